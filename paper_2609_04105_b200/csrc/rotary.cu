// Rotary positions of Q and K, and the transposed rotation for their gradients.
//
// Bound by HBM: every element is read once and written once, so a launch takes Q and K together and every access is 16 bytes
// wide (2 x 4096 tokens of 32 + 8 heads, d = 128, bf16: 33 us, 5.1 TB/s; fp32 57 us, 5.8 TB/s; 4 x 4095 of 32, d = 64, half of each head turned
// in neighbouring pairs: 37 us, 3.6 TB/s).  A block takes a few tokens and a range of heads.  The cosines and sines of its tokens are worked out once (in 64
// bits, see cos_sin) into shared memory and serve all of its heads.
#include "kv_cache.cuh"

namespace fp4attn {
namespace {

constexpr int kThreads = 256;
constexpr int kMostPairs = 128;                                   // of a head: d up to 256

template <typename T>
struct RotaryParams {
  View<T> in[2], out[2];                                          // Q, K
  int heads[2];
  const int* positions;                                           // [B, N]
  const float* inv_freq;                                          // [pairs]
  int B, N, d, pairs, tokens_per_block, heads_per_block;
  float factor;
  float sign;                                                     // -1: the transposed rotation
};

// One unit of work of a row.  VECTOR: 16 bytes of the first elements of the pairs and 16 bytes of the second ones (half layout), 16 bytes of
// neighbouring pairs (interleaved), or 16 bytes behind the rotated part.  Otherwise one pair, or one element behind it.
template <typename T, bool INTERLEAVED, bool VECTOR>
__device__ __forceinline__ void rotary_unit(const T* x, T* y, int u, int pairs, const float2* cs) {
  constexpr int V = 16 / (int)sizeof(T);
  if constexpr (!VECTOR) {
    if (u < pairs) {
      const int i = INTERLEAVED ? 2 * u : u, j = INTERLEAVED ? 2 * u + 1 : u + pairs;
      float a = to_float(x[i]), b = to_float(x[j]);
      rotate_pair(a, b, cs[u]);
      y[i] = from_float<T>(a);
      y[j] = from_float<T>(b);
    } else {
      y[pairs + u] = x[pairs + u];
    }
  } else {
    alignas(16) T a[V], b[V];
    const int units = INTERLEAVED ? 2 * pairs / V : pairs / V;
    if (u >= units) {                                              // carried over as it is
      const int i = 2 * pairs + (u - units) * V;
      *reinterpret_cast<uint4*>(y + i) = *reinterpret_cast<const uint4*>(x + i);
    } else if (INTERLEAVED) {
      *reinterpret_cast<uint4*>(a) = *reinterpret_cast<const uint4*>(x + u * V);
#pragma unroll
      for (int k = 0; k < V; k += 2) {
        float p = to_float(a[k]), q = to_float(a[k + 1]);
        rotate_pair(p, q, cs[(u * V + k) / 2]);
        a[k] = from_float<T>(p);
        a[k + 1] = from_float<T>(q);
      }
      *reinterpret_cast<uint4*>(y + u * V) = *reinterpret_cast<const uint4*>(a);
    } else {
      *reinterpret_cast<uint4*>(a) = *reinterpret_cast<const uint4*>(x + u * V);
      *reinterpret_cast<uint4*>(b) = *reinterpret_cast<const uint4*>(x + pairs + u * V);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float p = to_float(a[k]), q = to_float(b[k]);
        rotate_pair(p, q, cs[u * V + k]);
        a[k] = from_float<T>(p);
        b[k] = from_float<T>(q);
      }
      *reinterpret_cast<uint4*>(y + u * V) = *reinterpret_cast<const uint4*>(a);
      *reinterpret_cast<uint4*>(y + pairs + u * V) = *reinterpret_cast<const uint4*>(b);
    }
  }
}

template <typename T, bool INTERLEAVED, bool VECTOR>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const RotaryParams<T> p) {
  extern __shared__ float2 table[];                               // [tokens_per_block][pairs]
  launch_dependents();
  wait_prior_grids();
  constexpr int V = 16 / (int)sizeof(T);
  const long long tokens = (long long)p.B * p.N, first = (long long)blockIdx.x * p.tokens_per_block;
  const int n_tok = (int)min((long long)p.tokens_per_block, tokens - first);
  for (int i = threadIdx.x; i < n_tok * p.pairs; i += kThreads) {
    const int t = i / p.pairs, f = i - t * p.pairs;
    float2 cs = cos_sin(load(p.positions + first + t), load(p.inv_freq + f), p.factor);
    cs.y *= p.sign;
    table[i] = cs;
  }
  __syncthreads();
  // A thread keeps its unit and steps through the rows (heads of a token, token by token): no division per unit, which took as long as the
  // rest (2 x 4096 tokens of 40 heads, d = 128: 38.6 us with three).
  const int units = VECTOR ? (INTERLEAVED ? p.d / V : (p.d - p.pairs) / V) : p.d - p.pairs;
  const int h0 = blockIdx.y * p.heads_per_block;
  const int n_heads = min(p.heads_per_block, p.heads[0] + p.heads[1] - h0);
  const int at_once = kThreads / units, u = threadIdx.x % units;   // rows of a pass (units: at most d, 256)
  int hh = threadIdx.x / units, t = 0;
  if (hh >= at_once) return;
  int b = (int)(first / p.N), n = (int)(first - (long long)b * p.N);
  for (;;) {
    while (hh >= n_heads) {
      hh -= n_heads;
      if (++t >= n_tok) return;
      if (++n == p.N) {
        n = 0;
        ++b;
      }
    }
    const int h = h0 + hh, w = h >= p.heads[0], head = w ? h - p.heads[0] : h;
    rotary_unit<T, INTERLEAVED, VECTOR>(p.in[w].row(b, head, n), p.out[w].row(b, head, n), u, p.pairs, table + t * p.pairs);
    hh += at_once;
  }
}

template <typename T>
int launch(const fp4attn_view* x, const fp4attn_view* y, int Hq, int Hk, int B, int N, int d, const int* positions,
           const float* inv_freq, int pairs, bool interleaved, bool transposed, float factor, cudaStream_t st) {
  RotaryParams<T> p;
  bool vector = true;
  const int V = 16 / (int)sizeof(T);
  for (int i = 0; i < 2; ++i) {
    p.in[i] = view_of<T>(x[i]);
    p.out[i] = view_of<T>(y[i]);
    p.heads[i] = i ? Hk : Hq;
    if (p.heads[i]) vector = vector && view_vectors(x[i], sizeof(T)) && view_vectors(y[i], sizeof(T));
  }
  vector = vector && d % V == 0 && (interleaved ? 2 * pairs : pairs) % V == 0 && (2 * pairs) % V == 0;
  p.positions = positions; p.inv_freq = inv_freq;
  p.B = B; p.N = N; p.d = d; p.pairs = pairs; p.factor = factor; p.sign = transposed ? -1.f : 1.f;
  const int sms = device_sms();
  if (!sms) return FP4ATTN_ERR_CUDA;
  const long long tokens = (long long)B * N;
  const int heads = Hq + Hk;
  // up to four tokens a block while that leaves eight blocks an SM; heads split while there are fewer
  long long per = tokens / (8ll * sms);
  p.tokens_per_block = (int)(per < 1 ? 1 : per > 4 ? 4 : per);
  const long long blocks = (tokens + p.tokens_per_block - 1) / p.tokens_per_block;
  long long split = blocks < 2ll * sms ? (2ll * sms + blocks - 1) / blocks : 1;
  if (split > heads) split = heads;
  p.heads_per_block = (int)((heads + split - 1) / split);
  const dim3 grid((unsigned)blocks, (unsigned)((heads + p.heads_per_block - 1) / p.heads_per_block));
  const size_t smem = sizeof(float2) * p.tokens_per_block * pairs;
  cudaError_t e;
  if (vector)
    e = interleaved ? launch_overlapped(rotary_kernel<T, true, true>, grid, kThreads, smem, st, p)
                    : launch_overlapped(rotary_kernel<T, false, true>, grid, kThreads, smem, st, p);
  else
    e = interleaved ? launch_overlapped(rotary_kernel<T, true, false>, grid, kThreads, smem, st, p)
                    : launch_overlapped(rotary_kernel<T, false, false>, grid, kThreads, smem, st, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
}

}  // namespace
}  // namespace fp4attn

using namespace fp4attn;

extern "C" int fp4attn_rotary(const fp4attn_view* q, const fp4attn_view* k, const fp4attn_view* q_out, const fp4attn_view* k_out, int type,
                              int B, int H, int kv_heads, int N, int d, const int* positions, const float* inv_freq, int pairs,
                              int interleaved, int transposed, float factor, fp4attn_stream_t stream) {
  if (!q || !q_out || !q->data || !q_out->data || !positions || !inv_freq) return FP4ATTN_ERR_INVALID_ARG;
  if (B <= 0 || H <= 0 || N <= 0 || d <= 0 || pairs <= 0 || kv_heads < 0) return FP4ATTN_ERR_INVALID_ARG;
  if (kv_heads > 0 && (!k || !k_out || !k->data || !k_out->data)) return FP4ATTN_ERR_INVALID_ARG;
  if (type < FP4ATTN_TYPE_BF16 || type > FP4ATTN_TYPE_FP32 || (interleaved & ~1) || (transposed & ~1)) return FP4ATTN_ERR_INVALID_ARG;
  if (2ll * pairs > d || d > 2 * kMostPairs || (long long)H + kv_heads > 65535) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  if ((long long)B * N >= (1ll << 31)) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  const fp4attn_view none = {nullptr, 0, 0, 0};
  const fp4attn_view x[2] = {*q, kv_heads ? *k : none}, y[2] = {*q_out, kv_heads ? *k_out : none};
  const uintptr_t size = type == FP4ATTN_TYPE_FP32 ? 4 : 2;
  for (int i = 0; i < 2; ++i)
    if (((uintptr_t)x[i].data | (uintptr_t)y[i].data) & (size - 1)) return FP4ATTN_ERR_ALIGNMENT;
  if (((uintptr_t)positions | (uintptr_t)inv_freq) & 3) return FP4ATTN_ERR_ALIGNMENT;
  const int rc = check_device_sm100();
  if (rc != FP4ATTN_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  switch (type) {
    case FP4ATTN_TYPE_BF16:
      return launch<__nv_bfloat16>(x, y, H, kv_heads, B, N, d, positions, inv_freq, pairs, interleaved, transposed, factor, st);
    case FP4ATTN_TYPE_FP16:
      return launch<__half>(x, y, H, kv_heads, B, N, d, positions, inv_freq, pairs, interleaved, transposed, factor, st);
    default:
      return launch<float>(x, y, H, kv_heads, B, N, d, positions, inv_freq, pairs, interleaved, transposed, factor, st);
  }
}
