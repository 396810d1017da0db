// Attention of one token, or of a tree of drafted tokens, of every sequence over its pages of a quantized cache.
//
// Row (b, h, t) sees the first context[b] tokens of the sequence, and of the T drafted tokens at positions context[b] ..
// context[b] + T - 1 those whose bit of its mask is set.  One warp takes a row and walks its keys with a running maximum and sum.
#include "kv_cache.cuh"

namespace fp4attn {

int check_cache(const fp4attn_cache* c, int B, const int* block_table, int max_pages, const int* start, const int* count, CacheRef* ref);

namespace {

struct TreeParams {
  const void* q;
  long long q_sb, q_sh, q_sn;
  CacheRef cache;
  const int *context, *count;
  const unsigned long long* mask;    // [B, T] or null: token t sees 0 .. t
  void* out;                         // [B, H, T, d]
  float* lse;                        // [B, H, T]
  int* status;
  int B, H, T, group;
  float scale;
};

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(128) tree_row_kernel(const TreeParams p) {
  using L = RecordLayout<FMT, D>;
  launch_dependents();
  wait_prior_grids();
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= (long long)p.B * p.H * p.T) return;
  const int t = (int)(row % p.T), h = (int)(row / p.T % p.H), b = (int)(row / p.T / p.H), kvh = h / p.group;
  if (p.count && t >= __ldg(p.count + b)) return;
  constexpr int E = D / 32;
  const int P = 1 << p.cache.log_page;
  const T* q = static_cast<const T*>(p.q) + b * p.q_sb + h * p.q_sh + t * p.q_sn;
  float qv[E], o[E];
  for (int i = 0; i < E; ++i) {
    qv[i] = to_float(q[2 * lane + 64 * (i >> 1) + (i & 1)]);
    o[i] = 0.f;
  }
  const float c = p.scale * 1.4426950408889634f / __ldg(p.cache.k_G + kvh);
  const unsigned long long bits = p.mask ? __ldg(p.mask + (size_t)b * p.T + t) : (2ull << t) - 1;
  const int ctx = max(0, __ldg(p.context + b));
  float m = -INFINITY, l = 0.f;
  const long long held = (long long)p.cache.max_pages << p.cache.log_page, end = min((long long)ctx + p.T, held);
  if ((long long)ctx + p.T > held && p.status) *p.status = FP4ATTN_ERR_PAGE;
  for (long long k = 0; k < end; ++k) {
    if (k >= ctx && !(bits >> (k - ctx) & 1)) continue;
    const int page = p.cache.page_of(b, k);
    if (page < 0) {
      if (p.status) *p.status = FP4ATTN_ERR_PAGE;
      continue;
    }
    const uint8_t* const rec = p.cache.rec(page, kvh);
    const int at = (int)(k & (P - 1));
    float s = 0.f, v[E];
    for (int i = 0; i < E; ++i) {
      const int e = 2 * lane + 64 * (i >> 1) + (i & 1);
      float kv, vv;
      if (L::kFp4) {
        const float2 kp = half2_of(cvt_f16x2_e2m1x2<0>(rec[(e / 32 * P + at) * 16 + e % 32 / 2]));
        const float2 vp = half2_of(cvt_f16x2_e2m1x2<0>(rec[L::v_codes(P) + (at / 16 * L::kRow + e / 2) * 16 + at % 16]));
        kv = (e & 1 ? kp.y : kp.x) * e4m3_value(rec[L::k_scales(P) + at * L::kScales + e / 16]);
        vv = (e & 1 ? vp.y : vp.x) * e4m3_value(rec[L::v_scales(P) + e / 16 * P + v_scale_place(at)]);
      } else {
        kv = e4m3_value(rec[(e / 16 * P + at) * 16 + e % 16]);
        vv = e4m3_value(rec[L::v_codes(P) + (at / 16 * L::kRow + e) * 16 + at % 16]);
      }
      s += qv[i] * kv;
      v[i] = vv;
    }
    for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= c;
    const float m2 = fmaxf(m, s);
    const float old = m == -INFINITY ? 0.f : exp2f(m - m2), w = exp2f(s - m2);
    l = l * old + w;
    for (int i = 0; i < E; ++i) o[i] = o[i] * old + w * v[i];
    m = m2;
  }
  const float r = l > 0.f ? 1.f / (l * __ldg(p.cache.v_G + kvh)) : l;     // a NaN stays one
  T* const y = static_cast<T*>(p.out) + row * D;
  for (int i = 0; i < E; ++i) y[2 * lane + 64 * (i >> 1) + (i & 1)] = from_float<T>(l == 0.f ? 0.f : o[i] * r);
  if (lane == 0 && p.lse) p.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

template <typename T, int FMT, int D>
int launch_tree(const TreeParams& p, cudaStream_t st) {
  const long long rows = (long long)p.B * p.H * p.T;
  const cudaError_t e = launch_overlapped(tree_row_kernel<T, FMT, D>, dim3((unsigned)((rows + 3) / 4)), 128u, 0, st, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
}

}  // namespace
}  // namespace fp4attn

using namespace fp4attn;

extern "C" size_t fp4attn_tree_attention_workspace_bytes(int B, int H, int kv_heads, int T, int d) {
  (void)B; (void)H; (void)kv_heads; (void)T; (void)d;
  return 0;
}

extern "C" int fp4attn_tree_attention(const fp4attn_view* q, int type, const fp4attn_cache* cache, int B, int H, int T, const int* block_table,
                                      int max_pages, const int* context, const int* count, const unsigned long long* tree_mask,
                                      float softmax_scale, void* O, float* LSE, int* device_status, void* workspace, size_t workspace_bytes,
                                      fp4attn_stream_t stream) {
  CacheRef ref;
  int rc = check_cache(cache, B, block_table, max_pages, context, count, &ref);
  if (rc != FP4ATTN_OK) return rc;
  if (!q || !q->data || !O || H <= 0 || T <= 0 || !(softmax_scale >= 0.f)) return FP4ATTN_ERR_INVALID_ARG;
  if (type != FP4ATTN_TYPE_BF16 && type != FP4ATTN_TYPE_FP16) return FP4ATTN_ERR_INVALID_ARG;
  if (H % cache->kv_heads != 0) return FP4ATTN_ERR_INVALID_ARG;
  if (T > FP4ATTN_MOST_TREE_TOKENS || (long long)B * H * T >= (1ll << 31)) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  if (((uintptr_t)q->data & 1) || ((uintptr_t)O & 15) || ((uintptr_t)tree_mask & 7) || ((uintptr_t)LSE | (uintptr_t)device_status) & 3)
    return FP4ATTN_ERR_ALIGNMENT;
  if ((rc = check_device_sm100()) != FP4ATTN_OK) return rc;
  (void)workspace; (void)workspace_bytes;
  TreeParams p = {};
  p.q = q->data; p.q_sb = q->stride_b; p.q_sh = q->stride_h; p.q_sn = q->stride_n;
  p.cache = ref;
  p.context = context; p.count = count; p.mask = tree_mask;
  p.out = O; p.lse = LSE; p.status = device_status;
  p.B = B; p.H = H; p.T = T; p.group = H / cache->kv_heads;
  p.scale = softmax_scale > 0.f ? softmax_scale : (float)(1.0 / sqrt((double)cache->d));
  cudaStream_t st = (cudaStream_t)stream;
#define FP4ATTN_TREE(T_)                                                                                                              \
  if (cache->fmt == FP4ATTN_FMT_NVFP4)                                                                                                \
    return cache->d == 64 ? launch_tree<T_, FP4ATTN_FMT_NVFP4, 64>(p, st) : launch_tree<T_, FP4ATTN_FMT_NVFP4, 128>(p, st);           \
  return cache->d == 64 ? launch_tree<T_, FP4ATTN_FMT_E4M3, 64>(p, st) : launch_tree<T_, FP4ATTN_FMT_E4M3, 128>(p, st);
  if (type == FP4ATTN_TYPE_BF16) { FP4ATTN_TREE(__nv_bfloat16) }
  FP4ATTN_TREE(__half)
#undef FP4ATTN_TREE
}
