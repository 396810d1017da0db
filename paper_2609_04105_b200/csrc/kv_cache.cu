// Quantizing K and V into the pages of a cache, and reading them back.
//
// Both are bound by HBM: 2 bytes an element on the 16-bit side, 9/16 or 1 in the cache.  A block takes the tokens of one batch
// entry that stand in an aligned sixteen of the sequence - the unit in which V is kept - for a range of heads; a thread takes
// sixteen elements of one token, which is one NVFP4 block: 32 bytes in, no exchange with other threads for the block's
// maximum.  The bytes of K and V of the sixteen tokens are put together in shared memory as they lie in the page and leave
// in 16-byte stores.  Where the call's tokens do not fill a sixteen, V's bytes leave one by one: the others belong to
// tokens that are there already.
#include "kv_cache.cuh"

namespace fp4attn {
namespace {

constexpr int kTok = 16;                                          // tokens of a block

template <typename T>
struct WriteParams {
  View<const T> k, v;
  CacheRef cache;
  const int *start, *count, *positions;
  const float* inv_freq;
  int* status;
  int B, N, groups, heads_per_block, pairs;
  float factor;
  bool vector, interleaved;
};

// sixteen elements from x[first] on
template <typename T>
__device__ __forceinline__ void load16(const T* x, bool vector, float* v) {
  if (vector) {
    uint32_t w[8];
    *reinterpret_cast<uint4*>(w) = __ldg(reinterpret_cast<const uint4*>(x));
    *reinterpret_cast<uint4*>(w + 4) = __ldg(reinterpret_cast<const uint4*>(x) + 1);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = unpack2<T>(w[i]);
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = to_float(x[i]);
  }
}

// sixteen elements from element e0 of a row on, rotated and rounded to T as fp4attn_rotary would have left them
template <typename T, int D>
__device__ __forceinline__ void rotate16(const T* row, int e0, bool vector, bool interleaved, int pairs, const float2* cs, float* v) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      if (e0 + i >= 2 * pairs) break;
      rotate_pair(v[i], v[i + 1], cs[(e0 + i) >> 1]);
    }
  } else {
    const bool whole = vector && pairs % 16 == 0;                 // the partners are sixteen neighbours too
    float w[16];
    const int other = e0 < pairs ? e0 + pairs : e0 - pairs;
    if (whole && e0 < 2 * pairs) load16(row + other, true, w);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int e = e0 + i;
      if (e >= 2 * pairs) break;
      const bool first = e < pairs;
      float x = whole ? w[i] : to_float(row[first ? e + pairs : e - pairs]);
      if (first) rotate_pair(v[i], x, cs[e]);
      else rotate_pair(x, v[i], cs[e - pairs]);
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = to_float(from_float<T>(v[i]));
}

// NVFP4 block: eight bytes of codes; the scale byte.  NaN counts as 0 (the cache holds finite values only).
__device__ __forceinline__ uint2 nvfp4_block(float* v, float G, uint32_t* scale) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    v[i] = v[i] == v[i] ? v[i] : 0.f;
    a = fmaxf(a, fabsf(v[i]));
  }
  const uint32_t byte = cvt_e4m3x2(__fdiv_rn(__fmul_rn(a, G), 6.f), 0.f) & 0xFFu;
  const float S = e4m3_value(byte);
  const float r = S > 0.f ? __fdiv_rn(G, S) : 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __fmul_rn(v[i], r);
  *scale = byte;
  return make_uint2(cvt_e2m1x8(v), cvt_e2m1x8(v + 8));
}
// sixteen E4M3 bytes
__device__ __forceinline__ uint4 e4m3_block(float* v, float G) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = v[i] == v[i] ? __fmul_rn(v[i], G) : 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = cvt_e4m3x2(v[4 * i], v[4 * i + 1]) | cvt_e4m3x2(v[4 * i + 2], v[4 * i + 3]) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Threads: token (of sixteen) fastest, then the head's sixteens of elements.  Grid: sixteens of the sequence, batch, head ranges.
template <typename T, int FMT, int D>
__global__ void __launch_bounds__(D) cache_write_kernel(const WriteParams<T> p) {
  using L = RecordLayout<FMT, D>;
  // one head's bytes as they lie in the page, K: codes by chunk of 16 bytes and token, scales by token; V: codes by index and token,
  // scales by block and place
  __shared__ alignas(16) uint8_t sk[kTok * L::kRow], sv[kTok * L::kRow], sks[kTok * (L::kScales + 1)], svs[kTok * (L::kScales + 1)];
  extern __shared__ float2 table[];                               // [16][pairs]: cosines and sines of the tokens
  launch_dependents();
  wait_prior_grids();
  const int b = blockIdx.y, tid = threadIdx.x, tok = tid & 15, blk = tid >> 4;
  const int start = __ldg(p.start + b), n = p.count ? max(0, min(__ldg(p.count + b), p.N)) : p.N;
  // the sixteen that this block takes; a start below 0 counts from there (its tokens in front of 0 have no page)
  const long long pos0 = ((long long)(start >> 4) + blockIdx.x) << 4;
  const long long first = max((long long)start, pos0), last = min((long long)start + n, pos0 + kTok);
  if (first >= last) return;
  const int P = 1 << p.cache.log_page;
  const long long pos = pos0 + tok;
  const bool mine = pos >= first && pos < last;
  const int page = p.cache.page_of(b, pos0);                      // a page holds whole sixteens
  if (page < 0) {
    if (tid == 0 && blockIdx.z == 0 && p.status) *p.status = FP4ATTN_ERR_PAGE;
    return;
  }
  const int t0 = (int)(pos0 & (P - 1)), i = (int)(pos - start);                 // place in the page; index in the call
  if (p.pairs) {
    for (int j = tid; j < kTok * p.pairs; j += D) {
      const int t = j / p.pairs, f = j - t * p.pairs;
      if (pos0 + t < first || pos0 + t >= last) continue;
      const int at = p.positions ? __ldg(p.positions + (size_t)b * p.N + (pos0 + t - start)) : (int)(pos0 + t);
      table[j] = cos_sin(at, __ldg(p.inv_freq + f), p.factor);
    }
    __syncthreads();
  }
  const bool whole = last - first == kTok;
  const int h_end = min((int)(blockIdx.z + 1) * p.heads_per_block, p.cache.kv_heads);
  for (int h = blockIdx.z * p.heads_per_block; h < h_end; ++h) {
    if (mine) {
      const T* krow = p.k.row(b, h, i);
      float x[16], y[16];
      load16(krow + blk * 16, p.vector, x);
      load16(p.v.row(b, h, i) + blk * 16, p.vector, y);
      if (p.pairs) rotate16<T, D>(krow, blk * 16, p.vector, p.interleaved, p.pairs, table + tok * p.pairs, x);
      const float kG = __ldg(p.cache.k_G + h), vG = __ldg(p.cache.v_G + h);
      if (L::kFp4) {
        uint32_t ks, vs;
        const uint2 kc = nvfp4_block(x, kG, &ks), vc = nvfp4_block(y, vG, &vs);
        *reinterpret_cast<uint2*>(sk + ((blk >> 1) * kTok + tok) * 16 + (blk & 1) * 8) = kc;
        sks[tok * L::kScales + blk] = (uint8_t)ks;
        svs[blk * kTok + v_scale_place(tok)] = (uint8_t)vs;
#pragma unroll
        for (int r = 0; r < 8; ++r) sv[(blk * 8 + r) * kTok + tok] = (uint8_t)((r < 4 ? vc.x : vc.y) >> (8 * (r & 3)));
      } else {
        *reinterpret_cast<uint4*>(sk + (blk * kTok + tok) * 16) = e4m3_block(x, kG);
        const uint4 vc = e4m3_block(y, vG);
        const uint32_t w[4] = {vc.x, vc.y, vc.z, vc.w};
#pragma unroll
        for (int r = 0; r < 16; ++r) sv[(blk * 16 + r) * kTok + tok] = (uint8_t)(w[r >> 2] >> (8 * (r & 3)));
      }
    }
    __syncthreads();
    uint8_t* const rec = p.cache.rec(page, h);
    // K: a token's 16-byte chunks
    for (int j = tid; j < kTok * L::kRow / 16; j += D) {
      const int c = j >> 4, t = j & 15;
      if (whole || (pos0 + t >= first && pos0 + t < last))
        *reinterpret_cast<uint4*>(rec + (c * P + t0 + t) * 16) = *reinterpret_cast<const uint4*>(sk + j * 16);
    }
    uint8_t* const vrec = rec + L::v_codes(P) + t0 * L::kRow;
    if (whole) {
      for (int j = tid; j < L::kRow; j += D) *reinterpret_cast<uint4*>(vrec + j * 16) = *reinterpret_cast<const uint4*>(sv + j * 16);
      if (L::kFp4 && tid < L::kScales)                             // K: sixteen rows of scales in a run; V: a run of sixteen per block
        *reinterpret_cast<uint4*>(rec + L::k_scales(P) + t0 * L::kScales + tid * 16) = *reinterpret_cast<const uint4*>(sks + tid * 16);
      else if (L::kFp4 && tid < 2 * L::kScales)
        *reinterpret_cast<uint4*>(rec + L::v_scales(P) + (tid - L::kScales) * P + t0) = *reinterpret_cast<const uint4*>(svs + (tid - L::kScales) * 16);
    } else {
      for (int j = tid; j < kTok * L::kRow; j += D) {
        const int t = j & 15;
        if (pos0 + t >= first && pos0 + t < last) vrec[j] = sv[j];
      }
      if (L::kFp4 && mine) {
        rec[L::k_scales(P) + (t0 + tok) * L::kScales + blk] = sks[tok * L::kScales + blk];
        rec[L::v_scales(P) + blk * P + t0 + v_scale_place(tok)] = svs[blk * kTok + v_scale_place(tok)];
      }
    }
    __syncthreads();
  }
}

template <typename T>
struct ReadParams {
  View<T> k, v;
  CacheRef cache;
  const int *start, *count;
  int* status;
  int B, N, groups, heads_per_block;
  bool vector;
};

template <typename T>
__device__ __forceinline__ void store16(T* y, bool vector, const float* v) {
  if (vector) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = pack_pair<T>(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4*>(y) = make_uint4(w[0], w[1], w[2], w[3]);
    *(reinterpret_cast<uint4*>(y) + 1) = make_uint4(w[4], w[5], w[6], w[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = from_float<T>(v[i]);
  }
}
__device__ __forceinline__ void e4m3x16_values(uint4 raw, float scale, float* v) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 f = half2_of(cvt_f16x2_e4m3x2(w[i >> 1] >> (16 * (i & 1)) & 0xFFFFu));
    v[2 * i] = f.x * scale;
    v[2 * i + 1] = f.y * scale;
  }
}

// As cache_write_kernel.  A value is code * scale (exact) * fl(1 / G), rounded once more to T: two units in the last place of
// fp32 beside the quotient by G, which would take as long as reading the cache.
template <typename T, int FMT, int D>
__global__ void __launch_bounds__(D) cache_read_kernel(const ReadParams<T> p) {
  using L = RecordLayout<FMT, D>;
  __shared__ alignas(16) uint8_t sv[kTok * L::kRow], svs[kTok * (L::kScales + 1)];
  launch_dependents();
  wait_prior_grids();
  const int b = blockIdx.y, tid = threadIdx.x, tok = tid & 15, blk = tid >> 4;
  const int start = __ldg(p.start + b), n = p.count ? max(0, min(__ldg(p.count + b), p.N)) : p.N;
  const long long pos0 = ((long long)(start >> 4) + blockIdx.x) << 4;
  const long long first = max((long long)start, pos0), last = min((long long)start + n, pos0 + kTok);
  if (first >= last) return;
  const int P = 1 << p.cache.log_page;
  const long long pos = pos0 + tok;
  const bool mine = pos >= first && pos < last;
  const int page = p.cache.page_of(b, pos0);
  if (page < 0 && tid == 0 && blockIdx.z == 0 && p.status) *p.status = FP4ATTN_ERR_PAGE;
  const int t0 = (int)(pos0 & (P - 1)), i = (int)(pos - start);
  const int h_end = min((int)(blockIdx.z + 1) * p.heads_per_block, p.cache.kv_heads);
  for (int h = blockIdx.z * p.heads_per_block; h < h_end; ++h) {
    float x[16], y[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = y[r] = 0.f;                // no page: zeros
    if (page >= 0) {
      const uint8_t* const rec = p.cache.rec(page, h);
      const uint8_t* const vrec = rec + L::v_codes(P) + t0 * L::kRow;
      const float kr = __fdiv_rn(1.f, __ldg(p.cache.k_G + h)), vr = __fdiv_rn(1.f, __ldg(p.cache.v_G + h));
      __syncthreads();                                             // the head before is out of shared memory
      for (int j = tid; j < L::kRow; j += D) *reinterpret_cast<uint4*>(sv + j * 16) = __ldg(reinterpret_cast<const uint4*>(vrec) + j);
      if (L::kFp4 && tid < L::kScales)
        *reinterpret_cast<uint4*>(svs + tid * 16) = __ldg(reinterpret_cast<const uint4*>(rec + L::v_scales(P) + tid * P + t0));
      if (L::kFp4) {
        const uint2 kc = __ldg(reinterpret_cast<const uint2*>(rec + ((blk >> 1) * P + t0 + tok) * 16 + (blk & 1) * 8));
        const float ks = e4m3_value(__ldg(rec + L::k_scales(P) + (t0 + tok) * L::kScales + blk));
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t c = w ? kc.y : kc.x;
          const float2 f0 = half2_of(cvt_f16x2_e2m1x2<0>(c)), f1 = half2_of(cvt_f16x2_e2m1x2<1>(c));
          const float2 f2 = half2_of(cvt_f16x2_e2m1x2<2>(c)), f3 = half2_of(cvt_f16x2_e2m1x2<3>(c));
          const float e[8] = {f0.x, f0.y, f1.x, f1.y, f2.x, f2.y, f3.x, f3.y};
#pragma unroll
          for (int r = 0; r < 8; ++r) x[8 * w + r] = e[r] * ks * kr;
        }
      } else {
        e4m3x16_values(__ldg(reinterpret_cast<const uint4*>(rec + (blk * P + t0 + tok) * 16)), kr, x);
      }
      __syncthreads();
      if (L::kFp4) {
        const float vs = e4m3_value(svs[blk * kTok + v_scale_place(tok)]);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float2 f = half2_of(cvt_f16x2_e2m1x2<0>(sv[(blk * 8 + r) * kTok + tok]));
          y[2 * r] = f.x * vs * vr;
          y[2 * r + 1] = f.y * vs * vr;
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) y[r] = e4m3_value(sv[(blk * 16 + r) * kTok + tok]) * vr;
      }
    }
    if (mine) {
      store16(p.k.row(b, h, i) + blk * 16, p.vector, x);
      store16(p.v.row(b, h, i) + blk * 16, p.vector, y);
    }
  }
}

// grid of either kernel; false where the device does not tell its size
bool cover(int B, int N, int kv_heads, dim3* grid, int* heads_per_block) {
  const int sms = device_sms();
  if (!sms) return false;
  const int groups = (N + 14) / kTok + 1;                          // N tokens touch at most so many aligned sixteens
  // heads of a block: as many as leave eight blocks an SM
  long long per = (long long)groups * B * kv_heads / (8ll * sms);
  if (per < 1) per = 1;
  if (per > kv_heads) per = kv_heads;
  *heads_per_block = (int)per;
  *grid = dim3((unsigned)groups, (unsigned)B, (unsigned)((kv_heads + per - 1) / per));
  return true;
}

template <typename T, int FMT, int D>
int launch_write(WriteParams<T> p, cudaStream_t st) {
  dim3 grid;
  if (!cover(p.B, p.N, p.cache.kv_heads, &grid, &p.heads_per_block)) return FP4ATTN_ERR_CUDA;
  const cudaError_t e = launch_overlapped(cache_write_kernel<T, FMT, D>, grid, D, sizeof(float2) * kTok * p.pairs, st, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
}
template <typename T, int FMT, int D>
int launch_read(ReadParams<T> p, cudaStream_t st) {
  dim3 grid;
  if (!cover(p.B, p.N, p.cache.kv_heads, &grid, &p.heads_per_block)) return FP4ATTN_ERR_CUDA;
  const cudaError_t e = launch_overlapped(cache_read_kernel<T, FMT, D>, grid, D, 0, st, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
}

}  // namespace

// What is wrong with a cache, a batch's block table and its starts; fills `ref`
int check_cache(const fp4attn_cache* c, int B, const int* block_table, int max_pages, const int* start, const int* count, CacheRef* ref) {
  if (!c || !c->pages || !c->k_G || !c->v_G || !block_table || !start) return FP4ATTN_ERR_INVALID_ARG;
  if (c->fmt != FP4ATTN_FMT_NVFP4 && c->fmt != FP4ATTN_FMT_E4M3) return FP4ATTN_ERR_INVALID_ARG;
  if (B <= 0 || max_pages <= 0 || c->num_pages <= 0 || c->kv_heads <= 0 || c->d <= 0 || c->page_size <= 0) return FP4ATTN_ERR_INVALID_ARG;
  const size_t record = fp4attn_cache_record_bytes(c->fmt, c->page_size, c->d);
  if (!record || B > 65535 || c->kv_heads > 65535) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  if ((long long)max_pages * c->page_size >= (1ll << 30)) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;      // a token's place is an int
  if ((uintptr_t)c->pages & 15) return FP4ATTN_ERR_ALIGNMENT;
  if (((uintptr_t)c->k_G | (uintptr_t)c->v_G | (uintptr_t)block_table | (uintptr_t)start | (uintptr_t)count) & 3) return FP4ATTN_ERR_ALIGNMENT;
  ref->pages = (uint8_t*)c->pages;
  ref->k_G = c->k_G; ref->v_G = c->v_G;
  ref->table = block_table;
  ref->max_pages = max_pages; ref->num_pages = c->num_pages; ref->kv_heads = c->kv_heads;
  ref->log_page = log2_page(c->page_size);
  ref->record = (int)record;
  return FP4ATTN_OK;
}

}  // namespace fp4attn

using namespace fp4attn;

extern "C" size_t fp4attn_cache_record_bytes(int fmt, int page_size, int d) {
  if ((fmt != FP4ATTN_FMT_NVFP4 && fmt != FP4ATTN_FMT_E4M3) || log2_page(page_size) < 0 || (d != 64 && d != 128)) return 0;
  return (size_t)2 * page_size * (fmt == FP4ATTN_FMT_NVFP4 ? d / 2 + d / 16 : d);
}

#define FP4ATTN_CACHE_CASES(CALL, T, PARAMS)                                                                       \
  if (cache->fmt == FP4ATTN_FMT_NVFP4)                                                                             \
    return cache->d == 64 ? CALL<T, FP4ATTN_FMT_NVFP4, 64>(PARAMS, st) : CALL<T, FP4ATTN_FMT_NVFP4, 128>(PARAMS, st); \
  return cache->d == 64 ? CALL<T, FP4ATTN_FMT_E4M3, 64>(PARAMS, st) : CALL<T, FP4ATTN_FMT_E4M3, 128>(PARAMS, st);

extern "C" int fp4attn_cache_write(const fp4attn_cache* cache, const fp4attn_view* k, const fp4attn_view* v, int type, int B, int N,
                                   const int* block_table, int max_pages, const int* start, const int* count, const int* positions,
                                   const float* inv_freq, int pairs, int interleaved, float factor, int* device_status,
                                   fp4attn_stream_t stream) {
  CacheRef ref;
  int rc = check_cache(cache, B, block_table, max_pages, start, count, &ref);
  if (rc != FP4ATTN_OK) return rc;
  if (!k || !v || !k->data || !v->data || N <= 0 || pairs < 0 || (interleaved & ~1)) return FP4ATTN_ERR_INVALID_ARG;
  if (type != FP4ATTN_TYPE_BF16 && type != FP4ATTN_TYPE_FP16) return FP4ATTN_ERR_INVALID_ARG;
  if ((pairs > 0) != (inv_freq != nullptr) || (positions && !inv_freq)) return FP4ATTN_ERR_INVALID_ARG;
  if (2ll * pairs > cache->d || N >= (1 << 30)) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  if (((uintptr_t)k->data | (uintptr_t)v->data) & 1 || ((uintptr_t)positions | (uintptr_t)inv_freq | (uintptr_t)device_status) & 3)
    return FP4ATTN_ERR_ALIGNMENT;
  if ((rc = check_device_sm100()) != FP4ATTN_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  auto params = [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    WriteParams<T> p = {};
    p.k = View<const T>{(const T*)k->data, k->stride_b, k->stride_h, k->stride_n};
    p.v = View<const T>{(const T*)v->data, v->stride_b, v->stride_h, v->stride_n};
    p.cache = ref;
    p.start = start; p.count = count; p.positions = positions; p.inv_freq = inv_freq; p.status = device_status;
    p.B = B; p.N = N; p.pairs = pairs; p.factor = factor; p.interleaved = interleaved != 0;
    p.vector = view_vectors(*k, 2) && view_vectors(*v, 2);
    return p;
  };
  if (type == FP4ATTN_TYPE_BF16) { FP4ATTN_CACHE_CASES(launch_write, __nv_bfloat16, params((__nv_bfloat16*)nullptr)) }
  FP4ATTN_CACHE_CASES(launch_write, __half, params((__half*)nullptr))
}

extern "C" int fp4attn_cache_read(const fp4attn_cache* cache, const fp4attn_view* k_out, const fp4attn_view* v_out, int type, int B, int N,
                                  const int* block_table, int max_pages, const int* start, const int* count, int* device_status,
                                  fp4attn_stream_t stream) {
  CacheRef ref;
  int rc = check_cache(cache, B, block_table, max_pages, start, count, &ref);
  if (rc != FP4ATTN_OK) return rc;
  if (!k_out || !v_out || !k_out->data || !v_out->data || N <= 0) return FP4ATTN_ERR_INVALID_ARG;
  if (type != FP4ATTN_TYPE_BF16 && type != FP4ATTN_TYPE_FP16) return FP4ATTN_ERR_INVALID_ARG;
  if (N >= (1 << 30)) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  if (((uintptr_t)k_out->data | (uintptr_t)v_out->data) & 1 || ((uintptr_t)device_status & 3)) return FP4ATTN_ERR_ALIGNMENT;
  if ((rc = check_device_sm100()) != FP4ATTN_OK) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  auto params = [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    ReadParams<T> p = {};
    p.k = view_of<T>(*k_out);
    p.v = view_of<T>(*v_out);
    p.cache = ref;
    p.start = start; p.count = count; p.status = device_status;
    p.B = B; p.N = N;
    p.vector = view_vectors(*k_out, 2) && view_vectors(*v_out, 2);
    return p;
  };
  if (type == FP4ATTN_TYPE_BF16) { FP4ATTN_CACHE_CASES(launch_read, __nv_bfloat16, params((__nv_bfloat16*)nullptr)) }
  FP4ATTN_CACHE_CASES(launch_read, __half, params((__half*)nullptr))
}
