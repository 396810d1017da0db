// Attention of any number of tokens of every sequence over its pages of a quantized cache, and of a batch that shares long prefixes.
//
// Row (b, h, t) at position p sees keys [first, last), clipped to the keys that are there.  With s the scaled product of q and a key,
//     x = cap tanh(s / cap) (if capped) - slope_h |p - j|,   O = sum_j e^(x_j - m) v_j / sum_j e^(x_j - m),   LSE = m + ln sum_j e^(x_j - m).
//
// The simplest form: a warp per row, a key after another, everything in fp32.
#include "kv_cache.cuh"

#include <limits.h>
#include <math.h>

#include <algorithm>

namespace fp4attn {

int check_cache(const fp4attn_cache* c, int B, const int* block_table, int max_pages, const int* start, const int* count, CacheRef* ref);

namespace {

struct PagedParams {
  const void* q;
  long long q_sb, q_sh, q_sn;
  CacheRef cache;
  const int *context, *count, *first, *last;
  // shared prefixes: of each group, and where its entries begin
  const int *prefix_table, *prefix_length, *group_start;
  int groups, prefix_pages;
  const unsigned long long* mask;
  const float* slopes;
  void* out;
  float* lse;
  int* status;
  int B, H, T, group;
  float scale, cap;
  bool half;
};

template <int FMT, int D>
__global__ void __launch_bounds__(128) row_kernel(const PagedParams p) {
  using L = RecordLayout<FMT, D>;
  constexpr int E = D / 32;
  wait_prior_grids();
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, P = 1 << p.cache.log_page;
  if (row >= (long long)p.B * p.H * p.T) return;
  const int t = (int)(row % p.T), h = (int)(row / p.T % p.H), b = (int)(row / ((long long)p.T * p.H)), kvh = h / p.group;
  const int n = p.count ? max(0, min(load(p.count + b), p.T)) : p.T;
  if (t >= n) return;
  const int ctx = max(0, load(p.context + b));
  float q[E];
  for (int x = 0; x < E; ++x) {
    const uint16_t w = load(static_cast<const uint16_t*>(p.q) + b * p.q_sb + h * p.q_sh + t * p.q_sn + lane * E + x);
    q[x] = p.half ? __half2float(__ushort_as_half(w)) : __bfloat162float(__ushort_as_bfloat16(w));
  }
  const float c = __fdiv_rn(p.scale, load(p.cache.k_G + kvh)), slope = p.slopes ? load(p.slopes + h) : 0.f;
  float m = -INFINITY, l = 0.f, o[E] = {};
  bool lost = false;
  auto run = [&](const int* table, int max_pages, long long lo, long long hi, long long reported, long long at, const unsigned long long* mask, int ctx) {
    const long long room = (long long)max_pages << p.cache.log_page;
    lost |= reported > room;                                        // the table has no room for the last tokens
    for (long long j = lo; j < min(hi, room); ++j) {
      if (mask && j >= ctx && !(*mask >> (j - ctx) & 1)) continue;
      const long long i = j >> p.cache.log_page;
      const int page = i < max_pages ? load(table + i) : -1;
      if (page < 0 || page >= p.cache.num_pages) {
        lost |= j < reported;
        continue;
      }
      const uint8_t* const rec = p.cache.rec(page, kvh);
      const int tok = (int)(j & (P - 1)), e = lane * E;
      float k[E], v[E];
      for (int x = 0; x < E; ++x) {
        const int f = e + x;
        if (L::kFp4) {
          const uint32_t kb = load(rec + (f / 32 * P + tok) * 16 + f % 32 / 2) >> 4 * (f & 1) & 15u;
          const uint32_t vb = load(rec + L::v_codes(P) + (tok / 16 * (D / 2) + f / 2) * 16 + tok % 16) >> 4 * (f & 1) & 15u;
          k[x] = half2_of(cvt_f16x2_e2m1x2<0>(kb)).x * e4m3_value(load(rec + L::k_scales(P) + tok * L::kScales + f / 16));
          v[x] = half2_of(cvt_f16x2_e2m1x2<0>(vb)).x * e4m3_value(load(rec + L::v_scales(P) + f / 16 * P + v_scale_place(tok)));
        } else {
          k[x] = e4m3_value(load(rec + (f / 16 * P + tok) * 16 + f % 16));
          v[x] = e4m3_value(load(rec + L::v_codes(P) + (tok / 16 * D + f) * 16 + tok % 16));
        }
      }
      float s = 0.f;
      for (int x = 0; x < E; ++x) s = fmaf(q[x], k[x], s);
      for (int y = 16; y; y >>= 1) s += __shfl_xor_sync(0xffffffffu, s, y);
      s *= c;
      if (p.cap > 0.f) s = p.cap * tanhf(s / p.cap);
      s -= slope * fabsf((float)(at - j));
      const float top = fmaxf(m, s), f = m == -INFINITY ? 0.f : expf(m - top), w = top == -INFINITY ? 0.f : expf(s - top);
      m = top;
      l = l * f + w;
      for (int x = 0; x < E; ++x) o[x] = o[x] * f + w * v[x];
    }
  };
  if (p.groups) {
    int before = 0;
    for (int g = 0; g < p.groups; ++g) {
      if (b < load(p.group_start + g) || b >= load(p.group_start + g + 1)) continue;
      before = max(0, load(p.prefix_length + g));
      run(p.prefix_table + (size_t)g * p.prefix_pages, p.prefix_pages, 0, before, before, (long long)before + ctx + t, nullptr, 0);
    }
    const unsigned long long mask = p.mask ? load(p.mask + (size_t)b * p.T + t) : (2ull << t) - 1;
    run(p.cache.table + (size_t)b * p.cache.max_pages, p.cache.max_pages, 0, (long long)ctx + n, (long long)ctx + n, (long long)ctx + t, &mask, ctx);
  } else {
    const long long there = (long long)ctx + n;
    const long long lo = p.first ? max(0, load(p.first + (size_t)b * p.T + t)) : 0;
    const long long hi = min(there, p.last ? (long long)load(p.last + (size_t)b * p.T + t) : (long long)ctx + t + 1);
    run(p.cache.table + (size_t)b * p.cache.max_pages, p.cache.max_pages, lo, hi, hi, (long long)ctx + t, nullptr, 0);
  }
  const float f = l == 0.f ? 0.f : __fdiv_rn(1.f, l * load(p.cache.v_G + kvh));
  for (int x = 0; x < E; ++x) {
    const float y = l == 0.f ? 0.f : o[x] * f;
    static_cast<uint16_t*>(p.out)[row * D + lane * E + x] = p.half ? __half_as_ushort(__float2half_rn(y)) : __bfloat16_as_ushort(__float2bfloat16_rn(y));
  }
  if (lane == 0 && p.lse) p.lse[row] = l == 0.f ? -INFINITY : m + logf(l);
  if (lost && lane == 0 && p.status) *p.status = FP4ATTN_ERR_PAGE;
}

int launch(const PagedParams& p, int fmt, int d, cudaStream_t st) {
  const dim3 grid((unsigned)(((long long)p.B * p.H * p.T + 3) / 4));
  auto go = [&](auto* kernel) {
    const cudaError_t e = launch_overlapped(kernel, grid, 128u, 0, st, p);
    return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
  };
  if (fmt == FP4ATTN_FMT_NVFP4) return d == 64 ? go(row_kernel<FP4ATTN_FMT_NVFP4, 64>) : go(row_kernel<FP4ATTN_FMT_NVFP4, 128>);
  return d == 64 ? go(row_kernel<FP4ATTN_FMT_E4M3, 64>) : go(row_kernel<FP4ATTN_FMT_E4M3, 128>);
}

// what the two calls have in common
int check(const fp4attn_view* q, int type, const fp4attn_cache* cache, int B, int H, int T, const int* block_table, int max_pages, const int* context,
          const int* count, float softmax_scale, float soft_cap, const float* slopes, void* O, float* LSE, int* device_status, PagedParams* p) {
  const int rc = check_cache(cache, B, block_table, max_pages, context, count, &p->cache);
  if (rc != FP4ATTN_OK) return rc;
  if (!q || !q->data || !O || H <= 0 || T <= 0 || !(softmax_scale >= 0.f) || !(soft_cap >= 0.f) || isinf(softmax_scale) || isinf(soft_cap))
    return FP4ATTN_ERR_INVALID_ARG;
  if (type != FP4ATTN_TYPE_BF16 && type != FP4ATTN_TYPE_FP16) return FP4ATTN_ERR_INVALID_ARG;
  if (H % cache->kv_heads != 0) return FP4ATTN_ERR_INVALID_ARG;
  if ((long long)B * H * T >= (1ll << 31)) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  if (((uintptr_t)q->data & 1) || ((uintptr_t)O & 15) || ((uintptr_t)LSE | (uintptr_t)device_status | (uintptr_t)slopes) & 3) return FP4ATTN_ERR_ALIGNMENT;
  p->q = q->data; p->q_sb = q->stride_b; p->q_sh = q->stride_h; p->q_sn = q->stride_n;
  p->half = type == FP4ATTN_TYPE_FP16;
  p->context = context; p->count = count; p->slopes = slopes;
  p->out = O; p->lse = LSE; p->status = device_status;
  p->B = B; p->H = H; p->T = T; p->group = H / cache->kv_heads;
  p->scale = softmax_scale > 0.f ? softmax_scale : (float)(1.0 / sqrt((double)cache->d));
  p->cap = soft_cap;
  return FP4ATTN_OK;
}

}  // namespace
}  // namespace fp4attn

using namespace fp4attn;

extern "C" size_t fp4attn_paged_attention_workspace_bytes(int B, int H, int kv_heads, int T, int d) {
  if (B <= 0 || H <= 0 || kv_heads <= 0 || H % kv_heads != 0 || T <= 0 || (d != 64 && d != 128) || (long long)B * H * T >= (1ll << 31)) return 0;
  return 16;
}

extern "C" int fp4attn_paged_attention(const fp4attn_view* q, int type, const fp4attn_cache* cache, int B, int H, int T, const int* block_table,
                                       int max_pages, const int* context, const int* count, const int* first, const int* last, float softmax_scale,
                                       float soft_cap, const float* slopes, void* O, float* LSE, int* device_status, void* workspace,
                                       size_t workspace_bytes, fp4attn_stream_t stream) {
  PagedParams p = {};
  int rc = check(q, type, cache, B, H, T, block_table, max_pages, context, count, softmax_scale, soft_cap, slopes, O, LSE, device_status, &p);
  if (rc != FP4ATTN_OK) return rc;
  if (((uintptr_t)first | (uintptr_t)last) & 3) return FP4ATTN_ERR_ALIGNMENT;
  if (!workspace || workspace_bytes < fp4attn_paged_attention_workspace_bytes(B, H, cache->kv_heads, T, cache->d)) return FP4ATTN_ERR_WORKSPACE;
  if ((uintptr_t)workspace & 15) return FP4ATTN_ERR_ALIGNMENT;
  if ((rc = check_device_sm100()) != FP4ATTN_OK) return rc;
  p.first = first; p.last = last;
  return launch(p, cache->fmt, cache->d, (cudaStream_t)stream);
}

extern "C" size_t fp4attn_shared_prefix_attention_workspace_bytes(int B, int H, int kv_heads, int T, int d, int groups) {
  if (groups <= 0 || groups > 65535 || T > FP4ATTN_MOST_TREE_TOKENS) return 0;
  return fp4attn_paged_attention_workspace_bytes(B, H, kv_heads, T, d);
}

extern "C" int fp4attn_shared_prefix_attention(const fp4attn_view* q, int type, const fp4attn_cache* cache, int B, int H, int T, int groups,
                                               const int* prefix_table, int prefix_pages, const int* prefix_length, const int* group_start,
                                               const int* block_table, int max_pages, const int* context, const int* count,
                                               const unsigned long long* tree_mask, float softmax_scale, float soft_cap, const float* slopes, void* O,
                                               float* LSE, int* device_status, void* workspace, size_t workspace_bytes, fp4attn_stream_t stream) {
  PagedParams p = {};
  int rc = check(q, type, cache, B, H, T, block_table, max_pages, context, count, softmax_scale, soft_cap, slopes, O, LSE, device_status, &p);
  if (rc != FP4ATTN_OK) return rc;
  if (!prefix_table || !prefix_length || !group_start || groups <= 0 || prefix_pages <= 0) return FP4ATTN_ERR_INVALID_ARG;
  if (groups > 65535 || T > FP4ATTN_MOST_TREE_TOKENS || (long long)prefix_pages * cache->page_size >= (1ll << 30)) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  if (((uintptr_t)prefix_table | (uintptr_t)prefix_length | (uintptr_t)group_start) & 3 || ((uintptr_t)tree_mask & 7)) return FP4ATTN_ERR_ALIGNMENT;
  if (!workspace || workspace_bytes < fp4attn_shared_prefix_attention_workspace_bytes(B, H, cache->kv_heads, T, cache->d, groups)) return FP4ATTN_ERR_WORKSPACE;
  if ((uintptr_t)workspace & 15) return FP4ATTN_ERR_ALIGNMENT;
  if ((rc = check_device_sm100()) != FP4ATTN_OK) return rc;
  p.groups = groups; p.prefix_table = prefix_table; p.prefix_pages = prefix_pages; p.prefix_length = prefix_length; p.group_start = group_start;
  p.mask = tree_mask;
  return launch(p, cache->fmt, cache->d, (cudaStream_t)stream);
}
