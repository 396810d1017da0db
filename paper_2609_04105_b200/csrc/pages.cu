// Pages of a cache out of a stack of free ones, and back onto it: block tables, slots and positions without a word from the host.
//
// assign   tokens start[b] .. start[b] + count[b] - 1 of entry b need pages ceil(start / P) .. ceil((start + count) / P) - 1 of its table.  The i-th
//          new page of the call, in the order of entries and of their tables, is free[n - 1 - i] of the n free ones: where an entry's begin is a
//          prefix sum over the entries, which every block makes for itself (8 bytes an entry out of L2 cost less than a second launch).
// release  pages ceil(keep / P) .. ceil(length / P) - 1 of an entry's table go back, the call's last one first: what an assign took lies on the
//          stack afterwards as it lay before.  Tables may have holes, so the pages are counted by a kernel of their own first.
//
// Bound by launches and by dependent loads (start - page - slot); a prompt's slots by writing them: 48 sequences of up to 16384 tokens are 9 MB.  Every block
// sums over all entries for itself (release: a block an entry), which is little up to some thousands of them and quadratic beyond: one token each, assigned and
// released, 12 us for 1024 entries, 59 for 8192, 2.1 ms for 65535, the most there may be (of which the assign is 40 us).
#include "kv_cache.cuh"

namespace fp4attn {
namespace {

constexpr int kThreads = 256;

struct AssignParams {
  int *free, *left, *turn;             // the stack, how many are on it, blocks that are through
  int num_pages, log_page;
  int* table;
  int max_pages;
  const int *start, *count;
  long long* slots;
  int* positions;
  int* status;
  int B, N, entries, chunk;            // a block: so many entries, so many of their tokens
};

// pages that n tokens take
__device__ __forceinline__ int pages_of(long long n, int log_page) { return n <= 0 ? 0 : (int)((n + (1 << log_page) - 1) >> log_page); }

struct Need {
  int start, has, fresh;               // fresh: new pages
  bool cut;                            // the table has no room for all of them
};
__device__ __forceinline__ Need need_of(const AssignParams& p, int b) {
  Need n;
  n.start = load(p.start + b);
  const long long s = max(0, n.start), c = p.count ? max(0, load(p.count + b)) : p.N;
  n.has = pages_of(s, p.log_page);
  const int until = pages_of(n.start < 0 ? 0 : s + c, p.log_page), room = min(until, p.max_pages);
  n.fresh = c ? max(0, room - n.has) : 0;
  n.cut = c && until > p.max_pages;
  return n;
}

// sums of two values over the block, of which every thread gets both
__device__ __forceinline__ void block_sums(long long& a, long long& b, long long* scratch) {
#pragma unroll
  for (int s = 16; s; s >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, s);
    b += __shfl_xor_sync(0xffffffffu, b, s);
  }
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0) {
    scratch[2 * warp] = a;
    scratch[2 * warp + 1] = b;
  }
  __syncthreads();
  a = b = 0;
  for (int i = 0; i < kThreads / 32; ++i) {
    a += scratch[2 * i];
    b += scratch[2 * i + 1];
  }
}

constexpr int kMostEntries = kThreads;  // of a block

__global__ void __launch_bounds__(kThreads) assign_kernel(const AssignParams p) {
  __shared__ long long scratch[2 * (kThreads / 32)];
  __shared__ int s_start[kMostEntries], s_has[kMostEntries], s_fresh[kMostEntries];
  __shared__ long long s_base[kMostEntries];
  __shared__ int s_last;
  launch_dependents();
  wait_prior_grids();
  const int e0 = blockIdx.x * p.entries, n_here = min(p.entries, p.B - e0), P = 1 << p.log_page;
  const long long left = max(0, min(load(p.left), p.num_pages));
  long long before = 0, total = 0;
  for (int b = threadIdx.x; b < p.B; b += kThreads) {
    const int f = need_of(p, b).fresh;
    total += f;
    before += b < e0 ? f : 0;
  }
  block_sums(before, total, scratch);
  bool lost = false;
  if ((int)threadIdx.x < n_here) {
    const Need n = need_of(p, e0 + threadIdx.x);
    s_start[threadIdx.x] = n.start;
    s_has[threadIdx.x] = n.has;
    s_fresh[threadIdx.x] = n.fresh;
    lost = n.cut;
  }
  __syncthreads();
  {
    // bases of this block's entries: a scan by the first warps, one entry a thread
    const int f = (int)threadIdx.x < n_here ? s_fresh[threadIdx.x] : 0;
    long long incl = f;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, incl, s);
      if ((threadIdx.x & 31) >= s) incl += o;
    }
    if ((threadIdx.x & 31) == 31) scratch[threadIdx.x >> 5] = incl;
    __syncthreads();
    for (int i = 0; i < (int)threadIdx.x >> 5; ++i) incl += scratch[i];
    if ((int)threadIdx.x < n_here) s_base[threadIdx.x] = before + incl - f;
  }
  // every thread has read the count: the block that is through last writes the new one
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    s_last = atomicAdd(p.turn, 1) == (int)(gridDim.x * gridDim.y) - 1;
  }
  // ---- new pages
  auto fresh_page = [&](int e, int i) {
    const long long at = left - 1 - (s_base[e] + i);
    return at >= 0 ? load(p.free + at) : -1;
  };
  const int per_chunk = p.chunk >> p.log_page, i0 = blockIdx.y * per_chunk;
  const bool last_chunk = blockIdx.y == gridDim.y - 1;
  // a warp an entry; where there are few pages of many entries, a thread an entry
  const bool thread_each = p.entries > kThreads / 32;
  for (int e = thread_each ? threadIdx.x : threadIdx.x >> 5; e < n_here; e += thread_each ? kThreads : kThreads / 32) {
    const int until = last_chunk ? s_fresh[e] : min(s_fresh[e], i0 + per_chunk);
    int* const row = p.table + (size_t)(e0 + e) * p.max_pages + s_has[e];
    for (int i = i0 + (thread_each ? 0 : threadIdx.x & 31); i < until; i += thread_each ? 1 : 32) {
      const int page = fresh_page(e, i);
      row[i] = page;
      lost |= page < 0;
    }
  }
  // ---- slots and positions
  const int t0 = blockIdx.y * p.chunk, tokens = max(0, min(p.chunk, p.N - t0));
  if (p.slots || p.positions) {
    for (unsigned j = threadIdx.x; j < (unsigned)(n_here * tokens); j += kThreads) {
      const int e = j / (unsigned)tokens, t = t0 + (int)(j - (unsigned)e * tokens);
      const int pos = (int)((unsigned)s_start[e] + (unsigned)t);
      const size_t at = (size_t)(e0 + e) * p.N + t;
      if (p.positions) p.positions[at] = pos;
      if (p.slots) {
        long long slot = -1;
        const int i = pos >> p.log_page, has = s_has[e];
        if (pos >= 0 && i < p.max_pages && (!p.count || t < load(p.count + e0 + e))) {
          const int page = i < has ? load(p.table + (size_t)(e0 + e) * p.max_pages + i) : i < has + s_fresh[e] ? fresh_page(e, i - has) : -1;
          if (page >= 0 && page < p.num_pages) slot = ((long long)page << p.log_page) + (pos & (P - 1));
        }
        p.slots[at] = slot;
      }
    }
  }
  if (lost && p.status) *p.status = FP4ATTN_ERR_PAGE;
  __syncthreads();
  if (threadIdx.x == 0 && s_last) {
    __threadfence();
    *p.left = (int)max(0ll, left - total);
    *p.turn = 0;
  }
}

struct ReleaseParams {
  int *free, *left;
  int num_pages, log_page;
  int* table;
  int max_pages;
  const int *length, *keep;
  int* counts;                         // [B] pages of an entry that go; [B]: how many were free before
  int* status;
  int B;
};
__device__ __forceinline__ int2 range_of(const ReleaseParams& p, int b) {
  return make_int2(p.keep ? pages_of(load(p.keep + b), p.log_page) : 0, min(pages_of(load(p.length + b), p.log_page), p.max_pages));
}
constexpr int kMostReleaseThreads = 512;                            // of a block: 128, or as many for long tables
__global__ void __launch_bounds__(kMostReleaseThreads) release_count_kernel(const ReleaseParams p) {
  launch_dependents();
  wait_prior_grids();
  const int b = blockIdx.x, threads = blockDim.x;
  const int2 r = range_of(p, b);
  int mine = 0;
  for (int i = r.x + threadIdx.x; i < r.y; i += threads) {
    const int page = load(p.table + (size_t)b * p.max_pages + i);
    mine += page >= 0 && page < p.num_pages;
  }
  __shared__ int warps[kMostReleaseThreads / 32];
  mine = __reduce_add_sync(0xffffffffu, mine);
  if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < threads / 32; ++i) mine += warps[i];
    p.counts[b] = mine;
    if (b == 0) p.counts[p.B] = max(0, min(load(p.left), p.num_pages));
  }
}
__global__ void __launch_bounds__(kMostReleaseThreads) release_push_kernel(const ReleaseParams p) {
  __shared__ int warps[kMostReleaseThreads / 32];
  __shared__ long long sums[2 * (kMostReleaseThreads / 32)];
  launch_dependents();
  wait_prior_grids();
  const int b = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, threads = blockDim.x;
  const int2 r = range_of(p, b);
  if (b != 0 && r.x >= r.y) return;
  long long before = 0, total = 0;
  for (int i = threadIdx.x; i < p.B; i += threads) {
    const int c = load(p.counts + i);
    total += c;
    before += i < b ? c : 0;
  }
#pragma unroll
  for (int s = 16; s; s >>= 1) {
    before += __shfl_xor_sync(0xffffffffu, before, s);
    total += __shfl_xor_sync(0xffffffffu, total, s);
  }
  if (lane == 0) {
    sums[2 * warp] = before;
    sums[2 * warp + 1] = total;
  }
  __syncthreads();
  before = total = 0;
  for (int i = 0; i < threads / 32; ++i) {
    before += sums[2 * i];
    total += sums[2 * i + 1];
  }
  const long long left = load(p.counts + p.B);
  bool lost = left + total > p.num_pages;
  if (b == 0 && threadIdx.x == 0) *p.left = (int)min(left + total, (long long)p.num_pages);
  for (int i0 = r.x; i0 < r.y; i0 += threads) {
    const int i = i0 + threadIdx.x;
    int* const at = p.table + (size_t)b * p.max_pages + i;
    const int page = i < r.y ? load(at) : -1;
    const bool goes = page >= 0 && page < p.num_pages;
    const uint32_t votes = __ballot_sync(0xffffffffu, goes);
    if (lane == 0) warps[warp] = __popc(votes);
    __syncthreads();
    long long rank = before + __popc(votes & ((1u << lane) - 1));
    for (int k = 0; k < threads / 32; ++k) {
      if (k < warp) rank += warps[k];
      before += warps[k];
    }
    __syncthreads();
    if (goes) {
      const long long to = left + total - 1 - rank;
      if (to < p.num_pages) p.free[to] = page;                      // (more than there are: released twice)
    }
    if (i < r.y) *at = -1;
  }
  if (lost && threadIdx.x == 0 && p.status) *p.status = FP4ATTN_ERR_PAGE;
}

int check_pool(const fp4attn_page_pool* pool, int B, const int* table, int max_pages) {
  if (!pool || !pool->free || !pool->count || !pool->turn || !table || B <= 0 || max_pages <= 0 || pool->num_pages <= 0 || pool->page_size <= 0)
    return FP4ATTN_ERR_INVALID_ARG;
  if (log2_page(pool->page_size) < 0 || B > 65535 || (long long)max_pages * pool->page_size >= (1ll << 30)) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  if (((uintptr_t)pool->free | (uintptr_t)pool->count | (uintptr_t)pool->turn | (uintptr_t)table) & 3) return FP4ATTN_ERR_ALIGNMENT;
  return FP4ATTN_OK;
}

}  // namespace
}  // namespace fp4attn

using namespace fp4attn;

extern "C" int fp4attn_pages_assign(const fp4attn_page_pool* pool, int B, int N, int* block_table, int max_pages, const int* start, const int* count,
                                    long long* slots, int* positions, int* device_status, fp4attn_stream_t stream) {
  int rc = check_pool(pool, B, block_table, max_pages);
  if (rc != FP4ATTN_OK) return rc;
  if (!start || N < 0 || (!count && !N) || ((slots || positions) && !N)) return FP4ATTN_ERR_INVALID_ARG;
  if (N >= (1 << 30)) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  if (((uintptr_t)start | (uintptr_t)count | (uintptr_t)positions | (uintptr_t)device_status) & 3 || ((uintptr_t)slots & 7)) return FP4ATTN_ERR_ALIGNMENT;
  if ((rc = check_device_sm100()) != FP4ATTN_OK) return rc;
  AssignParams p = {};
  p.free = pool->free; p.left = pool->count; p.turn = pool->turn;
  p.num_pages = pool->num_pages; p.log_page = log2_page(pool->page_size);
  p.table = block_table; p.max_pages = max_pages;
  p.start = start; p.count = count; p.slots = slots; p.positions = positions; p.status = device_status;
  p.B = B; p.N = N;
  const int tokens = N < 1 ? 1 : N;
  p.chunk = 2048;                                                   // a multiple of every page
  p.entries = tokens >= p.chunk ? 1 : p.chunk / tokens < kMostEntries ? p.chunk / tokens : kMostEntries;
  if ((tokens + p.chunk - 1) / p.chunk > 65535) p.chunk = 1 << 15;
  const dim3 grid((unsigned)((B + p.entries - 1) / p.entries), (unsigned)((tokens + p.chunk - 1) / p.chunk));
  const cudaError_t e = launch_overlapped(assign_kernel, grid, kThreads, 0, (cudaStream_t)stream, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
}

extern "C" size_t fp4attn_pages_release_workspace_bytes(int B) { return B <= 0 || B > 65535 ? 0 : ((size_t)B + 1) * 4; }

extern "C" int fp4attn_pages_release(const fp4attn_page_pool* pool, int B, int* block_table, int max_pages, const int* length, const int* keep,
                                     int* device_status, void* workspace, size_t workspace_bytes, fp4attn_stream_t stream) {
  int rc = check_pool(pool, B, block_table, max_pages);
  if (rc != FP4ATTN_OK) return rc;
  if (!length) return FP4ATTN_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < fp4attn_pages_release_workspace_bytes(B)) return FP4ATTN_ERR_WORKSPACE;
  if (((uintptr_t)length | (uintptr_t)keep | (uintptr_t)device_status | (uintptr_t)workspace) & 3) return FP4ATTN_ERR_ALIGNMENT;
  if ((rc = check_device_sm100()) != FP4ATTN_OK) return rc;
  ReleaseParams p = {};
  p.free = pool->free; p.left = pool->count;
  p.num_pages = pool->num_pages; p.log_page = log2_page(pool->page_size);
  p.table = block_table; p.max_pages = max_pages;
  p.length = length; p.keep = keep; p.counts = (int*)workspace; p.status = device_status;
  p.B = B;
  const unsigned threads = max_pages > 256 ? kMostReleaseThreads : 128;
  cudaError_t e = launch_overlapped(release_count_kernel, dim3((unsigned)B), threads, 0, (cudaStream_t)stream, p);
  if (e == cudaSuccess) e = launch_overlapped(release_push_kernel, dim3((unsigned)B), threads, 0, (cudaStream_t)stream, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
}
