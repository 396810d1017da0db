// Quantizing K and V into the pages of a cache, and reading them back.
//
// Both are bound by HBM: 2 bytes an element on the 16-bit side, 9/16 or 1 in the cache.  A block takes some tokens of one KV head, half
// of its threads K and half V, 64 elements a thread (128: too few threads); nothing goes through shared memory and no thread waits for another block's work.
//   K  is kept token by token: a thread takes sixteen elements of one token (an NVFP4 block) to write, eight to read.
//   V  is kept in chunks of sixteen tokens at one pair of elements (E4M3: one element): a thread takes eight elements of eight tokens, half of
//      such chunks, and turns bytes around in registers, so that the 16-bit side is accessed 16 bytes and the cache 8 bytes at a time, neighbouring
//      lanes at neighbouring addresses.  Where a call's tokens do not fill an eight, V's bytes are written one by one: the others belong to
//      tokens that are there already.
// NVFP4, d = 128, 8 KV heads: write of 4 x 4096 tokens 25 us (3.4 TB/s; through shared memory, a head after another, 50), read of 4 x 8192 39 us
// (4.4 TB/s; 57).  What is left is instructions (ALU 54 %, issue 59 % of the write and 70 % of the read) at the occupancy that registers allow: two
// divisions a block (for V in both lanes that share it), a page looked up for every piece of K.  With rotary positions the same write takes
// 96 us: 122 to 128 registers, and ranges of heads that divide unevenly; rotary of K and a plain write after it take less than half.
#include "kv_cache.cuh"

namespace fp4attn {
namespace {

constexpr int kThreads = 128, kHalf = 64;
template <int D> constexpr int kBlockTokens = 4096 / D;           // 64 threads of 64 elements

template <typename T>
struct WriteParams {
  View<const T> k, v;
  CacheRef cache;
  const int *start, *count, *positions;
  const float* inv_freq;
  int* status;
  int B, N, heads_per_block, pairs;
  float factor;
  bool vector, interleaved;
};

// eight elements from x on, as four words
template <typename T>
__device__ __forceinline__ uint4 load8(const T* x, bool vector) {
  if (vector) return load(reinterpret_cast<const uint4*>(x));
  const uint16_t* y = reinterpret_cast<const uint16_t*>(x);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (uint32_t)load(y + 2 * i) | (uint32_t)load(y + 2 * i + 1) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void store8(T* y, bool vector, uint4 raw) {
  if (vector) {
    *reinterpret_cast<uint4*>(y) = raw;
    return;
  }
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  uint16_t* z = reinterpret_cast<uint16_t*>(y);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    z[2 * i] = (uint16_t)w[i];
    z[2 * i + 1] = (uint16_t)(w[i] >> 16);
  }
}
template <typename T>
__device__ __forceinline__ void unpack8(uint4 raw, float* v) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack2<T>(w[i]);
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
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
    if (whole && e0 < 2 * pairs) {
      unpack8<T>(load8(row + other, true), w);
      unpack8<T>(load8(row + other + 8, true), w + 8);
    }
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

// NaN counts as 0 (the cache holds finite values only)
template <int N>
__device__ __forceinline__ float clean_max(float* v) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = v[i] == v[i] ? v[i] : 0.f;
    a = fmaxf(a, fabsf(v[i]));
  }
  return a;
}
// scale byte of an NVFP4 block of largest magnitude a, and the factor on its elements
__device__ __forceinline__ float nvfp4_scale(float a, float G, uint32_t* byte) {
  *byte = cvt_e4m3x2(__fdiv_rn(__fmul_rn(a, G), 6.f), 0.f) & 0xFFu;
  const float S = e4m3_value(*byte);
  return S > 0.f ? __fdiv_rn(G, S) : 0.f;
}
__device__ __forceinline__ uint32_t e4m3x4(const float* v, float G) {
  return cvt_e4m3x2(__fmul_rn(v[0], G), __fmul_rn(v[1], G)) | cvt_e4m3x2(__fmul_rn(v[2], G), __fmul_rn(v[3], G)) << 16;
}
// byte j of word i <-> byte i of word j
__device__ __forceinline__ void transpose_bytes(uint32_t (&w)[4]) {
  const uint32_t a = __byte_perm(w[0], w[1], 0x5140), b = __byte_perm(w[2], w[3], 0x5140);
  const uint32_t c = __byte_perm(w[0], w[1], 0x7362), d = __byte_perm(w[2], w[3], 0x7362);
  w[0] = __byte_perm(a, b, 0x5410);
  w[1] = __byte_perm(a, b, 0x7632);
  w[2] = __byte_perm(c, d, 0x5410);
  w[3] = __byte_perm(c, d, 0x7632);
}

// the tokens of a block: `pos0` its first place in the sequence, a multiple of its tokens; first .. last - 1 those that the call has
template <int D>
struct Span {
  long long pos0, first, last;
  int start;
  __device__ __forceinline__ Span(const int* starts, const int* counts, int N, int b) {
    start = load(starts + b);
    const int n = counts ? max(0, min(load(counts + b), N)) : N;
    constexpr int kTokens = kBlockTokens<D>;
    pos0 = ((long long)(start >= 0 ? start / kTokens : -((kTokens - 1 - (long long)start) / kTokens)) + blockIdx.x) * kTokens;
    first = max((long long)start, pos0);
    last = min((long long)start + n, pos0 + kTokens);
  }
  __device__ __forceinline__ bool has(int tok) const { return pos0 + tok >= first && pos0 + tok < last; }
  __device__ __forceinline__ int index(int tok) const { return (int)(pos0 + tok - start); }
};

// Grid: blocks of the sequence, batch, head ranges.  GENERAL: with rotary positions, or rows that take no 16-byte accesses (an instance of
// its own: either costs the plain one registers that it does not have).
template <typename T, int FMT, int D, bool GENERAL>
__global__ void __launch_bounds__(kThreads, GENERAL ? 4 : 6) cache_write_kernel(const WriteParams<T> p) {
  using L = RecordLayout<FMT, D>;
  extern __shared__ float2 table[];                               // [tokens][pairs]: cosines and sines
  launch_dependents();
  wait_prior_grids();
  const int b = blockIdx.y, tid = threadIdx.x;
  const Span<D> span(p.start, p.count, p.N, b);
  if (span.first >= span.last) return;
  const int P = 1 << p.cache.log_page;
  const bool vector = GENERAL ? p.vector : true;
  if (GENERAL && p.pairs) {
    const int t_first = (int)(span.first - span.pos0), t_count = (int)(span.last - span.first);
    for (int j = tid; j < t_count * p.pairs; j += kThreads) {
      const int t = t_first + j / p.pairs, f = j % p.pairs;
      const int at = p.positions ? load(p.positions + (size_t)b * p.N + span.index(t)) : (int)(span.pos0 + t);
      table[t * p.pairs + f] = cos_sin(at, load(p.inv_freq + f), p.factor);
    }
    __syncthreads();
  }
  bool lost = false;
  const int h_end = min((int)(blockIdx.z + 1) * p.heads_per_block, p.cache.kv_heads);
  for (int h = blockIdx.z * p.heads_per_block; h < h_end; ++h) {
    if (tid < kHalf) {
      // ---- V: eight elements of eight tokens
      constexpr int kLanes = D / 8, kRows = L::kFp4 ? 4 : 8;        // chunks of a thread, half of each
      const int t0 = tid / kLanes * 8, e8 = tid % kLanes;
      if (span.pos0 + t0 >= span.last || span.pos0 + t0 + 8 <= span.first) continue;
      const int page = p.cache.page_of(b, span.pos0 + t0);          // a page holds whole eights
      lost |= page < 0;
      if (page < 0) continue;
      const float G = load(p.cache.v_G + h);
      uint32_t rows[kRows][2], sc[2] = {0u, 0u};
      uint32_t have = 0;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        uint4 raw[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int t = t0 + 4 * q + y;
          raw[y] = make_uint4(0u, 0u, 0u, 0u);
          if (span.has(t)) {
            raw[y] = load8(p.v.row(b, h, span.index(t)) + 8 * e8, vector);
            have |= 1u << (4 * q + y);
          }
        }
        uint32_t lo[4], hi[4];                                      // codes of the four tokens; E4M3: of elements 0-3 and 4-7
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          float v[8];
          unpack8<T>(raw[y], v);
          float a = clean_max<8>(v);
          if (L::kFp4) {
            a = fmaxf(a, __shfl_xor_sync(3u << (tid & 30), a, 1));
            uint32_t byte;
            const float r = nvfp4_scale(a, G, &byte);
#pragma unroll
            for (int z = 0; z < 8; ++z) v[z] = __fmul_rn(v[z], r);
            lo[y] = cvt_e2m1x8(v);
            const int at = v_scale_place(4 * q + y);
            sc[at >> 2] |= byte << (8 * (at & 3));
          } else {
            lo[y] = e4m3x4(v, G);
            hi[y] = e4m3x4(v + 4, G);
          }
        }
        transpose_bytes(lo);
        if (!L::kFp4) transpose_bytes(hi);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          rows[y][q] = lo[y];
          if (!L::kFp4) rows[kRows - 4 + y][q] = hi[y];
        }
      }
      uint8_t* const rec = p.cache.rec(page, h);
      const int in_page = (int)((span.pos0 + t0) & (P - 1));
      uint8_t* const chunks = rec + L::v_codes(P) + (in_page & ~15) * L::kRow + kRows * e8 * 16 + (in_page & 8);
      uint8_t* const scales = rec + L::v_scales(P) + (e8 >> 1) * P + in_page;
      if (have == 0xFFu) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) *reinterpret_cast<uint2*>(chunks + 16 * r) = make_uint2(rows[r][0], rows[r][1]);
        if (L::kFp4 && !(e8 & 1)) *reinterpret_cast<uint2*>(scales) = make_uint2(sc[0], sc[1]);
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          if (!(have >> t & 1)) continue;
#pragma unroll
          for (int r = 0; r < kRows; ++r) chunks[16 * r + t] = (uint8_t)(rows[r][t >> 2] >> (8 * (t & 3)));
          const int at = v_scale_place(t);
          if (L::kFp4 && !(e8 & 1)) scales[at] = (uint8_t)(sc[at >> 2] >> (8 * (at & 3)));
        }
      }
    } else {
      // ---- K: sixteen elements of a token at a time
      constexpr int kParts = D / 16, kPieces = kBlockTokens<D> * kParts / kHalf, kAtOnce = 2;
      const float G = load(p.cache.k_G + h);
#pragma unroll 1
      for (int q0 = 0; q0 < kPieces; q0 += kAtOnce) {
        uint4 raw[kAtOnce][2];
        int page[kAtOnce];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
          const int j = (q0 + q) * kHalf + tid - kHalf, t = j / kParts, part = j % kParts;
          page[q] = -1;
          if (!span.has(t)) continue;
          const T* const x = p.k.row(b, h, span.index(t)) + 16 * part;
          raw[q][0] = load8(x, vector);
          raw[q][1] = load8(x + 8, vector);
          page[q] = p.cache.page_of(b, span.pos0 + t);
          lost |= page[q] < 0;
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
          if (page[q] < 0) continue;
          const int j = (q0 + q) * kHalf + tid - kHalf, t = j / kParts, part = j % kParts;
          float v[16];
          unpack8<T>(raw[q][0], v);
          unpack8<T>(raw[q][1], v + 8);
          if (GENERAL && p.pairs) rotate16<T, D>(p.k.row(b, h, span.index(t)), 16 * part, vector, p.interleaved, p.pairs, table + t * p.pairs, v);
          const float a = clean_max<16>(v);
          uint8_t* const rec = p.cache.rec(page[q], h);
          const int in_page = (int)((span.pos0 + t) & (P - 1));
          if (L::kFp4) {
            uint32_t byte;
            const float r = nvfp4_scale(a, G, &byte);
#pragma unroll
            for (int z = 0; z < 16; ++z) v[z] = __fmul_rn(v[z], r);
            *reinterpret_cast<uint2*>(rec + ((part >> 1) * P + in_page) * 16 + (part & 1) * 8) = make_uint2(cvt_e2m1x8(v), cvt_e2m1x8(v + 8));
            rec[L::k_scales(P) + in_page * L::kScales + part] = (uint8_t)byte;
          } else {
            *reinterpret_cast<uint4*>(rec + (part * P + in_page) * 16) = make_uint4(e4m3x4(v, G), e4m3x4(v + 4, G), e4m3x4(v + 8, G), e4m3x4(v + 12, G));
          }
        }
      }
    }
  }
  if (lost && p.status) *p.status = FP4ATTN_ERR_PAGE;
}

template <typename T>
struct ReadParams {
  View<T> k, v;
  CacheRef cache;
  const int *start, *count;
  int* status;
  int B, N;
  bool vector;
};

// eight values, of eight E2M1 codes and their scale or of eight E4M3 bytes: code * scale is exact in f16
template <typename T>
__device__ __forceinline__ uint4 values_e2m1(uint32_t codes, uint32_t scale_splat, float r) {
  uint32_t h[4], w[4];
  cvt_f16x2_e2m1x8(codes, h);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&h[i]), *reinterpret_cast<const __half2*>(&scale_splat));
    const float2 f = __half22float2(x);
    w[i] = pack_pair<T>(f.x * r, f.y * r);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ uint4 values_e4m3(uint32_t lo, uint32_t hi, float r) {
  uint32_t h[4], w[4];
  cvt_f16x2_e4m3x4(lo, h);
  cvt_f16x2_e4m3x4(hi, h + 2);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = half2_of(h[i]);
    w[i] = pack_pair<T>(f.x * r, f.y * r);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint32_t e4m3_splat(uint32_t byte) { return cvt_f16x2_e4m3x2(byte * 0x0101u); }

// As cache_write_kernel.  A value is code * scale (exact) * fl(1 / G), rounded once more to T: two units in the last place of
// fp32 beside the quotient by G, which would take as long as reading the cache.
template <typename T, int FMT, int D>
__global__ void __launch_bounds__(kThreads, 8) cache_read_kernel(const ReadParams<T> p) {
  using L = RecordLayout<FMT, D>;
  launch_dependents();
  wait_prior_grids();
  const int b = blockIdx.y, h = blockIdx.z, tid = threadIdx.x;
  const Span<D> span(p.start, p.count, p.N, b);
  if (span.first >= span.last) return;
  const int P = 1 << p.cache.log_page;
  constexpr int kLanes = D / 8;
  bool lost = false;
  if (tid < kHalf) {
    // ---- V: eight elements of eight tokens
    constexpr int kRows = L::kFp4 ? 4 : 8;
    const int t0 = tid / kLanes * 8, e8 = tid % kLanes;
    if (span.pos0 + t0 < span.last && span.pos0 + t0 + 8 > span.first) {
      const int page = p.cache.page_of(b, span.pos0 + t0);
      lost |= page < 0;
      uint2 rows[kRows], sc = make_uint2(0u, 0u);
#pragma unroll
      for (int r = 0; r < kRows; ++r) rows[r] = make_uint2(0u, 0u);
      if (page >= 0) {
        const uint8_t* const rec = p.cache.rec(page, h);
        const int in_page = (int)((span.pos0 + t0) & (P - 1));
        const uint8_t* const chunks = rec + L::v_codes(P) + (in_page & ~15) * L::kRow + kRows * e8 * 16 + (in_page & 8);
#pragma unroll
        for (int r = 0; r < kRows; ++r) rows[r] = load(reinterpret_cast<const uint2*>(chunks + 16 * r));
        if (L::kFp4) sc = load(reinterpret_cast<const uint2*>(rec + L::v_scales(P) + (e8 >> 1) * P + in_page));
      }
      const float r = __fdiv_rn(1.f, load(p.cache.v_G + h));
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          lo[y] = q ? rows[y].y : rows[y].x;
          hi[y] = q ? rows[kRows - 4 + y].y : rows[kRows - 4 + y].x;
        }
        transpose_bytes(lo);
        if (!L::kFp4) transpose_bytes(hi);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int t = t0 + 4 * q + y, at = v_scale_place(4 * q + y);
          if (!span.has(t)) continue;
          const uint4 out = L::kFp4 ? values_e2m1<T>(lo[y], e4m3_splat((at & 4 ? sc.y : sc.x) >> (8 * (at & 3)) & 0xFFu), r)
                                    : values_e4m3<T>(lo[y], hi[y], r);
          store8(p.v.row(b, h, span.index(t)) + 8 * e8, p.vector, out);
        }
      }
    }
  } else {
    // ---- K: eight elements of a token at a time
    constexpr int kPieces = kBlockTokens<D> * kLanes / kHalf, kAtOnce = 8;
    const float r = __fdiv_rn(1.f, load(p.cache.k_G + h));
#pragma unroll 1
    for (int q0 = 0; q0 < kPieces; q0 += kAtOnce) {
      uint2 raw[kAtOnce];                                           // NVFP4: codes and the scale's byte
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        const int j = (q0 + q) * kHalf + tid - kHalf, t = j / kLanes, e8 = j % kLanes;
        raw[q] = make_uint2(0u, 0u);
        if (!span.has(t)) continue;
        const int page = p.cache.page_of(b, span.pos0 + t);
        lost |= page < 0;
        if (page < 0) continue;                                     // zeros
        const uint8_t* const rec = p.cache.rec(page, h);
        const int in_page = (int)((span.pos0 + t) & (P - 1));
        if (L::kFp4) {
          raw[q].x = load(reinterpret_cast<const uint32_t*>(rec + ((e8 >> 2) * P + in_page) * 16 + (e8 & 3) * 4));
          raw[q].y = load(rec + L::k_scales(P) + in_page * L::kScales + (e8 >> 1));
        } else {
          raw[q] = load(reinterpret_cast<const uint2*>(rec + ((e8 >> 1) * P + in_page) * 16 + (e8 & 1) * 8));
        }
      }
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        const int j = (q0 + q) * kHalf + tid - kHalf, t = j / kLanes, e8 = j % kLanes;
        if (!span.has(t)) continue;
        const uint4 out = L::kFp4 ? values_e2m1<T>(raw[q].x, e4m3_splat(raw[q].y), r) : values_e4m3<T>(raw[q].x, raw[q].y, r);
        store8(p.k.row(b, h, span.index(t)) + 8 * e8, p.vector, out);
      }
    }
  }
  if (lost && p.status) *p.status = FP4ATTN_ERR_PAGE;
}

template <typename T, int FMT, int D>
int launch_write(WriteParams<T> p, cudaStream_t st) {
  const int sms = device_sms(), blocks = (int)(((long long)p.N + kBlockTokens<D> - 2) / kBlockTokens<D> + 1);    // N tokens touch at most so many
  if (!sms) return FP4ATTN_ERR_CUDA;
  // Heads of a block: one - its loads then wait for nothing but each other -, or where they share the cosines and sines of their tokens as
  // many as leave four blocks an SM
  long long per = p.pairs ? (long long)blocks * p.B * p.cache.kv_heads / (4ll * sms) : 1;
  if (per < 1) per = 1;
  if (per > p.cache.kv_heads) per = p.cache.kv_heads;
  p.heads_per_block = (int)per;
  const dim3 grid((unsigned)blocks, (unsigned)p.B, (unsigned)((p.cache.kv_heads + per - 1) / per));
  const cudaError_t e = p.pairs || !p.vector
                            ? launch_overlapped(cache_write_kernel<T, FMT, D, true>, grid, kThreads, sizeof(float2) * kBlockTokens<D> * p.pairs, st, p)
                            : launch_overlapped(cache_write_kernel<T, FMT, D, false>, grid, kThreads, 0, st, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
}
template <typename T, int FMT, int D>
int launch_read(ReadParams<T> p, cudaStream_t st) {
  const int blocks = (int)(((long long)p.N + kBlockTokens<D> - 2) / kBlockTokens<D> + 1);
  const cudaError_t e = launch_overlapped(cache_read_kernel<T, FMT, D>, dim3((unsigned)blocks, (unsigned)p.B, (unsigned)p.cache.kv_heads), kThreads, 0, st, p);
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
