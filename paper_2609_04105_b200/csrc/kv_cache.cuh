// The paged key/value cache as the kernels see it: where a token's bytes are, and how its values are coded.
//
// A (page, KV head) record holds P tokens: K codes, K scales, V codes, V scales (include/fp4attn.h states the layout).  What
// decided it: attention reads a record with one bulk copy and turns it into two tensor-core operands, K with a key per lane
// and V^T with a head-dimension index per lane.  So K is kept in 16-byte chunks of one token, neighbouring tokens side by side
// (a warp reads 32 tokens' chunks without bank conflicts), and V in 16-byte chunks of sixteen tokens at one index.
#pragma once
#include "common.cuh"

namespace fp4attn {

// Every load of a kernel of this path is a coherent one.  A kernel begins before its predecessor has ended, and what it reads (pages, rows,
// tables, positions) may be what that one writes: the non-coherent path (__ldg, ld.global.nc) is defined only for memory that nobody writes
// while the kernel lives.  wait_prior_grids makes what was written visible to ordinary loads.  (As an explicit load, not `*p`: the compiler
// moved the dereferences of the attention kernel's walk to other places, 320 instead of 252 bytes of spills and 102 instead of 98 us.)
template <typename T>
__device__ __forceinline__ T load(const T* p) { return __ldca(p); }

struct CacheRef {
  uint8_t* pages;
  const float *k_G, *v_G;            // one factor per KV head
  const int* table;                  // [B, max_pages]
  int max_pages, num_pages, kv_heads;
  int log_page;                      // log2 of the tokens of a page
  int record;                        // bytes of a (page, head) record

  // page of token `pos` of batch entry b; -1 where the table has none or names none of the cache's
  __device__ __forceinline__ int page_of(int b, long long pos) const {
    const long long i = pos >> log_page;
    if (pos < 0 || i >= max_pages) return -1;
    const int id = load(table + (size_t)b * max_pages + i);
    return id >= 0 && id < num_pages ? id : -1;
  }
  __device__ __forceinline__ uint8_t* rec(int page, int head) const {
    return pages + ((size_t)page * kv_heads + head) * (size_t)record;
  }
};

// Places inside a record of P tokens.  FMT: FP4ATTN_FMT_NVFP4 or FP4ATTN_FMT_E4M3.
template <int FMT, int D>
struct RecordLayout {
  static constexpr bool kFp4 = FMT == FP4ATTN_FMT_NVFP4;
  static constexpr int kRow = kFp4 ? D / 2 : D;          // code bytes of a token
  static constexpr int kScales = kFp4 ? D / 16 : 0;      // scale bytes of a token
  static constexpr int kToken = kRow + kScales;          // bytes of one token's K or V
  __host__ __device__ static constexpr int bytes(int P) { return 2 * P * kToken; }
  __host__ __device__ static constexpr int k_scales(int P) { return P * kRow; }
  __host__ __device__ static constexpr int v_codes(int P) { return P * kToken; }
  __host__ __device__ static constexpr int v_scales(int P) { return P * (kToken + kRow); }
};
// V scales: where in a row of tokens token t stands.  Each eight in the order 0 4 1 5 2 6 3 7: the codes of tokens i and i + 4
// meet in one byte when a lane takes its index's nibbles out of two words, so their scales are kept side by side.
__host__ __device__ __forceinline__ constexpr int v_scale_place(int t) { return (t & ~7) | ((t & 3) << 1) | ((t >> 2) & 1); }

// fp32 x2 -> two E4M3 bytes, to nearest, saturating at 448
__device__ __forceinline__ uint32_t cvt_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(r) : "f"(lo), "f"(hi));
  return r;
}
// two E4M3 bytes -> f16x2, exact
__device__ __forceinline__ uint32_t cvt_f16x2_e4m3x2(uint32_t two_bytes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two_bytes));
  return r;
}
// the two E2M1 codes of byte I of a word -> f16x2 (bits 0-3 in the low half), exact
template <int I>
__device__ __forceinline__ uint32_t cvt_f16x2_e2m1x2(uint32_t word) {
  uint32_t r;
  asm("{\n\t.reg .b8 b;\n\t.reg .b32 s;\n\tshr.b32 s, %1, %2;\n\tcvt.u8.u32 b, s;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(r) : "r"(word), "n"(8 * I));
  return r;
}
// The eight codes of a word, or the four E4M3 bytes, at once: the byte is then taken by the conversion itself (64 conversions a clock
// and SM; 32 with a shift in front of each).  Right for every value of every byte, of words out of memory, permuted, masked, united or extended
// with zeros alike.  (One byte alone so, the other three names unused, gave wrong values where the word was a byte extended with
// zeros: cvt_f16x2_e2m1x2 shifts.)
__device__ __forceinline__ void cvt_f16x2_e2m1x8(uint32_t word, uint32_t* h) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(word));
}
__device__ __forceinline__ void cvt_f16x2_e4m3x4(uint32_t word, uint32_t* h) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(h[0]), "=r"(h[1]) : "r"(word));
}
__device__ __forceinline__ float2 half2_of(uint32_t h2) { return __half22float2(*reinterpret_cast<const __half2*>(&h2)); }
__device__ __forceinline__ float e4m3_value(uint32_t byte) { return half2_of(cvt_f16x2_e4m3x2(byte)).x; }

// ---- 16-bit elements of a tensor, bf16 or fp16
template <typename T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float(float x) { return x; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float(float x) { return __float2half_rn(x); }
// two elements of a 32-bit word
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) { return half2_of(w); }
template <typename T> __device__ __forceinline__ uint32_t pack_pair(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(float lo, float hi) {
  const __half2 p = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// [B, heads, N, d] with any strides (in elements) but the last, which is 1
template <typename T>
struct View {
  T* data;
  long long sb, sh, sn;
  __device__ __forceinline__ T* row(int b, int h, int n) const { return data + b * sb + h * sh + n * sn; }
};
template <typename T>
static inline View<T> view_of(const fp4attn_view& v) {
  return View<T>{static_cast<T*>(v.data), v.stride_b, v.stride_h, v.stride_n};
}
// may every row be read and written in 16-byte pieces?
static inline bool view_vectors(const fp4attn_view& v, int type_bytes) {
  const long long any = v.stride_b | v.stride_h | v.stride_n;
  return (((uintptr_t)v.data | (uintptr_t)(any * type_bytes)) & 15) == 0;
}

// cos and sin of p * f, each to about 2^-50, rounded to fp32 once they are multiplied by the factor.  p * f, its reduction to
// [-pi/4, pi/4] and the Taylor polynomials (to x^15 and x^16: the first terms left out are below 2^-50) are in 64 bits: in fp32 an
// angle of a position of a million is off by 0.03.
__device__ __forceinline__ float2 cos_sin(int p, float f, float factor) {
  const double t = (double)p * (double)f;
  const double n = rint(t * 0.63661977236758134308);                      // 2 / pi
  double x = fma(n, -1.57079632679489655800, t);                          // pi / 2 in two parts
  x = fma(n, -6.12323399573676603587e-17, x);
  const double z = x * x;
  double s = fma(z, -1.0 / 1307674368000.0, 1.0 / 6227020800.0);          // x^15, x^13 ..
  s = fma(z, s, -1.0 / 39916800.0);
  s = fma(z, s, 1.0 / 362880.0);
  s = fma(z, s, -1.0 / 5040.0);
  s = fma(z, s, 1.0 / 120.0);
  s = fma(z, s, -1.0 / 6.0);
  s = fma(z * x, s, x);
  double c = fma(z, 1.0 / 20922789888000.0, -1.0 / 87178291200.0);        // x^16, x^14 ..
  c = fma(z, c, 1.0 / 479001600.0);
  c = fma(z, c, -1.0 / 3628800.0);
  c = fma(z, c, 1.0 / 40320.0);
  c = fma(z, c, -1.0 / 720.0);
  c = fma(z, c, 1.0 / 24.0);
  c = fma(z, c, -0.5);
  c = fma(z, c, 1.0);
  const long long q = (long long)n;
  const double cs = (q & 1) ? s : c, sn = (q & 1) ? c : s;
  const double a = (double)factor;
  return make_float2((float)(a * ((q + 1) & 2 ? -cs : cs)), (float)(a * (q & 2 ? -sn : sn)));
}
// the rotation of one pair: products and sum each rounded to fp32, so that every path gives the same bits
__device__ __forceinline__ void rotate_pair(float& a, float& b, float2 cs) {
  const float x = a, y = b;
  a = __fsub_rn(__fmul_rn(x, cs.x), __fmul_rn(y, cs.y));
  b = __fadd_rn(__fmul_rn(y, cs.x), __fmul_rn(x, cs.y));
}

// a power of two from 16 to 128?
static inline int log2_page(int page_size) {
  for (int l = 4; l <= 7; ++l)
    if (page_size == 1 << l) return l;
  return -1;
}

}  // namespace fp4attn
