// What the kernels that attend over a cache have in common: waits, arithmetic on pairs, equal runs of tiles for the CTAs.
#pragma once
#include "kv_cache.cuh"
#include "ptx.cuh"

namespace fp4attn {

// Attention of few rows per KV head with the masks and scores of fp4attn_paged_attention (tree_attn.cu): does a call have few, the workspace, the launch.
struct FewRows {
  const fp4attn_view* q;
  CacheRef cache;
  const int *context, *count, *first, *last;
  const float* slopes;
  void* out;
  float* lse;
  int* status;
  int type, fmt, d, B, H, T;
  float scale, cap;
  bool changed() const { return first || last || slopes || cap > 0.f; }       // else: attention over a tree in which every token sees those before it
};
bool few_rows(int rows, int fmt, int d, bool changed);
size_t few_rows_workspace(int B, int H, int kv_heads, int T, int d, int fmt);
int launch_few_rows(const FewRows& a, void* workspace, cudaStream_t st);
int check_cache(const fp4attn_cache* c, int B, const int* block_table, int max_pages, const int* start, const int* count, CacheRef* ref);

namespace {
using namespace ptx;

constexpr int kTile = 128;                 // keys of a tile
constexpr float kLag = 8.f;                // octaves by which a score may exceed its row's reference
constexpr float kShift = 7.f;              // a probability of 1 is 2^7: with the lag just inside f16, whose subnormals then begin at 2^-21

__device__ __forceinline__ bool rare(bool x) { return __builtin_expect(x, 0); }
// Waits for a barrier's phase; the whole warp goes on together.  A wait that runs out, or sees that another one did, sets the abort word
// and returns as if the phase had come: what the roles then read and multiply means nothing, but stays in bounds, and every wait of
// theirs ends at once, so that they run out of tiles.  (Who brings copies asks given_up() behind it.)  The phase has come at the first look,
// or while that look was suspended, in nearly every wait.  CALL: the loop behind it is a function of its own: inlined at each wait it took
// up to 12 % of the time, in instruction fetches.  (Code that shares out registers by setmaxnreg may not call.)
__device__ __forceinline__ void poll_phase(uint32_t bar, uint32_t parity, uint32_t abort_at) {
  uint32_t since = 0;
  for (uint32_t n = 1;; ++n) {
    uint32_t gone;
    asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(gone) : "r"(abort_at) : "memory");
    if (gone || mbar_try_wait(bar, parity)) return;
    if (n % kPolls) continue;
    uint32_t now;
    asm volatile("mov.u32 %0, %%clock;" : "=r"(now));
    if (n == kPolls) since = now;
    if (now - since >= kWaitClocks) break;
  }
  asm volatile("st.volatile.shared.u32 [%0], 1;" ::"r"(abort_at) : "memory");
}
__device__ __noinline__ void wait_longer(uint32_t bar, uint32_t parity, uint32_t abort_at) { poll_phase(bar, parity, abort_at); }
template <bool CALL>
__device__ __forceinline__ void wait_phase(uint32_t bar, uint32_t parity, uint32_t abort_at) {
  if (rare(!mbar_try_wait(bar, parity))) {
    if (CALL) wait_longer(bar, parity, abort_at);
    else poll_phase(bar, parity, abort_at);
  }
  __syncwarp();
}
// Behind a wait for a stage, before anything is brought into it: has some wait run out?  Then those who read stages no longer wait for what
// they read, so that the stage may seem free while its last copies are still under way: a barrier that still expects bytes takes no second
// arrival, and no copy may go where another is.  (One who gives up sets the word before it arrives anywhere, so an arrival that is seen shows
// it.  By a shuffle: a vote, or the wait's own answer voted on, made attention over trees of 64 tokens 2 to 3 % slower.)
__device__ __forceinline__ bool given_up(uint32_t abort_at) {
  uint32_t gone;
  asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(gone) : "r"(abort_at) : "memory");
  return __shfl_sync(0xffffffffu, gone, 0) != 0;
}
// which of N buffers, and the phase of its barriers
template <int N>
struct Turn {
  int at = 0, phase = 0;
  __device__ __forceinline__ void next(int n = 1) {
    if ((at += n) >= N) {
      at -= N;
      phase ^= 1;
    }
  }
};

// The last copies into a ring of STAGES end before the warp that brought `parts` does, also where the others have given up on them: whatever the abort word says,
// but no longer than some tens of milliseconds.  ring: behind the last part.
template <int STAGES>
__device__ __forceinline__ void drain(Turn<STAGES> ring, uint32_t full, int parts) {
#pragma unroll 1
  for (int k = 0; k < STAGES && k < parts; ++k) {
    ring.at = ring.at ? ring.at - 1 : (ring.phase ^= 1, STAGES - 1);
    for (int spin = 0; spin < (1 << 13) && !mbar_try_wait(full + 8 * ring.at, (uint32_t)ring.phase); ++spin) {}
  }
  __syncwarp();
}

template <bool HALF>
__device__ __forceinline__ float2 unpack16(uint32_t w) { return HALF ? unpack2<__half>(w) : unpack2<__nv_bfloat16>(w); }

__device__ __forceinline__ uint32_t splat_half(uint32_t h2, int hi) { return __byte_perm(h2, 0, hi ? 0x3232 : 0x1010); }
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// x = a * b + c, l += a: two at a time
__device__ __forceinline__ void fma_pair(float& x0, float& x1, uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1, uint32_t c0, uint32_t c1) {
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(x0), "=f"(x1) : "r"(a0), "r"(a1), "r"(b0), "r"(b1), "r"(c0), "r"(c1));
}
// x = a * b
__device__ __forceinline__ void mul_pair(float& x0, float& x1, float a0, float a1, float b0, float b1) {
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(x0), "=f"(x1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ void fma_pair(float& x0, float& x1, float a0, float a1, float b0, float b1, float c0, float c1) {
  fma_pair(x0, x1, __float_as_uint(a0), __float_as_uint(a1), __float_as_uint(b0), __float_as_uint(b1), __float_as_uint(c0), __float_as_uint(c1));
}
__device__ __forceinline__ void add_pair(float& l0, float& l1, float a0, float a1) {
  asm("{\n\t.reg .b64 a, l;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 l, {%0, %1};\n\tadd.rn.f32x2 l, l, a;\n\tmov.b64 {%0, %1}, l;\n\t}"
      : "+f"(l0), "+f"(l1) : "f"(a0), "f"(a1));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Biased exponent of the factor of a row of Q whose largest magnitude is a: 2^(14 - exponent of a), at most 2^100 (rows below 2^-86 lose
// bits of scores that are nothing beside any others)
__device__ __forceinline__ uint32_t row_exponent(float a) { return a == 0.f ? 127u : min(268u - (__float_as_uint(a) >> 23), 227u); }

// bits [a, b) of a word, whatever a and b are
__device__ __forceinline__ uint32_t bits_between(int a, int b) {
  const uint32_t from = a <= 0 ? 0xFFFFFFFFu : a >= 32 ? 0u : 0xFFFFFFFFu << a, until = b >= 32 ? 0xFFFFFFFFu : b <= 0 ? 0u : (1u << b) - 1;
  return from & until;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// f16 pairs: NaN and infinities of bytes that nobody wrote become numbers, everything that a cache holds stays (E4M3 ends at 448): a probability
// of 0 times any of them is 0
__device__ __forceinline__ uint32_t finite(uint32_t h2) {
  const __half2 most = __float2half2_rn(448.f), r = __hmin2(*reinterpret_cast<const __half2*>(&h2), most);
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Capped scores, cap tanh u with u = s / cap, are off by no more than 2^-20 of themselves, in every kernel and every job alike (roundings of u beside it):
//   |u| <= 1.25   cap u P(u^2), P of least largest relative error (2^-20.6; by Lawson's weights), seven multiply-adds, two scores at a time
//   beyond        cap - 2 cap / (1 + e^(2|u|)) with the sign of u: the second term, off by 2^-21 of itself, is less than a fifth of the result
// The second form alone is off by 2^-21 of the cap: near 0 it is a difference of two numbers as large as the cap (scores of 10 under a cap of 1e7 were 9.7,
// under 1e9 nothing).  The special-function unit's own tanh is off by 2^-11.
constexpr float kTanhReach = 1.25f * 1.25f;                         // of u^2
__device__ __forceinline__ void tanh_pair(float& t0, float& t1, float w0, float w1) {               // P(w)
  fma_pair(t0, t1, w0, w1, 5.84494090e-4f, 5.84494090e-4f, -4.62690555e-3f, -4.62690555e-3f);
  fma_pair(t0, t1, t0, t1, w0, w1, 1.82291232e-2f, 1.82291232e-2f);
  fma_pair(t0, t1, t0, t1, w0, w1, -5.22054434e-2f, -5.22054434e-2f);
  fma_pair(t0, t1, t0, t1, w0, w1, 1.32906482e-1f, 1.32906482e-1f);
  fma_pair(t0, t1, t0, t1, w0, w1, -3.33293408e-1f, -3.33293408e-1f);
  fma_pair(t0, t1, t0, t1, w0, w1, 9.99999404e-1f, 9.99999404e-1f);
}
// N scores in octaves (of e^s) from their u; out = cap log2 e.  (One look for all of them: with a branch for each pair prompts of 4095 and 1774 tokens with capped
// documents took 254 us instead of 235, and of 4 x 2047 with a bias, which is the same code, 296 instead of 251.)
template <int N>
__device__ __forceinline__ void cap_scores(float (&x)[N], const float (&u)[N], float out) {
  float wide = 0.f;
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    float w0, w1, t0, t1;
    mul_pair(w0, w1, u[i], u[i + 1], u[i], u[i + 1]);
    wide = max3(wide, w0, w1);
    tanh_pair(t0, t1, w0, w1);
    mul_pair(x[i], x[i + 1], u[i], u[i + 1], out, out);
    mul_pair(x[i], x[i + 1], t0, t1, x[i], x[i + 1]);
  }
  if (rare(wide > kTanhReach)) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (u[i] * u[i] > kTanhReach) x[i] = copysignf(fmaf(-2.f * out, rcp_approx(1.f + exp2_approx(fabsf(u[i]) * 2.885390082f)), out), u[i]);
  }
}
// u of a product is it times this, of a row's constant and 1 / out: a number, so that a product of 0 stays 0
__device__ __forceinline__ float cap_constant(float con, float inverse) { return fminf(con * inverse, 0x1.fffffep127f); }
// floor(a * b / c), floor((a + 1) * b / c), ... of tile numbers: in 32 bits where they are enough (64-bit divisions took 0.5 us of the
// smallest calls)
__device__ __forceinline__ constexpr long long div_short(long long a, long long c) {
  return (a | c) < (1ll << 31) ? (long long)((uint32_t)a / (uint32_t)c) : a / c;
}
__device__ __forceinline__ constexpr long long mul_div(long long a, long long b, long long c) { return div_short(a * b, c); }
// the CTA that has a tile of the list, of `total` tiles in equal runs for `ctas`
__device__ __forceinline__ constexpr int cta_of(long long tile, long long total, long long ctas) { return (int)div_short((tile + 1) * ctas - 1, total); }
static_assert(cta_of(0, 5, 2) == 0 && cta_of(1, 5, 2) == 0 && cta_of(2, 5, 2) == 1 && cta_of(4, 5, 2) == 1, "runs 0-1, 2-4");
static_assert(mul_div(1, 5, 2) == 2 && mul_div(2, 5, 2) == 5, "where they begin");
static_assert(cta_of(7, (1ll << 32) + 1, 592) == 0 && cta_of((1ll << 32), (1ll << 32) + 1, 592) == 591 && mul_div(591, 1ll << 33, 592) < 1ll << 33 &&
              cta_of(mul_div(591, 1ll << 33, 592), 1ll << 33, 592) == 591 && cta_of(mul_div(591, 1ll << 33, 592) - 1, 1ll << 33, 592) == 590,
              "more tiles than 32 bits hold");

}  // namespace
}  // namespace fp4attn
