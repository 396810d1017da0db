// Attention of any number of tokens of every sequence over its pages of a quantized cache, and of a batch that shares long prefixes.
//
// Row (b, h, t) at position p sees keys [first, last), clipped to the keys that are there.  With s the scaled product of q and a key,
//     x = cap tanh(s / cap) (if capped) - slope_h |p - j|,   O = sum_j e^(x_j - m) v_j / sum_j e^(x_j - m),   LSE = m + ln sum_j e^(x_j - m).
//
// Rows are in lanes: S = Q K^T (128 rows x 64 or 128 keys), O += P V (128 rows x d), both on the fifth-generation tensor core with fp32 sums in tensor
// memory.  The rows that read one KV head (tokens x heads of its group, tokens first) are an item's, 256 at a time or, where there are no more,
// 128.  A row's maximum and sum then belong to one thread, and a key is converted once for all rows of the item:
//
//   producer   items, and the pages of a tile of 128 keys -> a ring of stages, K and V by themselves: one bulk copy a page
//   K          codes -> f16 (exact) -> shared memory, a key a row
//   V          codes -> f16 (exact) -> shared memory, V^T: an index of the head dimension a row
//              both: Q of an item, times a power of two per row, -> f16 -> shared memory
//   issuers    of S and of O
//   softmax    two groups of 128 threads, a thread a row: scores -> P, f16, over its own scores in tensor memory, where the product reads it
//
// A job of a softmax group is 64 keys, and it has two places for their scores, so that those of the next job are there when it comes to them (with one place of
// 128 it stood still for two products in between: a chunk of 2048 tokens 1229 us instead of 1112).  Items of more than 128 rows give each group half of the
// rows; those of fewer give it half of the keys of a tile, with a reference, a sum and an O of its own, joined at the item's end.
//
// Few rows (up to 16 a KV head; up to 8 in NVFP4 with d = 128) go to the kernel of warps in tree_attn.cu, and up to 32 with neither mask nor cap nor bias to its
// roles, but for shared prefixes.  (Rule and measurements: at few_rows there.)
//
// What bounds it: instructions.  A softmax warp executes one about every five clocks (waits, branches and instruction fetches among them), a job of 64
// keys is some 250, and an item costs as much as three or four tiles (bringing Q, the first references, writing O).  All 19 warps have 96 registers, so that every instance
// spills, 8 to 96 bytes of stores and 4 to 128 of loads a thread.  2048 tokens of 32 heads over 8 behind 30720, d = 128, NVFP4: 1.04 to 1.07 ms, 1000 to 1025
// TFLOP/s (power: 1780 MHz); two prompts of 4096: 345 to 361 us, 760 to 800 TFLOP/s.  Beside the products of N = 64, whose operands
// come from shared memory (48 clocks instead of 32) and which take longer to issue than to compute (90), exponentials do not count: without them nothing changes.
//
// A row's keys are walked from its last to its first: what a mask cuts off comes where a reference has to be looked for anyway, and a bias by distance falls
// from there on, so that references do not move.
//
// All tiles of all items stand in one list of which every CTA takes an equal run; what an item leaves in several CTAs (maximum, sum, O) is joined by a
// second kernel in the order of its keys, so results repeat bit by bit.  With shared prefixes an item is a prefix's rows of all members of its group, or
// a sequence's rows over its own tokens; every row is joined from both.
//
// References, f16 probabilities and the scale of Q are those of attention over drafted trees (tree_attn.cu).
#include "cache_attn.cuh"

#include <limits.h>
#include <math.h>

#include <algorithm>

namespace fp4attn {

namespace {

constexpr int kMostCtas = 160;             // one an SM; each may leave two partial results
constexpr int kMostGroup = (1 << 16) - 1;  // query heads of a KV head: see divide()

// how a product becomes a score: scaled; scaled and capped; with a bias, and perhaps capped
enum { kScaled, kCapped, kBiased };

struct PagedParams {
  const void* q;
  long long q_sb, q_sh, q_sn;
  CacheRef cache;
  const int *context, *count, *first, *last;
  const int2* ranges;                      // [B * row_tiles]: of the keys that a tile of rows sees, with first or last
  // shared prefixes: of each group, and where its entries begin
  const int *prefix_table, *prefix_length, *group_start;
  int groups, prefix_pages;
  const unsigned long long* mask;          // [B, T] or null
  const float* slopes;
  void* out;
  float* lse;
  int* status;
  float* part;                             // [2 * kMostCtas][rows of an item][D]
  float2* part_ml;                         // [2 * kMostCtas][rows of an item]: reference, sum
  int4* begun;                             // [kMostCtas]: the item that began in a CTA and went on in others: its x, its u, the last CTA; w: is there one
  int2* split;                             // shared: of every item its first and last CTA; first = -1: whole
  float* whole;                            // shared: [2][B, H, T][D] of whole items
  float2* whole_ml;                        // [2][B, H, T]
  int B, H, T, group, row_tiles;           // row_tiles: of a sequence's rows
  unsigned long long by_group, by_tokens;  // for divide()
  float scale, cap;
  bool half, q_vector, out_wide;           // out_wide: O begins at a multiple of 32 bytes
};

// What a CTA has of an item: written by the producer, read by the other roles
struct Item {
  int tiles;                               // of the item here; 0: no item, the end
  int first;                               // first key of the first of them; tiles go from the last keys to the first (see below)
  int lo, hi, ctx;                         // as in Desc
  int b, g, kvh;
  int row0, here, v0, h0;                  // its first row, how many it has; token and head of the first
  int two, copies;                         // more than 128 rows; how often rows are kept (see copies_of)
  int begins, whole;                       // does it begin here, and does all of it lie here
  int last_cta, slot;                      // where it ends; place of its partial result
  long long split;                         // place in p.split
};
constexpr float kMostSum = 32768.f;        // of a job's probabilities: none of them is beyond f16 then
constexpr int kItems = 32;                 // the producer is some ten tiles, hence items, ahead at most

template <int FMT, int D, int RT>
struct PagedCfg {
  using L = RecordLayout<FMT, D>;
  static constexpr int kRows = 128 * RT;                           // of an item
  // warps
  static constexpr int kFirstV = 4, kFirstSoftmax = 8, kProducer = 16, kIssuerS = 17, kIssuerO = 18, kThreads = 32 * 19;
  static constexpr int kStage = kTile * L::kToken;                 // K or V of a tile
  static constexpr int kQ = kRows * D * 2, kOp = kTile * D * 2;    // an operand tile
  static constexpr int kKB = 2, kVB = RT == 2 && D == 128 && !L::kFp4 ? 1 : 2;
  static constexpr int kJoin = RT == 1 ? 8 * 32 * 16 * 4 : 0;      // sixteen columns of O of all copies
  static constexpr int kRing = 32, kRingC = 4;                     // tiles whose pages, items whose constants are remembered
  static constexpr int kItemBytes = kItems * (int)sizeof(Item);
  static constexpr int kFixed = kQ + (kKB + kVB) * kOp + 2048 + 4 * kRows * kRingC + 2048 + 4 * kRing + 256 + 64 + 1024 + 1024 + kJoin + kItemBytes;
  static constexpr int kStages = (227 * 1024 - kFixed) / kStage < 8 ? (227 * 1024 - kFixed) / kStage : 8;
  static_assert(kStages >= 2, "shared memory");
  static constexpr int kOffQ = 0, kOffK = kOffQ + kQ, kOffV = kOffK + kKB * kOp, kOffStage = kOffV + kVB * kOp;
  static constexpr int kOffVScale = kOffStage + kStages * kStage;  // f16 [4 V warps][2 blocks][128 tokens]
  static constexpr int kOffC = kOffVScale + 2048;                  // float [kRingC][kRows]: score constants of the last items
  static constexpr int kOffML = kOffC + 4 * kRows * kRingC;        // float2 [2][128]
  static constexpr int kOffJoin = kOffML + 2048;                   // float [8 softmax warps][32][16]
  static constexpr int kOffValid = kOffJoin + kJoin;                  // u32 [kRing]: pages of a tile that are there
  static constexpr int kOffItems = kOffValid + 4 * kRing;
  static constexpr int kOffScan = kOffItems + kItemBytes;           // i64 [18]
  static constexpr int kOffFind = kOffScan + 256;                  // i64 [2], Desc
  static constexpr int kOffBar = kOffFind + 64;
  static constexpr int kSmem = kOffBar + 1024 + 1024;
  static_assert(kSmem <= 227 * 1024 && kOffStage % 1024 == 0 && kStage % 16 == 0, "shared memory");
  enum { K_FULL = 0, K_FREE = K_FULL + kKB, V_FULL = K_FREE + kKB, V_FREE = V_FULL + kVB, Q_FULL = V_FREE + kVB, Q_FREE, S_FULL, P_FULL = S_FULL + 4,
         PV_DONE = P_FULL + 4, DRAIN = PV_DONE + 4, MEET = DRAIN + 2, RING_FULL, RING_FREE = RING_FULL + kStages, ITEM = RING_FREE + kStages, kBars = ITEM + kItems };
  static_assert(kBars * 8 + 16 <= 1024, "barriers");
  static constexpr int kS = 0, kO = 256;                           // tensor memory: scores (and P) of the two groups, their O
  // a group's two places for scores; with the same rows for both, those of a tile are neighbours
  __device__ static constexpr uint32_t scores_at(uint32_t group, uint32_t place) { return kS + (RT == 1 ? 128 * place + 64 * group : 128 * group + 64 * place); }
};

// tokens that entry b has
__device__ __forceinline__ int tokens_of(const PagedParams& p, int b) { return p.count ? max(0, min(load(p.count + b), p.T)) : p.T; }

// its context: what lies behind every table's room is all the same
__device__ __forceinline__ int context_of(const PagedParams& p, int b) { return max(0, min(load(p.context + b), (1 << 30) - 1)); }

// ---- items.  x: a tile of rows of a sequence (paged); a group's prefix, or a sequence by itself (shared).  All items of an x have as many tiles.
struct Desc {
  int nt;                                  // tiles of an item; 0: no item
  int k0;                                  // its first tile of keys
  int lo, hi, need;                        // keys of the item that may be seen; need: before they are clipped to the table
  int row0, rows, rts;                     // first row (of x's only tile), rows of x, tiles of rows
  int b;                                   // entry, or (prefix) the first of the group
  int g;                                   // group of a prefix, -1
  int ctx, n;                              // of the entry: context, tokens
};
template <int ROWS>
__device__ __forceinline__ void describe(const PagedParams& p, int x, Desc& d) {
  d.g = -1;
  d.row0 = 0;
  d.k0 = 0;
  d.lo = 0;
  long long need;
  int room = p.cache.max_pages << p.cache.log_page;
  if (!p.groups) {
    d.b = x / p.row_tiles;
    d.row0 = (x - d.b * p.row_tiles) * ROWS;
    d.n = tokens_of(p, d.b);
    d.ctx = context_of(p, d.b);
    d.rows = d.n * p.group;
    d.rts = 1;
    d.nt = 0;
    if (d.row0 >= d.rows) return;
    if (p.ranges) {
      const int2 r = load(p.ranges + x);
      d.lo = r.x;
      need = r.y;
    } else {
      need = (long long)d.ctx + (min(d.row0 + ROWS, d.rows) - 1) / p.group + 1;
    }
  } else if (x < p.groups) {
    const int b0 = max(0, min(load(p.group_start + x), p.B)), b1 = max(b0, min(load(p.group_start + x + 1), p.B));
    d.g = x;
    d.b = b0;
    d.ctx = 0;
    d.n = p.T;
    d.rows = (b1 - b0) * p.T * p.group;
    d.rts = (d.rows + ROWS - 1) / ROWS;
    room = p.prefix_pages << p.cache.log_page;
    need = max(0, load(p.prefix_length + x));
    d.nt = 0;
    if (!d.rows || !need) return;
  } else {
    d.b = x - p.groups;
    d.n = tokens_of(p, d.b);
    d.ctx = context_of(p, d.b);
    d.rows = d.n * p.group;
    d.rts = (d.rows + ROWS - 1) / ROWS;
    d.nt = 0;
    if (!d.rows) return;
    need = (long long)d.ctx + d.n;
    room = (int)min((long long)room, (long long)d.ctx + (p.mask ? p.T : d.n));       // (a mask may look behind the count)
  }
  d.need = (int)min(need, (long long)INT_MAX);
  d.hi = p.groups && d.g < 0 ? room : min(d.need, room);
  if (d.lo >= d.hi) {                      // rows that see nothing: one tile, all of it hidden
    d.lo = d.hi = 0;
    d.nt = 1;
  } else {
    d.k0 = d.lo / kTile;
    d.nt = (d.hi + kTile - 1) / kTile - d.k0;
  }
}
// of an item among the entries of p.split.  (Prefixes: those of a group begin behind as many whole tiles as the groups before it can fill.)
template <int ROWS>
__device__ __forceinline__ size_t split_place(const PagedParams& p, const Desc& d, int u) {
  const int kvh = u / d.rts, rt = u - kvh * d.rts;
  const long long rows = (long long)p.T * p.group;
  const long long at = d.g >= 0 ? d.b * rows / ROWS + d.g + rt : p.B * rows / ROWS + p.groups + 1 + (long long)d.b * p.row_tiles + rt;
  return (size_t)at * p.cache.kv_heads + kvh;
}
// n / d for n up to 2^24 (d < 2^12) or 2^17 (d < 2^16): m = ceil(2^36 / d), so that n (m d - 2^36) < n d stays below 2^36.  d is a KV head's query heads (n
// less than 256 more) or a call's tokens (n those of a group): more heads than that are refused.
__device__ __forceinline__ int divide(int n, unsigned long long m) { return (int)((unsigned long long)n * m >> 36); }

// This CTA's run of the list, in units: a tile is one, and an item that many more (bringing Q, writing O), which come before its tiles.  x, the run's
// first unit among x's, how many, the first one's number in the list, all units, CTAs.  Barriers of the block.
constexpr int kItemCost = 3;
struct Run {
  int x;
  long long at, tiles, first, total, ctas;
};
template <int ROWS, int THREADS>
__device__ __forceinline__ Run find_run(const PagedParams& p, long long* scan, long long* find) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int X = p.groups ? p.groups + p.B : p.B * p.row_tiles;
  const int per = (X + THREADS - 1) / THREADS, x0 = min(X, (int)threadIdx.x * per), x1 = min(X, x0 + per);
  Desc d;
  auto tiles = [&](int x) {
    describe<ROWS>(p, x, d);
    return d.nt ? (long long)(d.nt + kItemCost) * d.rts * p.cache.kv_heads : 0ll;
  };
  long long mine = 0;
#pragma unroll 1
  for (int x = x0; x < x1; ++x) mine += tiles(x);
  long long incl = mine;
#pragma unroll 1
  for (int s = 1; s < 32; s <<= 1) {
    const long long o = __shfl_up_sync(0xffffffffu, incl, s);
    if (lane >= s) incl += o;
  }
  if (lane == 31) scan[warp] = incl;
  __syncthreads();
  Run r;
  long long before = 0;
  r.total = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 32; ++i) {
    const long long here = scan[i];
    before += i < warp ? here : 0;
    r.total += here;
  }
  before += incl - mine;
  r.ctas = min((long long)gridDim.x, r.total);
  r.first = blockIdx.x < r.ctas ? mul_div(blockIdx.x, r.total, r.ctas) : r.total;
  r.tiles = blockIdx.x < r.ctas ? mul_div(blockIdx.x + 1, r.total, r.ctas) - r.first : 0;
  if (r.tiles && before <= r.first && r.first < before + mine) {    // one thread
    int x = x0;
    if (per > 1)
      for (;; ++x) {
        const long long here = tiles(x);
        if (r.first < before + here) break;
        before += here;
      }
    find[0] = x;
    find[1] = r.first - before;
    *reinterpret_cast<Desc*>(find + 2) = d;                         // (of x: the one described last)
  }
  __syncthreads();
  r.x = r.tiles ? (int)find[0] : 0;
  r.at = r.tiles ? find[1] : 0;
  return r;
}

// entry, token and head of row r of an item (or of x: the same with v0 = h0 = 0 where r * group is small)
template <class I>
__device__ __forceinline__ void row_token(const PagedParams& p, const I& i, int r, int* b, int* t, int* h) {
  const int at = i.h0 + r, v = divide(at, p.by_group);
  *h = at - v * p.group;
  *b = i.b;
  *t = i.v0 + v;
  if (i.g >= 0) {
    const int e = divide(*t, p.by_tokens);
    *b = i.b + e;
    *t -= e * p.T;
  }
}

// How often the rows of an item stand among the 128 lanes.  A warp's instructions cost the same for one row as for 32, and it sees only its own 32
// lanes of tensor memory: few rows are kept twice or four times, and each copy takes a half or a quarter of the keys of a tile, with a reference, a
// sum and an O of its own, its other probabilities 0.
template <int ROWS>
__device__ __forceinline__ int copies_of(int rows) { return ROWS > 128 || rows > 64 ? 1 : rows > 32 ? 2 : 4; }

// the larger of two magnitudes as row_exponent wants it: a NaN counts as the largest number there is
__device__ __forceinline__ float finite_max(float a, float b) { return fminf(fmaxf(a, b), 0x1.fffffep127f); }
// 32 bytes at once, so aligned
__device__ __forceinline__ void store_32(void* dst, const uint32_t* h) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(dst), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]), "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7]) : "memory");
}
// place of 16-byte chunk c of a row of 128 bytes in a swizzled operand
__device__ __forceinline__ uint32_t chunk_at(int row, int c) { return (uint32_t)(row * 128 + ((c ^ (row & 7)) << 4)); }

template <int FMT, int D, int RT, int SCORES>
__global__ void __launch_bounds__(PagedCfg<FMT, D, RT>::kThreads, 1) paged_kernel(const PagedParams p) {
  using C = PagedCfg<FMT, D, RT>;
  using L = typename C::L;
  constexpr int ROWS = C::kRows;
  constexpr bool CAP = SCORES == kCapped, ANY = SCORES == kBiased;     // ANY: a bias, and perhaps a cap
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const sgen = smem_raw + (sbase - smem_u32(smem_raw));
  const uint32_t abort_at = sbase + C::kOffBar + 8 * C::kBars, tslot = abort_at + 4;
  volatile uint32_t* const abort_word = reinterpret_cast<volatile uint32_t*>(sgen + C::kOffBar + 8 * C::kBars);
  auto bar = [&](int i) { return sbase + C::kOffBar + 8u * i; };
  auto wait = [&](int b, int phase) { wait_phase<true>(bar(b), (uint32_t)phase, abort_at); };
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kBars; ++i) {
      const bool four = (i < C::K_FREE) || (i >= C::V_FULL && i < C::V_FREE) || (i >= C::P_FULL && i < C::PV_DONE) || (i >= C::RING_FREE && i < C::ITEM);
      mbar_init(bar(i), i == C::Q_FULL || i == C::MEET ? 8 : four ? 4 : 1);
    }
    *abort_word = 0;
    fence_barrier_init();
  }
  if (warp == C::kIssuerS) { tmem_alloc(tslot, 512); tmem_relinquish(); }
  tc_fence_before();
  launch_dependents();                                              // the joining kernel: its launch lies under this one
  wait_prior_grids();
  if (threadIdx.x == 0 && p.begun) p.begun[blockIdx.x].w = 0;
  const Run run = find_run<ROWS, C::kThreads>(p, reinterpret_cast<long long*>(sgen + C::kOffScan), reinterpret_cast<long long*>(sgen + C::kOffFind));
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(sgen + C::kOffBar + 8 * C::kBars + 4);
  uint32_t* const valid_ring = reinterpret_cast<uint32_t*>(sgen + C::kOffValid);
  Item* const items = reinterpret_cast<Item*>(sgen + C::kOffItems);
  const int log_page = p.cache.log_page, P = 1 << log_page, half_record = p.cache.record / 2;
  const uint32_t all_pages = (1u << (kTile >> log_page)) - 1;
  // item i of this CTA; none (0 tiles) where some wait ran out
  auto next_item = [&](int i) -> const Item* {
    wait(C::ITEM + (i & (kItems - 1)), i / kItems & 1);
    return items + (i & (kItems - 1));
  };
  auto none = [&](const Item* it) { return it->tiles == 0 || *abort_word; };

  // Q of an item, by the 256 threads that convert K and V.  Rows are scaled by a power of two into f16's range (the largest element to [2^14,
  // 2^15)): exact for 8-bit significands, and a row's scores are scaled back by its constant.  Rows up to the next 32 are written, since a warp of softmax
  // threads takes all of its 32 or none; few rows are written as often as their copies are (see copies_of).
  // All of an item's rows are in these threads' registers, converted, before the buffer is free: then only stores stand between the last scores of an item
  // and the first of the next.
  auto bring_q = [&](const Item* it, int item, int& q_phase) {
    constexpr int kParts = D / 16, kStep = 256 / kParts, kMost = ROWS / kStep;       // threads of a row; how far apart a thread's rows are; how many
    const int here = it->here, kvh = it->kvh, copies = it->copies, rows32 = (here + 31) & ~31, e = (threadIdx.x % kParts) * 16, r0 = threadIdx.x / kParts;
    const float c = __fdiv_rn(p.scale * 1.4426950408889634f, load(p.cache.k_G + kvh));
    uint32_t words[kMost][8];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int r = r0 + kStep * i;
#pragma unroll
      for (int x = 0; x < 8; ++x) words[i][x] = 0u;
      if (r < here) {
        int b, tok, hl;
        row_token(p, *it, r, &b, &tok, &hl);
        const uint16_t* q = static_cast<const uint16_t*>(p.q) + b * p.q_sb + (long long)(kvh * p.group + hl) * p.q_sh + tok * p.q_sn + e;
        if (p.q_vector) {
          *reinterpret_cast<uint4*>(words[i]) = load(reinterpret_cast<const uint4*>(q));
          *reinterpret_cast<uint4*>(words[i] + 4) = load(reinterpret_cast<const uint4*>(q) + 1);
        } else {
#pragma unroll 1
          for (int x = 0; x < 8; ++x) {                               // (shifted in, so that no register is named by a variable)
            const uint32_t w = (uint32_t)load(q + 2 * x) | (uint32_t)load(q + 2 * x + 1) << 16;
#pragma unroll
            for (int y = 0; y < 7; ++y) words[i][y] = words[i][y + 1];
            words[i][7] = w;
          }
        }
      }
    }
    uint32_t ups[(kMost + 3) / 4];                                    // exponents of the rows' factors, a byte each
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      if (r0 + kStep * i >= rows32) break;                            // (a warp's rows are a few neighbours: all or none)
      // the largest magnitude, of pairs as they are (bits without their sign are in order in either type; NaN and infinity come out on top)
      uint32_t a2 = 0u;
#pragma unroll
      for (int x = 0; x < 8; ++x) a2 = __vmaxu2(a2, words[i][x] & 0x7FFF7FFFu);
#pragma unroll
      for (int x = 1; x < kParts; x <<= 1) a2 = __vmaxu2(a2, __shfl_xor_sync(0xffffffffu, a2, x));
      const float2 both = p.half ? unpack16<true>(a2) : unpack16<false>(a2);
      const uint32_t up = row_exponent(finite_max(both.x, both.y));
      const float f = __uint_as_float(up << 23);
      if (p.half) {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const float2 v = unpack16<true>(words[i][x]);
          words[i][x] = pack_pair<__half>(v.x * f, v.y * f);
        }
      } else {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const float2 v = unpack16<false>(words[i][x]);
          words[i][x] = pack_pair<__half>(v.x * f, v.y * f);
        }
      }
      ups[i / 4] = i % 4 ? ups[i / 4] | up << (8 * (i % 4)) : up;
    }
    wait(C::Q_FREE, q_phase);
    q_phase ^= 1;
    float* const con = reinterpret_cast<float*>(sgen + C::kOffC) + (item & (C::kRingC - 1)) * ROWS;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      const int r = r0 + kStep * i;
      if (r >= rows32) break;
      uint8_t* const panel = sgen + C::kOffQ + (r >> 7) * (128 * D * 2) + (e >> 6) * 16384;
#pragma unroll 1
      for (int k = 0; k < copies; ++k) {
        const int to = (r & 127) + k * (128 / copies);
        *reinterpret_cast<uint4*>(panel + chunk_at(to, (e & 63) >> 3)) = *reinterpret_cast<const uint4*>(words[i]);
        *reinterpret_cast<uint4*>(panel + chunk_at(to, ((e & 63) >> 3) + 1)) = *reinterpret_cast<const uint4*>(words[i] + 4);
      }
      if (e == 0) con[r] = c * __uint_as_float((254u - (ups[i / 4] >> (8 * (i % 4)) & 255u)) << 23);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(C::Q_FULL));
  };

  if (warp == C::kProducer) {
    // ===================================================================== items, and pages -> shared memory
    Turn<C::kStages> ring;
    bool lost = false, going = true;                                  // going: every stage waited for has become free
    int parts = 0, x = run.x, u = 0, i = 0;
    long long left = run.tiles, number = run.first, at = run.at;      // number: of the first unit of the run, at: its place in the item
    Desc d;
    if (left > 0) {
      d = *reinterpret_cast<const Desc*>(sgen + C::kOffFind + 16);
      u = (int)mul_div(at, 1, d.nt + kItemCost);
      at -= (long long)u * (d.nt + kItemCost);
    }
    int n = 0;                                                        // items
#pragma unroll 1
    while (left > 0 && going && !*abort_word) {
      // units [at, end) of the item; its tiles are those from unit kItemCost on
      const int from = (int)at, end = (int)min((long long)(d.nt + kItemCost), at + left), tile = max(0, from - kItemCost);
      const long long item0 = number - from;
      left -= end - from;
      number += end - from;
      at = 0;
      const int kvh = u / d.rts, rt = u - kvh * d.rts;
      Item it;
      it.tiles = max(0, end - kItemCost - tile);
      it.first = (d.k0 + d.nt - 1 - tile) * kTile;
      it.lo = d.lo; it.hi = d.hi; it.ctx = d.ctx; it.b = d.b; it.g = d.g; it.kvh = kvh;
      it.row0 = d.row0 + rt * ROWS;
      it.here = min(ROWS, d.rows - it.row0);
      it.v0 = it.row0 / p.group;
      it.h0 = it.row0 - it.v0 * p.group;
      it.two = it.here > 128;
      it.copies = copies_of<ROWS>(it.here);
      it.begins = tile == 0;
      it.whole = it.tiles == d.nt;
      it.last_cta = cta_of(item0 + kItemCost + d.nt - 1, run.total, run.ctas);
      it.slot = 2 * (int)blockIdx.x + it.begins;
      it.split = p.groups ? (long long)split_place<ROWS>(p, d, u) : 0;
      if (lane == 0 && it.tiles) {
        items[n & (kItems - 1)] = it;
        if (!p.groups && it.begins && !it.whole) p.begun[blockIdx.x] = make_int4(x, u, it.last_cta, 1);
        mbar_arrive(bar(C::ITEM + (n & (kItems - 1))));
      }
      __syncwarp();
      n += it.tiles > 0;
      // Q into L2, while the tiles before it are worked on.  (Of a prefix's members some may have no tokens: what only those would see is nobody's loss.)
      bool missing = false, someone = it.g < 0;
#pragma unroll 1
      for (int r = lane; r < it.here && it.tiles; r += 32) {
        int b, tok, hl;
        row_token(p, it, r, &b, &tok, &hl);
        const uint16_t* q = static_cast<const uint16_t*>(p.q) + b * p.q_sb + (long long)(kvh * p.group + hl) * p.q_sh + tok * p.q_sn;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(q));
        if (D == 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + 64));
        if (it.g >= 0) someone |= tok < tokens_of(p, b);
      }
      const int room = (d.g >= 0 ? p.prefix_pages : p.cache.max_pages) << log_page;
      missing |= it.tiles && d.need > d.hi && d.need > room;
      const int* const table = d.g >= 0 ? p.prefix_table + (size_t)d.g * p.prefix_pages : p.cache.table + (size_t)d.b * p.cache.max_pages;
      const uint8_t* const pages = p.cache.pages + (size_t)kvh * p.cache.record;
      const size_t page_bytes = (size_t)p.cache.kv_heads * p.cache.record;
      auto page_at = [&](int first) {                                 // of this lane, -1: none, or not needed
        const int pos = first + lane * P;
        if (lane >= kTile >> log_page || pos >= d.hi || pos + P <= d.lo) return -1;
        const int id = load(table + (pos >> log_page));               // (d.hi is inside the table)
        if (id >= 0 && id < p.cache.num_pages) return id;
        missing |= pos < d.need;
        return -1;
      };
      int page = page_at(it.first);
#pragma unroll 1
      for (int k = 0; k < it.tiles && going; ++k) {
        const uint32_t held = __ballot_sync(0xffffffffu, page >= 0);
        const uint8_t* const rec = pages + (size_t)max(page, 0) * page_bytes;
        const bool mine = page >= 0;
        if (k + 1 < it.tiles) page = page_at(it.first - (k + 1) * kTile);            // (its entry comes while a stage is waited for)
#pragma unroll 1
        for (int part = 0; part < 2; ++part) {
          wait(C::RING_FREE + ring.at, ring.phase ^ 1);
          going = !given_up(abort_at);
          if (rare(!going)) break;
          if (lane == 0) {
            if (part == 0) valid_ring[i % C::kRing] = held;
            mbar_arrive_expect_tx(bar(C::RING_FULL + ring.at), __popc(held) * half_record);
          }
          __syncwarp();
          if (mine)
            bulk_load_1d(sbase + C::kOffStage + ring.at * C::kStage + lane * half_record, rec + part * half_record, half_record, bar(C::RING_FULL + ring.at));
          ring.next();
          ++parts;
        }
        ++i;
      }
      lost |= __any_sync(0xffffffffu, missing) && __any_sync(0xffffffffu, someone);
      if (left > 0 && going && ++u == d.rts * p.cache.kv_heads) {
        u = 0;
        do describe<ROWS>(p, ++x, d);
        while (d.nt == 0);                                            // (there is another item: the run goes on)
      }
    }
    if (lane == 0) {
      items[n & (kItems - 1)].tiles = 0;
      mbar_arrive(bar(C::ITEM + (n & (kItems - 1))));
    }
    if (__any_sync(0xffffffffu, lost) && lane == 0 && p.status) *p.status = FP4ATTN_ERR_PAGE;
    drain(ring, bar(C::RING_FULL), parts);
  } else if (warp == C::kIssuerS || warp == C::kIssuerO) {
    // ===================================================================== products
    // Jobs: 128 rows and 64 keys, of the softmax groups in turn.  A tile has four (both halves of the rows, both of the keys) or, with up to 128 rows,
    // two (a group has a half of the keys).  A group has two places for its scores, so that those of its next job are there when it comes to them; P
    // stands where S did.  A warp each for S and O: what an issuer executes besides products is one chain of instructions, which shares its scheduler with five
    // other warps; in one warp it took twice the time of the products.
    int item = -1, tiles = 0, two = 0, in_item = 0;                   // tiles: left of the item; in_item: jobs of the item so far
    int job = 0;                                                      // of the tile
    uint32_t n = 0;                                                   // jobs so far
    auto another = [&] {                                              // before a job: is there one?
      if (rare(tiles == 0)) {
        const Item* const it = next_item(++item);
        if (none(it)) return false;
        tiles = it->tiles;
        two = it->two;
        in_item = 0;
      }
      return true;
    };
    auto next = [&](bool last) {
      ++n;
      ++in_item;
      ++job;
      if (last) {
        job = 0;
        --tiles;
      }
    };
    if (warp == C::kIssuerS && RT == 1) {
      // Both groups have the same rows and a half of the keys each: one product of N = 128 for both (eight of 64 clocks instead of sixteen, which take more to
      // issue than to compute: 40 sequences of 5 drafted tokens behind six prefixes 43 -> 38 us)
      constexpr uint32_t kIdesc = make_idesc_f16(128, kTile, false);
      const uint64_t q_desc = make_smem_desc(sbase + C::kOffQ, 16, 1024, kSwz128), k_desc = make_smem_desc(sbase + C::kOffK, 16, 1024, kSwz128);
      Turn<C::kKB> kb;
      int q_phase = 0;
#pragma unroll 1
      while (another()) {
        const uint32_t place = n & 1;
        if (rare(in_item == 0)) {
          wait(C::Q_FULL, q_phase);
          q_phase ^= 1;
        }
        wait(C::K_FULL + kb.at, kb.phase);
        wait(C::PV_DONE + place, (n >> 1 & 1) ^ 1);                   // what stood in this place has been read
        wait(C::PV_DONE + 2 + place, (n >> 1 & 1) ^ 1);
        tc_fence_after();
        const uint64_t b = k_desc + (uint32_t)(kb.at * C::kOp >> 4);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const int at = (k >> 2) * (16384 >> 4) + (k & 3) * 2;
            tc_mma_f16(tmem + C::kS + 128 * place, q_desc + at, b + at, kIdesc, k > 0);
          }
          tc_commit(bar(C::S_FULL + place));
          tc_commit(bar(C::K_FREE + kb.at));
          if (tiles == 1) tc_commit(bar(C::Q_FREE));
        }
        __syncwarp();
        kb.next();
        ++n;
        in_item = 1;
        --tiles;
      }
    } else if (warp == C::kIssuerS) {
      constexpr uint32_t kIdesc = make_idesc_f16(128, 64, false);
      const uint64_t q_desc = make_smem_desc(sbase + C::kOffQ, 16, 1024, kSwz128), k_desc = make_smem_desc(sbase + C::kOffK, 16, 1024, kSwz128);
      Turn<C::kKB> kb;
      int q_phase = 0;
#pragma unroll 1
      while (another()) {
        const bool last = job == (two ? 3 : 1);
        const uint32_t group = n & 1, place = n >> 1 & 1;
        if (rare(in_item == 0)) {
          wait(C::Q_FULL, q_phase);
          q_phase ^= 1;
        }
        if (job == 0) wait(C::K_FULL + kb.at, kb.phase);
        wait(C::PV_DONE + 2 * group + place, (n >> 2 & 1) ^ 1);       // what stood in this place has been read
        tc_fence_after();
        // (an address is a sum in a descriptor's low bits)
        const uint64_t a = q_desc + (two ? group * (128 * D * 2 >> 4) : 0u), b = k_desc + (uint32_t)(kb.at * C::kOp + (two ? 1 - (job >> 1) : job) * 8192 >> 4);
        const uint32_t to = tmem + C::scores_at(group, place);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const int at = (k >> 2) * (16384 >> 4) + (k & 3) * 2;
            tc_mma_f16(to, a + at, b + at, kIdesc, k > 0);
          }
          tc_commit(bar(C::S_FULL + 2 * group + place));
          if (last) tc_commit(bar(C::K_FREE + kb.at));
          if (last && tiles == 1) tc_commit(bar(C::Q_FREE));
        }
        __syncwarp();
        if (last) kb.next();
        next(last);
      }
    } else {
      constexpr uint32_t kIdesc = make_idesc_f16(128, D, false);
      const uint64_t v_desc = make_smem_desc(sbase + C::kOffV, 16, 1024, kSwz128);
      Turn<C::kVB> vb;
#pragma unroll 1
      while (another()) {
        const bool last = job == (two ? 3 : 1);
        const uint32_t group = n & 1, place = n >> 1 & 1;
        if (job == 0) wait(C::V_FULL + vb.at, vb.phase);
        const uint64_t b = v_desc + (uint32_t)(vb.at * C::kOp + (two ? 1 - (job >> 1) : job) * (D * 128) >> 4);
        const uint32_t p_at = tmem + C::scores_at(group, place), more = in_item >= 2;         // not the item's first of this group
        wait(C::P_FULL + 2 * group + place, n >> 2 & 1);
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < 4; ++k) tc_mma_f16_ta(tmem + C::kO + D * group, p_at + 8 * k, b + 2 * k, kIdesc, k > 0 ? 1u : more);
          tc_commit(bar(C::PV_DONE + 2 * group + place));
          if (last) tc_commit(bar(C::V_FREE + vb.at));
        }
        __syncwarp();
        if (last) vb.next();
        next(last);
      }
    }
    if (elect_one()) tc_commit(bar(C::DRAIN + (warp == C::kIssuerO)));
    __syncwarp();
  } else if (warp < C::kFirstSoftmax) {
    // ===================================================================== K, V and Q
    const bool is_v = warp >= C::kFirstV;
    // K: a thread a key
    const int tid = threadIdx.x & 127, key = tid, slot = key >> log_page, t = key & (P - 1);
    const uint32_t mine = (uint32_t)(slot * half_record + t * 16), my_scales = (uint32_t)(slot * half_record + P * L::kRow + t * L::kScales);
    // V: D = 128: a thread an index; D = 64: two threads, half of the tokens each
    const int e = D == 128 ? tid : tid & 63, tok0 = D == 128 ? 0 : tid & 64;
    constexpr int kTokens = D == 128 ? 128 : 64;                      // of a thread
    uint8_t* const scales = sgen + C::kOffVScale + (warp & 3) * 512;
    const uint32_t shift = 4 * (e & 1);
    // eight tokens whose scales of a block of this warp's indices a lane converts
    const int sc_tok = tok0 + 8 * (lane & (kTokens / 8 - 1)), sc_block = (e & ~31) / 16 + lane / (kTokens / 8);
    const uint32_t scale0 = (uint32_t)((sc_tok >> log_page) * half_record + P * L::kRow + sc_block * P + (sc_tok & (P - 1)));
    const uint8_t* const factors = scales + ((e >> 4) & 1) * (2 * kTokens);
    Turn<C::kStages> ring;
    Turn<C::kKB> kb;
    Turn<C::kVB> vb;
    int q_phase = 1, done = 0;
    if (is_v) ring.next();
#pragma unroll 1
    for (int item = 0;; ++item) {
      const Item* const it = next_item(item);
      if (none(it)) break;
      const int tiles = it->tiles, lo = it->lo, clean_end = p.ranges ? 0 : p.groups && it->g < 0 ? min(it->ctx, it->hi) : it->hi;
      int first = it->first;
      bring_q(it, item, q_phase);
      if (!is_v) {
#pragma unroll 1
        for (int i = 0; i < tiles; ++i) {
          wait(C::K_FREE + kb.at, kb.phase ^ 1);
          wait(C::RING_FULL + ring.at, ring.phase);
          const uint8_t* const stage = sgen + C::kOffStage + ring.at * C::kStage;
          const uint8_t* codes = stage + mine;
          uint8_t* const dst = sgen + C::kOffK + kb.at * C::kOp;
          uint2 sw = make_uint2(0u, 0u);
          if (L::kFp4 && D == 128) sw = *reinterpret_cast<const uint2*>(stage + my_scales);
          if (L::kFp4 && D == 64) sw.x = *reinterpret_cast<const uint32_t*>(stage + my_scales);
#pragma unroll 2
          for (int c = 0; c < D / 32; ++c) {
            uint32_t h[16];
            if (L::kFp4) {
              const uint4 raw = *reinterpret_cast<const uint4*>(codes);
              codes += P * 16;
              const uint32_t words[4] = {raw.x, raw.y, raw.z, raw.w}, both = cvt_f16x2_e4m3x2(sw.x & 0xFFFFu);
              sw.x = __funnelshift_r(sw.x, sw.y, 16);
              sw.y >>= 16;
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const uint32_t f = splat_half(both, x >> 1);
                cvt_f16x2_e2m1x8(words[x], h + 4 * x);
#pragma unroll
                for (int y = 0; y < 4; ++y) h[4 * x + y] = mul_half2(h[4 * x + y], f);
              }
            } else {
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const uint4 raw = *reinterpret_cast<const uint4*>(codes);
                codes += P * 16;
                const uint32_t words[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                for (int x = 0; x < 4; ++x) cvt_f16x2_e4m3x4(words[x], h + 8 * y + 2 * x);
              }
            }
            uint8_t* const panel = dst + (c >> 1) * 16384;
#pragma unroll
            for (int x = 0; x < 4; ++x)
              *reinterpret_cast<uint4*>(panel + chunk_at(key, 4 * (c & 1) + x)) = make_uint4(h[4 * x], h[4 * x + 1], h[4 * x + 2], h[4 * x + 3]);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(C::RING_FREE + ring.at));
            mbar_arrive(bar(C::K_FULL + kb.at));
          }
          ring.next(2);
          kb.next();
        }
      } else {
#pragma unroll 1
        for (int i = 0; i < tiles; ++i) {
          wait(C::V_FREE + vb.at, vb.phase ^ 1);
          wait(C::RING_FULL + ring.at, ring.phase);
          // is every byte one that some row sees, hence one that was written?
          const bool clean = L::kFp4 || (valid_ring[done % C::kRing] == all_pages && first >= lo && first + kTile <= clean_end);
          const uint8_t* const stage = sgen + C::kOffStage + ring.at * C::kStage;
          uint8_t* const dst = sgen + C::kOffV + vb.at * C::kOp;
          if (L::kFp4) {
            if (lane < kTokens / 4) {
              const uint2 sc = *reinterpret_cast<const uint2*>(stage + scale0);
              uint32_t f[4];
              cvt_f16x2_e4m3x4(sc.x, f);
              cvt_f16x2_e4m3x4(sc.y, f + 2);
              *reinterpret_cast<uint4*>(scales + lane * 16) = make_uint4(finite(f[0]), finite(f[1]), finite(f[2]), finite(f[3]));
            }
            __syncwarp();
          }
#pragma unroll 2
          for (int j = 0; j < kTokens; j += 16) {                       // sixteen tokens
            const int tok = tok0 + j;
            const uint4 raw = *reinterpret_cast<const uint4*>(stage + (tok >> log_page) * half_record + ((tok & (P - 1)) >> 4) * (16 * L::kRow) + (L::kFp4 ? e >> 1 : e) * 16);
            const uint32_t cw[4] = {raw.x, raw.y, raw.z, raw.w};
            uint32_t h[8];
            if (L::kFp4) {
#pragma unroll
              for (int x = 0; x < 2; ++x) {                             // eight tokens: i and i + 4 in a byte
                const uint4 f = *reinterpret_cast<const uint4*>(factors + 2 * j + 16 * x);
                cvt_f16x2_e2m1x8((cw[2 * x] >> shift & 0x0F0F0F0Fu) | (cw[2 * x + 1] << (4 - shift) & 0xF0F0F0F0u), h + 4 * x);
                h[4 * x] = mul_half2(h[4 * x], f.x);
                h[4 * x + 1] = mul_half2(h[4 * x + 1], f.y);
                h[4 * x + 2] = mul_half2(h[4 * x + 2], f.z);
                h[4 * x + 3] = mul_half2(h[4 * x + 3], f.w);
              }
            } else {
#pragma unroll
              for (int x = 0; x < 4; ++x) cvt_f16x2_e4m3x4(cw[x], h + 2 * x);
              if (rare(!clean)) {
#pragma unroll
                for (int x = 0; x < 8; ++x) h[x] = finite(h[x]);
              }
            }
            uint8_t* const panel = dst + (tok >> 6) * (D * 128);
            *reinterpret_cast<uint4*>(panel + chunk_at(e, (tok & 63) >> 3)) = make_uint4(h[0], h[1], h[2], h[3]);
            *reinterpret_cast<uint4*>(panel + chunk_at(e, ((tok & 63) >> 3) + 1)) = make_uint4(h[4], h[5], h[6], h[7]);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(C::RING_FREE + ring.at));
            mbar_arrive(bar(C::V_FULL + vb.at));
          }
          ring.next(2);
          vb.next();
          first -= kTile;
          ++done;
        }
      }
    }
  } else {
    // ===================================================================== softmax
    const int group = (warp - C::kFirstSoftmax) >> 2, quarter = warp & 3, in_tile = quarter * 32 + lane;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t o_at = tmem + lanes + C::kO + D * group;
    float2* const ml = reinterpret_cast<float2*>(sgen + C::kOffML);
    const float cap_out = p.cap * 1.4426950408889634f, cap_inverse = p.cap > 0.f ? __fdiv_rn(1.f, cap_out) : 0.f;
    int meet_phase = 0, done = 0;                                     // done: tiles of this CTA's run
    uint32_t n = 0;                                                   // jobs of this group
    // the group's last product on O.  (A barrier for each place: scores of a job say that the product before the last is done, so the last one is the
    // only one that this wait can be in doubt about.)
    auto o_done = [&] { wait(C::PV_DONE + 2 * group + (n - 1 & 1), (n - 1) >> 1 & 1); };
    auto meet = [&] {                                                 // both groups (a barrier whose wait ends, unlike that of the hardware's named ones)
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::MEET));
      wait(C::MEET, meet_phase);
      meet_phase ^= 1;
    };
#pragma unroll 1
    for (int item = 0;; ++item) {
      const Item* const it = next_item(item);
      if (none(it)) break;
      const bool two = it->two;
      const int copies = it->copies, tiles = it->tiles;
      // this thread's row of the item; of a job's four times sixteen keys, those of its copy
      const int row_in = two ? group * 128 + in_tile : in_tile & (128 / copies - 1);
      const int c_first = two ? 0 : in_tile / (128 / copies) * (4 / copies), c_end = c_first + 4 / copies;
      bool live = row_in < it->here;
      int b = 0, t = 0, hl = 0, lo = 0, hi = 0;
      float slope = 0.f;
      int pos = 0;
      unsigned long long mask = 0;
      if (live) {
        row_token(p, *it, row_in, &b, &t, &hl);
        const int ctx = it->ctx;
        if (ANY) {
          slope = p.slopes ? load(p.slopes + it->kvh * p.group + hl) * 1.4426950408889634f : 0.f;
          pos = (int)((unsigned)(it->g >= 0 ? it->hi + context_of(p, b) : ctx) + (unsigned)t);
        }
        if (it->g >= 0) {
          live = t < tokens_of(p, b);
          hi = it->hi;
        } else if (p.groups) {
          if (p.mask) {
            mask = load(p.mask + (size_t)b * p.T + t);
            if (p.T < 64) mask &= (1ull << p.T) - 1;
            hi = min(ctx, it->hi);
          } else {
            hi = min(ctx + t + 1, it->hi);
          }
        } else {
          lo = p.first ? max(0, load(p.first + (size_t)b * p.T + t)) : 0;
          hi = max(0, min(p.last ? load(p.last + (size_t)b * p.T + t) : ctx + t + 1, it->hi));
        }
      }
      const bool warp_live = __any_sync(0xffffffffu, live);
      if (!live) hi = INT_MAX;                                        // (a row of zeros, or one that is not written: never the reason to look at masks)
      const int mask_at = p.mask && it->g < 0 ? it->ctx : INT_MIN;    // where the drafted tokens begin
      // keys that every row of the warp sees
      const int plain_lo = __reduce_max_sync(0xffffffffu, lo), plain_hi = __reduce_min_sync(0xffffffffu, hi);
      bool have = false, settled = false;                             // a job of the item so far; a reference for every row
      float m = -INFINITY, l0 = 0.f, l1 = 0.f, con = 0.f;
      int first = it->first + (two ? 64 : 64 * group);                // first key of the job
      const int jobs = two ? 2 * tiles : tiles;
#pragma unroll 1
      for (int i = 0; i < jobs; ++i) {
        const uint32_t place = n & 1;
        wait(C::S_FULL + (RT == 1 ? 0 : 2 * group) + place, n >> 1 & 1);
        tc_fence_after();
        if (warp_live) {
          const uint32_t s_job = tmem + lanes + C::scores_at(group, place), held = valid_ring[done % C::kRing];
          if (rare(!have)) con = live ? reinterpret_cast<const float*>(sgen + C::kOffC)[(item & (C::kRingC - 1)) * ROWS + row_in] : 0.f;
          // Does every row see every key (with a bias: of those before it)?  Otherwise scores are changed, masked and put back before anything else; so are capped
          // scores beyond the polynomial's range.
          // (Scaled scores only: two votes fewer a job are 8 % of the time.  The others are as fast without, and have no registers for the bounds.)
          bool change = (SCORES == kScaled ? held != all_pages || first < plain_lo || first + 64 > plain_hi
                                           : !__all_sync(0xffffffffu, held == all_pages && lo <= first && hi >= first + 64 && (!ANY || pos >= first + 63))) ||
                        (ANY && p.cap > 0.f);
          // (by no row of the warp any of them: documents, the tile on the diagonal)
          const bool unseen = rare(change) && mask_at < 0 && __all_sync(0xffffffffu, hi <= first || lo >= first + 64);
          float lag = kLag;
          // The reference moves to the largest score seen so far.
          auto refer = [&] {
            float top = -INFINITY;
            const int in_tile0 = two ? 64 - 64 * (i & 1) : 64 * group;
            const float c = CAP || (ANY && p.cap > 0.f) ? cap_constant(con, cap_inverse) : con;
#pragma unroll 1
            for (int k = c_first; k < c_end; ++k) {
              uint32_t a[16];
              tmem_ld_32x32b_x16(s_job + 16 * k, a);
              const int at = first + 16 * k;
              const float far = (float)(pos - at);
              uint32_t seen = 0xFFFFu;
              if (change) {
                seen = bits_between(lo - at, hi - at);
                if (mask_at >= 0) {
                  const int o = mask_at - at;
                  seen |= o >= 32 || o <= -64 ? 0u : (uint32_t)(o >= 0 ? mask << o : mask >> -o);
                }
                seen = held >> ((in_tile0 + 16 * k) >> log_page) & 1 ? seen : 0u;
              }
              tmem_wait_ld();
              if (ANY || change) {
                float y[16];
#pragma unroll
                for (int x = 0; x < 16; ++x) y[x] = __uint_as_float(a[x]) * c;
                if (CAP || (ANY && p.cap > 0.f)) {
                  float u[16];
#pragma unroll
                  for (int x = 0; x < 16; ++x) u[x] = y[x];
                  cap_scores(y, u, cap_out);
                }
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                  if (ANY) y[x] = fmaf(-slope, fabsf(far - (float)x), y[x]);
                  a[x] = seen & 1u << x ? __float_as_uint(y[x]) : 0xFF800000u;
                }
                if (change) tmem_st_32x32b_x16(s_job + 16 * k, a);
              }
              float t2 = -INFINITY;
#pragma unroll
              for (int x = 0; x < 16; x += 4) {
                top = max3(top, __uint_as_float(a[x]), __uint_as_float(a[x + 1]));
                t2 = max3(t2, __uint_as_float(a[x + 2]), __uint_as_float(a[x + 3]));
              }
              top = fmaxf(top, t2);
            }
            if (!ANY && !change) {
              top *= c;
              if (CAP) {
                float x[2];
                const float u[2] = {top, 0.f};
                cap_scores(x, u, cap_out);
                top = x[0];
              }
            }
            if (change) tmem_wait_st();
            if (m == -INFINITY) m = top;                              // (so far nothing: its sum and O are 0)
            if (__any_sync(0xffffffffu, top > m + lag)) {
              // (of all rows of the warp: if only those moved that need it, some row would in many more jobs: prompt 371 -> 439 us)
              const float old = m;
              m = fmaxf(m, top);
              const float f = m == old ? 1.f : exp2_approx(old - m);
              l0 *= f;
              l1 *= f;
              if (have) {
                o_done();
                tc_fence_after();
#pragma unroll 1
                for (int k = 0; k < D; k += 16) {
                  uint32_t o[16];
                  tmem_ld_32x32b_x16(o_at + k, o);
                  tmem_wait_ld();
#pragma unroll
                  for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
                  tmem_st_32x32b_x16(o_at + k, o);
                }
                tmem_wait_st();
              }
            }
            settled = !__any_sync(0xffffffffu, m == -INFINITY);
          };
          // Probabilities of sixteen keys, eight words, and their sum.  HOW: scores times a constant; capped; with a
          // bias that falls along the keys.
          float wide, s0, s1, shift, c2;
          auto sixteen = [&](auto how, const uint32_t* raw, int k, uint32_t* h) {
            constexpr int HOW = decltype(how)::value;
#pragma unroll
            for (int y = 0; y < 16; y += 8) {
              float z[8];
#pragma unroll
              for (int x = 0; x < 8; x += 2) {
                const float r0 = __uint_as_float(raw[y + x]), r1 = __uint_as_float(raw[y + x + 1]);
                if (HOW == kCapped) {
                  // (ten instructions for two scores, where an exponential and a reciprocal each are 32 clocks of the special-function unit for a warp, as much
                  // again as exp2 twice over)
                  float u0, u1, w0, w1, t0, t1;
                  mul_pair(u0, u1, r0, r1, c2, c2);
                  mul_pair(w0, w1, u0, u1, u0, u1);
                  wide = max3(wide, w0, w1);
                  tanh_pair(t0, t1, w0, w1);
                  mul_pair(u0, u1, u0, u1, cap_out, cap_out);
                  fma_pair(z[x], z[x + 1], t0, t1, u0, u1, shift, shift);
                } else if (HOW == kBiased) {
                  float b0, b1;
                  fma_pair(b0, b1, slope, slope, (float)(16 * k + y + x), (float)(16 * k + y + x + 1), shift, shift);
                  fma_pair(z[x], z[x + 1], r0, r1, c2, c2, b0, b1);
                } else {
                  fma_pair(z[x], z[x + 1], r0, r1, c2, c2, shift, shift);
                }
                z[x] = exp2_approx(z[x]);
                z[x + 1] = exp2_approx(z[x + 1]);
                add_pair(s0, s1, z[x], z[x + 1]);
              }
              if (L::kFp4) {                                          // the order that V's tokens stand in: 0 4 1 5 2 6 3 7
#pragma unroll
                for (int x = 0; x < 4; ++x) h[y / 2 + x] = pack_pair<__half>(z[x], z[x + 4]);
              } else {
#pragma unroll
                for (int x = 0; x < 4; ++x) h[y / 2 + x] = pack_pair<__half>(z[2 * x], z[2 * x + 1]);
              }
            }
          };
          // Scores rarely exceed their reference by much: the largest is looked for first where there is none yet or scores have to be changed, and in all other
          // jobs only when their sum has turned out to be more than f16 is sure to hold of one of them; then the job is done again.
          bool sure = change || (SCORES == kScaled ? !settled : __any_sync(0xffffffffu, m == -INFINITY));
          s0 = s1 = 0.f;
          auto attempt = [&](auto pass) {
#pragma unroll 1
            while (true) {
              if (rare(sure)) refer();
              shift = m == -INFINITY ? 0.f : kShift - m;
              s0 = s1 = wide = 0.f;
              if (SCORES == kScaled || rare(change)) {
                c2 = change ? 1.f : con;
                pass(std::integral_constant<int, kScaled>());
              } else {
                c2 = CAP ? cap_constant(con, cap_inverse) : con;
                if (ANY) shift -= slope * (float)(pos - first);
                pass(std::integral_constant<int, SCORES>());
                if (CAP && rare(__any_sync(0xffffffffu, wide > kTanhReach))) {
                  change = sure = true;
                  continue;
                }
              }
              if (sure || !rare(__any_sync(0xffffffffu, s0 + s1 > kMostSum))) break;
              sure = true;
              lag = 1.f;                                              // (64 keys of that sum: one is 2^9 or more, two octaves above the reference's 2^7)
            }
          };
          if (unseen) {
            uint32_t h[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) h[x] = 0u;
            tmem_st_32x32b_x16(s_job, h);
            tmem_st_32x32b_x16(s_job + 16, h);
          } else if (ROWS > 128 || copies == 1) {
            uint32_t h[32];
            attempt([&](auto how) {
              uint32_t a[16], c[16];
              tmem_ld_32x32b_x16(s_job, a);
              tmem_wait_ld();
              tmem_ld_32x32b_x16(s_job + 16, c);
              sixteen(how, a, 0, h);
              tmem_wait_ld();
              tmem_ld_32x32b_x16(s_job + 32, a);
              sixteen(how, c, 1, h + 8);
              tmem_wait_ld();
              tmem_ld_32x32b_x16(s_job + 48, c);
              sixteen(how, a, 2, h + 16);
              tmem_wait_ld();
              sixteen(how, c, 3, h + 24);
            });
            tmem_st_32x32b_x16(s_job, h);                             // (over scores that have been read)
            tmem_st_32x32b_x16(s_job + 16, h + 16);
          } else {
            // (two pieces at most: what the one before the last has to store waits)
            uint32_t h[16];
            attempt([&](auto how) {
              uint32_t a[16];
              tmem_ld_32x32b_x16(s_job + 16 * c_first, a);
              tmem_wait_ld();
              sixteen(how, a, c_first, h);
              if (copies == 2) {
                tmem_ld_32x32b_x16(s_job + 16 * c_first + 16, a);
                tmem_wait_ld();
                sixteen(how, a, c_first + 1, h + 8);
              }
            });
            tmem_st_32x32b_x8(s_job + 8 * c_first, h);
            if (copies == 2) tmem_st_32x32b_x8(s_job + 8 * c_first + 8, h + 8);
#pragma unroll
            for (int x = 0; x < 8; ++x) h[x] = 0u;
#pragma unroll 1
            for (int k = 0; k < 4; ++k)                               // the other copies' keys
              if (k < c_first || k >= c_end) tmem_st_32x32b_x8(s_job + 8 * k, h);
          }
          l0 += s0;
          l1 += s1;
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::P_FULL + 2 * group + place));
        have = true;
        ++n;
        const bool tile_done = !two || (i & 1);
        first -= two ? 64 : kTile;
        done += tile_done;
      }
      // ---- end of the item, or of this CTA's part of it
      const int kvh = it->kvh;
      const bool whole = it->whole;
      const float v_G = load(p.cache.v_G + kvh);
      o_done();
      float f[2] = {1.f, 1.f}, top = m, sum = l0 + l1;
      if (!two) {                                                     // both groups, and every copy, have had tiles of these rows
        ml[group * 128 + in_tile] = make_float2(m, sum);
        meet();
        // (in one order, so that all have the same bits)
        float2 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          x[k] = k < 2 * copies ? ml[(k & 1) * 128 + row_in + (k >> 1) * (128 / copies)] : make_float2(-INFINITY, 0.f);
          top = fmaxf(top, x[k].x);
        }
        auto weight = [&](float2 y) { return y.x == -INFINITY && y.y == 0.f ? 0.f : y.x == top ? 1.f : exp2_approx(y.x - top); };
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float y = weight(x[k]);
          sum += y == 0.f ? 0.f : y * x[k].y;
        }
        f[0] = weight(ml[in_tile]);
        f[1] = weight(ml[128 + in_tile]);
      } else if (m == -INFINITY && sum == 0.f) {
        f[group] = 0.f;
      }
      tc_fence_after();
      const bool tells = two || (group == 0 && in_tile < 128 / copies);
      const long long at = ((long long)b * p.H + kvh * p.group + hl) * p.T + t;          // of the row among the outputs
      const bool out = whole && !p.groups;
      char* dst = nullptr;                                            // of the row's elements
      if (out) {
        const float inv = sum == 0.f ? 0.f : __fdiv_rn(1.f, sum * v_G);                  // nothing seen: 0, not 0 / 0
        f[0] *= inv;
        f[1] *= inv;
        if (live && p.lse && tells) p.lse[at] = sum == 0.f ? -INFINITY : (top - kShift + log2f(sum)) * 0.6931471805599453f;
        dst = static_cast<char*>(p.out) + at * (2 * D);
      } else if (live) {
        const long long place = whole ? (it->g < 0 ? (long long)p.B * p.H * p.T : 0) + at : (long long)it->slot * ROWS + row_in;
        dst = reinterpret_cast<char*>((whole ? p.whole : p.part) + place * D);
        if (tells) (whole ? p.whole_ml : p.part_ml)[place] = make_float2(top, sum);
      }
      if (p.groups && it->begins && group == 0 && in_tile == 0) p.split[it->split] = whole ? make_int2(-1, -1) : make_int2(blockIdx.x, it->last_cta);
      __syncwarp();
      // (Every group has had a job of the item, so what stands in O is a sum: 0 where nothing was seen, as P was 0 and V is finite.)
      auto write = [&](int e, const float* o) {                       // sixteen elements of a row, 32 bytes a store
        if (out) {
          uint32_t h[8];
          if (p.half) {
#pragma unroll
            for (int x = 0; x < 8; ++x) h[x] = pack_pair<__half>(o[2 * x], o[2 * x + 1]);
          } else {
#pragma unroll
            for (int x = 0; x < 8; ++x) h[x] = pack_pair<__nv_bfloat16>(o[2 * x], o[2 * x + 1]);
          }
          if (p.out_wide) {
            store_32(dst + 2 * e, h);
          } else {
            reinterpret_cast<uint4*>(dst + 2 * e)[0] = make_uint4(h[0], h[1], h[2], h[3]);
            reinterpret_cast<uint4*>(dst + 2 * e)[1] = make_uint4(h[4], h[5], h[6], h[7]);
          }
        } else {
          uint32_t h[16];
#pragma unroll
          for (int x = 0; x < 16; ++x) h[x] = __float_as_uint(o[x]);
          store_32(dst + 4 * e, h);
          store_32(dst + 4 * e + 32, h + 8);
        }
      };
      if (ROWS <= 128 && copies > 1) {
        // The copies' O meet in shared memory, as many elements at a time as there is room for of the rows that there are; then a thread takes four
        // elements of a row and adds them up.
        float* const join = reinterpret_cast<float*>(sgen + C::kOffJoin);
        const int here = it->here, most = here <= 4 ? 128 : here <= 8 ? 64 : here <= 16 ? 32 : 16, cols = min(D, most), stride = here > 32 ? 32 : here;
        // of this warp: [rows of the warp][cols]; row of the warp
        float* const put = join + ((warp - C::kFirstSoftmax) * stride + lane) * cols;
        const float g = f[group];
        char* const o_row = reinterpret_cast<char*>(whole ? (p.groups ? (void*)p.whole : p.out) : (void*)p.part);
        const long long whole0 = p.groups && it->g < 0 ? (long long)p.B * p.H * p.T : 0;
#pragma unroll 1
        for (int e0 = 0; e0 < D; e0 += cols) {
          if (warp_live) {
#pragma unroll 1
            for (int e = 0; e < cols; e += 16) {
              uint32_t v[16];
              tmem_ld_32x32b_x16(o_at + e0 + e, v);
              tmem_wait_ld();
              if (live) {
#pragma unroll
                for (int x = 0; x < 16; x += 4)
                  *reinterpret_cast<float4*>(put + ((e + x) ^ (lane & 3) * 4)) =
                      make_float4(__uint_as_float(v[x]) * g, __uint_as_float(v[x + 1]) * g, __uint_as_float(v[x + 2]) * g, __uint_as_float(v[x + 3]) * g);
              }
              __syncwarp();
            }
          }
          tc_fence_before();
          meet();
          const int quads = cols / 4;
#pragma unroll 1
          for (int j = threadIdx.x - 32 * C::kFirstSoftmax; j < here * quads; j += 256) {
            const int r = j / quads, c = (j - r * quads) * 4;
            int rb, rt, rh;
            row_token(p, *it, r, &rb, &rt, &rh);
            if (it->g >= 0 && rt >= tokens_of(p, rb)) continue;
            float o[4] = {0.f, 0.f, 0.f, 0.f};
            const float* const from = join + ((r >> 5) * stride + (r & 31)) * cols + (c ^ (r & 3) * 4);
#pragma unroll
            for (int k = 0; k < 8; ++k) {                             // (warp of the copy: of the group k & 1, as many warps on as a copy has)
              if (k >= 2 * copies) break;
              const float4 y = *reinterpret_cast<const float4*>(from + ((k & 1) * 4 + (k >> 1) * (4 / copies)) * stride * cols);
              o[0] += y.x; o[1] += y.y; o[2] += y.z; o[3] += y.w;
            }
            const long long row = whole ? whole0 + ((long long)rb * p.H + kvh * p.group + rh) * p.T + rt : (long long)it->slot * ROWS + r;
            if (out)
              *reinterpret_cast<uint2*>(o_row + (row * D + e0 + c) * 2) = p.half ? make_uint2(pack_pair<__half>(o[0], o[1]), pack_pair<__half>(o[2], o[3]))
                                                                                 : make_uint2(pack_pair<__nv_bfloat16>(o[0], o[1]), pack_pair<__nv_bfloat16>(o[2], o[3]));
            else
              *reinterpret_cast<float4*>(o_row + (row * D + e0 + c) * 4) = make_float4(o[0], o[1], o[2], o[3]);
          }
          meet();
        }
      } else {
        if (warp_live) {
          const int d0 = two ? 0 : group * (D / 2), d1 = two ? D : d0 + D / 2;
#pragma unroll 1
          for (int e = d0; e < d1; e += 16) {
            uint32_t v[16];
            float o[16];
            if (two) {
              tmem_ld_32x32b_x16(o_at + e, v);
              tmem_wait_ld();
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] = __uint_as_float(v[x]) * f[group];
            } else {
              uint32_t v2[16];
              tmem_ld_32x32b_x16(tmem + lanes + C::kO + e, v);
              tmem_ld_32x32b_x16(tmem + lanes + C::kO + D + e, v2);
              tmem_wait_ld();
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] = __uint_as_float(v[x]) * f[0] + __uint_as_float(v2[x]) * f[1];
            }
            if (live) write(e, o);
            __syncwarp();
          }
        }
        tc_fence_before();
        if (!two) meet();                                   // the next item's products may overwrite either O
      }
      tc_fence_before();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_word && threadIdx.x == 0 && p.status) *p.status = FP4ATTN_ERR_TIMEOUT;
  if (warp == C::kIssuerS) {
    if (*abort_word && lane == 0)                                   // given up: the products in flight end before tensor memory does
      for (int k = 0; k < 2; ++k)
        for (int spin = 0; spin < (1 << 14) && !mbar_try_wait(bar(C::DRAIN + k), 0); ++spin) {}
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ---- joining: a warp a row, in the order of the keys
template <int D>
struct Sum {
  static constexpr int E = D / 32;
  float m = -INFINITY, l = 0.f, o[E] = {};
  __device__ __forceinline__ void one(const float* src, float2 ml, int lane) {
    m = ml.x;
    l = ml.y;
    fetch(src, lane, o);
  }
  static __device__ __forceinline__ void fetch(const float* src, int lane, float* y) {
    if constexpr (E == 4) *reinterpret_cast<float4*>(y) = *reinterpret_cast<const float4*>(src + lane * E);
    else *reinterpret_cast<float2*>(y) = *reinterpret_cast<const float2*>(src + lane * E);
  }
  // row r of the parts that an item left in CTAs first .. last
  __device__ __forceinline__ void parts(const float* part_of, const float2* ml_of, int rows, int first, int last, int r, int lane) {
    const int n = last - first + 1;
    auto at = [&](int i) { return (size_t)(i ? 2 * (first + i) : 2 * first + 1) * rows + r; };
    for (int i = lane; i < n; i += 32) m = fmaxf(m, ml_of[at(i)].x);
    m = warp_max(m);
    for (int i0 = 0; i0 < n; i0 += 32) {
      const int i = i0 + lane;
      const float2 ml = i < n ? ml_of[at(i)] : make_float2(-INFINITY, 0.f);
      const float mine = m == -INFINITY || i >= n ? 0.f : exp2_approx(ml.x - m);
      const float weighted = ml.x == -INFINITY ? ml.y : mine * ml.y;
      constexpr int kAtOnce = 8;                                    // loads on their way together
      for (int k0 = 0; k0 < min(32, n - i0); k0 += kAtOnce) {
        float part[kAtOnce][E];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
#pragma unroll
          for (int x = 0; x < E; ++x) part[k][x] = 0.f;
          if (i0 + k0 + k < n) fetch(part_of + at(i0 + k0 + k) * D, lane, part[k]);
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {                         // (behind the last part: weights and parts of 0)
          const float f = __shfl_sync(0xffffffffu, mine, k0 + k);
          l += __shfl_sync(0xffffffffu, weighted, k0 + k);
#pragma unroll
          for (int x = 0; x < E; ++x) o[x] = fmaf(f, part[k][x], o[x]);
        }
      }
    }
  }
  __device__ __forceinline__ void add(const Sum& s) {
    const float top = fmaxf(m, s.m), f = top == -INFINITY || m == top ? 1.f : exp2_approx(m - top), g = top == -INFINITY || s.m == top ? 1.f : exp2_approx(s.m - top);
    m = top;
    l = l * f + s.l * g;
#pragma unroll
    for (int x = 0; x < E; ++x) o[x] = o[x] * f + s.o[x] * g;
  }
  __device__ __forceinline__ void give(const PagedParams& p, size_t at, int kvh, int lane) const {
    const float f = l == 0.f ? 0.f : __fdiv_rn(1.f, l * load(p.cache.v_G + kvh));
#pragma unroll
    for (int x = 0; x < E; x += 2) {
      const uint32_t two = p.half ? pack_pair<__half>(o[x] * f, o[x + 1] * f) : pack_pair<__nv_bfloat16>(o[x] * f, o[x + 1] * f);
      *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + at * D + lane * E + x) = two;
    }
    if (lane == 0 && p.lse) p.lse[at] = l == 0.f ? -INFINITY : (m - kShift + log2f(l)) * 0.6931471805599453f;
  }
};
constexpr int kJoinThreads = 256;
// the item that began in CTA blockIdx.x, if it went on in others
template <int D, int ROWS>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const PagedParams p) {
  wait_prior_grids();
  const int4 item = p.begun[blockIdx.x];
  const int first = blockIdx.x, last = item.z, lane = threadIdx.x & 31;
  if (!item.w || last <= first || last >= (int)gridDim.x) return;   // (or a kernel that gave up)
  Desc d;
  describe<ROWS>(p, item.x, d);
  const int kvh = item.y, here = min(ROWS, d.rows - d.row0);
  for (int r = blockIdx.y * (kJoinThreads / 32) + (threadIdx.x >> 5); r < here; r += gridDim.y * (kJoinThreads / 32)) {
    const int t = (d.row0 + r) / p.group, hl = d.row0 + r - t * p.group;
    Sum<D> s;
    s.parts(p.part, p.part_ml, ROWS, first, last, r, lane);
    s.give(p, ((size_t)d.b * p.H + (size_t)kvh * p.group + hl) * p.T + t, kvh, lane);
  }
}
// every row of a batch with shared prefixes: its prefix's part and its own
template <int D, int ROWS>
__global__ void __launch_bounds__(kJoinThreads) shared_join_kernel(const PagedParams p) {
  wait_prior_grids();
  const long long at = (long long)blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5), all = (long long)p.B * p.H * p.T;
  const int lane = threadIdx.x & 31;
  if (at >= all) return;
  const int t = (int)(at % p.T), h = (int)(at / p.T % p.H), b = (int)(at / p.T / p.H), kvh = h / p.group, hl = h - kvh * p.group;
  if (t >= tokens_of(p, b)) return;
  Sum<D> sum;
  auto take = [&](int x, int row) {
    Desc d;
    describe<ROWS>(p, x, d);
    if (!d.nt) return;
    const int2 ctas = p.split[split_place<ROWS>(p, d, kvh * d.rts + row / ROWS)];
    Sum<D> s;
    const long long w = d.g < 0 ? all + at : at;
    if (ctas.x < 0) s.one(p.whole + w * D, p.whole_ml[w], lane);
    else if (ctas.y >= ctas.x && ctas.y < kMostCtas) s.parts(p.part, p.part_ml, ROWS, ctas.x, ctas.y, row % ROWS, lane);
    sum.add(s);
  };
  // the last group that begins here or before
  int g = 0, end = p.groups;
  while (end - g > 1) {
    const int mid = (g + end) / 2;
    if (load(p.group_start + mid) <= b) g = mid;
    else end = mid;
  }
  const int b0 = load(p.group_start + g);
  if (b >= b0 && b < load(p.group_start + g + 1)) take(g, ((b - max(0, b0)) * p.T + t) * p.group + hl);
  take(p.groups + b, t * p.group + hl);
  sum.give(p, (size_t)at, kvh, lane);
}

// keys that each tile of rows sees, where first or last say so: a warp a tile
template <int ROWS>
__global__ void __launch_bounds__(128) range_kernel(const PagedParams p, int2* ranges) {
  launch_dependents();
  wait_prior_grids();
  const int x = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (x >= p.B * p.row_tiles) return;
  const int b = x / p.row_tiles, row0 = (x - b * p.row_tiles) * ROWS, n = tokens_of(p, b), ctx = context_of(p, b);
  int lo = INT_MAX, hi = 0;
  for (int t = row0 / p.group + lane; t < n && t <= (row0 + ROWS - 1) / p.group; t += 32) {
    const int from = p.first ? max(0, load(p.first + (size_t)b * p.T + t)) : 0, until = min(p.last ? load(p.last + (size_t)b * p.T + t) : ctx + t + 1, ctx + n);
    if (from < until) {
      lo = min(lo, from);
      hi = max(hi, until);
    }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) ranges[x] = hi ? make_int2(lo, hi) : make_int2(0, 0);
}

// ---- workspace
struct Plan {
  int rt, row_tiles;                       // 128-row halves of an item; items of a sequence's rows
  size_t ml, begun, ranges, split, whole, whole_ml, total;
};
size_t align32(size_t x) { return (x + 31) & ~(size_t)31; }
Plan plan(int B, int H, int kv_heads, int T, int d, int groups) {
  Plan t;
  const long long rows = (long long)(H / kv_heads) * T;
  // (a sequence by itself has few rows, and instances for those keep copies of them: prefixes go along.  48 sequences of 4 rows behind
  // a prefix of 16000 tokens, 192 rows: 80 us with 256 rows an item, 71 with 128)
  t.rt = !groups && rows > 128 ? 2 : 1;
  const long long R = 128 * t.rt, all = (long long)B * H * T;
  t.row_tiles = (int)((rows + R - 1) / R);
  const size_t slots = 2 * (size_t)kMostCtas * R;
  t.ml = slots * d * 4;
  t.begun = t.ml + slots * 8;
  t.ranges = t.begun + kMostCtas * 16;
  t.split = t.ranges + (groups ? 0 : align32((size_t)B * t.row_tiles * 8));
  t.whole = t.split + (groups ? align32((size_t)(B * rows / R + groups + 1 + (long long)B * t.row_tiles) * kv_heads * 8) : 0);
  t.whole_ml = t.whole + (groups ? (size_t)(2 * all) * d * 4 : 0);
  t.total = t.whole_ml + (groups ? align32((size_t)(2 * all) * 8) : 0);
  return t;
}

template <int FMT, int D, int RT, int SCORES>
int launch_scores(const PagedParams& p, cudaStream_t st) {
  using C = PagedCfg<FMT, D, RT>;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return FP4ATTN_ERR_CUDA;
  static std::atomic<bool> attr_set[kMaxDevices];
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(paged_kernel<FMT, D, RT, SCORES>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) != cudaSuccess) return FP4ATTN_ERR_CUDA;
    attr_set[dev].store(true, std::memory_order_release);
  }
  const int sms = device_sms();
  if (!sms) return FP4ATTN_ERR_CUDA;
  const unsigned grid = (unsigned)std::min(sms, kMostCtas);
  cudaError_t e = cudaSuccess;
  if (p.ranges)
    e = launch_overlapped(range_kernel<C::kRows>, dim3((unsigned)((p.B * p.row_tiles + 3) / 4)), 128u, 0, st, p, const_cast<int2*>(p.ranges));
  if (e == cudaSuccess) e = launch_overlapped(paged_kernel<FMT, D, RT, SCORES>, dim3(grid), C::kThreads, C::kSmem, st, p);
  const long long rows = (long long)p.B * p.H * p.T;
  if (e == cudaSuccess)
    e = p.groups ? launch_overlapped(shared_join_kernel<D, C::kRows>, dim3((unsigned)((rows + kJoinThreads / 32 - 1) / (kJoinThreads / 32))), kJoinThreads, 0, st, p)
                 : launch_overlapped(join_kernel<D, C::kRows>, dim3(grid, (unsigned)(std::min(p.group * p.T, C::kRows) + 7) / 8), kJoinThreads, 0, st, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
}
template <int FMT, int D, int RT>
int launch_rows(const PagedParams& p, cudaStream_t st) {
  if (p.slopes) return launch_scores<FMT, D, RT, kBiased>(p, st);
  return p.cap > 0.f ? launch_scores<FMT, D, RT, kCapped>(p, st) : launch_scores<FMT, D, RT, kScaled>(p, st);
}
int launch(PagedParams& p, const Plan& t, void* workspace, int fmt, int d, cudaStream_t st) {
  char* const ws = (char*)workspace;
  p.row_tiles = t.row_tiles;
  auto reciprocal = [](int n) { return ((1ull << 36) + n - 1) / n; };
  p.by_group = reciprocal(p.group);
  p.by_tokens = reciprocal(p.T);
  p.out_wide = ((uintptr_t)p.out & 31) == 0;
  p.part = (float*)ws;
  p.part_ml = (float2*)(ws + t.ml);
  if (p.groups) {
    p.split = (int2*)(ws + t.split);
    p.whole = (float*)(ws + t.whole);
    p.whole_ml = (float2*)(ws + t.whole_ml);
  } else {
    p.begun = (int4*)(ws + t.begun);
    if (p.first || p.last) p.ranges = (const int2*)(ws + t.ranges);
  }
  auto rows = [&](auto fmt_c, auto d_c) {
    return t.rt == 2 ? launch_rows<fmt_c.value, d_c.value, 2>(p, st) : launch_rows<fmt_c.value, d_c.value, 1>(p, st);
  };
  using std::integral_constant;
  if (fmt == FP4ATTN_FMT_NVFP4)
    return d == 64 ? rows(integral_constant<int, FP4ATTN_FMT_NVFP4>(), integral_constant<int, 64>())
                   : rows(integral_constant<int, FP4ATTN_FMT_NVFP4>(), integral_constant<int, 128>());
  return d == 64 ? rows(integral_constant<int, FP4ATTN_FMT_E4M3>(), integral_constant<int, 64>())
                 : rows(integral_constant<int, FP4ATTN_FMT_E4M3>(), integral_constant<int, 128>());
}

// what the two calls have in common
int check(const fp4attn_view* q, int type, const fp4attn_cache* cache, int B, int H, int T, const int* block_table, int max_pages, const int* context,
          const int* count, float softmax_scale, float soft_cap, const float* slopes, void* O, float* LSE, int* device_status, PagedParams* p) {
  const int rc = check_cache(cache, B, block_table, max_pages, context, count, &p->cache);
  if (rc != FP4ATTN_OK) return rc;
  if (!q || !q->data || !O || H <= 0 || T <= 0 || !(softmax_scale >= 0.f) || isinf(softmax_scale) || !(soft_cap == 0.f || (soft_cap >= 0x1p-60f && soft_cap <= 0x1p60f)))
    return FP4ATTN_ERR_INVALID_ARG;
  if (type != FP4ATTN_TYPE_BF16 && type != FP4ATTN_TYPE_FP16) return FP4ATTN_ERR_INVALID_ARG;
  if (H % cache->kv_heads != 0) return FP4ATTN_ERR_INVALID_ARG;
  if ((long long)B * H * T >= (1ll << 31) || T >= (1 << 30) || H / cache->kv_heads > kMostGroup) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;
  if (((uintptr_t)q->data & 1) || ((uintptr_t)O & 15) || ((uintptr_t)LSE | (uintptr_t)device_status | (uintptr_t)slopes) & 3) return FP4ATTN_ERR_ALIGNMENT;
  p->q = q->data; p->q_sb = q->stride_b; p->q_sh = q->stride_h; p->q_sn = q->stride_n;
  p->q_vector = view_vectors(*q, 2);
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

namespace {
// what a call needs, whatever its cache's format and its masks: of the kernels that may run, the one that needs the most (a step of one token of 32 heads over 8, d =
// 128: 5.3 MB, where the 128 rows in lanes, which it never takes, need 21.3)
size_t paged_workspace(int B, int H, int kv_heads, int T, int d) {
  const int rows = H / kv_heads * T;
  size_t most = 0;
  for (int fmt : {FP4ATTN_FMT_NVFP4, FP4ATTN_FMT_E4M3}) {
    if (few_rows(rows, fmt, d, false)) most = std::max(most, few_rows_workspace(B, H, kv_heads, T, d, fmt));
    if (!few_rows(rows, fmt, d, true)) most = std::max(most, plan(B, H, kv_heads, T, d, 0).total);
  }
  return most;
}
}  // namespace

extern "C" size_t fp4attn_paged_attention_workspace_bytes(int B, int H, int kv_heads, int T, int d) {
  if (B <= 0 || H <= 0 || kv_heads <= 0 || H % kv_heads != 0 || T <= 0 || (d != 64 && d != 128) || (long long)B * H * T >= (1ll << 31) || T >= (1 << 30) || H / kv_heads > kMostGroup)
    return 0;
  return paged_workspace(B, H, kv_heads, T, d);
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
  if ((uintptr_t)workspace & 31) return FP4ATTN_ERR_ALIGNMENT;
  if ((rc = check_device_sm100()) != FP4ATTN_OK) return rc;
  const FewRows few = {q, p.cache, context, count, first, last, slopes, O, LSE, device_status, type, cache->fmt, cache->d, B, H, T, p.scale, p.cap};
  if (few_rows(H / cache->kv_heads * T, cache->fmt, cache->d, few.changed())) return launch_few_rows(few, workspace, (cudaStream_t)stream);
  p.first = first; p.last = last;
  return launch(p, plan(B, H, cache->kv_heads, T, cache->d, 0), workspace, cache->fmt, cache->d, (cudaStream_t)stream);
}

extern "C" size_t fp4attn_shared_prefix_attention_workspace_bytes(int B, int H, int kv_heads, int T, int d, int groups) {
  if (groups <= 0 || groups > 65535 || T > FP4ATTN_MOST_TREE_TOKENS) return 0;
  return fp4attn_paged_attention_workspace_bytes(B, H, kv_heads, T, d) ? plan(B, H, kv_heads, T, d, groups).total : 0;
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
  if ((uintptr_t)workspace & 31) return FP4ATTN_ERR_ALIGNMENT;
  if ((rc = check_device_sm100()) != FP4ATTN_OK) return rc;
  p.groups = groups; p.prefix_table = prefix_table; p.prefix_pages = prefix_pages; p.prefix_length = prefix_length; p.group_start = group_start;
  p.mask = tree_mask;
  return launch(p, plan(B, H, cache->kv_heads, T, cache->d, groups), workspace, cache->fmt, cache->d, (cudaStream_t)stream);
}
