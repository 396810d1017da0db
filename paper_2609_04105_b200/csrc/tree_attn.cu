// Attention of one token, or of a tree of drafted tokens, of every sequence over its pages of a quantized cache.
//
// Row (b, h, t) sees the first context[b] tokens of the sequence, and of the T drafted tokens at positions context[b] ..
// context[b] + T - 1 those whose bit of its mask is set.
//
// The rows that read one KV head are few (1 to some hundreds), its keys are many, so keys and head dimension take the wide side of the
// tensor core and rows the narrow one:  S^T = K Q^T (128 keys x R rows),  O^T += V^T P^T (d x R rows), R = 32 or 64.  (Few rows - eight or
// sixteen, see rows_of_tile - have a kernel of their own, further down.)  Their A operands,
// K and V^T, live in tensor memory: a lane is a key of K, a head-dimension index of V^T, and the thread that turns a lane's
// codes into f16 writes them there without a word of shared memory.  Only Q and P, the narrow operands, are read from shared memory.
//
// One CTA per SM.  The 128-key tiles of all (batch entry, KV head, row tile) items stand in one list, of which every CTA takes an equal
// run, so that sequences of unlike lengths and few long ones fill the card alike.  An item whose tiles fall to several CTAs is left as
// partial (maximum, sum, O) in the workspace and joined by a second kernel in the order of its keys.
//
//   K            codes of a key -> f16 -> tensor memory; Q of an item, scaled by a power of two per row, -> f16 -> shared memory
//   V            codes of an index -> f16 -> tensor memory
//   softmax      a thread per key and 32 rows: exp2, P^T -> shared memory; rescale of O, end of an item
//   each in groups of four warps; tiles alternate between the two groups of V and, up to 32 rows, between two softmax groups with references,
//   sums and an O each: a tile is one long chain of instructions for a warp, and the time of a tile is that of the slowest chain.
//   then         one warp brings the pages in (one bulk copy per page: a (page, head) record is one run of bytes), two issue the products
//
// What bounds it: the softmax chain, 3400 clocks a tile of 64 rows (its products take 800, exp2 512, reading 800), and that every row tile of a
// KV head copies and converts the keys for itself: 4 sequences of 8192 tokens, 64 drafted tokens of 32 heads over 8 KV heads, d = 128,
// NVFP4: 98 us, 271 TFLOP/s; 16 drafted tokens of 16 heads over 4, d = 64, E4M3, 8 sequences of up to 4096: 26 us, of which starting,
// joining and the first tiles are more than half.
//
// The reference of a row, its maximum at some time, moves only when a score exceeds it by more than 2^8: probabilities up to 256 fit f16 as
// well, and neither a reduction over keys (they are in lanes) nor a pass over O is then part of an ordinary tile.  Probabilities are f16 because V
// is, exactly, and the product takes two operands of one type; each is off by at most 2^-11 of itself.  Beside bf16's rounding of O that is nothing
// (root mean square error against 64 bits 1.005 of a 32-bit form's); fp16 outputs have up to 1.28 times a 32-bit form's error.  Sums are of the
// values before they are rounded, for LSE's sake.
#include "cache_attn.cuh"

#include <limits.h>

#include <algorithm>

namespace fp4attn {

namespace {
using namespace ptx;

// CTAs of a call, each of which may leave two partial results: four an SM by warps, one by roles
constexpr int kMostWarpCtas = 640, kMostRoleCtas = 160;
template <int R> constexpr int kMostCtas = R <= 16 ? kMostWarpCtas : kMostRoleCtas;
struct TreeParams {
  const void* q;
  long long q_sb, q_sh, q_sn;
  CacheRef cache;
  const int *context, *count;
  const unsigned long long* mask;          // [B, T] or null: token t sees 0 .. t
  void* out;                               // [B, H, T, d]
  float* lse;                              // [B, H, T]
  int* status;
  float* part;                             // [2 * kMostCtas<R>][R][D]
  float2* part_ml;                         // [2 * kMostCtas<R>][R]: reference, sum
  int2* split;                             // [items]: first and last CTA of an item in parts; first = -1: whole
  int B, H, T, group, rows, row_tiles;     // rows = group * T of a KV head
  float scale;
  bool half, q_vector;
  // of fp4attn_paged_attention (PAGED instances)
  const int *seen_from, *seen_until;       // [B, T] or null
  const float* slopes;
  float cap;
};

// ---- what a CTA walks: tiles of items, in order.  The roles of a scheduler run in turn and each is one chain of instructions, so a tile
// costs what its loops execute besides the work: what changes with an item only is kept out of them (here: two instructions a tile).
struct Walk {
  int b, u;                                // batch entry, (KV head, row tile)
  int first, left;                         // first key of the tile, tiles of the item from here on
  int ctx, len;                            // context, keys (context and drafted tokens) that the table has room for
  int need;                                // keys that are there: a page that the table does not have among them is reported
  int begin, lowest;                       // PAGED: first tile of keys that rows see, first key
};
// drafted tokens that entry b has
__device__ __forceinline__ int drafted(const TreeParams& p, int b) { return p.count ? max(0, min(load(p.count + b), p.T)) : p.T; }
// tiles of an item: one at least, of no keys, where an entry has no rows
// PAGED: keys that some row sees lie between begin and len; ctx is the context all the same
template <bool PAGED = false>
__device__ __forceinline__ int load_entry(Walk& w, const TreeParams& p) {
  if (PAGED) {
    const int room = p.cache.max_pages << p.cache.log_page, n = drafted(p, w.b);
    w.ctx = max(0, min(load(p.context + w.b), (1 << 30) - 1));
    int lo = INT_MAX, hi = 0;
#pragma unroll 1
    for (int t = 0; t < n; ++t) {
      const int from = p.seen_from ? max(0, load(p.seen_from + (size_t)w.b * p.T + t)) : 0;
      const int until = min(p.seen_until ? load(p.seen_until + (size_t)w.b * p.T + t) : w.ctx + t + 1, w.ctx + n);
      if (from < until) {
        lo = min(lo, from);
        hi = max(hi, until);
      }
    }
    w.need = hi;
    w.len = min(hi, room);
    w.begin = lo < w.len ? lo / kTile * kTile : 0;
    w.lowest = lo;
    if (lo >= w.len) w.len = 0;
    return max(1, (w.len - w.begin + kTile - 1) / kTile);
  }
  const int room = p.cache.max_pages << p.cache.log_page, n = drafted(p, w.b), c = n ? max(0, load(p.context + w.b)) : 0;
  w.ctx = min(c, room);
  w.need = (int)min((long long)c + n, (long long)INT_MAX);
  w.len = n ? (int)min((long long)c + (p.mask ? p.T : n), (long long)room) : 0;        // (a mask may look behind the count)
  return max(1, (w.len + kTile - 1) / kTile);
}
template <bool PAGED = false>
__device__ __forceinline__ void next_item(Walk& w, const TreeParams& p, int units) {
  w.first = 0;
  if (++w.u == units) {
    w.u = 0;
    ++w.b;
  }
  if (w.b < p.B) w.left = load_entry<PAGED>(w, p);
  if (PAGED) w.first = w.begin;
}
// to the next tile; was this one the last of its item?
template <bool PAGED = false>
__device__ __forceinline__ bool advance(Walk& w, const TreeParams& p, int units) {
  w.first += kTile;
  if (!rare(--w.left == 0)) return false;
  next_item<PAGED>(w, p, units);
  return true;
}
// n tiles on; how many items ended on the way, and whether the tile is the first of its item
__device__ __forceinline__ int advance_by(Walk& w, const TreeParams& p, int units, int n, bool* fresh) {
  int ended = 0;
  for (int k = 0; k < n; ++k) {
    *fresh = advance(w, p, units);
    ended += *fresh;
  }
  return ended;
}
__device__ __forceinline__ unsigned long long row_mask(const TreeParams& p, int b, int t, int n) {
  if (t >= n) return 0ull;
  return p.mask ? load(p.mask + (size_t)b * p.T + t) : (2ull << t) - 1;
}

// R: rows of a tile, 32 or 64
template <int FMT, int D, int R>
struct TreeCfg {
  using L = RecordLayout<FMT, D>;
  static constexpr int kN = 32;                                    // rows of a softmax thread
  static constexpr int kColGroups = R / kN;
  static constexpr int kSets = R <= 32 ? 2 : 1;                    // sets of softmax groups that tiles alternate between
  static constexpr int kKGroups = 1, kVGroups = 2;                 // groups of four warps that tiles alternate between
  static constexpr int kFirstV = 4 * kKGroups, kFirstSoftmax = kFirstV + 4 * kVGroups;         // warps
  static constexpr int kProducer = kFirstSoftmax + 4 * kColGroups * kSets, kIssuerS = kProducer + 1, kIssuerO = kProducer + 2;
  static constexpr int kThreads = 32 * (kProducer + 4);            // the last warp only makes up a warpgroup
  // Registers: 80 a thread at launch.  A softmax thread needs 128 for its 32 rows (with 16 rows a thread and 64 registers a third of
  // its scores and sums were in local memory: 3850 clocks a tile of 64 rows); the other roles give up what it takes.  The compiler allots
  // for 80 all the same: 81 loads and 47 stores of local memory a tile of 64 rows, all warps together, of 5250 instructions.
  static constexpr int kRegsLaunch = 80, kRegsAux = 32, kRegsKV = 64, kRegsSoftmax = 128;
  static_assert(kThreads * kRegsLaunch <= 65536 &&
                kRegsAux + (kKGroups + kVGroups) * kRegsKV + kColGroups * kSets * kRegsSoftmax <= kThreads / 128 * kRegsLaunch, "register shares");
  static constexpr int kStage = kTile * 2 * L::kToken;
  static constexpr int kStages = kStage >= 32768 ? 4 : kStage > 16384 ? 6 : 8;
  // Buffers between the roles: deep enough that the hand-overs (some 200 clocks each) of one tile lie under the work on others
  static constexpr int kSB = kSets == 2 ? 4 : 2, kVB = 3;          // scores; V^T in tensor memory and P
  static constexpr int kKB = D == 64 ? 4 : 2;                      // K in tensor memory
  static constexpr int kQB = kKB;                                  // Q: see the K warps
  static constexpr int kQ = R * D * 2, kP = kTile * R * 2;
  // The softmax warps may be kKB + kSB tiles behind the K warps, and those kStages behind the producer: what they take from either
  // past the barriers is kept for as many items and tiles.
  static constexpr int kRingC = 8, kRing = 32;
  static_assert(kKB + kSB <= kRingC && kStages + kKB + kSB <= kRing, "rings");
  // shared memory
  static constexpr int kOffStage = 0;
  static constexpr int kOffQ = kOffStage + kStages * kStage;
  static constexpr int kOffP = kOffQ + kQB * kQ;
  static constexpr int kOffVScale = kOffP + kVB * kP;                // f16 [V warps][2 blocks][128 tokens]
  static constexpr int kOffCM = kOffVScale + 4 * kVGroups * 512;                 // float [kSets][2][R]: kShift minus the reference; score constant
  static constexpr int kOffC = kOffCM + 8 * R * kSets;             // float [kRingC][R]: score constants of the last items
  static constexpr int kOffBits = kOffC + 4 * R * kRingC;          // u32 [kSets][kColGroups][64]: rows that see a drafted token
  static constexpr int kOffWarp = kOffBits + 256 * kColGroups * kSets;         // float [kSets][4][R]: maxima or sums of the four warps
  static constexpr int kOffScale = kOffWarp + 16 * R * kSets;      // float [kSets][R]: factors on O
  static constexpr int kOffValid = kOffScale + 4 * R * kSets;      // u32 [kRing]
  static constexpr int kOffScan = kOffValid + 4 * kRing;           // i64 [32]
  static constexpr int kOffFind = kOffScan + 256;                  // i64 [5] (room for eight)
  static constexpr int kOffBar = kOffFind + 64;
  static constexpr int kSmem = kOffBar + 512 + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory");
  // barriers
  enum { KA_FULL = 0, KA_FREE = KA_FULL + kKB, VA_FULL = KA_FREE + kKB, P_FULL = VA_FULL + kVB, PV_DONE = P_FULL + kVB, S_FULL = PV_DONE + kVB,
         S_FREE = S_FULL + kSB, Q_FULL = S_FREE + kSB, DRAIN = Q_FULL + kQB, RING_FULL = DRAIN + 2, RING_FREE = RING_FULL + kStages };
  static constexpr int kBars = RING_FREE + kStages;
  static_assert(kBars * 8 + 16 <= 512, "barriers");
  // tensor memory columns
  static constexpr int kKA = 0, kVA = kKA + kKB * D / 2, kS = kVA + kVB * kTile / 2, kO = kS + kSB * R;
  static_assert(kO + R * kSets <= 512, "tensor memory");
};

// four bits -> byte masks of a word
__device__ __forceinline__ uint32_t byte_mask(uint32_t bits) { return ((bits & 15u) * 0x00204081u & 0x01010101u) * 0xFFu; }
// eight bits in the order V scales are kept in: 0 4 1 5 2 6 3 7
__device__ __forceinline__ uint32_t permute_eight(uint32_t v) {
  uint32_t lo = v & 15u, hi = v >> 4 & 15u;
  lo = (lo | lo << 2) & 0x33u; lo = (lo | lo << 1) & 0x55u;
  hi = (hi | hi << 2) & 0x33u; hi = (hi | hi << 1) & 0x55u;
  return lo | hi << 1;
}
// sum over the warp of each of N values: lane i ends with the total of value i % N
template <int N>
__device__ __forceinline__ float warp_sums(float (&v)[N], int lane) {
#pragma unroll
  for (int step = N / 2; step; step >>= 1) {
    const bool up = lane & step;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      if (i < step) {
        const float give = up ? v[i] : v[i + step], keep = up ? v[i + step] : v[i];
        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, step);
      }
    }
  }
  float s = v[0];
#pragma unroll
  for (int step = N; step < 32; step <<= 1) s += __shfl_xor_sync(0xffffffffu, s, step);
  return s;
}
template <int N>
__device__ __forceinline__ void tmem_ld_cols(uint32_t addr, uint32_t (&r)[N]) {
  if constexpr (N == 32) tmem_ld_32x32b_x32(addr, r);
  else tmem_ld_32x32b_x16(addr, r);
}
// of the eight tokens from position `pos` on, those that count (bit t: token t): the context, and the drafted tokens that some row sees
__device__ __forceinline__ uint32_t valid_eight(const Walk& w, unsigned long long seen, int pos) {
  const int in = w.ctx - pos, left = w.len - pos;                  // tokens of these in the context; that the table has room for
  uint32_t v = in >= 8 ? 0xFFu : in >= 0 ? (uint32_t)(seen << in) & 0xFFu : -in < 64 ? (uint32_t)(seen >> -in) & 0xFFu : 0u;
  if (in > 0 && in < 8) v |= (1u << in) - 1;
  return left >= 8 ? v : left > 0 ? v & ((1u << left) - 1) : 0u;
}

// This CTA's run of tiles: how many, and where it starts.  find: entry and place of the first tile, its number in the list, all tiles,
// CTAs.  A barrier of the block (two for a batch of more than 32): everything that the block wrote to shared memory before is visible after it.
template <int THREADS, bool PAGED = false>
__device__ __forceinline__ int find_run(const TreeParams& p, int units, Walk& w0, long long* scan, long long* find) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Walk w;
  long long t0, t1, total;
  auto run = [&] {
    const long long ctas = min((long long)gridDim.x, total);
    t0 = blockIdx.x < ctas ? mul_div(blockIdx.x, total, ctas) : total;
    t1 = blockIdx.x < ctas ? mul_div(blockIdx.x + 1, total, ctas) : total;
    if (threadIdx.x == 0) {
      find[2] = t0;
      find[3] = total;
      find[4] = ctas;
    }
  };
  long long at;                                                     // of the first tile among its entry's
  if (p.B <= 32) {                                                  // every warp for itself
    w.b = lane;
    const int nt = lane < p.B ? load_entry<PAGED>(w, p) : 0;
    const long long mine = (long long)nt * units;
    long long incl = mine;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, incl, s);
      if (lane >= s) incl += o;
    }
    total = __shfl_sync(0xffffffffu, incl, 31);
    run();
    const uint32_t behind = __ballot_sync(0xffffffffu, incl > t0);  // entries that end behind the first tile
    const int b = t0 < t1 ? __ffs(behind) - 1 : 0;
    w0.b = b;
    w0.ctx = __shfl_sync(0xffffffffu, w.ctx, b);
    w0.len = __shfl_sync(0xffffffffu, w.len, b);
    w0.need = __shfl_sync(0xffffffffu, w.need, b);
    if (PAGED) {
      w0.begin = __shfl_sync(0xffffffffu, w.begin, b);
      w0.lowest = __shfl_sync(0xffffffffu, w.lowest, b);
    }
    w0.left = __shfl_sync(0xffffffffu, nt, b);
    at = t0 < t1 ? t0 - __shfl_sync(0xffffffffu, incl - mine, b) : 0;
    __syncthreads();
  } else {
    const int per = (p.B + THREADS - 1) / THREADS, b0 = threadIdx.x * per, b1 = min(p.B, b0 + per);
    long long mine = 0;
#pragma unroll 1
    for (w.b = b0; w.b < b1; ++w.b) mine += (long long)load_entry<PAGED>(w, p) * units;
    long long incl = mine;
#pragma unroll 1
    for (int s = 1; s < 32; s <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, incl, s);
      if (lane >= s) incl += o;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    long long before = 0;
    total = 0;
#pragma unroll 1
    for (int i = 0; i < THREADS / 32; ++i) {
      if (i < warp) before += scan[i];
      total += scan[i];
    }
    before += incl - mine;
    run();
    if (t0 < t1 && before <= t0 && t0 < before + mine) {            // one thread
      for (w.b = b0;; ++w.b) {
        const long long here = (long long)load_entry<PAGED>(w, p) * units;
        if (t0 < before + here) break;
        before += here;
      }
      find[0] = w.b;
      find[1] = t0 - before;
    }
    __syncthreads();
    w0.b = t0 < t1 ? (int)find[0] : 0;
    w0.left = load_entry<PAGED>(w0, p);
    at = t0 < t1 ? find[1] : 0;
  }
  w0.u = (int)mul_div(at, 1, w0.left);
  const int kt = (int)(at - (long long)w0.u * w0.left);
  w0.first = kt * kTile + (PAGED ? w0.begin : 0);
  w0.left -= kt;
  return (int)min(t1 - t0, (long long)INT_MAX);
}

// Brings the pages of tiles into a ring of stages, one bulk copy each; a whole warp.  RING: stages for which `valid` remembers which of the
// pages exist.  PARTS = 2: K and V by themselves, each in a stage of its own.
template <int STAGES, int STAGE, int RING, int PARTS, bool CALL, bool PAGED = false>
struct Pages {
  Walk w;
  Turn<STAGES> ring;
  int i = 0;                                                        // part
  bool lost = false;
  int page = -1;                                                    // of this lane, of the tile
  __device__ __forceinline__ void find(const TreeParams& p) {
    const int lane = threadIdx.x & 31, P = 1 << p.cache.log_page, slots = kTile >> p.cache.log_page;       // pages of a tile: 1 to 8
    page = -1;
    if (lane < slots && w.first + lane * P < w.len && (!PAGED || w.first + lane * P + P > w.lowest)) {
      page = p.cache.page_of(w.b, w.first + lane * P);
      lost |= page < 0 && w.first + lane * P < w.need;
    }
    lost |= w.need > (PAGED ? p.cache.max_pages << p.cache.log_page : w.len);        // the table has no room for the last tokens
  }
  // false: the stage has not become free, some wait has run out; nothing was begun, and nothing more must be
  __device__ __forceinline__ bool bring(const TreeParams& p, uint32_t stages, uint32_t full, uint32_t free, uint32_t abort_at, uint32_t* valid) {
    const int lane = threadIdx.x & 31;
    const uint32_t held = __ballot_sync(0xffffffffu, page >= 0);
    wait_phase<CALL>(free + 8 * ring.at, ring.phase ^ 1, abort_at);
    if (rare(given_up(abort_at))) return false;
    const int bytes = p.cache.record / PARTS;
    if (lane == 0) {
      valid[i % RING] = held;
      mbar_arrive_expect_tx(full + 8 * ring.at, __popc(held) * bytes);
    }
    __syncwarp();
    if (page >= 0)
      bulk_load_1d(stages + ring.at * STAGE + lane * bytes, p.cache.rec(page, w.u / p.row_tiles) + (PARTS == 2 ? (i & 1) * bytes : 0), bytes,
                   full + 8 * ring.at);
    return true;
  }
  __device__ __forceinline__ void skip(const TreeParams& p, int units, int n) {
#pragma unroll 1
    for (int k = 0; k < n; ++k) {
      if (PARTS == 1 || (i & 1)) advance<PAGED>(w, p, units);
      ring.next();
      ++i;
    }
  }
  __device__ __forceinline__ void tell(const TreeParams& p) const {
    if (__any_sync(0xffffffffu, lost) && (threadIdx.x & 31) == 0 && p.status) *p.status = FP4ATTN_ERR_PAGE;
  }
};

template <int FMT, int D, int R>
__global__ void __launch_bounds__(TreeCfg<FMT, D, R>::kThreads, 1) tree_kernel(const TreeParams p) {
  using C = TreeCfg<FMT, D, R>;
  using L = typename C::L;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const sgen = smem_raw + (sbase - smem_u32(smem_raw));
  const uint32_t abort_at = sbase + C::kOffBar + 8 * C::kBars, tslot = abort_at + 4;
  volatile uint32_t* const abort_word = reinterpret_cast<volatile uint32_t*>(sgen + C::kOffBar + 8 * C::kBars);
  auto bar = [&](int i) { return sbase + C::kOffBar + 8u * i; };
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int units = p.cache.kv_heads * p.row_tiles;

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kKB; ++i) {
      mbar_init(bar(C::KA_FULL + i), 4);
      mbar_init(bar(C::KA_FREE + i), 1);
    }
    for (int i = 0; i < C::kVB; ++i) {
      mbar_init(bar(C::VA_FULL + i), 4);
      mbar_init(bar(C::P_FULL + i), 4 * C::kColGroups);
      mbar_init(bar(C::PV_DONE + i), 1);
    }
    for (int i = 0; i < C::kSB; ++i) {
      mbar_init(bar(C::S_FULL + i), 1);
      mbar_init(bar(C::S_FREE + i), 4 * C::kColGroups);
    }
    for (int i = 0; i < C::kQB; ++i) mbar_init(bar(C::Q_FULL + i), 4);
    for (int i = 0; i < 2; ++i) mbar_init(bar(C::DRAIN + i), 1);
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(bar(C::RING_FULL + s), 1);
      mbar_init(bar(C::RING_FREE + s), 8);
    }
    *abort_word = 0;
    fence_barrier_init();
  }
  if (warp == C::kIssuerS) { tmem_alloc(tslot, 512); tmem_relinquish(); }
  tc_fence_before();
  launch_dependents();                                              // the joining kernel: its launch lies under this one
  wait_prior_grids();
  Walk w0;
  long long* const find = reinterpret_cast<long long*>(sgen + C::kOffFind);
  const int n_tiles = find_run<C::kThreads>(p, units, w0, reinterpret_cast<long long*>(sgen + C::kOffScan), find);
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(sgen + C::kOffBar + 8 * C::kBars + 4);
  uint32_t* const valid_ring = reinterpret_cast<uint32_t*>(sgen + C::kOffValid);
  const int P = 1 << p.cache.log_page;
  auto wait = [&](int b, int phase) { wait_phase<false>(bar(b), (uint32_t)phase, abort_at); };

  if (warp >= C::kProducer) {
    registers_fewer<C::kRegsAux>();
    if (warp == C::kProducer) {
      // ===================================================================== pages -> shared memory
      Pages<C::kStages, C::kStage, C::kRing, 1, false> pages;
      pages.w = w0;
      if (n_tiles > 0) pages.find(p);
      while (pages.i < n_tiles) {
        if (rare(!pages.bring(p, sbase + C::kOffStage, bar(C::RING_FULL), bar(C::RING_FREE), abort_at, valid_ring))) break;
        pages.skip(p, units, 1);
        if (pages.i < n_tiles) pages.find(p);                         // the table's entries come while the stage is waited for
      }
      pages.tell(p);
      drain(pages.ring, bar(C::RING_FULL), pages.i);
    } else if (warp == C::kIssuerS) {
      // ===================================================================== S^T = K Q^T
      // Q: K-major, core matrices of 8 rows x 16 bytes, those along d neighbours.  A product takes 45 clocks or more whatever its N up to 64,
      // and its issue waits for the one before: two warps issue, so that the waits of one lie under the products of the other.
      constexpr uint32_t kIdesc = make_idesc_f16(128, R, false);
      Walk w = w0;
      Turn<C::kKB> kb;
      Turn<C::kSB> sb;
      Turn<C::kQB> qb;
      bool fresh = true;
      for (int i = 0; i < n_tiles; ++i) {
        if (rare(fresh)) wait(C::Q_FULL + qb.at, qb.phase);
        wait(C::S_FREE + sb.at, sb.phase ^ 1);
        wait(C::KA_FULL + kb.at, kb.phase);
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            tc_mma_f16_ta(tmem + C::kS + R * sb.at, tmem + C::kKA + (D / 2) * kb.at + 8 * k,
                          make_smem_desc(sbase + C::kOffQ + qb.at * C::kQ + k * 256, 128, (D / 8) * 128, kSwzNone), kIdesc, k > 0);
          tc_commit(bar(C::S_FULL + sb.at));
          tc_commit(bar(C::KA_FREE + kb.at));
        }
        __syncwarp();
        kb.next();
        sb.next();
        fresh = advance(w, p, units);
        if (rare(fresh)) qb.next();
      }
      if (elect_one()) tc_commit(bar(C::DRAIN));
      __syncwarp();
    } else if (warp == C::kIssuerO) {
      // ===================================================================== O^T += V^T P^T
      // P: rows are contiguous (MN-major), core matrices of 8 keys x 16 bytes (8 rows), those along rows neighbours
      constexpr uint32_t kIdesc = make_idesc_f16(128, R, true);
      Walk w = w0;
      int of_item = 0;                                                // tiles of the item so far
      Turn<C::kVB> vb;
      for (int i = 0; i < n_tiles; ++i) {
        wait(C::VA_FULL + vb.at, vb.phase);
        wait(C::P_FULL + vb.at, vb.phase);
        tc_fence_after();
        const uint32_t more = of_item >= C::kSets;                    // not the first tile of the item that this O gets
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < kTile / 16; ++k)
            tc_mma_f16_ta(tmem + C::kO + (C::kSets == 2 ? R * (i & 1) : 0), tmem + C::kVA + 64 * vb.at + 8 * k,
                          make_smem_desc(sbase + C::kOffP + vb.at * C::kP + k * 2 * (R / 8) * 128, (R / 8) * 128, 128, kSwzNone), kIdesc,
                          k > 0 ? 1u : more);
          tc_commit(bar(C::PV_DONE + vb.at));
        }
        __syncwarp();
        vb.next();
        of_item = advance(w, p, units) ? 0 : of_item + 1;
      }
      if (elect_one()) tc_commit(bar(C::DRAIN + 1));
      __syncwarp();
    }
  } else if (warp < C::kFirstSoftmax) {
    registers_fewer<C::kRegsKV>();
    if (warp < C::kFirstV) {
      // ===================================================================== Q and K
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
      const int group = warp >> 2, quarter = warp & 3;
      const int key = quarter * 32 + lane, slot = key >> p.cache.log_page, t = key & (P - 1);
      const float c0 = p.scale * 1.4426950408889634f;
      Walk w = w0;
      Turn<C::kStages> ring;
      Turn<C::kKB> kb;
      int item = 0;
      bool fresh = true;
      if (group && n_tiles > 0) {
        item = advance_by(w, p, units, group, &fresh);
        ring.next(group);
        kb.next(group);
      }
      for (int i = group; i < n_tiles; i += C::kKGroups) {
        wait(C::KA_FREE + kb.at, kb.phase ^ 1);
        if (rare(fresh)) {
          // Rows scaled by a power of two into f16's range (the largest element to [2^14, 2^15)): exact for 8-bit significands, and a row's
          // scores are scaled back by its constant.  The buffer is free: as many items back, the last tile that read it was tile i - kKB or
          // an earlier one, whose product is done.
          const int kvh = w.u / p.row_tiles, row0 = (w.u - kvh * p.row_tiles) * R, qb = item % C::kQB;
          const float c = __fdiv_rn(c0, load(p.cache.k_G + kvh));
          constexpr int kParts = D / 16;                              // threads of a row
#pragma unroll
          for (int j = key; j < R * kParts; j += 128) {
            const int r = j / kParts, e = (j % kParts) * 16, row = row0 + r;
            float v[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) v[x] = 0.f;
            if (row < p.rows) {
              const int hl = row / p.T, tok = row - hl * p.T;
              const uint16_t* q = static_cast<const uint16_t*>(p.q) + w.b * p.q_sb + (long long)(kvh * p.group + hl) * p.q_sh + tok * p.q_sn + e;
              uint32_t raw[8];
              if (p.q_vector) {
                *reinterpret_cast<uint4*>(raw) = load(reinterpret_cast<const uint4*>(q));
                *reinterpret_cast<uint4*>(raw + 4) = load(reinterpret_cast<const uint4*>(q) + 1);
              } else {
#pragma unroll
                for (int x = 0; x < 8; ++x) raw[x] = (uint32_t)load(q + 2 * x) | (uint32_t)load(q + 2 * x + 1) << 16;
              }
#pragma unroll
              for (int x = 0; x < 8; ++x) {
                const float2 f = p.half ? unpack16<true>(raw[x]) : unpack16<false>(raw[x]);
                v[2 * x] = f.x;
                v[2 * x + 1] = f.y;
              }
            }
            float a = 0.f;
#pragma unroll
            for (int x = 0; x < 16; ++x) a = fmaxf(a, fabsf(v[x]));
#pragma unroll
            for (int x = 1; x < kParts; x <<= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, x));
            const uint32_t up = row_exponent(a);
            const float f = __uint_as_float(up << 23);
            uint32_t h[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) h[x] = pack_pair<__half>(v[2 * x] * f, v[2 * x + 1] * f);
            uint8_t* const dst = sgen + C::kOffQ + qb * C::kQ + ((r >> 3) * (D / 8) + (e >> 3)) * 128 + (r & 7) * 16;
            *reinterpret_cast<uint4*>(dst) = make_uint4(h[0], h[1], h[2], h[3]);
            *reinterpret_cast<uint4*>(dst + 128) = make_uint4(h[4], h[5], h[6], h[7]);
            if (e == 0) reinterpret_cast<float*>(sgen + C::kOffC)[(item & (C::kRingC - 1)) * R + r] = c * __uint_as_float((254u - up) << 23);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::Q_FULL + qb));
        }
        wait(C::RING_FULL + ring.at, ring.phase);
        {
          tc_fence_after();
          const uint8_t* const rec = sgen + C::kOffStage + ring.at * C::kStage + slot * p.cache.record;
          const uint32_t dst = tmem + lanes + C::kKA + (D / 2) * kb.at;
          // (rolled loops: what the four roles of a scheduler run in turn has to stay in its instruction cache)
          const uint8_t* codes = rec + t * 16;
          uint2 sw = make_uint2(0u, 0u);
          if (L::kFp4 && D == 128) sw = *reinterpret_cast<const uint2*>(rec + L::k_scales(P) + t * L::kScales);
          if (L::kFp4 && D == 64) sw.x = *reinterpret_cast<const uint32_t*>(rec + L::k_scales(P) + t * L::kScales);
#pragma unroll 2
          for (int c = 0; c < D / 32; ++c) {
            uint32_t h[16];
            if (L::kFp4) {
              const uint4 raw = *reinterpret_cast<const uint4*>(codes);
              codes += P * 16;
              const uint32_t words[4] = {raw.x, raw.y, raw.z, raw.w}, two = cvt_f16x2_e4m3x2(sw.x & 0xFFFFu);
              sw.x = __funnelshift_r(sw.x, sw.y, 16);
              sw.y >>= 16;
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const uint32_t f = splat_half(two, x >> 1);
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
            tmem_st_32x32b_x16(dst + 16 * c, h);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::RING_FREE + ring.at));   // (the loads are done: their values have been used)
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::KA_FULL + kb.at));
        }
        ring.next(C::kKGroups);
        kb.next(C::kKGroups);
        item += advance_by(w, p, units, C::kKGroups, &fresh);
      }
    } else {
      // ===================================================================== V
      const int quarter = warp & 3, group = (warp - C::kFirstV) >> 2, e = quarter * 32 + lane;      // index of the head dimension
      const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
      uint8_t* const scales = sgen + C::kOffVScale + (warp - C::kFirstV) * 512;
      // this lane's codes in a stage: chunks of sixteen tokens, further in the page or at the same place of the next
      const int log_page = p.cache.log_page, record = p.cache.record;
      const uint32_t codes0 = (uint32_t)(L::v_codes(P) + (L::kFp4 ? e >> 1 : e) * 16);
      const uint32_t step16 = P == 16 ? (uint32_t)record : 16 * L::kRow;
      const uint32_t step32 = P <= 32 ? (uint32_t)((32 >> log_page) * record) : 32 * L::kRow;
      const uint32_t step64 = P <= 64 ? (uint32_t)((64 >> log_page) * record) : 64 * L::kRow;
      const int at_sc = 8 * (lane & 15);                              // eight tokens whose scales of block e / 16 this lane converts
      const uint32_t scale0 = (uint32_t)((at_sc >> log_page) * record + L::v_scales(P) + (e >> 4) * P + (at_sc & (P - 1)));
      Walk w = w0;
      Turn<C::kStages> ring;
      Turn<C::kVB> vb;
      int b_of = -1;
      unsigned long long seen = 0;                                    // drafted tokens that some row sees
      bool fresh;
      if (group && n_tiles > 0) {
        advance_by(w, p, units, group, &fresh);
        ring.next(group);
        vb.next(group);
      }
      for (int i = group; i < n_tiles; i += C::kVGroups) {
        if (rare(w.b != b_of)) {
          b_of = w.b;
          const int n = drafted(p, w.b);
          seen = row_mask(p, w.b, lane, n) | (lane + 32 < p.T ? row_mask(p, w.b, lane + 32, n) : 0ull);
          seen = (unsigned long long)__reduce_or_sync(0xffffffffu, (uint32_t)(seen >> 32)) << 32 | __reduce_or_sync(0xffffffffu, (uint32_t)seen);
        }
        wait(C::PV_DONE + vb.at, vb.phase ^ 1);
        wait(C::RING_FULL + ring.at, ring.phase);
        {
          tc_fence_after();
          const uint32_t held = valid_ring[i % C::kRing];
          const int first = w.first;
          // what no row sees counts as zero: it may be any bytes, and a probability of 0 times a NaN would be one
          const bool all = first + kTile <= w.ctx && held == (1u << (kTile >> p.cache.log_page)) - 1;
          const uint8_t* const stage = sgen + C::kOffStage + ring.at * C::kStage;
          const uint32_t dst = tmem + lanes + C::kVA + 64 * vb.at, shift = 4 * (e & 1);
          if (quarter * 32 < D) {
            if (L::kFp4) {
              // the scales of this warp's two blocks, once for all sixteen lanes that need them
              uint2 sc = *reinterpret_cast<const uint2*>(stage + scale0);
              if (rare(!all)) {
                const uint32_t v = held >> (at_sc >> log_page) & 1 ? permute_eight(valid_eight(w, seen, first + at_sc)) : 0u;
                sc.x &= byte_mask(v);
                sc.y &= byte_mask(v >> 4);
              }
              uint32_t f[4];
              cvt_f16x2_e4m3x4(sc.x, f);
              cvt_f16x2_e4m3x4(sc.y, f + 2);
              *reinterpret_cast<uint4*>(scales + lane * 16) = make_uint4(f[0], f[1], f[2], f[3]);
              __syncwarp();
            }
            const uint8_t* codes = stage + codes0;
            const uint8_t* factors = scales + (lane >> 4) * 256;
#pragma unroll 2
            for (int j = 0; j < kTile; j += 16) {                     // sixteen tokens
              uint4 raw = *reinterpret_cast<const uint4*>(j & 16 ? codes + step16 : codes);
              if (j & 16) codes = j & 32 ? stage + codes0 + step64 : codes + step32;
              uint32_t h[8];
              if (L::kFp4) {
                const uint32_t cw[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                for (int x = 0; x < 2; ++x) {                         // eight tokens: i and i + 4 in a byte
                  const uint4 f = *reinterpret_cast<const uint4*>(factors + 2 * j + 16 * x);
                  cvt_f16x2_e2m1x8((cw[2 * x] >> shift & 0x0F0F0F0Fu) | (cw[2 * x + 1] << (4 - shift) & 0xF0F0F0F0u), h + 4 * x);
                  h[4 * x] = mul_half2(h[4 * x], f.x);
                  h[4 * x + 1] = mul_half2(h[4 * x + 1], f.y);
                  h[4 * x + 2] = mul_half2(h[4 * x + 2], f.z);
                  h[4 * x + 3] = mul_half2(h[4 * x + 3], f.w);
                }
              } else {
                if (rare(!all)) {
                  const bool here = held >> (j >> log_page) & 1;
                  const uint32_t lo = here ? valid_eight(w, seen, first + j) : 0u;
                  const uint32_t hi = here ? valid_eight(w, seen, first + j + 8) : 0u;
                  raw.x &= byte_mask(lo); raw.y &= byte_mask(lo >> 4); raw.z &= byte_mask(hi); raw.w &= byte_mask(hi >> 4);
                }
                const uint32_t cw[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                for (int x = 0; x < 4; ++x) cvt_f16x2_e4m3x4(cw[x], h + 2 * x);
              }
              tmem_st_32x32b_x8(dst + (j >> 1), h);
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::RING_FREE + ring.at));
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::VA_FULL + vb.at));
        }
        ring.next(C::kVGroups);
        vb.next(C::kVGroups);
        advance_by(w, p, units, C::kVGroups, &fresh);
      }
    }
  } else {
    // ===================================================================== softmax
    registers_more<C::kRegsSoftmax>();
    constexpr int N = C::kN;
    const int group = (warp - C::kFirstSoftmax) >> 2, set = group / C::kColGroups, cols = group % C::kColGroups, c0 = cols * N;
    const int quarter = warp & 3, key = quarter * 32 + lane;
    const int id = 1 + group, id_all = 5 + cols;                    // named barriers: this group's 128 threads; the sets of these rows
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    float* const ref_all = reinterpret_cast<float*>(sgen + C::kOffCM) + c0;                      // [kSets][2] R apart: kShift - reference
    float* const ref = ref_all + set * 2 * R;
    float* const con = ref + R;                                                                  // score constants
    uint32_t* const bits = reinterpret_cast<uint32_t*>(sgen + C::kOffBits) + 64 * group;
    float* const warps_all = reinterpret_cast<float*>(sgen + C::kOffWarp) + c0;                  // [kSets][4] R apart
    float* const warps = warps_all + set * 4 * R;
    float* const factor_all = reinterpret_cast<float*>(sgen + C::kOffScale) + c0;
    float* const factor = factor_all + set * R;
    // where this key's probabilities stand among the keys of P: as V's tokens do in tensor memory
    const int place = L::kFp4 ? v_scale_place(key) : key;
    const uint32_t p_row = (uint32_t)((place >> 3) * (R / 8) * 128 + (c0 >> 3) * 128 + (place & 7) * 16);
    const uint32_t o_mine = tmem + lanes + C::kO + set * R + c0;
    Walk w = w0;
    Turn<C::kSB> sb;
    Turn<C::kVB> vb;
    int item = 0, part_first = 0;                                   // part_first: first key of the item that this CTA takes
    int last = 0, last_phase = 0;                                   // of this set's last tile: its buffer of P
    bool fresh = true, started = false;                             // of the item; has this set had a tile of it?
    float l[N];
    for (int i = 0; i < n_tiles; ++i) {
      if (rare(fresh)) {
        part_first = w.first;
        {
          // a lane has a row's mask; a word per drafted token, sixteen a warp
          const int row = w.u % p.row_tiles * R + c0 + lane;
          const unsigned long long mask = row < p.rows ? row_mask(p, w.b, row % p.T, drafted(p, w.b)) : 0ull;
          const uint32_t mine = (uint32_t)(mask >> (16 * quarter));
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const uint32_t word = __ballot_sync(0xffffffffu, mine >> j & 1);
            if (lane == j) bits[16 * quarter + j] = word;
          }
        }
#pragma unroll
        for (int r = 0; r < N; ++r) l[r] = 0.f;
        fresh = started = false;
      }
      if (C::kSets == 1 || (i & 1) == set) {
        wait(C::S_FULL + sb.at, sb.phase);
        if (rare(!started)) {                                       // (Q's constants were there before its products were issued)
          if (key < N) {
            con[key] = reinterpret_cast<const float*>(sgen + C::kOffC)[(item & (C::kRingC - 1)) * R + c0 + key];
            ref[key] = INFINITY;
          }
          bar_sync(id, 128);
        }
        tc_fence_after();
        const uint32_t scores = tmem + lanes + C::kS + R * sb.at + c0;
        uint32_t raw[N];
        tmem_ld_cols(scores, raw);
        tmem_wait_ld();
        const uint32_t held = valid_ring[i % C::kRing];
        // scores in octaves above the rows' references (+ kShift); those that are not seen go to -infinity
        float x[N], top = -INFINITY;
        uint32_t rows_seeing = 0xFFFFFFFFu;                             // rows of this thread that see its key
        const bool plain = w.first + kTile <= w.ctx && held == (1u << (kTile >> p.cache.log_page)) - 1;
        if (rare(!plain)) {
          const int pos = w.first + key;
          const bool here = held >> (key >> p.cache.log_page) & 1;
          rows_seeing = !here || pos >= w.len ? 0u : pos < w.ctx ? 0xFFFFFFFFu : bits[pos - w.ctx];
        }
        auto relative = [&](bool references) {
#pragma unroll
          for (int r = 0; r < N; r += 4) {
            const uint4 c = *reinterpret_cast<const uint4*>(con + r);
            uint4 k = *reinterpret_cast<const uint4*>(ref + r);
            if (!references) k = make_uint4(0u, 0u, 0u, 0u);
            fma_pair(x[r], x[r + 1], raw[r], raw[r + 1], c.x, c.y, k.x, k.y);
            fma_pair(x[r + 2], x[r + 3], raw[r + 2], raw[r + 3], c.z, c.w, k.z, k.w);
          }
          if (rare(!plain)) {
#pragma unroll
            for (int r = 0; r < N; ++r)
              if (!(rows_seeing >> r & 1)) x[r] = -INFINITY;
          }
        };
        relative(true);
#pragma unroll
        for (int r = 0; r < N; r += 2) top = max3(top, x[r], x[r + 1]);
        if (rare(bar_any(id, 128, !started || top > kLag + kShift))) {
          // the references move: to the largest score seen so far (the scores are read again: kept, they would cost as many registers)
          tmem_ld_cols(scores, raw);
          tmem_wait_ld();
          relative(false);
#pragma unroll
          for (int r = 0; r < N; ++r) {
            const float m = warp_max(x[r]);
            if (lane == 0) warps[quarter * R + r] = m;
          }
          bar_sync(id, 128);
          if (key < N) {
            const float old = kShift - ref[key];                   // -infinity: none yet
            const float m = fmaxf(fmaxf(fmaxf(warps[key], warps[R + key]), fmaxf(warps[2 * R + key], warps[3 * R + key])), old);
            factor[key] = m == -INFINITY ? 1.f : exp2_approx(old - m);
            ref[key] = kShift - m;
          }
          bar_sync(id, 128);
          tmem_ld_cols(scores, raw);
          tmem_wait_ld();
          relative(true);
#pragma unroll
          for (int r = 0; r < N; ++r) l[r] *= factor[r];
          if (started) {                                            // O of this set's tiles before
            wait(C::PV_DONE + last, last_phase);
            tc_fence_after();
            uint32_t o[N];
            tmem_ld_cols(o_mine, o);
            tmem_wait_ld();
#pragma unroll
            for (int r = 0; r < N; ++r) o[r] = __float_as_uint(__uint_as_float(o[r]) * factor[r]);
            tmem_st_32x32b_x16(o_mine, o);
            tmem_st_32x32b_x16(o_mine + 16, o + 16);
            tmem_wait_st();
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::S_FREE + sb.at));
        wait(C::PV_DONE + vb.at, vb.phase ^ 1);                     // what stood in this P has been read
        uint8_t* const dst = sgen + C::kOffP + vb.at * C::kP + p_row;
#pragma unroll
        for (int r = 0; r < N; r += 8) {
          uint32_t h[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float a = exp2_approx(x[r + 2 * y]), b = exp2_approx(x[r + 2 * y + 1]);
            add_pair(l[r + 2 * y], l[r + 2 * y + 1], a, b);
            h[y] = pack_pair<__half>(a, b);
          }
          *reinterpret_cast<uint4*>(dst + (r >> 3) * 128) = make_uint4(h[0], h[1], h[2], h[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::P_FULL + vb.at));
        started = true;
        last = vb.at;
        last_phase = vb.phase;
      }
      sb.next();
      vb.next();
      if (rare(w.left == 1 || i + 1 == n_tiles)) {
        // ---- end of the item, or of this CTA's part of it: the sets of these rows together
        const int kvh = w.u / p.row_tiles, row0 = (w.u - kvh * p.row_tiles) * R + c0;
        const bool whole = part_first == 0 && w.left == 1;
        const float sum = warp_sums(l, lane);
        if (lane < N) warps[quarter * R + lane] = sum;
        if (!started && key < N) ref[key] = INFINITY;
        if (started) wait(C::PV_DONE + last, last_phase);
        bar_sync(id_all, 128 * C::kSets);
        const int n = drafted(p, w.b);
        const long long out0 = ((long long)w.b * p.H + (long long)kvh * p.group) * p.T;
        const int slot = 2 * (int)blockIdx.x + (part_first == 0);
        if (set == 0 && key < N) {
          float m[C::kSets], part[C::kSets], f[C::kSets], top = -INFINITY, total_l = 0.f;
#pragma unroll
          for (int k = 0; k < C::kSets; ++k) {
            const float* const wk = warps_all + k * 4 * R + key;
            part[k] = wk[0] + wk[R] + wk[2 * R] + wk[3 * R];
            m[k] = kShift - ref_all[k * 2 * R + key];
            top = fmaxf(top, m[k]);
          }
#pragma unroll
          for (int k = 0; k < C::kSets; ++k) {
            f[k] = m[k] == top ? 1.f : exp2_approx(m[k] - top);     // (both -infinity: nothing seen)
            if (m[k] == -INFINITY && part[k] == 0.f) f[k] = 0.f;    // no tile, or nothing seen in them: what its O holds does not count
            total_l += f[k] * part[k];
          }
          const int row = row0 + key;
          float inv = 1.f;
          if (whole) {
            inv = total_l == 0.f ? 0.f : __fdiv_rn(1.f, total_l * load(p.cache.v_G + kvh));     // nothing seen: 0, not 0 / 0
            if (p.lse && row < p.rows && row % p.T < n)
              p.lse[out0 + row] = total_l == 0.f ? -INFINITY : (top - kShift + log2f(total_l)) * 0.6931471805599453f;
          } else {
            p.part_ml[(size_t)slot * R + c0 + key] = make_float2(top, total_l);
          }
#pragma unroll
          for (int k = 0; k < C::kSets; ++k) factor_all[k * R + key] = f[k] * inv;
        }
        if (group == 0 && key == 0 && part_first == 0)
          p.split[(size_t)w.b * units + w.u] = whole ? make_int2(-1, -1) : make_int2(blockIdx.x, cta_of(find[2] + i + w.left - 1, find[3], find[4]));
        bar_sync(id_all, 128 * C::kSets);
        tc_fence_after();
        // a set takes its share of the rows
        constexpr int M = N / C::kSets;
        const int r0 = set * M;
        float o[M];
        uint32_t v[C::kSets][M];
#pragma unroll
        for (int k = 0; k < C::kSets; ++k) {
          const uint32_t from = tmem + lanes + C::kO + k * R + c0 + r0;
          tmem_ld_cols(from, v[k]);
        }
        tmem_wait_ld();
#pragma unroll
        for (int r = 0; r < M; ++r) {
          o[r] = 0.f;
#pragma unroll
          for (int k = 0; k < C::kSets; ++k) {
            const float f = factor_all[k * R + r0 + r];
            o[r] += f == 0.f ? 0.f : __uint_as_float(v[k][r]) * f;
          }
        }
        tc_fence_before();
        if (C::kSets > 1) bar_sync(id_all, 128 * C::kSets);         // the next item's products may overwrite either O
        const uint32_t keep = __ballot_sync(0xffffffffu, lane < M && row0 + r0 + lane < p.rows && (row0 + r0 + lane) % p.T < n);
        if (key < D) {
          if (whole) {
            uint16_t* const dst = static_cast<uint16_t*>(p.out) + (size_t)(out0 + row0 + r0) * D + key;
#pragma unroll
            for (int r = 0; r < M; ++r) {
              const uint16_t h = p.half ? __half_as_ushort(__float2half_rn(o[r])) : __bfloat16_as_ushort(__float2bfloat16_rn(o[r]));
              if (keep >> r & 1) dst[r * D] = h;
            }
          } else {
            float* const dst = p.part + ((size_t)slot * R + c0 + r0) * D + key;
#pragma unroll
            for (int r = 0; r < M; ++r) dst[r * D] = o[r];
          }
        }
        fresh = true;
        ++item;
      }
      advance(w, p, units);
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

// ---------------------------------------------------------------- few rows: a warp by itself
// What should bound few rows is the reading; with the roles of the kernel above a tile costs more instructions for handing it from role to
// role than for its keys (4100 a tile of 128 keys, d = 128, half of them hand-overs; 32 sequences of up to 32768 tokens, 4 rows: 200 us, whose
// reading takes 94).  Here nothing is handed over (2700 a tile, 152 us; one token over 1000 keys 10 us instead of 11.7): a warp takes 32 keys
// of a tile from their codes to its own maximum, sum and O, all in registers, and the four warps of a CTA meet at the end of an item.  What bounds
// it is latency: four warps a scheduler do not cover the chain codes - convert - product - exp2 - transpose - product (issue 56 %, ALU 47 %, DRAM 41 %).
//
// The operands of the 16 x 8 x 16 products stay where they are loaded, because the orders of keys and of d are free:
//   S^T = K Q^T   A: keys x d, twice sixteen keys.  Lane (r, c) = (lane / 4, lane % 4) has keys r and r + 8: it takes D / 4 elements of either
//                 from d = c D / 4 on, in one piece; step j of the product over d is elements 4j .. 4j + 3 of each lane's piece.
//   O^T += V^T P^T  A: d x keys.  Lane (r, c) has tokens 8c .. 8c + 7, half a chunk of V; rows r and r + 8 of product t are elements 16t + 2r
//                 and 16t + 2r + 1, the two nibbles of a byte (sixteen elements are one block of scales).  NVFP4: step q has tokens
//                 8c + 2q + {0, 4 | 1, 5} (codes of tokens i and i + 4 meet in a byte, as their scales do), E4M3: 8c + 4q + {0, 1 | 2, 3}.
//                 B: P^T, which S^T leaves as keys x rows: 8 x 8 transposes.  So rows r and r + 8 of the q-th sixteen keys of S^T are those
//                 of the tokens that stand in columns r of the two halves of step q.
template <int FMT, int D, int NT>
struct WarpCfg {
  using L = RecordLayout<FMT, D>;
  static constexpr int kWarps = 4, kThreads = 32 * kWarps;
  static constexpr int R = 8 * NT;
  static constexpr int kStage = kTile * L::kToken;                 // K or V of a tile
  static constexpr int kCtas = kStage > 9216 ? 2 : NT == 2 ? 3 : 4;            // of an SM
  static constexpr int kStages = kStage > 9216 ? 6 : kStage > 8192 ? 5 : 6;
  static constexpr int kRow = D / 2;                               // floats of a row of half an O in shared memory (unpadded: it is full)
  static constexpr int kOffO = kStages * kStage;                   // float [4 warps][8 rows][kRow]
  static constexpr int kOffML = kOffO + kWarps * 8 * kRow * 4;     // float2 [4 warps][8 rows]
  static constexpr int kOffScale = kOffML + kWarps * 8 * 8;        // f16 [4 warps][D / 16][32 tokens]
  static constexpr int kOffValid = kOffScale + kWarps * (D / 16) * 64;
  static constexpr int kOffScan = kOffValid + 4 * 8;               // (room for kStages words)
  static_assert(kStages <= 8, "valid");
  static constexpr int kOffFind = kOffScan + 128;
  static constexpr int kOffBar = kOffFind + 64;
  static constexpr int kSmem = kOffBar + 2 * 8 * kStages + 16 + 128;
  static_assert(kCtas * (kSmem + 1024) <= 228 * 1024, "CTAs of an SM");
};
__device__ __forceinline__ void mma_16x8x16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// PAGED: rows see intervals of keys, and scores may be capped or biased (fp4attn_paged_attention)
template <int FMT, int D, int NT, bool PAGED>
__global__ void __launch_bounds__(WarpCfg<FMT, D, NT>::kThreads, WarpCfg<FMT, D, NT>::kCtas) tree_warp_kernel(const TreeParams p) {
  using C = WarpCfg<FMT, D, NT>;
  using L = typename C::L;
  constexpr int R = C::R, kSteps = D / 16;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (smem_u32(smem_raw) + 127u) & ~127u;
  uint8_t* const sgen = smem_raw + (sbase - smem_u32(smem_raw));
  const uint32_t full = sbase + C::kOffBar, free = full + 8 * C::kStages, abort_at = free + 8 * C::kStages;
  volatile uint32_t* const abort_word = reinterpret_cast<volatile uint32_t*>(sgen + C::kOffBar + 16 * C::kStages);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int units = p.cache.kv_heads * p.row_tiles;
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(free + 8 * s, C::kWarps);
    }
    *abort_word = 0;
    fence_barrier_init();
  }
  launch_dependents();                                              // the joining kernel: its launch lies under this one
  wait_prior_grids();
  Walk w0;
  long long* const find = reinterpret_cast<long long*>(sgen + C::kOffFind);
  const int n_tiles = find_run<C::kThreads, PAGED>(p, units, w0, reinterpret_cast<long long*>(sgen + C::kOffScan), find);
  uint32_t* const valid = reinterpret_cast<uint32_t*>(sgen + C::kOffValid);
  const int P = 1 << p.cache.log_page;

  // K and V of the first tiles; then the warps take turns, each bringing what takes the place of the K or V before the one they have just
  // been through (of that one the other warps may not be through yet).  A warp that fills a stage has itself been through what stood there
  // before: the stage's barrier cannot be further back than a wait by parity can tell.
  Pages<C::kStages, C::kStage, C::kStages, 2, true, PAGED> pages;
  pages.w = w0;
  const int n_parts = n_tiles > INT_MAX / 2 ? INT_MAX : 2 * n_tiles;
  if (warp == 0) {
    while (pages.i < C::kStages && pages.i < n_parts) {
      pages.find(p);
      if (rare(!pages.bring(p, sbase, full, free, abort_at, valid))) break;             // (they are free: no wait can have run out yet)
      pages.skip(p, units, 1);
    }
  } else if (C::kStages + warp < n_parts) {
    pages.skip(p, units, C::kStages + warp);
  } else {
    pages.i = n_parts;                                              // no turn
  }
  if (pages.i < n_parts) pages.find(p);
  auto next_pages = [&](int part) {                                 // this warp's turn?
    if (pages.i == part - 1 + C::kStages && pages.i < n_parts) {
      if (rare(!pages.bring(p, sbase, full, free, abort_at, valid)) || pages.i >= n_parts - C::kWarps) {
        pages.i = n_parts;
      } else {
        pages.skip(p, units, C::kWarps);
        pages.find(p);                                              // (the entries come until its next turn)
      }
    }
  };
  {
    const int r = lane >> 2, c = lane & 3;
    const int tok0 = 32 * warp;                                     // this warp's tokens of a tile
    // places in a stage of what the lane takes of them.  A sixteen of tokens is in one page, two may be in two.
    auto base_of = [&](int sixteen) {
      const int at = tok0 + 16 * sixteen;
      return (uint32_t)((at >> p.cache.log_page) * (p.cache.record / 2));
    };
    auto in_page = [&](int tok) { return (tok0 + tok) & (P - 1); };
    const int tok_k = 8 * (r >> 1) + (L::kFp4 ? 4 : 1) * (r & 1);   // token of row r of the first sixteen keys; row r + 8 and the second sixteen:
    constexpr int kSecondRow = L::kFp4 ? 1 : 2, kSecondStep = L::kFp4 ? 2 : 4;                   // so many further
    constexpr int kPiece = L::kRow / 4;                             // code bytes of a lane's piece of a key: 8, 16 or 32
    const uint32_t k_at = base_of(r >> 2) + (uint32_t)((c * kPiece / 16 * P + in_page(tok_k)) * 16 + c * kPiece % 16);
    const uint32_t ks_at = base_of(r >> 2) + (uint32_t)(L::k_scales(P) + in_page(tok_k) * L::kScales + c * (D / 64));
    const uint32_t v_at = base_of(c >> 1) + (uint32_t)(in_page(16 * (c >> 1)) * L::kRow + (L::kFp4 ? r : 2 * r) * 16 + 8 * (c & 1));
    uint8_t* const scales = sgen + C::kOffScale + warp * (D / 16) * 64;
    // scales of V that this lane converts: the eight tokens 8c .. of block lane / 4
    const uint32_t vs_at = base_of(c >> 1) + (uint32_t)(P * L::kRow + (lane >> 2) * P + in_page(8 * c));
    float* const o_smem = reinterpret_cast<float*>(sgen + C::kOffO);
    float2* const ml_smem = reinterpret_cast<float2*>(sgen + C::kOffML);

    const bool changed = PAGED && (p.cap > 0.f || p.slopes);
    Walk w = w0;
    Turn<C::kStages> ring;
    bool fresh = true;
    int part_first = 0, b_of = -1, n_drafted = 0, kvh = 0, row0 = 0;
    unsigned long long seen = 0;
    uint32_t qf[NT][kSteps][2];                                     // Q^T: rows 8n + lane / 4
    int from[NT][2], until[NT][2], at[NT][2], plain_from = 0, plain_until = 0;     // PAGED: keys that rows 8n + 2c, + 1 see, where they stand; that all rows see
    float slope[NT][2];
    const float cap_out = p.cap * 1.4426950408889634f, cap_inverse = PAGED && p.cap > 0.f ? __fdiv_rn(1.f, cap_out) : 0.f;
    float con[NT][2], ref[NT][2], l[NT][2];                         // of rows 8n + 2c, + 1: score constant, kShift minus the reference, sum
    float o[kSteps][NT][4];
#pragma unroll 1
    for (int i = 0; i < n_tiles; ++i) {
      if (rare(fresh)) {
        fresh = false;
        part_first = w.first;
        if (w.b != b_of) {
          b_of = w.b;
          n_drafted = drafted(p, w.b);
          if (!PAGED) {
            seen = row_mask(p, w.b, lane, n_drafted) | (lane + 32 < p.T ? row_mask(p, w.b, lane + 32, n_drafted) : 0ull);
            seen = (unsigned long long)__reduce_or_sync(0xffffffffu, (uint32_t)(seen >> 32)) << 32 | __reduce_or_sync(0xffffffffu, (uint32_t)seen);
          }
        }
        kvh = w.u / p.row_tiles;
        row0 = (w.u - kvh * p.row_tiles) * R;
        const float c0 = __fdiv_rn(p.scale * 1.4426950408889634f, load(p.cache.k_G + kvh));
        if (PAGED) {
          plain_from = 0;
          plain_until = INT_MAX;
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int row = row0 + 8 * n + 2 * c + y, hl = row / p.T, tok = row - hl * p.T;
              const bool is = row < p.rows && tok < n_drafted;
              from[n][y] = is && p.seen_from ? max(0, load(p.seen_from + (size_t)w.b * p.T + tok)) : 0;
              until[n][y] = !is ? INT_MAX : max(0, min(p.seen_until ? load(p.seen_until + (size_t)w.b * p.T + tok) : w.ctx + tok + 1, w.len));
              at[n][y] = w.ctx + tok;
              slope[n][y] = is && p.slopes ? load(p.slopes + kvh * p.group + hl) * 1.4426950408889634f : 0.f;
              plain_from = max(plain_from, from[n][y]);
              plain_until = min(plain_until, until[n][y]);
            }
          plain_from = __reduce_max_sync(0xffffffffu, plain_from);
          plain_until = __reduce_min_sync(0xffffffffu, plain_until);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          // Q scaled by a power of two per row, as above
          const int row = row0 + 8 * n + r;
          float v[D / 4];
          if (row < p.rows) {
            const int hl = row / p.T, tok = row - hl * p.T;
            const uint16_t* q = static_cast<const uint16_t*>(p.q) + w.b * p.q_sb + (long long)(kvh * p.group + hl) * p.q_sh + tok * p.q_sn + c * (D / 4);
#pragma unroll
            for (int x = 0; x < D / 4; x += 8) {
              uint32_t raw[4];
              if (p.q_vector) {
                *reinterpret_cast<uint4*>(raw) = load(reinterpret_cast<const uint4*>(q + x));
              } else {
#pragma unroll
                for (int y = 0; y < 4; ++y) raw[y] = (uint32_t)load(q + x + 2 * y) | (uint32_t)load(q + x + 2 * y + 1) << 16;
              }
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const float2 f = p.half ? unpack16<true>(raw[y]) : unpack16<false>(raw[y]);
                v[x + 2 * y] = f.x;
                v[x + 2 * y + 1] = f.y;
              }
            }
          } else {
#pragma unroll
            for (int x = 0; x < D / 4; ++x) v[x] = 0.f;
          }
          float a = 0.f;
#pragma unroll
          for (int x = 0; x < D / 4; ++x) a = fmaxf(a, fabsf(v[x]));
          a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
          a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
          const uint32_t up = row_exponent(a);
          const float f = __uint_as_float(up << 23), mine = c0 * __uint_as_float((254u - up) << 23);
#pragma unroll
          for (int x = 0; x < kSteps; ++x) {
            qf[n][x][0] = pack_pair<__half>(v[4 * x] * f, v[4 * x + 1] * f);
            qf[n][x][1] = pack_pair<__half>(v[4 * x + 2] * f, v[4 * x + 3] * f);
          }
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            con[n][y] = __shfl_sync(0xffffffffu, mine, (2 * c + y) * 4);
            if (PAGED && p.cap > 0.f) con[n][y] = cap_constant(con[n][y], cap_inverse);
            ref[n][y] = INFINITY;
            l[n][y] = 0.f;
          }
#pragma unroll
          for (int x = 0; x < kSteps; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) o[x][n][y] = 0.f;
        }
      }
      {
        wait_phase<true>(full + 8 * ring.at, ring.phase, abort_at);
        const uint8_t* stage = sgen + ring.at * C::kStage;
        const uint32_t held = valid[ring.at];
        const bool plain = (PAGED ? w.first >= plain_from && w.first + kTile <= plain_until : w.first + kTile <= w.ctx) &&
                           held == (1u << (kTile >> p.cache.log_page)) - 1;
        const bool v_here = held >> ((tok0 + 8 * c) >> p.cache.log_page) & 1;
        uint32_t v_mask = 0xFFu;                                    // of tokens 8c .., those that count
        if (!PAGED && rare(!plain)) v_mask = v_here ? valid_eight(w, seen, w.first + tok0 + 8 * c) : 0u;
        // ---- scores
        float s[NT][8];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int y = 0; y < 8; ++y) s[n][y] = 0.f;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t h[2][2 * kSteps];                                // f16 pairs of the two keys
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int on = kSecondStep * q + kSecondRow * k;
            const uint8_t* const at = stage + k_at + 16 * on;
            if (L::kFp4) {
              uint32_t words[D / 32], f[2];
              if (D == 128) *reinterpret_cast<uint4*>(words) = *reinterpret_cast<const uint4*>(at);
              else *reinterpret_cast<uint2*>(words) = *reinterpret_cast<const uint2*>(at);
              const uint8_t* const sat = stage + ks_at + L::kScales * on;
              const uint32_t two = cvt_f16x2_e4m3x2(D == 128 ? *reinterpret_cast<const uint16_t*>(sat) : *sat);
              f[0] = splat_half(two, 0);
              f[1] = splat_half(two, 1);
#pragma unroll
              for (int x = 0; x < D / 32; ++x) {
                cvt_f16x2_e2m1x8(words[x], h[k] + 4 * x);
#pragma unroll
                for (int y = 0; y < 4; ++y) h[k][4 * x + y] = mul_half2(h[k][4 * x + y], f[D == 128 ? x >> 1 : 0]);
              }
            } else {
#pragma unroll
              for (int x = 0; x < D / 64; ++x) {
                const uint4 raw = *reinterpret_cast<const uint4*>(at + x * P * 16);
                const uint32_t words[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                for (int y = 0; y < 4; ++y) cvt_f16x2_e4m3x4(words[y], h[k] + 8 * x + 2 * y);
              }
            }
          }
#pragma unroll
          for (int x = 0; x < kSteps; ++x)
#pragma unroll
            for (int n = 0; n < NT; ++n)
              mma_16x8x16(s[n] + 4 * q, h[0][2 * x], h[1][2 * x], h[0][2 * x + 1], h[1][2 * x + 1], qf[n][x][0], qf[n][x][1]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(free + 8 * ring.at);
        ring.next();
        next_pages(2 * i);
        // ---- probabilities: octaves above the rows' references (+ kShift); what is not seen goes to -infinity
        float x[NT][8], top = -INFINITY;
        uint32_t hidden = 0;                                        // bit 8n + y: s[n][y] is not seen
        if (PAGED) {
          if (rare(!plain)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int y = 0; y < 8; ++y) {
                const int tok = tok_k + kSecondStep * (y >> 2) + kSecondRow * (y >> 1 & 1), pos = w.first + tok0 + tok;
                const bool here = held >> ((tok0 + tok) >> p.cache.log_page) & 1;
                hidden |= (here && pos >= from[n][y & 1] && pos < until[n][y & 1] ? 0u : 1u) << (8 * n + y);
              }
          }
          if (changed) {                            // scores in octaves, changed; their constants are spent
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int y = 0; y < 8; ++y) s[n][y] *= con[n][y & 1];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              if (p.cap > 0.f) {
                cap_scores(x[n], s[n], cap_out);
#pragma unroll
                for (int y = 0; y < 8; ++y) s[n][y] = x[n][y];
              }
#pragma unroll
              for (int y = 0; y < 8; ++y) {
                const int tok = tok_k + kSecondStep * (y >> 2) + kSecondRow * (y >> 1 & 1), pos = w.first + tok0 + tok;
                s[n][y] = fmaf(-slope[n][y & 1], fabsf((float)(at[n][y & 1] - pos)), s[n][y]);
              }
            }
          }
        } else if (rare(!plain)) {
#pragma unroll 1
          for (int n = 0; n < NT; ++n) {
            unsigned long long mask[2];                             // drafted tokens that the rows see
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int row = row0 + 8 * n + 2 * c + y;
              mask[y] = row < p.rows ? row_mask(p, w.b, row % p.T, n_drafted) : 0ull;
            }
#pragma unroll
            for (int y = 0; y < 8; y += 2) {
              const int tok = tok_k + kSecondStep * (y >> 2) + kSecondRow * (y >> 1 & 1), pos = w.first + tok0 + tok, in = pos - w.ctx;
              const bool here = (held >> ((tok0 + tok) >> p.cache.log_page) & 1) && pos < w.len;
              const uint32_t m0 = in < 0 ? 1u : (uint32_t)(mask[0] >> (in & 63)) & 1u, m1 = in < 0 ? 1u : (uint32_t)(mask[1] >> (in & 63)) & 1u;
              hidden |= (here ? (m0 | m1 << 1) ^ 3u : 3u) << (8 * n + y);
            }
          }
        }
        auto relative = [&] {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int y = 0; y < 8; ++y) x[n][y] = fmaf(s[n][y], PAGED && changed ? 1.f : con[n][y & 1], ref[n][y & 1]);
          if (rare(hidden != 0)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int y = 0; y < 8; ++y)
                if (hidden >> (8 * n + y) & 1) x[n][y] = -INFINITY;
          }
        };
        relative();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int y = 0; y < 8; y += 2) top = max3(top, x[n][y], x[n][y + 1]);
        if (rare(__any_sync(0xffffffffu, top > kLag + kShift))) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float m = -INFINITY;                                  // the largest seen; max leaves NaN out
#pragma unroll
              for (int z = 0; z < 8; z += 2)
                if (!(hidden >> (8 * n + y + z) & 1)) m = fmaxf(m, s[n][y + z] * (PAGED && changed ? 1.f : con[n][y]));
              for (int z = 4; z < 32; z <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, z));
              const float old = kShift - ref[n][y];                 // -infinity: none yet
              m = fmaxf(m, old);
              const float f = m == -INFINITY ? 1.f : exp2_approx(old - m);
              ref[n][y] = kShift - m;
              l[n][y] *= f;
#pragma unroll
              for (int z = 0; z < kSteps; ++z) {
                o[z][n][y] *= f;
                o[z][n][y + 2] *= f;
              }
            }
          relative();
        }
        uint32_t pb[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float a = exp2_approx(x[n][2 * y]), b = exp2_approx(x[n][2 * y + 1]);
            add_pair(l[n][0], l[n][1], a, b);
            pb[n][y] = transpose_8x8(pack_pair<__half>(a, b));
          }
        wait_phase<true>(full + 8 * ring.at, ring.phase, abort_at);
        stage = sgen + ring.at * C::kStage;
        // ---- scales of V: f16, by block and token
        if (L::kFp4 && lane < D / 4) {
          uint2 sc = *reinterpret_cast<const uint2*>(stage + vs_at);
          if (!PAGED && rare(!plain)) {
            const uint32_t v = permute_eight(v_mask);
            sc.x &= byte_mask(v);
            sc.y &= byte_mask(v >> 4);
          }
          uint32_t f[4];
          cvt_f16x2_e4m3x4(sc.x, f);
          cvt_f16x2_e4m3x4(sc.y, f + 2);
          if (PAGED) {
#pragma unroll
            for (int y = 0; y < 4; ++y) f[y] = finite(f[y]);        // (what nobody sees has a probability of 0)
          }
          *reinterpret_cast<uint4*>(scales + lane * 16) = make_uint4(f[0], f[1], f[2], f[3]);
        }
        __syncwarp();
        // ---- O
#pragma unroll
        for (int z = 0; z < kSteps; ++z) {
          uint32_t even[4], odd[4];                                 // elements 16z + 2r and 16z + 2r + 1, pairs of tokens
          if (L::kFp4) {
            const uint2 raw = *reinterpret_cast<const uint2*>(stage + v_at + z * 128);
            const uint4 f = *reinterpret_cast<const uint4*>(scales + z * 64 + 16 * c);
            cvt_f16x2_e2m1x8((raw.x & 0x0F0F0F0Fu) | (raw.y << 4 & 0xF0F0F0F0u), even);
            cvt_f16x2_e2m1x8((raw.x >> 4 & 0x0F0F0F0Fu) | (raw.y & 0xF0F0F0F0u), odd);
            const uint32_t g[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              even[y] = mul_half2(even[y], g[y]);
              odd[y] = mul_half2(odd[y], g[y]);
            }
          } else {
            uint2 e = *reinterpret_cast<const uint2*>(stage + v_at + z * 256), d = *reinterpret_cast<const uint2*>(stage + v_at + z * 256 + 16);
            if (!PAGED && rare(!plain)) {
              const uint32_t lo = byte_mask(v_mask), hi = byte_mask(v_mask >> 4);
              e.x &= lo; e.y &= hi; d.x &= lo; d.y &= hi;
            }
            cvt_f16x2_e4m3x4(e.x, even);
            cvt_f16x2_e4m3x4(e.y, even + 2);
            cvt_f16x2_e4m3x4(d.x, odd);
            cvt_f16x2_e4m3x4(d.y, odd + 2);
            if (PAGED && rare(!plain)) {
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                even[y] = finite(even[y]);
                odd[y] = finite(odd[y]);
              }
            }
          }
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_16x8x16(o[z][n], even[2 * q], odd[2 * q], even[2 * q + 1], odd[2 * q + 1], pb[n][2 * q], pb[n][2 * q + 1]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(free + 8 * ring.at);
        ring.next();
        next_pages(2 * i + 1);
      }
      // ---- end of the item, or of this CTA's part of it: the warps together
      if (rare(w.left == 1 || i + 1 == n_tiles)) {
        const bool begins = part_first == (PAGED ? w.begin : 0), whole = begins && w.left == 1;
        const long long out0 = ((long long)w.b * p.H + (long long)kvh * p.group) * p.T;
        const int slot_of = 2 * (int)blockIdx.x + begins;
#pragma unroll
        for (int n = 0; n < NT; ++n)                                // eight rows and half the elements at a time
#pragma unroll
          for (int z0 = 0; z0 < kSteps; z0 += kSteps / 2) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int row = 2 * c + y;
              if (z0 == 0) {
                float sum = l[n][y];
                for (int z = 4; z < 32; z <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, z);
                if (lane < 4) ml_smem[warp * 8 + row] = make_float2(kShift - ref[n][y], sum);
              }
              float* const dst = o_smem + (warp * 8 + row) * C::kRow + 2 * r;
#pragma unroll
              for (int z = 0; z < kSteps / 2; ++z) *reinterpret_cast<float2*>(dst + 16 * z) = make_float2(o[z0 + z][n][y], o[z0 + z][n][y + 2]);
            }
            __syncthreads();
            // a thread per row and four elements
#pragma unroll 1
            for (int j = threadIdx.x; j < min(8, p.rows - row0 - 8 * n) * (D / 8); j += C::kThreads) {
              const int row8 = j / (D / 8), in_tile = 8 * n + row8, row = row0 + in_tile, e8 = j % (D / 8) * 4, e = 16 * z0 + e8;
              float top_m = -INFINITY, total_l = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
              for (int k = 0; k < C::kWarps; ++k) top_m = fmaxf(top_m, ml_smem[k * 8 + row8].x);
              for (int k = 0; k < C::kWarps; ++k) {
                const float2 ml = ml_smem[k * 8 + row8];
                const float f = ml.x == top_m ? 1.f : exp2_approx(ml.x - top_m);
                const float4 v = *reinterpret_cast<const float4*>(o_smem + (k * 8 + row8) * C::kRow + e8);
                total_l += f * ml.y;
                y[0] = fmaf(f, v.x, y[0]); y[1] = fmaf(f, v.y, y[1]); y[2] = fmaf(f, v.z, y[2]); y[3] = fmaf(f, v.w, y[3]);
              }
              if (whole) {
                if (row % p.T < n_drafted) {
                  const float inv = total_l == 0.f ? 0.f : __fdiv_rn(1.f, total_l * load(p.cache.v_G + kvh));     // nothing seen: 0
                  const uint2 h = p.half ? make_uint2(pack_pair<__half>(y[0] * inv, y[1] * inv), pack_pair<__half>(y[2] * inv, y[3] * inv))
                                         : make_uint2(pack_pair<__nv_bfloat16>(y[0] * inv, y[1] * inv), pack_pair<__nv_bfloat16>(y[2] * inv, y[3] * inv));
                  *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + (size_t)(out0 + row) * D + e) = h;
                  if (e == 0 && p.lse) p.lse[out0 + row] = total_l == 0.f ? -INFINITY : (top_m - kShift + log2f(total_l)) * 0.6931471805599453f;
                }
              } else {
                *reinterpret_cast<float4*>(p.part + ((size_t)slot_of * R + in_tile) * D + e) = make_float4(y[0], y[1], y[2], y[3]);
                if (e == 0) p.part_ml[(size_t)slot_of * R + in_tile] = make_float2(top_m, total_l);
              }
            }
            __syncthreads();
          }
        if (threadIdx.x == 0 && begins)
          p.split[(size_t)w.b * units + w.u] =
              whole ? make_int2(-1, -1) : make_int2(blockIdx.x, cta_of(find[2] + i + w.left - 1, find[3], find[4]));
        fresh = true;
      }
      advance<PAGED>(w, p, units);
    }
    pages.tell(p);
  }
  __syncthreads();
  if (rare(*abort_word != 0)) {                                     // given up: the copies in flight end before shared memory does
    if (threadIdx.x == 0 && p.status) *p.status = FP4ATTN_ERR_TIMEOUT;
    if (threadIdx.x < 2 * C::kStages)
      for (int spin = 0; spin < (1 << 10) && !mbar_try_wait(full + 8 * (threadIdx.x >> 1), threadIdx.x & 1); ++spin) {}
    __syncthreads();
  }
}

// Joins the parts of the items that fell to several CTAs, in the order of their keys; a warp per row.
template <int D, int R>
__global__ void __launch_bounds__(128) tree_join_kernel(const TreeParams p) {
  wait_prior_grids();
  const int units = p.cache.kv_heads * p.row_tiles;
  const int item = blockIdx.x, b = item / units, u = item - b * units, kvh = u / p.row_tiles, lane = threadIdx.x & 31;
  const int r = blockIdx.y * 4 + (threadIdx.x >> 5), row = (u - kvh * p.row_tiles) * R + r;
  if (r >= R || row >= p.rows || row % p.T >= drafted(p, b)) return;
  const int2 ctas = p.split[item];
  if (ctas.x < 0 || ctas.y < ctas.x || ctas.y >= kMostCtas<R>) return;   // whole (or a kernel that gave up)
  const int n = ctas.y - ctas.x + 1;
  auto slot = [&](int i) { return (size_t)(i ? 2 * (ctas.x + i) : 2 * ctas.x + 1); };
  float m = -INFINITY;
  for (int i = lane; i < n; i += 32) m = fmaxf(m, p.part_ml[slot(i) * R + r].x);
  m = warp_max(m);
  constexpr int E = D / 32;
  float o[E] = {}, l = 0.f;
  for (int i0 = 0; i0 < n; i0 += 32) {
    const int i = i0 + lane;
    const float2 ml = i < n ? p.part_ml[slot(i) * R + r] : make_float2(-INFINITY, 0.f);
    const float mine = m == -INFINITY || i >= n ? 0.f : exp2_approx(ml.x - m);
    const float weighted = ml.x == -INFINITY ? ml.y : mine * ml.y;
    constexpr int kAtOnce = 8;                                      // loads on their way together
    for (int k0 = 0; k0 < min(32, n - i0); k0 += kAtOnce) {
      float part[kAtOnce][E];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const bool is = i0 + k0 + k < n;
        const float* const src = p.part + (slot(is ? i0 + k0 + k : 0) * R + r) * D + lane * E;
        if constexpr (E == 4) *reinterpret_cast<float4*>(part[k]) = is ? *reinterpret_cast<const float4*>(src) : make_float4(0.f, 0.f, 0.f, 0.f);
        else *reinterpret_cast<float2*>(part[k]) = is ? *reinterpret_cast<const float2*>(src) : make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {                           // (behind the last part: weights and parts of 0)
        const float f = __shfl_sync(0xffffffffu, mine, k0 + k);
        l += __shfl_sync(0xffffffffu, weighted, k0 + k);
#pragma unroll
        for (int x = 0; x < E; ++x) o[x] = fmaf(f, part[k][x], o[x]);
      }
    }
  }
  const float f = l == 0.f ? 0.f : __fdiv_rn(1.f, l * load(p.cache.v_G + kvh));
  const size_t at = ((size_t)b * p.H + (size_t)kvh * p.group) * p.T + row;
#pragma unroll
  for (int x = 0; x < E; x += 2) {
    const uint32_t two = p.half ? pack_pair<__half>(o[x] * f, o[x + 1] * f) : pack_pair<__nv_bfloat16>(o[x] * f, o[x + 1] * f);
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + at * D + lane * E + x) = two;
  }
  if (lane == 0 && p.lse) p.lse[at] = l == 0.f ? -INFINITY : (m - kShift + log2f(l)) * 0.6931471805599453f;
}

// ---- workspace: partial O, their references and sums, what is split
// Few rows by warps (tiles of 8 or 16), more by roles (32 or 64).  By warps | by roles, us:
//   4 rows, NVFP4, d = 128, 32 sequences x up to 32768 tokens: 152 | 200
//   16 rows, 8 KV heads      1 x 1000      1 x 16000     8 x 4096      32 x 32000 (up to; 12 rows alike)
//     NVFP4, d = 64       10.8 | 11.1   26.4 | 26.9   21.7 | 27.9    169 | 260
//     E4M3, d = 64        11.0 | 11.1   26.5 | 26.1   21.4 | 29.3    158 | 273
//     E4M3, d = 128       12.3 | 12.1   24.7 | 25.3   28.0 | 31.0    263 | 294
//     NVFP4, d = 128      14.6 | 12.2   40.9 | 25.0   37.3 | 30.0    358 | 290    two groups of eight rows are more than its registers hold
//   32 rows, d = 128: 1 x 1000 18 | 13, 8 x 4096 41 | 24; 64 rows 22 | 16, 81 | 42; 256 rows 39 | 26, 265 | 114; E4M3 alike (d = 64: 1.1 to 1.3 times)
int rows_of_tile(int rows, int fmt, int d) {
  if (rows <= 8) return 8;
  if (rows <= 16 && !(fmt == FP4ATTN_FMT_NVFP4 && d == 128)) return 16;
  return rows <= 32 ? 32 : 64;
}
struct TreePlan {
  int R, row_tiles;
  size_t ml, split, total;
};
TreePlan plan(int B, int H, int kv_heads, int T, int d, int fmt) {
  TreePlan t;
  const int rows = H / kv_heads * T;
  t.R = rows_of_tile(rows, fmt, d);
  t.row_tiles = (rows + t.R - 1) / t.R;
  const size_t slots = 2 * (t.R <= 16 ? kMostWarpCtas : kMostRoleCtas);        // of the kernel that will run (launch_rows)
  t.ml = slots * t.R * d * 4;
  t.split = t.ml + slots * t.R * 8;
  t.total = t.split + (((size_t)B * kv_heads * t.row_tiles * 8 + 15) & ~(size_t)15);
  return t;
}

template <int FMT, int D, int R>
int launch_tree(const TreeParams& p, cudaStream_t st) {
  using C = TreeCfg<FMT, D, R>;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return FP4ATTN_ERR_CUDA;
  static std::atomic<bool> attr_set[kMaxDevices];
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(tree_kernel<FMT, D, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) != cudaSuccess) return FP4ATTN_ERR_CUDA;
    attr_set[dev].store(true, std::memory_order_release);
  }
  const int sms = device_sms();
  if (!sms) return FP4ATTN_ERR_CUDA;
  const int units = p.cache.kv_heads * p.row_tiles;
  const long long most_tiles = (((long long)p.cache.max_pages << p.cache.log_page) + kTile - 1) / kTile * p.B * units;
  const unsigned grid = (unsigned)std::min<long long>(std::min(sms, kMostCtas<R>), most_tiles);
  cudaError_t e = launch_overlapped(tree_kernel<FMT, D, R>, dim3(grid), C::kThreads, C::kSmem, st, p);
  if (e == cudaSuccess)
    e = launch_overlapped(tree_join_kernel<D, R>, dim3((unsigned)(p.B * units), (unsigned)(std::min(R, p.rows) + 3) / 4), 128u, 0, st, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
}
template <int FMT, int D, int NT, bool PAGED = false>
int launch_warps(const TreeParams& p, cudaStream_t st) {
  using C = WarpCfg<FMT, D, NT>;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return FP4ATTN_ERR_CUDA;
  static std::atomic<bool> attr_set[kMaxDevices];
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(tree_warp_kernel<FMT, D, NT, PAGED>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) != cudaSuccess) return FP4ATTN_ERR_CUDA;
    attr_set[dev].store(true, std::memory_order_release);
  }
  const int sms = device_sms();
  if (!sms) return FP4ATTN_ERR_CUDA;
  const long long most_tiles = (((long long)p.cache.max_pages << p.cache.log_page) + kTile - 1) / kTile * p.B * p.cache.kv_heads * p.row_tiles;
  const unsigned grid = (unsigned)std::min<long long>(std::min(C::kCtas * sms, kMostCtas<C::R>), most_tiles);
  cudaError_t e = launch_overlapped(tree_warp_kernel<FMT, D, NT, PAGED>, dim3(grid), C::kThreads, C::kSmem, st, p);
  if (e == cudaSuccess)
    e = launch_overlapped(tree_join_kernel<D, C::R>, dim3((unsigned)(p.B * p.cache.kv_heads * p.row_tiles), (unsigned)(std::min(p.rows, C::R) + 3) / 4), 128u, 0,
                          st, p);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? FP4ATTN_OK : FP4ATTN_ERR_CUDA;
}
template <int FMT, int D>
int launch_rows(const TreeParams& p, int R, cudaStream_t st) {
  if (R == 8) return launch_warps<FMT, D, 1>(p, st);
  if constexpr (!(FMT == FP4ATTN_FMT_NVFP4 && D == 128))
    if (R == 16) return launch_warps<FMT, D, 2>(p, st);
  return R == 32 ? launch_tree<FMT, D, 32>(p, st) : launch_tree<FMT, D, 64>(p, st);
}

template <int FMT, int D>
int launch_few(const TreeParams& p, int R, bool changed, cudaStream_t st) {
  if (R == 8) return changed ? launch_warps<FMT, D, 1, true>(p, st) : launch_warps<FMT, D, 1>(p, st);
  if constexpr (!(FMT == FP4ATTN_FMT_NVFP4 && D == 128))
    if (R == 16) return changed ? launch_warps<FMT, D, 2, true>(p, st) : launch_warps<FMT, D, 2>(p, st);
  return R == 32 && !changed ? launch_tree<FMT, D, 32>(p, st) : FP4ATTN_ERR_UNSUPPORTED_SHAPE;      // (not few)
}

}  // namespace

// The warps take up to 16 rows whatever the masks (8 where rows_of_tile says so); the roles, which know no masks, caps or biases, up to 32.  The roles of 32 or 64 rows
// against 128 rows in lanes (paged_attn.cu), without any, 8 KV heads, us:
//                       1 x 1000       8 x 4096       16 x 16000
//   32 rows
//     NVFP4, d = 128   13.5 | 22.4    35.2 | 43.8     123 | 151
//     E4M3,  d = 128   13.6 | 22.1    35.5 | 44.3     122 | 208
//     NVFP4, d = 64    12.3 | 17.4    32.3 | 33.9     112 | 121       (E4M3 alike)
//   64 rows
//     NVFP4, d = 128   15.4 | 22.3    44.0 | 45.2     196 | 159
//     E4M3,  d = 128   16.2 | 22.6    45.3 | 46.6     189 | 211
//     NVFP4, d = 64    12.6 | 17.4    36.9 | 35.3     178 | 136
//     E4M3,  d = 64    13.5 | 17.3    38.2 | 35.0     179 | 133
// One limit for every format and length: with 64 rows the lanes win where much is read in three of the four formats, by a fifth to a quarter, and lose 4 to 7 us on
// short calls and a tenth in E4M3 with d = 128.  32 rows with a mask, cap or bias take the lanes for want of roles that know them: 24, 45 and 152 us (E4M3: 218).
bool few_rows(int rows, int fmt, int d, bool changed) { return rows_of_tile(rows, fmt, d) <= (changed ? 16 : 32); }
size_t few_rows_workspace(int B, int H, int kv_heads, int T, int d, int fmt) { return plan(B, H, kv_heads, T, d, fmt).total; }
int launch_few_rows(const FewRows& a, void* workspace, cudaStream_t st) {
  const TreePlan t = plan(a.B, a.H, a.cache.kv_heads, a.T, a.d, a.fmt);
  TreeParams p = {};
  p.q = a.q->data; p.q_sb = a.q->stride_b; p.q_sh = a.q->stride_h; p.q_sn = a.q->stride_n;
  p.q_vector = view_vectors(*a.q, 2);
  p.half = a.type == FP4ATTN_TYPE_FP16;
  p.cache = a.cache;
  p.context = a.context; p.count = a.count;
  p.out = a.out; p.lse = a.lse; p.status = a.status;
  p.B = a.B; p.H = a.H; p.T = a.T; p.group = a.H / a.cache.kv_heads;
  p.rows = p.group * a.T;
  p.row_tiles = t.row_tiles;
  p.scale = a.scale;
  p.seen_from = a.first; p.seen_until = a.last; p.slopes = a.slopes; p.cap = a.cap;
  p.part = (float*)workspace;
  p.part_ml = (float2*)((char*)workspace + t.ml);
  p.split = (int2*)((char*)workspace + t.split);
  const bool changed = a.changed();
  if (a.fmt == FP4ATTN_FMT_NVFP4) return a.d == 64 ? launch_few<FP4ATTN_FMT_NVFP4, 64>(p, t.R, changed, st) : launch_few<FP4ATTN_FMT_NVFP4, 128>(p, t.R, changed, st);
  return a.d == 64 ? launch_few<FP4ATTN_FMT_E4M3, 64>(p, t.R, changed, st) : launch_few<FP4ATTN_FMT_E4M3, 128>(p, t.R, changed, st);
}
}  // namespace fp4attn

using namespace fp4attn;

extern "C" size_t fp4attn_tree_attention_workspace_bytes(int B, int H, int kv_heads, int T, int d) {
  if (B <= 0 || H <= 0 || kv_heads <= 0 || H % kv_heads != 0 || T <= 0 || T > FP4ATTN_MOST_TREE_TOKENS || (d != 64 && d != 128)) return 0;
  if ((long long)B * H * T >= (1ll << 31)) return 0;
  return std::max(plan(B, H, kv_heads, T, d, FP4ATTN_FMT_NVFP4).total, plan(B, H, kv_heads, T, d, FP4ATTN_FMT_E4M3).total);
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
  if (T > FP4ATTN_MOST_TREE_TOKENS || (long long)B * H * T >= (1ll << 31)) return FP4ATTN_ERR_UNSUPPORTED_SHAPE;     // (items are no more)
  if (((uintptr_t)q->data & 1) || ((uintptr_t)O & 15) || ((uintptr_t)tree_mask & 7) || ((uintptr_t)LSE | (uintptr_t)device_status) & 3)
    return FP4ATTN_ERR_ALIGNMENT;
  const TreePlan t = plan(B, H, cache->kv_heads, T, cache->d, cache->fmt);
  if (!workspace || workspace_bytes < fp4attn_tree_attention_workspace_bytes(B, H, cache->kv_heads, T, cache->d)) return FP4ATTN_ERR_WORKSPACE;
  if ((uintptr_t)workspace & 15) return FP4ATTN_ERR_ALIGNMENT;
  if ((rc = check_device_sm100()) != FP4ATTN_OK) return rc;
  TreeParams p = {};
  p.q = q->data; p.q_sb = q->stride_b; p.q_sh = q->stride_h; p.q_sn = q->stride_n;
  p.q_vector = view_vectors(*q, 2);
  p.half = type == FP4ATTN_TYPE_FP16;
  p.cache = ref;
  p.context = context; p.count = count; p.mask = tree_mask;
  p.out = O; p.lse = LSE; p.status = device_status;
  p.B = B; p.H = H; p.T = T; p.group = H / cache->kv_heads;
  p.rows = p.group * T;
  p.row_tiles = t.row_tiles;
  p.scale = softmax_scale > 0.f ? softmax_scale : (float)(1.0 / sqrt((double)cache->d));
  p.part = (float*)workspace;
  p.part_ml = (float2*)((char*)workspace + t.ml);
  p.split = (int2*)((char*)workspace + t.split);
  cudaStream_t st = (cudaStream_t)stream;
  if (cache->fmt == FP4ATTN_FMT_NVFP4)
    return cache->d == 64 ? launch_rows<FP4ATTN_FMT_NVFP4, 64>(p, t.R, st) : launch_rows<FP4ATTN_FMT_NVFP4, 128>(p, t.R, st);
  return cache->d == 64 ? launch_rows<FP4ATTN_FMT_E4M3, 64>(p, t.R, st) : launch_rows<FP4ATTN_FMT_E4M3, 128>(p, t.R, st);
}
