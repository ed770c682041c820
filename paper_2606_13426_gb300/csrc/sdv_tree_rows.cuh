// sdv_tree_rows.cuh - the tree attention for many rows, on the fifth-generation matrix unit.
//
// A CTA takes up to 128 rows (nodes times the query heads of a key head) through the keys in steps of whole pages, up to 128
// keys:
//   S = Q K' (tensor memory, fp32), P = 2^(S f - m) vs, O += P V.
// A row is a lane of tensor memory and a thread of a softmax warp, so that its maximum and sum need no exchange; a page's
// scales are one number for 16 keys or more.  Three kinds of warps work at once:
//   * one warp plans: which part of which item comes next, and what its nodes see of the tree;
//   * one warp copies: a step's pages of codes, in bulk, into rings of steps of keys and of values;
//   * loading warps widen them to f16 (exactly; a value's NaN becomes 0 and is told apart), the matrix unit's operands;
//   * two warps issue the products, scores and output, each as soon as it can;
//   * two groups of softmax warps take a half of each step's keys, each with references and sums of its own, joined
//     at the end of a segment.  The scores of the next step are had meanwhile, in the other half of their memory.
// Queries go through f16: bf16 ones under a power of two of their row.  Probabilities times their value's scale
// stand in tensor memory in place of their scores, as the sum of two f16: 22 bits, or 2^-32 of the row's largest.  So that they
// fit f16 whatever the scales of other pages, a row's reference m is taken on the score plus log2 of that scale;
// the sum of 2^(S f - m) is had from the same exponentials, in fp32.
//
// The steps of all (sequence, head) items, laid end to end, are cut into equal runs, one for each team of as many CTAs as
// an item has tiles of 128 rows: a team's CTAs read the same keys at about the same time, so that DRAM gives them once.
#pragma once

#include "sdv_attend.cuh"
#include "sdv_tcgen05.cuh"

namespace sdv {

constexpr int kTileRows = 128;
constexpr int kSoftWarps = 8, kLoadWarps = 8, kScoreWarp = kSoftWarps + kLoadWarps, kPlanWarp = kScoreWarp + 1, kCopyWarp = kScoreWarp + 2, kOutWarp = kScoreWarp + 3;
constexpr int kTreeThreads = 32 * (kScoreWarp + 4);
constexpr int kGroupWarps = kLoadWarps / 2, kGroupThreads = 32 * kGroupWarps;   // of the loading warps: keys, values
constexpr int kKStages = 1, kVStages = 2;          // of widened operands: keys are free again once the scores are had
constexpr int kRawK = 2, kRawV = 3;                // steps of codes under way
constexpr int kSegRing = 8, kScaleRing = 8;
constexpr int kTileChunks = kTileKeys / kChunk;
// Registers of a thread: softmax, loading, the others.  (96 at the launch.)
constexpr int kSoftRegs = 144, kLoadRegs = 72, kOtherRegs = 40;
static_assert(32 * (kSoftWarps * kSoftRegs + kLoadWarps * kLoadRegs + 4 * kOtherRegs) <= kTreeThreads * 96, "");
constexpr float kMostPlain = 0x1p20f;             // scores up to which a reference of one number serves
constexpr int kAside = 64;                        // steps whose products are summed in tensor memory (see put_aside)
constexpr int kMinTileSteps = 2;                  // of a run, where there are fewer steps than teams could take

// Steps [step0, step0 + steps) of an item; steps = 0: no more.
struct Segment {
  int b, h, step0, steps, len, count, whole, slot;
};

struct alignas(16) TreeSmall {
  uint64_t rk_full[kRawK], rk_free[kRawK], rv_full[kRawV], rv_free[kRawV];
  uint64_t k_full[kKStages], k_free[kKStages], v_full[kVStages], v_free[kVStages];
  uint64_t s_full[2], p_full[2][2], p_free[2], o_full, drained;   // scores, probabilities: of a step's parity (and a group)
  uint64_t seg_full[kSegRing], set_full[kSegRing], seg_done[kSegRing], q_full[kSegRing];
  uint64_t q_free;                                // of a segment: its last scores are had
  uint64_t soft;                                  // the softmax warps' meeting point
  Segment segs[kSegRing];
  uint64_t sets[kSegRing][SDV_MAX_TREE];          // what their nodes see of the tree
  int64_t before[kPrefixFrom + 1];                // steps before each sequence, where they are few
  uint16_t v_to[kTileChunks * 128];               // (Loader::init)
  float downs[kSegRing][kTileRows];               // what a row's queries were divided by
  float scales[kScaleRing][3 * kTileChunks];      // of a step's chunks: ks, then kPScale vs, then log2 |vs|
  uint32_t absent[kScaleRing];                    // chunks that are not there; bit 31: an ordinary step (see soft_probs)
  alignas(16) uint32_t nan_keys[kScaleRing][4];               // keys that have NaN among their values
  float ml[2][3][kTileRows];                      // the groups' references, sums, bases
  float* aside;                                   // what the groups have put aside: [group], as put_aside has it
  uint32_t tmem;
  int dead;
};

template <int kD>
struct TreeShape {
  static constexpr int kTile = kTileKeys * kD * 2;                  // bytes of an operand
  static constexpr int kBlock = kTileRows * 128;                     // of [128 rows][64 elements]
  static constexpr int kVBlock = kD * 128;                           // of [D rows][64 keys]
  static constexpr int kHalf = kTileKeys * kD;                       // codes of half a step
  static constexpr int kQ = 0, kK = kTile, kV = kK + kKStages * kTile, kRk = kV + kVStages * kTile, kRv = kRk + kRawK * kHalf, kSmallAt = kRv + kRawV * kHalf;
  static constexpr size_t kSmem = 1024 + kSmallAt + sizeof(TreeSmall);
  // floats of a partial: output [D / 4][row][4], so that a warp's rows are written together; reference (two numbers), sum
  static constexpr int kSlot = kTileRows * (kD + 3);
  static constexpr int kAsideAt = kTileRows * kD;                     // floats that a group has put aside, [D / 4][row][4]
  static constexpr int kLoads = kD / 16;                             // sixteens of a thread's keys, or of its values
  static_assert(kSmem <= 227 * 1024, "");
};

struct TreeRowsArgs {
  AttendArgs a;                    // RT: row tiles, R: rows; part: 2 slots a CTA
  int rows, teams;                 // rows of a tile; teams of RT CTAs
};

// Behind the partials and what was put aside, of each CTA: whether a wait of it gave up, so that what it was to write is not there.
template <int kD>
__device__ __forceinline__ int* gave_up(const TreeRowsArgs& T) {
  return reinterpret_cast<int*>(T.a.part + (int64_t)T.a.ctas * 2 * (TreeShape<kD>::kSlot + TreeShape<kD>::kAsideAt));
}

__device__ __forceinline__ int tree_runs(int64_t units, int teams) {
  return (int)min((int64_t)teams, (units + kMinTileSteps - 1) / kMinTileSteps);
}

// A warp's part in a meeting of several warps (bounded, unlike bar.sync).
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, int* dead) {
  return __all_sync(0xffffffffu, barrier_wait(bar, parity, dead));
}
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
  __syncwarp();
  if (lane == 0) barrier_arrive(bar);
}
struct Meeting {
  uint64_t* bar;
  uint32_t parity;
  __device__ __forceinline__ bool operator()(int lane, int* dead) {
    warp_arrive(bar, lane);
    const bool ok = warp_wait(bar, parity, dead);
    parity ^= 1;
    return ok;
  }
};

// The bytes' top bits tell which of four codes are NaN.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// log2 |vs| as a reference takes it: powers of two by it, their sums and their quotients by such sums stay in fp32's range.
// (Values smaller than that lose bits.)
__device__ __forceinline__ float log2_scale(float vs) { return fminf(fmaxf(log2f(fabsf(vs)), -100.f), 119.f); }

// Chunks of a step that the first group takes.
__device__ __forceinline__ int first_half(int chunks) { return (chunks + 1) / 2; }

// ------------------------------------------------------------------------------ the warp that plans
// The run's segments one after another, as far ahead as their ring allows.
__device__ __forceinline__ void plan_role(const TreeRowsArgs& T, TreeSmall& sm, int team, int lane) {
  const AttendArgs& A = T.a;
  const int per = A.c.H;
  int64_t total = 0;
  if (A.prefix) {
    total = A.prefix[A.B];
  } else {
    int64_t sum = 0;
    for (int b0 = 0; b0 < A.B; b0 += 32) {
      const int mine = b0 + lane < A.B ? seq_of<true, 0>(A, b0 + lane).steps : 0;
      int inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += x;
      }
      if (b0 + lane <= A.B) sm.before[b0 + lane] = sum + inc - mine;
      sum += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (lane == 0) sm.before[A.B] = sum;
    __syncwarp();
    total = sum;
  }
  const auto before = [&](int b) { return A.prefix ? A.prefix[b] : sm.before[b]; };
  // the last sequence whose steps begin at `at` or earlier, of which there are `total` in all: 32 places at a time
  const auto find = [&](int64_t at) {
    int lo = 0, hi = A.B;
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, here = lo + lane * step;
      const unsigned le = __ballot_sync(0xffffffffu, here < hi && before(here) <= at);
      const int k = 31 - __clz(le);                        // (lane 0 holds)
      hi = min(hi, lo + (k + 1) * step);
      lo += k * step;
    }
    return lo;
  };
  const int64_t units = total * per;
  const int runs = tree_runs(units, T.teams);
  int64_t u = 0, u_end = 0;
  if (team < runs) {
    u = run_start(units, team, runs);
    u_end = run_start(units, team + 1, runs);
  }
#pragma unroll 1
  for (int seg = 0;; ++seg) {
    Segment g{};
    if (u < u_end) {
      const int b = find(u / per);
      const int64_t seq_u = before(b) * per;
      const Seq sq = seq_of<true, 0>(A, b);
      if (u >= seq_u && u < seq_u + (int64_t)sq.steps * per) {   // (else the lengths have changed meanwhile)
        const int item = (int)((u - seq_u) / sq.steps);
        g.b = b, g.h = item, g.step0 = (int)(u - seq_u - (int64_t)item * sq.steps);
        g.steps = (int)min((int64_t)sq.steps - g.step0, u_end - u);
        g.len = sq.len, g.count = sq.count;
        g.whole = g.steps == sq.steps;
        g.slot = seg ? 1 : 0;
        u += g.steps;
      }
    }
    const int slot = seg & (kSegRing - 1);
    if (seg >= kSegRing && !warp_wait(&sm.seg_done[slot], (seg / kSegRing - 1) & 1, &sm.dead)) return;
    if (lane == 0) sm.segs[slot] = g;
    warp_arrive(&sm.seg_full[slot], lane);
    uint64_t a0 = 0, a1 = 0;
    if (g.steps) {
      bool bad = false;
      const int32_t* parents = A.parents + (int64_t)g.b * A.W;
      ancestors(lane < A.W ? parent_of(parents[lane], lane, bad) : -1, 32 + lane < A.W ? parent_of(parents[32 + lane], 32 + lane, bad) : -1,
                lane, a0, a1);
    }
    sm.sets[slot][lane] = a0;
    sm.sets[slot][32 + lane] = a1;
    warp_arrive(&sm.set_full[slot], lane);
    if (!g.steps) return;
  }
}

// ------------------------------------------------------------------------------ the warp that copies
// A place among the run's steps: step `n` of a segment.
struct Cursor {
  int seg, n;
  Segment g;                                              // (steps = 0: past the end)
};
__device__ __forceinline__ bool next_step(Cursor& c, TreeSmall& sm) {
  if (++c.n < c.g.steps) return true;
  c.n = 0;
  ++c.seg;
  if (!warp_wait(&sm.seg_full[c.seg & (kSegRing - 1)], c.seg / kSegRing & 1, &sm.dead)) return false;
  c.g = sm.segs[c.seg & (kSegRing - 1)];
  return true;
}

// Page `lane` of each step: its number two steps ahead, its scales one, then its keys and values.  `keys`, `values`: the steps
// whose copies were issued.
template <int kD>
__device__ __forceinline__ void copy_steps(const TreeRowsArgs& T, uint8_t* smem, TreeSmall& sm, int lane, int& keys, int& values) {
  using S = TreeShape<kD>;
  const AttendArgs& A = T.a;
  int* dead = &sm.dead;
  const int block = A.c.block, pages = A.step / block, chunks = block / kChunk;
  const uint32_t bytes = (uint32_t)(block * kD);
  const auto page_of = [&](const Cursor& c) {
    const int at = (c.g.step0 + c.n) * pages + lane;
    if (!c.g.steps || lane >= pages || (int64_t)at * block >= c.g.len) return -1;
    const int p = __ldg(A.c.table + (int64_t)c.g.b * A.c.max_pages + at);
    if (p >= 0 && p < (int)A.c.pages) return p;
    if (A.status) atomicOr(A.status + c.g.b, SDV_STATUS_BAD_PAGE);
    return -1;
  };
  const auto scale_of = [&](const float* of, int page, int h, float none) { return page < 0 ? none : __ldg(of + (int64_t)page * A.c.H + h); };
  Cursor c{0, 0, Segment{}};
  if (!warp_wait(&sm.seg_full[0], 0, dead)) return;
  c.g = sm.segs[0];
  int page = page_of(c), h = c.g.h, more = c.g.steps;      // this step's; its scales
  float ks = scale_of(A.c.ks, page, h, 1.f), vs = scale_of(A.c.vs, page, h, 0.f);
  if (more && !next_step(c, sm)) return;
  int page1 = page_of(c), h1 = c.g.h, more1 = c.g.steps;   // the next one's
#pragma unroll 1
  for (int t = 0; more; ++t) {
    const int64_t head = (int64_t)max(page, 0) * A.c.H + h;
    const unsigned there = __ballot_sync(0xffffffffu, page >= 0);
    {                                                        // the scales are read behind the keys' barrier
      const int slot = t % kRawK, turn = t / kRawK;
      if (turn && !warp_wait(&sm.rk_free[slot], (turn - 1) & 1, dead)) return;
      {
        const bool plain = lane >= pages || (page >= 0 && ks >= 0.f && ks < INFINITY && fabsf(vs) < INFINITY);
        const int at = t & (kScaleRing - 1);
        uint32_t absent = 0;
        const float lw = log2_scale(vs);
        if (lane < 4) sm.nan_keys[at][lane] = 0;
        if (lane < pages)
          for (int k = lane * chunks; k < (lane + 1) * chunks; ++k) {
            sm.scales[at][k] = ks;
            sm.scales[at][kTileChunks + k] = kPScale * vs;
            sm.scales[at][2 * kTileChunks + k] = lw;
            absent |= (uint32_t)(page < 0) << k;
          }
        absent = __reduce_or_sync(0xffffffffu, absent);
        const bool all = __all_sync(0xffffffffu, plain);
        if (lane == 0) sm.absent[at] = absent | (all ? 0x80000000u : 0u);
        __syncwarp();
      }
      if (lane == 0) barrier_expect(&sm.rk_full[slot], __popc(there) * bytes);
      __syncwarp();
      if (page >= 0) copy_bulk(smem_addr(smem + S::kRk + slot * S::kHalf) + lane * bytes, A.c.k + head * bytes, bytes, &sm.rk_full[slot]);
      keys = t + 1;
    }
    {
      const int slot = t % kRawV, turn = t / kRawV;
      if (turn && !warp_wait(&sm.rv_free[slot], (turn - 1) & 1, dead)) return;
      if (lane == 0) barrier_expect(&sm.rv_full[slot], __popc(there) * bytes);
      __syncwarp();
      if (page >= 0) copy_bulk(smem_addr(smem + S::kRv + slot * S::kHalf) + lane * bytes, A.c.v + head * bytes, bytes, &sm.rv_full[slot]);
      values = t + 1;
    }
    page = page1, h = h1, more = more1;
    ks = scale_of(A.c.ks, page, h, 1.f);
    vs = scale_of(A.c.vs, page, h, 0.f);
    if (more && !next_step(c, sm)) return;
    page1 = page_of(c), h1 = c.g.h, more1 = c.g.steps;
  }
}
// Whether all is done or a wait gave up: no copy is under way when the block ends.
template <int kD>
__device__ __forceinline__ void copy_role(const TreeRowsArgs& T, uint8_t* smem, TreeSmall& sm, int lane) {
  int keys = 0, values = 0, ignore = 0;
  copy_steps<kD>(T, smem, sm, lane, keys, values);
  for (int t = max(0, keys - kRawK); t < keys; ++t) warp_wait(&sm.rk_full[t % kRawK], t / kRawK & 1, &ignore);
  for (int t = max(0, values - kRawV); t < values; ++t) warp_wait(&sm.rv_full[t % kRawV], t / kRawV & 1, &ignore);
}

// ------------------------------------------------------------------------------ loading warps
// A thread's values again, with 0 for NaN; their keys are noted.
template <int kD>
__device__ __noinline__ void put_nan(const uint8_t* codes, uint8_t* tile, uint32_t* nan_keys, int block, int lt, int live) {
  const int chunks = block / kChunk, region = chunks * kD;
  for (int n = lt; n < live; n += kGroupThreads) {
    const int i = chunks == 8 ? n ^ (n & 4) << 1 : n;
    const uint4 y = reinterpret_cast<const uint4*>(codes)[i];
    const uint32_t x[4] = {y.x, y.y, y.z, y.w};
    const int page = i / region, r = i - page * region, d = r / chunks, c = page * chunks + r - d * chunks;
    uint32_t keys = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t n = nan_codes(x[k]);
      keys |= (n >> 7 & 1 | n >> 14 & 2 | n >> 21 & 4 | n >> 28 & 8) << (4 * k);
      uint2 f;
      widen4(x[k] & ~((n >> 7) * 0xffu), f.x, f.y);
      *reinterpret_cast<uint2*>(tile + (c >> 2) * TreeShape<kD>::kVBlock + swizzled(d, (c & 3) * 2 + (k >> 1)) + (k & 1) * 8) = f;
    }
    if (keys) atomicOr(&nan_keys[c >> 1], keys << (16 * (c & 1)));
  }
}

template <int kD>
struct Loader {
  using S = TreeShape<kD>;
  static constexpr int kN = S::kLoads;
  static constexpr int kPieces = kD / 16;                  // of a key
  const AttendArgs& A;
  uint8_t* smem;
  TreeSmall& sm;
  int lt, lane;

  // Where the sixteens of values go in the operand.
  __device__ __forceinline__ void init() {
    const int chunks = A.c.block / kChunk, region = chunks * kD;               // sixteens of a page's values: [D][chunks]
    for (int i = lt; i < kTileChunks * kD; i += kGroupThreads) {
      const int at = turn_pairs(i, chunks == 8), page = at / region, r = at - page * region, d = r / chunks, c = page * chunks + r - d * chunks;
      sm.v_to[i] = (uint16_t)((c >> 2) * S::kVBlock + swizzled(d, (c & 3) * 2));
    }
  }
  // Which of 1024 sixteens, eight to a row, thread i takes: rows change places in pairs for the second four of each, so
  // that no two of eight lanes meet in a bank, neither here nor where their pieces go.
  static __device__ __forceinline__ int turn_pairs(int i, bool eight) { return eight ? i ^ (i & 4) << 1 : i; }
  // A sixteen's two pieces, in places p and p ^ 16.
  __device__ __forceinline__ void put(uint8_t* at, const uint4& x) {
    uint4 a, b;
    widen4(x.x, a.x, a.y);
    widen4(x.y, a.z, a.w);
    widen4(x.z, b.x, b.y);
    widen4(x.w, b.z, b.w);
    *reinterpret_cast<uint4*>(at) = a;
    *reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(at) ^ 16) = b;
  }
  // Two of the thread's sixteens at a time (short loops, as elsewhere here).
  __device__ __forceinline__ void put_keys(const uint8_t* codes, int stage, int live) {
    const int first = turn_pairs(lt, kPieces == 8), p = first % kPieces, row = first / kPieces;
    uint8_t* to = smem + S::kK + stage * S::kTile + (p >> 2) * S::kBlock + swizzled(row, (p & 3) * 2);
    const uint4* from = reinterpret_cast<const uint4*>(codes) + first;
#pragma unroll 1
    for (int j = 0; j < kN; j += 2) {
      if (lt + j * kGroupThreads >= live) break;             // (whole rows of threads)
      const uint4 x = from[j * kGroupThreads], y = from[(j + 1) * kGroupThreads];
      put(to + j * (kGroupThreads / kPieces) * 128, x);
      if (lt + (j + 1) * kGroupThreads < live) put(to + (j + 1) * (kGroupThreads / kPieces) * 128, y);
    }
  }
  __device__ __forceinline__ void put_values(const uint8_t* codes, int stage, int t, int live) {
    uint8_t* tile = smem + S::kV + stage * S::kTile;
    const uint4* from = reinterpret_cast<const uint4*>(codes) + turn_pairs(lt, A.c.block == 128);
    __half2 nan = __float2half2_rn(0.f);                   // stays 0 unless a code is NaN
    const __half2 zero = nan;
#pragma unroll 1
    for (int j = 0; j < kN; j += 2) {
      if (lt + j * kGroupThreads >= live) break;
      const uint4 x[2] = {from[j * kGroupThreads], from[(j + 1) * kGroupThreads]};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (lt + (j + k) * kGroupThreads >= live) break;
        uint32_t w[8];
        widen4(x[k].x, w[0], w[1]);
        widen4(x[k].y, w[2], w[3]);
        widen4(x[k].z, w[4], w[5]);
        widen4(x[k].w, w[6], w[7]);
#pragma unroll
        for (int e = 0; e < 8; ++e) nan = __hfma2(*reinterpret_cast<const __half2*>(&w[e]), zero, nan);
        uint8_t* at = tile + sm.v_to[lt + (j + k) * kGroupThreads];
        *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(at) ^ 16) = make_uint4(w[4], w[5], w[6], w[7]);
      }
    }
    if (*reinterpret_cast<const uint32_t*>(&nan) & 0x7fff7fffu) put_nan<kD>(codes, tile, sm.nan_keys[t & (kScaleRing - 1)], A.c.block, lt, live);
  }
  // The rows' queries, by both groups' threads n, D / 8 lanes a row: first as they are, then, if bf16, made f16 in place.
  __device__ __forceinline__ void put_queries(const Segment& g, int rt, int rows, int seg, int n) {
    constexpr int kLanes = kD / 8, kAtOnce = 2 * kGroupThreads / kLanes;
    const int e8 = n % kLanes;
    uint8_t* block = smem + S::kQ + (e8 >> 3) * S::kBlock;
#pragma unroll 1
    for (int row = n / kLanes; row < kTileRows; row += kAtOnce) {
      const int r = rt * rows + row, i = r / A.G;
      const bool live = row < rows && r < A.R && i < g.count;
      const int64_t at = live ? g.b * A.q_sb + i * A.q_st + (int64_t)(g.h * A.G + r - i * A.G) * A.q_sh + e8 * 8 : 0;
      if (A.q_vec) copy16(smem_addr(block + swizzled(row, e8 & 7)), reinterpret_cast<const uint16_t*>(A.q) + at, live);
      else *reinterpret_cast<uint4*>(block + swizzled(row, e8 & 7)) = live ? q_load8(A, at) : make_uint4(0, 0, 0, 0);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");         // (a thread's own)
#pragma unroll 2
    for (int row = n / kLanes; row < kTileRows; row += kAtOnce) {
      int up = 0;
      if (A.bf16) {                                          // takes the row's largest to [2^15, 2^16)
        uint4* at = reinterpret_cast<uint4*>(block + swizzled(row, e8 & 7));
        uint4 v = *at;
        float most = q_largest(v, true);
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        up = most > 0.f ? min(max(15 - log2_of(most), -112), 100) : 0;
        float f[8];
        Num<SDV_BF16>::unpack(v, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= pow2(up);
        *at = Num<SDV_F16>::pack(f);
      }
      if (e8 == 0) sm.downs[seg & (kSegRing - 1)][row] = pow2(-up);
    }
  }
};

// The keys' group; both bring a segment's queries.
template <int kD>
__device__ __forceinline__ void keys_role(const TreeRowsArgs& T, uint8_t* smem, TreeSmall& sm, int rt, int tid) {
  using S = TreeShape<kD>;
  Loader<kD> L{T.a, smem, sm};
  L.lt = tid, L.lane = tid & 31;
  const int lane = L.lane, live = T.a.step * kD / 16;
  int* dead = &sm.dead;
  int t = 0;
#pragma unroll 1
  for (int seg = 0;; ++seg) {
    if (!warp_wait(&sm.seg_full[seg & (kSegRing - 1)], seg / kSegRing & 1, dead)) return;
    const Segment g = sm.segs[seg & (kSegRing - 1)];
    if (!g.steps) return;
    // its queries, once the last scores before are had.  (A barrier of its own: the values' warps may be two steps ahead of the
    // scores, where the parity of the keys' would tell them of the step before the last.)
    if (seg && !warp_wait(&sm.q_free, (seg - 1) & 1, dead)) return;
    L.put_queries(g, rt, T.rows, seg, tid);
    fence_async();
    warp_arrive(&sm.q_full[seg & (kSegRing - 1)], lane);
#pragma unroll 1
    for (const int end = t + g.steps; t < end; ++t) {
      const int slot = t % kRawK, st = t % kKStages, turn = t / kKStages;
      if (!warp_wait(&sm.rk_full[slot], t / kRawK & 1, dead)) return;
      if (turn && !warp_wait(&sm.k_free[st], (turn - 1) & 1, dead)) return;
      L.put_keys(smem + S::kRk + slot * S::kHalf, st, live);
      warp_arrive(&sm.rk_free[slot], lane);
      fence_async();
      warp_arrive(&sm.k_full[st], lane);
    }
  }
}
template <int kD>
__device__ __forceinline__ void values_role(const TreeRowsArgs& T, uint8_t* smem, TreeSmall& sm, int rt, int tid) {
  using S = TreeShape<kD>;
  Loader<kD> L{T.a, smem, sm};
  L.lt = tid, L.lane = tid & 31;
  L.init();
  const int lane = L.lane, live = T.a.step * kD / 16;
  int* dead = &sm.dead;
  int t = 0;
#pragma unroll 1
  for (int seg = 0;; ++seg) {
    if (!warp_wait(&sm.seg_full[seg & (kSegRing - 1)], seg / kSegRing & 1, dead)) return;
    const Segment g = sm.segs[seg & (kSegRing - 1)];
    if (!g.steps) return;
    if (seg && !warp_wait(&sm.q_free, (seg - 1) & 1, dead)) return;
    L.put_queries(g, rt, T.rows, seg, kGroupThreads + tid);
    fence_async();
    warp_arrive(&sm.q_full[seg & (kSegRing - 1)], lane);
#pragma unroll 1
    for (const int end = t + g.steps; t < end; ++t) {
      const int slot = t % kRawV, st = t % kVStages, turn = t / kVStages;
      if (!warp_wait(&sm.rv_full[slot], t / kRawV & 1, dead)) return;
      if (turn && !warp_wait(&sm.v_free[st], (turn - 1) & 1, dead)) return;
      L.put_values(smem + S::kRv + slot * S::kHalf, st, t, live);
      warp_arrive(&sm.rv_free[slot], lane);
      fence_async();
      warp_arrive(&sm.v_full[st], lane);
    }
  }
}

// ------------------------------------------------------------------------------ the warps that issue the products
// All of a warp's lanes go along, so that addresses and descriptors are the warp's (uniform registers); one of them issues.
// (With a single thread in this role a product took 100 cycles to issue, 64 to run.)
template <int kD>
__device__ __forceinline__ void scores_role(uint8_t* smem, TreeSmall& sm, int step) {
  using S = TreeShape<kD>;
  int* dead = &sm.dead;
  const uint32_t base = __shfl_sync(0xffffffffu, sm.tmem, 0);
  const uint64_t q = tile_desc(__shfl_sync(0xffffffffu, smem_addr(smem + S::kQ), 0)), k = q + (S::kK - S::kQ) / 16;
  const uint32_t score = mma_desc(kTileRows, step);
  const bool one = elected();
  int t = 0;
#pragma unroll 1
  for (int seg = 0;; ++seg) {
    const uint32_t turn = seg / kSegRing & 1;
    if (!warp_wait(&sm.seg_full[seg & (kSegRing - 1)], turn, dead)) break;
    const int steps = __shfl_sync(0xffffffffu, sm.segs[seg & (kSegRing - 1)].steps, 0);
    if (!steps || !warp_wait(&sm.q_full[seg & (kSegRing - 1)], turn, dead)) break;
    bool ok = true;
#pragma unroll 1
    for (const int end = t + steps; t < end; ++t) {
      const int st = t % kKStages;
      // the probabilities two steps ago, in whose place the scores go, are used
      ok = (t < 2 || warp_wait(&sm.p_free[t & 1], ((t >> 1) - 1) & 1, dead)) && warp_wait(&sm.k_full[st], t / kKStages & 1, dead);
      if (!ok) break;
      tmem_after_sync();
      const uint32_t to = base + (t & 1) * kTileKeys;
      const uint64_t kt = k + st * (S::kTile / 16);
      if (one) {
#pragma unroll 1
        for (int i = 0; i < kD / 16; ++i) {
          const int off = ((i >> 2) * S::kBlock + (i & 3) * 32) / 16;
          mma_ss(to, q + off, kt + off, score, i > 0);
        }
        mma_commit(&sm.s_full[t & 1]);
        mma_commit(&sm.k_free[st]);
        if (t + 1 == end) mma_commit(&sm.q_free);
      }
      __syncwarp();
    }
    if (!ok) break;
  }
  if (one) mma_commit(&sm.drained);                        // nothing is under way when the memory is given back
  __syncwarp();
}

template <int kD>
__device__ __forceinline__ void out_role(uint8_t* smem, TreeSmall& sm, int step) {
  using S = TreeShape<kD>;
  int* dead = &sm.dead;
  const uint32_t base = __shfl_sync(0xffffffffu, sm.tmem, 0);
  const uint64_t v = tile_desc(__shfl_sync(0xffffffffu, smem_addr(smem + S::kV), 0));
  constexpr uint32_t kOut = mma_desc(kTileRows, kD);
  const int chunks = step / kChunk, half = first_half(chunks);
  const bool one = elected();
  int t = 0;
#pragma unroll 1
  for (int seg = 0;; ++seg) {
    if (!warp_wait(&sm.seg_full[seg & (kSegRing - 1)], seg / kSegRing & 1, dead)) break;
    const int steps = __shfl_sync(0xffffffffu, sm.segs[seg & (kSegRing - 1)].steps, 0);
    if (!steps) break;
    bool ok = true;
#pragma unroll 1
    for (int n = 0; n < steps; ++n, ++t) {
      const int st = t % kVStages;
      const uint32_t p = base + (t & 1) * kTileKeys;
      const uint64_t vt = v + st * (S::kTile / 16);
      ok = warp_wait(&sm.v_full[st], t / kVStages & 1, dead);
#pragma unroll 1
      for (int h = 0; h < 2 && ok; ++h) {                  // a group's keys
        ok = warp_wait(&sm.p_full[t & 1][h], t >> 1 & 1, dead);
        if (!ok) break;
        tmem_after_sync();
        const uint32_t out = base + 2 * kTileKeys + h * 128;
        if (one) {
          const int i0 = h ? half : 0, i1 = h ? chunks : half;
#pragma unroll 1
          for (int i = i0; i < i1; ++i) {
            const int off = ((i >> 2) * S::kVBlock + (i & 3) * 32) / 16;
            mma_ts(out, p + i * 16, vt + off, kOut, n % kAside > 0 || i > i0);
            mma_ts(out, p + i * 16 + 8, vt + off, kOut, true);
          }
          if (h) {
            mma_commit(&sm.p_free[t & 1]);
            mma_commit(&sm.v_free[st]);
            if (n + 1 == steps) mma_commit(&sm.o_full);
          }
        }
        __syncwarp();
      }
      if (!ok) break;
    }
    if (!ok) break;
  }
  if (one) mma_commit(&sm.drained);
  __syncwarp();
  int ignore = 0;
  warp_wait(&sm.drained, 0, &ignore);
}

// ------------------------------------------------------------------------------ softmax warps
// What a row sees of 64 keys, as bits: the first n, and the set of the tree whose node 0 stands in place `at`.
__device__ __forceinline__ uint64_t below(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }
__device__ __forceinline__ uint64_t placed(uint64_t set, int at) {
  return at <= -64 || at >= 64 ? 0ull : at <= 0 ? set >> -at : set << at;
}

// A row's running state: its reference base + m (log2; base is 0 unless its scores are past 2^20), and the sum of
// 2^(score - reference).  lag: log2 of what takes the sums put aside to the reference, not above 0 (put_aside).
struct SoftRow {
  float m, l, base, lag;
};
// x 2^d for d <= 0, in two steps: neither factor underflows where the product does not.
__device__ __forceinline__ float scaled(float x, float half) { return x * half * half; }

// A chunk's sixteen probabilities p, which are added to the sums, times vs, as halves into the chunk's columns: eight of first
// ones, eight of second ones.  The first half is the number cut off after eleven bits, the second the rest of it, rounded.
__device__ __forceinline__ void put_probs(uint32_t at, const f32x2* p, float vs, f32x2* sum) {
  const f32x2 minus = pair(-1.f, -1.f);
  uint32_t o[16];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const f32x2 v = mul2(p[e], pair(vs, vs));
    sum[e & 1] = add2(sum[e & 1], p[e]);
    const float2 y = unpair(v);
    const float c0 = __uint_as_float(__float_as_uint(y.x) & 0xffffe000u), c1 = __uint_as_float(__float_as_uint(y.y) & 0xffffe000u);
    o[e] = pack_half(c0, c1);
    const float2 rest = unpair(fma2(pair(c0, c1), minus, v));
    o[8 + e] = pack_half(rest.x, rest.y);
  }
  tmem_store16(at, o);
}
__device__ __forceinline__ void add_sums(const f32x2* sum, SoftRow& s) {
  const float2 s2 = unpair(add2(sum[0], sum[1]));
  s.l += s2.x + s2.y;
  tmem_stored();
}

// A row's part of a step, up to 64 keys: scores in columns from `at` on (and in x) become probabilities times their values'
// scale; l goes on.  Every row sees every key, no scale of keys is negative, none without a number, no reference large.
__device__ __forceinline__ void soft_probs(uint32_t at, const uint32_t* x, int chunks, const float* scales, float f0, SoftRow& s) {
  f32x2 sum[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
  const f32x2 nm = pair(-s.m, -s.m);
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if (c >= chunks) break;
    const float f = f0 * scales[c];
    f32x2 p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 a = unpair(fma2(pair(__uint_as_float(x[16 * c + 2 * e]), __uint_as_float(x[16 * c + 2 * e + 1])), pair(f, f), nm));
      p[e] = pair(ex2(a.x), ex2(a.y));
    }
    put_probs(at + 16 * c, p, scales[kTileChunks + c], sum);
  }
  add_sums(sum, s);
}

// By how much the reference (m, base) exceeds that of (m0, base0).
__device__ __forceinline__ float reference_less(float m0, float base0, float m, float base) { return (base - base0) + (m - m0); }

// A step, of the CTA and of its segment: where the products of the steps before it end.
struct Before {
  TreeSmall* sm;
  int t, n;
  __device__ __forceinline__ bool any() const { return n > 0; }
  __device__ __forceinline__ bool aside() const { return n > 0 && n % kAside == 0; }       // their sums are put aside
  __device__ __forceinline__ void wait() const {             // (given up: so does the next wait)
    warp_wait(&sm->p_free[(t - 1) & 1], (t - 1) >> 1 & 1, &sm->dead);
    tmem_after_sync();
  }
};
// The matrix unit cuts its sums off instead of rounding them: where the products have one sign, 128 keys more cost 5e-7 of the
// sum, 1.6e-4 after 250 steps, a third of f16's half step and more with every key.  So what kAside steps have
// summed in tensor memory goes over into sums that are rounded to nearest, a group's and row's own in the workspace (in L2), and
// the next product begins from nothing: 3.1e-5 at most, whatever a sequence's length.  2 x 60 nodes of 8 x 8
// heads over 65000 keys take 374 us with and 362 without it, 32 x 32 of 8 x 4 heads over up to 16000 keys 241 and 236: about 2 us
// each time, and the code.  Both functions stay out of line, and away from where scores are live: a call from between
// scores and probabilities spilled them (277 us); the sums read in the epilogue's own loops took 249.
template <int kD>
__device__ __forceinline__ float4* aside_of(const TreeSmall& sm) {     // this thread's row and group
  return reinterpret_cast<float4*>(sm.aside + (threadIdx.x / kTileRows) * TreeShape<kD>::kAsideAt) + threadIdx.x % kTileRows;
}
// lag: log2 of what takes the sums put aside to the reference.
template <int kD>
__device__ __noinline__ void put_aside(uint32_t out, Before before, float lag) {
  float4* y = aside_of<kD>(*before.sm);
  const float by = ex2(.5f * lag);
  const bool first = before.n == kAside;
#pragma unroll 1
  for (int g = 0; g < kD / 64; ++g, y += 16 * kTileRows) {
    float4 b[16];                                            // (64 numbers of a row on their way at once)
#pragma unroll
    for (int e = 0; e < 16; ++e) b[e] = first ? make_float4(0.f, 0.f, 0.f, 0.f) : y[e * kTileRows];
    if (g == 0) before.wait();
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint32_t r[16];
      tmem_load16(out + 64 * g + 16 * c, r);
      tmem_loaded16(r);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float4 v = b[4 * c + e];
        y[(4 * c + e) * kTileRows] = make_float4(scaled(v.x, by) + __uint_as_float(r[4 * e]), scaled(v.y, by) + __uint_as_float(r[4 * e + 1]),
                                                 scaled(v.z, by) + __uint_as_float(r[4 * e + 2]), scaled(v.w, by) + __uint_as_float(r[4 * e + 3]));
      }
    }
  }
}
// At a segment's end: they are added to the last steps' sums in tensor memory.
template <int kD>
__device__ __noinline__ void put_back(uint32_t out, const TreeSmall& sm, float lag) {
  const float4* aside = aside_of<kD>(sm);
  const float by = ex2(.5f * lag);
#pragma unroll 1
  for (int g = 0; g < kD / 32; ++g, aside += 8 * kTileRows) {
    float4 b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = aside[e * kTileRows];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      uint32_t r[16];
      tmem_load16(out + 32 * g + 16 * c, r);
      tmem_loaded16(r);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float4 v = b[4 * c + e];
        r[4 * e] = __float_as_uint(__uint_as_float(r[4 * e]) + scaled(v.x, by));
        r[4 * e + 1] = __float_as_uint(__uint_as_float(r[4 * e + 1]) + scaled(v.y, by));
        r[4 * e + 2] = __float_as_uint(__uint_as_float(r[4 * e + 2]) + scaled(v.z, by));
        r[4 * e + 3] = __float_as_uint(__uint_as_float(r[4 * e + 3]) + scaled(v.w, by));
      }
      tmem_store16(out + 32 * g + 16 * c, r);
    }
  }
  tmem_stored();
}
// The sums of a row that goes over to a reference higher by 2^-d, half = 2^(d / 2).
template <int kD>
__device__ __noinline__ void move_out(uint32_t out, Before before, float half) {
  before.wait();
  uint32_t r[16];
#pragma unroll 1
  for (int g = 0; g < kD / 16; ++g) {
    tmem_load16(out + 16 * g, r);
    tmem_loaded16(r);
#pragma unroll
    for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(scaled(__uint_as_float(r[e]), half));
    tmem_store16(out + 16 * g, r);
  }
  tmem_stored();
}
template <int kD>
__device__ __forceinline__ void soft_move(uint32_t out, const Before& before, float d, SoftRow& s) {
  const float half = ex2(.5f * d);
  s.l = scaled(s.l, half);
  s.lag += d;
  if (before.any()) move_out<kD>(out, before, half);
}
__device__ __forceinline__ void soft_load(uint32_t at, uint32_t* x) {
  tmem_load32(at, x);
  tmem_load32(at + 32, x + 32);
  tmem_loaded(x);
  tmem_loaded(x + 32);
}

// The row's largest score less its base, plus log2 of the values' scale (`scale`: or without), of what it sees.
static __device__ __noinline__ float soft_top(uint32_t at, int chunks, const float* scales, float f0, uint64_t sees, float base, bool scale) {
  float top = -INFINITY;
#pragma unroll 1
  for (int c = 0; c < chunks; ++c) {
    uint32_t x[16];
    tmem_load16(at + 16 * c, x);
    const uint32_t w = (uint32_t)(sees >> (16 * c));
    const float f = f0 * scales[c], lw = scale ? scales[2 * kTileChunks + c] : 0.f;
    tmem_loaded16(x);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float y = (__fmul_rn(__uint_as_float(x[e]), f) - base) + lw;
      top = w >> e & 1 ? fmaxf(top, y) : top;
    }
  }
  return top;
}

// A step where some row does not see all, or of unusual scales or scores.  What a row does not see gets 0, what it sees of a scale
// without a number NaN; and the score is rounded before the reference is taken off: the fused product is off by half a step of
// the reference, which large scores make a large power.
// (This code runs once or twice a segment, and so from a cold instruction cache: short loops.  With its loops unrolled such a
// step took 7 us.  Where every step takes it, with key scales below 0 or a scale below 0, 32 x 32 nodes of 8 x 4 heads over 8000 keys
// take 363 us in place of 204, 2 x 64 of 8 x 8 over 65000 688 in place of 356.)
template <int kD>
__device__ __noinline__ SoftRow soft_any(uint32_t at, uint32_t out, int chunks, const float* scales, float f0, uint64_t sees, Before before,
                                         SoftRow s) {
  // a base for scores past 2^20: of the row's own, when they pass the old one or nothing has been seen
  float top = soft_top(at, chunks, scales, f0, sees, s.base, false);
  const bool large = fabsf(top) < INFINITY && (s.m > kNone ? top > kMostPlain : fabsf(top) > kMostPlain);
  if (__any_sync(0xffffffffu, large)) {
    const float base = large ? s.base + top : s.base;
    if (s.m > kNone) s.m = fmaxf(s.m + (s.base - base), kNone);
    s.base = base;
    __syncwarp();
  }
  top = soft_top(at, chunks, scales, f0, sees, s.base, true);
  const bool move = top > s.m + kSlack;
  if (__any_sync(0xffffffffu, move) ) {
    const float now = move ? top : s.m, d = s.m - now;
    s.m = now;
    soft_move<kD>(out, before, d, s);
  }
  f32x2 sum[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
#pragma unroll 1
  for (int c = 0; c < chunks; ++c) {
    uint32_t x[16];
    tmem_load16(at + 16 * c, x);
    const uint32_t w = (uint32_t)(sees >> (16 * c));
    const float f = f0 * scales[c], vs = scales[kTileChunks + c];
    const bool none = !(fabsf(vs) < INFINITY) || !(fabsf(f) < INFINITY);
    tmem_loaded16(x);
    f32x2 p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float2 a = make_float2(ex2((__fmul_rn(__uint_as_float(x[2 * e]), f) - s.base) - s.m),
                             ex2((__fmul_rn(__uint_as_float(x[2 * e + 1]), f) - s.base) - s.m));
      a.x = !(w >> (2 * e) & 1) ? 0.f : none ? NAN : a.x;
      a.y = !(w >> (2 * e + 1) & 1) ? 0.f : none ? NAN : a.y;
      p[e] = pair(a.x, a.y);
    }
    put_probs(at + 16 * c, p, none ? 1.f : vs, sum);
  }
  add_sums(sum, s);
  return s;
}

// An ordinary step: the row's largest score first, against which its reference may move.
template <int kD>
__device__ __forceinline__ void soft_tile(uint32_t at, uint32_t out, int chunks, const float* scales, float f0, const Before& before, SoftRow& s) {
  uint32_t x[64];
  soft_load(at, x);
  float top = -INFINITY;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if (c >= chunks) break;
    const uint32_t* r = x + 16 * c;
    float y[5];
#pragma unroll
    for (int e = 0; e < 5; ++e) y[e] = max3(__uint_as_float(r[3 * e]), __uint_as_float(r[3 * e + 1]), __uint_as_float(r[3 * e + 2]));
    const float most = fmaxf(max3(y[0], y[1], y[2]), max3(y[3], y[4], __uint_as_float(r[15])));
    top = fmaxf(top, fmaf(most, f0 * scales[c], scales[2 * kTileChunks + c]));
  }
  // the reference moves when a score passes it by 2^kSlack
  const bool move = top > s.m + kSlack;
  if (__any_sync(0xffffffffu, move || s.base != 0.f) ) {
    if (__any_sync(0xffffffffu, s.base != 0.f || (move && fabsf(top) > kMostPlain))) {
      s = soft_any<kD>(at, out, chunks, scales, f0, ~0ull, before, s);
      return;
    }
    const float now = move ? top : s.m, d = s.m - now;
    s.m = now;
    soft_move<kD>(out, before, d, s);
  }
  soft_probs(at, x, chunks, scales, f0, s);
}

template <int kD>
__device__ __forceinline__ void soft_role(const TreeRowsArgs& T, uint8_t* smem, TreeSmall& sm, int team, int rt, int tid) {
  using S = TreeShape<kD>;
  const AttendArgs& A = T.a;
  const int lane = tid & 31, warp = tid >> 5, s = warp >> 2, row = (warp & 3) * 32 + lane;
  int* dead = &sm.dead;
  const uint32_t lanes = sm.tmem + ((uint32_t)((warp & 3) * 32) << 16);
  const uint32_t out = lanes + 2 * kTileKeys;
  const int all = T.a.step / kChunk, chunk0 = s ? first_half(all) : 0, chunks = s ? all - chunk0 : first_half(all);   // this group's
  Meeting meet{&sm.soft, 0};
  const int r = rt * T.rows + row, i = r / A.G;
  int t = 0;
#pragma unroll 1
  for (int seg = 0;; ++seg) {
    const uint32_t turn = seg / kSegRing & 1;
    if (!warp_wait(&sm.seg_full[seg & (kSegRing - 1)], turn, dead)) return;
    const Segment g = sm.segs[seg & (kSegRing - 1)];
    if (!g.steps || !warp_wait(&sm.q_full[seg & (kSegRing - 1)], turn, dead)) return;
    const bool have = row < T.rows && r < A.R, live = have && i < g.count;
    const bool busy = __any_sync(0xffffffffu, live);
    if (!warp_wait(&sm.set_full[seg & (kSegRing - 1)], turn, dead)) return;
    const uint64_t set = live ? sm.sets[seg & (kSegRing - 1)][i] : 0;
    const float f0 = A.scale2 * sm.downs[seg & (kSegRing - 1)][row];
    const int at0 = g.len - g.count;                      // the root's place
    SoftRow mine{kNone, 0.f, 0.f, 0.f};
    // what the row sees of a step's keys from key0 on
    const auto seen = [&](int key0, uint32_t absent) {
      uint64_t can = (below(at0 - key0) | placed(set, at0 - key0)) & below(chunks * kChunk);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (absent >> (chunk0 + c) & 1) can &= ~(0xffffull << (16 * c));
      return live ? can : 0ull;
    };
    // NaN among the values that a row saw two steps ago, whose products are done: its own affair, since they are 0 for the others
    const auto look_for_nan = [&](int t, int n) {
      const int slot = t & (kScaleRing - 1);
      const uint4 nan = *reinterpret_cast<const uint4*>(sm.nan_keys[slot]);
      if (nan.x | nan.y | nan.z | nan.w) {
        const uint64_t lo = nan.x | (uint64_t)nan.y << 32, hi = nan.z | (uint64_t)nan.w << 32;
        const uint64_t keys = !chunk0 ? lo : chunk0 == 4 ? hi : lo >> (16 * chunk0) | hi << (64 - 16 * chunk0);
        if (seen((g.step0 + n) * A.step + chunk0 * kChunk, sm.absent[slot]) & keys) mine.l = NAN;
        __syncwarp();                                        // (tensor memory is read by all lanes at once)
      }
    };
#pragma unroll 1
    for (int n = 0; n < g.steps; ++n, ++t) {
      if (!warp_wait(&sm.s_full[t & 1], t >> 1 & 1, dead)) return;
      tmem_after_sync();
      if (n >= 2) look_for_nan(t - 2, n - 2);
      const int slot = t & (kScaleRing - 1), key0 = (g.step0 + n) * A.step + chunk0 * kChunk;
      const uint32_t absent = sm.absent[slot], at = lanes + (t & 1) * kTileKeys + chunk0 * kChunk;
      const float* scales = sm.scales[slot] + chunk0;
      const Before before{&sm, t, n};
      if (absent >> 31 && key0 + chunks * kChunk <= at0 && A.scale2 >= 0.f) {
        if (busy) soft_tile<kD>(at, out + s * 128, chunks, scales, f0, before, mine);
      } else if (busy) {
        const uint64_t sees = seen(key0, absent);
        __syncwarp();
        mine = soft_any<kD>(at, out + s * 128, chunks, scales, f0, sees, before, mine);
      }
      if (busy && before.aside()) {                          // (behind the probabilities: the products before are done by now)
        put_aside<kD>(out + s * 128, before, mine.lag);
        mine.lag = 0.f;
      }
      tmem_before_sync();
      warp_arrive(&sm.p_full[t & 1][s], lane);
    }
    // the segment's rows: both groups' sums, a half of the columns each
    if (!warp_wait(&sm.o_full, seg & 1, dead)) return;
    tmem_after_sync();
    if (g.steps > 1) look_for_nan(t - 2, g.steps - 2);
    look_for_nan(t - 1, g.steps - 1);
    if (busy && g.steps > kAside) {
      put_back<kD>(out + s * 128, sm, mine.lag);
      tmem_before_sync();
    }
    sm.ml[s][0][row] = mine.m;
    sm.ml[s][1][row] = mine.l;
    sm.ml[s][2][row] = mine.base;
    if (!meet(lane, dead)) return;
    tmem_after_sync();
    if (busy || (__any_sync(0xffffffffu, have))) {
      const float m0 = sm.ml[0][0][row], m1 = sm.ml[1][0][row], b0 = sm.ml[0][2][row], b1 = sm.ml[1][2][row];
      const float ahead = reference_less(m1, b1, m0, b0);    // of the first group's reference
      const float top = ahead >= 0.f ? m0 : m1, base = ahead >= 0.f ? b0 : b1;
      const float c0 = ex2(.5f * fminf(ahead, 0.f)), c1 = ex2(-.5f * fmaxf(ahead, 0.f));
      const float sum = live ? scaled(sm.ml[0][1][row], c0) + scaled(sm.ml[1][1][row], c1) : 0.f;
      const float by = !g.whole ? 1.f / kPScale : sum == 0.f ? 0.f : 1.f / sum / kPScale;
      const int64_t to = ((int64_t)g.b * A.W + i) * (A.c.H * A.G) + g.h * A.G + (r - i * A.G);
      float* part = A.part + ((int64_t)(blockIdx.x * 2 + g.slot)) * S::kSlot;
#pragma unroll 1
      for (int k = 0; k < kD / 64; ++k) {
        const int col = s * (kD / 2) + 32 * k;
        uint32_t a[32];
        float o[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0.f;
        if (busy) {
          tmem_load32(out + col, a);
          tmem_loaded(a);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = scaled(__uint_as_float(a[e]), c0);
          tmem_load32(out + 128 + col, a);
          tmem_loaded(a);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] += scaled(__uint_as_float(a[e]), c1);
        }
        if (have && g.whole) {
          const bool zero = sum == 0.f;
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = zero ? 0.f : o[e] * by;
          uint4* y = reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(A.out) + to * kD + col);
          if (A.out_vec) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = A.bf16 ? Num<SDV_BF16>::pack(o + 8 * e) : Num<SDV_F16>::pack(o + 8 * e);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) put_out(A, to * kD + col + e, o[e]);
          }
        } else if (have) {
          float4* y = reinterpret_cast<float4*>(part) + (col / 4) * kTileRows + row;
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e * kTileRows] = make_float4(o[4 * e] * by, o[4 * e + 1] * by, o[4 * e + 2] * by, o[4 * e + 3] * by);
        }
        __syncwarp();                                        // the next columns are read by all lanes at once
      }
      if (have && s == 0) {
        if (g.whole) {
          if (A.lse) A.lse[to] = lse_of(top, sum, base);
        } else {
          part[kTileRows * kD + row] = top;
          part[kTileRows * kD + kTileRows + row] = base;
          part[kTileRows * kD + 2 * kTileRows + row] = sum;
        }
      }
    }
    tmem_before_sync();
    if (!meet(lane, dead)) return;                         // the sums are read: the next products may come
    warp_arrive(&sm.seg_done[seg & (kSegRing - 1)], lane);
  }
}

// A step of 128 keys and 128 rows of 128 takes about 1.45 us.  What bounds it is shared memory: codes in (32 KB), operands out
// and in (128 KB), and read again by the products (96 KB) are 2048 cycles at 128 bytes a cycle, 1.07 us.  The products alone take
// 1540 cycles (a third of them for the second half of the probabilities), the exponentials of both groups 1680, HBM's pace 1390.
// 32 x 32 nodes of 8 x 4 heads over up to 16000 keys 234 to 244 us by their lengths, 2.5
// TB/s; 2 x 60 of 8 x 8 heads over up to 65000 371 us, 690
// TFLOP/s; k_attend on mma.sync takes 781 and 1124.  Tried without gain: one issuing warp for both products, groups that take
// every other step, scores in two halves of 64 keys (1.84 us a step), codes read by the widening warps themselves.
template <int kD>
__global__ void __launch_bounds__(kTreeThreads, 1) k_tree_rows(const TreeRowsArgs T) {
  using S = TreeShape<kD>;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = raw + (-smem_addr(raw) & 1023);
  TreeSmall& sm = *reinterpret_cast<TreeSmall*>(smem + S::kSmallAt);
  const int tid = threadIdx.x, warp = tid >> 5, team = blockIdx.x / T.a.RT, rt = blockIdx.x - team * T.a.RT;
  if (warp == kScoreWarp) tmem_alloc(&sm.tmem, 512);
  if (tid == 0) {
    for (int k = 0; k < 2; ++k) {
      barrier_init(&sm.s_full[k], 1);
      barrier_init(&sm.p_full[k][0], kSoftWarps / 2);
      barrier_init(&sm.p_full[k][1], kSoftWarps / 2);
      barrier_init(&sm.p_free[k], 1);
    }
    for (int k = 0; k < kSegRing; ++k) {
      barrier_init(&sm.seg_full[k], 1);
      barrier_init(&sm.set_full[k], 1);
      barrier_init(&sm.seg_done[k], kSoftWarps);
      barrier_init(&sm.q_full[k], kLoadWarps);
    }
    for (int k = 0; k < kKStages; ++k) {
      barrier_init(&sm.k_full[k], kGroupWarps);
      barrier_init(&sm.k_free[k], 1);
    }
    for (int k = 0; k < kVStages; ++k) {
      barrier_init(&sm.v_full[k], kGroupWarps);
      barrier_init(&sm.v_free[k], 1);
    }
    for (int k = 0; k < kRawK; ++k) {
      barrier_init(&sm.rk_full[k], 1);
      barrier_init(&sm.rk_free[k], kGroupWarps);
    }
    for (int k = 0; k < kRawV; ++k) {
      barrier_init(&sm.rv_full[k], 1);
      barrier_init(&sm.rv_free[k], kGroupWarps);
    }
    barrier_init(&sm.o_full, 1);
    barrier_init(&sm.q_free, 1);
    barrier_init(&sm.drained, 2);
    barrier_init(&sm.soft, kSoftWarps);
    sm.dead = 0;
    sm.aside = T.a.part + (int64_t)T.a.ctas * 2 * S::kSlot + (int64_t)blockIdx.x * 2 * S::kAsideAt;      // (behind all partials)
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tmem_before_sync();
  __syncthreads();
  tmem_after_sync();
  if (warp < kSoftWarps) {
    registers_up<kSoftRegs>();
    soft_role<kD>(T, smem, sm, team, rt, tid);
  } else if (warp < kScoreWarp) {
    registers_down<kLoadRegs>();
    if (warp < kSoftWarps + kGroupWarps) keys_role<kD>(T, smem, sm, rt, tid - 32 * kSoftWarps);
    else values_role<kD>(T, smem, sm, rt, tid - 32 * (kSoftWarps + kGroupWarps));
  } else {
    registers_down<kOtherRegs>();
    if (warp == kPlanWarp) plan_role(T, sm, team, tid & 31);
    else if (warp == kCopyWarp) copy_role<kD>(T, smem, sm, tid & 31);
    else if (warp == kScoreWarp) scores_role<kD>(smem, sm, T.a.step);
    else out_role<kD>(smem, sm, T.a.step);
  }
  __syncwarp();
  tmem_before_sync();
  __syncthreads();
  tmem_after_sync();
  if (warp == kScoreWarp) tmem_free(sm.tmem, 512);
  if (tid == 0) gave_up<kD>(T)[blockIdx.x] = sm.dead;      // k_tree_join tells
}

// Joins the partials of an item that several teams' runs hold; an item without steps gets zeros, one of which a part is missing
// NaN.  A CTA has 32 rows, a lane each.
// Its warps share out the partials for the rows' references and weights (kept in shared memory, a batch at a time), and the
// columns, eight at a time, for the sums.  Bound by latency: 14.7 us after a cold cache for 96 items of 128 rows, a few of them behind
// the kernel before.
constexpr int kJoinBatch = 64;
template <int kD>
__global__ void __launch_bounds__(kJoinThreads) k_tree_join(const TreeRowsArgs T) {
  using S = TreeShape<kD>;
  const AttendArgs& A = T.a;
  constexpr int kCtas = kTileRows / 32;                      // of an item
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int ib = blockIdx.x / kCtas, row = blockIdx.x % kCtas * 32 + lane;
  const int per = A.c.H * A.RT, b = ib / per, item = ib % per, h = item / A.RT, rt = item % A.RT, r = rt * T.rows + row;
  const Sums ts = step_sums<true, 0>(A, b, lane);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (A.status && item == 0 && blockIdx.x % kCtas == 0 && warp == 0) {
    bool bad = lane == 0 && A.lengths[b] < min(A.counts ? A.counts[b] : A.W, A.W);
    for (int i = lane; i < min(A.counts ? A.counts[b] : A.W, A.W); i += 32) parent_of(A.parents[(int64_t)b * A.W + i], i, bad);
    if (bad) atomicOr(A.status + b, SDV_STATUS_BAD_TREE);
    if (lane == 0 && A.lengths[b] > A.c.max_pages * A.c.block) atomicOr(A.status + b, SDV_STATUS_BAD_PAGE);
  }
  const Seq sq = seq_of<true, 0>(A, b);
  const int64_t units = ts.total * A.c.H, u0 = ts.before * A.c.H + (int64_t)h * sq.steps, u1 = min(u0 + sq.steps, units);
  const int runs = tree_runs(units, T.teams);
  int g0 = 0, g1 = -1;
  if (u0 < u1) {
    // the runs [units g / runs, units (g + 1) / runs) that meet [u0, u1)
    g0 = (int)((u0 * runs) / units);
    while (run_start(units, g0 + 1, runs) <= u0) ++g0;
    while (run_start(units, g0, runs) > u0) --g0;
    g1 = (int)(((u1 - 1) * runs) / units);
    while (run_start(units, g1 + 1, runs) <= u1 - 1) ++g1;
    while (run_start(units, g1, runs) > u1 - 1) --g1;
  }
  bool stuck = false;                                        // a run's CTA gave up: what it had of the item is not there
  for (int gi = g0 + lane; gi <= g1; gi += 32) stuck |= gave_up<kD>(T)[gi * A.RT + rt] != 0;
  stuck = __any_sync(0xffffffffu, stuck);
  if (stuck && A.status && threadIdx.x == 0) atomicOr(A.status + b, SDV_STATUS_STUCK);
  if (g0 == g1 && !stuck) return;                           // written by that run's CTA
  const bool live = row < T.rows && r < A.R;
  const int64_t first = g0 <= g1 && run_start(units, g0, runs) < u0 ? 1 : 0;
  const auto slot_of = [&](int gi) { return A.part + (((int64_t)gi * A.RT + rt) * 2 + (gi == g0 ? first : 0)) * S::kSlot; };
  __shared__ float ref[2][kJoinWarps][32], weights[kJoinBatch][32], sums[kJoinWarps][32];
  const auto scalar = [&](int gi, int which) { return slot_of(gi)[kTileRows * kD + which * kTileRows + row]; };
  float m = kNone, base = 0.f;
  if (live) {
#pragma unroll 4
    for (int gi = g0 + warp; gi <= g1; gi += kJoinWarps) {
      const float om = scalar(gi, 0), ob = scalar(gi, 1);
      if (reference_less(m, base, om, ob) > 0.f) m = om, base = ob;
    }
  }
  ref[0][warp][lane] = m;
  ref[1][warp][lane] = base;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) {
    const float om = ref[0][w][lane], ob = ref[1][w][lane];
    if (reference_less(m, base, om, ob) > 0.f) m = om, base = ob;
  }
  constexpr int kPer = kD / 8 / kJoinWarps;                  // eights of columns of a warp
  float l = 0.f, o[kPer][8];
#pragma unroll
  for (int k = 0; k < kPer; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) o[k][e] = 0.f;
  for (int first_of = g0; first_of <= g1; first_of += kJoinBatch) {
    const int n = min(kJoinBatch, g1 + 1 - first_of);
    __syncthreads();                                         // the weights before are used
    if (live) {
#pragma unroll 4
      for (int k = warp; k < n; k += kJoinWarps) {
        const float half = ex2(.5f * reference_less(m, base, scalar(first_of + k, 0), scalar(first_of + k, 1)));
        weights[k][lane] = half;
        l += scaled(scalar(first_of + k, 2), half);
      }
    }
    __syncthreads();
    if (live) {
#pragma unroll 4
      for (int k = 0; k < n; ++k) {
        const float4* x = reinterpret_cast<const float4*>(slot_of(first_of + k)) + row;
        const float half = weights[k][lane];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const float4 a = x[2 * (warp * kPer + j) * kTileRows], c = x[(2 * (warp * kPer + j) + 1) * kTileRows];
          const float f[8] = {a.x, a.y, a.z, a.w, c.x, c.y, c.z, c.w};
#pragma unroll
          for (int e = 0; e < 8; ++e) o[j][e] += scaled(f[e], half);
        }
      }
    }
  }
  sums[warp][lane] = l;
  __syncthreads();
  if (!live) return;
  l = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) l += sums[w][lane];
  const int i = r / A.G;
  if (i >= sq.count) l = 0.f;
  if (stuck) l = NAN;
  const int64_t to = ((int64_t)b * A.W + i) * (A.c.H * A.G) + h * A.G + (r - i * A.G);
  const float by = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int c8 = warp * kPer + j;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[j][e] = l == 0.f ? 0.f : o[j][e] * by;
    if (A.out_vec) {
      reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(A.out) + to * kD)[c8] = A.bf16 ? Num<SDV_BF16>::pack(o[j]) : Num<SDV_F16>::pack(o[j]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) put_out(A, to * kD + 8 * c8 + e, o[j][e]);
    }
  }
  if (A.lse && warp == 0) A.lse[to] = lse_of(m, l, base);
}

template <int kD>
static cudaError_t launch_tree_rows(const TreeRowsArgs& T, cudaStream_t s) {
  using S = TreeShape<kD>;
  const auto kern = k_tree_rows<kD>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
  if (e != cudaSuccess) return e;
  kern<<<(unsigned)(T.teams * T.a.RT), kTreeThreads, S::kSmem, s>>>(T);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)T.a.B * T.a.c.H * T.a.RT * (kTileRows / 32)));
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_tree_join<kD>, T);
}

}  // namespace sdv
