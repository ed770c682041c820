// sdv_tree_rows.cuh - the tree attention for many rows, on the fifth-generation matrix unit.
//
// A CTA takes up to 128 rows (nodes times the query heads of a key head) through the keys in steps of 128:
//   S = Q K' (tensor memory, fp32), P = 2^(S f - m) vs, O += P V.
// A row is a lane of tensor memory and a thread of a softmax warp, so that its maximum and sum need no exchange; a page's
// scales are one number for 16 keys or more.  Three kinds of warps work at once:
//   * loading warps read codes (registers, a step ahead) and widen them into the matrix unit's operands:
//     keys to f16 (exact, NaN stays NaN), values to bf16 (exact: an e4m3 code is a bf16 number times 2^120);
//   * one thread issues the products;
//   * two groups of softmax warps take the steps in turn, each with scores and sums of its own, joined at the
//     end of a segment.
// Queries go through f16: bf16 ones under a power of two of their row.  Probabilities times their value's scale
// stand in tensor memory in place of their scores, as the sum of two bf16 (2^-17 of each; bf16 has fp32's range, so
// that no page's scale costs another page's bits).
//
// The steps of all (sequence, head) items, laid end to end, are cut into equal runs, one for each team of as many CTAs as
// an item has tiles of 128 rows: a team's CTAs read the same keys at about the same time, so that DRAM gives them once.
#pragma once

#include "sdv_attend.cuh"
#include "sdv_tcgen05.cuh"

namespace sdv {

constexpr int kTileRows = 128;
constexpr int kSoftWarps = 8, kLoadWarps = 8;
constexpr int kTreeThreads = 32 * (kSoftWarps + kLoadWarps + 1);
constexpr int kLoadThreads = 32 * kLoadWarps;
constexpr int kStages = 2;
constexpr int kSegRing = 8, kScaleRing = 4;
constexpr int kTileChunks = kTileKeys / kChunk;
constexpr float kMostPlain = 0x1p20f;             // a reference from where on scores are rounded before it is taken off
constexpr int kMinTileSteps = 2;                  // of a run, where there are fewer steps than teams could take

// Steps [step0, step0 + steps) of an item; steps = 0: no more.
struct Segment {
  int b, h, step0, steps, len, count, whole, slot;
};

struct TreeSmall {
  uint64_t k_full[kStages], v_full[kStages], k_free[kStages], v_free[kStages];
  uint64_t s_full[2], p_full[2], o_full, drained;
  uint64_t q_full[kSegRing];
  uint64_t soft, load, half[2];                   // the softmax warps', loading warps', a group's meeting points
  Segment segs[kSegRing];
  float downs[kSegRing][kTileRows];               // what a row's queries were divided by
  float scales[kScaleRing][2 * kTileChunks];      // ks, then vs of a step's chunks
  uint32_t absent[kScaleRing];                    // chunks that are not there; bit 31: an ordinary step (see soft_tile)
  uint32_t nans[kScaleRing][kLoadWarps];          // whether a loading warp met NaN among the values
  uint32_t nan_keys[2][4];
  float ml[2][2][kTileRows];
  uint32_t tmem;
  int dead;
};

template <int kD>
struct TreeShape {
  static constexpr int kTile = kTileKeys * kD * 2;                  // bytes of an operand
  static constexpr int kBlock = kTileRows * 128;                     // of [128 rows][64 elements]
  static constexpr int kVBlock = kD * 128;                           // of [D rows][64 keys]
  static constexpr int kQ = 0, kK = kTile, kV = kK + kStages * kTile, kSmallAt = kV + kStages * kTile;
  static constexpr size_t kSmem = 1024 + kSmallAt + sizeof(TreeSmall);
  static constexpr int kSlot = kTileRows * (kD + 2);
  static constexpr int kLoads = kD / 32;                             // sixteens of a thread's keys, and of its values
  static_assert(kSmem <= 227 * 1024, "");
};

struct TreeRowsArgs {
  AttendArgs a;                    // RT: row tiles, R: rows; part: 2 slots a CTA
  int rows, teams;                 // rows of a tile; teams of RT CTAs
};

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

// Four codes as bf16: the exponent and mantissa bits stand for 2^-120 of the value, where bf16's are.
__device__ __forceinline__ uint32_t bf16_of(uint32_t x) {        // codes in bytes 1 and 3
  const uint32_t bits = (x & 0x80008000u) | (x >> 4 & 0x07f007f0u);
  const __nv_bfloat162 up = __halves2bfloat162(__ushort_as_bfloat16(0x7b80), __ushort_as_bfloat16(0x7b80));   // 2^120
  const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&bits), up);
  return *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ void widen4_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  lo = bf16_of(__byte_perm(w, 0, 0x1404));
  hi = bf16_of(__byte_perm(w, 0, 0x3424));
}
// The bytes' top bits tell which of four codes are NaN.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// ------------------------------------------------------------------------------ loading warps
template <int kD>
struct Loader {
  using S = TreeShape<kD>;
  static constexpr int kN = S::kLoads;
  static constexpr int kPieces = kD / 16;                 // of a key
  static constexpr int kKeysOf = kLoadThreads / kPieces;  // keys that the threads take at once
  const AttendArgs& A;
  uint8_t* smem;
  TreeSmall& sm;
  int lt, lane, warp;
  uint4 kr[kN], vr[kN];                                   // codes of the step to come
  float ks, vs;
  bool gone;                                              // this lane's chunk (lanes 0 .. 7 of the first warp)

  __device__ __forceinline__ int page_of(const Segment& g, int chunk) const {
    if (chunk * kChunk >= g.len) return -1;
    const int p = __ldg(A.c.table + (int64_t)g.b * A.c.max_pages + A.cpb.over(chunk));
    return p >= 0 && p < (int)A.c.pages ? p : -1;
  }
  __device__ __forceinline__ void load_keys(const Segment& g, int step) {
    const int c0 = step * kTileChunks;
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const int key = lt / kPieces + j * kKeysOf, chunk = c0 + key / kChunk, p = page_of(g, chunk);
      kr[j] = make_uint4(0, 0, 0, 0);
      if (p >= 0)
        kr[j] = __ldg(reinterpret_cast<const uint4*>(A.c.k + (((int64_t)p * A.c.H + g.h) * A.c.block + A.cpb.rest(chunk) * kChunk + (key & (kChunk - 1))) * kD +
                                                     lt % kPieces * 16));
    }
    if (warp == 0 && lane < kTileChunks) {
      const int chunk = c0 + lane, p = page_of(g, chunk);
      gone = p < 0;
      ks = gone ? 1.f : __ldg(A.c.ks + (int64_t)p * A.c.H + g.h);
      vs = gone ? 0.f : __ldg(A.c.vs + (int64_t)p * A.c.H + g.h);
      if (gone && chunk * kChunk < g.len && A.status) atomicOr(A.status + g.b, SDV_STATUS_BAD_PAGE);
    }
  }
  __device__ __forceinline__ void load_values(const Segment& g, int step) {
    const int chunk = step * kTileChunks + (lt & (kTileChunks - 1)), p = page_of(g, chunk);
    const uint8_t* from = A.c.v + (((int64_t)max(p, 0) * A.c.H + g.h) * kD + lt / kTileChunks) * A.c.block + A.cpb.rest(chunk) * kChunk;
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      vr[j] = make_uint4(0, 0, 0, 0);
      if (p >= 0) vr[j] = __ldg(reinterpret_cast<const uint4*>(from + (int64_t)j * (kLoadThreads / kTileChunks) * A.c.block));
    }
  }
  // A sixteen's two pieces; lanes of the second block write theirs the other way round: no two lanes meet in a bank.
  __device__ __forceinline__ void put(uint8_t* block, int row, int piece, bool other, const uint4& a, const uint4& b) {
    *reinterpret_cast<uint4*>(block + swizzled(row, piece + other)) = other ? b : a;
    *reinterpret_cast<uint4*>(block + swizzled(row, piece + !other)) = other ? a : b;
  }
  __device__ __forceinline__ void put_keys(int stage, int t) {
    uint8_t* tile = smem + S::kK + stage * S::kTile;
    const int p = lt % kPieces;
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      uint4 a, b;
      widen4(kr[j].x, a.x, a.y);
      widen4(kr[j].y, a.z, a.w);
      widen4(kr[j].z, b.x, b.y);
      widen4(kr[j].w, b.z, b.w);
      put(tile + (p >> 2) * S::kBlock, lt / kPieces + j * kKeysOf, (p & 3) * 2, p >> 2 & 1, a, b);
    }
    if (warp == 0) {
      const bool plain = gone ? false : ks >= 0.f && ks < INFINITY && fabsf(vs) < INFINITY;
      const uint32_t absent = __ballot_sync(0xffffffffu, lane < kTileChunks && gone), fine = __ballot_sync(0xffffffffu, lane >= kTileChunks || plain);
      if (lane < kTileChunks) {
        sm.scales[t & (kScaleRing - 1)][lane] = ks;
        sm.scales[t & (kScaleRing - 1)][kTileChunks + lane] = vs;
      }
      if (lane == 0) sm.absent[t & (kScaleRing - 1)] = absent | (fine == 0xffffffffu ? 0x80000000u : 0u);
    }
  }
  __device__ __forceinline__ void put_values(int stage, int t) {
    uint8_t* tile = smem + S::kV + stage * S::kTile;
    const int c = lt & (kTileChunks - 1);
    uint32_t nan = 0;
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      uint4 a, b;
      widen4_bf16(vr[j].x, a.x, a.y);
      widen4_bf16(vr[j].y, a.z, a.w);
      widen4_bf16(vr[j].z, b.x, b.y);
      widen4_bf16(vr[j].w, b.z, b.w);
      nan |= nan_codes(vr[j].x) | nan_codes(vr[j].y) | nan_codes(vr[j].z) | nan_codes(vr[j].w);
      put(tile + (c >> 2) * S::kVBlock, lt / kTileChunks + j * (kLoadThreads / kTileChunks), (c & 3) * 2, c >> 2 & 1, a, b);
    }
    const bool any = __any_sync(0xffffffffu, nan);
    if (lane == 0) sm.nans[t & (kScaleRing - 1)][warp] = any;
  }
  // The rows' queries, two threads a row.
  __device__ __forceinline__ void put_queries(const Segment& g, int rt, int rows, int seg) {
    const int row = lt >> 1, half = lt & 1, r = rt * rows + row, i = r / A.G;
    const bool live = row < rows && r < A.R && i < g.count;
    const int64_t at = live ? g.b * A.q_sb + i * A.q_st + (int64_t)(g.h * A.G + r - i * A.G) * A.q_sh : 0;
    constexpr int kEights = kD / 16;                      // of a thread
    float most = 0.f;
    uint4 v[kEights];
#pragma unroll
    for (int e = 0; e < kEights; ++e) {
      v[e] = live ? q_load8(A, at + (half * kEights + e) * 8) : make_uint4(0, 0, 0, 0);
      if (A.bf16) most = fmaxf(most, q_largest(v[e], true));
    }
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
    const int up = A.bf16 && most > 0.f ? min(max(15 - log2_of(most), -112), 100) : 0;   // takes the largest to [2^15, 2^16)
#pragma unroll
    for (int e = 0; e < kEights; ++e) {
      const int e8 = half * kEights + e;
      if (A.bf16) {
        float f[8];
        Num<SDV_BF16>::unpack(v[e], f);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] *= pow2(up);
        v[e] = Num<SDV_F16>::pack(f);
      }
      *reinterpret_cast<uint4*>(smem + S::kQ + (e8 >> 3) * S::kBlock + swizzled(row, e8 & 7)) = v[e];
    }
    if (half == 0) sm.downs[seg & (kSegRing - 1)][row] = pow2(-up);
  }
};

template <int kD>
__device__ __forceinline__ void load_role(const TreeRowsArgs& T, uint8_t* smem, TreeSmall& sm, int team, int rt, int tid) {
  using S = TreeShape<kD>;
  const AttendArgs& A = T.a;
  Loader<kD> L{A, smem, sm};
  L.lt = tid, L.lane = tid & 31, L.warp = tid >> 5;
  const int lane = L.lane;
  Meeting meet{&sm.load, 0};
  int* dead = &sm.dead;
  // the run's segments, by the first warp
  const int per = A.c.H;
  int64_t u = 0, u_end = 0, seq_u = 0;
  int b = 0;
  bool first = true;
  if (L.warp == 0) {
    const int64_t units = step_sums<true, kTileKeys>(A, 0, lane).total * per;
    const int runs = tree_runs(units, T.teams);
    if (team < runs) {
      u = run_start(units, team, runs);
      u_end = run_start(units, team + 1, runs);
      const Found f = find_sequence<true, kTileKeys>(A, u / per, lane);
      b = f.b;
      seq_u = f.before * per;
    }
  }
  auto next_segment = [&](int seg) {
    if (L.warp) return;
    Segment g{};
    while (u < u_end && b < A.B) {
      Seq sq = seq_of<true, kTileKeys>(A, b);
      const int64_t mine = (int64_t)sq.steps * per;
      if (u >= seq_u + mine) {                            // on to the next sequence, or over empty ones
        seq_u += mine;
        if (++b == A.B) break;
        if (!seq_of<true, kTileKeys>(A, b).steps) {
          const Found f = find_sequence<true, kTileKeys>(A, u / per, lane);
          b = f.b;
          seq_u = f.before * per;
        }
        continue;
      }
      if (u < seq_u) break;                               // (only if the lengths have changed meanwhile)
      const int item = (int)((u - seq_u) / sq.steps);
      const int64_t item_u = seq_u + (int64_t)item * sq.steps;
      g.b = b, g.h = item, g.step0 = (int)(u - item_u);
      g.steps = (int)min((int64_t)sq.steps, u_end - item_u) - g.step0;
      g.len = sq.len, g.count = sq.count;
      g.whole = g.steps == sq.steps;
      g.slot = first ? 0 : 1;
      first = false;
      u += g.steps;
      break;
    }
    if (lane == 0) sm.segs[seg & (kSegRing - 1)] = g;
  };
  next_segment(0);
  if (!meet(lane, dead)) return;
  int t = 0;
#pragma unroll 1
  for (int seg = 0;; ++seg) {
    const Segment g = sm.segs[seg & (kSegRing - 1)];
    if (g.steps && seg == 0) {
      L.load_keys(g, g.step0);
      L.load_values(g, g.step0);
    }
    if (g.steps) {
      next_segment(seg + 1);
      if (t && !warp_wait(&sm.k_free[(t - 1) % kStages], (t - 1) / kStages & 1, dead)) return;   // its last scores are had
      L.put_queries(g, rt, T.rows, seg);
      fence_async();
    }
    warp_arrive(&sm.q_full[seg & (kSegRing - 1)], lane);
    if (!g.steps) return;
#pragma unroll 1
    for (int n = 0; n < g.steps; ++n, ++t) {
      const int st = t % kStages;
      const uint32_t before = (t / kStages - 1) & 1;
      if (t >= kStages && !warp_wait(&sm.k_free[st], before, dead)) return;
      L.put_keys(st, t);
      fence_async();
      warp_arrive(&sm.k_full[st], lane);
      Segment ng = g;
      int step = g.step0 + n + 1;
      if (n + 1 == g.steps) {
        if (!meet(lane, dead)) return;
        ng = sm.segs[(seg + 1) & (kSegRing - 1)];
        step = ng.step0;
      }
      if (ng.steps) L.load_keys(ng, step);
      if (t >= kStages && !warp_wait(&sm.v_free[st], before, dead)) return;
      L.put_values(st, t);
      fence_async();
      warp_arrive(&sm.v_full[st], lane);
      if (ng.steps) L.load_values(ng, step);
    }
  }
}

// ------------------------------------------------------------------------------ the thread that issues the products
template <int kD>
__device__ __forceinline__ void mma_role(uint8_t* smem, TreeSmall& sm) {
  using S = TreeShape<kD>;
  int* dead = &sm.dead;
  const uint32_t base = sm.tmem, q = smem_addr(smem + S::kQ);
  constexpr uint32_t kScore = mma_desc(0, kTileRows, kTileKeys), kOut = mma_desc(1, kTileRows, kD);
  int t = 0;
  auto scores = [&](int t) {
    const int st = t % kStages;
    if (!barrier_wait(&sm.k_full[st], t / kStages & 1, dead)) return false;
    tmem_after_sync();
    const uint32_t k = smem_addr(smem + S::kK + st * S::kTile);
#pragma unroll
    for (int i = 0; i < kD / 16; ++i) {
      const uint32_t off = (i >> 2) * S::kBlock + (i & 3) * 32;
      mma_ss(base + (t & 1) * kTileKeys, tile_desc(q + off), tile_desc(k + off), kScore, i > 0);
    }
    mma_commit(&sm.s_full[t & 1]);
    mma_commit(&sm.k_free[st]);
    return true;
  };
#pragma unroll 1
  for (int seg = 0;; ++seg) {
    if (!barrier_wait(&sm.q_full[seg & (kSegRing - 1)], seg / kSegRing & 1, dead)) break;
    const int steps = sm.segs[seg & (kSegRing - 1)].steps;
    if (!steps || !scores(t)) break;
    bool ok = true;
#pragma unroll 1
    for (int n = 0; n < steps && ok; ++n, ++t) {
      if (n + 1 < steps) ok = scores(t + 1);
      const int st = t % kStages, s = t & 1;
      ok = ok && barrier_wait(&sm.p_full[s], t >> 1 & 1, dead) && barrier_wait(&sm.v_full[st], t / kStages & 1, dead);
      if (!ok) break;
      tmem_after_sync();
      const uint32_t v = smem_addr(smem + S::kV + st * S::kTile), out = base + 2 * kTileKeys + s * 128;
#pragma unroll
      for (int i = 0; i < kTileKeys / 16; ++i) {
        const uint64_t vd = tile_desc(v + (i >> 2) * S::kVBlock + (i & 3) * 32);
        const uint32_t p = base + s * kTileKeys + (i >> 1) * 32 + (i & 1) * 8;
        mma_ts(out, p, vd, kOut, i > 0 || n >= 2);
        mma_ts(out, p + 16, vd, kOut, true);
      }
      mma_commit(&sm.v_free[st]);
      if (n + 1 == steps) mma_commit(&sm.o_full);
    }
    if (!ok) break;
  }
  mma_commit(&sm.drained);                                // nothing is under way when the memory is given back
  int ignore = 0;
  barrier_wait(&sm.drained, 0, &ignore);
}

// ------------------------------------------------------------------------------ softmax warps
// What a row sees of a step's 128 keys, as bits.
struct Bits128 {
  uint64_t lo, hi;
};
__device__ __forceinline__ Bits128 below(int n) {         // the first n
  return Bits128{n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1, n >= 128 ? ~0ull : n <= 64 ? 0ull : (1ull << (n - 64)) - 1};
}
__device__ __forceinline__ Bits128 placed(uint64_t set, int at) {   // bit 0 in place `at`, -64 < at < 128
  if (at <= 0) return Bits128{set >> -at, 0};
  if (at < 64) return Bits128{set << at, set >> (64 - at)};
  return Bits128{0, set << (at - 64)};
}
__device__ __forceinline__ uint32_t word(const Bits128& x, int i) { return (uint32_t)((i & 2 ? x.hi : x.lo) >> (i & 1 ? 32 : 0)); }

// A row's step: scores in columns [at, at + 128) become probabilities times their values' scale, in halves (of each 32 scores
// sixteen columns of first ones, sixteen of second ones, in their place); l goes on.
// kPlain: every row sees every key, no scale is negative or none, no code NaN, no reference large.  Else what a row does
// not see gets 0, and of what it sees NaN is what has no number; and the score is rounded before the reference is
// taken off: the fused product is off by half a step of the reference, which large scores make a large power.
template <bool kPlain>
__device__ __forceinline__ void soft_probs(uint32_t at, const float* scales, float f0, const Bits128& sees, const Bits128& nans, float m, float& l) {
  uint32_t r[32];
  f32x2 sum = pair(0.f, 0.f);
  const f32x2 nm = pair(-m, -m);
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    tmem_load32(at + 32 * g, r);
    tmem_loaded(r);
    uint32_t w = 0, bad = 0;
    if constexpr (!kPlain) w = word(sees, g), bad = word(nans, g);
    uint32_t o[32];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float f = f0 * scales[2 * g + c], vs = scales[kTileChunks + 2 * g + c];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int k = 16 * c + 2 * e;
        const float x0 = __uint_as_float(r[k]), x1 = __uint_as_float(r[k + 1]);
        float2 p;
        f32x2 v;
        if constexpr (kPlain) {
          const float2 x = unpair(fma2(pair(x0, x1), pair(f, f), nm));
          p = make_float2(ex2(x.x), ex2(x.y));
          v = mul2(pair(p.x, p.y), pair(vs, vs));
        } else {
          const bool none = !(fabsf(vs) < INFINITY) || !(fabsf(f) < INFINITY);
          p = make_float2(ex2(__fmul_rn(x0, f) - m), ex2(__fmul_rn(x1, f) - m));
          p.x = !(w >> k & 1) ? 0.f : none || (bad >> k & 1) ? NAN : p.x;
          p.y = !(w >> (k + 1) & 1) ? 0.f : none || (bad >> (k + 1) & 1) ? NAN : p.y;
          v = none ? pair(p.x, p.y) : mul2(pair(p.x, p.y), pair(vs, vs));
        }
        sum = add2(sum, pair(p.x, p.y));
        const float2 y = unpair(v);
        const __nv_bfloat162 h = __floats2bfloat162_rn(y.x, y.y);
        const uint32_t hw = *reinterpret_cast<const uint32_t*>(&h);
        const __nv_bfloat162 lo = __floats2bfloat162_rn(y.x - __uint_as_float(hw << 16), y.y - __uint_as_float(hw & 0xffff0000u));
        o[8 * c + e] = hw;
        o[16 + 8 * c + e] = *reinterpret_cast<const uint32_t*>(&lo);
      }
    }
    tmem_store32(at + 32 * g, o);
  }
  const float2 s2 = unpair(sum);
  l += s2.x + s2.y;
  tmem_stored();
}

// The whole step: the row's largest score first, against which its reference m may move (`more`: O holds sums already).
template <int kD, bool kPlain>
__device__ __forceinline__ void soft_tile(uint32_t at, uint32_t out, const float* scales, float f0, const Bits128& sees, const Bits128& nans,
                                          bool more, float& m, float& l) {
  float top = -INFINITY;
  uint32_t r[32];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    tmem_load32(at + 32 * g, r);
    tmem_loaded(r);
    if constexpr (kPlain) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x = __uint_as_float(r[16 * c]);
#pragma unroll
        for (int e = 1; e < 16; ++e) x = fmaxf(x, __uint_as_float(r[16 * c + e]));
        top = fmaxf(top, x * (f0 * scales[2 * g + c]));
      }
    } else {
      const uint32_t w = word(sees, g);
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const float x = __uint_as_float(r[e]) * (f0 * scales[2 * g + e / 16]);
        top = w >> e & 1 ? fmaxf(top, x) : top;
      }
    }
  }
  // the reference moves when a score passes it by 2^kSlack
  const bool move = top > m + kSlack;
  if (__any_sync(0xffffffffu, move)) {
    const float now = move ? top : m, c = ex2(m - now);
    m = now;
    l *= c;
    if (more) {
#pragma unroll 1
      for (int g = 0; g < kD / 32; ++g) {
        tmem_load32(out + 32 * g, r);
        tmem_loaded(r);
#pragma unroll
        for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * c);
        tmem_store32(out + 32 * g, r);
      }
      tmem_stored();
    }
  }
  if (kPlain && !__any_sync(0xffffffffu, fabsf(m) > kMostPlain)) {
    soft_probs<true>(at, scales, f0, sees, nans, m, l);
  } else {
    const Bits128 all{~0ull, ~0ull};
    soft_probs<false>(at, scales, f0, kPlain ? all : sees, nans, m, l);
  }
}

template <int kD>
__device__ __forceinline__ void soft_role(const TreeRowsArgs& T, uint8_t* smem, TreeSmall& sm, int team, int rt, int tid) {
  using S = TreeShape<kD>;
  const AttendArgs& A = T.a;
  const int lane = tid & 31, warp = tid >> 5, s = warp >> 2, row = (warp & 3) * 32 + lane;
  int* dead = &sm.dead;
  const uint32_t lanes = sm.tmem + ((uint32_t)((warp & 3) * 32) << 16);
  const uint32_t at = lanes + s * kTileKeys, out = lanes + 2 * kTileKeys;
  Meeting meet{&sm.soft, 0}, meet_half{&sm.half[s], 0};
  const int r = rt * T.rows + row, i = r / A.G;
  int t = 0;
#pragma unroll 1
  for (int seg = 0;; ++seg) {
    if (!warp_wait(&sm.q_full[seg & (kSegRing - 1)], seg / kSegRing & 1, dead)) return;
    const Segment g = sm.segs[seg & (kSegRing - 1)];
    if (!g.steps) return;
    const bool have = row < T.rows && r < A.R, live = have && i < g.count;
    const bool busy = __any_sync(0xffffffffu, live);
    uint64_t set;
    {
      bool bad = false;
      const int32_t* parents = A.parents + (int64_t)g.b * A.W;
      uint64_t a0, a1;
      ancestors(lane < A.W ? parent_of(parents[lane], lane, bad) : -1, 32 + lane < A.W ? parent_of(parents[32 + lane], 32 + lane, bad) : -1,
                lane, a0, a1);
      const uint64_t lo = __shfl_sync(0xffffffffu, a0, i & 31), hi = __shfl_sync(0xffffffffu, a1, i & 31);
      set = !live ? 0 : i < 32 ? lo : hi;
    }
    const float f0 = A.scale2 * sm.downs[seg & (kSegRing - 1)][row];
    const int at0 = g.len - g.count;                      // the root's place
    float m = kNone, l = 0.f;
    int done = 0;                                          // this group's steps of the segment
    const int t_end = t + g.steps;
    const bool any0 = g.steps > 1 || !(t & 1), any1 = g.steps > 1 || (t & 1);
#pragma unroll 1
    for (int n = 0; t < t_end; ++t, ++n) {
      if ((t & 1) != s) continue;
      if (!warp_wait(&sm.v_full[t % kStages], t / kStages & 1, dead) || !warp_wait(&sm.s_full[s], t >> 1 & 1, dead)) return;
      tmem_after_sync();
      const int slot = t & (kScaleRing - 1), key0 = (g.step0 + n) * kTileKeys;
      const uint32_t absent = sm.absent[slot];
      uint32_t nan = 0;
#pragma unroll
      for (int k = 0; k < kLoadWarps; ++k) nan |= sm.nans[slot][k];
      const Bits128 none{0, 0};
      if (absent >> 31 && !nan && key0 + kTileKeys <= at0 && A.scale2 >= 0.f) {
        if (busy) soft_tile<kD, true>(at, out + s * 128, sm.scales[slot], f0, none, none, done > 0, m, l);
      } else {
        Bits128 nans = none;
        if (nan) {                                         // which keys' values: a thread a key
          const uint8_t* tile = smem + S::kV + (t % kStages) * S::kTile + (row >> 6) * S::kVBlock;
          bool mine = false;
#pragma unroll 1
          for (int d = 0; d < kD; ++d)
            mine |= (*reinterpret_cast<const uint16_t*>(tile + swizzled(d, (row & 63) >> 3) + (row & 7) * 2) & 0x7fff) == 0x43f0;   // 480
          const uint32_t w = __ballot_sync(0xffffffffu, mine);
          if (lane == 0) sm.nan_keys[s][warp & 3] = w;
          if (!meet_half(lane, dead)) return;
          nans = Bits128{sm.nan_keys[s][0] | (uint64_t)sm.nan_keys[s][1] << 32, sm.nan_keys[s][2] | (uint64_t)sm.nan_keys[s][3] << 32};
          if (!meet_half(lane, dead)) return;
        }
        if (busy) {
          Bits128 sees = below(at0 - key0);
          if (at0 - key0 > -64 && at0 - key0 < kTileKeys) {
            const Bits128 tree = placed(set, at0 - key0);
            sees.lo |= tree.lo, sees.hi |= tree.hi;
          }
#pragma unroll
          for (int c = 0; c < kTileChunks; ++c)
            if (absent >> c & 1) (c < 4 ? sees.lo : sees.hi) &= ~(0xffffull << (16 * (c & 3)));
          if (!live) sees = none;
          soft_tile<kD, false>(at, out + s * 128, sm.scales[slot], f0, sees, nans, done > 0, m, l);
        }
      }
      ++done;
      tmem_before_sync();
      warp_arrive(&sm.p_full[s], lane);
    }
    // the segment's rows: both groups' sums, a half of the columns each
    if (!warp_wait(&sm.o_full, seg & 1, dead)) return;
    tmem_after_sync();
    sm.ml[s][0][row] = m;
    sm.ml[s][1][row] = l;
    if (!meet(lane, dead)) return;
    if (busy || (__any_sync(0xffffffffu, have))) {
      const float m0 = sm.ml[0][0][row], m1 = sm.ml[1][0][row], l0 = sm.ml[0][1][row], l1 = sm.ml[1][1][row];
      const float top = fmaxf(m0, m1), c0 = ex2(m0 - top), c1 = ex2(m1 - top);
      const float sum = live ? l0 * c0 + l1 * c1 : 0.f, by = !g.whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
      const int64_t to = ((int64_t)g.b * A.W + i) * (A.c.H * A.G) + g.h * A.G + (r - i * A.G);
      float* part = A.part + ((int64_t)(blockIdx.x * 2 + g.slot)) * S::kSlot;
#pragma unroll 1
      for (int k = 0; k < kD / 64; ++k) {
        const int col = s * (kD / 2) + 32 * k;
        uint32_t a[32];
        float o[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0.f;
        if (busy && any0) {
          tmem_load32(out + col, a);
          tmem_loaded(a);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(a[e]) * c0;
        }
        if (busy && any1) {
          tmem_load32(out + 128 + col, a);
          tmem_loaded(a);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = fmaf(__uint_as_float(a[e]), c1, o[e]);
        }
        if (!have) continue;
        if (g.whole) {
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
        } else {
          float4* y = reinterpret_cast<float4*>(part + (int64_t)row * kD + col);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        }
      }
      if (have && s == 0) {
        if (g.whole) {
          if (A.lse) A.lse[to] = lse_of(top, sum, 0.f);
        } else {
          part[kTileRows * kD + row] = top;
          part[kTileRows * kD + kTileRows + row] = sum;
        }
      }
    }
    tmem_before_sync();
    if (!meet(lane, dead)) return;                         // the sums are read: the next products may come
  }
}

template <int kD>
__global__ void __launch_bounds__(kTreeThreads, 1) k_tree_rows(const TreeRowsArgs T) {
  using S = TreeShape<kD>;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = raw + (-smem_addr(raw) & 1023);
  TreeSmall& sm = *reinterpret_cast<TreeSmall*>(smem + S::kSmallAt);
  const int tid = threadIdx.x, warp = tid >> 5, team = blockIdx.x / T.a.RT, rt = blockIdx.x - team * T.a.RT;
  if (warp == kSoftWarps + kLoadWarps) tmem_alloc(&sm.tmem, 512);
  if (tid == 0) {
    for (int k = 0; k < kStages; ++k) {
      barrier_init(&sm.k_full[k], kLoadWarps);
      barrier_init(&sm.v_full[k], kLoadWarps);
      barrier_init(&sm.k_free[k], 1);
      barrier_init(&sm.v_free[k], 1);
    }
    for (int k = 0; k < 2; ++k) {
      barrier_init(&sm.s_full[k], 1);
      barrier_init(&sm.p_full[k], kSoftWarps / 2);
      barrier_init(&sm.half[k], kSoftWarps / 2);
    }
    for (int k = 0; k < kSegRing; ++k) barrier_init(&sm.q_full[k], kLoadWarps);
    barrier_init(&sm.o_full, 1);
    barrier_init(&sm.drained, 1);
    barrier_init(&sm.soft, kSoftWarps);
    barrier_init(&sm.load, kLoadWarps);
    sm.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tmem_before_sync();
  __syncthreads();
  tmem_after_sync();
  if (warp < kSoftWarps) soft_role<kD>(T, smem, sm, team, rt, tid);
  else if (warp < kSoftWarps + kLoadWarps) load_role<kD>(T, smem, sm, team, rt, tid - 32 * kSoftWarps);
  else if (tid == 32 * (kSoftWarps + kLoadWarps)) mma_role<kD>(smem, sm);
  __syncwarp();
  tmem_before_sync();
  __syncthreads();
  tmem_after_sync();
  if (warp == kSoftWarps + kLoadWarps) tmem_free(sm.tmem, 512);
  if (sm.dead && tid == 0 && T.a.status) atomicOr(T.a.status, SDV_STATUS_STUCK);
}

// Joins the partials of an item that several teams' runs hold; an item without steps gets zeros.  A warp a row.
template <int kD>
__global__ void __launch_bounds__(kJoinThreads) k_tree_join(const TreeRowsArgs T) {
  using S = TreeShape<kD>;
  constexpr int kV = kD / 32;
  const AttendArgs& A = T.a;
  constexpr int kCtas = kTileRows / kJoinWarps;             // of an item
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int ib = blockIdx.x / kCtas, row = blockIdx.x % kCtas * kJoinWarps + warp;
  const int per = A.c.H * A.RT, b = ib / per, item = ib % per, h = item / A.RT, rt = item % A.RT, r = rt * T.rows + row;
  const Sums ts = step_sums<true, kTileKeys>(A, b, lane);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (A.status && item == 0 && row == 0) {
    bool bad = lane == 0 && A.lengths[b] < min(A.counts ? A.counts[b] : A.W, A.W);
    for (int i = lane; i < min(A.counts ? A.counts[b] : A.W, A.W); i += 32) parent_of(A.parents[(int64_t)b * A.W + i], i, bad);
    if (bad) atomicOr(A.status + b, SDV_STATUS_BAD_TREE);
    if (lane == 0 && A.lengths[b] > A.c.max_pages * A.c.block) atomicOr(A.status + b, SDV_STATUS_BAD_PAGE);
  }
  if (row >= T.rows || r >= A.R) return;
  const Seq sq = seq_of<true, kTileKeys>(A, b);
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
    if (g0 == g1) return;                                   // written by that run's CTA
  }
  const int64_t first = g0 <= g1 && run_start(units, g0, runs) < u0 ? 1 : 0;
  auto slot_of = [&](int gi) { return A.part + (((int64_t)gi * A.RT + rt) * 2 + (gi == g0 ? first : 0)) * S::kSlot; };
  float m = kNone;
  for (int gi = g0 + lane; gi <= g1; gi += 32) m = fmaxf(m, slot_of(gi)[kTileRows * kD + row]);
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float l = 0.f, o[kV];
#pragma unroll
  for (int e = 0; e < kV; ++e) o[e] = 0.f;
#pragma unroll 4
  for (int gi = g0; gi <= g1; ++gi) {
    const float* slot = slot_of(gi);
    const float c = ex2(slot[kTileRows * kD + row] - m);
    l = fmaf(c, slot[kTileRows * kD + kTileRows + row], l);
#pragma unroll
    for (int e = 0; e < kV; ++e) o[e] = fmaf(c, slot[(int64_t)row * kD + e * 32 + lane], o[e]);
  }
  const int i = r / A.G;
  if (i >= sq.count) l = 0.f;
  const int64_t to = ((int64_t)b * A.W + i) * (A.c.H * A.G) + h * A.G + (r - i * A.G);
  const float by = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < kV; ++e) put_out(A, to * kD + e * 32 + lane, l == 0.f ? 0.f : o[e] * by);
  if (A.lse && lane == 0) A.lse[to] = lse_of(m, l, 0.f);
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
  cfg.gridDim = dim3((unsigned)((int64_t)T.a.B * T.a.c.H * T.a.RT * (kTileRows / kJoinWarps)));
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
