// sdv_attend.cuh - attention of a window's queries over the 8-bit cache: the kernels.
//
// For query i of sequence b (position len - count + i) and the keys up to its position:
//   s_j = scale ks_j (q . k_j),  p_j = e^{s_j - max} / sum,  out = sum_j p_j vs_j v_j.
// The G = Hq / H query heads of a key head and the window's queries are the rows of one item, so
// that a key is read once for up to 8 kMaxNt of them.  The (sequence, head, row tile) items' steps
// of 32 keys, laid end to end, are dealt out to the warps in equal runs, so that no warp waits for
// another; a run that does not hold an item's whole length leaves (max, sum, output) in the
// workspace, and k_attend_join joins them.
//
// Both products are taken transposed, S' = K Q' and O' = V' P': the cache is the operand with 16
// rows, the queries' rows come in eights, so that a single token's few heads waste little.  A warp
// reads its steps from a cp.async ring of its own.  Codes widen to f16
// exactly; with g = lane / 4 and t = lane % 4:
//   * key row g (g + 8) of score tile s is token 8 (g / 2) + 4 s + g % 2 (+ 2), which makes the tokens
//     that a thread multiplies in step s of the second product, 8 t + 4 s .. + 3, adjacent
//     bytes of a value row, and a thread's keys members of one chunk of 16 tokens: one
//     page, one pair of scales;
//   * a thread's sixteen contiguous elements of a key are its share of four steps of the first
//     product (the queries' fragments follow the same order of elements);
//   * an 8 x 8 tile of probabilities is transposed on its way to the second product (movmatrix).
//
// A row's exponentials are taken against a reference of its own, on score + log2(vs / U): what they are
// multiplied by with the values, p' = 2^(s + log2(vs / U) - m) kPScale, has to fit f16, and a row whose weight
// lies on pages of small values must keep its bits whatever the other pages hold.  The sum's terms 2^(s - m) are
// p' U / vs.  The unit U is a power of two near an item's first scale; from where a scale that rows see is far
// from it, or 0, the sums of the rest of the item are kept apart, against references on the score alone ("wide").
// Scores past 2^24, of which fp32 holds no fraction, are taken less a base of their row ("based"): an exact
// difference.  m moves only when a score passes it by 2^kSlack, so that most steps need no exchange between lanes and
// no rescaling of the output.
#pragma once

#include "sdv_cache.cuh"

namespace sdv {

constexpr int kSub = 32;                  // keys of a step
constexpr int kJoinWarps = 8;
constexpr int kJoinThreads = 32 * kJoinWarps;
constexpr int kMinSteps = 2;              // of a run, where there are fewer steps than warps could take (but see run_count)
constexpr int kMaxNt = 5;                 // eights of rows of an item
constexpr float kNone = -3e38f;           // the reference of a row that has seen nothing
constexpr float kSlack = 8.f;
constexpr float kPScale = 128.f, kLogPScale = 7.f;   // f16 holds 2^kSlack kPScale; its least step is 2^-31 of a row's largest
// What few items need: a power of two per query, sums kept apart, scores less a base (see above and k_attend).
constexpr int kUneven = 1, kWide = 2, kBased = 4;
constexpr float kMostScore = 0x1p24f;                 // a bound on the scores (as powers of 2) up to which half a step of theirs fits f16's range too
constexpr float kBaseRoom = 64.f;                     // scores less their base stay below
constexpr int kLeastUnit = -119, kMostUnit = 126;    // kPScale over the unit, and the unit over kPScale, are normal numbers
constexpr float kLeastPw = 0x1p-33f, kMostPw = 0x1p48f;   // kPScale vs / U where the sums are kept with p'

__device__ __forceinline__ float pow2(int n) { return __uint_as_float((uint32_t)(n + 127) << 23); }     // n from -126 to 127
// floor(log2 x) of x > 0 (-127 for what is below the normal numbers).
__device__ __forceinline__ int log2_of(float x) { return (int)(__float_as_uint(x) >> 23) - 127; }

// Division by the chunks of a page (up to 8) of numbers below 2^28: a product's upper half.
struct ChunkDiv {
  uint32_t magic, n;
  __device__ __forceinline__ int over(int x) const { return magic ? (int)__umulhi((uint32_t)x, magic) : x; }
  __device__ __forceinline__ int rest(int x) const { return x - over(x) * (int)n; }
};
inline ChunkDiv chunk_div(int n) { return ChunkDiv{n == 1 ? 0u : (uint32_t)((0x100000000ull + n - 1) / n), (uint32_t)n}; }

struct AttendArgs {
  const void* q;
  bool bf16, q_vec;                        // queries in whole aligned vectors of 16 bytes
  int64_t q_sb, q_st, q_sh;
  CacheView c;
  ChunkDiv cpb;
  int B, W, G, R, RT;                      // rows W * G, row tiles
  const int32_t* lengths;
  const int32_t* counts;
  float scale2;                            // scale * log2(e)
  int span;
  void* out;
  float* lse;
  uint32_t* status;
  const int64_t* prefix;                   // workspace: steps before each sequence, or NULL (few sequences)
  float* part;                             // workspace: 2 slots a warp
  int ctas;
};

// A sequence's tokens, new ones and steps.
struct Seq {
  int len, count, first, steps;            // first: the first step that a query sees
  int begin;                               // the first key that one sees
};
__device__ __forceinline__ Seq seq_of(const AttendArgs& A, int b) {
  Seq s;
  const int cap = A.c.max_pages * A.c.block;
  s.len = min(max(A.lengths[b], 0), cap);
  s.count = min(max(A.counts ? A.counts[b] : A.W, 0), A.W);
  s.begin = A.span > 0 ? max(0, s.len - s.count - A.span + 1) : 0;
  s.first = s.begin / kSub;
  s.steps = s.count && s.len ? (s.len + kSub - 1) / kSub - s.first : 0;
  return s;
}

// Steps of the sequences before b and of all (each for one head and row tile), by a warp: added up
// where the sequences are few, else looked up in what k_attend_prefix left.
struct Sums {
  int64_t before, total;
};
__device__ __forceinline__ Sums step_sums(const AttendArgs& A, int b, int lane) {
  if (A.prefix) return Sums{A.prefix[b], A.prefix[A.B]};
  Sums s{0, 0};
  for (int i = lane; i < A.B; i += 32) {
    const int t = seq_of(A, i).steps;
    s.total += t;
    if (i < b) s.before += t;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    s.before += __shfl_xor_sync(0xffffffffu, s.before, o);
    s.total += __shfl_xor_sync(0xffffffffu, s.total, o);
  }
  return s;
}
// The sequence that holds step u (of units of one head and row tile) and the steps before it, by a warp;
// b = B if there is none.
struct Found {
  int b;
  int64_t before;
};
__device__ __forceinline__ Found find_sequence(const AttendArgs& A, int64_t u, int lane) {
  if (A.prefix) {                                           // the last b with prefix[b] <= u, 32 places at a time
    int lo = 0, hi = A.B;                                   // prefix[lo] <= u < prefix[hi]
    if (u >= A.prefix[A.B]) return Found{A.B, A.prefix[A.B]};
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, at = lo + lane * step;
      const unsigned le = __ballot_sync(0xffffffffu, at < hi && A.prefix[at] <= u);
      const int k = 31 - __clz(le);                          // (lane 0 holds)
      hi = min(hi, lo + (k + 1) * step);
      lo += k * step;
    }
    return Found{lo, A.prefix[lo]};
  }
  int64_t before = 0;
  for (int b0 = 0; b0 < A.B; b0 += 32) {
    const int64_t mine = b0 + lane < A.B ? seq_of(A, b0 + lane).steps : 0;
    int64_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, before + inc > u);
    if (hit) {
      const int k = __ffs(hit) - 1;
      return Found{b0 + k, before + __shfl_sync(0xffffffffu, inc - mine, k)};
    }
    before += __shfl_sync(0xffffffffu, inc, 31);
  }
  return Found{A.B, before};
}

__device__ __forceinline__ int64_t run_start(int64_t units, int g, int runs) { return units * g / runs; }
// Runs for `units` steps of `items` items.  Where the items have a step each, a run has one: 53 x 25 rows over 8 keys and
// 8 heads take 21 us, and 29 with two steps a run; items of two steps want them together (62 x 32 rows over 48 keys and
// 4 heads: 17 us, and 23 apart).
__device__ __forceinline__ int run_count(int64_t units, int64_t items, int warps) {
  return (int)min((int64_t)warps, units <= items ? units : (units + kMinSteps - 1) / kMinSteps);
}

// Four e4m3 codes as two pairs of f16.
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{ .reg .b16 a, b;\n  mov.b32 {a, b}, %2;\n  cvt.rn.f16x2.e4m3x2 %0, a;\n  cvt.rn.f16x2.e4m3x2 %1, b; }"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void copy4(uint32_t to, const void* from, bool real) {
  const int n = real ? 4 : 0;
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(n));
}

// With more sequences than this their steps are added up once, by a kernel of its own; with fewer each
// warp does it.  4 heads of 60 tokens, without that kernel and with it: 12.5 us and 14.6 for 128
// sequences, 16.7 and 17.0 for 256, 36 and 30 for 512, 188 and 80 for 2048.
constexpr int kPrefixFrom = 256;
constexpr int kPrefixThreads = 1024;

// Warps of a CTA of k_attend, one CTA an SM, as many as its registers allow: 2 x 1 token of 64 query heads on 8, 131000
// keys, takes 97 us with 8 warps and 105 with 6, 16 x 4 tokens of 32 heads on 8, 16000 keys, 110 and 130.
constexpr int kAttendWarps = 8;

__device__ __forceinline__ void put_out(const AttendArgs& A, int64_t at, float x) {
  if (A.bf16) reinterpret_cast<__nv_bfloat16*>(A.out)[at] = __float2bfloat16_rn(x);
  else reinterpret_cast<__half*>(A.out)[at] = __float2half_rn(x);
}
__device__ __forceinline__ float lse_of(float m, float l, float base) {
  return l > 0.f ? (base + (m + log2f(l))) * kLn2f : (l == 0.f ? -INFINITY : NAN);
}

// A warp's ring holds kHalves half steps (32 keys, or their values): one in use, the others, 8 KB, under
// way; its queries' fragments are beside it.  (Four under way at D = 128, where few rows leave room: within
// 2 % either way for 4 to 36 rows.)
template <int kD, int kNt>
struct AttendShape {
  static constexpr int kWarps = kAttendWarps;
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kRows = 8 * kNt;
  static constexpr int kSlot = kRows * (kD + 2);         // floats of a partial: rows' output, max, sum
  static constexpr int kHalf = kSub * kD;                 // bytes
  static constexpr int kHalves = kD == 64 ? 5 : 3;
  static constexpr int kAhead = (kHalves - 1) / 2;        // steps
  static constexpr int kScaleSlots = kAhead + 1;
  static constexpr int kKv = kD / 64;                     // 16-byte pieces of a key for a thread
  static constexpr int kQBytes = kRows * kD * 2;
  static constexpr int kScaleBytes = kScaleSlots * 32;    // of a step: ks, vs of both chunks; absent chunks
  static constexpr int kRowBytes = kRows * 12;            // of a row: the sum's reference, the score's base, the query's power of two
  static constexpr int kWarpBytes = kHalves * kHalf + kQBytes + kScaleBytes + kRowBytes;
  static constexpr size_t kSmem = (size_t)kWarps * kWarpBytes;
  static_assert(kHalves % 2 == 1 && kSmem <= 227 * 1024, "");
};

// Eight elements of a query, as they are held.
__device__ __forceinline__ uint4 q_load8(const AttendArgs& A, int64_t at) {
  if (A.q_vec) return __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(A.q) + at));
  uint32_t w[4];
  const uint16_t* p = reinterpret_cast<const uint16_t*>(A.q) + at;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (uint32_t)p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The largest finite magnitude of eight elements of a query.
__device__ __forceinline__ float q_largest(uint4 v, bool bf16) {
  v.x &= 0x7fff7fffu, v.y &= 0x7fff7fffu, v.z &= 0x7fff7fffu, v.w &= 0x7fff7fffu;
  float m = bf16 ? vec_max_num<SDV_BF16>(v) : vec_max_num<SDV_F16>(v);
  if (!(m < INFINITY)) {
    float f[8];
    if (bf16) Num<SDV_BF16>::unpack(v, f);
    else Num<SDV_F16>::unpack(v, f);
    m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = f[e] < INFINITY ? fmaxf(m, f[e]) : m;
  }
  return m;
}

// Bytes: every key and value once for each row tile, 2 D codes a token and head; operations: 4 D a row of those.  Bound
// by DRAM where rows are few (4 or 8 a head, 2 x 131000 keys or 16 x 16000: 97 us, 5.4 to 5.5 TB/s with the join), by the two
// warps a scheduler waiting on their own instructions where there are 36 (32 windows of 9 tokens, 4 query heads a
// head, up to 16000 keys: 273 to 280 us, 2.1 TB/s and 0.15 PFLOP/s); the matrix instructions alone, 8 cycles each
// a scheduler, need 1920 cycles a step there, HBM's pace 1400.
// The probabilities go into the second product as a sum of two f16, 22 bits: with one, f16 outputs were off by as much
// as their own rounding again (2.9e-4 of their size, 2.0e-4 with two), and bf16 outputs were roundings of numbers
// up to 2^-12 off, so that some fell on the neighbouring value.  The second half costs those windows 48 us, few rows nothing.
template <int kD, int kNt>
__global__ void __launch_bounds__(AttendShape<kD, kNt>::kThreads, 1) k_attend(const AttendArgs A) {
  using S = AttendShape<kD, kNt>;
  constexpr int kKv = S::kKv;
  constexpr int kMt = kD / 16;                             // sixteens of the output
  constexpr int kR = 2 * kNt;                              // rows of a thread: 8 n + 2 t + e
  extern __shared__ __align__(16) uint8_t smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int H = A.c.H, per = H * A.RT;                     // items of a sequence
  uint8_t* ring = smem + warp * S::kWarpBytes;
  uint4* qf = reinterpret_cast<uint4*>(ring + S::kHalves * S::kHalf);
  float* scales = reinterpret_cast<float*>(ring + S::kHalves * S::kHalf + S::kQBytes);
  float* refs = reinterpret_cast<float*>(ring + S::kHalves * S::kHalf + S::kQBytes + S::kScaleBytes);   // the sums', where they are kept apart
  float* bases = refs + S::kRows;
  float* downs = bases + S::kRows;

  const int64_t units = step_sums(A, 0, lane).total * per;
  const int runs = run_count(units, (int64_t)A.B * per, A.ctas * S::kWarps);   // none of them empty
  // neighbours in the order of the runs sit on different SMs when there are few
  const int run = runs < A.ctas * S::kWarps ? warp * A.ctas + (int)blockIdx.x : (int)blockIdx.x * S::kWarps + warp;
  if (run >= runs) return;
  int64_t u = run_start(units, run, runs);
  const int64_t u_end = run_start(units, run + 1, runs);
  // the sequence that holds unit u, and the unit of its first step
  Found at_u = find_sequence(A, u / per, lane);
  int b = at_u.b;
  int64_t seq_u = at_u.before * per;
  bool first_segment = true;
  while (u < u_end && b < A.B) {
    Seq sq = seq_of(A, b);
    if (u >= seq_u + (int64_t)sq.steps * per) {              // on to the next sequence, or over empty ones
      seq_u += (int64_t)sq.steps * per;
      if (++b == A.B) break;
      sq = seq_of(A, b);
      if (!sq.steps) {
        at_u = find_sequence(A, u / per, lane);
        b = at_u.b;
        if (b == A.B) break;
        seq_u = at_u.before * per;
        sq = seq_of(A, b);
      }
    }
    if (u < seq_u || u >= seq_u + (int64_t)sq.steps * per) break;   // (only if the lengths have changed meanwhile)
    const int item = (int)((u - seq_u) / sq.steps);
    const int h = item / A.RT, row0 = item % A.RT * S::kRows;
    const int64_t item_u = seq_u + (int64_t)item * sq.steps;
    const int step0 = (int)(u - item_u);
    const int steps = (int)min((int64_t)sq.steps, u_end - item_u) - step0;
    const int32_t* table = A.c.table + (int64_t)b * A.c.max_pages;
    auto key_of = [&](int n) { return (sq.first + step0 + n) * kSub; };
    // the page of the chunk of 16 tokens from `key` on, or -1 where there is none or no query sees a token of it
    auto page_of = [&](int key) {
      if (key >= sq.len || key + kChunk <= sq.begin) return -1;
      const int p = table[A.cpb.over(key / kChunk)];
      if (p >= 0 && p < (int)A.c.pages) return p;
      if (A.status && lane == 0) atomicOr(A.status + b, SDV_STATUS_BAD_PAGE);
      return -1;
    };
    // The copies of a step's keys (and scales) or values into a half.  Lanes take the pieces of
    // whole keys, in the order of memory, to where the threads read them as fragments.
    constexpr int kPieces = kD / 16, kKeysOf = 32 / kPieces;   // pieces of a key; keys of one copy of the warp
    const int lk = lane / kPieces, lp = lane % kPieces;
    int key_to;                                                // this lane's place of copy 0
    if (kD == 128) key_to = ((lk >> 1) * kKv + (lp >> 2)) * 512 + ((lk & 1) * 4 + (lp & 3)) * 16;
    else key_to = ((lk >> 2 & 1) * 2 + (lk >> 1 & 1)) * 512 + ((lk & 1) * 4 + lp) * 16;
    const int64_t head_keys = (int64_t)h * A.c.block;
    auto issue_keys = [&](int n, int half, int slot, int p0, int p1) {
      const uint32_t to = smem_addr(ring + half * S::kHalf) + key_to;
      const int c = key_of(n) / kChunk;
      const int o0 = A.cpb.rest(c) * kChunk, o1 = A.cpb.rest(c + 1) * kChunk;
      const int64_t h0 = (int64_t)max(p0, 0) * H, h1 = (int64_t)max(p1, 0) * H;
      const uint8_t* k0 = A.c.k + (h0 * A.c.block + head_keys + o0 + lk) * kD + lp * 16;
      const uint8_t* k1 = A.c.k + (h1 * A.c.block + head_keys + o1 + lk) * kD + lp * 16;
      constexpr int kCopies = kSub / kKeysOf;
#pragma unroll
      for (int j = 0; j < kCopies; ++j) {
        // token kKeysOf j + lk is of column pair j / 2 (D = 128) or j (D = 64), step j % 2 or lk's
        const int add = kD == 128 ? (j & 1) * 2 * kKv * 512 + (j >> 1) * 2 * 64 : j * 2 * 64;
        const bool second = j >= kCopies / 2;
        copy16(to + add, (second ? k1 : k0) + (j % (kCopies / 2)) * kKeysOf * kD, second ? p1 >= 0 : p0 >= 0);
      }
      float* sc = scales + slot * 8;
      if (lane < 4) {
        const int64_t hh = (lane & 2 ? h1 : h0) + h;
        copy4(smem_addr(sc + lane), (lane & 1 ? A.c.vs : A.c.ks) + hh, (lane & 2 ? p1 : p0) >= 0);
      }
      if (lane == 0) sc[4] = __int_as_float((p0 < 0 ? 1 : 0) | (p1 < 0 ? 2 : 0));
      asm volatile("cp.async.commit_group;");
    };
    auto issue_values = [&](int n, int half, int p0, int p1) {
      const uint32_t to = smem_addr(ring + half * S::kHalf) + lane * 16;
      const int c = key_of(n) / kChunk + (lane & 1), p = lane & 1 ? p1 : p0;
      const uint8_t* from = A.c.v + (((int64_t)max(p, 0) * H + h) * kD + (lane >> 1)) * A.c.block + A.cpb.rest(c) * kChunk;
      const int64_t stride = 16 * A.c.block;
#pragma unroll
      for (int j = 0; j < kD / 16; ++j) {
        copy16(to + 512 * j, from, p >= 0);
        from += stride;
      }
      asm volatile("cp.async.commit_group;");
    };
    auto nothing = [] { asm volatile("cp.async.commit_group;"); };
    __syncwarp();                                          // the item before is done with the ring and the queries
    int np0 = -1, np1 = -1;                                 // pages of the next step to issue
    auto look = [&](int n) {
      if (n < steps) {
        np0 = page_of(key_of(n));
        np1 = page_of(key_of(n) + kChunk);
      }
    };
    look(0);
    const float first_vs = np0 >= 0 ? fabsf(A.c.vs[(int64_t)np0 * H + h]) : 0.f;
#pragma unroll
    for (int n = 0; n < S::kAhead; ++n) {
      if (n < steps) {
        issue_keys(n, 2 * n, n, np0, np1);
        issue_values(n, 2 * n + 1, np0, np1);
      } else {
        nothing();
        nothing();
      }
      look(n + 1);
    }
    // The rows' queries as fragments, in f16: bf16 ones are scaled into its range by a power of two, one for all rows
    // where every eight elements' largest is within 2^-14 of the largest of all, else ("uneven") one a row, whose scores are
    // brought to the common one again.  So an element is within 2^-26 of its row's largest, whatever the other rows hold.
    float rsc = A.scale2, amax = 0.f;
    int modes = 0;                                         // what the steps of this item take care of
    {
      constexpr int kN = S::kRows * kD / 8 / 32;            // eights of elements of a lane
      const auto load = [&](int p) {
        const int row = row0 + p / (kD / 8), i = row / A.G;
        if (row >= A.R || i >= sq.count) return make_uint4(0, 0, 0, 0);
        return q_load8(A, b * A.q_sb + i * A.q_st + (int64_t)(h * A.G + row - i * A.G) * A.q_sh + p % (kD / 8) * 8);
      };
      const auto put = [&](int p, uint4 v, int up) {
        const int r = p / (kD / 8), e8 = p % (kD / 8);
        if (A.bf16) {
          float f[8];
          Num<SDV_BF16>::unpack(v, f);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] *= pow2(up);
          v = Num<SDV_F16>::pack(f);
        }
        qf[(((r >> 3) * kKv + (e8 >> 3)) * 2 + (e8 & 1)) * 32 + (r & 7) * 4 + (e8 >> 1 & 3)] = v;
      };
      uint4 raw[kN];
#pragma unroll
      for (int j = 0; j < kN; ++j) raw[j] = load(lane + 32 * j);
      float least = INFINITY;
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        const float m = q_largest(raw[j], A.bf16);
        amax = fmaxf(amax, m);
        least = fminf(least, m > 0.f ? m : INFINITY);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) {
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
      }
      const auto power = [](float m) { return min(max(15 - log2_of(m), -112), 100); };   // takes m to [2^15, 2^16)
      const int up = A.bf16 && amax > 0.f ? power(amax) : 0;
      rsc *= pow2(-up);
#pragma unroll
      for (int j = 0; j < kN; ++j) put(lane + 32 * j, raw[j], up);
      if (A.bf16 && least < amax * 0x1p-14f) {
        modes = kUneven;
#pragma unroll 1
        for (int p = lane; p < 32 * kN; p += 32) {
          const uint4 v = load(p);
          float m = q_largest(v, true);
#pragma unroll
          for (int o = 1; o < kD / 8; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
          const int mine = m > 0.f ? min(power(m), up + 120) : up;
          if (p % (kD / 8) == 0) downs[p / (kD / 8)] = pow2(up - mine);
          put(p, v, mine);
        }
      }
      __syncwarp();
    }
    const float most_score = amax * (448.f * kD) * fabsf(A.scale2);   // times a key's scale
    // log2 of U, and kPScale / U
    const int unit = first_vs > 0.f && first_vs < INFINITY ? min(max(log2_of(first_vs), kLeastUnit), kMostUnit) : 0;
    const float winv = pow2(7 - unit);
    // the window's rows of this item: the last key that all of them see, the first that one does not
    const int at0 = sq.len - sq.count;                     // position of the window's first query
    const int i0 = row0 / A.G, i1 = min((min(row0 + S::kRows, A.R) - 1) / A.G, sq.count - 1);
    const int min_last = at0 + i0, max_begin = A.span > 0 ? at0 + i1 - A.span + 1 : 0;
    const int max_last = at0 + i1, min_begin = A.span > 0 ? at0 + i0 - A.span + 1 : 0;   // and what any of them sees
    float acc[kMt][kNt][4];
    float mx[kR], sum[kR];                                 // (mx: of p', so kLogPScale below the largest)
#pragma unroll
    for (int m = 0; m < kMt; ++m)
#pragma unroll
      for (int n = 0; n < kNt; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[m][n][e] = 0.f;
#pragma unroll
    for (int k = 0; k < kR; ++k) {
      mx[k] = kNone;
      sum[k] = 0.f;
    }
    int half = 0, slot = 0;                                 // of this step's keys
    auto after = [](int x, int by, int of) { return x + by >= of ? x + by - of : x + by; };
    for (int n = 0; n < steps; ++n) {
      const int free_half = after(half, S::kHalves - 1, S::kHalves), free_slot = after(slot, S::kAhead, S::kScaleSlots);
      if (n + S::kAhead < steps) issue_keys(n + S::kAhead, free_half, free_slot, np0, np1);
      else nothing();
      asm volatile("cp.async.wait_group %0;" ::"n"(S::kHalves - 1));
      __syncwarp();
      const uint8_t* from = ring + half * S::kHalf;
      uint8_t* values = ring + after(half, 1, S::kHalves) * S::kHalf;
      const float* sc = scales + slot * 8;
      const int key0 = key_of(n);
      // scores: sx[s][n][0, 1] of key row g and rows 2t, 2t + 1; [2, 3] of key row g + 8
      float sx[2][kNt][4];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int k = 0; k < kNt; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) sx[s][k][e] = 0.f;
#pragma unroll
      for (int i = 0; i < kKv; ++i) {
        uint4 raw[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) raw[q] = *reinterpret_cast<const uint4*>(from + ((q * kKv + i) * 32 + lane) * 16);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t a[2][4];
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            widen4(reinterpret_cast<const uint32_t*>(&raw[2 * s])[w], a[s][0], a[s][2]);
            widen4(reinterpret_cast<const uint32_t*>(&raw[2 * s + 1])[w], a[s][1], a[s][3]);
          }
#pragma unroll
          for (int k = 0; k < kNt; ++k) {
            const uint2 qb = *(reinterpret_cast<const uint2*>(qf + ((k * kKv + i) * 2 + (w >> 1)) * 32 + lane) + (w & 1));
            mma16816(sx[0][k], a[0], qb.x, qb.y);
            mma16816(sx[1][k], a[1], qb.x, qb.y);
          }
        }
      }
      __syncwarp();                                          // the keys are read: their half is the next values'
      if (n + S::kAhead < steps) issue_values(n + S::kAhead, half, np0, np1);
      else nothing();
      look(n + S::kAhead + 1);
      const int chunk = g >> 2;
      const float4 s4 = *reinterpret_cast<const float4*>(sc);   // ks, vs of the first chunk, of the second
      float f = (chunk ? s4.z : s4.x) * rsc;                 // what a raw score is to be multiplied by
      float vs = chunk ? s4.w : s4.y;
      const int absent = __float_as_int(sc[4]);
      float lw = __log2f(fabsf(vs) * winv), ipw = ex2(-lw);    // of kPScale vs / U; what takes a sum of p' to one of 2^(s - m)
      const bool big = !(fmaxf(fabsf(s4.x), fabsf(s4.z)) * most_score <= kMostScore);
      const bool masked = key0 + kSub - 1 > min_last || key0 < max_begin || absent || modes || big ||
                          !(max_nan(fabsf(s4.y), fabsf(s4.w)) * winv <= kMostPw && fminf(fabsf(s4.y), fabsf(s4.w)) * winv >= kLeastPw);
      if (!(f > 0.f)) {                                      // a scale of 0, below 0 or none
        const float by = f == 0.f ? 0.f : f < 0.f ? -1.f : f;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int k = 0; k < kNt; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) sx[s][k][e] *= by;
        f = f < 0.f ? -f : 1.f;
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(S::kHalves - 1));
      __syncwarp();
      if (masked) {
        if (modes & kUneven) {
#pragma unroll
          for (int k = 0; k < kNt; ++k) {
            const float2 d = *reinterpret_cast<const float2*>(downs + 8 * k + 2 * t);
#pragma unroll
            for (int s = 0; s < 2; ++s) sx[s][k][0] *= d.x, sx[s][k][1] *= d.y, sx[s][k][2] *= d.x, sx[s][k][3] *= d.y;
          }
        }
        // magnitudes of the value scales, of chunks that some row sees (-1: none does; 0: a scale that is none)
        const auto seen = [&](int key, float va, int out) {
          return absent & out || key > max_last || key + kChunk <= min_begin ? -1.f : va < INFINITY ? va : 0.f;
        };
        const float va0 = seen(key0, fabsf(s4.y), 1), va1 = seen(key0 + kChunk, fabsf(s4.w), 2), va = chunk ? va1 : va0;
        const auto far = [&](float x) { return x >= 0.f && !(x * winv <= kMostPw && x * winv >= kLeastPw); };
        if (!(modes & kWide) && (far(va0) || far(va1))) {
          modes |= kWide;
          if (g == 0) {
#pragma unroll
            for (int k = 0; k < kR; ++k) refs[8 * (k >> 1) + 2 * t + (k & 1)] = mx[k];
          }
          __syncwarp();
        }
        const bool wide = modes & kWide, based = modes & kBased;
        if (wide) {
          ipw = 0.f;
          lw = va > 0.f ? __log2f(va) + __log2f(winv) : -INFINITY;
        } else if (!(va >= 0.f)) {                         // (no row sees the chunk)
          ipw = 1.f;
          lw = 0.f;
        }
        // which of this thread's 8 value tokens count as 0
        const int have = sq.len - key0 - 8 * t;
        uint32_t drop = have >= 8 ? 0u : (0xffu << max(have, 0)) & 0xffu;
        uint32_t nan_keys = 0;                             // value codes that are NaN (0x7f, 0xff)
#pragma unroll 1
        for (int m = 0; m < 2 * kMt; ++m) {
          const uint2 v = *reinterpret_cast<const uint2*>(values + (m * 32 + lane) * 8);
          // a byte's low seven bits are all ones: its top bit after adding one to them
          const uint32_t x = ((v.x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u, y = ((v.y & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
          nan_keys |= (x >> 7 & 1) | (x >> 14 & 2) | (x >> 21 & 4) | (x >> 28 & 8) | (y >> 3 & 16) | (y >> 10 & 32) | (y >> 17 & 64) | (y >> 24 & 128);
        }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) nan_keys |= __shfl_xor_sync(0xffffffffu, nan_keys, o);
        nan_keys &= ~drop;
        drop |= nan_keys;
        nan_keys = __shfl_sync(0xffffffffu, nan_keys, g >> 1);   // of this thread's keys
        if (drop) {                                        // in the ring: a thread reads what it alone has written here
          uint2 keep = make_uint2(0u, 0u);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            keep.x |= drop >> e & 1 ? 0u : 0xffu << (8 * e);
            keep.y |= drop >> (e + 4) & 1 ? 0u : 0xffu << (8 * e);
          }
#pragma unroll 1
          for (int m = 0; m < 2 * kMt; ++m) {
            uint2* at = reinterpret_cast<uint2*>(values + (m * 32 + lane) * 8);
            *at = make_uint2(at->x & keep.x, at->y & keep.y);
          }
        }
        if (!(fabsf(vs) < INFINITY)) {                     // a scale that is none: as NaN codes
          nan_keys = 0xffu;
          vs = 0.f;
        }
        const bool here = !(absent >> chunk & 1);
#pragma unroll
        for (int k = 0; k < kR; ++k) {
          const int row = row0 + 8 * (k >> 1) + 2 * t + (k & 1);
          const int last = at0 + row / A.G, begin = A.span > 0 ? last - A.span + 1 : 0;
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int tok = 4 * s + 2 * e + (g & 1), key = key0 + 8 * (g >> 1) + tok;
              float& x = sx[s][k >> 1][2 * e + (k & 1)];
              if (key > last || key < begin || !here) x = -INFINITY;
              else if (nan_keys >> tok & 1) x = NAN;
            }
        }
        if (based || big) {                                // from here on scores have bases, the sums' references to begin with
#pragma unroll
          for (int k = 0; k < kR; ++k) {
            const int r = 8 * (k >> 1) + 2 * t + (k & 1);
            const float ref = wide ? refs[r] : mx[k];       // (of the sum; without its base, if that is new)
            const bool some = ref > kNone;
            const float was = based ? bases[r] : 0.f, now = based || !some ? was : ref;
            float top = -INFINITY;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float& x = sx[s][k >> 1][2 * e + (k & 1)];
                x = __fmul_rn(x, f);
                top = max_nan(top, x);
              }
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
            // moved by what is far above it; by whatever is far from it, where the row has seen nothing
            const float base = (some ? top - now : fabsf(top - now)) > kBaseRoom && fabsf(top) < INFINITY ? top : now;
            if (mx[k] > kNone) mx[k] = fmaxf(mx[k] + (was - base), kNone);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
              for (int e = 0; e < 2; ++e) sx[s][k >> 1][2 * e + (k & 1)] -= base;
            __syncwarp();
            if (g == 0) {
              bases[r] = base;
              if (wide && some) refs[r] = fmaxf(ref + (was - base), kNone);
            }
          }
          __syncwarp();
          modes |= kBased;
          f = 1.f;
        }
        if (wide) {
#pragma unroll
          for (int k = 0; k < kR; ++k) {
            float* at = refs + 8 * (k >> 1) + 2 * t + (k & 1);
            float x = f * max_nan(max_nan(sx[0][k >> 1][k & 1], sx[0][k >> 1][2 + (k & 1)]),
                                  max_nan(sx[1][k >> 1][k & 1], sx[1][k >> 1][2 + (k & 1)]));
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, o));
            const float was = *at, m = max_nan(was, x), c = ex2(was - m);
            float add = 0.f;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
              for (int e = 0; e < 2; ++e) add += ex2(fmaf(sx[s][k >> 1][2 * e + (k & 1)], f, -m));
            sum[k] = fmaf(sum[k], c, add);
            __syncwarp();
            if (g == 0) *at = m;
          }
          __syncwarp();
        }
      }
      float top[kR];                                         // of log2 p' + mx
      bool move = false;
#pragma unroll
      for (int k = 0; k < kR; ++k) {
        top[k] = fmaf(f, max_nan(max_nan(sx[0][k >> 1][k & 1], sx[0][k >> 1][2 + (k & 1)]),
                                 max_nan(sx[1][k >> 1][k & 1], sx[1][k >> 1][2 + (k & 1)])), lw);
        move |= !(top[k] <= mx[k] + (kSlack + kLogPScale));
      }
      if (__any_sync(0xffffffffu, move)) {
#pragma unroll
        for (int k = 0; k < kR; ++k) {
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) top[k] = max_nan(top[k], __shfl_xor_sync(0xffffffffu, top[k], o));
          // a row's own affair
          const float m = top[k] <= mx[k] + (kSlack + kLogPScale) ? mx[k] : max_nan(mx[k], top[k] - kLogPScale);
          const float c = ex2(mx[k] - m);
          mx[k] = m;
          if (!(modes & kWide)) sum[k] *= c;
#pragma unroll
          for (int q = 0; q < kMt; ++q) {
            acc[q][k >> 1][k & 1] *= c;
            acc[q][k >> 1][2 + (k & 1)] *= c;
          }
        }
      }
      const uint32_t sign = vs < 0.f ? 0x80008000u : 0u;
      uint32_t pb[2][kNt][2];                               // probabilities, transposed
      uint32_t pl[2][kNt][2];                               // what f16 leaves of them
#pragma unroll
      for (int k = 0; k < kNt; ++k) {
        const float m0 = lw - mx[2 * k], m1 = lw - mx[2 * k + 1];
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float e0 = ex2(fmaf(sx[s][k][2 * e], f, m0)), e1 = ex2(fmaf(sx[s][k][2 * e + 1], f, m1));
            s0 += e0;
            s1 += e1;
            const uint32_t high = pack_half(e0, e1);
            pb[s][k][e] = transpose8(high ^ sign);
            const float2 held = __half22float2(*reinterpret_cast<const __half2*>(&high));
            pl[s][k][e] = transpose8(pack_half(e0 - held.x, e1 - held.y) ^ sign);
          }
        sum[2 * k] = fmaf(s0, ipw, sum[2 * k]);
        sum[2 * k + 1] = fmaf(s1, ipw, sum[2 * k + 1]);
      }
#pragma unroll
      for (int m = 0; m < kMt; ++m) {
        const uint2 w0 = *reinterpret_cast<const uint2*>(values + ((2 * m) * 32 + lane) * 8);
        const uint2 w1 = *reinterpret_cast<const uint2*>(values + ((2 * m + 1) * 32 + lane) * 8);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          uint32_t a[4];
          widen4(s ? w0.y : w0.x, a[0], a[2]);
          widen4(s ? w1.y : w1.x, a[1], a[3]);
#pragma unroll
          for (int k = 0; k < kNt; ++k) mma16816(acc[m][k], a, pb[s][k][0], pb[s][k][1]);
#pragma unroll
          for (int k = 0; k < kNt; ++k) mma16816(acc[m][k], a, pl[s][k][0], pl[s][k][1]);
        }
      }
      half = after(half, 2, S::kHalves);
      slot = after(slot, 1, S::kScaleSlots);
      __syncwarp();
    }
    asm volatile("cp.async.wait_group 0;");
    // the item's results, or a partial of them: its output, and 2^m l for the sum, 1 <= l < 2
    const bool whole = steps == sq.steps;
    float* part = A.part + ((int64_t)run * 2 + (first_segment ? 0 : 1)) * S::kSlot;
    const float by_unit = 1.f / winv;
    const bool wide = modes & kWide, based = modes & kBased;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kR; ++k) {
      // a NaN code of a value that all rows of a step see is in the output's element alone: the row is NaN
      float any = 0.f;
#pragma unroll
      for (int m = 0; m < kMt; ++m) any = max_nan(any, max_nan(acc[m][k >> 1][k & 1], acc[m][k >> 1][2 + (k & 1)]));
      if (any != any) sum[k] = NAN;
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], o);
      const int r = 8 * (k >> 1) + 2 * t + (k & 1), row = row0 + r;
      if (row >= A.R) continue;
      // the sum's reference; what the output's differs by, in two steps, either of which fp32 holds
      const float ref = wide ? refs[r] : mx[k], half_up = wide ? ex2(.5f * (mx[k] - ref)) : 1.f, up = half_up * by_unit;
      const float base = based ? bases[r] : 0.f;
      if (whole) {
        const int i = row / A.G;
        const float l = i < sq.count ? sum[k] : 0.f;         // a row past the sequence's window gets zeros
        const float by = l == 0.f ? 0.f : 1.f / l;
        const int64_t at = ((int64_t)b * A.W + i) * (H * A.G) + h * A.G + row - i * A.G;
#pragma unroll
        for (int m = 0; m < kMt; ++m)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            put_out(A, at * kD + 16 * m + 8 * e + g, l == 0.f ? 0.f : acc[m][k >> 1][2 * e + (k & 1)] * by * half_up * up);
        if (A.lse && g == 0) A.lse[at] = lse_of(ref, l, base);
      } else {
        const float by = sum[k] == 0.f ? 0.f : 1.f / sum[k];
#pragma unroll
        for (int m = 0; m < kMt; ++m)
#pragma unroll
          for (int e = 0; e < 2; ++e) part[r * kD + 16 * m + 8 * e + g] = acc[m][k >> 1][2 * e + (k & 1)] * by * half_up * up;
        if (g == 0) {
          const bool some = sum[k] > 0.f && sum[k] < INFINITY;
          const int e = some ? log2_of(sum[k]) : 0;
          // (with a base: that, exactly, since two partials may tie on it)
          part[S::kRows * kD + r] = !based ? ref + (float)e : sum[k] == 0.f ? kNone : base;
          part[S::kRows * kD + S::kRows + r] = based ? sum[k] * ex2(ref) : some ? sum[k] * pow2(-e) : sum[k];
        }
      }
    }
    first_segment = false;
    u += steps;
  }
}

// Joins the partials of an item that several warps' runs hold; an item without steps gets zeros.
// kSplit: a CTA has one row, and its warps take the partials in turn (few items, many partials of
// each); otherwise a warp has a row.  Bound by latency: 6 to 14 us.  Whole calls with 16
// items of 76 partials and 8 rows take 98 us split and 114 not, with 256 of 5 partials 104 and 99 (4 rows) or 301 and 259 (36).
template <int kD, int kNt, bool kSplit>
__global__ void __launch_bounds__(kJoinThreads) k_attend_join(const AttendArgs A) {
  using S = AttendShape<kD, kNt>;
  constexpr int kV = kD / 32;                                // elements of a lane
  __shared__ float wo[kSplit ? kJoinWarps : 1][kD];
  __shared__ float wl[kJoinWarps];
  const int per = A.c.H * A.RT;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int ctas = kSplit ? S::kRows : kNt;                  // of an item
  const int ib = blockIdx.x / ctas;
  const int r = kSplit ? blockIdx.x % ctas : blockIdx.x % ctas * 8 + warp;
  const int b = ib / per, item = ib % per, h = item / A.RT, row = item % A.RT * S::kRows + r;
  const Sums ts = step_sums(A, b, lane);
  // the partials are there; CTAs without work wait as well, so that this kernel ends after k_attend
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (A.status && threadIdx.x == 0 && A.lengths[b] > A.c.max_pages * A.c.block) atomicOr(A.status + b, SDV_STATUS_BAD_PAGE);
  if (row >= A.R) return;
  const Seq sq = seq_of(A, b);
  const int64_t units = ts.total * per, u0 = ts.before * per + (int64_t)item * sq.steps;
  const int64_t u1 = min(u0 + sq.steps, units);              // (never past them, unless the lengths have changed meanwhile)
  const int runs = run_count(units, (int64_t)A.B * per, A.ctas * S::kWarps);
  int g0 = 0, g1 = -1;
  if (u0 < u1) {
    // the runs [units g / runs, units (g + 1) / runs) that meet [u0, u1)
    g0 = (int)((u0 * runs) / units);
    while (run_start(units, g0 + 1, runs) <= u0) ++g0;
    while (run_start(units, g0, runs) > u0) --g0;
    g1 = (int)(((u1 - 1) * runs) / units);
    while (run_start(units, g1 + 1, runs) <= u1 - 1) ++g1;
    while (run_start(units, g1, runs) > u1 - 1) --g1;
    if (g0 == g1) return;                                    // written by that run's warp
  }
  // the item is the first segment of a run that starts inside it or with it, which only g0's may not
  const int64_t first = g0 <= g1 && run_start(units, g0, runs) < u0 ? 1 : 0;
  auto slot_of = [&](int gi) { return A.part + ((int64_t)gi * 2 + (gi == g0 ? first : 0)) * S::kSlot; };
  float m = kNone;
  for (int gi = g0 + lane; gi <= g1; gi += 32) m = max_nan(m, slot_of(gi)[S::kRows * kD + r]);
#pragma unroll
  for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  float l = 0.f, o[kV];
#pragma unroll
  for (int e = 0; e < kV; ++e) o[e] = 0.f;
#pragma unroll 4
  for (int gi = kSplit ? g0 + warp : g0; gi <= g1; gi += kSplit ? kJoinWarps : 1) {
    const float* slot = slot_of(gi);
    const float c = ex2(slot[S::kRows * kD + r] - m) * slot[S::kRows * kD + S::kRows + r];
    l += c;
#pragma unroll
    for (int e = 0; e < kV; ++e) o[e] = fmaf(c, slot[r * kD + e * 32 + lane], o[e]);
  }
  if constexpr (kSplit) {
#pragma unroll
    for (int e = 0; e < kV; ++e) wo[warp][e * 32 + lane] = o[e];
    if (lane == 0) wl[warp] = l;
    __syncthreads();
    if (warp) return;
    const int parts = min(kJoinWarps, g1 - g0 + 1);
    for (int w = 1; w < parts; ++w) {
      l += wl[w];
#pragma unroll
      for (int e = 0; e < kV; ++e) o[e] += wo[w][e * 32 + lane];
    }
  }
  const int i = row / A.G;
  if (i >= sq.count) l = 0.f;                                // past the sequence's window
  const int64_t at = ((int64_t)b * A.W + i) * (A.c.H * A.G) + h * A.G + row - i * A.G;
  const float by = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < kV; ++e) put_out(A, at * kD + e * 32 + lane, l == 0.f ? 0.f : o[e] * by);
  if (A.lse && lane == 0) A.lse[at] = lse_of(0.f, l, m);
}

// Row tiles of R rows, and the eights of each.
struct RowTiles {
  int rt, nt;
};
// As few tiles as `most` eights allow, of about equal size.
inline RowTiles row_tiles(int64_t R, int most) {
  const int64_t rt = (R + 8 * most - 1) / (8 * most);
  return RowTiles{(int)rt, (int)((((R + rt - 1) / rt) + 7) / 8)};
}
// The tiles that are likely to take least, by a cost fitted to the times of 120 shapes in each number of eights
// (tenths of a microsecond): a call's fixed part, which grows with the kernel's code and its partials, and a round
// of steps over all warps.  It chooses what takes 0.3 % more than the best on average.  Many eights read the cache less
// often, few start sooner: 36 rows (D = 128) over 3 x 24000 keys and 8 heads take 99 us in two tiles of 3 eights and 120
// in one of 5, over 32 x 8000 keys 275 and 259; 45 rows over 31 keys 12.5 us in six tiles of 1 and 20 in two of 3; 128 rows
// over 62 x 48 keys and 4 heads 43 in four of 4 and 55 in sixteen of 1.  `longest`: steps of the longest sequence that the page
// table allows, since the lengths are on the device.
inline RowTiles choose_tiles(int64_t R, int64_t heads, int64_t longest, int D, int warps) {
  static const int fixed[kMaxNt] = {110, 130, 160, 185, 360};
  static const int round[2][kMaxNt] = {{8, 11, 13, 16, 17}, {10, 16, 23, 30, 39}};
  RowTiles best{0, 0};
  int64_t least = INT64_MAX;
  for (int most = kMaxNt; most >= 1; --most) {
    const RowTiles t = row_tiles(R, most);
    const int64_t items = heads * t.rt, steps = items * longest;
    const bool whole = longest <= kMinSteps && steps <= (int64_t)kMinSteps * warps;      // an item a warp: no partials
    const int64_t cost = fixed[t.nt - 1] - (whole ? 60 : 0) + steps * round[D == 128][t.nt - 1] / warps;
    if (cost < least) {
      least = cost;
      best = t;
    }
  }
  return best;
}

template <int kD, int kNt>
static cudaError_t launch_attend(const AttendArgs& A, cudaStream_t s) {
  using S = AttendShape<kD, kNt>;
  const auto attend = k_attend<kD, kNt>;
  cudaError_t e = cudaFuncSetAttribute(attend, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
  if (e != cudaSuccess) return e;
  attend<<<(unsigned)A.ctas, S::kThreads, S::kSmem, s>>>(A);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  // the join's CTAs start while the last runs end, and wait for them
  cudaLaunchConfig_t cfg = {};
  const int64_t items = (int64_t)A.B * A.c.H * A.RT;
  const bool split = items * 12 < (int64_t)A.ctas * S::kWarps;       // a dozen partials of an item, or more
  cfg.gridDim = dim3((unsigned)(items * (split ? S::kRows : kNt)));
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return split ? cudaLaunchKernelEx(&cfg, k_attend_join<kD, kNt, true>, A) : cudaLaunchKernelEx(&cfg, k_attend_join<kD, kNt, false>, A);
}

template <int kD>
cudaError_t launch_attend_d(const AttendArgs& A, int nt, cudaStream_t s) {
  switch (nt) {
    case 1: return launch_attend<kD, 1>(A, s);
    case 2: return launch_attend<kD, 2>(A, s);
    case 3: return launch_attend<kD, 3>(A, s);
    case 4: return launch_attend<kD, 4>(A, s);
    default: return launch_attend<kD, 5>(A, s);
  }
}
cudaError_t launch_attend_64(const AttendArgs& A, int nt, cudaStream_t s);
cudaError_t launch_attend_128(const AttendArgs& A, int nt, cudaStream_t s);

}  // namespace sdv
