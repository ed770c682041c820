// sdv_attend.cuh - attention of a window's queries over the 8-bit cache: the kernels.
//
// For query i of sequence b (position len - count + i) and the keys up to its position:
//   s_j = scale ks_j (q . k_j),  p_j = e^{s_j - max} / sum,  out = sum_j p_j vs_j v_j.
// The G = Hq / H query heads of a key head and the window's queries are the rows of one item, so
// that a key is read once for up to 8 kMaxNt of them.  The (sequence, head, row tile) items' tiles
// of 64 keys, laid end to end, are dealt out to the CTAs in equal runs; a run that does not hold
// an item's whole length leaves (max, sum, output) in the workspace, and k_attend_join joins them.
//
// Both products are taken transposed, S' = K Q' and O' = V' P': the cache is the operand with 16
// rows, the queries' rows come in eights, so that a single token's few heads waste little.  A warp
// works on 32 keys at a time, from a ring of cp.async stages of its own.  Codes widen to f16
// exactly; with g = lane / 4 and t = lane % 4:
//   * key row g (g + 8) of score tile s is token 8 (g / 2) + 4 s + g % 2 (+ 2), which makes the tokens
//     that a thread multiplies in step s of the second product, 8 t + 4 s .. + 3, adjacent
//     bytes of a value row, and a thread's keys members of one chunk of 16 tokens: one
//     page, one pair of scales;
//   * a thread's sixteen contiguous elements of a key are its share of four steps of the first
//     product (the queries' fragments follow the same order of elements);
//   * an 8 x 8 tile of probabilities is transposed on its way to the second product (movmatrix).
// The reference that a row's exponentials are taken against moves only when a score passes it by
// 2^kSlack (probabilities are held in f16 below that), so that most tiles need no exchange
// between lanes and no rescaling of the output.
#pragma once

#include "sdv_cache.cuh"

namespace sdv {

constexpr int kJoinThreads = 256;
constexpr int kTile = 64;                 // keys of a unit of work: two steps of kSub
constexpr int kSub = 32;
constexpr int kMaxNt = 5;                 // eights of rows of an item
constexpr float kNone = -3e38f;           // the reference of a row that has seen nothing
constexpr float kSlack = 8.f;
constexpr float kPScale = 128.f;          // f16 holds 2^kSlack * kPScale; what is below 2^-28 of the reference is lost

// Division by the chunks of a page (up to 8) of numbers below 2^28: a product's upper half.
struct ChunkDiv {
  uint32_t magic, n;
  __device__ __forceinline__ int over(int x) const { return magic ? (int)__umulhi((uint32_t)x, magic) : x; }
  __device__ __forceinline__ int rest(int x) const { return x - over(x) * (int)n; }
};
inline ChunkDiv chunk_div(int n) { return ChunkDiv{n == 1 ? 0u : (uint32_t)((0x100000000ull + n - 1) / n), (uint32_t)n}; }

struct AttendArgs {
  const void* q;
  bool bf16;
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
  float* part;                             // workspace: 2 slots a CTA
  int ctas;
};

// A sequence's tokens, new ones and tiles.
struct Seq {
  int len, count, first, tiles;            // first: the first tile that a query sees
};
__device__ __forceinline__ Seq seq_of(const AttendArgs& A, int b) {
  Seq s;
  const int cap = A.c.max_pages * A.c.block;
  s.len = min(max(A.lengths[b], 0), cap);
  s.count = min(max(A.counts ? A.counts[b] : A.W, 0), A.W);
  s.first = 0;
  if (A.span > 0) s.first = max(0, s.len - s.count - A.span + 1) / kTile;
  s.tiles = s.count && s.len ? (s.len + kTile - 1) / kTile - s.first : 0;
  return s;
}

// Tiles of the sequences before b and of all (each for one head and row tile).
struct Sums {
  int64_t before, total;
};
__device__ __forceinline__ Sums tile_sums(const AttendArgs& A, int b, int64_t* red) {
  int64_t mine = 0, all = 0;
  for (int i = threadIdx.x; i < A.B; i += blockDim.x) {
    const int t = seq_of(A, i).tiles;
    all += t;
    if (i < b) mine += t;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    mine += __shfl_xor_sync(0xffffffffu, mine, o);
    all += __shfl_xor_sync(0xffffffffu, all, o);
  }
  if ((threadIdx.x & 31) == 0) {
    red[2 * (threadIdx.x >> 5)] = mine;
    red[2 * (threadIdx.x >> 5) + 1] = all;
  }
  __syncthreads();
  Sums s{0, 0};
  for (int w = 0; w < (int)blockDim.x / 32; ++w) {
    s.before += red[2 * w];
    s.total += red[2 * w + 1];
  }
  __syncthreads();
  return s;
}
__device__ __forceinline__ int64_t run_start(int64_t units, int g, int ctas) { return units * g / ctas; }

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool real) {
  const int n = real ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n));
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

// A warp's ring holds kHalves half steps (32 keys, or their values): one in use, the others under
// way.  Few rows leave registers for sixteen warps, whose latencies overlap; more rows take
// eight.
template <int kD, int kNt>
struct AttendShape {
  static constexpr int kWarps = kNt <= 2 ? 16 : 8;
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kRows = 8 * kNt;
  static constexpr int kSlot = kRows * (kD + 2);         // floats of a partial: rows' output, max, sum
  static constexpr int kHalf = kSub * kD;                 // bytes
  static constexpr int kHalves = (kWarps == 16 ? 3 : 5) * (kD == 64 ? 2 : 1) - (kD == 64 ? 1 : 0);
  static constexpr int kAhead = (kHalves - 1) / 2;        // steps
  static constexpr int kScaleSlots = kAhead + 1;
  static constexpr int kKv = kD / 64;                     // 16-byte pieces of a key for a thread
  static constexpr int kOutStride = kD + 4;
  static constexpr int kRing = kWarps * kHalves * kHalf;
  static constexpr int kJoin = kWarps * kRows * kOutStride * 4;   // the warps' outputs join in its place
  static constexpr int kQAt = kRing > kJoin ? kRing : kJoin;
  static constexpr int kQBytes = kNt * kKv * 2 * 32 * 16;
  static constexpr int kScaleBytes = kWarps * kScaleSlots * 32;   // of a step: ks, vs of both chunks; absent chunks
  static constexpr size_t kSmem = (size_t)kQAt + kQBytes + kScaleBytes;
  static_assert(kHalves % 2 == 1 && kSmem <= 220 * 1024, "");
};

// Writes four elements of row `row` of an item's results, and its log sum with the first of them.
template <int kD>
__device__ __forceinline__ void put_row(const AttendArgs& A, int count, int b, int h, int row, int d, float4 o, float m, float l) {
  if (row >= A.R) return;
  const int i = row / A.G, head = h * A.G + row % A.G;
  if (i >= count) l = 0.f;                                  // past the sequence's window
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (l == 0.f) o = make_float4(0.f, 0.f, 0.f, 0.f);
  const int64_t at = ((int64_t)b * A.W + i) * (A.c.H * A.G) + head;
  uint2 w;
  if (A.bf16) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(o.x * inv, o.y * inv), y = __floats2bfloat162_rn(o.z * inv, o.w * inv);
    w = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
  } else {
    w = make_uint2(pack_half(o.x * inv, o.y * inv), pack_half(o.z * inv, o.w * inv));
  }
  *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(A.out) + at * kD + d) = w;
  if (A.lse && d == 0) A.lse[at] = l > 0.f ? (m + log2f(l)) * kLn2f : (l == 0.f ? -INFINITY : NAN);
}

__device__ __forceinline__ float q_value(const AttendArgs& A, int64_t at) {
  return A.bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(A.q)[at]) : __half2float(reinterpret_cast<const __half*>(A.q)[at]);
}

template <int kD, int kNt>
__global__ void __launch_bounds__(AttendShape<kD, kNt>::kThreads, 1) k_attend(const AttendArgs A) {
  using S = AttendShape<kD, kNt>;
  constexpr int kAttWarps = S::kWarps, kAttThreads = S::kThreads;
  constexpr int kKv = S::kKv;
  constexpr int kMt = kD / 16;                             // sixteens of the output
  constexpr int kR = 2 * kNt;                              // rows of a thread: 8 n + 2 t + e
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int64_t red[2 * kAttWarps];
  __shared__ int start_b;
  __shared__ int64_t start_before;
  __shared__ float row_scale[S::kRows];
  __shared__ float wm[kAttWarps][S::kRows], wl[kAttWarps][S::kRows];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int H = A.c.H, per = H * A.RT;                     // items of a sequence
  uint8_t* ring = smem + warp * S::kHalves * S::kHalf;
  uint4* qf = reinterpret_cast<uint4*>(smem + S::kQAt);
  float* scales = reinterpret_cast<float*>(smem + S::kQAt + S::kQBytes) + warp * S::kScaleSlots * 8;

  const int64_t units = tile_sums(A, 0, red).total * per;
  const int runs = (int)min((int64_t)A.ctas, units);       // none of them empty
  if ((int)blockIdx.x >= runs) return;
  int64_t u = run_start(units, blockIdx.x, runs);
  const int64_t u_end = run_start(units, blockIdx.x + 1, runs);
  // the sequence that holds unit u
  if (tid == 0) start_b = A.B;
  if (warp == 0) {
    int64_t before = 0;
    for (int b0 = 0; b0 < A.B; b0 += 32) {
      const int64_t mine = b0 + lane < A.B ? (int64_t)seq_of(A, b0 + lane).tiles * per : 0;
      int64_t inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += x;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, before + inc > u);
      if (hit) {
        const int k = __ffs(hit) - 1;
        if (lane == k) {
          start_b = b0 + k;
          start_before = before + inc - mine;
        }
        break;
      }
      before += __shfl_sync(0xffffffffu, inc, 31);
    }
  }
  __syncthreads();
  int b = start_b;
  int64_t seq_u = start_before;                            // unit of the sequence's first tile
  bool first_segment = true;
  while (u < u_end && b < A.B) {
    const Seq sq = seq_of(A, b);
    if (u >= seq_u + (int64_t)sq.tiles * per) {
      seq_u += (int64_t)sq.tiles * per;
      ++b;
      continue;
    }
    const int item = (int)((u - seq_u) / sq.tiles);
    const int h = item / A.RT, row0 = item % A.RT * S::kRows;
    const int64_t item_u = seq_u + (int64_t)item * sq.tiles;
    const int tile0 = (int)(u - item_u);
    const int tile1 = (int)min((int64_t)sq.tiles, u_end - item_u);
    const int32_t* table = A.c.table + (int64_t)b * A.c.max_pages;
    // this warp's steps: two of every kAttWarps-th unit
    const int steps = tile1 - tile0 > warp ? 2 * ((tile1 - tile0 - warp - 1) / kAttWarps + 1) : 0;
    auto key_of = [&](int n) { return (sq.first + tile0 + warp + (n >> 1) * kAttWarps) * kTile + (n & 1) * kSub; };
    // the page of the chunk of 16 tokens from `key` on, or -1 where there is none
    auto page_of = [&](int key) {
      if (key >= sq.len) return -1;
      const int p = table[A.cpb.over(key / kChunk)];
      if (p >= 0 && p < (int)A.c.pages) return p;
      if (A.status && lane == 0) atomicOr(A.status + b, SDV_STATUS_BAD_PAGE);
      return -1;
    };
    // The copies of a step's keys (and scales) or values into a half.  Lanes take the pieces of
    // whole keys, in the order of memory, to where the threads read them as fragments.
    constexpr int kPieces = kD / 16, kKeysOf = 32 / kPieces;   // pieces of a key; keys of one copy of the warp
    const int lk = lane / kPieces, lp = lane % kPieces;
    int key_to;                                                // this lane's place of copy 0, and what copy j adds
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
    __syncthreads();                                       // the rows before these are done with shared memory
    int np0 = -1, np1 = -1;                                 // pages of the next step to issue
    auto look = [&](int n) {
      if (n < steps) {
        np0 = page_of(key_of(n));
        np1 = page_of(key_of(n) + kChunk);
      }
    };
    look(0);
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
    // the rows' queries as fragments, in f16: bf16 rows are scaled by a power of two into its range
    for (int r = warp; r < S::kRows; r += kAttWarps) {
      const int row = row0 + r, i = row / A.G;
      float f[kD / 32];
      float amax = 0.f;
#pragma unroll
      for (int e = 0; e < kD / 32; ++e) {
        f[e] = 0.f;
        if (row < A.R) f[e] = q_value(A, b * A.q_sb + i * A.q_st + (int64_t)(h * A.G + row % A.G) * A.q_sh + lane + 32 * e);
        amax = fmaxf(amax, fabsf(f[e]));
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      float up = 1.f, down = 1.f;
      if (A.bf16 && amax > 0.f && amax < INFINITY) {
        const int k = min(max(139 - (int)(__float_as_uint(amax) >> 23), -100), 100);
        up = __uint_as_float((uint32_t)(127 + k) << 23);
        down = __uint_as_float((uint32_t)(127 - k) << 23);
      }
      if (lane == 0) row_scale[r] = down;
#pragma unroll
      for (int e = 0; e < kD / 32; ++e) {                  // element d: piece d / 16 is thread t's, i-th
        const int d = lane + 32 * e, piece = d / 16;
        __half* to = reinterpret_cast<__half*>(qf + (((r >> 3) * kKv + (piece >> 2)) * 2 + (d >> 3 & 1)) * 32 + (r & 7) * 4 + (piece & 3));
        to[d & 7] = __float2half_rn(f[e] * up);
      }
    }
    __syncthreads();
    float rsc[kR];
    int min_last = 0x7fffffff, max_begin = 0;
    const int at0 = sq.len - sq.count;                     // position of the window's first query
#pragma unroll
    for (int k = 0; k < kR; ++k) {
      const int r = 8 * (k >> 1) + 2 * t + (k & 1), row = row0 + r, i = row / A.G;
      rsc[k] = row_scale[r] * A.scale2;
      if (row < A.R && i < sq.count) {                     // what the other rows get is not written
        min_last = min(min_last, at0 + i);
        if (A.span > 0) max_begin = max(max_begin, at0 + i - A.span + 1);
      }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      min_last = min(min_last, __shfl_xor_sync(0xffffffffu, min_last, o));
      max_begin = max(max_begin, __shfl_xor_sync(0xffffffffu, max_begin, o));
    }
    float acc[kMt][kNt][4];
    float mx[kR], sum[kR];
    float vref = 0.f, winv = 0.f;
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
      const uint8_t* values = ring + after(half, 1, S::kHalves) * S::kHalf;
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
      const float ks = sc[2 * chunk];
      float vs = sc[2 * chunk + 1];
      const int absent = __float_as_int(sc[4]);
      const float v0 = fabsf(sc[1]), v1 = fabsf(sc[3]);
      const bool odd_scale = !(v0 < INFINITY) || !(v1 < INFINITY);
      const float va = fmaxf(v0 < INFINITY ? v0 : 0.f, v1 < INFINITY ? v1 : 0.f);
      const bool masked = key0 + kSub - 1 > min_last || key0 < max_begin || absent || odd_scale;
#pragma unroll
      for (int k = 0; k < kR; ++k) {
        const float f = ks * rsc[k];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          sx[s][k >> 1][k & 1] *= f;
          sx[s][k >> 1][2 + (k & 1)] *= f;
        }
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(S::kHalves - 1));
      __syncwarp();
      uint32_t drop = 0;                                   // which of this thread's 8 value tokens count as 0
      if (masked) {
        const int have = sq.len - key0 - 8 * t;
        drop = have >= 8 ? 0u : (0xffu << max(have, 0)) & 0xffu;
        uint32_t nan_keys = 0;                             // value codes that are NaN (0x7f, 0xff)
#pragma unroll
        for (int m = 0; m < 2 * kMt; ++m) {
          const uint2 v = *reinterpret_cast<const uint2*>(values + (m * 32 + lane) * 8);
#pragma unroll
          for (int e = 0; e < 8; ++e) nan_keys |= (uint32_t)(((e < 4 ? v.x : v.y) >> (8 * (e & 3)) & 0x7f) == 0x7f) << e;
        }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) nan_keys |= __shfl_xor_sync(0xffffffffu, nan_keys, o);
        nan_keys &= ~drop;
        drop |= nan_keys;
        nan_keys = __shfl_sync(0xffffffffu, nan_keys, g >> 1);   // of this thread's keys
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
      }
      float top[kR];
      bool move = va > vref;
#pragma unroll
      for (int k = 0; k < kR; ++k) {
        top[k] = max_nan(max_nan(sx[0][k >> 1][k & 1], sx[0][k >> 1][2 + (k & 1)]),
                         max_nan(sx[1][k >> 1][k & 1], sx[1][k >> 1][2 + (k & 1)]));
        move |= !(top[k] <= mx[k] + kSlack);
      }
      if (__any_sync(0xffffffffu, move)) {
        float vc = 1.f;
        if (va > vref) {
          vc = vref / (4.f * va);
          vref = 4.f * va;
          winv = kPScale / vref;
        }
#pragma unroll
        for (int k = 0; k < kR; ++k) {
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) top[k] = max_nan(top[k], __shfl_xor_sync(0xffffffffu, top[k], o));
          const float m = top[k] <= mx[k] + kSlack ? mx[k] : max_nan(mx[k], top[k]);   // a row's own affair
          const float c = ex2(mx[k] - m);
          mx[k] = m;
          sum[k] *= c;
#pragma unroll
          for (int q = 0; q < kMt; ++q) {
            acc[q][k >> 1][k & 1] *= c * vc;
            acc[q][k >> 1][2 + (k & 1)] *= c * vc;
          }
        }
      }
      const float pw = vs * winv;
      uint32_t pb[2][kNt][2];                               // probabilities, transposed
#pragma unroll
      for (int k = 0; k < kNt; ++k)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float e0 = ex2(sx[s][k][2 * e] - mx[2 * k]), e1 = ex2(sx[s][k][2 * e + 1] - mx[2 * k + 1]);
            sum[2 * k] += e0;
            sum[2 * k + 1] += e1;
            pb[s][k][e] = transpose8(pack_half(e0 * pw, e1 * pw));
          }
#pragma unroll
      for (int m = 0; m < kMt; ++m) {
        uint2 v0 = *reinterpret_cast<const uint2*>(values + ((2 * m) * 32 + lane) * 8);
        uint2 v1 = *reinterpret_cast<const uint2*>(values + ((2 * m + 1) * 32 + lane) * 8);
        if (drop) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (drop >> e & 1) {
              const uint32_t keep = ~(0xffu << (8 * (e & 3)));
              if (e < 4) v0.x &= keep, v1.x &= keep;
              else v0.y &= keep, v1.y &= keep;
            }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          uint32_t a[4];
          widen4(s ? v0.y : v0.x, a[0], a[2]);
          widen4(s ? v1.y : v1.x, a[1], a[3]);
#pragma unroll
          for (int k = 0; k < kNt; ++k) mma16816(acc[m][k], a, pb[s][k][0], pb[s][k][1]);
        }
      }
      half = after(half, 2, S::kHalves);
      slot = after(slot, 1, S::kScaleSlots);
      __syncwarp();
    }
    asm volatile("cp.async.wait_group 0;");
    // the warps' states join in shared memory (the ring is free): output rows in value units
#pragma unroll
    for (int k = 0; k < kR; ++k) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], o);
      if (g == 0) {
        wm[warp][8 * (k >> 1) + 2 * t + (k & 1)] = mx[k];
        wl[warp][8 * (k >> 1) + 2 * t + (k & 1)] = sum[k];
      }
    }
    __syncthreads();
    float* wo = reinterpret_cast<float*>(smem);            // [warp][row][kOutStride]
    const float unit = vref * (1.f / kPScale);
#pragma unroll
    for (int k = 0; k < kR; ++k) {
      float* to = wo + (warp * S::kRows + 8 * (k >> 1) + 2 * t + (k & 1)) * S::kOutStride + g;
#pragma unroll
      for (int m = 0; m < kMt; ++m) {
        to[16 * m] = acc[m][k >> 1][k & 1] * unit;
        to[16 * m + 8] = acc[m][k >> 1][2 + (k & 1)] * unit;
      }
    }
    __syncthreads();
    const bool whole = tile0 == 0 && tile1 == sq.tiles;
    const int live = min(kAttWarps, tile1 - tile0);         // warps that had any
    float* part = A.part + ((int64_t)blockIdx.x * 2 + (first_segment ? 0 : 1)) * S::kSlot;
    for (int i = tid; i < S::kRows * kD / 4; i += kAttThreads) {
      const int r = i / (kD / 4), d = i % (kD / 4) * 4;
      if (row0 + r >= A.R) break;
      float m = wm[0][r];
      for (int w = 1; w < live; ++w) m = max_nan(m, wm[w][r]);
      float l = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = 0; w < live; ++w) {
        const float c = ex2(wm[w][r] - m);
        const float4 x = *reinterpret_cast<const float4*>(wo + (w * S::kRows + r) * S::kOutStride + d);
        l = fmaf(c, wl[w][r], l);
        o.x = fmaf(c, x.x, o.x);
        o.y = fmaf(c, x.y, o.y);
        o.z = fmaf(c, x.z, o.z);
        o.w = fmaf(c, x.w, o.w);
      }
      if (whole) {
        put_row<kD>(A, sq.count, b, h, row0 + r, d, o, m, l);
      } else {
        *reinterpret_cast<float4*>(part + r * kD + d) = o;
        if (d == 0) {
          part[S::kRows * kD + r] = m;
          part[S::kRows * kD + S::kRows + r] = l;
        }
      }
    }
    first_segment = false;
    u = item_u + tile1;
  }
}

// Joins the partials of an item that several CTAs' runs hold; an item without tiles gets zeros.
// A CTA has eight rows of an item, a warp each.
template <int kD, int kNt>
__global__ void __launch_bounds__(kJoinThreads) k_attend_join(const AttendArgs A) {
  using S = AttendShape<kD, kNt>;
  __shared__ int64_t red[2 * (kJoinThreads / 32)];
  const int per = A.c.H * A.RT;
  const int rows8 = blockIdx.x % kNt, ib = blockIdx.x / kNt;
  const int b = ib / per, item = ib % per, h = item / A.RT, row0 = item % A.RT * S::kRows;
  const int r = 8 * rows8 + (int)threadIdx.x / 32, lane = threadIdx.x & 31;
  if (row0 + 8 * rows8 >= A.R) return;
  const Sums ts = tile_sums(A, b, red);
  const Seq sq = seq_of(A, b);
  const int64_t units = ts.total * per, u0 = ts.before * per + (int64_t)item * sq.tiles, u1 = u0 + sq.tiles;
  const int runs = (int)min((int64_t)A.ctas, units);
  int g0 = 0, g1 = -1;
  if (sq.tiles) {
    // the CTAs whose runs [units g / runs, units (g + 1) / runs) meet [u0, u1)
    g0 = (int)((u0 * runs) / units);
    while (run_start(units, g0 + 1, runs) <= u0) ++g0;
    while (run_start(units, g0, runs) > u0) --g0;
    g1 = (int)(((u1 - 1) * runs) / units);
    while (run_start(units, g1 + 1, runs) <= u1 - 1) ++g1;
    while (run_start(units, g1, runs) > u1 - 1) --g1;
    if (g0 == g1) return;                                  // written by that CTA
  }
  // the item is the first segment of a run that starts inside it or with it, which only g0's may not
  const int64_t first = g0 <= g1 && run_start(units, g0, runs) < u0 ? 1 : 0;
  auto slot_of = [&](int gi) { return A.part + ((int64_t)gi * 2 + (gi == g0 ? first : 0)) * S::kSlot; };
  float m = kNone;
  for (int gi = g0 + lane; gi <= g1; gi += 32) m = max_nan(m, slot_of(gi)[S::kRows * kD + r]);
#pragma unroll
  for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  const int d = 4 * lane;
#pragma unroll 4
  for (int gi = g0; gi <= g1; ++gi) {
    const float* slot = slot_of(gi);
    const float c = ex2(slot[S::kRows * kD + r] - m);
    l = fmaf(c, slot[S::kRows * kD + S::kRows + r], l);
    if (d < kD) {
      const float4 x = *reinterpret_cast<const float4*>(slot + r * kD + d);
      o.x = fmaf(c, x.x, o.x);
      o.y = fmaf(c, x.y, o.y);
      o.z = fmaf(c, x.z, o.z);
      o.w = fmaf(c, x.w, o.w);
    }
  }
  if (d < kD) put_row<kD>(A, sq.count, b, h, row0 + r, d, o, m, l);
}

// Row tiles of R rows (as few as kMaxNt eights allow, of about equal size), and the eights of each.
struct RowTiles {
  int rt, nt;
};
inline RowTiles row_tiles(int64_t R) {
  const int64_t rt = (R + 8 * kMaxNt - 1) / (8 * kMaxNt);
  return RowTiles{(int)rt, (int)((((R + rt - 1) / rt) + 7) / 8)};
}

template <int kD, int kNt>
static cudaError_t launch_attend(const AttendArgs& A, cudaStream_t s) {
  using S = AttendShape<kD, kNt>;
  cudaError_t e = cudaFuncSetAttribute(k_attend<kD, kNt>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
  if (e != cudaSuccess) return e;
  k_attend<kD, kNt><<<(unsigned)A.ctas, S::kThreads, S::kSmem, s>>>(A);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  k_attend_join<kD, kNt><<<(unsigned)((int64_t)A.B * A.c.H * A.RT * kNt), kJoinThreads, 0, s>>>(A);
  return cudaGetLastError();
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
