// sdv_attend.cu - attention of a window's queries over the 8-bit cache.
//
// For query i of sequence b (position len - count + i) and the keys up to its position:
//   s_j = scale ks_j (q . k_j),  p_j = e^{s_j - max} / sum,  out = sum_j p_j vs_j v_j.
// The G = Hq / H query heads of a key head and the window's queries are the rows of one tile, so
// that a key is read once for all of them.  The (sequence, head, row tile) items' tiles of 64
// keys, laid end to end, are dealt out to the CTAs in equal runs; a run that does not hold an
// item's whole length leaves (max, sum, output) in the workspace, and k_attend_join joins them.
//
// A warp's tile goes through cp.async into a ring of its own: every thread copies exactly the
// bytes that it will multiply, laid out as it reads them, so that no barrier and no shuffle is
// needed.  With g = lane / 4 and t = lane % 4, keys of column g of score tile j are tokens
// 16 (g / 2) + 2 j + g % 2, which gives thread t's scores (columns 2t, 2t + 1 of all eight
// tiles) the tokens 16t .. 16t + 15: one chunk, one page, one pair of scales, and sixteen
// contiguous bytes of a value row.
#include "sdv_cache.cuh"

namespace sdv {

constexpr int kAttWarps = 4;
constexpr int kAttThreads = 32 * kAttWarps;
constexpr int kTile = 64;                 // keys of a tile
constexpr int kTileChunks = kTile / kChunk;
constexpr float kPScale = 4096.f;         // probabilities are rounded to f16 above 2^-36 of the largest

struct AttendArgs {
  const void* q;
  int64_t q_sb, q_st, q_sh;
  CacheView c;
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
__device__ Sums tile_sums(const AttendArgs& A, int b, int64_t* red) {
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

// The state of an item's rows in one CTA or warp: maximum (log2 units), sum, and the output in
// units of vref / kPScale.
template <int kD, int kM>
struct AttendShape {
  static constexpr int kRows = 16 * kM;
  static constexpr int kSlot = kRows * (kD + 2);        // floats of a partial: rows' output, max, sum
  static constexpr int kStage = 2 * kTile * kD;          // bytes of a warp's stage
  static constexpr int kStages = kD == 128 ? 3 : 6;
  static constexpr int kScaleBytes = kStages * kTileChunks * 8;
  static constexpr int kQBytes = kM * (kD / 16) * 32 * 16;
  static constexpr size_t kSmem = (size_t)kAttWarps * (kStages * kStage + kScaleBytes) + kQBytes;
};

template <int kDtype>
__device__ __forceinline__ void store2(void* out, int64_t at, float a, float b) {
  if constexpr (kDtype == SDV_BF16) {
    *reinterpret_cast<__nv_bfloat162*>(reinterpret_cast<__nv_bfloat16*>(out) + at) = __floats2bfloat162_rn(a, b);
  } else {
    *reinterpret_cast<__half2*>(reinterpret_cast<__half*>(out) + at) = __floats2half2_rn(a, b);
  }
}

// Writes two elements of row `row` of an item's results, and its log sum with the first of them.
template <int kDtype, int kD>
__device__ __forceinline__ void put_row(const AttendArgs& A, int count, int b, int h, int row, int d, float a0, float a1, float m,
                                        float l) {
  if (row >= A.R) return;
  const int i = row / A.G, head = h * A.G + row % A.G;
  if (i >= count) a0 = a1 = l = 0.f;                        // past the sequence's window
  const int64_t at = ((int64_t)b * A.W + i) * (A.c.H * A.G) + head;
  store2<kDtype>(A.out, at * kD + d, a0, a1);
  if (A.lse && d == 0) A.lse[at] = l > 0.f ? (m + log2f(l)) * kLn2f : (l == 0.f ? -INFINITY : NAN);
}

template <int kDtype, int kD, int kM>
__global__ void __launch_bounds__(kAttThreads) k_attend(const AttendArgs A) {
  using S = AttendShape<kD, kM>;
  using T = typename Num<kDtype>::T;
  constexpr int kSteps = kD / 16;                          // k-steps of q . k; kD / 64 vectors of a key for a thread
  constexpr int kKv = kD / 64;
  constexpr int kNt = kD / 8;                              // n-tiles of the output
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int64_t red[2 * kAttWarps];
  __shared__ int start_b;
  __shared__ int64_t start_before;
  __shared__ float row_scale[S::kRows];
  __shared__ float wm[kAttWarps][S::kRows], wl[kAttWarps][S::kRows];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int H = A.c.H, per = H * A.RT;                     // items of a sequence
  uint8_t* ring = smem + (size_t)warp * S::kStages * S::kStage;
  float2* scales = reinterpret_cast<float2*>(smem + (size_t)kAttWarps * S::kStages * S::kStage) + warp * S::kStages * kTileChunks;
  uint4* qf = reinterpret_cast<uint4*>(smem + (size_t)kAttWarps * (S::kStages * S::kStage + S::kScaleBytes));

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
    const int h = item / A.RT, rt = item % A.RT;
    const int64_t item_u = seq_u + (int64_t)item * sq.tiles;
    const int tile0 = (int)(u - item_u);
    const int tile1 = (int)min((int64_t)sq.tiles, u_end - item_u);
    const int row0 = rt * S::kRows;
    __syncthreads();                                       // the rows before these are done with shared memory
    // the rows' queries as fragments, in f16: bf16 rows are scaled by a power of two into its range
    for (int r = warp; r < S::kRows; r += kAttWarps) {
      const int row = row0 + r, i = row / A.G;
      float f[kD / 32];
      float amax = 0.f;
#pragma unroll
      for (int e = 0; e < kD / 32; ++e) {
        f[e] = 0.f;
        if (row < A.R)
          f[e] = Num<kDtype>::to(reinterpret_cast<const T*>(A.q)[b * A.q_sb + i * A.q_st + (int64_t)(h * A.G + row % A.G) * A.q_sh + lane + 32 * e]);
        amax = fmaxf(amax, fabsf(f[e]));
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      float up = 1.f, down = 1.f;
      if (kDtype == SDV_BF16) {
        const int e = (int)(__float_as_uint(amax) >> 23) - 127;
        if (amax > 0.f && amax < INFINITY) {
          const int k = min(max(12 - e, -100), 100);
          up = __uint_as_float((uint32_t)(127 + k) << 23);
          down = __uint_as_float((uint32_t)(127 - k) << 23);
        }
      }
      if (lane == 0) row_scale[r] = down;
      // element d goes to step (i, s) and place of its thread: d = 16 (tq + 4 i) + 4 s + e
#pragma unroll
      for (int e = 0; e < kD / 32; ++e) {
        const int d = lane + 32 * e;
        const int chunk = d / 16, tq = chunk % 4, half_i = chunk / 4, s = d / 4 % 4, el = d % 4;
        const int step = half_i * 4 + s;
        const int reg = (el / 2) * 2 + ((r & 15) >= 8);
        const int ln = (r & 7) * 4 + tq;
        __half* to = reinterpret_cast<__half*>(qf + ((r >> 4) * kSteps + step) * 32 + ln) + reg * 2 + (el & 1);
        *to = __float2half_rn(f[e] * up);
      }
    }
    __syncthreads();
    int last[2 * kM], begin[2 * kM];                       // the rows' last and first keys
    float rsc[2 * kM];
    int min_last = 0x7fffffff, max_begin = 0;
#pragma unroll
    for (int k = 0; k < 2 * kM; ++k) {
      const int r = (k >> 1) * 16 + (k & 1) * 8 + g, row = row0 + r, i = row / A.G;
      last[k] = sq.len - sq.count + i;
      begin[k] = A.span > 0 ? max(0, last[k] - A.span + 1) : 0;
      rsc[k] = row_scale[r] * A.scale2;
      if (row < A.R && i < sq.count) {                       // what the other rows get is not written
        min_last = min(min_last, last[k]);
        max_begin = max(max_begin, begin[k]);
      }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      min_last = min(min_last, __shfl_xor_sync(0xffffffffu, min_last, o));
      max_begin = max(max_begin, __shfl_xor_sync(0xffffffffu, max_begin, o));
    }
    float acc[kM][kNt][4];
    float mx[2 * kM], sum[2 * kM];
    float vref = 0.f;
#pragma unroll
    for (int k = 0; k < kM; ++k)
#pragma unroll
      for (int n = 0; n < kNt; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[k][n][e] = 0.f;
#pragma unroll
    for (int k = 0; k < 2 * kM; ++k) {
      mx[k] = -INFINITY;
      sum[k] = 0.f;
    }
    const int32_t* table = A.c.table + (int64_t)b * A.c.max_pages;
    const int cpb = A.c.block / kChunk;                    // chunks of a page
    // the page of a chunk of 16 tokens, or -1 where there is none
    auto page_of = [&](int chunk) -> int64_t {
      if (chunk * kChunk >= sq.len) return -1;
      const int p = table[chunk / cpb];
      if (p < 0 || p >= A.c.pages) {
        if (A.status) atomicOr(A.status + b, SDV_STATUS_BAD_PAGE);
        return -1;
      }
      return p;
    };
    auto issue = [&](int tile, int stage) {
      uint8_t* to = ring + stage * S::kStage;
      const int c0 = (sq.first + tile) * kTileChunks;
      const int ck = c0 + (g >> 1), cv = c0 + t;
      const int64_t pk = page_of(ck), pv = page_of(cv);
      const uint8_t* kp = A.c.k + ((max(pk, (int64_t)0) * H + h) * A.c.block + ck % cpb * kChunk + (g & 1)) * kD + 16 * t;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < kKv; ++i)
          copy16(smem_addr(to + ((j * kKv + i) * 32 + lane) * 16), kp + 2 * j * kD + 64 * i, pk >= 0);
      const uint8_t* vp = A.c.v + ((max(pv, (int64_t)0) * H + h) * kD + g) * A.c.block + cv % cpb * kChunk;
#pragma unroll
      for (int n = 0; n < kNt; ++n)
        copy16(smem_addr(to + kTile * kD + (n * 32 + lane) * 16), vp + (int64_t)8 * n * A.c.block, pv >= 0);
      if (g == 0) {
        float2 sc = make_float2(0.f, -1.f);                // a chunk that is not there
        if (pv >= 0) sc = make_float2(A.c.ks[pv * H + h], fabsf(A.c.vs[pv * H + h]));
        scales[stage * kTileChunks + t] = sc;
      }
    };
    int next = tile0 + warp;
#pragma unroll
    for (int s = 0; s < S::kStages - 1; ++s) {
      if (next < tile1) issue(next, s);
      asm volatile("cp.async.commit_group;");
      next += kAttWarps;
    }
    int stage = 0;
    for (int tile = tile0 + warp; tile < tile1; tile += kAttWarps) {
      if (next < tile1) issue(next, stage == 0 ? S::kStages - 1 : stage - 1);
      asm volatile("cp.async.commit_group;");
      next += kAttWarps;
      asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 1));
      __syncwarp();                                        // the scales of the stage
      const uint8_t* from = ring + stage * S::kStage;
      const float2 sc = scales[stage * kTileChunks + t];
      const bool here = sc.y >= 0.f || sc.y != sc.y;
      const float vs = here ? sc.y : 0.f;
      const int key0 = (sq.first + tile) * kTile + kChunk * t;
      const bool masked = (sq.first + tile + 1) * kTile - 1 > min_last || (sq.first + tile) * kTile < max_begin ||
                          __any_sync(0xffffffffu, !here);
      // scores
      float sx[kM][8][4];
#pragma unroll
      for (int k = 0; k < kM; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) sx[k][j][e] = 0.f;
#pragma unroll
      for (int i = 0; i < kKv; ++i) {
        uint4 qa[kM][4];
#pragma unroll
        for (int k = 0; k < kM; ++k)
#pragma unroll
          for (int s = 0; s < 4; ++s) qa[k][s] = qf[(k * kSteps + 4 * i + s) * 32 + lane];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint4 kv = *reinterpret_cast<const uint4*>(from + ((j * kKv + i) * 32 + lane) * 16);
          const uint32_t w[4] = {kv.x, kv.y, kv.z, kv.w};
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            uint32_t b0, b1;
            widen4(w[s], b0, b1);
#pragma unroll
            for (int k = 0; k < kM; ++k) mma16816(sx[k][j], reinterpret_cast<const uint32_t*>(&qa[k][s]), b0, b1);
          }
        }
      }
      uint32_t drop = 0;                                   // tokens of the chunk whose value codes count as 0
      uint32_t nan_keys = 0;
      if (masked) {
        const int have = min(max(sq.len - key0, 0), kChunk);
        drop = 0xffffu & ~((1u << have) - 1u);
#pragma unroll
        for (int n = 0; n < kNt; ++n) {                    // value codes that are NaN (0x7f, 0xff)
          const uint4 vv = *reinterpret_cast<const uint4*>(from + kTile * kD + (n * 32 + lane) * 16);
          const uint32_t w[4] = {vv.x, vv.y, vv.z, vv.w};
#pragma unroll
          for (int e = 0; e < 16; ++e) nan_keys |= (uint32_t)((w[e / 4] >> (8 * (e % 4)) & 0x7f) == 0x7f) << e;
        }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) nan_keys |= __shfl_xor_sync(0xffffffffu, nan_keys, o);
        nan_keys &= ~drop;
        drop |= nan_keys;
      }
      const float f0 = sc.x;
      float mnew[2 * kM];
#pragma unroll
      for (int k = 0; k < 2 * kM; ++k) {
        float top = -INFINITY;
        const float f = f0 * rsc[k];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float& x = sx[k >> 1][j][2 * (k & 1) + e];
            x *= f;
            if (masked) {
              const int tok = 2 * j + e, key = key0 + tok;
              if (key > last[k] || key < begin[k] || !here) x = -INFINITY;
              else if (nan_keys >> tok & 1) x = NAN;
            }
            top = max_nan(top, x);
          }
        top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 2));
        mnew[k] = max_nan(mx[k], top);
      }
      // the values' scales, relative to the largest so far
      float vnew = fmaxf(vs, __shfl_xor_sync(0xffffffffu, vs, 1));
      vnew = fmaxf(vnew, __shfl_xor_sync(0xffffffffu, vnew, 2));
      vnew = fmaxf(vref, vnew);
      const float vcorr = vnew > vref ? vref / vnew : 1.f;
      vref = vnew;
      const float pw = vref > 0.f ? vs / vref * kPScale : 0.f;
      bool moved = vcorr != 1.f;
#pragma unroll
      for (int k = 0; k < 2 * kM; ++k) moved |= !(mnew[k] == mx[k]);
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int k = 0; k < 2 * kM; ++k) {
          const float c = mx[k] == -INFINITY ? 0.f : ex2(mx[k] - mnew[k]);
          sum[k] *= c;
          const float oc = c * vcorr;
#pragma unroll
          for (int n = 0; n < kNt; ++n) {
            acc[k >> 1][n][2 * (k & 1)] *= oc;
            acc[k >> 1][n][2 * (k & 1) + 1] *= oc;
          }
          mx[k] = mnew[k];
        }
      }
      uint32_t pa[kM][4][4];
#pragma unroll
      for (int k = 0; k < 2 * kM; ++k) {
        const float ms = mx[k] == -INFINITY ? 0.f : mx[k];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float e0 = ex2(sx[k >> 1][j][2 * (k & 1)] - ms), e1 = ex2(sx[k >> 1][j][2 * (k & 1) + 1] - ms);
          sum[k] += e0 + e1;
          pa[k >> 1][j >> 1][(j & 1) * 2 + (k & 1)] = pack_half(e0 * pw, e1 * pw);
        }
      }
#pragma unroll
      for (int n = 0; n < kNt; ++n) {
        uint4 vv = *reinterpret_cast<const uint4*>(from + kTile * kD + (n * 32 + lane) * 16);
        uint32_t w[4] = {vv.x, vv.y, vv.z, vv.w};
        if (masked) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (drop >> e & 1) w[e / 4] &= ~(0xffu << (8 * (e % 4)));
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          uint32_t b0, b1;
          widen4(w[s], b0, b1);
#pragma unroll
          for (int k = 0; k < kM; ++k) mma16816(acc[k][n], pa[k][s], b0, b1);
        }
      }
      stage = stage + 1 == S::kStages ? 0 : stage + 1;
      __syncwarp();
    }
    asm volatile("cp.async.wait_group 0;");
    // the warps' states join in shared memory (the ring is free): output rows in value units
#pragma unroll
    for (int k = 0; k < 2 * kM; ++k) {
      sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], 1);
      sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], 2);
      const int r = (k >> 1) * 16 + (k & 1) * 8 + g;
      if (t == 0) {
        wm[warp][r] = mx[k];
        wl[warp][r] = sum[k];
      }
    }
    __syncthreads();
    float* wo = reinterpret_cast<float*>(smem);            // [warp][row][kD]
    const float unit = vref / kPScale;
#pragma unroll
    for (int k = 0; k < 2 * kM; ++k) {
      const int r = (k >> 1) * 16 + (k & 1) * 8 + g;
#pragma unroll
      for (int n = 0; n < kNt; ++n)
        *reinterpret_cast<float2*>(wo + ((size_t)warp * S::kRows + r) * kD + 8 * n + 2 * t) =
            make_float2(acc[k >> 1][n][2 * (k & 1)] * unit, acc[k >> 1][n][2 * (k & 1) + 1] * unit);
    }
    __syncthreads();
    const bool whole = tile0 == 0 && tile1 == sq.tiles;
    float* slot = A.part + ((int64_t)blockIdx.x * 2 + (first_segment ? 0 : 1)) * S::kSlot;
    for (int i = tid; i < S::kRows * kD / 2; i += kAttThreads) {
      const int r = i / (kD / 2), d = i % (kD / 2) * 2;
      float m = wm[0][r];
      for (int w = 1; w < kAttWarps; ++w) m = max_nan(m, wm[w][r]);
      const float ms = m == -INFINITY ? 0.f : m;
      float l = 0.f, a0 = 0.f, a1 = 0.f;
      for (int w = 0; w < kAttWarps; ++w) {
        const float c = ex2(wm[w][r] - ms);
        const float2 o = *reinterpret_cast<const float2*>(wo + ((size_t)w * S::kRows + r) * kD + d);
        l += c * wl[w][r];
        a0 = fmaf(c, o.x, a0);
        a1 = fmaf(c, o.y, a1);
      }
      if (whole) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        put_row<kDtype, kD>(A, sq.count, b, h, row0 + r, d, a0 * inv, a1 * inv, m, l);
      } else {
        *reinterpret_cast<float2*>(slot + r * kD + d) = make_float2(a0, a1);
        if (d == 0) {
          slot[S::kRows * kD + r] = m;
          slot[S::kRows * kD + S::kRows + r] = l;
        }
      }
    }
    first_segment = false;
    u = item_u + tile1;
  }
}

// Joins the partials of an item that several CTAs' runs hold; an item without tiles gets zeros.
template <int kDtype, int kD, int kM>
__global__ void __launch_bounds__(kAttThreads) k_attend_join(const AttendArgs A) {
  using S = AttendShape<kD, kM>;
  __shared__ int64_t red[2 * kAttWarps];
  const int per = A.c.H * A.RT;
  const int b = blockIdx.x / per, item = blockIdx.x % per, h = item / A.RT, row0 = item % A.RT * S::kRows;
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
  for (int i = threadIdx.x; i < S::kRows * kD / 2; i += kAttThreads) {
    const int r = i / (kD / 2), d = i % (kD / 2) * 2;
    float m = -INFINITY, l = 0.f, a0 = 0.f, a1 = 0.f;
    for (int gi = g0; gi <= g1; ++gi) {
      // the item is the first segment of a run that starts inside it or with it
      const bool first = run_start(units, gi, runs) >= u0;
      const float* slot = A.part + ((int64_t)gi * 2 + (first ? 0 : 1)) * S::kSlot;
      const float om = slot[S::kRows * kD + r], ol = slot[S::kRows * kD + S::kRows + r];
      const float2 o = *reinterpret_cast<const float2*>(slot + r * kD + d);
      const float mn = max_nan(m, om), ms = mn == -INFINITY ? 0.f : mn;
      const float c0 = ex2(m - ms), c1 = ex2(om - ms);
      l = c0 * l + c1 * ol;
      a0 = c0 * a0 + c1 * o.x;
      a1 = c0 * a1 + c1 * o.y;
      m = mn;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    put_row<kDtype, kD>(A, sq.count, b, h, row0 + r, d, a0 * inv, a1 * inv, m, l);
  }
}

static int attend_rows(int rows) { return rows <= 16 ? 1 : 2; }

template <int kDtype, int kD, int kM>
static cudaError_t launch_attend(AttendArgs A, cudaStream_t s) {
  using S = AttendShape<kD, kM>;
  A.RT = (A.R + S::kRows - 1) / S::kRows;
  cudaError_t e = cudaFuncSetAttribute(k_attend<kDtype, kD, kM>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
  if (e != cudaSuccess) return e;
  k_attend<kDtype, kD, kM><<<(unsigned)A.ctas, kAttThreads, S::kSmem, s>>>(A);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  k_attend_join<kDtype, kD, kM><<<(unsigned)((int64_t)A.B * A.c.H * A.RT), kAttThreads, 0, s>>>(A);
  return cudaGetLastError();
}

template <int kDtype>
static cudaError_t launch_attend_d(const AttendArgs& A, cudaStream_t s) {
  if (A.c.D == 128) return attend_rows(A.R) == 1 ? launch_attend<kDtype, 128, 1>(A, s) : launch_attend<kDtype, 128, 2>(A, s);
  return attend_rows(A.R) == 1 ? launch_attend<kDtype, 64, 1>(A, s) : launch_attend<kDtype, 64, 2>(A, s);
}

}  // namespace sdv

using namespace sdv;

extern "C" {

size_t sdv_attend_workspace_bytes(int W, int Hq, int H, int D) {
  if (W < 1 || H < 1 || Hq < H || Hq % H || (D != 64 && D != 128)) return 0;
  const int64_t R = (int64_t)W * (Hq / H);
  return (size_t)sm_count() * 2 * 16 * (R <= 16 ? 1 : 2) * (size_t)(D + 2) * 4;
}

int sdv_cache_attend(const void* q, int64_t q_stride_b, int64_t q_stride_t, int64_t q_stride_h, int dtype, int B, int W,
                     int Hq, int H, int D, int block, const void* k_codes, const void* v_codes, const float* k_scale,
                     const float* v_scale, int64_t pages, const int32_t* page_table, int max_pages,
                     const int32_t* lengths, const int32_t* counts, float scale, int span, void* out, float* lse,
                     uint32_t* status, void* workspace, size_t workspace_bytes, sdv_stream_t stream) {
  if ((dtype != SDV_BF16 && dtype != SDV_F16) || B < 1 || W < 1 || H < 1 || Hq < H || Hq % H || !q || !lengths || !out)
    return SDV_EINVAL;
  int rc = check_cache(k_codes, v_codes, k_scale, v_scale, pages, page_table, max_pages, H, D, block);
  if (rc) return rc;
  if (q_stride_b < 0 || q_stride_t < 0 || q_stride_h < 0 || span < 0 || !(fabsf(scale) < INFINITY)) return SDV_EINVAL;
  const int64_t R = (int64_t)W * (Hq / H);
  if (R > (1 << 24) || (int64_t)B * H * ((R + 15) / 16) > 0x7fffffff) return SDV_EINVAL;
  if (!aligned_to(q, 2) || !aligned_to(out, 4) || !aligned_to(lse, 4) || !aligned_to(status, 4) || !aligned_to(lengths, 4) ||
      !aligned_to(counts, 4))
    return SDV_EALIGN;
  if (!workspace || workspace_bytes < sdv_attend_workspace_bytes(W, Hq, H, D)) return SDV_ENOWORKSPACE;
  if (!aligned_to(workspace, 256)) return SDV_EALIGN;
  AttendArgs A{};
  A.q = q;
  A.q_sb = q_stride_b, A.q_st = q_stride_t, A.q_sh = q_stride_h;
  A.c = CacheView{(uint8_t*)k_codes, (uint8_t*)v_codes, (float*)k_scale, (float*)v_scale, page_table, pages, max_pages, H, D, block};
  A.B = B, A.W = W, A.G = Hq / H, A.R = (int)R;
  A.lengths = lengths, A.counts = counts;
  A.scale2 = scale * kLog2E;
  A.span = span;
  A.out = out, A.lse = lse, A.status = status;
  A.part = (float*)workspace;
  A.ctas = sm_count();
  cudaStream_t s = (cudaStream_t)stream;
  return launched(dtype == SDV_BF16 ? launch_attend_d<SDV_BF16>(A, s) : launch_attend_d<SDV_F16>(A, s));
}

}  // extern "C"
