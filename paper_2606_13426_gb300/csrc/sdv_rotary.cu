// sdv_rotary.cu - appending keys and values to the 8-bit cache, the keys (and the queries) turned by
// their positions on the way.
//
// Pair i of a head's first `rot` elements is a plane, turned by pos f_i radians:
//   (x_a, x_b) -> (x_a cos - x_b sin, x_b cos + x_a sin).
// The angle is had modulo a turn without a large argument: t_i = f_i / 2 pi mod 1 as a 64-bit fraction, and pos t_i
// modulo 2^64 is the fraction of a turn, within pos (2^-52 |f_i| / 2 pi + 2^-64) turns (1 / 2 pi and the product, both rounded to
// 53 bits; the fraction cut off).  Its nearest quarter turn is taken off as an integer, so that sine and cosine see an eighth of a
// turn at most, in steps of 2^-32.
//
// Codes and scales are those of sdv_cache_append for the turned keys, rounded once, from fp32.
#include "sdv_codes.cuh"

namespace sdv {

constexpr int kRotThreads = 256;
constexpr int kRotQueryElems = 16384;    // elements of a CTA that turns queries, about
constexpr int kQueryTokens = 32;         // of it at most
// CTAs on an SM above which they take more heads each, so that a page's cosines are computed fewer times.  With 6 and with 1, 64 x 1
// tokens of 8 heads of 128 take 9.8 and 12.5 us in place of 8.8, 32 x 32 17.6 and 20.8 in
// place of 17.2.
constexpr int kGroupCtas = 3;
constexpr int kQueriesApart = 6;         // CTAs of queries on an SM from which on they have a launch of their own
constexpr int kQueryItems = 4;           // pairs of 16-byte vectors that a thread asks for at once
enum : int { kNeighbours = 0, kHalvesOfUnits = 1, kHalves = 2 };

struct RotaryArgs {
  const void* k;
  const void* v;
  const void* q;
  void* q_out;
  int64_t sb, st, sh;                    // keys and values
  int64_t q_sb, q_st, q_sh, o_sb, o_st, o_sh;
  CacheView c;
  int B, W, Hq, nb;                      // new tokens at most, pages of a sequence they may touch
  const double* freqs;
  const int32_t* positions;              // [B, W] or NULL: from the lengths on
  int rot, halves;
  int group, groups;                     // heads of a CTA, and CTAs of a page
  int append_ctas;
  int q_tokens;                          // of a CTA
  const int32_t* lengths;
  const int32_t* counts;
  uint32_t* status;
};

// Cosine and sine of pos turns / 2^64.  An eighth of a turn at most is left, |x| <= pi / 4, where the power series to
// x^9 and x^10 are within 2^-29 and 2^-33 of them: their roundings in fp32 are what is left.
__device__ __forceinline__ float2 turned(uint64_t turn, int pos) {
  const uint64_t at = turn * (uint64_t)(int64_t)pos;
  const uint32_t quarter = (uint32_t)((at + (1ull << 61)) >> 62);
  const int rest = (int)(uint32_t)((at - ((uint64_t)quarter << 62) + (1ull << 31)) >> 32);     // of 2^32, an eighth at most
  const float x = (float)rest * (float)(3.14159265358979323846 * 0x1p-31), y = x * x;
  float s = fmaf(y, 1.f / 362880.f, -1.f / 5040.f), c = fmaf(y, -1.f / 3628800.f, 1.f / 40320.f);
  s = fmaf(fmaf(fmaf(y, s, 1.f / 120.f), y, -1.f / 6.f) * y, x, x);
  c = fmaf(fmaf(fmaf(fmaf(y, c, -1.f / 720.f), y, 1.f / 24.f), y, -.5f), y, 1.f);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_float2(quarter == 1 || quarter == 2 ? -a : a, quarter & 2 ? -b : b);
}
__device__ __forceinline__ uint64_t turn_of(double f) {
  const double t = fabs(f) * 0.15915494309189533577;             // 1 / 2 pi
  const uint64_t turn = (uint64_t)((t - floor(t)) * 0x1p64);     // (exact: of a number above 0, no bits are lost)
  return f < 0. ? 0 - turn : turn;
}

// The pairs' turns per position: 64-bit products and a floor, which this machine has few units for, so once a CTA.
__device__ __forceinline__ void fill_turns(uint64_t* turns, const RotaryArgs& A, int tid) {
  if (tid < A.rot / 2) turns[tid] = turn_of(__ldg(A.freqs + tid));
}
// A table of cosines and sines: token t's pair i at t * table_row(pairs) + table_at(i).  Without the gaps the lanes of a warp,
// which read pairs 8 or 16 apart and of several tokens, would meet in the same banks, up to 32 at once.  Two pairs from an even
// one on are read together.
__host__ __device__ __forceinline__ int table_at(int i) { return i + (i >> 3) * 2; }
__host__ __device__ constexpr int table_row(int pairs) { return (pairs + (pairs >> 3) * 2 + 15) / 16 * 16 + 2; }
__device__ __forceinline__ float4 two_pairs(const float2* cs, int i) { return *reinterpret_cast<const float4*>(cs + table_at(i)); }
// `tokens` tokens' table; pos: a token's position.
template <typename F>
__device__ __forceinline__ void fill_table(float2* table, const uint64_t* turns, int pairs, int tokens, int tid, F pos) {
  const bool keeps = kRotThreads % pairs == 0;
  int t = tid / pairs, p = tid - t * pairs;
  const int step = kRotThreads / pairs, row = table_row(pairs);
  for (int i = tid; i < tokens * pairs; i += kRotThreads) {
    if (!keeps) t = i / pairs, p = i - t * pairs;
    table[t * row + table_at(p)] = turned(turns[p], pos(t));
    t += step;
  }
}

// Four elements, two pairs (the second, if it is one).
__device__ __forceinline__ void turn_neighbours(const float4& c, bool both, float* f) {
  const float a = f[0], b = f[1], x = f[2], y = f[3];
  f[0] = a * c.x - b * c.y;
  f[1] = b * c.x + a * c.y;
  f[2] = both ? x * c.z - y * c.w : x;
  f[3] = both ? y * c.z + x * c.w : y;
}

// Sixteen consecutive elements from x on, as fp32.
template <int kDtype>
__device__ __forceinline__ void load16(const typename Num<kDtype>::T* x, bool vec, float* f) {
  using E = Num<kDtype>;
  Sixteen<kDtype> s;
  s.load(x, vec);
#pragma unroll
  for (int i = 0; i < Sixteen<kDtype>::kN; ++i) E::unpack(s.raw[i], f + i * E::kPer16);
}

// A thread's 32 elements of a key: units (sixteens) u0 and u1 of its head, turned.
template <int kDtype, int kPairs>
__device__ __forceinline__ void turn_key(const typename Num<kDtype>::T* x, bool vec, const float2* cs, int rot, int u0, int u1, float* f) {
  using E = Num<kDtype>;
  load16<kDtype>(x + u0 * 16, vec, f);
  load16<kDtype>(x + u1 * 16, vec, f + 16);
  if constexpr (kPairs == kHalvesOfUnits) {
    if (u1 * 16 < rot) {
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float4 c = two_pairs(cs, u0 * 16 + e);
        const float a = f[e], b = f[16 + e], x = f[e + 1], y = f[17 + e];
        f[e] = a * c.x - b * c.y;
        f[16 + e] = b * c.x + a * c.y;
        f[e + 1] = x * c.z - y * c.w;
        f[17 + e] = y * c.z + x * c.w;
      }
    }
  } else if constexpr (kPairs == kNeighbours) {
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
      const int at = (e < 16 ? u0 * 16 : u1 * 16 - 16) + e;
      if (at < rot) turn_neighbours(two_pairs(cs, at / 2), at + 2 < rot, f + e);
    }
  } else {                               // halves that end inside a sixteen: the other half is read again, element by element
    // (4 x 8000 tokens of 8 key heads of 128, keys alone: 113 to 134 us for 16 and 48 turned elements, 68 for 64)
    const int half = rot / 2;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      const int at = (e < 16 ? u0 * 16 : u1 * 16 - 16) + e;
      if (at < rot) {
        const bool low = at < half;
        const float2 c = cs[table_at(low ? at : at - half)];
        const float o = E::to(x[low ? at + half : at - half]);
        f[e] = low ? f[e] * c.x - o * c.y : f[e] * c.x + o * c.y;
      }
    }
  }
}
__device__ __forceinline__ float largest16(const float* f, bool finite) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float a = fabsf(f[e]);
    m = fmaxf(m, finite && !(a < INFINITY) ? 0.f : a);
  }
  return m;
}
__device__ __forceinline__ uint4 codes16(const float* f, bool pow2, float inv, float s) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = pow2 ? codes4(f[4 * i] * inv, f[4 * i + 1] * inv, f[4 * i + 2] * inv, f[4 * i + 3] * inv)
                : codes4_over(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3], s);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A CTA's queries: tokens [t0, t0 + q_tokens) of all sequences' in their order.  A thread's item is two 16-byte vectors that
// are each other's other half, or neighbours; it asks for kQueryItems of them before the first is used.
template <int kDtype>
__device__ __forceinline__ void turn_queries(const RotaryArgs& A, float2* table, uint64_t* turns, int cta) {
  using E = Num<kDtype>;
  using T = typename E::T;
  constexpr int kPer = E::kPer16;
  __shared__ int64_t from[kQueryTokens], to[kQueryTokens];
  __shared__ int where[kQueryTokens], live[kQueryTokens];
  const int tid = threadIdx.x, D = A.c.D, rot = A.rot, pairs = rot / 2;
  const int64_t total = (int64_t)A.B * A.W, t0 = (int64_t)cta * A.q_tokens;
  const int n = (int)min((int64_t)A.q_tokens, total - t0);
  int b = 0, w = 0;
  if (tid < n) {
    const int64_t at = t0 + tid;
    b = (int)(at / A.W), w = (int)(at - (int64_t)b * A.W);
    from[tid] = b * A.q_sb + w * A.q_st;
    to[tid] = b * A.o_sb + w * A.o_st;
  }
  __syncthreads();
  const auto fill = [&] {
    fill_turns(turns, A, tid);
    if (tid < n) {
      live[tid] = !A.counts || w < A.counts[b];
      where[tid] = A.positions ? A.positions[t0 + tid] : (int)((int64_t)max(A.lengths[b], 0) + w);
    }
    __syncthreads();
    fill_table(table, turns, pairs, n, tid, [&](int t) { return where[t]; });
    __syncthreads();
  };
  const T* q = reinterpret_cast<const T*>(A.q);
  T* out = reinterpret_cast<T*>(A.q_out);
  const bool vec = aligned16(q) && aligned16(out) && ((A.q_sb | A.q_st | A.q_sh | A.o_sb | A.o_st | A.o_sh) * (int64_t)sizeof(T)) % 16 == 0;
  if (vec && (!A.halves || pairs % kPer == 0)) {
    const int lper = __ffs(D / kPer / 2) - 1, per = A.Hq << lper, items = n * per;
    const int hv = A.halves ? pairs / kPer : 0;                   // vectors of a half
    bool filled = false;
    for (int i0 = tid; i0 - tid < items; i0 += kRotThreads * kQueryItems) {
      uint4 raw[kQueryItems][2];
      int tok[kQueryItems], head[kQueryItems], e0[kQueryItems], e1[kQueryItems];
#pragma unroll
      for (int k = 0; k < kQueryItems; ++k) {
        const int i = i0 + k * kRotThreads;
        tok[k] = -1;
        if (i < items) {
          const int t = i / per, r = i - t * per, p = r & ((1 << lper) - 1);
          tok[k] = t;
          head[k] = r >> lper;
          e0[k] = (p < hv ? p : 2 * p) * kPer;
          e1[k] = (p < hv ? p + hv : 2 * p + 1) * kPer;
          const T* x = q + from[t] + head[k] * A.q_sh;
          raw[k][0] = *reinterpret_cast<const uint4*>(x + e0[k]);
          raw[k][1] = *reinterpret_cast<const uint4*>(x + e1[k]);
        }
      }
      if (!filled) {                                              // while they are on their way
        fill();
        filled = true;
      }
#pragma unroll
      for (int k = 0; k < kQueryItems; ++k) {
        if (tok[k] < 0) continue;
        const float2* cs = table + tok[k] * table_row(pairs);
        if (!live[tok[k]]) {
          raw[k][0] = raw[k][1] = make_uint4(0, 0, 0, 0);
        } else if (e0[k] < rot) {                                 // (neighbours: the second may lie behind the turned ones)
          float a[kPer], b[kPer];
          E::unpack(raw[k][0], a);
          E::unpack(raw[k][1], b);
          if (A.halves) {
#pragma unroll
            for (int e = 0; e < kPer; e += 2) {
              const float4 c = two_pairs(cs, e0[k] + e);
              const float x = a[e], y = b[e], z = a[e + 1], w = b[e + 1];
              a[e] = x * c.x - y * c.y;
              b[e] = y * c.x + x * c.y;
              a[e + 1] = z * c.z - w * c.w;
              b[e + 1] = w * c.z + z * c.w;
            }
          } else {
#pragma unroll
            for (int e = 0; e < kPer; e += 4) {
              if (e0[k] + e < rot) turn_neighbours(two_pairs(cs, (e0[k] + e) / 2), e0[k] + e + 2 < rot, a + e);
              if (e1[k] + e < rot) turn_neighbours(two_pairs(cs, (e1[k] + e) / 2), e1[k] + e + 2 < rot, b + e);
            }
          }
          raw[k][0] = E::pack(a);
          raw[k][1] = E::pack(b);
        }
        T* y = out + to[tok[k]] + head[k] * A.o_sh;
        *reinterpret_cast<uint4*>(y + e0[k]) = raw[k][0];
        *reinterpret_cast<uint4*>(y + e1[k]) = raw[k][1];
      }
    }
    return;
  }
  // by elements: a pair by the thread that has its first
  fill();
  const int per = A.Hq * D;
  for (int i = tid; i < n * per; i += kRotThreads) {
    const int t = i / per, r = i - t * per, h = r / D, e = r - h * D;
    const T* x = q + from[t] + h * A.q_sh;
    T* y = out + to[t] + h * A.o_sh;
    const int p = A.halves ? e : e / 2, other = A.halves ? e + pairs : e + 1;
    if (!live[t]) {
      y[e] = E::from(0.f);
    } else if (e >= rot) {
      y[e] = x[e];
    } else if (A.halves ? e < pairs : e % 2 == 0) {
      const float2 c = table[t * table_row(pairs) + table_at(p)];
      const float a = E::to(x[e]), b = E::to(x[other]);
      y[e] = E::from(a * c.x - b * c.y);
      y[other] = E::from(b * c.x + a * c.y);
    }
  }
}

// Bound by what an SM has under way: a head's keys and values are read, their scales found by the CTA together, and written, with two
// CTAs on an SM (three spill: 64-token pages of 4 x 8000 tokens then take 107 us in place of 89; asking for the next head's rows
// ahead 94).  The queries go at the pace of a copy.  4 x 8000 tokens of 8 key and 32 query heads of 128, bf16: 165 us, 720 MB,
// 4.4 TB/s; before the cosines' table was laid out without bank conflicts and the queries asked for four vectors at a time 264.
//
// One CTA per (sequence, page, group of heads), and behind them the queries' CTAs.  Cosines and sines of the page's new
// tokens are computed once for the group's heads, in shared memory; a thread has two sixteens of a key that are each other's
// other half.  The rest is k_cache_append's.
template <int kDtype, int kItems, int kPairs>
__global__ void __launch_bounds__(kRotThreads, kItems == 1 ? 2 : 1) k_append_rotary(const RotaryArgs A) {
  using T = typename Num<kDtype>::T;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float red[2][kRotThreads / 32];
  __shared__ uint64_t turns[64];
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= A.append_ctas) {
    turn_queries<kDtype>(A, reinterpret_cast<float2*>(smem), turns, (int)blockIdx.x - A.append_ctas);
    return;
  }
  const int T_ = A.c.block, D = A.c.D;
  uint8_t* tile = smem;                                          // values: codes [row of the page][D]
  float2* table = reinterpret_cast<float2*>(smem + T_ * D);
  const uint32_t u = blockIdx.x, bj = u / (uint32_t)A.groups;
  const int hg = (int)(u - bj * (uint32_t)A.groups), b = (int)(bj / (uint32_t)A.nb), j = (int)(bj - (uint32_t)b * (uint32_t)A.nb);
  const int n = max(A.lengths[b], 0);
  const int count = min(A.counts ? A.counts[b] : A.W, A.W);
  const int64_t page_at = n / T_ + j;
  const int64_t start = page_at * T_;                            // the page's first token
  const int r0 = (int)max((int64_t)0, n - start), r1 = (int)min((int64_t)T_, n + (int64_t)count - start);   // its new rows
  if (r0 >= r1) return;
  const int m = r1 - r0, first = (int)(start + r0 - n);           // of the new tokens
  const int64_t page = page_at < A.c.max_pages ? A.c.table[(int64_t)b * A.c.max_pages + page_at] : -1;
  if (page < 0 || page >= A.c.pages) {
    if (A.status && tid == 0) atomicOr(A.status + b, SDV_STATUS_BAD_PAGE);
    return;
  }
  fill_turns(turns, A, tid);
  __syncthreads();
  fill_table(table, turns, A.rot / 2, m, tid, [&](int t) { return A.positions ? A.positions[(int64_t)b * A.W + first + t] : (int)((int64_t)n + first + t); });
  __syncthreads();
  const int per = D / 32, lper = per == 4 ? 2 : 1, lrow = lper + 1, items = m * per;
  const int hu = kPairs == kHalvesOfUnits ? A.rot / 32 : 0;       // sixteens of a half
  const int h1 = min((hg + 1) * A.group, A.c.H);
  for (int h = hg * A.group; h < h1; ++h) {
    const int64_t ph = page * A.c.H + h;
    const T* kx = reinterpret_cast<const T*>(A.k) + (int64_t)b * A.sb + first * A.st + h * A.sh;
    const T* vx = reinterpret_cast<const T*>(A.v) + (int64_t)b * A.sb + first * A.st + h * A.sh;
    const bool kvec = aligned16(kx) && (A.st * sizeof(T)) % 16 == 0, vvec = aligned16(vx) && (A.st * sizeof(T)) % 16 == 0;
    float kf[kItems][32];
    Sixteen<kDtype> vr[kItems][2];
    int u0[kItems], u1[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int i = tid + k * kRotThreads, row = i >> lper, p = i & (per - 1);
      u0[k] = p < hu ? p : 2 * p;
      u1[k] = p < hu ? p + hu : 2 * p + 1;
      if (i < items) {
        vr[k][0].load(vx + row * A.st + u0[k] * 16, vvec);
        vr[k][1].load(vx + row * A.st + u1[k] * 16, vvec);
        turn_key<kDtype, kPairs>(kx + row * A.st, kvec, table + row * table_row(A.rot / 2), A.rot, u0[k], u1[k], kf[k]);
      }
    }
    float was[2];                                                 // (r0 > 0: the page holds tokens)
    was[0] = r0 ? A.c.ks[ph] : 0.f;
    was[1] = r0 ? A.c.vs[ph] : 0.f;
    float amax[2];
#pragma unroll 1
    for (int finite = 0;; ++finite) {                             // infinities do not count for the scale
      amax[0] = amax[1] = 0.f;
#pragma unroll
      for (int k = 0; k < kItems; ++k)
        if (tid + k * kRotThreads < items) {
          amax[0] = fmaxf(amax[0], fmaxf(largest16(kf[k], finite), largest16(kf[k] + 16, finite)));
          if (!finite) {
            amax[1] = fmaxf(amax[1], fmaxf(vr[k][0].amax(), vr[k][1].amax()));
          } else {
#pragma unroll
            for (int i = 0; i < Sixteen<kDtype>::kN; ++i)
              amax[1] = fmaxf(amax[1], fmaxf(finite_max<kDtype>(vr[k][0].raw[i]), finite_max<kDtype>(vr[k][1].raw[i])));
          }
        }
#pragma unroll
      for (int kind = 0; kind < 2; ++kind) {
#pragma unroll
        for (int o = 16; o; o >>= 1) amax[kind] = fmaxf(amax[kind], __shfl_xor_sync(0xffffffffu, amax[kind], o));
        if ((tid & 31) == 0) red[kind][tid >> 5] = amax[kind];
      }
      __syncthreads();
#pragma unroll
      for (int kind = 0; kind < 2; ++kind) {
        amax[kind] = red[kind][tid & (kRotThreads / 32 - 1)];
#pragma unroll
        for (int o = 1; o < kRotThreads / 32; o <<= 1) amax[kind] = fmaxf(amax[kind], __shfl_xor_sync(0xffffffffu, amax[kind], o));
      }
      __syncthreads();                                            // red, and the old scales, are read
      if (finite || (amax[0] < INFINITY && amax[1] < INFINITY)) break;
    }
#pragma unroll
    for (int kind = 1; kind >= 0; --kind) {
      const float need = scale_for(amax[kind]);
      const float s_old = r0 ? was[kind] : need;
      const float s = fmaxf(fabsf(s_old), need);                  // (a caller's own may be negative: codes change sign)
      const bool restate = r0 && s != s_old;
      const float ratio = s_old / s;
      const bool pow2 = (__float_as_uint(s) & 0x807fffffu) == 0 && s >= 0x1p-126f && s <= 0x1p126f;
      const float inv = pow2 ? __uint_as_float((254u << 23) - __float_as_uint(s)) : 0.f;
      uint8_t* codes = (kind ? A.c.v : A.c.k) + ph * T_ * D;
      uint4* to = reinterpret_cast<uint4*>(kind ? tile : codes) + (r0 << lrow);
#pragma unroll
      for (int k = 0; k < kItems; ++k) {
        const int i = tid + k * kRotThreads, at = (i >> lper) << lrow;
        if (i < items) {
          if (kind) {
            to[at + u0[k]] = pow2 ? vr[k][0].codes(inv) : codes_over<kDtype>(vr[k][0], s);
            to[at + u1[k]] = pow2 ? vr[k][1].codes(inv) : codes_over<kDtype>(vr[k][1], s);
          } else {
            to[at + u0[k]] = codes16(kf[k], pow2, inv, s);
            to[at + u1[k]] = codes16(kf[k] + 16, pow2, inv, s);
          }
        }
      }
      if (kind == 0) {
        if (restate) restate_keys(reinterpret_cast<uint4*>(codes), r0 << lrow, ratio, tid, kRotThreads);
      } else {
        __syncthreads();
        put_values(tile, codes, T_, D, r0, r1, restate, ratio, tid, kRotThreads);
      }
      if (tid == 0 && (!r0 || restate)) (kind ? A.c.vs : A.c.ks)[ph] = s;
    }
  }
}

// The queries alone, where there are many: with the keys' registers a third fewer of these CTAs would be in flight.  Bound by issue slots
// (65 % busy) as much as by DRAM.
template <int kDtype>
__global__ void __launch_bounds__(kRotThreads, 3) k_turn_queries(const RotaryArgs A) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ uint64_t turns[64];
  turn_queries<kDtype>(A, reinterpret_cast<float2*>(smem), turns, (int)blockIdx.x);
}

template <int kDtype, int kItems, int kPairs>
static cudaError_t launch_rotary_as(const RotaryArgs& A, int64_t grid, size_t smem, cudaStream_t s) {
  const auto kern = k_append_rotary<kDtype, kItems, kPairs>;
  if (smem > 40 << 10) {                                           // (48 KB with the kernel's own, without asking)
    // the limit is shared by all host threads: its largest value
    constexpr int kMost = SDV_MAX_BLOCK * (128 + table_row(128 / 2) * (int)sizeof(float2));
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
  }
  kern<<<(unsigned)grid, kRotThreads, smem, s>>>(A);
  return cudaGetLastError();
}
template <int kDtype>
static cudaError_t launch_rotary(const RotaryArgs& A, int64_t grid, cudaStream_t s) {
  const int rows = min_int(A.W, A.c.block);
  const size_t table = (size_t)table_row(A.rot / 2) * sizeof(float2), append = (size_t)A.c.block * A.c.D + rows * table;
  size_t query = A.q ? A.q_tokens * table : 0;
  if (A.q && grid - A.append_ctas > kQueriesApart * (int64_t)sm_count()) {
    k_turn_queries<kDtype><<<(unsigned)(grid - A.append_ctas), kRotThreads, query, s>>>(A);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    grid = A.append_ctas;
    query = 0;
  }
  const size_t smem = append > query ? append : query;
  const int pairs = !A.halves ? kNeighbours : A.rot % 32 == 0 ? kHalvesOfUnits : kHalves;
  const bool one = rows * A.c.D / 32 <= kRotThreads;
  if (pairs == kNeighbours) return one ? launch_rotary_as<kDtype, 1, kNeighbours>(A, grid, smem, s) : launch_rotary_as<kDtype, 2, kNeighbours>(A, grid, smem, s);
  if (pairs == kHalvesOfUnits)
    return one ? launch_rotary_as<kDtype, 1, kHalvesOfUnits>(A, grid, smem, s) : launch_rotary_as<kDtype, 2, kHalvesOfUnits>(A, grid, smem, s);
  return one ? launch_rotary_as<kDtype, 1, kHalves>(A, grid, smem, s) : launch_rotary_as<kDtype, 2, kHalves>(A, grid, smem, s);
}
static_assert(SDV_MAX_BLOCK * 128 / 32 <= 2 * kRotThreads, "");

}  // namespace sdv

using namespace sdv;

extern "C" int sdv_cache_append_rotary(const void* k_new, const void* v_new, int64_t stride_b, int64_t stride_t, int64_t stride_h,
                                       const void* q, int64_t q_stride_b, int64_t q_stride_t, int64_t q_stride_h, void* q_out,
                                       int64_t out_stride_b, int64_t out_stride_t, int64_t out_stride_h, int dtype, int B, int W,
                                       int Hq, int H, int D, int block, const double* freqs, int rot, int halves,
                                       const int32_t* positions, void* k_codes, void* v_codes, float* k_scale, float* v_scale,
                                       int64_t pages, const int32_t* page_table, int max_pages, const int32_t* lengths,
                                       const int32_t* counts, uint32_t* status, sdv_stream_t stream) {
  if (!token_dtype(dtype) || B < 1 || W < 1 || W > (1 << 30) || !k_new || !v_new || !lengths || !freqs) return SDV_EINVAL;
  int rc = check_cache(k_codes, v_codes, k_scale, v_scale, pages, page_table, max_pages, H, D, block);
  if (rc) return rc;
  if (stride_b < 0 || stride_t < 0 || stride_h < 0 || rot < 2 || rot > D || rot % 2 || (halves != 0 && halves != 1)) return SDV_EINVAL;
  if (!q != !q_out) return SDV_EINVAL;
  if (q && (Hq < 1 || Hq > (1 << 20) || q_stride_b < 0 || q_stride_t < 0 || q_stride_h < 0 || out_stride_b < 0 || out_stride_t < 0 || out_stride_h < 0))
    return SDV_EINVAL;
  // (rows that share memory would be written by several threads)
  if (q && ((B > 1 && !out_stride_b) || (W > 1 && !out_stride_t) || (Hq > 1 && !out_stride_h))) return SDV_EINVAL;
  if (q == q_out && q && (q_stride_b != out_stride_b || q_stride_t != out_stride_t || q_stride_h != out_stride_h)) return SDV_EINVAL;
  const size_t es = elem_bytes(dtype);
  if (!aligned_to(k_new, es) || !aligned_to(v_new, es) || !aligned_to(q, es) || !aligned_to(q_out, es) || !aligned_to(freqs, 8) ||
      !aligned_to(positions, 4) || !aligned_to(lengths, 4) || !aligned_to(counts, 4) || !aligned_to(status, 4))
    return SDV_EALIGN;
  RotaryArgs A{};
  A.nb = (W + block - 2) / block + 1;
  // the heads of a CTA: as few as keep to kGroupCtas CTAs an SM
  const int64_t pages_most = (int64_t)B * A.nb;
  A.group = 1;
  while (A.group < H && pages_most * ((H + A.group - 1) / A.group) > kGroupCtas * (int64_t)sm_count()) A.group *= 2;
  if (A.group > H) A.group = H;
  A.groups = (H + A.group - 1) / A.group;
  int64_t grid = pages_most * A.groups;
  if (grid > 0x7fffffff) return SDV_EINVAL;
  A.append_ctas = (int)grid;
  if (q) {
    const int64_t tokens = (int64_t)B * W;
    int per = kRotQueryElems / (Hq * D);
    per = per < 1 ? 1 : per > kQueryTokens ? kQueryTokens : per;
    while (per > 1 && (tokens + per - 1) / per < 4 * sm_count()) per /= 2;
    A.q_tokens = per;
    grid += (tokens + per - 1) / per;
    if (grid > 0x7fffffff) return SDV_EINVAL;
  }
  A.k = k_new, A.v = v_new, A.q = q, A.q_out = q_out;
  A.sb = stride_b, A.st = stride_t, A.sh = stride_h;
  A.q_sb = q_stride_b, A.q_st = q_stride_t, A.q_sh = q_stride_h;
  A.o_sb = out_stride_b, A.o_st = out_stride_t, A.o_sh = out_stride_h;
  A.c = CacheView{(uint8_t*)k_codes, (uint8_t*)v_codes, k_scale, v_scale, page_table, pages, max_pages, H, D, block};
  A.B = B, A.W = W, A.Hq = Hq;
  A.freqs = freqs, A.positions = positions, A.rot = rot, A.halves = halves;
  A.lengths = lengths, A.counts = counts, A.status = status;
  cudaStream_t s = (cudaStream_t)stream;
  return launched(dtype == SDV_F32    ? launch_rotary<SDV_F32>(A, grid, s)
                  : dtype == SDV_BF16 ? launch_rotary<SDV_BF16>(A, grid, s)
                                      : launch_rotary<SDV_F16>(A, grid, s));
}
