// sdv_cache.cu - appending keys and values to the 8-bit cache.
//
// A page's scale for a head is the least power of two whose 448-fold (the largest e4m3 value)
// holds every magnitude in it: s = 2^k, k = ceil(log2(amax / 448)); codes are rn(x / s).  Tokens
// that a page already holds keep their codes unless the scale grows; then they are restated
// under the new one, which is exact (powers of two) but for what underflows.  Between the reads
// and the writes a CTA owns its page and head, so that nothing is shared.
#include "sdv_cache.cuh"

namespace sdv {

constexpr int kAppendThreads = 256;

struct AppendArgs {
  const void* x[2];                 // keys, values: [B, W, H, D] by strides
  int64_t sb, st, sh;
  CacheView c;
  int W, nb;                        // new tokens at most, pages of a sequence they may touch
  const int32_t* lengths;
  const int32_t* counts;
  uint32_t* status;
};

// The least power of two, 2^-126 or more, whose 448-fold holds amax (finite, >= 0).
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int k = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);   // 448 = 1.75 * 2^8
  return __uint_as_float((uint32_t)(max(k, -126) + 127) << 23);
}

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}
__device__ __forceinline__ float code_value(uint32_t byte) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
}
__device__ __forceinline__ uint32_t restate4(uint32_t w, float ratio) {
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = code_value(w >> (8 * i) & 0xff) * ratio;
  return codes4(f[0], f[1], f[2], f[3]);
}

// Sixteen consecutive elements as they are held.
template <int kDtype>
struct Sixteen {
  using E = Num<kDtype>;
  static constexpr int kN = 16 / E::kPer16;
  uint4 raw[kN];
  __device__ __forceinline__ void load(const typename E::T* p, bool vec) {
    if (vec) {
#pragma unroll
      for (int i = 0; i < kN; ++i) raw[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        float f[E::kPer16];
#pragma unroll
        for (int e = 0; e < E::kPer16; ++e) f[e] = E::to(p[i * E::kPer16 + e]);
        raw[i] = E::pack(f);
      }
    }
  }
  // The largest magnitude (infinity if one is infinite).
  __device__ __forceinline__ float amax() const {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      uint4 v = raw[i];
      const uint32_t sign = kDtype == SDV_F32 ? 0x7fffffffu : 0x7fff7fffu;
      v.x &= sign, v.y &= sign, v.z &= sign, v.w &= sign;
      m = fmaxf(m, vec_max_num<kDtype>(v));
    }
    return m;
  }
  __device__ __forceinline__ uint4 codes(float inv) const {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      float f[E::kPer16];
      E::unpack(raw[i], f);
#pragma unroll
      for (int e = 0; e < E::kPer16; e += 4) w[(i * E::kPer16 + e) / 4] = codes4(f[e] * inv, f[e + 1] * inv, f[e + 2] * inv, f[e + 3] * inv);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// What few calls need, kept out of the way of the others: the largest finite magnitude of eight or
// four elements, and codes under a scale that is no power of two (a caller's own): x / s, rounded
// once, sixteen elements at a time.
template <int kDtype>
static __device__ __noinline__ float finite_max(uint4 v) {
  float f[Num<kDtype>::kPer16], m = 0.f;
  Num<kDtype>::unpack(v, f);
#pragma unroll
  for (int e = 0; e < Num<kDtype>::kPer16; ++e) m = fmaxf(m, fabsf(f[e]) < INFINITY ? fabsf(f[e]) : 0.f);
  return m;
}
static __device__ __noinline__ uint32_t codes4_over(float a, float b, float c, float d, float s) { return codes4(a / s, b / s, c / s, d / s); }
template <int kDtype>
__device__ __forceinline__ uint4 codes_over(const Sixteen<kDtype>& x, float s) {
  using E = Num<kDtype>;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < Sixteen<kDtype>::kN; ++i) {
    float f[E::kPer16];
    E::unpack(x.raw[i], f);
#pragma unroll
    for (int e = 0; e < E::kPer16; e += 4) w[(i * E::kPer16 + e) / 4] = codes4_over(f[e], f[e + 1], f[e + 2], f[e + 3], s);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Bytes of the word of tokens t .. t + 3 that are in [lo, hi).
__device__ __forceinline__ uint32_t bytes_in(int t, int lo, int hi) {
  const int a = min(max(lo - t, 0), 4), b = min(max(hi - t, 0), 4);
  const uint32_t below_b = b == 4 ? 0xffffffffu : (1u << (8 * b)) - 1u, below_a = a == 4 ? 0xffffffffu : (1u << (8 * a)) - 1u;
  return below_b & ~below_a;
}

// CTAs of an SM that the registers of the elements held leave room for.
constexpr int append_ctas(int dtype, int units) {
  const int regs = 2 * units * (dtype == SDV_F32 ? 16 : 8);
  return regs <= 32 ? 4 : regs <= 64 ? 2 : 1;
}

// One CTA per (sequence, head, page).  The new keys and values are read once and kept in registers
// (kUnits sixteens of elements of each a thread) between the largest magnitude and the codes: the
// loads of both are under way together.  Values go through shared memory as codes, and are
// turned in 4 x 4 bytes on the way out.
// 4 x 8000 tokens, 8 heads of 128, bf16: 42 us, 4.7 TB/s (131 MB in, 66 out); bound by issue slots (56 % busy:
// conversions, the transposition) and by the chain of length, page, scale in each CTA.  64 windows
// of 9 tokens: 6.5 us, latency.
template <int kDtype, int kUnits>
__global__ void __launch_bounds__(kAppendThreads, append_ctas(kDtype, kUnits)) k_cache_append(const AppendArgs A) {
  using T = typename Num<kDtype>::T;
  extern __shared__ __align__(16) uint8_t tile[];      // values: codes [row of the page][D]
  __shared__ float red[2][kAppendThreads / 32];
  const uint32_t u = blockIdx.x, bh = u / (uint32_t)A.nb;
  const int j = (int)(u - bh * (uint32_t)A.nb), b = (int)(bh / (uint32_t)A.c.H), h = (int)(bh - (uint32_t)b * (uint32_t)A.c.H);
  const int tid = threadIdx.x, T_ = A.c.block, D = A.c.D;
  const int n = max(A.lengths[b], 0);
  const int count = min(A.counts ? A.counts[b] : A.W, A.W);
  const int page_at = n / T_ + j;
  const int64_t start = (int64_t)page_at * T_;                   // the page's first token
  const int r0 = (int)max((int64_t)0, n - start), r1 = (int)min((int64_t)T_, n + (int64_t)count - start);   // its new rows
  if (r0 >= r1) return;
  const int m = r1 - r0;
  const int per = D / 16, lper = per == 8 ? 3 : 2, units = m * per;
  Sixteen<kDtype> s16[2][kUnits];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    const T* x = reinterpret_cast<const T*>(A.x[kind]) + (int64_t)b * A.sb + (start + r0 - n) * A.st + h * A.sh;
    const bool vec = aligned16(x) && (A.st * sizeof(T)) % 16 == 0;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
      const int i = tid + k * kAppendThreads;
      if (i < units) s16[kind][k].load(x + (i >> lper) * A.st + (i & (per - 1)) * 16, vec);
    }
  }
  const int64_t page = page_at < A.c.max_pages ? A.c.table[(int64_t)b * A.c.max_pages + page_at] : -1;
  if (page < 0 || page >= A.c.pages) {
    if (A.status && tid == 0) atomicOr(A.status + b, SDV_STATUS_BAD_PAGE);
    return;
  }
  const int64_t ph = page * A.c.H + h;
  float was[2];                                                   // (r0 > 0: the page holds tokens)
  was[0] = r0 ? A.c.ks[ph] : 0.f;
  was[1] = r0 ? A.c.vs[ph] : 0.f;
  float amax[2];
#pragma unroll 1
  for (int finite = 0;; ++finite) {                               // infinities do not count for the scale
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      amax[kind] = 0.f;
#pragma unroll
      for (int k = 0; k < kUnits; ++k)
        if (tid + k * kAppendThreads < units) {
          if (!finite) {
            amax[kind] = fmaxf(amax[kind], s16[kind][k].amax());
          } else {
#pragma unroll
            for (int i = 0; i < Sixteen<kDtype>::kN; ++i) amax[kind] = fmaxf(amax[kind], finite_max<kDtype>(s16[kind][k].raw[i]));
          }
        }
#pragma unroll
      for (int o = 16; o; o >>= 1) amax[kind] = fmaxf(amax[kind], __shfl_xor_sync(0xffffffffu, amax[kind], o));
      if ((tid & 31) == 0) red[kind][tid >> 5] = amax[kind];
    }
    __syncthreads();
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      amax[kind] = red[kind][tid & (kAppendThreads / 32 - 1)];
#pragma unroll
      for (int o = 1; o < kAppendThreads / 32; o <<= 1) amax[kind] = fmaxf(amax[kind], __shfl_xor_sync(0xffffffffu, amax[kind], o));
    }
    __syncthreads();                                              // red, and the old scales, are read
    if (finite || (amax[0] < INFINITY && amax[1] < INFINITY)) break;
  }
#pragma unroll
  for (int kind = 1; kind >= 0; --kind) {
    const float need = scale_for(amax[kind]);
    const float s_old = r0 ? was[kind] : need;
    const float s = fmaxf(fabsf(s_old), need);                    // (a caller's own may be negative: codes change sign)
    const bool restate = r0 && s != s_old;
    const float ratio = s_old / s;
    const bool pow2 = (__float_as_uint(s) & 0x807fffffu) == 0 && s >= 0x1p-126f && s <= 0x1p126f;
    const float inv = pow2 ? __uint_as_float((254u << 23) - __float_as_uint(s)) : 0.f;
    uint8_t* codes = (kind ? A.c.v : A.c.k) + ph * T_ * D;
    uint4* to = reinterpret_cast<uint4*>(kind ? tile : codes) + (r0 << lper);
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
      const int i = tid + k * kAppendThreads;
      if (i < units) to[i] = pow2 ? s16[kind][k].codes(inv) : codes_over<kDtype>(s16[kind][k], s);
    }
    if (kind == 0) {
      if (restate)
        for (int i = tid; i < r0 << lper; i += kAppendThreads) {
          uint4* at = reinterpret_cast<uint4*>(codes) + i;
          uint4 c = *at;
          c.x = restate4(c.x, ratio);
          c.y = restate4(c.y, ratio);
          c.z = restate4(c.z, ratio);
          c.w = restate4(c.w, ratio);
          *at = c;
        }
    } else {
      __syncthreads();
      // sixteen tokens of four elements a thread
      const int c0 = restate ? 0 : r0 / kChunk, c1 = (r1 - 1) / kChunk + 1, quads = D / 4, lq = quads == 32 ? 5 : 4;
#pragma unroll 1
      for (int i = tid; i < (c1 - c0) << lq; i += kAppendThreads) {
        const int d = (i & (quads - 1)) * 4, t0 = (c0 + (i >> lq)) * kChunk;
        uint32_t w[4][4];                                         // [element][four tokens]
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t a[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) a[e] = *reinterpret_cast<const uint32_t*>(tile + (t0 + 4 * q + e) * D + d);
          const uint32_t x0 = __byte_perm(a[0], a[1], 0x5140), x1 = __byte_perm(a[2], a[3], 0x5140);
          const uint32_t y0 = __byte_perm(a[0], a[1], 0x7362), y1 = __byte_perm(a[2], a[3], 0x7362);
          w[0][q] = __byte_perm(x0, x1, 0x5410);
          w[1][q] = __byte_perm(x0, x1, 0x7632);
          w[2][q] = __byte_perm(y0, y1, 0x5410);
          w[3][q] = __byte_perm(y0, y1, 0x7632);
        }
        uint4* at = reinterpret_cast<uint4*>(codes + (int64_t)d * T_ + t0);
        if (t0 < r0 || t0 + kChunk > r1) {                        // some of the tokens are old, or not there yet
          uint4 old[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) old[e] = *reinterpret_cast<const uint4*>(reinterpret_cast<uint8_t*>(at) + (int64_t)e * T_);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t fresh = bytes_in(t0 + 4 * q, r0, r1), kept = restate ? bytes_in(t0 + 4 * q, 0, r0) : 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t o = q == 0 ? old[e].x : q == 1 ? old[e].y : q == 2 ? old[e].z : old[e].w;
              if (kept) o = (restate4(o, ratio) & kept) | (o & ~kept);
              w[e][q] = (w[e][q] & fresh) | (o & ~fresh);
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(at) + (int64_t)e * T_) = make_uint4(w[e][0], w[e][1], w[e][2], w[e][3]);
      }
    }
    if (tid == 0 && (!r0 || restate)) (kind ? A.c.vs : A.c.ks)[ph] = s;
  }
}

template <int kDtype>
static cudaError_t launch_append(const AppendArgs& A, int64_t grid, cudaStream_t s) {
  const size_t smem = (size_t)A.c.block * A.c.D;
  const int most = (A.W < A.c.block ? A.W : A.c.block) * A.c.D / 16;              // sixteens of a page's new tokens
  if (most <= kAppendThreads) k_cache_append<kDtype, 1><<<(unsigned)grid, kAppendThreads, smem, s>>>(A);
  else if (most <= 2 * kAppendThreads) k_cache_append<kDtype, 2><<<(unsigned)grid, kAppendThreads, smem, s>>>(A);
  else k_cache_append<kDtype, 4><<<(unsigned)grid, kAppendThreads, smem, s>>>(A);
  return cudaGetLastError();
}
static_assert(SDV_MAX_BLOCK * 128 / 16 <= 4 * kAppendThreads, "");

}  // namespace sdv

using namespace sdv;

extern "C" int sdv_cache_append(const void* k_new, const void* v_new, int64_t stride_b, int64_t stride_t, int64_t stride_h,
                                int dtype, int B, int W, int H, int D, int block, void* k_codes, void* v_codes, float* k_scale,
                                float* v_scale, int64_t pages, const int32_t* page_table, int max_pages,
                                const int32_t* lengths, const int32_t* counts, uint32_t* status, sdv_stream_t stream) {
  if (!token_dtype(dtype) || B < 1 || W < 1 || W > (1 << 30) || !k_new || !v_new || !lengths) return SDV_EINVAL;
  int rc = check_cache(k_codes, v_codes, k_scale, v_scale, pages, page_table, max_pages, H, D, block);
  if (rc) return rc;
  if (stride_b < 0 || stride_t < 0 || stride_h < 0) return SDV_EINVAL;
  if (!aligned_to(k_new, elem_bytes(dtype)) || !aligned_to(v_new, elem_bytes(dtype)) || !aligned_to(lengths, 4) ||
      !aligned_to(counts, 4) || !aligned_to(status, 4))
    return SDV_EALIGN;
  const int nb = (W + block - 2) / block + 1;
  const int64_t grid = (int64_t)B * H * nb;
  if (grid > 0x7fffffff) return SDV_EINVAL;
  const AppendArgs A{{k_new, v_new}, stride_b, stride_t, stride_h,
                     CacheView{(uint8_t*)k_codes, (uint8_t*)v_codes, k_scale, v_scale, page_table, pages, max_pages, H, D, block},
                     W, nb, lengths, counts, status};
  cudaStream_t s = (cudaStream_t)stream;
  return launched(dtype == SDV_F32    ? launch_append<SDV_F32>(A, grid, s)
                  : dtype == SDV_BF16 ? launch_append<SDV_BF16>(A, grid, s)
                                      : launch_append<SDV_F16>(A, grid, s));
}
