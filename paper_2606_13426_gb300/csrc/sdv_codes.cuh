// sdv_codes.cuh - e4m3 codes under a page's scale: what the kernels that write the 8-bit cache share.
#pragma once

#include "sdv_cache.cuh"

namespace sdv {

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

// Restates n vectors of sixteen codes.
__device__ __forceinline__ void restate_keys(uint4* at, int n, float ratio, int tid, int threads) {
  for (int i = tid; i < n; i += threads) {
    uint4 c = at[i];
    c.x = restate4(c.x, ratio);
    c.y = restate4(c.y, ratio);
    c.z = restate4(c.z, ratio);
    c.w = restate4(c.w, ratio);
    at[i] = c;
  }
}

// The values' codes of a page's rows [r0, r1), tile [row][D] in shared memory, into codes [D][rows_of], turned in 4 x 4
// bytes; restate: those of the rows before them come under the new scale.  Sixteen tokens of four elements a thread.
__device__ __forceinline__ void put_values(const uint8_t* tile, uint8_t* codes, int rows_of, int D, int r0, int r1, bool restate,
                                           float ratio, int tid, int threads) {
  const int c0 = restate ? 0 : r0 / kChunk, c1 = (r1 - 1) / kChunk + 1, quads = D / 4, lq = quads == 32 ? 5 : 4;
#pragma unroll 1
  for (int i = tid; i < (c1 - c0) << lq; i += threads) {
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
    uint4* at = reinterpret_cast<uint4*>(codes + (int64_t)d * rows_of + t0);
    if (t0 < r0 || t0 + kChunk > r1) {                        // some of the tokens are old, or not there yet
      uint4 old[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) old[e] = *reinterpret_cast<const uint4*>(reinterpret_cast<uint8_t*>(at) + (int64_t)e * rows_of);
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
      *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(at) + (int64_t)e * rows_of) = make_uint4(w[e][0], w[e][1], w[e][2], w[e][3]);
  }
}

}  // namespace sdv
