// sdv_cache.cu - appending keys and values to the 8-bit cache.
//
// A page's scale for a head is the least power of two whose 448-fold (the largest e4m3 value)
// holds every magnitude in it: s = 2^k, k = ceil(log2(amax / 448)); codes are rn(x / s).  Tokens
// that a page already holds keep their codes unless the scale grows; then they are restated
// under the new one, which is exact (powers of two) but for what underflows.  Between the reads
// and the writes a CTA owns its page and head, so that nothing is shared.
#include "sdv_cache.cuh"

namespace sdv {

constexpr int kAppendThreads = 128;

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

// x / s, rounded once: a product where s is a power of two.
struct Divide {
  float s, inv;
  bool pow2;
  __device__ __forceinline__ explicit Divide(float s_) : s(s_) {
    pow2 = (__float_as_uint(s) & 0x807fffffu) == 0 && s >= 0x1p-126f && s <= 0x1p126f;
    inv = pow2 ? 1.f / s : 0.f;
  }
  __device__ __forceinline__ float operator()(float x) const { return pow2 ? x * inv : x / s; }
};

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

// Sixteen consecutive elements, in 32 bits.
template <int kDtype>
__device__ __forceinline__ void load16(const typename Num<kDtype>::T* p, bool vec, float* f) {
  using E = Num<kDtype>;
  if (vec) {
#pragma unroll
    for (int i = 0; i < 16 / E::kPer16; ++i) E::unpack(__ldg(reinterpret_cast<const uint4*>(p) + i), f + i * E::kPer16);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = E::to(p[i]);
  }
}

// One CTA per (sequence, head, page, keys or values).
template <int kDtype>
__global__ void __launch_bounds__(kAppendThreads) k_cache_append(const AppendArgs A) {
  using T = typename Num<kDtype>::T;
  extern __shared__ __align__(16) uint8_t tile[];      // values: codes [token][D]
  __shared__ float red[kAppendThreads / 32];
  const int kind = blockIdx.x & 1;
  int64_t u = blockIdx.x >> 1;
  const int j = (int)(u % A.nb);
  u /= A.nb;
  const int h = (int)(u % A.c.H);
  const int64_t b = u / A.c.H;
  const int tid = threadIdx.x, T_ = A.c.block, D = A.c.D;
  const int64_t n = max(A.lengths[b], 0);
  const int count = min(A.counts ? A.counts[b] : A.W, A.W);
  const int64_t block_id = n / T_ + j;
  const int64_t lo = max(n, block_id * T_), hi = min(n + count, (block_id + 1) * T_);
  if (lo >= hi) return;
  const int64_t page = block_id < A.c.max_pages ? A.c.table[b * A.c.max_pages + block_id] : -1;
  if (page < 0 || page >= A.c.pages) {
    if (A.status && tid == 0) atomicOr(A.status + b, SDV_STATUS_BAD_PAGE);
    return;
  }
  const int kept = (int)max((int64_t)0, n - block_id * T_);      // tokens the page holds already
  const int r0 = (int)(lo - block_id * T_), m = (int)(hi - lo);
  const T* x = reinterpret_cast<const T*>(A.x[kind]) + b * A.sb + (lo - n) * A.st + h * A.sh;
  const bool vec = aligned16(x) && (A.st * sizeof(T)) % 16 == 0;
  const int per = D / 16, units = m * per;
  float amax = 0.f;
  for (int i = tid; i < units; i += kAppendThreads) {
    float f[16];
    load16<kDtype>(x + (i / per) * A.st + (i % per) * 16, vec, f);
#pragma unroll
    for (int e = 0; e < 16; ++e) amax = fmaxf(amax, fabsf(f[e]) < INFINITY ? fabsf(f[e]) : 0.f);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if ((tid & 31) == 0) red[tid >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kAppendThreads / 32; ++w) amax = fmaxf(amax, red[w]);
  const int64_t ph = page * A.c.H + h;
  float* scale = (kind ? A.c.vs : A.c.ks) + ph;
  const float need = scale_for(amax);
  const float s_old = kept ? *scale : need;
  __syncthreads();                                     // read by all before it is replaced below
  const float s = fmaxf(s_old, need);
  const bool restate = kept && s != s_old;
  const float ratio = s_old / s;
  const Divide by(s);
  uint8_t* codes = (kind ? A.c.v : A.c.k) + ph * T_ * D;
  if (kind == 0) {
    for (int i = tid; i < units; i += kAppendThreads) {
      float f[16];
      load16<kDtype>(x + (i / per) * A.st + (i % per) * 16, vec, f);
#pragma unroll
      for (int e = 0; e < 16; ++e) f[e] = by(f[e]);
      uint4 c;
      c.x = codes4(f[0], f[1], f[2], f[3]);
      c.y = codes4(f[4], f[5], f[6], f[7]);
      c.z = codes4(f[8], f[9], f[10], f[11]);
      c.w = codes4(f[12], f[13], f[14], f[15]);
      *reinterpret_cast<uint4*>(codes + (int64_t)r0 * D + i * 16) = c;
    }
    if (restate)
      for (int i = tid; i < kept * per; i += kAppendThreads) {
        uint4* at = reinterpret_cast<uint4*>(codes) + i;
        uint4 c = *at;
        c.x = restate4(c.x, ratio);
        c.y = restate4(c.y, ratio);
        c.z = restate4(c.z, ratio);
        c.w = restate4(c.w, ratio);
        *at = c;
      }
  } else {
    for (int i = tid; i < units; i += kAppendThreads) {
      float f[16];
      load16<kDtype>(x + (i / per) * A.st + (i % per) * 16, vec, f);
#pragma unroll
      for (int e = 0; e < 16; ++e) f[e] = by(f[e]);
      uint4 c;
      c.x = codes4(f[0], f[1], f[2], f[3]);
      c.y = codes4(f[4], f[5], f[6], f[7]);
      c.z = codes4(f[8], f[9], f[10], f[11]);
      c.w = codes4(f[12], f[13], f[14], f[15]);
      reinterpret_cast<uint4*>(tile)[i] = c;
    }
    __syncthreads();
    // the page's rows along the tokens, sixteen tokens at a time
    const int c0 = restate ? 0 : r0 / kChunk, c1 = (r0 + m - 1) / kChunk + 1;
    for (int i = tid; i < (c1 - c0) * D; i += kAppendThreads) {
      const int d = i % D, t0 = (c0 + i / D) * kChunk;
      uint4* at = reinterpret_cast<uint4*>(codes + (int64_t)d * T_ + t0);
      uint32_t w[4];
      const bool whole = t0 >= r0 && t0 + kChunk <= r0 + m;
      if (!whole) {
        const uint4 c = *at;
        w[0] = c.x, w[1] = c.y, w[2] = c.z, w[3] = c.w;
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t v = 0;
        const uint32_t was = whole ? 0 : w[q];
        const uint32_t again = restate && t0 + 4 * q < kept ? restate4(was, ratio) : was;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = t0 + 4 * q + e;
          const uint32_t byte = t >= r0 && t < r0 + m ? tile[(t - r0) * D + d]
                                                      : ((t < kept ? again : was) >> (8 * e) & 0xff);
          v |= byte << (8 * e);
        }
        w[q] = v;
      }
      *at = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  if (tid == 0 && (!kept || restate)) *scale = s;
}

template <int kDtype>
static cudaError_t launch_append(const AppendArgs& A, int64_t grid, cudaStream_t s) {
  k_cache_append<kDtype><<<(unsigned)grid, kAppendThreads, (size_t)A.c.block * A.c.D, s>>>(A);
  return cudaGetLastError();
}

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
  const int64_t grid = 2 * (int64_t)B * H * nb;
  if (grid > 0x7fffffff) return SDV_EINVAL;
  const AppendArgs A{{k_new, v_new}, stride_b, stride_t, stride_h,
                     CacheView{(uint8_t*)k_codes, (uint8_t*)v_codes, k_scale, v_scale, page_table, pages, max_pages, H, D, block},
                     W, nb, lengths, counts, status};
  cudaStream_t s = (cudaStream_t)stream;
  return launched(dtype == SDV_F32    ? launch_append<SDV_F32>(A, grid, s)
                  : dtype == SDV_BF16 ? launch_append<SDV_BF16>(A, grid, s)
                                      : launch_append<SDV_F16>(A, grid, s));
}
