// sdv_cache.cu - appending keys and values to the 8-bit cache.
//
// A page's scale for a head is the least power of two whose 448-fold (the largest e4m3 value)
// holds every magnitude in it: s = 2^k, k = ceil(log2(amax / 448)); codes are rn(x / s).  Tokens
// that a page already holds keep their codes unless the scale grows; then they are restated
// under the new one, which is exact (powers of two) but for what underflows.  Between the reads
// and the writes a CTA owns its page and head, so that nothing is shared.
#include "sdv_codes.cuh"

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
      if (restate) restate_keys(reinterpret_cast<uint4*>(codes), r0 << lper, ratio, tid, kAppendThreads);
    } else {
      __syncthreads();
      put_values(tile, codes, T_, D, r0, r1, restate, ratio, tid, kAppendThreads);
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
