// sdv_keep.cu - moving the rows of an accepted path to the front of a sequence's new tokens.
//
// Row lengths + path[j] of a sequence goes to lengths + j.  A page's scale stays, or grows to the least power of two whose
// 448-fold holds the rows that come into it; where it grows all of the page's codes are restated under it.
// A code c of a page with scale s is code rn(c s / s') under s'.
//
// Rows may come from any page of the sequence's into any other: a CTA has one sequence and head, and holds all
// that moves in shared memory before it writes.
#include "sdv_codes.cuh"
#include "sdv_tree.cuh"

namespace sdv {

constexpr int kKeepThreads = 128;
constexpr int kKeepPages = (SDV_MAX_TREE + kChunk - 2) / kChunk + 1;   // that a tree's rows touch

struct KeepArgs {
  CacheView c;
  const int32_t* path;                   // [B, W]
  const int32_t* lengths;
  uint32_t* status;
  int W;
};

// Four codes that stand for c s, under the scale `to`.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float s, float to) {
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = code_value(w >> (8 * i) & 0xff) * s / to;
  return codes4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ float code_max4(uint32_t w) {        // of the magnitudes that are numbers
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, fabsf(code_value(w >> (8 * i) & 0xff)));
  return m;
}

// Bound by latency: length, then page and scales, then the rows, then the writes, one after another.  A row's values stand a byte
// to a place of `dim`, 32 bytes of DRAM each, so that a moved row of 128 costs 4 KB read and written.  8 sequences x 8 heads,
// up to 6 rows of 128: 4.4 to 5.5 us, a launch's time; 256 x 8, up to 12, pages of 16: 14 to 16.5.
__global__ void __launch_bounds__(kKeepThreads) k_cache_keep(const KeepArgs A) {
  const int b = blockIdx.x / A.c.H, h = blockIdx.x - b * A.c.H, tid = threadIdx.x;
  const int D = A.c.D, T_ = A.c.block, words = D / 4;
  __shared__ uint32_t rows[2][SDV_MAX_TREE][128 / 4];           // codes of keys, values that move
  __shared__ float scale[2][kKeepPages];                        // of the pages
  __shared__ int pages[kKeepPages], from[SDV_MAX_TREE], to[SDV_MAX_TREE], moved_s;
  __shared__ int need[2][kKeepPages];                           // largest magnitudes that come in, as bits of floats
  const int n = min(max(A.lengths[b], 0), (int)kMaxTokens), first = n / T_;
  if (tid < 32) {
    // the path's entries up to the first negative one, two a lane
    int p[2];
    unsigned end[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = 32 * k + tid;
      p[k] = j < A.W ? A.path[(int64_t)b * A.W + j] : -1;
      end[k] = __ballot_sync(0xffffffffu, p[k] < 0);
    }
    const int kept = end[0] ? __ffs(end[0]) - 1 : 32 + (end[1] ? __ffs(end[1]) - 1 : 32);
    bool bad = false;
    int moved = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = 32 * k + tid;
      const bool in = j < kept, ok = p[k] < A.W;
      bad |= in && !ok;
      const unsigned m = __ballot_sync(0xffffffffu, in && ok && p[k] != j);
      if (m >> tid & 1) {
        const int at = moved + __popc(m & ((1u << tid) - 1));
        from[at] = p[k];
        to[at] = j;
      }
      moved += __popc(m);
    }
    if (A.status && h == 0 && bad) atomicOr(A.status + b, SDV_STATUS_BAD_TREE);
    if (tid == 0) moved_s = moved;
  } else if (tid < 32 + kKeepPages) {
    const int k = tid - 32, at = first + k;
    int page = -1;
    if ((int64_t)at * T_ < (int64_t)n + A.W && at < A.c.max_pages) page = A.c.table[(int64_t)b * A.c.max_pages + at];
    if (page >= A.c.pages) page = -1;
    pages[k] = page < 0 ? -1 : page;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      scale[kind][k] = page < 0 ? 1.f : (kind ? A.c.vs : A.c.ks)[(int64_t)page * A.c.H + h];
      need[kind][k] = 0;
    }
  }
  __syncthreads();
  const int moved = moved_s;
  if (!moved) return;
  const auto page_of = [&](int node) { return (n + node) / T_ - first; };        // of the sequence's touched ones
  const auto row_of = [&](int node) { return (n + node) % T_; };
  // the rows, and what their pages need; a row without a page, or on its way to none, is left out
  for (int i = tid; i < moved * words; i += kKeepThreads) {
    const int r = i / words, d4 = i - r * words, pf = page_of(from[r]), pt = page_of(to[r]), page = pages[pf];
    if (page < 0 || pages[pt] < 0) {
      if (A.status && d4 == 0 && h == 0) atomicOr(A.status + b, SDV_STATUS_BAD_PAGE);
      continue;
    }
    const int64_t at = ((int64_t)page * A.c.H + h) * T_ * D;
    const int row = row_of(from[r]);
    const uint32_t k4 = *reinterpret_cast<const uint32_t*>(A.c.k + at + (int64_t)row * D + d4 * 4);
    uint32_t v4 = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) v4 |= (uint32_t)A.c.v[at + (int64_t)(d4 * 4 + e) * T_ + row] << (8 * e);
    rows[0][r][d4] = k4;
    rows[1][r][d4] = v4;
    const float mk = code_max4(k4) * fabsf(scale[0][pf]), mv = code_max4(v4) * fabsf(scale[1][pf]);
    if (mk < INFINITY) atomicMax(&need[0][pt], __float_as_int(mk));              // (the order of maxima changes nothing)
    if (mv < INFINITY) atomicMax(&need[1][pt], __float_as_int(mv));
  }
  __syncthreads();
#pragma unroll 1
  for (int kind = 0; kind < 2; ++kind) {
    uint8_t* codes = kind ? A.c.v : A.c.k;
    for (int k = 0; k < kKeepPages; ++k) {                       // pages whose scale grows
      if (pages[k] < 0) continue;
      const float was = scale[kind][k], s = scale_for(__int_as_float(need[kind][k]));
      if (need[kind][k] == 0 || !(s > fabsf(was))) continue;
      const float ratio = was / s;
      restate_keys(reinterpret_cast<uint4*>(codes + ((int64_t)pages[k] * A.c.H + h) * T_ * D), T_ * D / 16, ratio, tid, kKeepThreads);
      if (tid == 0) (kind ? A.c.vs : A.c.ks)[(int64_t)pages[k] * A.c.H + h] = s;
    }
  }
  __syncthreads();
  for (int i = tid; i < moved * words; i += kKeepThreads) {
    const int r = i / words, d4 = i - r * words, pf = page_of(from[r]), pt = page_of(to[r]), page = pages[pt];
    if (pages[pf] < 0 || page < 0) continue;
    const int64_t at = ((int64_t)page * A.c.H + h) * T_ * D;
    const int row = row_of(to[r]);
    uint32_t w[2];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const float was = scale[kind][pt], s = need[kind][pt] ? scale_for(__int_as_float(need[kind][pt])) : 0.f, now = s > fabsf(was) ? s : was;
      const float sf = scale[kind][pf];
      w[kind] = sf == now ? rows[kind][r][d4] : rescale4(rows[kind][r][d4], sf, now);
    }
    *reinterpret_cast<uint32_t*>(A.c.k + at + (int64_t)row * D + d4 * 4) = w[0];
#pragma unroll
    for (int e = 0; e < 4; ++e) A.c.v[at + (int64_t)(d4 * 4 + e) * T_ + row] = (uint8_t)(w[1] >> (8 * e));
  }
}

}  // namespace sdv

using namespace sdv;

extern "C" int sdv_cache_keep(const int32_t* path, int B, int W, int H, int D, int block, void* k_codes, void* v_codes, float* k_scale,
                              float* v_scale, int64_t pages, const int32_t* page_table, int max_pages, const int32_t* lengths,
                              uint32_t* status, sdv_stream_t stream) {
  if (B < 1 || W < 1 || W > SDV_MAX_TREE || !path || !lengths) return SDV_EINVAL;
  int rc = check_cache(k_codes, v_codes, k_scale, v_scale, pages, page_table, max_pages, H, D, block);
  if (rc) return rc;
  if ((int64_t)B * H > 0x7fffffff) return SDV_EINVAL;
  if (!aligned_to(path, 4) || !aligned_to(lengths, 4) || !aligned_to(status, 4)) return SDV_EALIGN;
  const KeepArgs A{CacheView{(uint8_t*)k_codes, (uint8_t*)v_codes, k_scale, v_scale, page_table, pages, max_pages, H, D, block},
                   path, lengths, status, W};
  k_cache_keep<<<(unsigned)(B * H), kKeepThreads, 0, (cudaStream_t)stream>>>(A);
  return launched(cudaGetLastError());
}
