// sdv_attend.cu - the entry points of the attention over the 8-bit cache.
#include "sdv_attend.cuh"

using namespace sdv;

extern "C" {

size_t sdv_attend_workspace_bytes(int W, int Hq, int H, int D) {
  if (W < 1 || H < 1 || Hq < H || Hq % H || (D != 64 && D != 128)) return 0;
  const int nt = row_tiles((int64_t)W * (Hq / H)).nt;
  return (size_t)sm_count() * (size_t)attend_warps(nt) * 2 * 8 * (size_t)nt * (size_t)(D + 2) * 4;
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
  if (R > (1 << 24) || (int64_t)B * H * ((R + 7) / 8 + kMaxNt) > 0x7fffffff) return SDV_EINVAL;
  if (!aligned_to(q, 2) || !aligned_to(out, 2) || !aligned_to(lse, 4) || !aligned_to(status, 4) || !aligned_to(lengths, 4) ||
      !aligned_to(counts, 4))
    return SDV_EALIGN;
  if (!workspace || workspace_bytes < sdv_attend_workspace_bytes(W, Hq, H, D)) return SDV_ENOWORKSPACE;
  if (!aligned_to(workspace, 256)) return SDV_EALIGN;
  AttendArgs A{};
  const RowTiles tiles = row_tiles(R);
  A.q = q;
  A.bf16 = dtype == SDV_BF16;
  A.q_vec = aligned_to(q, 16) && q_stride_b % 8 == 0 && q_stride_t % 8 == 0 && q_stride_h % 8 == 0;
  A.q_sb = q_stride_b, A.q_st = q_stride_t, A.q_sh = q_stride_h;
  A.c = CacheView{(uint8_t*)k_codes, (uint8_t*)v_codes, (float*)k_scale, (float*)v_scale, page_table, pages, max_pages, H, D, block};
  A.cpb = chunk_div(block / kChunk);
  A.B = B, A.W = W, A.G = Hq / H, A.R = (int)R, A.RT = tiles.rt;
  A.lengths = lengths, A.counts = counts;
  A.scale2 = scale * kLog2E;
  A.span = span;
  A.out = out, A.lse = lse, A.status = status;
  A.part = (float*)workspace;
  A.ctas = sm_count();
  cudaStream_t s = (cudaStream_t)stream;
  return launched(D == 64 ? launch_attend_64(A, tiles.nt, s) : launch_attend_128(A, tiles.nt, s));
}

}  // extern "C"
