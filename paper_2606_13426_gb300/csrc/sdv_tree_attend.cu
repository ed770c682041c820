// sdv_tree_attend.cu - the entry points of the attention of a drafted tree over the 8-bit cache.
#include "sdv_attend.cuh"

namespace sdv {

constexpr int kTileRowsMost = 128;          // rows of a tile of the matrix unit's kernels

// The time of a call of those kernels, in tenths of a microsecond, as choose_tiles has it for the others: a fixed part, the
// steps of a team and the items that it begins or ends.  Fitted to 60 shapes of 20 to 256 rows whose page tables are as wide as their
// sequences (the lengths are on the device: a wider table counts as long sequences); both kernels (us), heads of 128,
// 8 key heads: 64 rows over 1 x 3000 keys 22 and 29 here, 8 x 1000 37 and 28, 32 x 600 77 and 53, 32 x 3000 164 and 101,
// 128 x 200 155 and 116; 20 rows over 32 x 3000 79 and 100, 48 rows 130 and 101; heads of 64: 64 rows over 32 x 3000 105 and 88,
// 32 rows 67 and 70.
static int64_t rows_cost(int64_t rt, int64_t heads, int64_t longest, int step, int D) {
  const int64_t teams = sm_count() / rt;
  return (D == 128 ? 190 : 150) + heads * ((longest + step - 1) / step) * (D == 128 ? 15 : 11) / teams + (heads / teams + 1) * 90;
}

static AttendSpace tree_space(int B, int W, int Hq, int H, int D) {
  AttendSpace space = attend_space(B, W, Hq, H, D);
  const size_t part = tree_rows_part(D);
  if (part > space.part) {
    space.total += part - space.part;
    space.part = part;
  }
  return space;
}

// How a call is laid out: the tiles of rows, and which kernels take them.
struct TreeChoice {
  RowTiles tiles;
  int step;                                 // keys of a step of the kernels for many rows
  bool many;                                // those kernels
};
static TreeChoice choose_tree(int64_t R, int64_t heads, int D, int block, int max_pages) {
  TreeChoice c;
  const int64_t longest = (int64_t)max_pages * block, rt = (R + kTileRowsMost - 1) / kTileRowsMost;
  int64_t cost = 0;
  c.step = kTileKeys / block * block;
  c.tiles = choose_tiles(R, heads, (longest + kSub - 1) / kSub, D, sm_count() * kAttendWarps, &cost);
  c.many = rt <= sm_count() && rows_cost(rt, heads, longest, c.step, D) < cost;
  if (c.many) c.tiles.rt = (int)rt;
  return c;
}
// Two partials a CTA, with a row's references and sum, what its two groups put aside, and whether it gave up.
size_t tree_rows_part(int D) { return (size_t)sm_count() * (2 * kTileRowsMost * (size_t)(D + 3 + D) + 1) * 4 / 256 * 256 + 256; }

}  // namespace sdv

using namespace sdv;

extern "C" {

size_t sdv_tree_attend_workspace_bytes(int B, int W, int Hq, int H, int D) {
  if (B < 1 || W < 1 || W > SDV_MAX_TREE || H < 1 || Hq < H || Hq % H || (D != 64 && D != 128)) return 0;
  return tree_space(B, W, Hq, H, D).total;
}

int sdv_tree_attend_row_tiles(int B, int W, int Hq, int H, int D, int block, int max_pages) {
  if (!sdv_tree_attend_workspace_bytes(B, W, Hq, H, D) || block < 16 || block % 16 || block > SDV_MAX_BLOCK || max_pages < 1 ||
      (int64_t)max_pages * block > kMaxTokens)
    return SDV_EINVAL;
  const TreeChoice c = choose_tree((int64_t)W * (Hq / H), (int64_t)B * H, D, block, max_pages);
  return c.many ? c.tiles.rt : 0;
}

int sdv_tree_attend(const void* q, int64_t q_stride_b, int64_t q_stride_t, int64_t q_stride_h, int dtype, int B, int W, int Hq,
                    int H, int D, int block, const void* k_codes, const void* v_codes, const float* k_scale,
                    const float* v_scale, int64_t pages, const int32_t* page_table, int max_pages, const int32_t* lengths,
                    const int32_t* parents, const int32_t* counts, float scale, void* out, float* lse, uint32_t* status,
                    void* workspace, size_t workspace_bytes, sdv_stream_t stream) {
  if ((dtype != SDV_BF16 && dtype != SDV_F16) || B < 1 || W < 1 || W > SDV_MAX_TREE || H < 1 || Hq < H || Hq % H || !q || !lengths ||
      !parents || !out)
    return SDV_EINVAL;
  int rc = check_cache(k_codes, v_codes, k_scale, v_scale, pages, page_table, max_pages, H, D, block);
  if (rc) return rc;
  if (q_stride_b < 0 || q_stride_t < 0 || q_stride_h < 0 || !(fabsf(scale) < INFINITY)) return SDV_EINVAL;
  const int64_t R = (int64_t)W * (Hq / H);
  if (R > (1 << 24) || (int64_t)B * H * ((R + 7) / 8 + kMaxNt) > 0x7fffffff) return SDV_EINVAL;
  if (!aligned_to(q, 2) || !aligned_to(out, 2) || !aligned_to(lse, 4) || !aligned_to(status, 4) || !aligned_to(lengths, 4) ||
      !aligned_to(parents, 4) || !aligned_to(counts, 4))
    return SDV_EALIGN;
  const AttendSpace space = tree_space(B, W, Hq, H, D);
  if (!workspace || workspace_bytes < space.total) return SDV_ENOWORKSPACE;
  if (!aligned_to(workspace, 256)) return SDV_EALIGN;
  AttendArgs A{};
  const TreeChoice choice = choose_tree(R, (int64_t)B * H, D, block, max_pages);
  const RowTiles tiles = choice.tiles;
  A.q = q;
  A.bf16 = dtype == SDV_BF16;
  A.q_vec = aligned_to(q, 16) && q_stride_b % 8 == 0 && q_stride_t % 8 == 0 && q_stride_h % 8 == 0;
  A.out_vec = aligned_to(out, 16);
  A.q_sb = q_stride_b, A.q_st = q_stride_t, A.q_sh = q_stride_h;
  A.c = CacheView{(uint8_t*)k_codes, (uint8_t*)v_codes, (float*)k_scale, (float*)v_scale, page_table, pages, max_pages, H, D, block};
  A.cpb = chunk_div(block / kChunk);
  A.B = B, A.W = W, A.G = Hq / H, A.R = (int)R, A.RT = tiles.rt;
  A.lengths = lengths, A.counts = counts, A.parents = parents;
  A.scale2 = scale * kLog2E;
  A.out = out, A.lse = lse, A.status = status;
  A.part = (float*)workspace;
  A.ctas = sm_count();
  A.step = choice.many ? choice.step : 0;
  cudaStream_t s = (cudaStream_t)stream;
  if (B > kPrefixFrom) {
    int64_t* prefix = (int64_t*)((char*)workspace + space.part);
    const cudaError_t e = launch_attend_prefix(A, prefix, s);
    if (e != cudaSuccess) return launched(e);
    A.prefix = prefix;
  }
  if (choice.many) {
    const int rows = (int)((R + tiles.rt - 1) / tiles.rt);
    return launched(D == 64 ? launch_tree_rows_64(A, rows, s) : launch_tree_rows_128(A, rows, s));
  }
  return launched(D == 64 ? launch_tree_attend_64(A, tiles.nt, s) : launch_tree_attend_128(A, tiles.nt, s));
}

}  // extern "C"
