// sdv_attend.cu - the entry points of the attention over the 8-bit cache.
#include "sdv_attend.cuh"

namespace sdv {

// prefix[b]: the steps of the sequences before b, b = 0 .. B.
template <bool kTree, int kStep>
__global__ void __launch_bounds__(kPrefixThreads) k_attend_prefix(const AttendArgs A, int64_t* prefix) {
  __shared__ int64_t warps[kPrefixThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31;
  int64_t before = 0;
  for (int b0 = 0; b0 < A.B; b0 += kPrefixThreads) {
    const int64_t mine = b0 + tid < A.B ? seq_of<kTree, kStep>(A, b0 + tid).steps : 0;
    int64_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    if (lane == 31) warps[tid / 32] = inc;
    __syncthreads();
    int64_t base = before;
    for (int w = 0; w < kPrefixThreads / 32; ++w) {
      if (w < tid / 32) base += warps[w];
      before += warps[w];
    }
    if (b0 + tid < A.B) prefix[b0 + tid] = base + inc - mine;
    __syncthreads();
  }
  if (tid == 0) prefix[A.B] = before;
}

cudaError_t launch_attend_prefix(const AttendArgs& A, int64_t* prefix, cudaStream_t s) {
  const auto kern = !A.parents ? k_attend_prefix<false, kSub> : !A.step ? k_attend_prefix<true, kSub> : k_attend_prefix<true, 0>;
  kern<<<1, kPrefixThreads, 0, s>>>(A, prefix);
  return cudaGetLastError();
}

AttendSpace attend_space(int B, int W, int Hq, int H, int D) {
  const int nt = row_tiles((int64_t)W * (Hq / H), kMaxNt).nt;             // (no choice of tiles has more)
  const size_t part = ((size_t)sm_count() * kAttendWarps * 2 * 8 * (size_t)nt * (size_t)(D + 2) * 4 + 255) / 256 * 256;
  return AttendSpace{part, part + (B > kPrefixFrom ? ((size_t)B + 1) * sizeof(int64_t) : 0)};
}

}  // namespace sdv

using namespace sdv;

extern "C" {

size_t sdv_attend_workspace_bytes(int B, int W, int Hq, int H, int D) {
  if (B < 1 || W < 1 || H < 1 || Hq < H || Hq % H || (D != 64 && D != 128)) return 0;
  return attend_space(B, W, Hq, H, D).total;
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
  const AttendSpace space = attend_space(B, W, Hq, H, D);
  if (!workspace || workspace_bytes < space.total) return SDV_ENOWORKSPACE;
  if (!aligned_to(workspace, 256)) return SDV_EALIGN;
  AttendArgs A{};
  A.span = span < max_pages * block ? span : 0;             // as many as there can be, or more: all
  const int64_t tokens = min(A.span > 0 ? (int64_t)A.span + W + kSub : kMaxTokens, (int64_t)max_pages * block);
  const RowTiles tiles = choose_tiles(R, (int64_t)B * H, (tokens + kSub - 1) / kSub, D, sm_count() * kAttendWarps);
  A.q = q;
  A.bf16 = dtype == SDV_BF16;
  A.q_vec = aligned_to(q, 16) && q_stride_b % 8 == 0 && q_stride_t % 8 == 0 && q_stride_h % 8 == 0;
  A.q_sb = q_stride_b, A.q_st = q_stride_t, A.q_sh = q_stride_h;
  A.c = CacheView{(uint8_t*)k_codes, (uint8_t*)v_codes, (float*)k_scale, (float*)v_scale, page_table, pages, max_pages, H, D, block};
  A.cpb = chunk_div(block / kChunk);
  A.B = B, A.W = W, A.G = Hq / H, A.R = (int)R, A.RT = tiles.rt;
  A.lengths = lengths, A.counts = counts;
  A.scale2 = scale * kLog2E;
  A.out = out, A.lse = lse, A.status = status;
  A.part = (float*)workspace;
  A.ctas = sm_count();
  cudaStream_t s = (cudaStream_t)stream;
  if (B > kPrefixFrom) {
    int64_t* prefix = (int64_t*)((char*)workspace + space.part);
    const cudaError_t e = launch_attend_prefix(A, prefix, s);
    if (e != cudaSuccess) return launched(e);
    A.prefix = prefix;
  }
  return launched(D == 64 ? launch_attend_64(A, tiles.nt, s) : launch_attend_128(A, tiles.nt, s));
}

}  // extern "C"
