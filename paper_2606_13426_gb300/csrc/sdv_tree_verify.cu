// sdv_tree_verify.cu - verification of a tree of drafted tokens, and the next token.
//
// At node u with q = softmax(target row / T), p = softmax(draft row / T') the children's tokens x, drawn from p, are tried
// in turn.  Recursive rejection takes x with probability min{1, r(x) / p(x)} and goes on with r' = max{0, r - p}
// normalised, from r = q.  By induction r_k = max{0, q - beta_k p} / M_k with
//   M_k = sum_v max{0, q(v) - beta_k p(v)},  beta_{k+1} = beta_k + M_k,  beta_1 = 0, M_1 = 1
// (where q < beta p, all later remainders are 0 too), so that what is left after any number of rejections is one number
// more and one pass over two rows.  Children without a draft distribution were chosen, not drawn: x is taken with
// probability q(x) / M, M the mass of the tokens not rejected yet.
//
// A cluster of CTAs walks down the tree of one sequence, each with a part of every row's columns, and reads the rows of the
// nodes on the path alone.  What it decides on (tree, tokens, their logits, coins) comes from its first CTA, so that
// all of its CTAs decide alike and meet at the same barriers, even if the caller's arrays change meanwhile.
#include "sdv_token_rows.cuh"
#include "sdv_tree.cuh"

namespace sdv {

constexpr int64_t kAheadBytes = 8 << 20;

struct TreeVerifyArgs {
  const void* q;
  const void* p;                       // NULL: children chosen without chance
  int64_t q_sb, q_sr, p_sb, p_sr;
  const int32_t* tokens;
  const int32_t* parents;
  int W, V;
  float cq, cp, iq, ip;                // log2(e) / T and 1 / T of target and draft
  int ahead;                           // children whose rows are asked for before it is known which is taken
  const int32_t* counts;
  uint64_t seed;
  const float* coins;
  const float* race;
  int32_t* accepted;
  int32_t* path;
  int32_t* next;
  float* ell;
  uint32_t* status;
};

// Tokens that are out of the running, and 64 bits that tell which are surely not among them.
struct Tried {
  int n;
  uint64_t maybe;
};
__device__ __forceinline__ bool tried_before(const Tried& t, const int* list, int v) {
  if (!(t.maybe >> (v & 63) & 1)) return false;
  for (int k = 0; k < t.n; ++k)
    if (list[k] == v) return true;
  return false;
}

// Asks for part `rank` of a row of V elements before it is read.
__device__ __forceinline__ void ask_ahead(const void* row, int V, int bytes, int rank, int log_c, int tid) {
  const int64_t all = (int64_t)V * bytes;
  const char* x = static_cast<const char*>(row);
  const int64_t end = (all * (rank + 1) >> log_c);
  for (int64_t i = (all * rank >> log_c) + tid * 128; i < end; i += kVerThreads * 128)
    asm volatile("prefetch.global.L2 [%0];" ::"l"(x + i));
}

// Statistics of this thread's parts of two rows (the second of none, if !pairs), both on their way at once.  Few vectors a
// turn: a thread's part is often no longer, and the code is run cold.
template <int kDtype>
__device__ __forceinline__ void read_two(const Row<kDtype>& Q, const Row<kDtype>& P, bool pairs, int rank, int log_c, float cq, float cp,
                                         Run& a, Run& c) {
  using E = Num<kDtype>;
  constexpr int kVecs = 4;
  const Part<kDtype, false, kVerThreads> q(Q, rank, log_c), p(P, rank, log_c);
  const int p1 = pairs ? p.v1 : 0, tid = (int)threadIdx.x;
  a = run_empty();
  c = run_empty();
  const auto add = [&](Run& r, const uint4* raw, float scale, int some) {
    float top = vec_max<kDtype>(raw[0]);
#pragma unroll
    for (int u = 1; u < kVecs; ++u) top = max_nan(top, vec_max<kDtype>(raw[u]));
    run_see(r, top, scale);
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      if (u * kVerThreads >= some) break;                    // (for all threads of the CTA)
      float f[E::kPer16];
      E::unpack(raw[u], f);
      run_add<E::kPer16, false>(r, f, scale);
    }
  };
#pragma unroll 1
  for (int v = q.v0, w = p.v0; v - tid < q.v1 || w - tid < p1; v += kVecs * kVerThreads, w += kVecs * kVerThreads) {
    uint4 x[kVecs], y[kVecs];
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      x[u] = y[u] = vec_masked<kDtype>();
      if (v + u * kVerThreads < q.v1) x[u] = q.vec[v + u * kVerThreads];
      if (w + u * kVerThreads < p1) y[u] = p.vec[w + u * kVerThreads];
    }
    add(a, x, cq, q.v1 - v + tid);
    if (pairs) add(c, y, cp, p1 - w + tid);
  }
  if (q.single >= 0) run_one(a, q.x, cq);
  if (pairs && p.single >= 0) run_one(c, p.x, cp);
}

// Bound by latency: a node is a read of its rows' parts, a barrier for their statistics, and with each rejection that leaves
// children a pass and a barrier more.  From cold rows: about 9 us for a root without children and its draw, 4 for each node
// (5.4 before both rows were read at once and the children's asked for ahead), 1 to 2 for a rejection.  1 x 16 x 32768 bf16: 13 us
// with one node taken, 25 with four; 16 x 32 x 131072 42 to 53 by their paths; 48 x 24 x 50001 fp32, children chosen, 26.
template <int kDtype, bool kDrawn>
__global__ void __launch_bounds__(kVerThreads, 3) k_tree_verify(const TreeVerifyArgs A) {
  using E = Num<kDtype>;
  using T = typename E::T;
  constexpr int kPer = E::kPer16;
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), log_c = __ffs(C) - 1;
  const int b = blockIdx.x >> log_c, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int W = A.W, V = A.V;
  __shared__ int tok_s[SDV_MAX_TREE], tried_s[SDV_MAX_TREE];
  __shared__ float eta_s[SDV_MAX_TREE], xq_s[SDV_MAX_TREE], xp_s[SDV_MAX_TREE];
  __shared__ unsigned long long kids_s[SDV_MAX_TREE];
  __shared__ int n_s;
  __shared__ uint32_t bad_s;                                 // rank 0's: status bits found on the way in
  __shared__ float ell_s[SDV_MAX_TREE];
  __shared__ int path_s[SDV_MAX_TREE];
  __shared__ Stat warp_stat[2][kVerWarps], part_stat[2][2][kVerMaxCluster];
  __shared__ float warp_sum[kVerWarps], part_sum[2][kVerMaxCluster];
  __shared__ Best best_w[kVerWarps];
  __shared__ Best best_c[2][kVerMaxCluster];
  const auto at_rank = [&](auto* p, int k) { return C > 1 ? cl.map_shared_rank(p, k) : p; };
  const auto meet = [&] {
    if (C > 1) cl.sync();
    else __syncthreads();
  };
  // Cleared before the arrival: the first CTA writes into all of them as soon as all have arrived.
  for (int i = tid; i < SDV_MAX_TREE; i += kVerThreads) {
    kids_s[i] = 0;
    ell_s[i] = 0.f;
    path_s[i] = -1;
  }
  if (tid == 0) bad_s = 0;
  if (C > 1) cl.barrier_arrive();
  const T* q0 = reinterpret_cast<const T*>(A.q) + b * A.q_sb;
  const T* p0 = kDrawn ? reinterpret_cast<const T*>(A.p) + b * A.p_sb : nullptr;
  const float* race = A.race ? A.race + (int64_t)b * V : nullptr;
  ask_ahead(q0, V, sizeof(T), rank, log_c, tid);             // the root's
  if (kDrawn) ask_ahead(p0, V, sizeof(T), rank, log_c, tid);
  if (race)
    for (int i = share(V, rank, log_c) + tid * 32; i < share(V, rank + 1, log_c); i += kVerThreads * 32)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(race + i));
  __syncthreads();
  if (C > 1) cl.barrier_wait();                              // every CTA of the cluster has started, and has its kids_s cleared
  if (rank == 0) {
    const int64_t at = (int64_t)b * W + tid;
    int up = 0, t = 0;
    float coin = 0.f;
    if (tid < W) {                                           // (beside the counts, not behind them)
      up = A.parents[at];
      t = A.tokens[at];
      if (A.coins) coin = A.coins[at];
    }
    const int n = A.counts ? min(A.counts[b], W) : W;
    if (tid < n) {
      bool bad = false;
      const int p = parent_of(up, tid, bad);
      if (p >= 0) atomicOr(&kids_s[p], 1ull << tid);
      if (bad) atomicOr(&bad_s, SDV_STATUS_BAD_TREE);
      const float eta = A.coins ? coin : ((float)philox_block(A.seed, (uint32_t)b, (uint32_t)tid, kStreamCoin, 0).x + 0.5f) * 0x1p-32f;
      for (int k = 0; k < C; ++k) {
        at_rank(tok_s, k)[tid] = t;
        at_rank(eta_s, k)[tid] = eta;
      }
    }
    __syncthreads();
    for (int k = tid / SDV_MAX_TREE; k < C; k += kVerThreads / SDV_MAX_TREE) {
      const int i = tid % SDV_MAX_TREE;
      if (k) at_rank(kids_s, k)[i] = kids_s[i];
      if (i == 0) *at_rank(&n_s, k) = n;
    }
  }
  meet();
  const int n = n_s;
  if (n <= 0) {                                              // not verified
    if (rank == 0) {
      if (tid == 0) {
        A.accepted[b] = 0;
        A.next[b] = -1;
        if (A.status) A.status[b] = 0;
      }
      if (tid < W) {
        A.path[(int64_t)b * W + tid] = -1;
        if (A.ell) A.ell[(int64_t)b * W + tid] = 0.f;
      }
    }
    if (C > 1) cl.sync();                                    // (no CTA leaves while its shared memory is written)
    return;
  }
  int u = 0, length = 0, sums = 0;
  uint32_t status = 0;
  float beta = 0.f;
  Tried tried{0, 0};
  RowStat rq, rp;
#pragma unroll 1
  for (;; ++length) {
    unsigned long long kids = kids_s[u];
    const bool pairs = kDrawn && kids;
    const T* q = q0 + u * A.q_sr;
    const T* p = pairs ? p0 + u * A.p_sr : q;
    const bool child = rank == 0 && tid < SDV_MAX_TREE && (kids >> tid & 1);
    float xq = 0.f, xp = 0.f;
    if (child) {
      const int t = tok_s[tid];
      if (t >= 0 && t < V) {
        xq = E::to(q[t]);
        if (kDrawn) xp = E::to(p[t]);
      }
    }
    // the rows' statistics
    {
      Run mine, other;
      read_two<kDtype>(Row<kDtype>(q, V), Row<kDtype>(p, V), pairs, rank, log_c, A.cq, A.cp, mine, other);
      const Stat a = run_warp(mine, A.cq);
      if (lane == 0) warp_stat[0][warp] = a;
      if (pairs) {
        const Stat c = run_warp(other, A.cp);
        if (lane == 0) warp_stat[1][warp] = c;
      }
      if (child)
        for (int k = 0; k < C; ++k) {
          at_rank(xq_s, k)[tid] = xq;
          at_rank(xp_s, k)[tid] = xp;
        }
      // the rows of the children likeliest to be taken, while the CTAs meet
      unsigned long long next = kids;
      for (int k = 0; next && k < A.ahead; ++k, next &= next - 1) {
        const int c = __ffsll((long long)next) - 1;
        ask_ahead(q0 + c * A.q_sr, V, sizeof(T), rank, log_c, tid);
        if (kDrawn && kids_s[c]) ask_ahead(p0 + c * A.p_sr, V, sizeof(T), rank, log_c, tid);
      }
      __syncthreads();
      if (warp < 2 && (warp == 0 || pairs)) {
        const Stat c = stat_gather(warp_stat[warp], kVerWarps, lane, warp ? A.cp : A.cq);
        if (lane < C) at_rank(&part_stat[length & 1][warp][0], lane)[rank] = c;
      }
      meet();
      const Stat all = stat_gather(part_stat[length & 1][0], C, lane, A.cq);
      rq = RowStat{all.m, log2f(all.s), all.s};
      rp = RowStat{-INFINITY, 0.f, 1.f};
      if (pairs) {
        const Stat c = stat_gather(part_stat[length & 1][1], C, lane, A.cp);
        rp = RowStat{c.m, log2f(c.s), c.s};
      }
    }
    if (!(rq.m < INFINITY) || !(rp.m < INFINITY)) status |= SDV_STATUS_NONFINITE;
    if (rq.m == -INFINITY || (pairs && rp.m == -INFINITY)) status |= SDV_STATUS_EMPTY_ROW;
    if (tid == 0) path_s[length] = u;
    const bool fair = row_ok(rq) && rp.m < INFINITY;         // the node's children can be tried
    int went = -1;
    float mass = 1.f, gone = 0.f;                            // gone: of q, with the tokens rejected (chosen children)
    beta = 0.f;
    tried = Tried{0, 0};
#pragma unroll 1
    while (kids) {
      const int c = __ffsll((long long)kids) - 1;
      kids &= kids - 1;
      const int x = tok_s[c];
      if (x < 0 || x >= V) {
        status |= SDV_STATUS_BAD_TOKEN;
        continue;
      }
      if (!fair) continue;
      const float dq = (xq_s[c] - rq.m) * A.iq;              // -inf for a masked token
      float ell, value;
      if constexpr (kDrawn) {
        const float dp = row_ok(rp) ? (xp_s[c] - rp.m) * A.ip : -INFINITY;
        // the sums' logarithms are large and nearly equal: that of their ratio, near 0, costs no bits
        ell = !(dq > -INFINITY) ? -INFINITY : dp > -INFINITY ? (dq - dp) + logf(__fdividef(rp.s, rq.s)) : INFINITY;
        value = expf(ell) - beta;
      } else {
        ell = dq - logf(rq.s);
        value = tried_before(tried, tried_s, x) ? 0.f : prob(rq, xq_s[c], A.cq, 0.f);
      }
      if (tid == 0) ell_s[c] = ell;
      if (mass > 0.f && eta_s[c] * mass < value) {
        went = c;
        break;
      }
      if constexpr (kDrawn) {
        if (!row_ok(rp)) continue;                           // nothing to take off q
        beta += mass;
        if (!kids) break;
      } else {
        if (!tried_before(tried, tried_s, x)) {
          gone += value;
          __syncthreads();                                   // the list is read
          if (tid == 0) tried_s[tried.n] = x;
          __syncthreads();
          tried.n += 1;
          tried.maybe |= 1ull << (x & 63);
        }
        if (!kids) break;
        if (gone <= .5f) {                                   // (1 - gone is within two roundings; nearer 1 it would lose bits)
          mass = 1.f - gone;
          continue;
        }
      }
      // what is left of q
      float sum = 0.f;
      each_pair<kDtype>(q, p, V, rank, log_c, tid, kVerThreads, [&](int i, int, const float* y, const float* z) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const float a = prob(rq, y[e], A.cq, 0.f);
          if constexpr (kDrawn) sum += fmaxf(fmaf(-beta, prob(rp, z[e], A.cp, 0.f), a), 0.f);
          else sum += tried_before(tried, tried_s, i + e) ? 0.f : a;
        }
      });
#pragma unroll
      for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      __syncthreads();                                       // the sums before are read
      if (lane == 0) warp_sum[warp] = sum;
      __syncthreads();
      if (tid < C) {
        float s = 0.f;
        for (int k = 0; k < kVerWarps; ++k) s += warp_sum[k];
        at_rank(part_sum[sums & 1], tid)[rank] = s;
      }
      meet();
      mass = 0.f;
      for (int k = 0; k < C; ++k) mass += part_sum[sums & 1][k];
      ++sums;
    }
    if (went < 0) break;
    u = went;
  }
  // the next token
  const T* q = q0 + u * A.q_sr;
  Best best{0.f, -1};
  uint32_t zero = 0;
  for (int attempt = 0; attempt < 2; ++attempt) {
    const bool rest = attempt == 0 && (kDrawn ? beta > 0.f && row_ok(rp) : tried.n > 0);
    Racer top{0.f, 1.f, 0x7fffffff};
    if (row_ok(rq))
      race_part<kDtype>(q, kDrawn && rest ? p0 + u * A.p_sr : q, V, rank, log_c, tid, kVerThreads, race, A.seed, (uint32_t)b, top,
                        [&](int, float x, float y) {
                          const float a = prob(rq, x, A.cq, 0.f);
                          if constexpr (kDrawn) {
                            if (rest) return fmaf(-beta, prob(rp, y, A.cp, 0.f), a);
                          }
                          return a;
                        },
                        [&](int i) { return kDrawn || !rest || !tried_before(tried, tried_s, i); });
    Best me{top.r > 0.f ? top.r / top.e : 0.f, top.i};
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const float ox = __shfl_xor_sync(0xffffffffu, me.x, o);
      const int oi = __shfl_xor_sync(0xffffffffu, me.i, o);
      if (before(ox, oi, me.x, me.i)) me = Best{ox, oi};
    }
    if (lane == 0) best_w[warp] = me;
    __syncthreads();
    if (tid < C) {
      me = best_w[0];
      for (int k = 1; k < kVerWarps; ++k)
        if (before(best_w[k].x, best_w[k].i, me.x, me.i)) me = best_w[k];
      at_rank(best_c[attempt], tid)[rank] = me;
    }
    meet();
    me = best_c[attempt][0];
    for (int k = 1; k < C; ++k)
      if (before(best_c[attempt][k].x, best_c[attempt][k].i, me.x, me.i)) me = best_c[attempt][k];
    if (me.x > 0.f) {
      best = me;
      break;
    }
    if (!rest) break;
    zero = SDV_STATUS_ZERO_DELTA;                            // nothing is left: the target's own
  }
  if (rank == 0) {
    if (tid == 0) {
      A.accepted[b] = length;
      A.next[b] = best.i;
      if (A.status) A.status[b] = status | zero | bad_s;
    }
    if (tid < W) {
      A.path[(int64_t)b * W + tid] = path_s[tid];
      if (A.ell) A.ell[(int64_t)b * W + tid] = ell_s[tid];
    }
  }
}

template <int kDtype>
static cudaError_t launch_tree_verify(const TreeVerifyArgs& A, int B, int dtype, cudaStream_t s) {
  const int C = verify_cluster(B, A.V, dtype);
  const auto verify = A.p ? k_tree_verify<kDtype, true> : k_tree_verify<kDtype, false>;
  if (C > 8) {
    const cudaError_t e = cudaFuncSetAttribute(verify, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return launch_cluster(verify, dim3((unsigned)B * (unsigned)C), kVerThreads, 0, (unsigned)C, false, s, A);
}

}  // namespace sdv

using namespace sdv;

extern "C" int sdv_tree_verify(const void* target, int64_t target_stride_b, int64_t target_stride_row, const void* draft,
                               int64_t draft_stride_b, int64_t draft_stride_row, const int32_t* tokens, const int32_t* parents,
                               int B, int W, int V, int dtype, float temperature, float draft_temperature, const int32_t* counts,
                               uint64_t seed, const float* coins, const float* race, int32_t* accepted_len, int32_t* path,
                               int32_t* next_token, float* log_ratio_out, uint32_t* status_out, sdv_stream_t stream) {
  if (B < 1 || B > (1 << 20) || W < 1 || W > SDV_MAX_TREE || V < 1 || V > (1 << 30) || !token_dtype(dtype)) return SDV_EINVAL;
  if (!temperature_ok(temperature) || !temperature_ok(draft_temperature)) return SDV_EINVAL;
  if (!target || !tokens || !parents || !accepted_len || !path || !next_token) return SDV_EINVAL;
  if (target_stride_row < V || target_stride_b < 0 || (draft && (draft_stride_row < V || draft_stride_b < 0))) return SDV_EINVAL;
  if (!aligned_to(target, elem_bytes(dtype)) || !aligned_to(draft, elem_bytes(dtype))) return SDV_EALIGN;
  const void* four[] = {tokens, parents, counts, coins, race, accepted_len, path, next_token, log_ratio_out, status_out};
  for (const void* p : four)
    if (!aligned_to(p, 4)) return SDV_EALIGN;
  // as many as make 8 MB of all sequences' rows: with one 48 x 24 x 50001 fp32, chosen, take 27.6 us in place of 25.8
  const int64_t rows = (int64_t)B * V * (int64_t)elem_bytes(dtype) * (draft ? 2 : 1);
  const int ahead = (int)(kAheadBytes / rows > SDV_MAX_TREE ? SDV_MAX_TREE : kAheadBytes / rows);
  const TreeVerifyArgs A{target, draft, target_stride_b, target_stride_row, draft_stride_b, draft_stride_row, tokens, parents, W, V,
                         kLog2E / temperature, kLog2E / draft_temperature, 1.f / temperature, 1.f / draft_temperature, ahead,
                         counts, seed, coins, race, accepted_len, path, next_token, log_ratio_out, status_out};
  cudaStream_t s = (cudaStream_t)stream;
  return launched(dtype == SDV_F32    ? launch_tree_verify<SDV_F32>(A, B, dtype, s)
                  : dtype == SDV_BF16 ? launch_tree_verify<SDV_BF16>(A, B, dtype, s)
                                      : launch_tree_verify<SDV_F16>(A, B, dtype, s));
}
