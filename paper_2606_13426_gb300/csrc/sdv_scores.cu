// sdv_scores.cu - log probabilities of given tokens, entropy and the top alternatives of rows
// of logits (k_scores), the gradient from given statistics (k_scores_grad), and statistics and
// gradient in one pass over the logits (k_scores_train).
//
// With d_v = x_v - m, m = max x, and s = sum e^{d_v/T}:
//   log p_t = d_t/T - log s,     H = log s - (1/T) sum p_v d_v,
//   dx_v = (1/T) [g_lp (1[v = t] - p_v) - g_H p_v (log p_v + H)].
// A row is split over the CTAs of a cluster, which join their statistics through distributed
// shared memory.
#include <cstdint>

#include "sdv_tokens.cuh"

namespace sdv {

// Groups of threads whose maxima give the alternatives' threshold, the k-th largest of them: 32, or twice as
// many where k is near 32, the least of 32 maxima being a low one (32 alternatives of 26 x 128050 fp32:
// 36 us with 32 groups).
constexpr int kGroups = 32, kManyGroups = 64, kManyFrom = 25;
constexpr int kCandMax = 512;          // candidates a CTA ranks; more: k passes over its part

struct ScoreArgs {
  const void* x;
  int64_t stride;
  int V;
  const int32_t* tokens;
  float c;                             // log2(e) / T
  float inv_t;
  int top_k;
  float* logprob;
  float* entropy;
  float* row_max;
  float* log_sum;
  int32_t* top_ids;
  float* top_lp;
  uint32_t* status;
};

struct Cand {
  float x;
  int i;
};

// The token of a row and its logit, read before any gradient is written (which may be in place).
struct Token {
  int t;
  float x;
};
template <int kDtype>
__device__ __forceinline__ Token row_token(const ScoreArgs& A, const typename Num<kDtype>::T* row, int64_t n) {
  Token k{A.tokens ? A.tokens[n] : -1, 0.f};
  if (k.t >= 0 && k.t < A.V) k.x = Num<kDtype>::to(row[k.t]);
  return k;
}

// The outputs of a row other than its alternatives.
__device__ __forceinline__ void write_row(const ScoreArgs& A, int64_t n, const Stat& a, const Token& tok) {
  uint32_t st = 0;
  const bool bad = !(a.m < INFINITY);                    // NaN or +inf
  const bool empty = a.m == -INFINITY;
  if (bad) st |= SDV_STATUS_NONFINITE;
  if (empty) st |= SDV_STATUS_EMPTY_ROW;
  const float log_s = bad ? NAN : (empty ? -INFINITY : logf(a.s));
  if (A.row_max) A.row_max[n] = bad ? NAN : a.m;
  if (A.log_sum) A.log_sum[n] = log_s;
  if (A.entropy) A.entropy[n] = bad ? NAN : (empty ? 0.f : log_s - a.w / a.s * A.inv_t);
  if (A.tokens) {
    const int t = tok.t;
    float lp = 0.f;
    if (t != -1) {
      if (t < 0 || t >= A.V) {
        st |= SDV_STATUS_BAD_TOKEN;
        lp = NAN;
      } else if (bad) {
        lp = NAN;
      } else {
        lp = empty ? -INFINITY : (tok.x - a.m) * A.inv_t - log_s;
      }
    }
    A.logprob[n] = lp;
  }
  if (A.status) A.status[n] = st;
}

// Ranks the n candidates in `c` by counting, eight lanes a candidate, and hands those of rank < k to
// put(rank, candidate).
template <typename Put>
__device__ __forceinline__ void rank_candidates(const Cand* c, int n, int k, Put put) {
#pragma unroll 1
  for (int i = threadIdx.x / 8; i - (int)(threadIdx.x & 31) / 8 < n; i += kScoreThreads / 8) {
    const Cand me = i < n ? c[i] : Cand{0.f, 0};
    int r = 0;
#pragma unroll 1
    for (int j = threadIdx.x & 7; j < n; j += 8) {
      const Cand o = c[j];
      r += before(o.x, o.i, me.x, me.i);
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
    if (i < n && r < k && (threadIdx.x & 7) == 0) put(r, me);
  }
}

// Statistics of a row in one read: a thread keeps sums against a reference that moves only when a logit
// passes it by 2^8, a warp, then the cluster's leader rebase them to the row's maximum.  Alternatives: the
// k-th largest of 32 groups' maxima (64 groups' from k = 25 on) is a threshold that at least k logits reach; the few threads above it
// read their vectors again (from the L2), and what reaches it is ranked by counting.
// Bound by the read where rows are many (600 x 131072 bf16 without alternatives 26.8 us, 5.9 TB/s; 38 with
// 20), by latency where they are few (8 x 65536: 3.7 us, 5.7 with 8; 144 x 131072: 10.3 us, 15 with 20).
// What follows the row's read runs once a CTA, mostly from a cold instruction cache (a line of eight
// instructions took about 350 cycles where rows fill the L2): loops there are not unrolled.
template <int kDtype, bool kTop>
__global__ void __launch_bounds__(kScoreThreads, 4) k_scores(const ScoreArgs A) {
  using E = Num<kDtype>;
  using T = typename E::T;
  constexpr int kPer = E::kPer16;
  constexpr int kWarps = kScoreThreads / 32;
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), log_c = __ffs(C) - 1;
  const int64_t n = blockIdx.x >> log_c;
  const int tid = threadIdx.x;
  __shared__ Stat stats[kScoreMaxCluster * kWarps];           // the leader's: every warp's
  __shared__ int listed[kScoreMaxCluster];
  __shared__ __align__(16) float gmax[kManyGroups];
  __shared__ int ncand, nhot;
  __shared__ int hot[kTop ? kCandMax : 1];
  __shared__ Cand cand[kTop ? kCandMax : 1];
  __shared__ Cand lists[kTop ? kScoreMaxCluster * SDV_MAX_TOP : 1];
  __shared__ Cand best_w[kWarps];
  __shared__ uint8_t who[kWarps][32];
  if (C > 1) cl.barrier_arrive();
  const T* row = reinterpret_cast<const T*>(A.x) + n * A.stride;
  const Row<kDtype> R(row, A.V);
  Token tok{-1, 0.f};
  if (rank == 0 && tid == 0) tok = row_token<kDtype>(A, row, n);   // (under way with the row)
  const Part<kDtype, true> P(R, rank, log_c);
  const int first = P.v0;
  const Run run = P.read(A.c);
  const float tm = run.top;                   // the largest of this thread's logits
  Stat a = run_warp(run, A.c);
  if constexpr (kTop) {
    float g = tm;                             // a group's
    const int of = kScoreThreads / (A.top_k < kManyFrom ? kGroups : kManyGroups);
#pragma unroll 1
    for (int o = 1; o < of; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, o));
    if ((tid & (of - 1)) == 0) gmax[tid / of] = g;
    if (tid == 0) ncand = nhot = 0;
    __syncthreads();
  }
  if (C > 1) cl.barrier_wait();               // the leader has started: its memory can be written
  if ((tid & 31) == 0) (C > 1 ? cl.map_shared_rank(stats, 0) : stats)[rank * kWarps + tid / 32] = a;
  if constexpr (kTop) {
    // At least k of the part's logits are at or above the k-th largest of the groups' maxima.
    float thr = INFINITY;
    const int groups = A.top_k < kManyFrom ? kGroups : kManyGroups;
#pragma unroll 1
    for (int i = tid & 31; i < groups; i += 32) {
      const float mine_max = gmax[i];
      int above = 0;
#pragma unroll 8
      for (int j = 0; j < groups; j += 4) {
        const float4 o = *reinterpret_cast<const float4*>(gmax + j);
        above += (o.x > mine_max) + (o.y > mine_max) + (o.z > mine_max) + (o.w > mine_max);
      }
      if (above < A.top_k) thr = fminf(thr, mine_max);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) thr = fminf(thr, __shfl_xor_sync(0xffffffffu, thr, o));
    auto keep = [&](float x, int i) {
      if (x >= thr && x > -INFINITY) {
        const int at = atomicAdd(&ncand, 1);     // their order does not matter: they are ranked
        if (at < kCandMax) cand[at] = Cand{x, i};
      }
    };
    // The vectors of the threads that have candidates (about as many as alternatives are wanted) are
    // read again, a warp's threads' together, and then those that hold some, an element a thread.
    const unsigned flagged = __ballot_sync(0xffffffffu, tm >= thr && tm > -INFINITY);
    if (flagged) {
      const int nf = __popc(flagged), w0 = first - (tid & 31);           // the warp's first vector
      if (flagged >> (tid & 31) & 1) who[tid / 32][__popc(flagged & ((1u << (tid & 31)) - 1u))] = (uint8_t)(tid & 31);
      __syncwarp();
      const int log_v = 32 - __clz(max((P.v1 - w0 + kScoreThreads - 1) / kScoreThreads - 1, 0));   // vectors a thread, as a power of two
#pragma unroll 1
      for (int i = tid & 31; i < nf << log_v; i += 64) {
        const int i2 = i + 32;
        const int va = w0 + who[tid / 32][i >> log_v] + (i & ((1 << log_v) - 1)) * kScoreThreads;
        const int vb = i2 < nf << log_v ? w0 + who[tid / 32][i2 >> log_v] + (i2 & ((1 << log_v) - 1)) * kScoreThreads : P.v1;
        const uint4 ra = va < P.v1 ? __ldg(P.vec + va) : vec_masked<kDtype>(), rb = vb < P.v1 ? __ldg(P.vec + vb) : vec_masked<kDtype>();
        const float ta = vec_max<kDtype>(ra), tb = vec_max<kDtype>(rb);
        if (ta >= thr && va < P.v1) {
          const int at = atomicAdd(&nhot, 1);
          if (at < kCandMax) hot[at] = va;
        }
        if (tb >= thr && vb < P.v1) {
          const int at = atomicAdd(&nhot, 1);
          if (at < kCandMax) hot[at] = vb;
        }
      }
      if (P.single >= 0) keep(P.x, P.single);
    }
    __syncthreads();
    const int hots = nhot;
#pragma unroll 1
    for (int i = tid; i < min(hots, kCandMax) * kPer; i += kScoreThreads) {
      const int at = R.head + hot[i / kPer] * kPer + i % kPer;
      keep(E::to(row[at]), at);
    }
    __syncthreads();
    Cand* mine = (C > 1 ? cl.map_shared_rank(lists, 0) : lists) + rank * A.top_k;
    int nc = ncand;
    if (nc <= kCandMax && hots <= kCandMax) {
      rank_candidates(cand, nc, A.top_k, [&](int r, Cand c) { mine[r] = c; });
      nc = min(nc, A.top_k);
    } else {                                      // many equal logits: one alternative per pass
      Cand last{INFINITY, -1};
      for (nc = 0; nc < A.top_k; ++nc) {
        Cand b{-INFINITY, 0x7fffffff};
        auto see = [&](float x, int i) {
          if (x > -INFINITY && before(last.x, last.i, x, i) && before(x, i, b.x, b.i)) b = Cand{x, i};
        };
        for (int v = first; v < P.v1; v += kScoreThreads) {
          float f[kPer];
          E::unpack(__ldg(P.vec + v), f);
#pragma unroll
          for (int e = 0; e < kPer; ++e) see(f[e], R.head + v * kPer + e);
        }
        if (P.single >= 0) see(P.x, P.single);
#pragma unroll
        for (int o = 16; o; o >>= 1) {
          const float ox = __shfl_xor_sync(0xffffffffu, b.x, o);
          const int oi = __shfl_xor_sync(0xffffffffu, b.i, o);
          if (before(ox, oi, b.x, b.i)) b = Cand{ox, oi};
        }
        __syncthreads();
        if ((tid & 31) == 0) best_w[tid >> 5] = b;
        __syncthreads();
        b = best_w[0];
        for (int w = 1; w < kWarps; ++w)
          if (before(best_w[w].x, best_w[w].i, b.x, b.i)) b = best_w[w];
        if (!(b.x > -INFINITY)) break;
        if (tid == 0) mine[nc] = b;
        last = b;
      }
    }
    if (tid == 0) (C > 1 ? cl.map_shared_rank(listed, 0) : listed)[rank] = nc;
  }
  if (C > 1) {
    cl.sync();
    if (rank) return;
  } else {
    __syncthreads();
  }
  if (!kTop && tid >= 32) return;
  a = stat_gather(stats, C * kWarps, tid & 31, A.c);
  if (tid == 0) write_row(A, n, a, tok);
  if constexpr (kTop) {
    const bool bad = !(a.m < INFINITY);
    const float log_s = logf(a.s);
    const int k = A.top_k;
    auto put = [&](int r, Cand c) {
      const bool none = bad || c.i < 0;
      A.top_ids[n * k + r] = none ? -1 : c.i;
      A.top_lp[n * k + r] = bad ? NAN : (none ? -INFINITY : (c.x - a.m) * A.inv_t - log_s);
    };
    int total = 0;
#pragma unroll 1
    for (int r = 0; r < C; ++r) total += listed[r];
    if (bad) {
      total = 0;
    } else if (C == 1) {
      if (tid < min(total, k)) put(tid, lists[tid]);
    } else {
      // a lane for each list that an alternative has its place in: its own, and the others by bisection
#pragma unroll 1
      for (int i = tid / 8; i - (tid & 31) / 8 < C * k; i += kScoreThreads / 8) {
        const int q = i / k, j = i - q * k, p = tid & 7;
        const bool is = i < C * k && j < listed[q];
        const Cand me = is ? lists[i] : Cand{0.f, 0};
        int lo = 0, hi = p < C ? listed[p] : 0;
        if (p == q) lo = hi = j;
#pragma unroll 1
        while (lo < hi) {
          const int mid = (lo + hi) / 2;
          const Cand o = lists[p * k + mid];
          if (before(o.x, o.i, me.x, me.i)) lo = mid + 1;
          else hi = mid;
        }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) lo += __shfl_xor_sync(0xffffffffu, lo, o);
        if (is && lo < k && p == 0) put(lo, me);
      }
    }
#pragma unroll 1
    for (int r = total + tid; r < k; r += kScoreThreads) put(r, Cand{-INFINITY, -1});
  }
}

struct GradArgs {
  const void* x;
  int64_t stride;
  int V;
  const int32_t* tokens;
  float c, inv_t;
  const float* row_max;
  const float* log_sum;
  const float* entropy;
  const float* g_lp;
  const float* g_h;
  void* dx;
  int64_t dstride;
};

// The gradient of a row: p_v (a + b d_v), and at the token g more.
struct RowGrad {
  float m, ls2;          // maximum, log2 s
  float a, b, g;
  int t;                 // the token, or -1
};
__device__ __forceinline__ RowGrad row_grad(float m, float log_s, float H, int t, int V, float g_lp, float g_h, float inv_t) {
  RowGrad r;
  const bool token = t >= 0 && t < V;
  r.t = token ? t : -1;
  r.m = m;
  r.ls2 = log_s * kLog2E;
  const float gl = token ? g_lp : 0.f;
  r.a = -inv_t * (gl + g_h * (H - log_s));
  r.b = -inv_t * inv_t * g_h;
  r.g = inv_t * gl;
  if (m == -INFINITY) r.ls2 = r.a = r.b = 0.f, r.t = -1;      // an empty row: p = 0
  if (!(m < INFINITY)) r.a = NAN, r.t = -1;
  return r;
}
__device__ __forceinline__ float grad_one(const RowGrad& r, float x, int i, float c) {
  const float d = fmaxf(x - r.m, kFar);
  const float o = ex2(fmaf(d, c, -r.ls2)) * fmaf(r.b, d, r.a);
  return i == r.t && x > -INFINITY ? o + r.g : o;
}
// Without the token's part, which grad_one writes afterwards.
template <int kPer>
__device__ __forceinline__ void grad_vec(const RowGrad& r, const float* f, float* o, float c) {
  const f32x2 m = pair(-r.m, -r.m), c2 = pair(c, c), l = pair(-r.ls2, -r.ls2), a = pair(r.a, r.a), b = pair(r.b, r.b);
#pragma unroll
  for (int e = 0; e < kPer; e += 2) {
    const f32x2 d = far2(add2(pair(f[e], f[e + 1]), m));
    const float2 t = unpair(fma2(d, c2, l));
    const float2 y = unpair(mul2(pair(ex2(t.x), ex2(t.y)), fma2(b, d, a)));
    o[e] = y.x;
    o[e + 1] = y.y;
  }
}
// Stores a vector of results whose place need not be on a 16-byte boundary.
template <int kDtype>
__device__ __forceinline__ void put_vec(typename Num<kDtype>::T* to, const float* o, bool vec) {
  using E = Num<kDtype>;
  if (vec) {
    *reinterpret_cast<uint4*>(to) = E::pack(o);
  } else {
#pragma unroll
    for (int e = 0; e < E::kPer16; ++e) to[e] = E::from(o[e]);
  }
}
template <int kDtype>
__device__ __forceinline__ bool same_phase(const void* a, const void* b) {
  return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15) == 0;
}

// One read of the logits and one write, by parts of rows (a power of two of them, while there are fewer than
// eight CTAs an SM): 4096 x 65536 bf16 167 us, 6.4 TB/s; bound by the copy.
template <int kDtype>
__global__ void __launch_bounds__(kScoreThreads) k_scores_grad(const GradArgs A, int log_parts) {
  using E = Num<kDtype>;
  using T = typename E::T;
  constexpr int kPer = E::kPer16;
  const int64_t n = blockIdx.x >> log_parts;
  const int part = blockIdx.x & ((1 << log_parts) - 1);
  const T* row = reinterpret_cast<const T*>(A.x) + n * A.stride;
  T* out = reinterpret_cast<T*>(A.dx) + n * A.dstride;
  const Row<kDtype> R(row, A.V);
  const bool vec_out = same_phase<kDtype>(row, out);
  const RowGrad g = row_grad(A.row_max[n], A.log_sum[n], A.entropy ? A.entropy[n] : 0.f, A.tokens ? A.tokens[n] : -1, A.V,
                             A.g_lp ? A.g_lp[n] : 0.f, A.g_h ? A.g_h[n] : 0.f, A.inv_t);
  const int v0 = share(R.nvec, part, log_parts), v1 = share(R.nvec, part + 1, log_parts);
  const uint4* vec = R.vec();
  for (int v = v0 + threadIdx.x; v < v1; v += kScoreThreads) {
    float f[kPer], o[kPer];
    E::unpack(vec[v], f);
    grad_vec<kPer>(g, f, o, A.c);
    if ((unsigned)(g.t - R.head - v * kPer) < (unsigned)kPer) {
#pragma unroll
      for (int e = 0; e < kPer; ++e)
        if (g.t - R.head - v * kPer == e) o[e] = grad_one(g, f[e], g.t, A.c);
    }
    put_vec<kDtype>(out + R.head + v * kPer, o, vec_out);
  }
  if (part == 0 && threadIdx.x < R.singles()) {
    const int i = R.single(threadIdx.x);
    out[i] = E::from(grad_one(g, E::to(row[i]), i, A.c));
  }
}

struct TrainArgs {
  ScoreArgs S;
  const float* g_lp;
  const float* g_h;
  void* dx;
  int64_t dstride;
};

constexpr int kTrainThreads = 256;
constexpr int kTrainMaxVecs = 24;      // vectors of a thread: 96 KB of shared memory a CTA, two an SM

// Statistics and gradient with the row read once: a cluster takes row after row, each thread's vectors
// of a row in shared memory that it alone reads and writes.  A vector's place is filled with the
// next row's (asynchronously) as soon as its gradient is out, so that the reads never stop.  The
// statistics of all warps are exchanged in one cluster barrier a row, their places taken in turn.
// 4096 x 65536 bf16: 210 us (5.1 TB/s), where scores and gradient apart take 83 + 167; bound by issue slots,
// 65 % of them busy with 20 instructions an element (two exponentials, 11 others of arithmetic, the
// conversions and shared memory).  333 x 50001 fp32: 30 us, three rounds of rows.
template <int kDtype>
__global__ void __launch_bounds__(kTrainThreads, 4) k_scores_train(const TrainArgs A, int N) {
  using E = Num<kDtype>;
  using T = typename E::T;
  constexpr int kPer = E::kPer16, kThreads = kTrainThreads, kWarps = kThreads / 32;
  extern __shared__ __align__(16) uint4 buffer[];               // [vecs][kThreads]
  __shared__ Stat stats[2][kScoreMaxCluster * kWarps];
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), log_c = __ffs(C) - 1;
  const int tid = threadIdx.x;
  const int step = gridDim.x >> log_c;
  struct Mine {                                                  // this thread's part of a row
    const T* row;
    const uint4* vec;                                            // its first vector
    int first, have, single, t;                                  // the vector's first element, vectors
    float x, g_lp, g_h;
  };
  auto locate = [&](int64_t n) {
    Mine p;
    p.row = reinterpret_cast<const T*>(A.S.x) + n * A.S.stride;
    const Row<kDtype> R(p.row, A.S.V);
    const int v0 = share(R.nvec, rank, log_c) + tid, v1 = share(R.nvec, rank + 1, log_c);
    p.vec = R.vec() + v0;
    p.first = R.head + v0 * kPer;
    p.have = v0 < v1 ? (v1 - v0 - 1) / kThreads + 1 : 0;
    p.single = rank == 0 && tid < R.singles() ? R.single(tid) : -1;
    p.x = p.single >= 0 ? E::to(p.row[p.single]) : 0.f;
    p.t = A.S.tokens ? A.S.tokens[n] : -1;
    p.g_lp = A.g_lp ? A.g_lp[n] : 0.f;
    p.g_h = A.g_h ? A.g_h[n] : 0.f;
    return p;
  };
  uint4* mine = buffer + tid;
  const uint32_t place = smem_addr(mine);
  if (C > 1) cl.barrier_arrive();
  int64_t n = blockIdx.x >> log_c;
  Mine p = locate(n);
  for (int u = 0; u < p.have; ++u) copy16(place + u * kThreads * 16, p.vec + u * kThreads, true);
  asm volatile("cp.async.commit_group;");
  Token tok{p.t, p.t >= 0 && p.t < A.S.V ? E::to(p.row[p.t]) : 0.f};
  if (C > 1) cl.barrier_wait();
#pragma unroll 1
  for (int turn = 0;; turn ^= 1) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    Run run = run_empty();
#pragma unroll 1
    for (int u = 0; u < p.have; u += 4) {
      uint4 raw[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        raw[k] = vec_masked<kDtype>();
        if (u + k < p.have) raw[k] = mine[(u + k) * kThreads];
      }
      run_see(run, max_nan(max_nan(vec_max<kDtype>(raw[0]), vec_max<kDtype>(raw[1])),
                           max_nan(vec_max<kDtype>(raw[2]), vec_max<kDtype>(raw[3]))), A.S.c);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float f[kPer];
        E::unpack(raw[k], f);
        run_add<kPer>(run, f, A.S.c);
      }
    }
    if (p.single >= 0) run_one(run, p.x, A.S.c);
    Stat a = run_warp(run, A.S.c);
    if ((tid & 31) < C) (C > 1 ? cl.map_shared_rank(stats[turn], tid & 31) : stats[turn])[rank * kWarps + tid / 32] = a;
    const int64_t next = n + step;
    Mine q = p;
    q.have = 0;
    if (next < N) q = locate(next);
    if (C > 1) cl.sync();
    else __syncthreads();
    a = stat_gather(stats[turn], C * kWarps, tid & 31, A.S.c);
    if (rank == 0 && tid == 0) write_row(A.S, n, a, tok);
    const float log_s = logf(a.s);
    const RowGrad g = row_grad(a.m, log_s, log_s - a.w / a.s * A.S.inv_t, tok.t, A.S.V, p.g_lp, p.g_h, A.S.inv_t);
    // the next row's token, before that row's gradient can be written
    tok = Token{q.t, q.t >= 0 && q.t < A.S.V ? E::to(q.row[q.t]) : 0.f};
    T* out = reinterpret_cast<T*>(A.dx) + n * A.dstride;
    const bool vec = same_phase<kDtype>(p.row, out);
    T* to = out + p.first;
#pragma unroll 2
    for (int u = 0; u < p.have; ++u) {
      float f[kPer], o[kPer];
      E::unpack(mine[u * kThreads], f);
      grad_vec<kPer>(g, f, o, A.S.c);
      if ((unsigned)(g.t - p.first - u * kThreads * kPer) < (unsigned)kPer) {     // the token's vector
#pragma unroll
        for (int e = 0; e < kPer; ++e)
          if (g.t - p.first - u * kThreads * kPer == e) o[e] = grad_one(g, f[e], g.t, A.S.c);
      }
      put_vec<kDtype>(to + u * kThreads * kPer, o, vec);
      if (u < q.have) copy16(place + u * kThreads * 16, q.vec + u * kThreads, true);
    }
    for (int u = p.have; u < q.have; ++u) copy16(place + u * kThreads * 16, q.vec + u * kThreads, true);
    asm volatile("cp.async.commit_group;");
    if (p.single >= 0) out[p.single] = E::from(grad_one(g, p.x, p.single, A.S.c));
    if (next >= N) break;
    n = next;
    p = q;
  }
}

static int check_rows(const void* x, int64_t stride, int N, int V, int dtype, float temperature) {
  if (!token_dtype(dtype) || N < 0 || V < 1 || V > (1 << 30) || stride < V) return SDV_EINVAL;
  if (!temperature_ok(temperature) || !x) return SDV_EINVAL;
  if (!aligned_to(x, elem_bytes(dtype))) return SDV_EALIGN;
  return SDV_OK;
}

template <int kDtype>
static cudaError_t launch_scores(const ScoreArgs& A, int N, int dtype, cudaStream_t s) {
  const int C = score_cluster(N, A.V, dtype);
  const dim3 grid((unsigned)(N * (int64_t)C));
  if (A.top_k) return launch_cluster(k_scores<kDtype, true>, grid, kScoreThreads, 0, (unsigned)C, false, s, A);
  return launch_cluster(k_scores<kDtype, false>, grid, kScoreThreads, 0, (unsigned)C, false, s, A);
}

// How k_scores_train runs: CTAs per row, vectors per thread, clusters.  As many clusters as are resident
// together (a few SMs' worth less: clusters do not fill every part of the chip) take the rows in
// rounds; a CTA's row costs its vectors and about five more for what is done once a row (of
// 4096 rows of 65536 bf16, two CTAs a row: 500 of 1450 instructions a warp).  c = 0 if no cluster
// holds a row.
struct TrainShape {
  int c, vecs, clusters;
};
static TrainShape train_shape(int N, int V, int dtype) {
  const int64_t nvec = ((int64_t)V * (int64_t)elem_bytes(dtype) + 15) / 16;
  TrainShape best{0, 0, 0};
  int64_t least = INT64_MAX;
  for (int c = 1; c <= kScoreMaxCluster; c *= 2) {
    const int64_t vecs = ((nvec + c - 1) / c + kTrainThreads - 1) / kTrainThreads;
    if (vecs > kTrainMaxVecs) continue;
    const int per_sm = min_int(4, (int)(225 * 1024 / (vecs * kTrainThreads * 16 + 3 * 1024)));
    const int most = (sm_count() - 6) * per_sm / c;
    const int rounds = (N + most - 1) / most;
    const int64_t cost = (int64_t)rounds * per_sm * (vecs + 5);
    if (cost < least) {
      least = cost;
      best = TrainShape{c, (int)vecs, (N + rounds - 1) / rounds};
    }
  }
  return best;
}

template <int kDtype>
static cudaError_t launch_grad(const GradArgs& G, int N, int dtype, cudaStream_t s) {
  const int64_t nvec = (int64_t)G.V * (int64_t)elem_bytes(dtype) / 16;
  int parts = 0;                                                  // (a logarithm)
  while (parts < 6 && ((int64_t)N << parts) < 8 * sm_count() && nvec >> (parts + 1) >= kScoreThreads) ++parts;
  k_scores_grad<kDtype><<<(unsigned)((int64_t)N << parts), kScoreThreads, 0, s>>>(G, parts);
  return cudaGetLastError();
}

template <int kDtype>
static cudaError_t launch_train(const TrainArgs& A, int N, TrainShape t, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(k_scores_train<kDtype>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             kTrainMaxVecs * kTrainThreads * 16);
  if (e != cudaSuccess) return e;
  return launch_cluster(k_scores_train<kDtype>, dim3((unsigned)(t.clusters * t.c)), kTrainThreads,
                        (size_t)t.vecs * kTrainThreads * 16, (unsigned)t.c, false, s, A, N);
}

}  // namespace sdv

using namespace sdv;

extern "C" {

int sdv_token_scores(const void* logits, int64_t row_stride, int N, int V, int dtype, const int32_t* tokens,
                     float temperature, int top_k, float* logprob, float* entropy, float* row_max, float* log_sum,
                     int32_t* top_ids, float* top_logprob, uint32_t* status, sdv_stream_t stream) {
  if (N == 0) return token_dtype(dtype) && V >= 1 ? SDV_OK : SDV_EINVAL;
  int rc = check_rows(logits, row_stride, N, V, dtype, temperature);
  if (rc) return rc;
  if (N > (1 << 27) || top_k < 0 || top_k > SDV_MAX_TOP || top_k > V) return SDV_EINVAL;
  if ((tokens == nullptr) != (logprob == nullptr)) return SDV_EINVAL;
  if (top_k && (!top_ids || !top_logprob)) return SDV_EINVAL;
  if (!logprob && !entropy && !row_max && !log_sum && !top_k && !status) return SDV_EINVAL;
  const void* four[] = {tokens, logprob, entropy, row_max, log_sum, top_ids, top_logprob, status};
  for (const void* p : four)
    if (!aligned_to(p, 4)) return SDV_EALIGN;
  const ScoreArgs A{logits, row_stride, V, tokens, kLog2E / temperature, 1.f / temperature, top_k, logprob, entropy,
                    row_max, log_sum, top_ids, top_logprob, status};
  cudaStream_t s = (cudaStream_t)stream;
  return launched(dtype == SDV_F32    ? launch_scores<SDV_F32>(A, N, dtype, s)
                  : dtype == SDV_BF16 ? launch_scores<SDV_BF16>(A, N, dtype, s)
                                      : launch_scores<SDV_F16>(A, N, dtype, s));
}

int sdv_token_scores_grad(const void* logits, int64_t row_stride, int N, int V, int dtype, const int32_t* tokens,
                          float temperature, const float* row_max, const float* log_sum, const float* entropy,
                          const float* g_logprob, const float* g_entropy, void* d_logits, int64_t d_stride,
                          sdv_stream_t stream) {
  if (N == 0) return token_dtype(dtype) && V >= 1 ? SDV_OK : SDV_EINVAL;
  int rc = check_rows(logits, row_stride, N, V, dtype, temperature);
  if (rc) return rc;
  if (N > (1 << 25) || d_stride < V || !d_logits || !row_max || !log_sum) return SDV_EINVAL;
  if ((!g_logprob && !g_entropy) || (tokens == nullptr) != (g_logprob == nullptr) || (g_entropy && !entropy)) return SDV_EINVAL;
  if (!aligned_to(d_logits, elem_bytes(dtype))) return SDV_EALIGN;
  const void* four[] = {tokens, row_max, log_sum, entropy, g_logprob, g_entropy};
  for (const void* p : four)
    if (!aligned_to(p, 4)) return SDV_EALIGN;
  const GradArgs G{logits, row_stride, V, tokens, kLog2E / temperature, 1.f / temperature, row_max, log_sum, entropy,
                   g_logprob, g_entropy, d_logits, d_stride};
  cudaStream_t s = (cudaStream_t)stream;
  return launched(dtype == SDV_F32    ? launch_grad<SDV_F32>(G, N, dtype, s)
                  : dtype == SDV_BF16 ? launch_grad<SDV_BF16>(G, N, dtype, s)
                                      : launch_grad<SDV_F16>(G, N, dtype, s));
}

int sdv_token_scores_train(const void* logits, int64_t row_stride, int N, int V, int dtype, const int32_t* tokens,
                           float temperature, const float* g_logprob, const float* g_entropy, float* logprob,
                           float* entropy, float* row_max, float* log_sum, uint32_t* status, void* d_logits,
                           int64_t d_stride, sdv_stream_t stream) {
  if (N == 0) return token_dtype(dtype) && V >= 1 ? SDV_OK : SDV_EINVAL;
  int rc = check_rows(logits, row_stride, N, V, dtype, temperature);
  if (rc) return rc;
  if (N > (1 << 27) || d_stride < V || !d_logits || !entropy || !row_max || !log_sum) return SDV_EINVAL;
  if ((!g_logprob && !g_entropy) || (tokens == nullptr) != (logprob == nullptr) || (g_logprob && !tokens)) return SDV_EINVAL;
  if (!aligned_to(d_logits, elem_bytes(dtype))) return SDV_EALIGN;
  const void* four[] = {tokens, g_logprob, g_entropy, logprob, entropy, row_max, log_sum, status};
  for (const void* p : four)
    if (!aligned_to(p, 4)) return SDV_EALIGN;
  const TrainShape t = train_shape(N, V, dtype);
  if (!t.c) {                                   // rows that no cluster holds: read twice
    rc = sdv_token_scores(logits, row_stride, N, V, dtype, tokens, temperature, 0, logprob, entropy, row_max, log_sum,
                          nullptr, nullptr, status, stream);
    if (rc) return rc;
    return sdv_token_scores_grad(logits, row_stride, N, V, dtype, g_logprob ? tokens : nullptr, temperature, row_max,
                                 log_sum, entropy, g_logprob, g_entropy, d_logits, d_stride, stream);
  }
  const TrainArgs A{ScoreArgs{logits, row_stride, V, tokens, kLog2E / temperature, 1.f / temperature, 0, logprob, entropy,
                              row_max, log_sum, nullptr, nullptr, status},
                    g_logprob, g_entropy, d_logits, d_stride};
  cudaStream_t s = (cudaStream_t)stream;
  return launched(dtype == SDV_F32    ? launch_train<SDV_F32>(A, N, t, s)
                  : dtype == SDV_BF16 ? launch_train<SDV_BF16>(A, N, t, s)
                                      : launch_train<SDV_F16>(A, N, t, s));
}

}  // extern "C"
