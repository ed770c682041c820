// sdv_token_verify.cu - sample and block verification of drafted tokens, and the next token.
//
// With q_j = softmax(target row j / T), p_j = softmax(draft row j / T') and the tokens t_j:
//   ell_j = log q_j(t_j) - log p_j(t_j),  log alpha_{j+1} = min{0, log alpha_j + ell_j},
//   v_j = sum_v max{0, alpha_j q_j(v) - p_j(v)},  h_j = v_j / (v_j + 1 - alpha_j)  (j < n),
//   h_n = alpha_n; accepted = max{j : eta_j < h_j} (block), or the tokens before the first
//   eta_j >= e^ell_j (sample).  The next token has the probabilities max{0, alpha q - p} of the
// row behind the accepted tokens, normalised, or q of the last row on full accept: the index of
// the largest r_v / E_v, the E_v exponential variates (a race, which needs no cumulated sums).
//
// k_token_stats takes every row's softmax statistics, one read of the logits with all rows alike, a
// cluster of CTAs each (in small calls k_token_verify does it).  k_token_verify has a cluster of
// CTAs per chain, each with a part of every row's columns: the masses v_j that can matter and the
// race are taken from a second read of those rows, which the L2 still holds.  h_j <= alpha_j, so that a step with eta_j >= alpha_j
// fails, and one with alpha_j = 1 succeeds, without its mass.
#include "sdv_device.cuh"
#include "sdv_tokens.cuh"

namespace sdv {

constexpr int kVerThreads = 256;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kVerMaxCluster = 16;
constexpr int kLogVerSegs = 3;
constexpr int kVerSegs = kVerWarps;    // segments of a CTA's part of a row, a warp each
constexpr int kVerRows = 2 * SDV_MAX_L + 1;
constexpr uint32_t kStreamRace = 7;
constexpr int64_t kOwnBytes = 72 << 10;

static_assert(kVerSegs == 1 << kLogVerSegs, "");

struct TokenVerifyArgs {
  const void* q;
  const void* p;
  int64_t q_sb, q_sr, p_sb, p_sr;
  const int32_t* tokens;
  int L, V, mode;
  float cq, cp, iq, ip;                // log2(e) / T and 1 / T of target and draft
  const int32_t* L_eff;
  uint64_t seed;
  const float* coins;
  const float* race;
  int32_t* accepted;
  int32_t* next;
  float* ell;
  uint32_t* status;
  struct RowStat* stats;                // workspace [B, 2 L + 1]: target rows, then draft rows
  struct StepIn* steps;                 // workspace [B, L]
  int* windows;                         // workspace [B]
};

struct Best {
  float x;
  int i;
};
struct Racer {
  float r, e;
  int i;
};

// A row's softmax as e^{(x - m)/T} / s: m, log2 s and s.
struct RowStat {
  float m, l2, s;
};
__device__ __forceinline__ bool row_ok(const RowStat& r) { return r.m > -INFINITY && r.m < INFINITY; }
// log2 of the probability, with `shift` (a log2) added.
__device__ __forceinline__ float prob(const RowStat& r, float x, float c, float shift) {
  return ex2(fmaf(fmaxf(x - r.m, kFar), c, shift - r.l2));
}

// What a step needs beside its rows' statistics: its token, the token's logits and the coin.
struct StepIn {
  int t;
  float xq, xp, eta;
};
template <int kDtype>
__device__ __forceinline__ StepIn step_in(const TokenVerifyArgs& A, int b, int j) {
  using E = Num<kDtype>;
  using T = typename E::T;
  StepIn s{A.tokens[(int64_t)b * A.L + j], 0.f, 0.f, 0.f};
  if (s.t >= 0 && s.t < A.V) {
    s.xq = E::to((reinterpret_cast<const T*>(A.q) + b * A.q_sb + j * A.q_sr)[s.t]);
    s.xp = E::to((reinterpret_cast<const T*>(A.p) + b * A.p_sb + j * A.p_sr)[s.t]);
  }
  s.eta = A.coins ? A.coins[(int64_t)b * A.L + j]
                  : ((float)philox_block(A.seed, (uint32_t)b, (uint32_t)j, kStreamCoin, 0).x + 0.5f) * 0x1p-32f;
  return s;
}

// Four exponential variates: E_v of elements 4 block .. 4 block + 3 of chain b, from the seed.
static __device__ __noinline__ float4 race4(uint64_t seed, uint32_t b, uint32_t block) {
  const uint4 w = philox_block(seed, b, block, kStreamRace, 0);
  return make_float4(-log_uniform(w.x), -log_uniform(w.y), -log_uniform(w.z), -log_uniform(w.w));
}

// Calls f(first index, n, q, p) with n <= 8 (kPer) consecutive elements of two rows at a time: this
// thread's share (of `step` threads) of part `part` of 2^log_parts.  Rows in the same phase of 16 bytes
// are read as vectors, others element by element; what is before and behind the groups of kPer comes
// one at a time (n = 1, the other places masked).  The passes over the rows run from a cold instruction
// cache: two groups under way, not more (four: no gain).
template <int kDtype, typename F>
__device__ __forceinline__ void each_pair(const typename Num<kDtype>::T* q, const typename Num<kDtype>::T* p, int V, int part,
                                          int log_parts, int lane, int step, F f) {
  using E = Num<kDtype>;
  constexpr int kPer = E::kPer16, kUn = 2;
  const bool vec = ((reinterpret_cast<uintptr_t>(q) ^ reinterpret_cast<uintptr_t>(p)) & 15) == 0;
  const Row<kDtype> R(q, V);
  const int total = vec ? R.nvec : V / kPer;          // groups of kPer
  const int g0 = share(total, part, log_parts), g1 = share(total, part + 1, log_parts);
  const uint4* vq = R.vec();
  const uint4* vp = reinterpret_cast<const uint4*>(p + R.head);
  const int done = vec ? R.head + R.nvec * kPer : total * kPer, head = vec ? R.head : 0;
  // elements outside of the groups first: at most 2 kPer - 2
  if (part == 0) {
    const int rest = head + V - done;
    for (int s = lane; s < rest; s += step) {
      const int i = s < head ? s : done + s - head;
      float x[kPer], y[kPer];
      x[0] = E::to(q[i]);
      y[0] = E::to(p[i]);
#pragma unroll
      for (int e = 1; e < kPer; ++e) x[e] = y[e] = -INFINITY;
      f(i, 1, x, y);
    }
  }
#pragma unroll 1
  for (int g = g0 + lane; g - lane < g1; g += kUn * step) {
    float x[kUn][kPer], y[kUn][kPer];
    if (vec) {
      uint4 a[kUn], b[kUn];
#pragma unroll
      for (int u = 0; u < kUn; ++u) {
        a[u] = b[u] = vec_masked<kDtype>();
        if (g + u * step < g1) {
          a[u] = __ldg(vq + g + u * step);
          b[u] = __ldg(vp + g + u * step);
        }
      }
#pragma unroll
      for (int u = 0; u < kUn; ++u) {
        E::unpack(a[u], x[u]);
        E::unpack(b[u], y[u]);
      }
    } else {
#pragma unroll
      for (int u = 0; u < kUn; ++u)
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const bool in = g + u * step < g1;
          const int i = (g + u * step) * kPer + e;
          x[u][e] = in ? E::to(q[i]) : -INFINITY;
          y[u][e] = in ? E::to(p[i]) : -INFINITY;
        }
    }
#pragma unroll
    for (int u = 0; u < kUn; ++u)
      if (g + u * step < g1) f(head + (g + u * step) * kPer, kPer, x[u], y[u]);
  }
}

// Bound by the read: 272 rows of 131072 bf16 (71 MB) take 15 us, 4.7 TB/s.
// The statistics of one row a cluster (rows past a chain's window are left out), and beside them what
// the CTAs of k_token_verify's clusters must all see alike: the windows, tokens, their logits and coins.
template <int kDtype>
__global__ void __launch_bounds__(kScoreThreads, 4) k_token_stats(const TokenVerifyArgs A) {
  using T = typename Num<kDtype>::T;
  constexpr int kWarps = kScoreThreads / 32;
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), log_c = __ffs(C) - 1;
  const int n = blockIdx.x >> log_c, per = 2 * A.L + 1, b = n / per, r = n % per;
  const int window = A.L_eff ? min(A.L_eff[b], A.L) : A.L;
  __shared__ Stat stats[kScoreMaxCluster * kWarps];
  if (C > 1) cl.barrier_arrive();
  const bool first = rank == 0 && threadIdx.x == 0;
  if (first && r == 0) A.windows[b] = window;
  if (r <= A.L ? r > window : r - A.L - 1 >= window) {
    if (C > 1) {                               // with as many barriers as the other CTAs, whatever they read
      cl.barrier_wait();
      cl.sync();
    }
    return;
  }
  StepIn in{};
  if (first && r < window) in = step_in<kDtype>(A, b, r);
  const T* row = r <= A.L ? reinterpret_cast<const T*>(A.q) + b * A.q_sb + r * A.q_sr
                          : reinterpret_cast<const T*>(A.p) + b * A.p_sb + (r - A.L - 1) * A.p_sr;
  const float c = r <= A.L ? A.cq : A.cp;
  const Part<kDtype, false> P(Row<kDtype>(row, A.V), rank, log_c);
  const Stat a = run_warp(P.read(c), c);
  if (C > 1) cl.barrier_wait();
  if ((threadIdx.x & 31) == 0) (C > 1 ? cl.map_shared_rank(stats, 0) : stats)[rank * kWarps + threadIdx.x / 32] = Stat{a.m, a.s, 0.f};
  if (C > 1) cl.sync();
  else __syncthreads();
  if (rank || threadIdx.x >= 32) return;
  const Stat all = stat_gather(stats, C * kWarps, threadIdx.x, c);
  if (threadIdx.x == 0) {
    A.stats[n] = RowStat{all.m, log2f(all.s), all.s};
    if (r < window) A.steps[(int64_t)b * A.L + r] = in;
  }
}

// kOwn: the cluster takes its chain's statistics itself (see own_stats), a warp a row's part.
// A chain of dependent phases, bound by their latency: 16 chains of 8 steps, V = 131072 bf16, 18 us in block mode
// (masses of the steps that may succeed, a warp a segment of a row, 8 of them; then the race), 12 in sample mode; one chain
// of 4 steps, V = 32768, with its statistics 11 us.  Three CTAs an SM: with four (64 registers) spills cost 2 to 4 %,
// with two 48 chains wait for places (26 us become 33).
// The CTAs of a cluster decide alike, and so meet at the same barriers: what they decide on comes from one
// place, k_token_stats' workspace or the first CTA, even if the caller's arrays change meanwhile.
template <int kDtype, bool kOwn>
__global__ void __launch_bounds__(kVerThreads, 3) k_token_verify(const TokenVerifyArgs A) {
  using E = Num<kDtype>;
  using T = typename E::T;
  constexpr int kPer = E::kPer16;
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), log_c = __ffs(C) - 1;
  const int b = blockIdx.x >> log_c, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int L = A.L, V = A.V;
  __shared__ RowStat rs[kVerRows];
  __shared__ StepIn in[SDV_MAX_L];
  __shared__ float mass_seg[SDV_MAX_L * kVerSegs];
  __shared__ float mass_part[kVerMaxCluster * SDV_MAX_L];
  __shared__ float la[SDV_MAX_L + 1], ell_s[SDV_MAX_L];
  __shared__ int need[SDV_MAX_L];
  __shared__ int n_need, acc_s, window_s;
  __shared__ uint32_t status_s;
  __shared__ Best best_w[kVerWarps];
  __shared__ Best best_c[2][kVerMaxCluster];
  static_assert(SDV_MAX_L <= kVerThreads, "a thread per step");
  if (C > 1) cl.barrier_arrive();
  if (tid == 0) status_s = 0;
  const T* q0 = reinterpret_cast<const T*>(A.q) + b * A.q_sb;
  const T* p0 = reinterpret_cast<const T*>(A.p) + b * A.p_sb;
  if (A.race) {
    const float* race = A.race + (int64_t)b * V;
    for (int i = share(V, rank, log_c) + tid * 32; i < share(V, rank + 1, log_c); i += kVerThreads * 32)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(race + i));
  }
  int n_in;                                                  // the chain's window
  if constexpr (kOwn) {
    __shared__ Stat own[kVerRows], all[kVerRows * kVerMaxCluster];
    const int window = A.L_eff ? A.L_eff[b] : L, nw = max(min(window, L), 0);
    const bool sends = rank == 0 && tid < nw;
    StepIn mine{};
    if (sends) mine = step_in<kDtype>(A, b, tid);
    auto log_segs = [](int rows) { return rows >= kVerWarps ? 0 : rows >= kVerWarps / 2 ? 1 : 2; };   // few rows: parts of them
    int log_seg = log_segs(2 * nw + 1);
    for (int u = warp; u < (2 * nw + 1) << log_seg; u += kVerWarps) {
      const int r = u >> log_seg;
      const float c = r <= nw ? A.cq : A.cp;
      const Part<kDtype, false, 32> P(Row<kDtype>(r <= nw ? q0 + r * A.q_sr : p0 + (r - nw - 1) * A.p_sr, V),
                                      (rank << log_seg) + (u & ((1 << log_seg) - 1)), log_c + log_seg);
      const Stat a = run_warp(P.read(c), c);
      if (lane == 0) own[u] = Stat{a.m, a.s, 0.f};
    }
    __syncthreads();
    if (C > 1) cl.barrier_wait();                            // every CTA of the cluster has started
    for (int i = tid; i < (2 * nw + 1) << (log_seg + log_c); i += kVerThreads) {
      const int u = i >> log_c, k = i & (C - 1);
      (C > 1 ? cl.map_shared_rank(all, k) : all)[(u << log_c) + rank] = own[u];
    }
    for (int k = 0; k < C; ++k) {
      if (sends) (C > 1 ? cl.map_shared_rank(in, k) : in)[tid] = mine;
      if (rank == 0 && tid == 0) *(C > 1 ? cl.map_shared_rank(&window_s, k) : &window_s) = window;
    }
    if (C > 1) cl.sync();
    else __syncthreads();
    n_in = window_s;
    const int n = max(min(n_in, L), 0);
    log_seg = log_segs(2 * n + 1);
    for (int r = warp; r < 2 * n + 1; r += kVerWarps) {
      const Stat a = stat_gather(all + (r << (log_seg + log_c)), 1 << (log_seg + log_c), lane, r <= n ? A.cq : A.cp);
      if (lane == 0) rs[r] = RowStat{a.m, log2f(a.s), a.s};
    }
  } else {
    asm volatile("griddepcontrol.wait;" ::: "memory");       // the rows' statistics are there
    n_in = A.windows[b];
    const int n = max(min(n_in, L), 0);
    for (int r = tid; r < 2 * n + 1; r += kVerThreads) rs[r] = A.stats[(int64_t)b * (2 * L + 1) + (r <= n ? r : L + r - n)];
    if (tid < n) in[tid] = A.steps[(int64_t)b * L + tid];
    if (C > 1) cl.barrier_wait();
  }
  if (n_in < 0) {                                            // an inactive chain
    if (rank == 0) {
      if (tid == 0) {
        A.accepted[b] = 0;
        A.next[b] = -1;
        if (A.status) A.status[b] = 0;
      }
      if (A.ell)
        for (int j = tid; j < L; j += kVerThreads) A.ell[(int64_t)b * L + j] = 0.f;
    }
    return;
  }
  const int n = min(n_in, L), rows = 2 * n + 1;
  __syncthreads();
  for (int r = tid; r < rows; r += kVerThreads) {
    uint32_t st = 0;
    if (!(rs[r].m < INFINITY)) st |= SDV_STATUS_NONFINITE;
    if (rs[r].m == -INFINITY) st |= SDV_STATUS_EMPTY_ROW;
    if (st) atomicOr(&status_s, st);
  }
  // log ratios
  if (tid < n) {
    const int j = tid, t = in[j].t;
    float ell = NAN;
    if (t >= 0 && t < V) {
      const RowStat rq = rs[j], rp = rs[n + 1 + j];
      const float xq = in[j].xq, xp = in[j].xp;
      if (rq.m < INFINITY && rp.m < INFINITY) {
        // The sums' logarithms are large and nearly equal: that of their ratio, near 0, costs no bits.  (Divisions rounded
        // to the last bit, here and by the temperatures, took 0.4 us of one chain's 11.6: this runs from a cold cache.)
        const float dq = row_ok(rq) ? (xq - rq.m) * A.iq : -INFINITY, dp = row_ok(rp) ? (xp - rp.m) * A.ip : -INFINITY;
        ell = !(dq > -INFINITY) ? -INFINITY : dp > -INFINITY ? (dq - dp) + logf(__fdividef(rp.s, rq.s)) : INFINITY;
      }
    } else {
      atomicOr(&status_s, SDV_STATUS_BAD_TOKEN);
    }
    ell_s[j] = ell;
  }
  __syncthreads();
  if (tid == 0) {                                             // the recursion, which is sequential
    float run = 0.f;
    la[0] = 0.f;
    for (int j = 0; j < n; ++j) {
      const float next = run + ell_s[j];
      run = next == next ? fminf(0.f, next) : -INFINITY;      // NaN: a step without a ratio, or -inf + inf
      la[j + 1] = A.mode == SDV_MODE_SAMPLE ? 0.f : run;
    }
  }
  __syncthreads();
  if (warp == 0) {                                            // and what each step's coin says, a lane a step
    uint64_t sure = 0, open = 0;                              // steps that succeed, steps whose mass decides
    for (int j0 = 0; j0 < n; j0 += 32) {
      const int j = j0 + lane;
      bool hit = false, may = false;
      if (j < n) {
        if (A.mode == SDV_MODE_SAMPLE) {
          hit = ell_s[j] >= 0.f || in[j].eta < expf(ell_s[j]);
        } else {
          const bool below = in[j].eta < expf(la[j + 1]);
          hit = la[j + 1] == 0.f || (j == n - 1 && below);
          may = !hit && j < n - 1 && below;
        }
      }
      sure |= (uint64_t)__ballot_sync(0xffffffffu, hit) << j0;
      open |= (uint64_t)__ballot_sync(0xffffffffu, may) << j0;
    }
    int acc;
    if (A.mode == SDV_MODE_SAMPLE) acc = sure == ~0ull ? n : min(n, __ffsll((long long)~sure) - 1);
    else acc = 64 - __clzll((long long)sure);                 // the last success so far; steps before it cannot matter
    const uint64_t rest = acc >= 64 ? 0 : open >> acc << acc;
    if (A.mode == SDV_MODE_BLOCK)
      for (int j0 = 0; j0 < n; j0 += 32) {
        const int j = j0 + lane;
        if (j < n && (rest >> j & 1)) need[__popcll((unsigned long long)(rest & ((1ull << j) - 1)))] = j + 1;
      }
    if (lane == 0) {
      acc_s = acc;
      n_need = A.mode == SDV_MODE_BLOCK ? __popcll((unsigned long long)rest) : 0;
    }
  }
  __syncthreads();
  int acc = acc_s;
  const int nn = n_need;
  if (nn) {                                                  // masses of the steps that may succeed
    for (int u = warp; u < nn * kVerSegs; u += kVerWarps) {
      const int j = need[u / kVerSegs];
      const RowStat rq = rs[j], rp = rs[n + 1 + j];
      const float sh = la[j] * kLog2E;
      float sum = 0.f;
      const bool has_p = row_ok(rp);
      each_pair<kDtype>(q0 + j * A.q_sr, has_p ? p0 + j * A.p_sr : q0 + j * A.q_sr, V, rank * kVerSegs + u % kVerSegs, log_c + kLogVerSegs, lane, 32,
                        [&](int, int, const float* x, const float* y) {
#pragma unroll
                          for (int e = 0; e < kPer; ++e)
                            sum += fmaxf(prob(rq, x[e], A.cq, sh) - (has_p ? prob(rp, y[e], A.cp, 0.f) : 0.f), 0.f);
                        });
#pragma unroll
      for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) mass_seg[u] = row_ok(rq) ? sum : NAN;
    }
    __syncthreads();
    for (int i = tid; i < nn; i += kVerThreads) {
      float s = 0.f;
      for (int k = 0; k < kVerSegs; ++k) s += mass_seg[i * kVerSegs + k];
      for (int k = 0; k < C; ++k) {
        float* to = C > 1 ? cl.map_shared_rank(mass_part, k) : mass_part;
        to[rank * SDV_MAX_L + i] = s;
      }
    }
    if (C > 1) cl.sync();
    else __syncthreads();
    for (int i = nn - 1; i >= 0; --i) {
      const int j = need[i];
      float s = 0.f;
      for (int k = 0; k < C; ++k) s += mass_part[k * SDV_MAX_L + i];
      const float h = s / (s + 1.f - expf(la[j]));
      if (in[j - 1].eta < h) {
        acc = max(acc, j);
        break;
      }
    }
  }
  // the next token
  const RowStat rq = rs[acc], rp = acc < n ? rs[n + 1 + acc] : RowStat{-INFINITY, 0.f, 1.f};
  const float sh = la[acc] * kLog2E;
  const T* q = q0 + acc * A.q_sr;
  Best best{0.f, -1};
  uint32_t zero = 0;
  for (int attempt = 0; attempt < 2; ++attempt) {
    const bool rest = attempt == 0 && acc < n && row_ok(rp);
    const T* p = rest ? p0 + acc * A.p_sr : q;
    Racer top{0.f, 1.f, 0x7fffffff};
    const float* race = A.race ? A.race + (int64_t)b * V : nullptr;
    if (row_ok(rq))
      each_pair<kDtype>(q, p, V, rank, log_c, tid, kVerThreads, [&](int i, int count, const float* x, const float* y) {
        float r[kPer], e[kPer];
        bool any = false;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          r[k] = prob(rq, x[k], A.cq, rest ? sh : 0.f) - (rest ? prob(rp, y[k], A.cp, 0.f) : 0.f);
          any |= r[k] > 0.f;
        }
        if (!any) return;
        if (race && count == kPer && aligned16(race + i)) {
#pragma unroll
          for (int k = 0; k < kPer; k += 4) *reinterpret_cast<float4*>(e + k) = __ldg(reinterpret_cast<const float4*>(race + i + k));
        } else if (race) {
#pragma unroll
          for (int k = 0; k < kPer; ++k) e[k] = k < count ? __ldg(race + i + k) : 1.f;
        } else {
          float4 four = race4(A.seed, (uint32_t)b, (uint32_t)i >> 2);
#pragma unroll
          for (int k = 0; k < kPer; ++k) {
            if (k && ((i + k) & 3) == 0) four = race4(A.seed, (uint32_t)b, (uint32_t)(i + k) >> 2);
            const int w = (i + k) & 3;
            e[k] = w == 0 ? four.x : w == 1 ? four.y : w == 2 ? four.z : four.w;
          }
        }
#pragma unroll
        for (int k = 0; k < kPer; ++k) {                            // r / e against the best so far
          const float mine = r[k] * top.e, theirs = top.r * e[k];
          if (mine > theirs || (mine == theirs && r[k] > 0.f && i + k < top.i)) top = Racer{r[k], e[k], i + k};
        }
      });
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
      Best* to = C > 1 ? cl.map_shared_rank(best_c[attempt], tid) : best_c[attempt];
      to[rank] = me;
    }
    if (C > 1) cl.sync();
    else __syncthreads();
    me = best_c[attempt][0];
    for (int k = 1; k < C; ++k)
      if (before(best_c[attempt][k].x, best_c[attempt][k].i, me.x, me.i)) me = best_c[attempt][k];
    if (me.x > 0.f) {
      best = me;
      break;
    }
    if (!rest) break;
    zero = SDV_STATUS_ZERO_DELTA;                            // no mass is left: the target's own
  }
  if (rank == 0) {
    if (tid == 0) {
      A.accepted[b] = acc;
      A.next[b] = best.i;
      if (A.status) A.status[b] = status_s | zero;
    }
    if (A.ell)
      for (int j = tid; j < L; j += kVerThreads) A.ell[(int64_t)b * L + j] = j < n ? ell_s[j] : 0.f;
  }
}

// CTAs per chain: as many as fit beside the other chains' (three an SM), as long as each thread has a vector
// of a row.  With half as many 16 x 8 x 131072 bf16 take 35 us in place of 33 and 48 x 7 x 50001 fp32 29 in
// place of 26; with twice as many, more than are resident together, the latter 37.
static int verify_cluster(int B, int V, int dtype) {
  const int64_t nvec = (int64_t)V * (int64_t)elem_bytes(dtype) / 16;
  int c = 1;
  while (c < kVerMaxCluster && (int64_t)B * 2 * c <= 3 * sm_count() && nvec >= 2 * c * kVerThreads) c *= 2;
  return c;
}

// Whether k_token_verify takes the statistics itself: where a CTA's parts of the rows are small.  Calls one
// after another, two kernels and one (bf16): 1 chain of 4 steps, V = 32768 (37 KB a CTA), 24.6 us
// and 20.7; 16 of 1, V = 131072 (49 KB), 24.9 and 20.9; 16 of 8, V = 32768 (70 KB), 24.5 and 23.0; 128
// of 8, V = 4096 (70 KB), 27.2 and 20.3; 48 of 8, V = 32768 (139 KB), 25.5 and 27.2.
static bool own_stats(int B, int L, int V, int dtype, int C) {
  return (int64_t)(2 * L + 1) * V * (int64_t)elem_bytes(dtype) / C <= kOwnBytes;
}

template <int kDtype>
static cudaError_t launch_token_verify(const TokenVerifyArgs& A, int B, int dtype, cudaStream_t s) {
  const int C = verify_cluster(B, A.V, dtype);
  const bool own = own_stats(B, A.L, A.V, dtype, C);
  const auto verify = own ? k_token_verify<kDtype, true> : k_token_verify<kDtype, false>;
  if (C > 8) {
    const cudaError_t e = cudaFuncSetAttribute(verify, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  if (own) return launch_cluster(verify, dim3((unsigned)B * (unsigned)C), kVerThreads, 0, (unsigned)C, false, s, A);
  const int rows = B * (2 * A.L + 1), Cs = score_cluster(rows, A.V, dtype);
  const cudaError_t e = launch_cluster(k_token_stats<kDtype>, dim3((unsigned)rows * (unsigned)Cs), kScoreThreads, 0, (unsigned)Cs, false, s, A);
  if (e != cudaSuccess) return e;
  return launch_cluster(verify, dim3((unsigned)B * (unsigned)C), kVerThreads, 0, (unsigned)C, true, s, A);
}

}  // namespace sdv

using namespace sdv;

extern "C" {

size_t sdv_token_verify_workspace_bytes(int B, int L) {
  if (B < 1 || B > (1 << 20) || L < 1 || L > SDV_MAX_L) return 0;
  return ((size_t)B * ((2 * L + 1) * sizeof(RowStat) + L * sizeof(StepIn) + sizeof(int)) + 255) / 256 * 256;
}

int sdv_token_verify(const void* target, int64_t target_stride_b, int64_t target_stride_row, const void* draft,
                     int64_t draft_stride_b, int64_t draft_stride_row, const int32_t* tokens, int B, int L, int V, int dtype,
                     float temperature, float draft_temperature, int mode, const int32_t* L_eff, uint64_t seed,
                     const float* coins, const float* race, int32_t* accepted_len, int32_t* next_token,
                     float* log_ratio_out, uint32_t* status_out, void* workspace, size_t workspace_bytes,
                     sdv_stream_t stream) {
  if (B < 1 || B > (1 << 20) || L < 1 || L > SDV_MAX_L || V < 1 || V > (1 << 30) || !token_dtype(dtype)) return SDV_EINVAL;
  if (mode != SDV_MODE_SAMPLE && mode != SDV_MODE_BLOCK) return SDV_EINVAL;
  if (!temperature_ok(temperature) || !temperature_ok(draft_temperature)) return SDV_EINVAL;
  if (!target || !draft || !tokens || !accepted_len || !next_token) return SDV_EINVAL;
  if (target_stride_row < V || draft_stride_row < V || target_stride_b < 0 || draft_stride_b < 0) return SDV_EINVAL;
  if (!aligned_to(target, elem_bytes(dtype)) || !aligned_to(draft, elem_bytes(dtype))) return SDV_EALIGN;
  const void* four[] = {tokens, L_eff, coins, race, accepted_len, next_token, log_ratio_out, status_out};
  for (const void* p : four)
    if (!aligned_to(p, 4)) return SDV_EALIGN;
  if (!workspace || workspace_bytes < sdv_token_verify_workspace_bytes(B, L)) return SDV_ENOWORKSPACE;
  if (!aligned_to(workspace, 256)) return SDV_EALIGN;
  const TokenVerifyArgs A{target, draft, target_stride_b, target_stride_row, draft_stride_b, draft_stride_row, tokens, L, V,
                          mode, kLog2E / temperature, kLog2E / draft_temperature, 1.f / temperature,
                          1.f / draft_temperature, L_eff, seed, coins, race, accepted_len, next_token, log_ratio_out, status_out,
                          (RowStat*)workspace, (StepIn*)((RowStat*)workspace + (size_t)B * (2 * L + 1)),
                          (int*)((StepIn*)((RowStat*)workspace + (size_t)B * (2 * L + 1)) + (size_t)B * L)};
  cudaStream_t s = (cudaStream_t)stream;
  return launched(dtype == SDV_F32    ? launch_token_verify<SDV_F32>(A, B, dtype, s)
                  : dtype == SDV_BF16 ? launch_token_verify<SDV_BF16>(A, B, dtype, s)
                                      : launch_token_verify<SDV_F16>(A, B, dtype, s));
}

}  // extern "C"
