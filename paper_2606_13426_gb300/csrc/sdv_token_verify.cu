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
// One cluster of CTAs per chain; each CTA has a part of every row's columns.  The statistics of
// all rows come first (one read of the logits), are joined through distributed shared memory,
// and the masses v_j that can matter and the race are taken from a second read of those rows,
// which the L2 still holds.  h_j <= alpha_j, so that a step with eta_j >= alpha_j fails, and one
// with alpha_j = 1 succeeds, without its mass.
#include "sdv_device.cuh"
#include "sdv_tokens.cuh"

namespace sdv {

constexpr int kVerThreads = 512;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kVerMaxCluster = 8;
constexpr int kVerSegs = 8;            // segments of a CTA's part of a row, a warp each
constexpr int kBatch = 8;
constexpr int kVerRows = 2 * SDV_MAX_L + 1;
constexpr uint32_t kStreamRace = 7;

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
};

struct Best {
  float x;
  int i;
};
struct Racer {
  float r, e;
  int i;
};

// A row's softmax as e^{(x - m)/T} / s: m and log2 s.  mass: 1, or 0 for a row that has none.
struct RowStat {
  float m, l2;
};
__device__ __forceinline__ bool row_ok(const RowStat& r) { return r.m > -INFINITY && r.m < INFINITY; }
// log2 of the probability, with `shift` (a log2) added.
__device__ __forceinline__ float prob(const RowStat& r, float x, float c, float shift) {
  return ex2(fmaf(fmaxf(x - r.m, kFar), c, shift - r.l2));
}

// Calls f(index, q, p) for this thread's share (of `step` threads) of elements [.., ..) of two rows;
// part `part` of `parts`.  Rows in the same phase of 16 bytes are read as vectors.
template <int kDtype, typename F>
__device__ __forceinline__ void each_pair(const typename Num<kDtype>::T* q, const typename Num<kDtype>::T* p, int V, int part,
                                          int parts, int lane, int step, F f) {
  using E = Num<kDtype>;
  constexpr int kPer = E::kPer16;
  if (((reinterpret_cast<uintptr_t>(q) ^ reinterpret_cast<uintptr_t>(p)) & 15) == 0) {
    const Row<kDtype> R(q, V);
    const uint4* vq = R.vec();
    const uint4* vp = reinterpret_cast<const uint4*>(p + R.head);
    const int v0 = (int)((int64_t)R.nvec * part / parts), v1 = (int)((int64_t)R.nvec * (part + 1) / parts);
    int v = v0 + lane;
    for (; v + 3 * step < v1; v += 4 * step) {
      uint4 a[4], b[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        a[u] = __ldg(vq + v + u * step);
        b[u] = __ldg(vp + v + u * step);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float x[kPer], y[kPer];
        E::unpack(a[u], x);
        E::unpack(b[u], y);
#pragma unroll
        for (int e = 0; e < kPer; ++e) f(R.head + (v + u * step) * kPer + e, x[e], y[e]);
      }
    }
    for (; v < v1; v += step) {
      float x[kPer], y[kPer];
      E::unpack(__ldg(vq + v), x);
      E::unpack(__ldg(vp + v), y);
#pragma unroll
      for (int e = 0; e < kPer; ++e) f(R.head + v * kPer + e, x[e], y[e]);
    }
    if (part == 0)
      for (int s = lane; s < R.singles(); s += step) f(R.single(s), E::to(q[R.single(s)]), E::to(p[R.single(s)]));
  } else {
    const int e0 = (int)((int64_t)V * part / parts), e1 = (int)((int64_t)V * (part + 1) / parts);
    int e = e0 + lane;
    for (; e + 7 * step < e1; e += 8 * step) {
      float x[8], y[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        x[u] = E::to(q[e + u * step]);
        y[u] = E::to(p[e + u * step]);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) f(e + u * step, x[u], y[u]);
    }
    for (; e < e1; e += step) f(e, E::to(q[e]), E::to(p[e]));
  }
}

// Calls f(index, q, p, race) for this thread's share of part `part` of `parts` of the rows.
template <int kDtype, typename F>
__device__ __forceinline__ void each_race(const typename Num<kDtype>::T* q, const typename Num<kDtype>::T* p, const float* race,
                                          int V, int part, int parts, int tid, F f) {
  using E = Num<kDtype>;
  constexpr int kPer = E::kPer16, kUn = kPer == 8 ? 2 : 4;
  const Row<kDtype> R(q, V);
  const bool whole = ((reinterpret_cast<uintptr_t>(q) ^ reinterpret_cast<uintptr_t>(p)) & 15) == 0 && aligned16(race + R.head);
  if (whole) {
    const uint4* vq = R.vec();
    const uint4* vp = reinterpret_cast<const uint4*>(p + R.head);
    const float4* vr = reinterpret_cast<const float4*>(race + R.head);
    const int v0 = (int)((int64_t)R.nvec * part / parts), v1 = (int)((int64_t)R.nvec * (part + 1) / parts);
    for (int v = v0 + tid; v < v1; v += kUn * kVerThreads) {
      uint4 a[kUn], b[kUn];
      float4 e[kUn * kPer / 4];
#pragma unroll
      for (int u = 0; u < kUn; ++u) {
        const int w = v + u * kVerThreads;
        if (w < v1) {
          a[u] = __ldg(vq + w);
          b[u] = __ldg(vp + w);
#pragma unroll
          for (int k = 0; k < kPer / 4; ++k) e[u * (kPer / 4) + k] = __ldg(vr + (int64_t)w * (kPer / 4) + k);
        }
      }
#pragma unroll
      for (int u = 0; u < kUn; ++u) {
        const int w = v + u * kVerThreads;
        if (w < v1) {
          float x[kPer], y[kPer];
          E::unpack(a[u], x);
          E::unpack(b[u], y);
#pragma unroll
          for (int k = 0; k < kPer; ++k) {
            const float4 ev = e[u * (kPer / 4) + k / 4];
            f(R.head + w * kPer + k, x[k], y[k], k % 4 == 0 ? ev.x : k % 4 == 1 ? ev.y : k % 4 == 2 ? ev.z : ev.w);
          }
        }
      }
    }
    if (part == 0 && tid < R.singles()) {
      const int i = R.single(tid);
      f(i, E::to(q[i]), E::to(p[i]), race[i]);
    }
  } else {
    const int e0 = (int)((int64_t)V * part / parts), e1 = (int)((int64_t)V * (part + 1) / parts);
    for (int e = e0 + tid; e < e1; e += 8 * kVerThreads) {
      float x[8], y[8], z[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = e + u * kVerThreads;
        if (i < e1) {
          x[u] = E::to(q[i]);
          y[u] = E::to(p[i]);
          z[u] = race[i];
        }
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (e + u * kVerThreads < e1) f(e + u * kVerThreads, x[u], y[u], z[u]);
    }
  }
}

template <int kDtype>
__global__ void __launch_bounds__(kVerThreads) k_token_verify(const TokenVerifyArgs A) {
  using E = Num<kDtype>;
  using T = typename E::T;
  constexpr int kPer = E::kPer16;
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int b = blockIdx.x / C, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int L = A.L, V = A.V;
  const int n_in = A.L_eff ? A.L_eff[b] : L;
  if (n_in < 0) {                                  // an inactive chain
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
  const int n = min(n_in, L);
  const int rows = 2 * n + 1;
  __shared__ RowStat seg[kVerRows * kVerSegs];              // a CTA's segments of a row: m and s
  __shared__ RowStat part_s[kVerMaxCluster * kVerRows];      // the CTAs' parts
  __shared__ RowStat rs[kVerRows];
  __shared__ float mass_seg[SDV_MAX_L * kVerSegs];
  __shared__ float mass_part[kVerMaxCluster * SDV_MAX_L];
  __shared__ float la[SDV_MAX_L + 1], ell_s[SDV_MAX_L], eta[SDV_MAX_L];
  __shared__ int need[SDV_MAX_L];
  __shared__ int n_need, acc_s;
  __shared__ uint32_t status_s;
  __shared__ Best best_w[kVerWarps];
  __shared__ Best best_c[2][kVerMaxCluster];
  if (C > 1) cl.barrier_arrive();
  if (tid == 0) status_s = 0;
  const T* q0 = reinterpret_cast<const T*>(A.q) + b * A.q_sb;
  const T* p0 = reinterpret_cast<const T*>(A.p) + b * A.p_sb;
  auto row_of = [&](int r) { return r <= n ? q0 + r * A.q_sr : p0 + (r - n - 1) * A.p_sr; };
  // statistics: target rows 0 .. n, then draft rows 0 .. n - 1, a warp per segment of a row; the
  // next kBatch vectors of each lane are under way while it works on the last ones
  const int parts = C * kVerSegs;
  {
    struct At {
      int u, v, v1;                                            // unit, this lane's vector, the unit's end
    };
    auto unit = [&](int u) {
      At a{u, 0, 0};
      if (u < rows * kVerSegs) {
        const Row<kDtype> R(row_of(u / kVerSegs), V);
        const int sg = rank * kVerSegs + u % kVerSegs;
        a.v = (int)((int64_t)R.nvec * sg / parts) + lane;
        a.v1 = (int)((int64_t)R.nvec * (sg + 1) / parts);
      }
      return a;
    };
    auto load = [&](const At& a, uint4* raw) {
      if (a.u >= rows * kVerSegs) return;
      const uint4* vec = Row<kDtype>(row_of(a.u / kVerSegs), V).vec() + a.v;
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (a.v + 32 * k < a.v1) raw[k] = __ldg(vec + 32 * k);
    };
    uint4 raw[kBatch], ahead[kBatch];
    At at = unit(warp);
    load(at, raw);
    Run run = run_empty();
    while (at.u < rows * kVerSegs) {
      const int r = at.u / kVerSegs;
      const float c = r <= n ? A.cq : A.cp;
      At next = at;
      next.v += 32 * kBatch;
      const bool last = next.v - lane >= at.v1;
      if (last) next = unit(at.u + kVerWarps);
      load(next, ahead);
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (at.v + 32 * k < at.v1) {
          float f[kPer];
          run_see(run, vec_max<kDtype>(raw[k]), c);
          E::unpack(raw[k], f);
          run_add<kPer>(run, f, c);
        }
      if (last) {
        if (rank == 0 && at.u % kVerSegs == 0) {
          const T* row = row_of(r);
          const Row<kDtype> R(row, V);
          if (lane < R.singles()) run_one(run, E::to(row[R.single(lane)]), c);
        }
        const Stat a = run_warp(run, c);
        if (lane == 0) seg[at.u] = RowStat{a.m, a.s};
        run = run_empty();
      }
      at = next;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) raw[k] = ahead[k];
    }
  }
  __syncthreads();
  if (C > 1) cl.barrier_wait();
  auto join = [&](const RowStat* from, int count, int stride, float c) {
    Stat a{from[0].m, from[0].l2, 0.f};
    for (int i = 1; i < count; ++i) a = stat_join(a, Stat{from[i * stride].m, from[i * stride].l2, 0.f}, c);
    return a;
  };
  for (int r = tid; r < rows; r += kVerThreads) {
    const Stat a = join(seg + r * kVerSegs, kVerSegs, 1, r <= n ? A.cq : A.cp);
    for (int k = 0; k < C; ++k) {
      RowStat* to = C > 1 ? cl.map_shared_rank(part_s, k) : part_s;
      to[rank * kVerRows + r] = RowStat{a.m, a.s};
    }
  }
  if (C > 1) cl.sync();
  else __syncthreads();
  for (int r = tid; r < rows; r += kVerThreads) {
    const Stat a = join(part_s + r, C, kVerRows, r <= n ? A.cq : A.cp);
    rs[r] = RowStat{a.m, log2f(a.s)};
    uint32_t st = 0;
    if (!(a.m < INFINITY)) st |= SDV_STATUS_NONFINITE;
    if (a.m == -INFINITY) st |= SDV_STATUS_EMPTY_ROW;
    if (st) atomicOr(&status_s, st);
  }
  __syncthreads();
  // log ratios and coins
  for (int j = tid; j < n; j += kVerThreads) {
    const int t = A.tokens[(int64_t)b * L + j];
    float ell = NAN;
    if (t >= 0 && t < V) {
      const RowStat rq = rs[j], rp = rs[n + 1 + j];
      const float xq = E::to(q0[j * A.q_sr + t]), xp = E::to(p0[j * A.p_sr + t]);
      if (rq.m < INFINITY && rp.m < INFINITY) {
        const float lq = row_ok(rq) && xq > -INFINITY ? (xq - rq.m) * A.iq - rq.l2 * kLn2f : -INFINITY;
        const float lp = row_ok(rp) && xp > -INFINITY ? (xp - rp.m) * A.ip - rp.l2 * kLn2f : -INFINITY;
        ell = lq > -INFINITY ? lq - lp : -INFINITY;
      }
    } else {
      atomicOr(&status_s, SDV_STATUS_BAD_TOKEN);
    }
    ell_s[j] = ell;
    eta[j] = A.coins ? A.coins[(int64_t)b * L + j]
                     : ((float)philox_block(A.seed, (uint32_t)b, (uint32_t)j, kStreamCoin, 0).x + 0.5f) * 0x1p-32f;
  }
  __syncthreads();
  if (tid == 0) {
    int acc = 0, m = 0;
    la[0] = 0.f;
    if (A.mode == SDV_MODE_SAMPLE) {
      while (acc < n && (ell_s[acc] >= 0.f || eta[acc] < expf(ell_s[acc]))) ++acc;
      for (int j = 0; j < n; ++j) la[j + 1] = 0.f;
    } else {
      float run = 0.f;
      for (int j = 0; j < n; ++j) {
        const float e = ell_s[j];
        run = e == e ? fminf(0.f, run + e) : -INFINITY;
        if (!(run == run)) run = -INFINITY;                 // -inf + inf
        la[j + 1] = run;
        const float alpha = expf(run);
        if (run == 0.f || (j == n - 1 && eta[j] < alpha)) {
          acc = j + 1;
          m = 0;                                            // what is below cannot matter any more
        } else if (j < n - 1 && eta[j] < alpha) {
          need[m++] = j + 1;
        }
      }
    }
    acc_s = acc;
    n_need = m;
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
      each_pair<kDtype>(q0 + j * A.q_sr, p0 + j * A.p_sr, V, rank * kVerSegs + u % kVerSegs, parts, lane, 32,
                        [&](int, float x, float y) {
                          const float d = prob(rq, x, A.cq, sh) - (has_p ? prob(rp, y, A.cp, 0.f) : 0.f);
                          sum += fmaxf(d, 0.f);
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
      if (eta[j - 1] < h) {
        acc = max(acc, j);
        break;
      }
    }
  }
  // the next token
  const RowStat rq = rs[acc], rp = acc < n ? rs[n + 1 + acc] : RowStat{-INFINITY, 0.f};
  const float sh = la[acc] * kLog2E;
  const T* q = q0 + acc * A.q_sr;
  Best best{0.f, -1};
  uint32_t zero = 0;
  for (int attempt = 0; attempt < 2; ++attempt) {
    const bool rest = attempt == 0 && acc < n && row_ok(rp);
    const T* p = rest ? p0 + acc * A.p_sr : q;
    Racer top{0.f, 1.f, 0x7fffffff};
    if (row_ok(rq)) {
      if (A.race) {
        const float* race = A.race + (int64_t)b * V;
        each_race<kDtype>(q, p, race, V, rank, C, tid, [&](int i, float x, float y, float e) {
          const float r = prob(rq, x, A.cq, rest ? sh : 0.f) - (rest ? prob(rp, y, A.cp, 0.f) : 0.f);
          const float mine = r * top.e, theirs = top.r * e;      // r / e against the best so far
          if (mine > theirs || (mine == theirs && r > 0.f && i < top.i)) top = Racer{r, e, i};
        });
      } else {
        int blk = -1;
        uint4 w = make_uint4(0, 0, 0, 0);
        each_pair<kDtype>(q, p, V, rank, C, tid, kVerThreads, [&](int i, float x, float y) {
          const float r = prob(rq, x, A.cq, rest ? sh : 0.f) - (rest ? prob(rp, y, A.cp, 0.f) : 0.f);
          if (!(r > 0.f)) return;
          if ((i >> 2) != blk) {
            blk = i >> 2;
            w = philox_block(A.seed, (uint32_t)b, (uint32_t)blk, kStreamRace, 0);
          }
          const uint32_t k = i & 3;
          const float e = -log_uniform(k == 0 ? w.x : k == 1 ? w.y : k == 2 ? w.z : w.w);
          const float mine = r * top.e, theirs = top.r * e;
          if (mine > theirs || (mine == theirs && i < top.i)) top = Racer{r, e, i};
        });
      }
    }
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

// CTAs per chain.
static int verify_cluster(int B, int V, int dtype) {
  const int64_t nvec = (int64_t)V * (int64_t)elem_bytes(dtype) / 16;
  int c = 1;
  while (c < kVerMaxCluster && (int64_t)B * c < 2 * sm_count() && nvec / (2 * c) >= 32 * kVerSegs) c *= 2;
  return c;
}

template <int kDtype>
static cudaError_t launch_token_verify(const TokenVerifyArgs& A, int B, int dtype, cudaStream_t s) {
  const int C = verify_cluster(B, A.V, dtype);
  return launch_cluster(k_token_verify<kDtype>, dim3((unsigned)B * (unsigned)C), kVerThreads, 0, (unsigned)C, s, A);
}

}  // namespace sdv

using namespace sdv;

extern "C" {

int sdv_token_verify(const void* target, int64_t target_stride_b, int64_t target_stride_row, const void* draft,
                     int64_t draft_stride_b, int64_t draft_stride_row, const int32_t* tokens, int B, int L, int V, int dtype,
                     float temperature, float draft_temperature, int mode, const int32_t* L_eff, uint64_t seed,
                     const float* coins, const float* race, int32_t* accepted_len, int32_t* next_token,
                     float* log_ratio_out, uint32_t* status_out, sdv_stream_t stream) {
  if (B < 1 || B > (1 << 27) || L < 1 || L > SDV_MAX_L || V < 1 || V > (1 << 30) || !token_dtype(dtype)) return SDV_EINVAL;
  if (mode != SDV_MODE_SAMPLE && mode != SDV_MODE_BLOCK) return SDV_EINVAL;
  const float t[2] = {temperature, draft_temperature};
  for (float x : t)
    if (!(x > 0.f) || !(x < INFINITY) || !(kLog2E / x < INFINITY)) return SDV_EINVAL;
  if (!target || !draft || !tokens || !accepted_len || !next_token) return SDV_EINVAL;
  if (target_stride_row < V || draft_stride_row < V || target_stride_b < 0 || draft_stride_b < 0) return SDV_EINVAL;
  if (!aligned_to(target, elem_bytes(dtype)) || !aligned_to(draft, elem_bytes(dtype))) return SDV_EALIGN;
  const void* four[] = {tokens, L_eff, coins, race, accepted_len, next_token, log_ratio_out, status_out};
  for (const void* p : four)
    if (!aligned_to(p, 4)) return SDV_EALIGN;
  const TokenVerifyArgs A{target, draft, target_stride_b, target_stride_row, draft_stride_b, draft_stride_row, tokens, L, V,
                          mode, kLog2E / temperature, kLog2E / draft_temperature, 1.f / temperature,
                          1.f / draft_temperature, L_eff, seed, coins, race, accepted_len, next_token, log_ratio_out,
                          status_out};
  cudaStream_t s = (cudaStream_t)stream;
  return launched(dtype == SDV_F32    ? launch_token_verify<SDV_F32>(A, B, dtype, s)
                  : dtype == SDV_BF16 ? launch_token_verify<SDV_BF16>(A, B, dtype, s)
                                      : launch_token_verify<SDV_F16>(A, B, dtype, s));
}

}  // extern "C"
