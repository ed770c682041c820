// sdv_token_rows.cuh - what the verifications of windows and of trees share: probabilities from a row's
// statistics, passes over pairs of rows, the race that draws a token.
#pragma once

#include "sdv_device.cuh"
#include "sdv_tokens.cuh"

namespace sdv {

constexpr int kVerThreads = 256;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kVerMaxCluster = 16;
constexpr uint32_t kStreamRace = 7;

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

struct AnyToken {
  __device__ __forceinline__ bool operator()(int) const { return true; }
};
// A thread's best of the race for r / E over its share of two rows (each_pair's), r = rest(index, q's logit, p's), among the
// tokens that are `in`: asked of those that would win alone.
template <int kDtype, typename F, typename G = AnyToken>
__device__ __forceinline__ void race_part(const typename Num<kDtype>::T* q, const typename Num<kDtype>::T* p, int V, int part,
                                          int log_parts, int lane, int step, const float* race, uint64_t seed, uint32_t b, Racer& top,
                                          F rest, G in = G()) {
  constexpr int kPer = Num<kDtype>::kPer16;
  each_pair<kDtype>(q, p, V, part, log_parts, lane, step, [&](int i, int count, const float* x, const float* y) {
    float r[kPer], e[kPer];
    bool any = false;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      r[k] = rest(i + k, x[k], y[k]);
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
      float4 four = race4(seed, b, (uint32_t)i >> 2);
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        if (k && ((i + k) & 3) == 0) four = race4(seed, b, (uint32_t)(i + k) >> 2);
        const int w = (i + k) & 3;
        e[k] = w == 0 ? four.x : w == 1 ? four.y : w == 2 ? four.z : four.w;
      }
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {                            // r / e against the best so far
      const float mine = r[k] * top.e, theirs = top.r * e[k];
      if ((mine > theirs || (mine == theirs && r[k] > 0.f && i + k < top.i)) && in(i + k)) top = Racer{r[k], e[k], i + k};
    }
  });
}

// CTAs per chain: as many as fit beside the other chains' (three an SM), as long as each thread has a vector
// of a row.  With half as many 16 x 8 x 131072 bf16 take 35 us in place of 33 and 48 x 7 x 50001 fp32 29 in
// place of 26; with twice as many, more than are resident together, the latter 37.
inline int verify_cluster(int B, int V, int dtype) {
  const int64_t nvec = (int64_t)V * (int64_t)elem_bytes(dtype) / 16;
  int c = 1;
  while (c < kVerMaxCluster && (int64_t)B * 2 * c <= 3 * sm_count() && nvec >= 2 * c * kVerThreads) c *= 2;
  return c;
}

}  // namespace sdv
