// sdv_tokens.cuh - what the token operators' kernels share: rows of logits read as 16-byte
// vectors from wherever they start, running softmax statistics, clusters.
#pragma once

#include <cooperative_groups.h>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "../../include/specdiff.h"
#include "sdv_host.h"

namespace sdv {

namespace cg = cooperative_groups;

constexpr float kLog2E = 1.44269504088896341f;   // log2 e
constexpr float kLn2f = 0.69314718055994531f;    // log 2
// Far below any difference of two logits that leaves a probability, and finite: 0 * kFar is 0
// where 0 * -inf would be NaN.  The temperatures allowed keep it so: kFar / T is -1000 or less,
// and kFar / T^2, a factor in the entropy's gradient, finite.
constexpr float kFar = -1e12f;
constexpr float kLeastTemperature = 1e-9f, kMostTemperature = 1e9f;

template <int kDtype>
struct Num;
template <>
struct Num<SDV_F32> {
  using T = float;
  static constexpr int kPer16 = 4;
  static __device__ __forceinline__ float to(T x) { return x; }
  static __device__ __forceinline__ T from(float x) { return x; }
  static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <>
struct Num<SDV_BF16> {
  using T = __nv_bfloat16;
  static constexpr int kPer16 = 8;
  static __device__ __forceinline__ float to(T x) { return __bfloat162float(x); }
  static __device__ __forceinline__ T from(float x) { return __float2bfloat16_rn(x); }
  static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Num<SDV_F16> {
  using T = __half;
  static constexpr int kPer16 = 8;
  static __device__ __forceinline__ float to(T x) { return __half2float(x); }
  static __device__ __forceinline__ T from(float x) { return __float2half_rn(x); }
  static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      f[2 * i] = p.x;
      f[2 * i + 1] = p.y;
    }
  }
  static __device__ __forceinline__ uint4 pack(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// A row of V elements as `head` single elements up to the next 16-byte boundary, `nvec`
// vectors and `tail` single elements.
template <int kDtype>
struct Row {
  using T = typename Num<kDtype>::T;
  static constexpr int kPer = Num<kDtype>::kPer16;
  const T* p;
  int V, head, nvec, tail;
  __device__ __forceinline__ Row(const T* row, int V_) : p(row), V(V_) {
    const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    head = off ? min(V, kPer - off) : 0;
    nvec = (V - head) / kPer;
    tail = V - head - nvec * kPer;
  }
  __device__ __forceinline__ const uint4* vec() const { return reinterpret_cast<const uint4*>(p + head); }
  // Element of single i (the head's, then the tail's).
  __device__ __forceinline__ int single(int i) const { return i < head ? i : V - tail + (i - head); }
  __device__ __forceinline__ int singles() const { return head + tail; }
};

// The first of part `part`'s share of n (below 2^28) things in 2^log_parts parts, part at most 2^log_parts.
// (A shift: 64-bit divisions took a third of the instructions of the kernels with one row a CTA.)
__device__ __forceinline__ int share(int n, int part, int log_parts) {
  return (int)((uint64_t)(uint32_t)n * (uint32_t)part >> log_parts);
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Maximum that keeps a NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// Running softmax statistics of x_v / T: the maximum m of x, s = sum e^{(x - m)/T} and
// w = sum e^{(x - m)/T} (x - m).  A NaN or +inf logit shows as such in m.
struct Stat {
  float m, s, w;
};
__device__ __forceinline__ Stat stat_empty() { return Stat{-INFINITY, 0.f, 0.f}; }

// c = log2(e) / T
__device__ __forceinline__ void stat_rebase(Stat& a, float m, float c) {
  const float d = fmaxf(a.m - m, kFar);          // a.m = -inf holds nothing: s = w = 0
  const float f = ex2(d * c);
  a.w = f * fmaf(a.s, d, a.w);
  a.s *= f;
  a.m = m;
}
__device__ __forceinline__ Stat stat_join(Stat a, Stat b, float c) {
  const float m = max_nan(a.m, b.m);
  stat_rebase(a, m, c);
  stat_rebase(b, m, c);
  return Stat{m, a.s + b.s, a.w + b.w};
}
// Two fp32 operations an instruction.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpair(f32x2 x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 far2(f32x2 d) {             // max(d, kFar)
  const float2 x = unpair(d);
  return pair(fmaxf(x.x, kFar), fmaxf(x.y, kFar));
}

// A vector of masked logits.
template <int kDtype>
__device__ __forceinline__ uint4 vec_masked() {
  const uint32_t w = kDtype == SDV_F32 ? 0xff800000u : kDtype == SDV_BF16 ? 0xff80ff80u : 0xfc00fc00u;
  return make_uint4(w, w, w, w);
}

// The largest value of a 16-byte vector (a NaN stays).
template <int kDtype>
__device__ __forceinline__ float vec_max(const uint4& v) {
  if constexpr (kDtype == SDV_F32) {
    return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
  } else {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (kDtype == SDV_BF16) {
      const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(w);
      const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3]));
      return max_nan(__low2float(m), __high2float(m));
    } else {
      const __half2* p = reinterpret_cast<const __half2*>(w);
      const __half2 m = __hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3]));
      return max_nan(__low2float(m), __high2float(m));
    }
  }
}

// The same without regard to NaN.
template <int kDtype>
__device__ __forceinline__ float vec_max_num(const uint4& v) {
  if constexpr (kDtype == SDV_F32) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  } else {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (kDtype == SDV_BF16) {
      const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(w);
      const __nv_bfloat162 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
      return fmaxf(__low2float(m), __high2float(m));
    } else {
      const __half2* p = reinterpret_cast<const __half2*>(w);
      const __half2 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
      return fmaxf(__low2float(m), __high2float(m));
    }
  }
}

// A thread's running statistics: sums against a reference that moves only when a logit passes it by
// 2^8 (in e^{d/T}), and the largest logit.
struct Run {
  float ref, lim, top;
  f32x2 s, w;
};
__device__ __forceinline__ Run run_empty() { return Run{-INFINITY, -INFINITY, -INFINITY, 0ull, 0ull}; }
// Makes room for logits up to `top`.
__device__ __forceinline__ void run_see(Run& r, float top, float c) {
  r.top = max_nan(r.top, top);
  if (!(top <= r.lim)) {
    const float d = fmaxf(r.ref - top, kFar), f = ex2(d * c);      // ref = -inf holds nothing
    r.w = mul2(pair(f, f), fma2(r.s, pair(d, d), r.w));
    r.s = mul2(pair(f, f), r.s);
    r.ref = top;
    r.lim = top + 8.f / c;
  }
}
// Adds n (even) logits that it has made room for.
template <int n, bool kEntropy = true>
__device__ __forceinline__ void run_add(Run& r, const float* x, float c) {
  const f32x2 m = pair(-r.ref, -r.ref), c2 = pair(c, c);
#pragma unroll
  for (int i = 0; i < n; i += 2) {
    const f32x2 d = far2(add2(pair(x[i], x[i + 1]), m));
    const float2 t = unpair(mul2(d, c2));
    const f32x2 e = pair(ex2(t.x), ex2(t.y));
    r.s = add2(r.s, e);
    if (kEntropy) r.w = fma2(e, d, r.w);
  }
}
// A warp's statistics, against its largest logit.
__device__ __forceinline__ Stat run_warp(const Run& r, float c) {
  const float2 s = unpair(r.s), w = unpair(r.w);
  Stat a{r.ref, s.x + s.y, w.x + w.y};
  float m = r.top;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  stat_rebase(a, m, c);
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.w += __shfl_xor_sync(0xffffffffu, a.w, o);
  }
  return a;
}
// A single logit.
__device__ __forceinline__ void run_one(Run& r, float x, float c) {
  run_see(r, x, c);
  const float two[2] = {x, -INFINITY};
  run_add<2>(r, two, c);
}
// The warp's statistics: one rebase a lane to the common maximum, then plain sums.
__device__ __forceinline__ Stat stat_warp(Stat a, float c) {
  float m = a.m;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  stat_rebase(a, m, c);
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.w += __shfl_xor_sync(0xffffffffu, a.w, o);
  }
  return a;
}
// The statistics of n parts, by a whole warp.
__device__ __forceinline__ Stat stat_gather(const Stat* part, int n, int lane, float c) {
  Stat a = stat_empty();
  for (int i = lane; i < n; i += 32) a = i == lane ? part[i] : stat_join(a, part[i], c);
  return stat_warp(a, c);
}

// The order of the alternatives: the larger logit first, of equal ones the lower index.
__device__ __forceinline__ bool before(float a, int ia, float b, int ib) { return a > b || (a == b && ia < ib); }

constexpr int kScoreThreads = 256;
constexpr int kScoreVecs = 8;          // 16-byte vectors of a thread under way at once
constexpr int kScoreMaxCluster = 8;

// A thread's part of a row: vectors v0 + tid + u kStep < v1, and one of the row's single elements;
// kStep threads share the row's part.
template <int kDtype, bool kEntropy, int kStep = kScoreThreads>
struct Part {
  using E = Num<kDtype>;
  static __device__ __forceinline__ int tid() { return (int)threadIdx.x & (kStep - 1); }
  const uint4* vec;
  int v0, v1, single;
  float x;
  __device__ __forceinline__ Part(const Row<kDtype>& R, int rank, int log_c) {
    vec = R.vec();
    v0 = share(R.nvec, rank, log_c) + tid();
    v1 = share(R.nvec, rank + 1, log_c);
    single = rank == 0 && tid() < R.singles() ? R.single(tid()) : -1;
    x = single >= 0 ? E::to(R.p[single]) : 0.f;
  }
  // Its statistics; what is past the part counts as masked: one copy of the code for whole and partial
  // batches, which are run once and so from a cold instruction cache.
  __device__ __forceinline__ Run read(float c) const {
    Run r = run_empty();
#pragma unroll 1
    for (int v = v0; v - tid() < v1; v += kScoreVecs * kStep) {
      uint4 raw[kScoreVecs];
#pragma unroll
      for (int u = 0; u < kScoreVecs; ++u) {
        raw[u] = vec_masked<kDtype>();
        if (v + u * kStep < v1) raw[u] = vec[v + u * kStep];
      }
#pragma unroll
      for (int u = 0; u < kScoreVecs; ++u) {
        float f[E::kPer16];
        if (u % 4 == 0) {
          float top = vec_max<kDtype>(raw[u]);
#pragma unroll
          for (int k = 1; k < 4; ++k) top = max_nan(top, vec_max<kDtype>(raw[u + k]));
          run_see(r, top, c);
        }
        E::unpack(raw[u], f);
        run_add<E::kPer16, kEntropy>(r, f, c);
      }
    }
    if (single >= 0) run_one(r, x, c);
    return r;
  }
};

// CTAs per row: while there are fewer than four an SM, as many as leave every thread sixteen vectors.  With
// 16, 4 and 32 of them, without alternatives / with 20 (us, bf16): 128 rows of 32768 4.3 / 8.5, 5.8 / 11.5
// and 4.2 / 7.0; 300 of 8192 3.8 / 6.2, 6.0 / 10.9, 3.9 / 6.3; 32 of 65536 3.8 / 8.1, 4.2 / 9.8, 4.6 / 8.6; 1 of
// 131072 3.3 / 8.4, 3.7 / 8.8, 4.1 / 8.4.  With up to two CTAs an SM 144 of 131072 take 11.4 in place of 10.3.
inline int score_cluster(int64_t N, int V, int dtype) {
  const int64_t nvec = (int64_t)V * (dtype == SDV_F32 ? 4 : 2) / 16;
  int c = 1;
  while (c < kScoreMaxCluster && N * 2 * c <= 4 * sm_count() && nvec >= 16 * c * kScoreThreads) c *= 2;
  return c;
}

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool real) {
  const int n = real ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n));
}

// A launch in clusters of `cluster` CTAs along x; early: it may start before the kernel before it
// ends (and waits for it itself).
template <typename Kern, typename... Args>
inline cudaError_t launch_cluster(Kern kern, dim3 grid, unsigned threads, size_t smem, unsigned cluster, bool early,
                                  cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cluster;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = early ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline int min_int(int a, int b) { return a < b ? a : b; }
inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t elem_bytes(int dtype) { return dtype == SDV_F32 ? 4 : 2; }
inline bool temperature_ok(float t) { return t >= kLeastTemperature && t <= kMostTemperature; }
inline bool token_dtype(int dtype) { return dtype == SDV_F32 || dtype == SDV_BF16 || dtype == SDV_F16; }

// The return code of a launch.
inline int launched(cudaError_t e) {
  if (e == cudaSuccess) return SDV_OK;
  cudaGetLastError();
  set_last_cuda_error((int)e);
  return SDV_ECUDA;
}

}  // namespace sdv
