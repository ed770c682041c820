// What the tree attention's kernels for many rows do when a wait gives up, without one that does: the joining kernel on partials
// of the host's, with a CTA marked as having given up; the copying warp when another has; and a barrier that nothing reaches.
// Prints a line for each; the test reads them.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../paper_2606_13426_gb300/csrc/sdv_tree_rows.cuh"

using namespace sdv;

#define OK(call)                                                             \
  do {                                                                       \
    const cudaError_t e_ = (call);                                           \
    if (e_ != cudaSuccess) {                                                 \
      std::printf("%s: %s\n", #call, cudaGetErrorString(e_));                \
      std::exit(1);                                                          \
    }                                                                        \
  } while (0)

template <typename T>
static T* put(const std::vector<T>& x) {
  T* d = nullptr;
  OK(cudaMalloc(&d, x.size() * sizeof(T)));
  OK(cudaMemcpy(d, x.data(), x.size() * sizeof(T), cudaMemcpyHostToDevice));
  return d;
}
template <typename T>
static std::vector<T> get(const T* d, size_t n) {
  std::vector<T> x(n);
  OK(cudaMemcpy(x.data(), d, n * sizeof(T), cudaMemcpyDeviceToHost));
  return x;
}

// Sixteen steps of three sequences, 10, 1 and 5, in four runs: the first two and a half for sequence 0; sequence 1 whole in run 2.
static void check_join(int marked) {
  constexpr int kD = 64;
  using S = TreeShape<kD>;
  const int B = 3, W = 64, G = 2, teams = 4;
  TreeRowsArgs T{};
  AttendArgs& A = T.a;
  A.B = B, A.W = W, A.G = G, A.R = W * G, A.RT = 1, A.step = 128, A.ctas = teams, A.bf16 = false, A.out_vec = true;
  A.c.H = 1, A.c.D = kD, A.c.block = 128, A.c.max_pages = 16;
  T.rows = 128, T.teams = teams;
  const size_t slots = (size_t)teams * 2 * S::kSlot, floats = slots + (size_t)teams * 2 * S::kAsideAt;
  std::vector<float> part(floats + teams, 0.f);
  for (int s = 0; s < teams * 2; ++s)
    for (int i = 0; i < 128; ++i) {
      for (int d = 0; d < kD; ++d) part[s * S::kSlot + (size_t)i * kD + d] = 6.f;         // (all alike, so in any order)
      part[s * S::kSlot + 128 * (kD + 2) + i] = 3.f;
    }
  for (int c = 0; c < teams; ++c) reinterpret_cast<int*>(part.data() + floats)[c] = c == marked;
  const std::vector<int32_t> lengths{1280, 128, 640}, parents((size_t)B * W, -1);
  std::vector<uint16_t> out((size_t)B * W * G * kD, 0x1234);                              // (not to be touched)
  std::vector<float> lse((size_t)B * W * G, -7.f);
  std::vector<uint32_t> status(B, 0);
  A.part = put(part), A.lengths = put(lengths), A.parents = put(parents), A.out = put(out), A.lse = put(lse), A.status = put(status);
  k_tree_join<kD><<<B * (kTileRows / 32), kJoinThreads>>>(T);
  OK(cudaGetLastError());
  OK(cudaDeviceSynchronize());
  out = get((const uint16_t*)A.out, out.size()), lse = get(A.lse, lse.size()), status = get(A.status, status.size());
  std::printf("join %d:", marked);
  for (int b = 0; b < B; ++b) {
    int nan = 0, two = 0, kept = 0;
    for (int i = 0; i < W * G * kD; ++i) {
      const uint16_t x = out[(size_t)b * W * G * kD + i];
      nan += (x & 0x7c00) == 0x7c00 && (x & 0x3ff), two += x == 0x4000, kept += x == 0x1234;
    }
    int lnan = 0, lkept = 0;
    for (int i = 0; i < W * G; ++i) lnan += std::isnan(lse[b * W * G + i]), lkept += lse[b * W * G + i] == -7.f;
    const int all = W * G * kD, rows = W * G;
    const char* what = nan == all && lnan == rows ? "nan" : two == all && !lnan && !lkept ? "joined" : kept == all && lkept == rows ? "kept" : "mixed";
    std::printf(" %s/%u", what, status[b]);
  }
  std::printf("\n");
}

__global__ void k_copy(const TreeRowsArgs T, uint8_t* got) {
  constexpr int kD = 64;
  using S = TreeShape<kD>;
  extern __shared__ uint8_t raw[];
  uint8_t* smem = raw + (-smem_addr(raw) & 1023);
  TreeSmall& sm = *reinterpret_cast<TreeSmall*>(smem + S::kSmallAt);
  const int lane = threadIdx.x;
  if (lane == 0) {
    for (int k = 0; k < kSegRing; ++k) barrier_init(&sm.seg_full[k], 1);
    for (int k = 0; k < kRawK; ++k) barrier_init(&sm.rk_full[k], 1), barrier_init(&sm.rk_free[k], kGroupWarps);
    for (int k = 0; k < kRawV; ++k) barrier_init(&sm.rv_full[k], 1), barrier_init(&sm.rv_free[k], kGroupWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sm.dead = 1;                                            // another warp has given up
    Segment g{};
    g.steps = 10, g.len = 1280, g.count = 1;
    sm.segs[0] = g;
  }
  warp_arrive(&sm.seg_full[0], lane);
  copy_role<kD>(T, smem, sm, lane);
  for (int i = lane; i < kRawK * S::kHalf; i += 32) got[i] = smem[S::kRk + i];            // the first steps' keys, values
  for (int i = lane; i < kRawK * S::kHalf; i += 32) got[kRawK * S::kHalf + i] = smem[S::kRv + i];
}
static void check_copy() {
  constexpr int kD = 64, kPages = 10;
  using S = TreeShape<kD>;
  TreeRowsArgs T{};
  AttendArgs& A = T.a;
  A.step = 128, A.c.H = 1, A.c.D = kD, A.c.block = 128, A.c.max_pages = kPages, A.c.pages = kPages;
  std::vector<uint8_t> codes((size_t)2 * kPages * S::kHalf);
  for (size_t i = 0; i < codes.size(); ++i) codes[i] = (uint8_t)(i * 2654435761u >> 13);
  std::vector<int32_t> table(kPages);
  for (int i = 0; i < kPages; ++i) table[i] = (i * 3 + 4) % kPages;
  A.c.k = put(codes), A.c.v = A.c.k + (size_t)kPages * S::kHalf, A.c.table = put(table);
  A.c.ks = A.c.vs = put(std::vector<float>(kPages, 1.f));
  std::vector<uint8_t> got((size_t)2 * kRawK * S::kHalf, 0);
  uint8_t* d = put(got);
  OK(cudaFuncSetAttribute(k_copy, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem));
  k_copy<<<1, 32, S::kSmem>>>(T, d);
  OK(cudaGetLastError());
  OK(cudaDeviceSynchronize());
  got = get(d, got.size());
  size_t same = 0;
  for (int kind = 0; kind < 2; ++kind)
    for (int t = 0; t < kRawK; ++t)
      for (int i = 0; i < S::kHalf; ++i)
        same += got[((size_t)kind * kRawK + t) * S::kHalf + i] == codes[((size_t)kind * kPages + table[t]) * S::kHalf + i];
  std::printf("copies: %s\n", same == got.size() ? "there" : "missing");
}

__global__ void k_wait(int* said) {
  __shared__ uint64_t bar;
  __shared__ int dead;
  barrier_init(&bar, 1);
  dead = 0;
  said[0] = barrier_wait(&bar, 0, &dead);                   // nothing arrives
  said[1] = dead;
  said[2] = barrier_wait(&bar, 0, &dead);                   // at once, now that one has given up
}
static void check_wait() {
  int* d = put(std::vector<int>(3, 9));
  k_wait<<<1, 1>>>(d);
  OK(cudaGetLastError());
  OK(cudaDeviceSynchronize());
  const std::vector<int> said = get(d, 3);
  std::printf("wait: %d %d %d\n", said[0], said[1], said[2]);
}

int main() {
  for (int marked : {-1, 0, 2, 3}) check_join(marked);
  check_copy();
  check_wait();
  return 0;
}
