// The mixed-batch entry points (csrc/batch.cpp) on the host under AddressSanitizer
// and UndefinedBehaviorSanitizer: the kernels' launch is a stand-in that reads the
// tables (host memory here) and touches the ends of every region the kernels address
// for the rows, widths and ranks in them, so that a size that the checks let through
// or pass on wrongly becomes an out-of-bounds access.  Test infrastructure only.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../include/dif.h"
#include "../../paper_2607_06631_amd/csrc/kernels.h"

hipError_t hipEventCreate(hipEvent_t*) { return hipErrorInvalidValue; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipErrorInvalidValue; }
const char* hipGetErrorString(hipError_t) { return "stub error"; }

static long g_launches = 0;
static hipError_t g_result = hipSuccess;
static volatile unsigned char g_sink;

template <typename T>
static void ends(const T* base, int64_t rows, int64_t ld, int64_t width, bool write = false) {
  if (rows <= 0 || width <= 0) return;
  for (int64_t r : {int64_t(0), rows - 1})
    for (int64_t k : {int64_t(0), width - 1}) {
      unsigned char* p = (unsigned char*)(base + r * ld + k);
      if (write) *p = 1;
      else g_sink = *p;
    }
}

namespace dif {
template <typename T, typename OutT>
hipError_t launch_gemm_batch(const T* A, int64_t lda, const T* B, int64_t ldb, OutT* C, int64_t ldc, int M, int N,
                             int K, int, const float* bias, const float* gate0, const float* gate1,
                             const BatchGroups* g, const BatchLora* l, hipStream_t) {
  ++g_launches;
  ends(A, M, lda, K);
  ends(C, M, ldc, N, true);
  if (gate0) ends(gate0, 1, 0, N);
  const int groups = g ? g->n_groups : 1, weights = g ? g->n_weights : 1;
  for (int i = 0; i < groups; ++i) {
    const int w = g && g->index ? g->index[i] : i;
    if (g) g_sink = (unsigned char)(g->off[i] + g->off[i + 1]);
    if (w < 0 || w >= weights) continue;
    const int n = g && g->n_kept ? g->n_kept[w] : N, k = g && g->k_kept ? g->k_kept[w] : K;
    ends(B + (g ? w * g->b_stride : 0), std::min(n, N), ldb, std::min(k, K));
    if (bias) ends(bias + (g ? w * g->bias_stride : 0), 1, 0, N);
    if (gate1) ends(gate1 + (g ? w * g->gate_stride : 0), 1, 0, N);
  }
  if (l) {
    for (int q = 0; q < l->n_requests; ++q) {
      g_sink = (unsigned char)(l->off[q] + l->off[q + 1]);
      const int a = l->adapter[q];
      if (a < 0 || a >= l->n_adapters || K == 0) continue;
      if (l->scales) g_sink = (unsigned char)l->scales[a];
      const int r = l->ranks ? std::min(std::max(l->ranks[a], 0), l->rank) : l->rank;
      ends((const T*)l->down + a * l->down_stride, r, l->ld_down, K);
      ends((const T*)l->up + a * l->up_stride, N, l->ld_up, r);
    }
    if (l->n_adapters > 0 && K > 0) ends(l->low, (int64_t)l->max_parts * M, l->ld_low, l->ld_low, true);
  }
  return g_result;
}
#define INST(T, O)                                                                                              \
  template hipError_t launch_gemm_batch<T, O>(const T*, int64_t, const T*, int64_t, O*, int64_t, int, int, int, \
                                              int, const float*, const float*, const float*, const BatchGroups*, \
                                              const BatchLora*, hipStream_t);
INST(__bf16, __bf16)
INST(__bf16, float)
INST(float, float)
}  // namespace dif

static void expect(dif_status got, dif_status want, const char* what) {
  if (got != want) {
    std::fprintf(stderr, "%s: status %d, expected %d\n", what, got, want);
    std::exit(1);
  }
}

// exactly sized, 256-byte aligned memory
template <typename T>
struct Mem {
  T* p;
  explicit Mem(size_t n) {
    void* v = nullptr;
    if (posix_memalign(&v, 256, n ? n * sizeof(T) : 1)) std::abort();
    p = (T*)v;
    for (size_t i = 0; i < n; ++i) p[i] = T();
  }
  Mem(const Mem&) = delete;
  ~Mem() { std::free(p); }
};

template <typename T, typename O>
static void sizes(int dt, int out) {
  const int64_t vec = 16 / sizeof(T);
  for (int M : {1, 3, 40})
    for (int N : {1, 33})
      for (int K : {0, 1, 7, 64})
        for (int rank : {1, 5, 64})
          for (int W : {1, 3}) {
            const int64_t lda = std::max<int64_t>((K + vec - 1) / vec * vec, vec), ldu = (rank + vec - 1) / vec * vec;
            // (the last row ends with its last element)
            const size_t nb = ((size_t)W * N - 1) * lda + K, nd = ((size_t)W * rank - 1) * lda + K;
            Mem<T> A((size_t)(M - 1) * lda + K), B(nb), down(nd), up(((size_t)W * N - 1) * ldu + rank);
            Mem<O> C((size_t)(M - 1) * N + N);
            Mem<float> bias((size_t)W * N), gate0(N), gate1((size_t)W * N), scales(W);
            Mem<int32_t> off(W + 1), index(W), kept_n(W), kept_k(W), ranks(W);
            for (int i = 0; i < W; ++i) {
              off.p[i + 1] = M * (i + 1) / W;
              index.p[i] = (i + 1) % W;
              kept_n.p[i] = i ? N : 1 << 30;
              kept_k.p[i] = i ? K : -3;
              ranks.p[i] = i ? rank : 1 << 30;
            }
            dif_groups g{W, W, off.p, index.p, kept_n.p, kept_k.p, N * lda, N, N};
            expect(dif_gemm_grouped(dt, out, A.p, lda, B.p, lda, C.p, N, M, N, K, DIF_EPI_RESIDUAL, bias.p, gate0.p,
                                    gate1.p, &g, nullptr),
                   DIF_OK, "grouped");
            g.k_kept = nullptr;
            size_t need = 0;
            expect(dif_lora_workspace_bytes(M, rank, &need), DIF_OK, "workspace bytes");
            Mem<char> ws(need);
            dif_lora l{W, W, rank, off.p, index.p, ranks.p, scales.p, down.p, lda, rank * lda, up.p, ldu, N * ldu};
            expect(dif_gemm_lora(dt, out, A.p, lda, B.p, lda, C.p, N, M, N, K, DIF_EPI_GELU, bias.p, nullptr, nullptr,
                                 &g, &l, ws.p, need, nullptr),
                   DIF_OK, "lora");
            expect(dif_gemm_lora(dt, out, A.p, lda, B.p, lda, C.p, N, M, N, K, DIF_EPI_STORE, nullptr, nullptr,
                                 nullptr, nullptr, &l, ws.p, need, nullptr),
                   DIF_OK, "lora, one matrix");
            if (K) {
              expect(dif_gemm_lora(dt, out, A.p, lda, B.p, lda, C.p, N, M, N, K, DIF_EPI_STORE, nullptr, nullptr,
                                   nullptr, nullptr, &l, ws.p, need - 1, nullptr),
                     DIF_E_WORKSPACE, "small workspace");
            }
            l.n_adapters = 0;
            l.down = l.up = nullptr;
            expect(dif_gemm_lora(dt, out, A.p, lda, B.p, lda, C.p, N, M, N, K, DIF_EPI_STORE, nullptr, nullptr,
                                 nullptr, nullptr, &l, nullptr, 0, nullptr),
                   DIF_OK, "no adapters");
          }
}

int main() {
  sizes<__bf16, __bf16>(DIF_BF16, DIF_BF16);
  sizes<__bf16, float>(DIF_BF16, DIF_F32);
  sizes<float, float>(DIF_F32, DIF_F32);
  g_result = hipErrorInvalidValue;
  Mem<float> A(64), C(4);
  Mem<int32_t> off(2);
  off.p[1] = 1;
  dif_groups g{1, 1, off.p, nullptr, nullptr, nullptr, 0, 0, 0};
  expect(dif_gemm_grouped(DIF_F32, DIF_F32, A.p, 64, A.p, 64, C.p, 4, 1, 1, 64, 0, nullptr, nullptr, nullptr, &g, nullptr),
         DIF_E_HIP, "a failing launch");
  std::printf("harness: %ld launches, all cases passed\n", g_launches);
  return 0;
}
