// Launches of the mixed-batch products (gemm_batch.h).
#include "gemm_ring.h"

namespace dif {

template <typename T, typename OutT>
hipError_t launch_gemm_batch(const T* A, int64_t lda, const T* B, int64_t ldb, OutT* C, int64_t ldc, int M, int N,
                             int K, int epi, const float* bias, const float* gate0, const float* gate1,
                             const BatchGroups* groups, const BatchLora* lora, hipStream_t stream) {
  if (M <= 0 || N <= 0) return hipSuccess;
  BatchParams<T, OutT> p{};
  p.A = A;
  p.Bs[0] = B;
  p.C = C;
  p.lda = lda;
  p.ldb = ldb;
  p.ldc = ldc;
  p.M = M;
  p.N = N;
  p.K = K;
  p.biases[0] = bias;
  p.nseg = 1;
  p.gate0 = gate0;
  p.gate1 = gate1;
  p.vec4 = ldc % 4 == 0 && reinterpret_cast<uintptr_t>(C) % (4 * sizeof(OutT)) == 0;
  p.n_groups = p.n_weights = 1;
  if (groups) {
    p.group_off = groups->off;
    p.w_index = groups->index;
    p.n_groups = groups->n_groups;
    p.n_weights = groups->n_weights;
    p.n_kept = groups->n_kept;
    p.k_kept = groups->k_kept;
    p.b_stride = groups->b_stride;
    p.bias_stride = groups->bias_stride;
    p.gate_stride = groups->gate_stride;
  }
  if (lora) {
    p.request_off = lora->off;
    p.adapter = lora->adapter;
    p.n_requests = lora->n_requests;
    p.n_adapters = lora->n_adapters;
    p.rank = lora->rank;
    p.ranks = lora->ranks;
    p.scales = lora->scales;
    p.low = lora->low;
    p.ld_low = lora->ld_low;
    p.up = static_cast<const T*>(lora->up);
    p.ld_up = lora->ld_up;
    p.up_stride = lora->up_stride;
    if (K > 0 && lora->rank > 0 && lora->n_adapters > 0) {
      // low = A down^T: requests as groups, adapters as matrices, ranks as widths
      BatchParams<T, float> q{};
      q.A = A;
      q.Bs[0] = static_cast<const T*>(lora->down);
      q.C = lora->low;
      q.lda = lda;
      q.ldb = lora->ld_down;
      q.ldc = lora->ld_low;
      q.M = M;
      q.N = lora->rank;
      q.K = K;
      q.nseg = 1;
      q.vec4 = 1;
      q.group_off = lora->off;
      q.w_index = lora->adapter;
      q.n_groups = lora->n_requests;
      q.n_weights = lora->n_adapters;
      q.n_kept = lora->ranks;
      q.b_stride = lora->down_stride;
      const int shape = pick_tile<T>(M, lora->rank, 1, K, EPI_STORE, q.n_groups < M ? q.n_groups : M);
      const hipError_t e = launch_gemm_batch_ring<T, float>(shape, q, EPI_STORE, stream);
      if (e != hipSuccess) return e;
    } else {
      p.request_off = lora->off;   // (rows of no request stay untouched)
      p.n_adapters = 0;            // no term
    }
  }
  const int shape = pick_tile<T>(M, N, 1, K, epi, p.n_groups < M ? p.n_groups : M);
  return launch_gemm_batch_ring<T, OutT>(shape, p, epi, stream);
}

#define INST(T, OutT)                                                                                             \
  template hipError_t launch_gemm_batch<T, OutT>(const T*, int64_t, const T*, int64_t, OutT*, int64_t, int, int, \
                                                 int, int, const float*, const float*, const float*,             \
                                                 const BatchGroups*, const BatchLora*, hipStream_t);
INST(bf16, bf16)
INST(bf16, float)
INST(float, float)
#undef INST

}  // namespace dif
