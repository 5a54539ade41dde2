// Launches of the mixed-batch products (gemm_batch.h).
#include "gemm_ring.h"

namespace dif {

// Parts of the reduction of low = A down^T: few rows make few tiles, each a long
// chain of k-tiles (16 rows, rank 16, K = 5120: 12.4 us in one part, 4.8 in 16).  As many as
// fill the chip with 32 x 32 tiles twice, of about four k-tiles each, that the
// workspace holds.
static int low_parts(int M, int rank, int groups, int nk, int most) {
  const int64_t tiles = (int64_t)groups * ((M / groups + 31) / 32) * ((rank + 31) / 32);
  int64_t parts = 2 * kCus / tiles;
  if (parts > nk / 4) parts = nk / 4;
  if (parts > most) parts = most;
  return parts < 2 ? 1 : (int)parts;
}

// Tile shape of low where it is not split.  Ranks of their own lie anywhere up to the
// widest, so that what the host sees of low is its largest size: 32 x 32 tiles are the
// fastest while no CU has two (a CU then streams its rows alone), 64 x 64 with more.
// Up to 5/3 tiles a CU at the largest size the first lose less on full ranks than the
// second on small ones (bf16, K = 5120, eight requests, us on 32 x 32 and on 64 x 64: 392
// tiles with all ranks 64 of 64 20.6 and 19.5, 32 14.0 and 19.0, 16 to 64 20.4 and 19.2; 500
// tiles 29.7 and 19.9, 18.2 and 19.0, 25.5 and 19.2).  A rank of 32 or less is one column of
// tiles whatever the ranks (391 tiles 24.7 and 22.2).
template <typename T>
static int low_shape(int M, int rank, bool ranks, int groups, int K) {
  const int64_t tiles = (int64_t)((M + 31) / 32) * ((rank + 31) / 32);
  if (ranks && rank > 32 && tiles * 3 <= 5 * kCus) return TS_32;
  return pick_tile<T>(M, rank, 1, K, EPI_STORE, groups);
}

template <typename T, typename OutT>
static hipError_t launch_shape(int shape, const BatchParams<T, OutT>& p, int epi, hipStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (shape == TS_256) return launch_gemm_batch_256<OutT>(p, epi, s);
  return launch_gemm_batch_ring<T, OutT>(shape, p, epi, s);
}

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
    if (K > 0 && lora->n_adapters > 0) {
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
      const int groups_met = lora->n_requests < M ? lora->n_requests : M;
      int shape = low_shape<T>(M, lora->rank, lora->ranks != nullptr, groups_met, K);
      const int parts = low_parts(M, lora->rank, groups_met, K / (128 / (int)sizeof(T)), lora->max_parts);
      p.low_parts = 1;
      if (parts > 1) {
        shape = TS_32;
        const int kt = 128 / (int)sizeof(T), nk = (K + kt - 1) / kt;
        q.parts = p.low_parts = parts;   // (the last may be empty: zeros)
        q.k_part = (nk + parts - 1) / parts * kt;
        q.c_part = p.low_stride = (int64_t)M * lora->ld_low;
      }
      const hipError_t e = launch_shape<T, float>(shape, q, EPI_STORE, stream);
      if (e != hipSuccess) return e;
    } else {
      p.n_adapters = 0;   // no term (rows of no request still stay untouched)
    }
  }
  const int shape = pick_tile<T>(M, N, 1, K, epi, p.n_groups < M ? p.n_groups : M, p.n_adapters > 0 ? p.n_requests : 0, p.rank);
  return launch_shape<T, OutT>(shape, p, epi, stream);
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
