// C ABI of the mixed-batch products: matrices grouped by rows, adapters per
// request.  Host side only: argument checks and the launches (gemm_batch.hip).
#include <algorithm>
#include <cstdint>

#include "host.h"
#include "kernels.h"

using namespace dif;

namespace {

// a 256-row block of any matrix is addressed through 32-bit buffer offsets: the
// bytes of a row
constexpr int64_t kRowLimit = (int64_t(1) << 31) / 256;

struct Product {
  int32_t dtype, out_dtype;
  const void* A;
  int64_t lda;
  const void* B;
  int64_t ldb;
  void* C;
  int64_t ldc;
  int32_t M, N, K, epilogue;
  const float *bias, *gate0, *gate1;
};

inline bool misaligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

// A matrix of `rows` long rows of 16-byte pieces: its row stride, and the stride
// between such matrices where there are several.
dif_status check_rows(const char* name, const void* p, int64_t ld, int64_t width, int64_t es, int64_t count,
                      int64_t stride) {
  if (!p) return fail(DIF_E_ARG, "%s is null", name);
  if (misaligned(p, 16)) return fail(DIF_E_ARG, "%s must be 16-byte aligned", name);
  if (ld < width) return fail(DIF_E_SHAPE, "%s: row stride %lld below the width %lld", name, (long long)ld,
                              (long long)width);
  if (ld >= kRowLimit / es) return fail(DIF_E_SHAPE, "%s: 256 rows span 2 GiB or more", name);
  if (ld * es % 16) return fail(DIF_E_SHAPE, "%s: row stride must be a multiple of 16 bytes", name);
  if (count > 1 && (stride < 0 || stride % (16 / es)))
    return fail(DIF_E_SHAPE, "%s: stride between matrices must be >= 0 and a multiple of 16 bytes", name);
  return DIF_OK;
}

dif_status check_product(const Product& p) {
  if (p.dtype != DIF_BF16 && p.dtype != DIF_F32) return fail(DIF_E_ARG, "bad dtype");
  if (p.out_dtype != p.dtype && p.out_dtype != DIF_F32) return fail(DIF_E_ARG, "bad out_dtype");
  if (p.epilogue < 0 || p.epilogue > 2) return fail(DIF_E_ARG, "bad epilogue");
  if (p.M < 0 || p.N < 0 || p.K < 0) return fail(DIF_E_SHAPE, "negative size");
  return DIF_OK;
}

dif_status check_operands(const Product& p, int64_t n_weights, int64_t b_stride) {
  const int64_t es = esize(p.dtype), oes = esize(p.out_dtype);
  if (!p.C) return fail(DIF_E_ARG, "null output");
  if (misaligned(p.C, oes)) return fail(DIF_E_ARG, "the output must be aligned to its element");
  if (p.ldc < p.N) return fail(DIF_E_SHAPE, "ldc < N");
  if (p.ldc >= kRowLimit / oes) return fail(DIF_E_SHAPE, "256 rows of C span 2 GiB or more");
  if (p.K > 0) {   // A and B are read only when K > 0
    DIF_TRY(check_rows("A", p.A, p.lda, p.K, es, 1, 0));
    DIF_TRY(check_rows("B", p.B, p.ldb, p.K, es, n_weights, b_stride));
  }
  if (p.epilogue != DIF_EPI_RESIDUAL && (p.gate0 || p.gate1))
    return fail(DIF_E_ARG, "gates belong to DIF_EPI_RESIDUAL");
  if (p.gate1 && !p.gate0) return fail(DIF_E_ARG, "gate1 without gate0");
  if (misaligned(p.bias, 4) || misaligned(p.gate0, 4) || misaligned(p.gate1, 4))
    return fail(DIF_E_ARG, "bias and gates must be 4-byte aligned");
  return DIF_OK;
}

dif_status check_groups(const dif_groups* g) {
  if (!g) return fail(DIF_E_ARG, "groups is null");
  if (g->n_groups < 1 || g->n_groups > DIF_MAX_GROUPS)
    return fail(DIF_E_SHAPE, "n_groups %d outside 1 .. %d", g->n_groups, DIF_MAX_GROUPS);
  if (g->n_weights < 1) return fail(DIF_E_SHAPE, "n_weights < 1");
  if (!g->weight_index && g->n_weights < g->n_groups)
    return fail(DIF_E_SHAPE, "%d groups need as many matrices, or a weight_index", g->n_groups);
  if (!g->row_offsets) return fail(DIF_E_ARG, "row_offsets is null");
  if (misaligned(g->row_offsets, 4) || misaligned(g->weight_index, 4) || misaligned(g->n_kept, 4) ||
      misaligned(g->k_kept, 4))
    return fail(DIF_E_ARG, "tables must be 4-byte aligned");
  if (g->bias_stride < 0 || g->gate_stride < 0) return fail(DIF_E_SHAPE, "negative stride");
  return DIF_OK;
}

// The launch must have a tile shape whose grid fits: 96 x 128, which both types have.
dif_status check_extent(int64_t M, int64_t N, int64_t groups) {
  if (M > INT32_MAX - 512 || N > INT32_MAX - 512 || batch_tiles(M, N, std::min(groups, M), 96, 128) > kMostTiles)
    return fail(DIF_E_SHAPE, "problem too large: split the rows over several calls");
  return DIF_OK;
}

BatchGroups to_groups(const dif_groups& g) {
  BatchGroups b;
  b.off = g.row_offsets;
  b.index = g.weight_index;
  b.n_groups = g.n_groups;
  b.n_weights = g.n_weights;
  b.n_kept = g.n_kept;
  b.k_kept = g.k_kept;
  b.b_stride = g.b_stride;
  b.bias_stride = g.bias_stride;
  b.gate_stride = g.gate_stride;
  return b;
}

dif_status run(const Product& p, const BatchGroups* groups, const BatchLora* lora, hipStream_t s) {
  // (the split is in device memory: counted as if every row ran the full widths
  // and every adapter were used)
  const double m = p.M, n = p.N, k = p.K, es = (double)esize(p.dtype), oes = (double)esize(p.out_dtype);
  const double nw = groups ? std::min(groups->n_weights, p.M) : 1, na = lora ? std::min(lora->n_adapters, p.M) : 0;
  const double r = lora ? lora->rank : 0;
  const ProfScope prof(PK_GEMM_IO, s, 2.0 * m * n * k + 2.0 * m * r * (n + k),
                       es * (m * k + nw * n * k + na * r * (n + k)) +
                           oes * m * n * (p.epilogue == DIF_EPI_RESIDUAL ? 2 : 1));
#define CALL(T, O)                                                                                         \
  HIP_TRY((launch_gemm_batch<T, O>((const T*)p.A, p.lda, (const T*)p.B, p.ldb, (O*)p.C, p.ldc, p.M, p.N,   \
                                   p.K, p.epilogue, p.bias, p.gate0, p.gate1, groups, lora, s)))
  if (p.dtype == DIF_BF16 && p.out_dtype == DIF_BF16) CALL(bf16, bf16);
  else if (p.dtype == DIF_BF16) CALL(bf16, float);
  else CALL(float, float);
#undef CALL
  return DIF_OK;
}

inline int64_t low_width(int32_t rank) { return round_up(rank, 8); }

// Parts of low that the workspace holds: few rows split the reduction
// (gemm_batch.hip; at most 32 MiB of it).
inline int low_max_parts(int32_t M) { return M <= 128 ? 16 : M <= 512 ? 8 : M <= 2048 ? 4 : 1; }

// Rows of low, all parts together, of the largest of all batches of up to M rows
// (the most rows of each number of parts among them): a workspace serves every
// batch smaller than its own.
inline int64_t low_rows(int32_t M) {
  int64_t rows = 0;
  for (const int32_t m : {std::min(M, 128), std::min(M, 512), std::min(M, 2048), M})
    rows = std::max(rows, (int64_t)m * low_max_parts(m));
  return rows;
}

}  // namespace

extern "C" {

dif_status dif_gemm_grouped(int32_t dtype, int32_t out_dtype, const void* A, int64_t lda, const void* B,
                            int64_t ldb, void* C, int64_t ldc, int32_t M, int32_t N, int32_t K,
                            int32_t epilogue, const float* bias, const float* gate0, const float* gate1,
                            const dif_groups* groups, dif_stream stream) {
  GUARD_BEGIN
  const Product p{dtype, out_dtype, A, lda, B, ldb, C, ldc, M, N, K, epilogue, bias, gate0, gate1};
  DIF_TRY(check_product(p));
  DIF_TRY(check_groups(groups));
  if (M == 0 || N == 0) return DIF_OK;
  DIF_TRY(check_operands(p, groups->n_weights, groups->b_stride));
  DIF_TRY(check_extent(M, N, groups->n_groups));
  const BatchGroups g = to_groups(*groups);
  return run(p, &g, nullptr, reinterpret_cast<hipStream_t>(stream));
  GUARD_END
}

dif_status dif_lora_workspace_bytes(int32_t M, int32_t rank, size_t* bytes) {
  GUARD_BEGIN
  if (!bytes) return fail(DIF_E_ARG, "null output");
  if (M < 0) return fail(DIF_E_SHAPE, "negative size");
  if (rank < 1 || rank > DIF_MAX_RANK) return fail(DIF_E_SHAPE, "rank %d outside 1 .. %d", rank, DIF_MAX_RANK);
  *bytes = align256((size_t)low_rows(M) * low_width(rank) * sizeof(float));
  return DIF_OK;
  GUARD_END
}

dif_status dif_gemm_lora(int32_t dtype, int32_t out_dtype, const void* A, int64_t lda, const void* B, int64_t ldb,
                         void* C, int64_t ldc, int32_t M, int32_t N, int32_t K, int32_t epilogue,
                         const float* bias, const float* gate0, const float* gate1, const dif_groups* groups,
                         const dif_lora* lora, void* ws, size_t ws_bytes, dif_stream stream) {
  GUARD_BEGIN
  const Product p{dtype, out_dtype, A, lda, B, ldb, C, ldc, M, N, K, epilogue, bias, gate0, gate1};
  DIF_TRY(check_product(p));
  if (groups) {
    DIF_TRY(check_groups(groups));
    if (groups->k_kept) return fail(DIF_E_UNSUPPORTED, "adapters beside groups of their own reduction widths");
  }
  if (!lora) return fail(DIF_E_ARG, "lora is null");
  if (lora->n_requests < 1 || lora->n_requests > DIF_MAX_GROUPS)
    return fail(DIF_E_SHAPE, "n_requests %d outside 1 .. %d", lora->n_requests, DIF_MAX_GROUPS);
  if (lora->n_adapters < 0) return fail(DIF_E_SHAPE, "n_adapters < 0");
  size_t need = 0;
  DIF_TRY(dif_lora_workspace_bytes(M, lora->rank, &need));
  if (!lora->row_offsets || !lora->adapter) return fail(DIF_E_ARG, "row_offsets or adapter is null");
  if (misaligned(lora->row_offsets, 4) || misaligned(lora->adapter, 4) || misaligned(lora->ranks, 4) ||
      misaligned(lora->scales, 4))
    return fail(DIF_E_ARG, "tables must be 4-byte aligned");
  if (M == 0 || N == 0) return DIF_OK;
  DIF_TRY(check_operands(p, groups ? groups->n_weights : 1, groups ? groups->b_stride : 0));
  DIF_TRY(check_extent(M, std::max(N, lora->rank), std::max(groups ? groups->n_groups : 1, lora->n_requests)));
  const int64_t es = esize(dtype);
  if (lora->n_adapters > 0 && K > 0) {
    DIF_TRY(check_rows("down", lora->down, lora->ld_down, K, es, lora->n_adapters, lora->down_stride));
    DIF_TRY(check_rows("up", lora->up, lora->ld_up, lora->rank, es, lora->n_adapters, lora->up_stride));
    if (!ws || misaligned(ws, 256) || ws_bytes < need)
      return fail(DIF_E_WORKSPACE, "workspace must be 256-byte aligned and hold %zu bytes", need);
  }
  BatchLora l{};
  l.off = lora->row_offsets;
  l.adapter = lora->adapter;
  l.n_requests = lora->n_requests;
  l.n_adapters = lora->n_adapters;
  l.rank = lora->rank;
  l.ranks = lora->ranks;
  l.scales = lora->scales;
  l.down = lora->down;
  l.ld_down = lora->ld_down;
  l.down_stride = lora->down_stride;
  l.up = lora->up;
  l.ld_up = lora->ld_up;
  l.up_stride = lora->up_stride;
  l.low = static_cast<float*>(ws);
  l.ld_low = (int)low_width(lora->rank);
  l.max_parts = low_max_parts(M);
  BatchGroups g;
  if (groups) g = to_groups(*groups);
  return run(p, groups ? &g : nullptr, &l, reinterpret_cast<hipStream_t>(stream));
  GUARD_END
}

}  // extern "C"
