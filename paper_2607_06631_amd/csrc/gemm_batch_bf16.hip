// gemm_ring.h over mixed batches for (operand, output) types bf16, bf16.
#include "gemm_ring.h"

namespace dif {
DIF_BATCH_INSTANCE(bf16, bf16)
}  // namespace dif
