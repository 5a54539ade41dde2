// gemm_ring.h over mixed batches for (operand, output) types bf16, float.
#include "gemm_ring.h"

namespace dif {
DIF_BATCH_INSTANCE(bf16, float)
}  // namespace dif
