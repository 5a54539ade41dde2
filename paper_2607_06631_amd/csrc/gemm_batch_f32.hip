// gemm_ring.h over mixed batches for (operand, output) types float, float.
#include "gemm_ring.h"

namespace dif {
DIF_BATCH_INSTANCE(float, float)
}  // namespace dif
