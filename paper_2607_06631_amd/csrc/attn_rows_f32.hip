// attn_rows.h for float.
#include "attn_rows.h"

namespace dif {
DIF_ROWS_INSTANCE(float)
}  // namespace dif
