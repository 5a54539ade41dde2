// attn_stream.h for float32.
#include "attn_stream.h"

namespace dif {
DIF_STREAM_INSTANCE(float)
}  // namespace dif
