// attn_stream.h for bf16.
#include "attn_stream.h"

namespace dif {
DIF_STREAM_INSTANCE(bf16)

size_t attention_rows_bytes(int head_dim) {
  const size_t rows = (size_t)kRowsRule.limit * kRowsTile, tokens = (size_t)kTokensRule.limit * kTokensTile;
  const size_t wide = (size_t)kWideRule.limit * kWideTile;
  return (kNoteFloats + std::max({rows, tokens, wide}) * (head_dim + 2)) * sizeof(float);
}
}  // namespace dif
