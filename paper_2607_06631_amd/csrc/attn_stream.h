// Which kernel attends, and whether key ranges may be split (attn_rows.h, attn_tokens.h).
#pragma once
#include <cmath>

#include "attn_rows.h"
#include "attn_tokens.h"
#include "attn_wide.h"

namespace dif {

template <typename T>
hipError_t launch_attention_rows(const KeyView& kv, int head_dim, const T* q, int64_t ldq, T* out, int64_t ldo,
                                 int heads, const SeenMask& mask, bool q_scaled, float* part, hipStream_t stream) {
  RowsParams<T> p{kv, q, out, ldq, ldo, heads, heads / kv.kv_heads, mask,
                  q_scaled ? 1.f : (float)(1.4426950408889634 / std::sqrt((double)head_dim)), part};
  // rows of a sequence, on average, with the heads that share a key head
  const int64_t rows = (int64_t)kv.rows * p.group;
  const bool tokens = rows <= (int64_t)kTokensTile * kv.n_seqs;
  // (a wide tile at least half full on average)
  const bool wide = sizeof(T) == 2 && head_dim == 128 && !tokens && rows >= (int64_t)(kWideTile / 2) * kv.n_seqs;
  const SplitRule& rule = tokens ? kTokensRule : wide ? kWideRule : kRowsRule;
  const int bmq = tokens ? kTokensTile : wide ? kWideTile : kRowsTile, bn = tokens || sizeof(T) == 4 ? 32 : 64;
  // nothing to split: so many items whatever the sequences, or so few keys
  const int most = tokens ? kTokensShort : 2 * rule.least * bn;
  if ((rows + bmq - 1) / bmq * kv.kv_heads >= 2 * rule.slots || kv.max_keys <= most) p.part = nullptr;
  hipError_t e;
  if (tokens) {
    e = launch_tokens<T>(p, head_dim, stream);
  } else if constexpr (sizeof(T) == 2) {
    e = wide ? launch_wide(p, stream) : launch_rows<T>(p, head_dim, stream);
  } else {
    e = launch_rows<T>(p, head_dim, stream);
  }
  if (e != hipSuccess || !p.part) return e;
  if (tokens) return launch_join<T, kTokensTile>(p, head_dim, rule, stream);
  if constexpr (sizeof(T) == 2) {
    if (wide) return launch_join<T, kWideTile>(p, head_dim, rule, stream);
  }
  return launch_join<T, kRowsTile>(p, head_dim, rule, stream);
}

#define DIF_STREAM_INSTANCE(T)                                                                                   \
  template hipError_t launch_attention_rows<T>(const KeyView&, int, const T*, int64_t, T*, int64_t, int,        \
                                               const SeenMask&, bool, float*, hipStream_t);

}  // namespace dif
