// Which kernel attends, and whether key ranges may be split (attn_rows.h, attn_tokens.h).
#pragma once
#include <cmath>

#include "attn_rows.h"
#include "attn_tokens.h"
#include "attn_wide.h"

namespace dif {

enum RowsKernel { ROWS_TOKENS, ROWS_CHUNKS, ROWS_WIDE };

template <typename T>
hipError_t launch_kind(RowsParams<T> p, int head_dim, RowsKernel kind, hipStream_t stream) {
  const KeyView& kv = p.kv;
  const int64_t rows = (int64_t)kv.rows * p.group;
  const SplitRule rule = kind == ROWS_TOKENS ? kTokensRule : kind == ROWS_WIDE ? kWideRule : kRowsRule;
  const int bmq = kind == ROWS_TOKENS ? kTokensTile : kind == ROWS_WIDE ? kWideTile : kRowsTile;
  const int bn = kind == ROWS_TOKENS || sizeof(T) == 4 ? 32 : 64;
  // nothing to split: so many items whatever the sequences, or so few keys
  const int most = kind == ROWS_TOKENS ? kTokensShort : 2 * rule.least * bn;
  if ((kv.least_rows <= 1 && kv.most_rows >= kv.rows && (rows + bmq - 1) / bmq * kv.kv_heads >= 2 * rule.slots) ||
      kv.max_keys <= most)
    p.part = nullptr;
  hipError_t e;
  if (kind == ROWS_TOKENS) {
    e = launch_tokens<T>(p, head_dim, stream);
  } else if constexpr (sizeof(T) == 2) {
    e = kind == ROWS_WIDE ? launch_wide(p, stream) : launch_rows<T>(p, head_dim, stream);
  } else {
    e = launch_rows<T>(p, head_dim, stream);
  }
  if (e != hipSuccess || !p.part) return e;
  if (kind == ROWS_TOKENS) return launch_join<T, kTokensTile>(p, head_dim, rule, stream);
  if constexpr (sizeof(T) == 2) {
    if (kind == ROWS_WIDE) return launch_join<T, kWideTile>(p, head_dim, rule, stream);
  }
  return launch_join<T, kRowsTile>(p, head_dim, rule, stream);
}

template <typename T>
hipError_t launch_attention_rows(const KeyView& kv, int head_dim, const T* q, int64_t ldq, T* out, int64_t ldo,
                                 int heads, const SeenMask& mask, bool q_scaled, float* part, hipStream_t stream) {
  RowsParams<T> p{kv, q, out, ldq, ldo, heads, heads / kv.kv_heads, mask,
                  q_scaled ? 1.f : (float)(1.4426950408889634 / std::sqrt((double)head_dim)), part};
  // Rows of a sequence, on average, with the heads that share a key head: up to 16 take the
  // single tokens' kernel, a wide tile at least half full the wide one (bf16, heads of
  // 128), the rest the other.  Where the average is low because some sequences
  // have a chunk and many a token or none (more rows than sequences), those of more than
  // four of its tiles have a launch of their own: the single tokens' kernel reads the cache once per 16 rows.
  const int64_t rows = (int64_t)kv.rows * p.group;
  // (the wide kernel's code is long, and short caches end before it has paid: 16 heads of 2048 causal
  // tokens take 71 us without it, 82 with it, of 4096 152 and 140.  Windows shorter than the blocks
  // over pages leave it few tiles that all its rows see: 2000 rows over 8000 keys, 12 heads, blocks of
  // 1000 and windows of 700 take 134 us without it, 172 with it)
  const bool wide = sizeof(T) == 2 && head_dim == 128 && kv.max_keys > 2048 && !(kv.table && mask.gaps());
  if (rows > (int64_t)kTokensTile * kv.n_seqs) {
    return launch_kind<T>(p, head_dim, wide && rows >= (int64_t)(kWideTile / 2) * kv.n_seqs ? ROWS_WIDE : ROWS_CHUNKS,
                          stream);
  }
  const int most = 4 * kTokensTile / p.group;
  if (kv.rows <= kv.n_seqs || kv.rows <= most) return launch_kind<T>(p, head_dim, ROWS_TOKENS, stream);
  p.kv.most_rows = most;
  const hipError_t e = launch_kind<T>(p, head_dim, ROWS_TOKENS, stream);
  if (e != hipSuccess) return e;
  p.kv.least_rows = most + 1;
  p.kv.most_rows = 0x7fffffff;
  return launch_kind<T>(p, head_dim, wide ? ROWS_WIDE : ROWS_CHUNKS, stream);
}

#define DIF_STREAM_INSTANCE(T)                                                                                   \
  template hipError_t launch_attention_rows<T>(const KeyView&, int, const T*, int64_t, T*, int64_t, int,        \
                                               const SeenMask&, bool, float*, hipStream_t);

}  // namespace dif
