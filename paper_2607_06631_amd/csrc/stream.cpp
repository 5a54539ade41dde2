// C ABI of streamed generation: appending to a paged cache, attention of new tokens
// over it and over packed sequences.  Host side only: argument checks and the launches
// (append.hip, attn_rows.h).
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "host.h"
#include "kernels.h"

using namespace dif;

namespace {

// the kernels round a sequence's keys up to whole tiles in 32 bits
constexpr int64_t kMostKeys = INT32_MAX - 65535;

inline bool misaligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

dif_status check_types(int32_t dtype, int32_t head_dim) {
  if (dtype != DIF_BF16 && dtype != DIF_F32) return fail(DIF_E_ARG, "bad dtype");
  if (head_dim != 64 && head_dim != 128) return fail(DIF_E_UNSUPPORTED, "head_dim %d is not 64 or 128", head_dim);
  return DIF_OK;
}

// `heads` heads beside each other in rows `ld` elements apart.
dif_status check_rows(const char* name, const void* p, int64_t ld, int64_t heads, int64_t head_dim, int64_t es) {
  if (!p) return fail(DIF_E_ARG, "%s is null", name);
  if (misaligned(p, 16)) return fail(DIF_E_ARG, "%s must be 16-byte aligned", name);
  if (ld < heads * head_dim) return fail(DIF_E_SHAPE, "%s: row stride %lld below the width", name, (long long)ld);
  if (ld * es % 16) return fail(DIF_E_SHAPE, "%s: row stride must be a multiple of 16 bytes", name);
  if (ld >= (int64_t(1) << 24)) return fail(DIF_E_SHAPE, "%s: row stride of 2^24 elements or more", name);
  return DIF_OK;
}

dif_status check_stride(const char* name, int64_t stride, int64_t least, int64_t es) {
  if (stride < least || stride > (int64_t(1) << 40) || stride * es % 16)
    return fail(DIF_E_SHAPE, "cache: %s stride must be >= %lld and a multiple of 16 bytes", name, (long long)least);
  return DIF_OK;
}

dif_status check_seqs(int64_t n_seqs, const int32_t* row_offsets) {
  if (n_seqs < 1 || n_seqs > DIF_MAX_GROUPS)
    return fail(DIF_E_SHAPE, "n_seqs %lld outside 1 .. %d", (long long)n_seqs, DIF_MAX_GROUPS);
  if (!row_offsets || misaligned(row_offsets, 4)) return fail(DIF_E_ARG, "row_offsets is null or misaligned");
  return DIF_OK;
}

dif_status to_view(const dif_kv_cache* c, int32_t dtype, int32_t rows, KeyView* kv) {
  if (!c) return fail(DIF_E_ARG, "cache is null");
  DIF_TRY(check_types(dtype, c->head_dim));
  const int64_t es = esize(dtype);
  if (rows < 0) return fail(DIF_E_SHAPE, "negative size");
  DIF_TRY(check_seqs(c->n_seqs, c->row_offsets));
  if (c->n_pages < 1 || c->max_pages < 1 || c->n_kv_heads < 1)
    return fail(DIF_E_SHAPE, "n_pages, max_pages and n_kv_heads must be >= 1");
  if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)))
    return fail(DIF_E_SHAPE, "page_size %d is not a power of two from 16 to 65536", c->page_size);
  if ((int64_t)c->max_pages * c->page_size > kMostKeys)
    return fail(DIF_E_SHAPE, "max_pages pages hold more than %lld tokens", (long long)kMostKeys);
  if (c->ld_table < c->max_pages || c->ld_table > (int64_t(1) << 40)) return fail(DIF_E_SHAPE, "ld_table < max_pages");
  if (!c->k || !c->v || misaligned(c->k, 16) || misaligned(c->v, 16))
    return fail(DIF_E_ARG, "the cache's k and v must be 16-byte aligned, not null");
  if (!c->table || !c->lengths || misaligned(c->table, 4) || misaligned(c->lengths, 4))
    return fail(DIF_E_ARG, "table or lengths is null or misaligned");
  DIF_TRY(check_stride("page", c->page_stride, 0, es));
  DIF_TRY(check_stride("head", c->head_stride, c->n_kv_heads > 1 ? c->head_dim : 0, es));
  DIF_TRY(check_stride("slot", c->slot_stride, c->head_dim, es));
  // (the kernels address within a page, and runs of 32 tokens, through 32-bit offsets)
  if (c->slot_stride >= (int64_t(1) << 24) || c->page_size * c->slot_stride * es >= (int64_t(1) << 31))
    return fail(DIF_E_SHAPE, "cache: a slot stride of 2^24 elements, or a page's tokens spanning 2 GiB");
  if (c->page_stride * es >= (int64_t(1) << 32)) return fail(DIF_E_SHAPE, "cache: pages 4 GiB or more apart");
  *kv = KeyView{};
  kv->k = c->k;
  kv->v = c->v;
  kv->page_stride = c->page_stride;
  kv->k_head = kv->v_head = c->head_stride;
  kv->k_slot = kv->v_slot = c->slot_stride;
  kv->table = c->table;
  kv->ld_table = c->ld_table;
  kv->lengths = c->lengths;
  kv->row_off = c->row_offsets;
  kv->n_seqs = c->n_seqs;
  kv->rows = rows;
  kv->kv_heads = c->n_kv_heads;
  kv->max_keys = c->max_pages * c->page_size;
  kv->n_pages = c->n_pages;
  kv->page_shift = __builtin_ctz((unsigned)c->page_size);
  return DIF_OK;
}

dif_status check_heads(int32_t heads, int32_t kv_heads) {
  if (heads < 1 || kv_heads < 1 || heads % kv_heads)
    return fail(DIF_E_SHAPE, "%d query heads are no multiple of %d key heads", heads, kv_heads);
  return DIF_OK;
}

// The mask, the output and the launch that both attention calls share.
dif_status attend(int32_t dtype, int32_t head_dim, int32_t flags, const KeyView& kv, const void* q, int64_t ldq,
                  void* out, int64_t ldo, int32_t heads, const dif_seen* seen, void* ws, size_t ws_bytes,
                  hipStream_t s) {
  const int64_t es = esize(dtype);
  if (flags & ~DIF_ATTN_Q_PRESCALED) return fail(DIF_E_ARG, "unknown flags");
  if (!seen) return fail(DIF_E_ARG, "seen is null");
  if (seen->block < 0 || seen->window < 0 || seen->sinks < 0)
    return fail(DIF_E_SHAPE, "block, window and sinks must be >= 0");
  if (seen->sinks > 0 && seen->window == 0) return fail(DIF_E_ARG, "sinks belong to a window");
  DIF_TRY(check_heads(heads, kv.kv_heads));
  if (ws && (misaligned(ws, 256) || ws_bytes < attention_rows_bytes(head_dim)))
    return fail(DIF_E_WORKSPACE, "workspace must be 256-byte aligned and hold %zu bytes", attention_rows_bytes(head_dim));
  if (kv.rows == 0) return DIF_OK;
  DIF_TRY(check_rows("q", q, ldq, heads, head_dim, es));
  DIF_TRY(check_rows("out", out, ldo, heads, head_dim, es));
  // rows times shared heads are counted in 32 bits, a launch's threads too
  if ((int64_t)kv.rows * (heads / kv.kv_heads) > INT32_MAX - 65536 ||
      rows_items(kv.rows, heads, kv.kv_heads, kv.n_seqs, 16) > kMostTiles)
    return fail(DIF_E_SHAPE, "problem too large: split the sequences over several calls");
  // (lengths are in device memory: booked as if every row saw all keys there may be)
  const double keys = kv.max_keys, m = kv.rows;
  const ProfScope prof(PK_ATTN_SELF, s, 4.0 * head_dim * heads * m * keys,
                       2.0 * es * head_dim * (m * heads + keys * kv.kv_heads * (kv.table ? kv.n_seqs : 1)));
  const SeenMask mask{seen->block, seen->window, seen->sinks};
  const bool scaled = flags & DIF_ATTN_Q_PRESCALED;
  float* part = static_cast<float*>(ws);
  if (dtype == DIF_BF16)
    HIP_TRY(launch_attention_rows<bf16>(kv, head_dim, (const bf16*)q, ldq, (bf16*)out, ldo, heads, mask, scaled, part, s));
  else
    HIP_TRY(launch_attention_rows<float>(kv, head_dim, (const float*)q, ldq, (float*)out, ldo, heads, mask, scaled, part, s));
  return DIF_OK;
}

}  // namespace

extern "C" {

dif_status dif_cache_append(int32_t dtype, const dif_kv_cache* cache, const void* k, int64_t ldk, const void* v,
                            int64_t ldv, const void* q, int64_t ldq, void* q_out, int64_t ldqo, int32_t M,
                            int32_t n_heads, const dif_append* how, dif_stream stream) {
  GUARD_BEGIN
  KeyView kv;
  DIF_TRY(to_view(cache, dtype, M, &kv));
  if (!how) return fail(DIF_E_ARG, "how is null");
  const int64_t es = esize(dtype), dh = cache->head_dim;
  if (q) DIF_TRY(check_heads(n_heads, kv.kv_heads));
  if (!q && (q_out || how->gain_q)) return fail(DIF_E_ARG, "q_out or gain_q without q");
  if (how->axes != 0 && how->axes != 1 && how->axes != 3) return fail(DIF_E_ARG, "axes %d is not 0, 1 or 3", how->axes);
  if (how->axes > 0 && !(how->theta > 0.f && std::isfinite(how->theta))) return fail(DIF_E_ARG, "theta must be > 0");
  if (how->axes == 3 && !how->positions) return fail(DIF_E_ARG, "three axes need positions");
  if (how->axes == 0 && how->positions) return fail(DIF_E_ARG, "positions without a rotation");
  if (how->gain_k || how->gain_q) {
    if (!(how->eps > 0.f)) return fail(DIF_E_ARG, "eps must be > 0");
    if (how->norm_dim < 0) return fail(DIF_E_SHAPE, "norm_dim < 0");
    const int64_t most = dtype == DIF_BF16 ? kMostNormed<bf16> : kMostNormed<float>;
    if ((how->gain_k && kv.kv_heads * dh > most) || (how->gain_q && n_heads * dh > most))
      return fail(DIF_E_SHAPE, "normalised rows are at most %lld wide", (long long)most);
  }
  if (misaligned(how->gain_k, 16) || misaligned(how->gain_q, 16) || misaligned(how->positions, 4))
    return fail(DIF_E_ARG, "gains must be 16-byte aligned, positions 4-byte");
  if (M == 0) return DIF_OK;
  DIF_TRY(check_rows("k", k, ldk, kv.kv_heads, dh, es));
  DIF_TRY(check_rows("v", v, ldv, kv.kv_heads, dh, es));
  if (q) {
    DIF_TRY(check_rows("q", q, ldq, n_heads, dh, es));
    DIF_TRY(check_rows("q_out", q_out, ldqo, n_heads, dh, es));
  }
  // (a launch counts its threads in 32 bits)
  if (M > (int32_t)(kMostTiles * 4 / 3)) return fail(DIF_E_SHAPE, "too many rows: split them over several calls");
  AppendDesc d{};
  d.gain_q = how->gain_q;
  d.gain_k = how->gain_k;
  const int64_t nd = how->norm_dim;
  d.inv_dim_k = 1.f / (float)(nd ? nd : kv.kv_heads * dh);
  d.inv_dim_q = q ? 1.f / (float)(nd ? nd : n_heads * dh) : 0.f;
  d.eps = how->eps;
  d.q_scale = how->q_scale;
  d.positions = how->positions;
  d.axes = how->axes;
  const int per = how->axes == 3 ? (int)(dh / 6) : 0;   // pairs of the second and of the third axis
  const int pairs[3] = {(int)dh / 2 - 2 * per, per, per};
  d.axis1 = pairs[0];
  d.axis2 = pairs[0] + per;
  if (how->axes > 0) {
    // turns per position, theta^(-j / pairs) / 2 pi, as fractions of 2^64 (whole turns left
    // out), by repeated multiplication: off by at most 64 roundings of 2^-64
    int at = 0;
    for (const int n : pairs) {
      if (n == 0) continue;
      const long double step = std::pow((long double)how->theta, -1.0L / n);
      if (step < 1.0L) {   // (in whole numbers: 64 multiplications in long double took 2 us of a call's 12)
        const uint64_t by = (uint64_t)(step * 18446744073709551616.0L);
        uint64_t f = 2935890503282001226u;   // 2^64 / 2 pi
        for (int j = 0; j < n; ++j, f = (uint64_t)(((unsigned __int128)f * by) >> 64)) d.freq[at++] = f;
      } else {
        long double f = 0.159154943091895335768883763372514362L;
        for (int j = 0; j < n; ++j, f *= step) d.freq[at++] = (uint64_t)((f - std::floor(f)) * 18446744073709551616.0L);
      }
    }
  }
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const double wide = (double)dh * (2.0 * kv.kv_heads + (q ? n_heads : 0));
  const ProfScope prof(PK_QK_NORM, s, 0.0, 2.0 * es * M * wide);
#define CALL(T)                                                                                                    \
  HIP_TRY((launch_append<T>(kv, (int)dh, (const T*)k, ldk, (const T*)v, ldv, (const T*)q, ldq, (T*)q_out, ldqo,    \
                            n_heads, d, s)))
  if (dtype == DIF_BF16) CALL(bf16);
  else CALL(float);
#undef CALL
  return DIF_OK;
  GUARD_END
}

dif_status dif_attention_paged_bytes(int32_t head_dim, size_t* bytes) {
  GUARD_BEGIN
  if (!bytes) return fail(DIF_E_ARG, "null output");
  if (head_dim != 64 && head_dim != 128) return fail(DIF_E_UNSUPPORTED, "head_dim %d is not 64 or 128", head_dim);
  *bytes = attention_rows_bytes(head_dim);
  return DIF_OK;
  GUARD_END
}

dif_status dif_attention_paged(int32_t dtype, int32_t flags, const void* q, int64_t ldq, const dif_kv_cache* cache,
                               void* out, int64_t ldo, int32_t M, int32_t n_heads, const dif_seen* seen, void* ws,
                               size_t ws_bytes, dif_stream stream) {
  GUARD_BEGIN
  KeyView kv;
  DIF_TRY(to_view(cache, dtype, M, &kv));
  return attend(dtype, cache->head_dim, flags, kv, q, ldq, out, ldo, n_heads, seen, ws, ws_bytes,
                reinterpret_cast<hipStream_t>(stream));
  GUARD_END
}

dif_status dif_attention_window(int32_t dtype, int32_t head_dim, int32_t flags, const void* q, int64_t ldq,
                                const void* k, int64_t ldk, const void* v, int64_t ldv, void* out, int64_t ldo,
                                int32_t M, int32_t N, int32_t n_heads, int32_t n_kv_heads, int32_t n_seqs,
                                const int32_t* row_offsets, const int32_t* key_offsets, const dif_seen* seen, void* ws,
                                size_t ws_bytes, dif_stream stream) {
  GUARD_BEGIN
  DIF_TRY(check_types(dtype, head_dim));
  if (M < 0 || N < 0) return fail(DIF_E_SHAPE, "negative size");
  if (N > kMostKeys) return fail(DIF_E_SHAPE, "more than %lld keys", (long long)kMostKeys);
  DIF_TRY(check_seqs(n_seqs, row_offsets));
  if (!key_offsets && N != M) return fail(DIF_E_SHAPE, "%d rows and %d keys need key_offsets", M, N);
  if (misaligned(key_offsets, 4)) return fail(DIF_E_ARG, "key_offsets is misaligned");
  DIF_TRY(check_heads(n_heads, n_kv_heads));
  const int64_t es = esize(dtype);
  if (M > 0 && N > 0) {
    DIF_TRY(check_rows("k", k, ldk, n_kv_heads, head_dim, es));
    DIF_TRY(check_rows("v", v, ldv, n_kv_heads, head_dim, es));
  }
  KeyView kv{};
  kv.k = const_cast<void*>(k);
  kv.v = const_cast<void*>(v);
  kv.k_head = kv.v_head = head_dim;
  kv.k_slot = ldk;
  kv.v_slot = ldv;
  kv.row_off = row_offsets;
  kv.key_off = key_offsets ? key_offsets : row_offsets;
  kv.n_seqs = n_seqs;
  kv.rows = M;
  kv.kv_heads = n_kv_heads;
  kv.max_keys = N;
  return attend(dtype, head_dim, flags, kv, q, ldq, out, ldo, n_heads, seen, ws, ws_bytes,
                reinterpret_cast<hipStream_t>(stream));
  GUARD_END
}

}  // extern "C"
