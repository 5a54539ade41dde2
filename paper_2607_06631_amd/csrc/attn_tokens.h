// Attention of single tokens (few rows of a sequence, up to 16 with the heads that
// share a key head) over long caches: bound by reading the keys and values once.
//
// A workgroup takes the rows of one sequence and key head and a range of its keys; its
// waves walk tiles of 32 keys in turn, each with its own running maximum and
// sum, and join at the end.  Operands go from memory to registers in the MFMAs'
// layout, so no tile passes through LDS and no wave waits for another:
//   S^T = K Q^T      16x16 tiles, rows keys, columns the 16 rows.  A lane reads 16-byte
//                    pieces of its key's row; the order of dims is the same on both
//                    sides and nothing else.
//   O^T += V^T P^T   The keys of an S^T column lie in a lane's registers as the B operand
//                    wants them.  For V^T a lane reads the same few dims of eight keys (a
//                    wave whole rows) and bf16 pairs are swapped between registers
//                    (v_perm_b32), 32 of them for 32 keys.
// K's registers are loaded again as soon as the scores are taken, V's as soon as the
// products are, so loads are in flight all the time: 16 KB a wave, 8 waves a CU.
// Masks as in attn_rows.h.
#pragma once
#include <algorithm>
#include <type_traits>

#include "stream.h"

namespace dif {

// The MFMA steps of the two types on 16x16 tiles.
template <typename T> struct Tok;
template <> struct Tok<bf16> {
  // key (of 32) in row r of S^T tile a: its register e of lane group g is key 8 g + 4 a + e
  __device__ static constexpr int key(int a, int r) { return 8 * (r >> 2) + 4 * a + (r & 3); }
  __device__ static void step(f32x4& acc, const u32x4& a, const u32x4& b) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0,
                                                  0, 0);
  }
};
template <> struct Tok<float> {
  __device__ static constexpr int key(int a, int r) { return 16 * a + r; }
  __device__ static void step(f32x4& acc, const u32x4& a, const u32x4& b) {
    const f32x4 fa = __builtin_bit_cast(f32x4, a), fb = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fb[e], acc, 0, 0, 0);
  }
};

// NW waves: four, two workgroups a CU, or eight for short caches, whose few tiles are then
// a shorter chain (257 keys, float32: 10.3 against 11.7 us; 64 sequences of 16 to 16384
// keys took 202 against 136 us with eight).
// GAP: windows shorter than the blocks over pages, in an instance of its own (in all of them it
// cost 3 to 6 % for float32 heads of 128).
template <typename T, int DH, bool PAGED, int NW, bool GAP>
__global__ __launch_bounds__(64 * NW, 2) void attn_tokens_kernel(RowsParams<T> p) {
  constexpr int BMQ = kTokensTile, BN = 32;
  constexpr int ES = (int)sizeof(T), VEC = 16 / ES;
  constexpr int NST = DH / VEC / 4;        // pieces of a key's row in a lane
  constexpr int VB = DH / 16;              // dims of V in a lane, NV of them each turn
  constexpr int NVD = VB * ES / 4;         // dwords of one key's dims in a lane: 4 or 2 (bf16), 8 or 4 (float32)
  __shared__ float sums[NW][BMQ][DH];
  __shared__ float stats[NW][BMQ][2];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 4, col = lane & 15;
  const KeyView& kv = p.kv;

  Sequences seqs;
  const Plan plan = make_plan<BN>(kv, p.mask, p.group, BMQ, p.part != nullptr, kTokensRule, &seqs);
  leave_plan(p.part, plan);
  const int64_t all = (int64_t)plan.pieces * kv.kv_heads;
  if ((int64_t)blockIdx.x >= all) return;
  const int idx = blockIdx.x;
  const int i = idx / kv.kv_heads, h = idx - i * kv.kv_heads;   // heads beside each other in memory run together
  const Place at = find_place<BN>(kv, p.mask, p.group, BMQ, plan, seqs, i);
  const int slot = h * plan.pieces + i;
  const int s = at.seq;
  const Sequence sq = at.sq;
  const int nrows = sq.rows * p.group;
  const int r0 = (((nrows + BMQ - 1) / BMQ) - 1 - at.tile) * BMQ;
  leave_note(p.part, plan, at, slot, r0, nrows);
  if (r0 < 0 || r0 >= nrows) return;   // (offsets that are not ascending)
  const int shift = sq.keys - sq.rows;
  const int rlast = min(r0 + BMQ, nrows) - 1;
  const Seen first = seen_by(p.mask, shift + r0 / p.group, sq.keys);
  const Seen last = seen_by(p.mask, shift + rlast / p.group, sq.keys);
  const Extent<BN, GAP> ex = extent<BN, GAP>(p.mask, shift + r0 / p.group, shift + rlast / p.group, sq.keys);
  const int hi = ex.hi, sinks = ex.sinks;
  const int t0 = (int)((int64_t)ex.ntiles * at.part / at.parts);
  const int t1 = (int)((int64_t)ex.ntiles * (at.part + 1) / at.parts);

  const int row = min(r0 + col, nrows - 1);
  const int token = row / p.group, head = h * p.group + row - token * p.group;
  const Seen mine = seen_by(p.mask, shift + token, sq.keys);
  u32x4 qf[NST];
  {
    const T* qr = p.q + (int64_t)(sq.row0 + token) * p.ldq + head * DH;
#pragma unroll
    for (int st = 0; st < NST; ++st) qf[st] = *reinterpret_cast<const u32x4*>(qr + (4 * st + g) * VEC);
  }

  const char* kbase = reinterpret_cast<const char*>(static_cast<const T*>(kv.k) + h * kv.k_head);
  const char* vbase = reinterpret_cast<const char*>(static_cast<const T*>(kv.v) + h * kv.v_head);
  typedef const __attribute__((address_space(4))) int32_t* table_t;
  [[maybe_unused]] const table_t table = (table_t)(uintptr_t)(kv.table + s * kv.ld_table);

  // Places of a tile's keys: one run of 32 in one page, or two of 16.  Keys that no row sees
  // are read from the place of one in the tile that is seen.
  struct Where {
    int64_t k[2], v[2];   // bytes to the first key of each run
    int tile;             // absolute
    bool whole;           // every key is seen by some row
    uint32_t seen;        // (GAP) a bit for each key that is; none: the first run begins at a key before the tile
  };
  auto offset = [&](uint32_t page, int key, int64_t slot_stride) __attribute__((always_inline)) {
    if constexpr (PAGED)
      return ((int64_t)min(page, (uint32_t)kv.n_pages - 1) * kv.page_stride +
              (int64_t)(key & ((1 << kv.page_shift) - 1)) * slot_stride) * ES;
    else
      return (int64_t)(sq.key0 + key) * slot_stride * ES;
  };
  auto locate = [&](int t) __attribute__((always_inline)) {
    Where w;
    w.tile = ex.tile(t);
    const int k0 = w.tile * BN;
    w.whole = ex.whole(w.tile);
    int from = k0;
    if constexpr (GAP) {
      w.seen = __builtin_amdgcn_readfirstlane((uint32_t)__ballot(ex.sees(k0 + (lane & 31))));
      if (w.seen == 0) from = __builtin_amdgcn_readfirstlane(ex.before(w.tile));
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      // (a run without a seen key is not read; its page may lie behind the table)
      const int k = from + 16 * r;
      uint32_t page = 0;
      if constexpr (PAGED) page = (uint32_t)table[min(k, hi - 1) >> kv.page_shift];
      w.k[r] = offset(page, k, kv.k_slot);
      w.v[r] = offset(page, k, kv.v_slot);
    }
    return w;
  };
  // key `key` of the tile, or one that is seen
  auto seen_key = [&](const Where& w, int key) __attribute__((always_inline)) {
    if constexpr (GAP) return w.seen >> key & 1 ? key : w.seen ? __builtin_ctz(w.seen) : 0;
    const int k0 = w.tile * BN;
    if (w.tile < ex.w0) return min(key, sinks - 1 - k0);
    if (key >= sinks - k0) key = max(key, ex.lo - k0);
    return min(key, hi - 1 - k0);
  };
  u32x4 kf[2][NST];
  uint32_t vr[8][NVD];
  auto load_k = [&](const Where& w) __attribute__((always_inline)) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      int key = Tok<T>::key(a, col);
      if (!w.whole) key = seen_key(w, key);
      const char* at_row = kbase + (key >= 16 ? w.k[1] : w.k[0]) + (int64_t)(key & 15) * kv.k_slot * ES;
#pragma unroll
      for (int st = 0; st < NST; ++st) kf[a][st] = *reinterpret_cast<const u32x4*>(at_row + 16 * (4 * st + g));
    }
  };
  auto load_v = [&](const Where& w) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      int key = Tok<T>::key(e >> 2, 4 * g + (e & 3));
      if (!w.whole) key = seen_key(w, key);
      const char* at_row = vbase + (key >= 16 ? w.v[1] : w.v[0]) + (int64_t)(key & 15) * kv.v_slot * ES;
      // dims VB col .. ; float32: 4 col + 64 j ..
      if constexpr (ES == 2 && NVD == 2) {
        const u32x2 d = *reinterpret_cast<const u32x2*>(at_row + 8 * col);
        vr[e][0] = d[0];
        vr[e][1] = d[1];
      } else {
#pragma unroll
        for (int j = 0; j < NVD / 4; ++j) {
          const u32x4 d = *reinterpret_cast<const u32x4*>(at_row + 16 * col + 256 * j);
#pragma unroll
          for (int w4 = 0; w4 < 4; ++w4) vr[e][4 * j + w4] = d[w4];
        }
      }
    }
  };
  // dim (of head_dim) of V that MFMA t's row r stands for
  auto dim_of = [&](int t, int r) __attribute__((always_inline)) {
    return ES == 2 ? VB * r + t : 4 * r + (t & 3) + 64 * (t >> 2);
  };

  f32x4 o[VB];
#pragma unroll
  for (int t = 0; t < VB; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float l_run = 0.f, m_run = kNoBase;

  // acc[t] += V^T P^T for MFMA t; P as eight probabilities of a lane; `only`: of the key
  // whose number (lane group times 8 + register) it is, -1: all keys
  auto products = [&](f32x4& acc, int t, const float* pv, const u32x4& pb, const u32x4& pl, int only) __attribute__((always_inline)) {
    if constexpr (ES == 2) {
      u32x4 f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        f[w] = __builtin_amdgcn_perm(vr[2 * w + 1][t / 2], vr[2 * w][t / 2], t & 1 ? 0x07060302u : 0x05040100u);
        if (only >= 0) f[w] = g == only >> 3 && w == (only & 7) >> 1 ? f[w] & (only & 1 ? 0xffff0000u : 0xffffu) : 0u;
      }
      Tok<T>::step(acc, f, pb);
      Tok<T>::step(acc, f, pl);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t v = vr[e][t];
        if (only >= 0) v = g == only >> 3 && e == (only & 7) ? v : 0u;
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, v), pv[e], acc, 0, 0, 0);
      }
    }
  };

  Where now, next;
  int t = t0 + wave;
  if (t < t1) {
    now = locate(t);
    load_k(now);
    load_v(now);
    if (t + NW < t1) next = locate(t + NW);
  }
  for (; t < t1; t += NW) {
    f32x4 sc[2];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      sc[a] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NST; ++st) Tok<T>::step(sc[a], kf[a][st], qf[st]);
    }
    const bool more = t + NW < t1;
    if (more) load_k(next);
    const int k0 = ex.tile(t) * BN;
    const bool masked = !(k0 + BN <= first.end && (k0 >= last.start || k0 + BN <= sinks));
    if (masked) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int k = k0 + Tok<T>::key(e >> 2, 4 * g + (e & 3));
        if (!(k < mine.end && (k >= mine.start || k < sinks))) sc[e >> 2][e & 3] = -INFINITY;
      }
    }
    float pv[8], lh;
    // (bf16: probabilities in two terms, 15 bits; the matrix units have the time, and the output's
    // rounding is then the only one that counts.  The first is the probability cut to less than
    // itself, so that both are above 0 where it is: their products with an infinite value are
    // that infinity, where a rest of 0 would give NaN and one below 0 the other sign.)
    u32x4 pb = u32x4{0u, 0u, 0u, 0u}, pl = pb;
    auto probs = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) pv[e] = __builtin_amdgcn_exp2f(fmaf(sc[e >> 2][e & 3], p.c, -m_run));
      if constexpr (ES == 2) {
        float rest[8];
        uint32_t cut[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t bits = __builtin_bit_cast(uint32_t, pv[e]);
          cut[e] = (bits - (bits != 0u)) & 0xffff0000u;
          rest[e] = pv[e] - __builtin_bit_cast(float, cut[e]);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) pb[w] = cut[2 * w] >> 16 | cut[2 * w + 1];
        pl = Chunk<T>::pack(rest);
      }
      lh = ((pv[0] + pv[1]) + (pv[2] + pv[3])) + ((pv[4] + pv[5]) + (pv[6] + pv[7]));
    };
    probs();
    if (__any(!(lh <= (float)(1 << (int)kRowsSlack)))) {   // the base moves (attn_rows.h)
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) mx = fmaxf(mx, sc[e >> 2][e & 3]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m_run, mx * p.c);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < VB; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[d][r] *= alpha;
      m_run = m_new;
      probs();
    }
    l_run += lh;
    // Is a value of a masked tile not finite?  (Where all rows see the same keys too: the places of
    // the others are copies of seen ones, and a zero probability makes NaN of an infinity.)
    bool odd = false;
    if (masked) {
      if constexpr (ES == 2) {
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        u16x2 top = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int w = 0; w < NVD; ++w) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vr[e][w] & 0x7fff7fffu));
        odd = __any(top[0] >= 0x7f80 || top[1] >= 0x7f80);
      } else {
        float z = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int w = 0; w < NVD; ++w) z = fmaf(__builtin_bit_cast(float, vr[e][w]), 0.f, z);
        odd = __any(z != 0.f);
      }
    }
    if (!odd) {
#pragma unroll
      for (int d = 0; d < VB; ++d) products(o[d], d, pv, pb, pl, -1);
    } else {
#pragma unroll 1
      for (int e = 0; e < 32; ++e) {
        const int k = k0 + Tok<T>::key((e >> 2) & 1, 4 * (e >> 3) + (e & 3));
        const bool see = k < mine.end && (k >= mine.start || k < sinks);
#pragma unroll
        for (int d = 0; d < VB; ++d) {
          f32x4 add = f32x4{0.f, 0.f, 0.f, 0.f};
          products(add, d, pv, pb, pl, e);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[d][r] += see ? add[r] : 0.f;
        }
      }
    }
    if (more) {
      load_v(next);
      if (t + 2 * NW < t1) next = locate(t + 2 * NW);
    }
  }

  // the waves' sums, joined
  float l = l_run + __shfl_xor(l_run, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int d = 0; d < VB; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) sums[wave][col][dim_of(d, 4 * g + r)] = o[d][r];
  if (g == 0) {
    stats[wave][col][0] = m_run;
    stats[wave][col][1] = l;
  }
  __syncthreads();
  constexpr int PER = BMQ * DH / (64 * NW);   // dims of a thread
  const int q = threadIdx.x / (DH / PER), d0 = (threadIdx.x % (DH / PER)) * PER;
  if (r0 + q >= nrows) return;
  float m = kNoBase, a[NW];
#pragma unroll
  for (int w = 0; w < NW; ++w) m = fmaxf(m, stats[w][q][0]);
  l = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    a[w] = __builtin_amdgcn_exp2f(stats[w][q][0] - m);
    l += a[w] * stats[w][q][1];
  }
  float e[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    e[j] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) e[j] += a[w] * sums[w][q][d0 + j];
  }
  if (at.parts > 1) {
    float* po = part_sums(p.part, slot, q, BMQ, DH) + d0;
#pragma unroll
    for (int j = 0; j < PER; ++j) po[j] = e[j];
    if (d0 == 0) {
      float* ml = part_stats(p.part, kTokensRule.limit, slot, q, BMQ, DH);
      ml[0] = m;
      ml[1] = l;
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int tk = (r0 + q) / p.group, hd = h * p.group + r0 + q - tk * p.group;
  T* dst = p.out + (int64_t)(sq.row0 + tk) * p.ldo + hd * DH + d0;
#pragma unroll
  for (int j = 0; j < PER; ++j) dst[j] = from_f32<T>(e[j] * inv);
}

// Joins the pieces of split row tiles: with m the largest base and a_k = 2^(m_k - m),
// out = sum a_k O_k / sum a_k l_k, in one pass with a running m.  A workgroup (several for many
// rows) per first piece of a row tile.  A wave takes R rows at once; its lanes hold a
// row's dims, four each, and several pieces at a time.  What it costs is memory round
// trips: some 400 pieces of 256 rows take 9 us, row by row with m first they took 15.
template <typename T, int DH, int BMQ>
__global__ __launch_bounds__(256) void attn_join_kernel(RowsParams<T> p, SplitRule rule) {
  const Plan plan = *reinterpret_cast<const Plan*>(p.part);
  const Note note = *part_note(p.part, blockIdx.x);
  if (plan.most == kWhole || (int)blockIdx.x >= plan.pieces * p.kv.kv_heads || note.parts < 2) return;
  const int slot0 = blockIdx.x, h = slot0 / plan.pieces;
  constexpr int LPR = DH / 4, NP = 64 / LPR;   // lanes of a row; pieces at a time
  constexpr int R = BMQ == kTokensTile ? 1 : 4;
  const int lane = threadIdx.x & 63, sub = lane / LPR, d = (lane % LPR) * 4, wave = (int)threadIdx.x >> 6;
  const int rows = min(BMQ, note.rows - note.r0);
#pragma unroll 1
  for (int q0 = (blockIdx.y * 4 + wave) * R; q0 < rows; q0 += 4 * R * gridDim.y) {
    float m[R], l[R];
    f32x4 acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      m[r] = kNoBase;
      l[r] = 0.f;
      acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll 4
    for (int k = sub; k < note.parts; k += NP) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int q = min(q0 + r, rows - 1);
        const float* ml = part_stats(p.part, rule.limit, slot0 + k, q, BMQ, DH);
        const f32x4 o = *reinterpret_cast<const f32x4*>(part_sums(p.part, slot0 + k, q, BMQ, DH) + d);
        const float top = fmaxf(m[r], ml[0]);
        const float was = __builtin_amdgcn_exp2f(m[r] - top), a = __builtin_amdgcn_exp2f(ml[0] - top);
        m[r] = top;
        l[r] = l[r] * was + a * ml[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][e] = acc[r][e] * was + a * o[e];
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int x = LPR; x < 64; x *= 2) {
        const float top = fmaxf(m[r], __shfl_xor(m[r], x)), a = __builtin_amdgcn_exp2f(m[r] - top);
        m[r] = top;
        l[r] *= a;
        l[r] += __shfl_xor(l[r], x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[r][e] *= a;
          acc[r][e] += __shfl_xor(acc[r][e], x);
        }
      }
      if (sub != 0 || q0 + r >= rows) continue;
      const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
      const int row = note.r0 + q0 + r, tk = row / p.group, hd = h * p.group + row - tk * p.group;
      T* dst = p.out + (int64_t)(note.row0 + tk) * p.ldo + hd * DH + d;
#pragma unroll
      for (int e = 0; e < 4; ++e) dst[e] = from_f32<T>(acc[r][e] * inv);
    }
  }
}

template <typename T>
hipError_t launch_tokens(const RowsParams<T>& p, int head_dim, hipStream_t stream) {
  const KeyView& kv = p.kv;
  int64_t grid = rows_items(kv.rows, p.heads, kv.kv_heads, kv.n_seqs, kTokensTile);
  if (p.part) grid = std::max<int64_t>(grid, kTokensRule.limit);
  auto go = [&](auto dh, auto paged, auto gap) {
    if (kv.max_keys <= kTokensShort)
      hipLaunchKernelGGL((attn_tokens_kernel<T, decltype(dh)::value, decltype(paged)::value, 8, decltype(gap)::value>),
                         dim3((unsigned)grid), dim3(512), 0, stream, p);
    else
      hipLaunchKernelGGL((attn_tokens_kernel<T, decltype(dh)::value, decltype(paged)::value, 4, decltype(gap)::value>),
                         dim3((unsigned)grid), dim3(256), 0, stream, p);
  };
  auto by_kind = [&](auto dh) {
    if (!kv.table) go(dh, std::false_type{}, std::false_type{});
    else if (p.mask.gaps()) go(dh, std::true_type{}, std::true_type{});
    else go(dh, std::true_type{}, std::false_type{});
  };
  if (head_dim == 128) by_kind(std::integral_constant<int, 128>{});
  else if (head_dim == 64) by_kind(std::integral_constant<int, 64>{});
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

template <typename T, int BMQ>
hipError_t launch_join(const RowsParams<T>& p, int head_dim, const SplitRule& rule, hipStream_t stream) {
  const dim3 grid(rule.limit, BMQ == kTokensTile ? 1 : BMQ / 16);
  if (head_dim == 128) hipLaunchKernelGGL((attn_join_kernel<T, 128, BMQ>), grid, dim3(256), 0, stream, p, rule);
  else hipLaunchKernelGGL((attn_join_kernel<T, 64, BMQ>), grid, dim3(256), 0, stream, p, rule);
  return hipGetLastError();
}

}  // namespace dif
