// Attention of new tokens over the keys of their sequences, in pages or packed, under
// a mask by token or block, a window and first keys that stay visible (SeenMask).
//
// Work split: a workgroup takes BMQ rows of one sequence and one key head.  A row is
// a token and one of the query heads that share the key head, in that order, so
// shared heads share the key tiles.  Four waves of 32 rows walk the tiles of keys
// that any of the rows sees, BN keys each, copied global -> LDS (one buffer ahead).
//
// Arithmetic as in attention.hip: S^T = K Q^T on 32x32 MFMAs, so a lane owns a row
// and 16 keys of 32; K's rows are placed so that accumulator register r of lane group
// g is key 16 g + r, which makes the probabilities the B operand of O^T += V^T P^T as
// they are.  V lies in memory as K does (token by token).  V^T's operand needs the
// keys of one dim in a lane: for bf16 the LDS reads transpose (four keys a read), for
// float32 each lane reads its own dim.  Softmax in base 2, the base of a row moving
// only when a half tile's probabilities sum above 2^kSlack.
//
// Masks: tiles that none of a wave's rows sees are passed over, tiles that all of
// them see whole run without masks.  In the others hidden scores are -inf.  A zero
// probability times a value that is not finite would be NaN: such tiles are found by
// a product with zeros, and take their keys one by one, leaving out the rows that do
// not see them.
//
// Keys that are copied but seen by no row (tails of a tile) are read from the place
// of a key that is seen, so pages without one are never touched.
#pragma once
#include <algorithm>
#include <type_traits>

#include "attn_tile.h"

namespace dif {

// PAGED: kv has a table.  GAP: windows shorter than the blocks over it (stream.h), in an instance
// of its own (in all of them it cost 5 to 8 %: bf16 heads of 64, 4096 causal tokens 110 against 102 us).
template <typename T, int DH, int BN, bool PAGED, bool GAP>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(RowsParams<T> p) {
  constexpr int NW = 4, BMQ = 32 * NW;
  static_assert(BMQ == kRowsTile, "rows of a workgroup");
  constexpr int VEC = Chunk<T>::VEC, ES = (int)sizeof(T);
  constexpr int CH = DH / VEC;             // pieces per K / V row
  constexpr int NQS = DH / Mma<T>::KS;     // MMA steps over head_dim
  constexpr int NPC = 16 / VEC;            // P pieces per 32 keys
  constexpr int NH = BN / 32;
  typedef TileCopies<T, DH, BN, NW, PAGED, GAP> Copies;
  constexpr int NI = Copies::NI;
  // (a variable per buffer, so that the compiler sees that copies into one are not
  // what it reads from the other)
  typedef typename Copies::Tile Tile;
  __shared__ Tile ks0, vs0, ks1, vs1;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 5, col = lane & 31;
  const KeyView& kv = p.kv;

  Sequences seqs;
  const Plan plan = make_plan<BN>(kv, p.mask, p.group, BMQ, p.part != nullptr, kRowsRule, &seqs);
  leave_plan(p.part, plan);
  int i, h;
  if (!turn_of(blockIdx.x, plan.pieces, kv.kv_heads, &i, &h)) return;
  const Place at = find_place<BN>(kv, p.mask, p.group, BMQ, plan, seqs, i);
  const int slot = h * plan.pieces + i;
  const int s = at.seq;
  const Sequence sq = at.sq;
  const int nrows = sq.rows * p.group;
  // the last tiles see the most keys: first
  const int r0 = (((nrows + BMQ - 1) / BMQ) - 1 - at.tile) * BMQ;
  leave_note(p.part, plan, at, slot, r0, nrows);
  if (r0 < 0 || r0 >= nrows) return;   // (offsets that are not ascending)
  const int shift = sq.keys - sq.rows;     // position of the first row

  const int rlast = min(r0 + BMQ, nrows) - 1;
  const Extent<BN, GAP> ex = extent<BN, GAP>(p.mask, shift + r0 / p.group, shift + rlast / p.group, sq.keys);
  const int sinks = ex.sinks;
  // the piece's tiles [t0, ntiles)
  const int t0 = (int)((int64_t)ex.ntiles * at.part / at.parts);
  const int ntiles = (int)((int64_t)ex.ntiles * (at.part + 1) / at.parts);
  auto key_of = [&](int i) __attribute__((always_inline)) { return ex.tile(i) * BN; };

  // this lane's row; rows past the last repeat it
  const int wr0 = r0 + wave * 32;
  const bool idle = wr0 >= nrows;          // (wave-uniform) no rows
  const int row = min(wr0 + col, nrows - 1);
  const int token = row / p.group, head = h * p.group + row - token * p.group;
  const Seen mine = seen_by(p.mask, shift + token, sq.keys);
  const Seen wfirst = seen_by(p.mask, shift + min(wr0, nrows - 1) / p.group, sq.keys);
  const Seen wlast = seen_by(p.mask, shift + min(wr0 + 31, nrows - 1) / p.group, sq.keys);

  u32x4 qf[NQS];
  {
    const T* qr = p.q + (int64_t)(sq.row0 + token) * p.ldq + head * DH;
#pragma unroll
    for (int st = 0; st < NQS; ++st) qf[st] = *reinterpret_cast<const u32x4*>(qr + (2 * st + g) * VEC);
  }

  const Copies copies(kv, sq, s, h, ex);
  int32_t page[NI];   // of the next tile's instructions

  f32x16 o[DH / 32];
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  float l_run = 0.f, m_run = kNoBase;
  f32x16 zero;
#pragma unroll
  for (int r = 0; r < 16; ++r) zero[r] = 0.f;

  // A lane's places in the tiles' rows: of its K pieces, and of its V pieces per 32
  // dims.  (Opaque, so that the buffers and halves are offsets of the reads and not addresses of their own.)
  uint32_t kat[4], vat[DH / 32];
#pragma unroll
  for (int st = 0; st < 4; ++st) {
    kat[st] = col * CH * 16 + 16 * k_swz(col, 2 * st + g);
    asm volatile("" : "+v"(kat[st]));
  }
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt) {
    if constexpr (ES == 2) {
      const int r = 4 * g + ((lane & 15) >> 2), c = 4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      vat[dt] = r * CH * 16 + 16 * v_swz<T, CH>(r, c) + 8 * (lane & 1);
    } else {
      vat[dt] = 4 * g * CH * 16 + 16 * v_swz<T, CH>(4 * g, 8 * dt + (col >> 2)) + 4 * (col & 3);
    }
    asm volatile("" : "+v"(vat[dt]));
  }
  auto scores = [&](const Tile& ks, int kk, const f32x16& c0) __attribute__((always_inline)) {
    constexpr int KB = NQS >= 8 ? NQS / 2 : NQS;
    f32x16 sc = c0;
#pragma unroll
    for (int s0 = 0; s0 < NQS; s0 += KB) {
      u32x4 kf[KB];
#pragma unroll
      for (int st = 0; st < KB; ++st)
        kf[st] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(&ks[kk * 32][0]) + 128 * ((s0 + st) / 4) + kat[(s0 + st) & 3]);
#pragma unroll
      for (int st = 0; st < KB; ++st) Mma<T>::step(sc, kf[st], qf[s0 + st]);
    }
    return sc;
  };
  // Hidden keys of the 32 from key0 on: of this lane's sixteen, numbers below end that
  // are at or past start or below sunk are seen.
  struct Half {
    int start, end, sunk;
    __device__ __forceinline__ bool sees(int r) const { return r < end && (r >= start || r < sunk); }
  };
  auto half_of = [&](int key0) __attribute__((always_inline)) {
    int k = key0 + 16 * g;
    asm volatile("" : "+v"(k));   // (sixteen comparisons with constants, none of them kept)
    return Half{mine.start - k, mine.end - k, sinks - k};
  };
  auto mask = [&](f32x16& sc, int key0) __attribute__((always_inline)) {
    const Half hf = half_of(key0);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (!hf.sees(r)) sc[r] = -INFINITY;
  };
  // V^T piece u of dims 32 dt + col: this lane group's keys 16 g + VEC u .. of half kk
  // (rows of a piece lie eight apart, or beside each other for float32: the swizzle is the lane's)
  auto v_piece = [&](const Tile& vs, int kk, int u, int dt) __attribute__((always_inline)) {
    u32x4 f;
    if constexpr (ES == 2) {
#if defined(__HIP_DEVICE_COMPILE__)
      typedef short s4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s4 lds4_t;
      u32x2 part[2];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const char* at = reinterpret_cast<const char*>(&vs[kk * 32 + 8 * (2 * u + hh)][0]) + vat[dt];
        part[hh] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t*)at));
      }
      f = u32x4{part[0][0], part[0][1], part[1][0], part[1][1]};
#endif
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        f[e] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(&vs[kk * 32 + 8 * u + e][0]) + vat[dt]);
    }
    return f;
  };

  auto tile = [&](int i, const Tile& ks, const Tile& vs, auto masked_c) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked_c)::value;
    const int key0 = key_of(i);
    auto half = [&](int kk) __attribute__((always_inline)) {
      __builtin_amdgcn_sched_barrier(0);
      f32x16 sc = scores(ks, kk, zero);
      if (MASKED) mask(sc, key0 + 32 * kk);
      constexpr bool EARLY = !MASKED && ES == 2;   // V^T's operands on their way during the softmax
      u32x4 vf[NPC][DH / 32];
      if constexpr (EARLY) {
#pragma unroll
        for (int u = 0; u < NPC; ++u)
#pragma unroll
          for (int dt = 0; dt < DH / 32; ++dt) vf[u][dt] = v_piece(vs, kk, u, dt);
      }
      __builtin_amdgcn_sched_barrier(0);
      u32x4 pc[NPC];
      float lh = 0.f;
      auto probs = [&](float scale, float base) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NPC; ++u) {
          float pv[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float x = sc[u * VEC + e];
            pv[e] = __builtin_amdgcn_exp2f(fmaf(x, scale, -base));
          }
          // (bf16: rounded for the matrix units, their sum below is not.  The output's error grows
          // from 1.7e-3 to 2.3e-3 of its size; a second term would be half as many MFMAs again)
          pc[u] = Chunk<T>::pack(pv);
          float t[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) t[e] = pv[e];
#pragma unroll
          for (int w = VEC / 2; w > 0; w /= 2)
#pragma unroll
            for (int e = 0; e < w; ++e) t[e] += t[e + w];
          lh = u == 0 ? t[0] : lh + t[0];
        }
      };
      probs(p.c, m_run);
      // The base moves when a half's probabilities sum above 2^kRowsSlack (or are not
      // numbers); so it does at the first key of every row.
      if (__any(!(lh <= (float)(1 << (int)kRowsSlack)))) {
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
        const float m_new = fmaxf(m_run, fmaxf(mx, __shfl_xor(mx, 32)) * p.c);
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
        m_run = m_new;
        probs(p.c, m_new);
      }
      l_run += lh;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (MASKED) {
        // is a value of the half not finite?
        f32x16 z = zero;
#pragma unroll
        for (int u = 0; u < NPC; ++u)
#pragma unroll
          for (int dt = 0; dt < DH / 32; ++dt) Mma<T>::step(z, v_piece(vs, kk, u, dt), u32x4{0u, 0u, 0u, 0u});
        bool odd = false;
#pragma unroll
        for (int r = 0; r < 16; ++r) odd |= z[r] != 0.f;
        if (__any(odd)) {
          // key by key: the products of one key alone, added where it is seen
#pragma unroll 1
          for (int ke = 0; ke < 32; ++ke) {
            const int gk = ke >> 4, u = (ke & 15) / VEC, e = ke % VEC;
            const int k = key0 + 32 * kk + ke;
            const bool see = k < mine.end && (k >= mine.start || k < sinks);
            u32x4 pu = pc[0];
#pragma unroll
            for (int t = 1; t < NPC; ++t) pu = u == t ? pc[t] : pu;
#pragma unroll
            for (int dt = 0; dt < DH / 32; ++dt) {
              u32x4 one = v_piece(vs, kk, u, dt);
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const uint32_t bits = ES == 4 ? 0xffffffffu : e & 1 ? 0xffff0000u : 0xffffu;
                one[w] = g == gk && w == e * ES / 4 ? one[w] & bits : 0u;
              }
              f32x16 add = zero;
              Mma<T>::step(add, one, pu);
#pragma unroll
              for (int r = 0; r < 16; ++r) o[dt][r] += see ? add[r] : 0.f;
            }
          }
          return;
        }
      }
#pragma unroll
      for (int u = 0; u < NPC; ++u) {
        if constexpr (ES == 4) __builtin_amdgcn_sched_barrier(0);   // (a few operands in registers at a time)
#pragma unroll
        for (int dt = 0; dt < DH / 32; ++dt) {
          if constexpr (EARLY) Mma<T>::step(o[dt], vf[u][dt], pc[u]);
          else Mma<T>::step(o[dt], v_piece(vs, kk, u, dt), pc[u]);
        }
      }
    };
    if constexpr (MASKED) {
#pragma unroll 1
      for (int kk = 0; kk < NH; ++kk) half(kk);
    } else {
#pragma unroll
      for (int kk = 0; kk < NH; ++kk) half(kk);
    }
  };
  auto visit = [&](int i, const Tile& ks, const Tile& vs, Tile& next_ks, Tile& next_vs) __attribute__((always_inline)) {
    // the next tile's copies (its buffer was last read before the barrier), the places of the one after it
    if (i + 1 < ntiles) {
      copies.template copy<false>(ex.tile(i + 1), page, next_ks);
      copies.template copy<true>(ex.tile(i + 1), page, next_vs);
    }
    if (i + 2 < ntiles) copies.look_up(ex.tile(i + 2), page);
    const int k0 = key_of(i), k1 = k0 + BN;
    if (!idle && k0 < wlast.end && (k1 > wfirst.start || k0 < sinks)) {
      if (k1 <= wfirst.end && (k0 >= wlast.start || k1 <= sinks)) tile(i, ks, vs, std::false_type{});
      else tile(i, ks, vs, std::true_type{});
    }
    wait_vmcnt<0>();   // this wave's copies have landed
    __syncthreads();   // ... and every other wave's
  };
  if (t0 < ntiles) {
    copies.look_up(ex.tile(t0), page);
    copies.template copy<false>(ex.tile(t0), page, ks0);
    copies.template copy<true>(ex.tile(t0), page, vs0);
    if (t0 + 1 < ntiles) copies.look_up(ex.tile(t0 + 1), page);
    wait_vmcnt<0>();
    __syncthreads();
  }
  for (int i = t0; i < ntiles; i += 2) {
    visit(i, ks0, vs0, ks1, vs1);
    if (i + 1 < ntiles) visit(i + 1, ks1, vs1, ks0, vs0);
  }
  if (idle) return;

  static_assert(32 * DH * ES <= (int)sizeof(Tile), "staging");
  char* stage = reinterpret_cast<char*>(wave == 0 ? &ks0 : wave == 1 ? &vs0 : wave == 2 ? &ks1 : &vs1);
  finish_rows<T, DH>(p, sq, h, o, l_run, m_run, stage, r0, wave * 32, nrows, BMQ, at.parts > 1, slot, kRowsRule.limit);
}

template <typename T>
hipError_t launch_rows(const RowsParams<T>& p, int head_dim, hipStream_t stream) {
  constexpr int BN = sizeof(T) == 2 ? 64 : 32;
  const KeyView& kv = p.kv;
  int64_t grid = rows_items(kv.rows, p.heads, kv.kv_heads, kv.n_seqs, kRowsTile);
  if (p.part) grid = std::max<int64_t>(grid, kRowsRule.limit);
  grid = turns(grid, kv.kv_heads);
  auto go = [&](auto dh, auto paged, auto gap) {
    hipLaunchKernelGGL((attn_rows_kernel<T, decltype(dh)::value, BN, decltype(paged)::value, decltype(gap)::value>),
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

}  // namespace dif
