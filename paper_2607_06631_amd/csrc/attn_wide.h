// Attention of long chunks, bf16, head_dim 128: attn_rows.h's arithmetic with two groups of
// 32 rows a wave, 256 rows a workgroup, one wave per SIMD, and the software pipeline of
// attention.hip's two-group kernel.
//
// Every K and V fragment read from LDS feeds the MFMAs of both groups g0, g1.  (With 32 rows a
// wave LDS has to deliver 128 bytes a clock to keep the matrix units busy, all that
// it can: 0.8 PFLOP/s.)  The lone wave of a SIMD hides its own softmax, in blocks of 16 MFMAs for
// each half tile (t, H) of 32 keys:
//   X(t,H): S(t,H,g1) = K Q1^T and O1 += V^T P(before,g1);  softmax of S(t,H,g0)
//   Y(t,H): S(next,g0) = K Q0^T and O0 += V^T P(t,H,g0);    softmax of S(t,H,g1)
// Score and output MFMAs alternate; the exponentials, packs and sums of a half are dealt
// over the block's slots; a fragment is read again right behind its last use.  Ahead of
// the first half the pipeline holds P = 0 and V = 0, behind the last one it computes
// scores that nobody uses, so there is one form of each block.
//
// Tiles sit in a ring of three LDS buffers, a barrier per tile in X(t,1): tile t+1 has landed,
// tile t-1 is done with, and tile t+2 is sent for into its buffer, an instruction behind
// each score MFMA, from addresses that the scalar unit worked out during X(t,0).
//
// A row's base is kept in the accumulator that its scores start from (-m in MFMA units).
// A row without a base yet (it has seen no key) has 0 there and a limit below any sum,
// so its first half with a seen key sets it.
//
// Masked tiles (some row does not see some key) come through registers, not straight into LDS:
// V entries that are not finite are stored as 0, since the zero probability of a row
// that does not see them would make NaN of them; such entries are added to the rows that do
// see them when all is done (the sum is not finite either way).
//
// The MFMAs are inline assembly, so that Q^T and O^T stay in AGPRs and the rest in VGPRs;
// the distances that the hardware needs between them and VALU code are kept here by wait
// states and empty register constraints, as attention.hip explains, and checked on the compiled
// code (tests/test_stream_mfma_hazards.py).
#pragma once
#include <algorithm>
#include <type_traits>

#include "attn_tile.h"

namespace dif {

constexpr int kWideTile = 256;
// (what a piece costs beside its tiles: 14 us, most of it the first run of the code from a cold
// instruction cache, and its part of the joining launch)
constexpr SplitRule kWideRule{256, 512, 8, 12};

namespace wide {
__device__ __forceinline__ void mma_sc(f32x16& d, const u32x4& a, const u32x4& b, const f32x16& c) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %3" : "=&v"(d) : "v"(a), "a"(b), "v"(c));
}
__device__ __forceinline__ void mma_s(f32x16& d, const u32x4& a, const u32x4& b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(d) : "v"(a), "a"(b));
}
__device__ __forceinline__ void mma_o(f32x16& d, const u32x4& a, const u32x4& b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(d) : "v"(a), "v"(b));
}
// behind VALU code that wrote an operand
__device__ __forceinline__ void mma_o_first(f32x16& d, const u32x4& a, const u32x4& b) {
  asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(d) : "v"(a), "v"(b));
}
__device__ __forceinline__ void drain() { asm volatile("s_nop 15\n\ts_nop 15" ::); }
__device__ __forceinline__ void valu_to_mfma() { asm volatile("s_nop 4" ::); }
template <typename X>
__device__ __forceinline__ void pin(X& x) { asm volatile("" : "+v"(x)); }
template <typename X>
__device__ __forceinline__ void pin_a(X& x) { asm volatile("" : "+a"(x)); }
}  // namespace wide

// SC: queries arrive multiplied by log2(e) / sqrt(dh).
template <bool SC, bool PAGED>
__global__ __launch_bounds__(256, 1) void attn_wide_kernel(RowsParams<bf16> p) {
  typedef bf16 T;
  constexpr int DH = 128, NW = 4, BMQ = 64 * NW, BN = 64, VEC = 8, CH = DH / VEC, NQS = DH / 16, ND = DH / 32;
  static_assert(BMQ == kWideTile, "rows of a workgroup");
  typedef TileCopies<T, DH, BN, NW, PAGED, false> Copies;
  constexpr int NI = Copies::NI;
  typedef typename Copies::Tile Tile;
  // (a variable per buffer: attn_rows.h)
  __shared__ Tile ks0, ks1, ks2, vs0, vs1, vs2;
  __shared__ int odd;   // a masked tile held values that are not finite
  auto kbuf = [&](int b) __attribute__((always_inline)) -> Tile& { return b == 0 ? ks0 : b == 1 ? ks1 : ks2; };
  auto vbuf = [&](int b) __attribute__((always_inline)) -> Tile& { return b == 0 ? vs0 : b == 1 ? vs1 : vs2; };

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 5, col = lane & 31;
  const KeyView& kv = p.kv;

  Sequences seqs;
  const Plan plan = make_plan<BN>(kv, p.mask, p.group, BMQ, p.part != nullptr, kWideRule, &seqs);
  leave_plan(p.part, plan);
  int i, h;
  if (!turn_of(blockIdx.x, plan.pieces, kv.kv_heads, &i, &h)) return;
  const Place at = find_place<BN>(kv, p.mask, p.group, BMQ, plan, seqs, i);
  const int slot = h * plan.pieces + i;
  const int s = at.seq;
  const Sequence sq = at.sq;
  const int nrows = sq.rows * p.group;
  const int r0 = (((nrows + BMQ - 1) / BMQ) - 1 - at.tile) * BMQ;   // the last tiles see the most keys: first
  leave_note(p.part, plan, at, slot, r0, nrows);
  if (r0 < 0 || r0 >= nrows) return;   // (offsets that are not ascending)
  const int shift = sq.keys - sq.rows;
  const int rlast = min(r0 + BMQ, nrows) - 1;
  const Extent<BN, false> ex = extent<BN, false>(p.mask, shift + r0 / p.group, shift + rlast / p.group, sq.keys);
  const int sinks = ex.sinks;
  const int t0 = (int)((int64_t)ex.ntiles * at.part / at.parts);
  const int ntiles = (int)((int64_t)ex.ntiles * (at.part + 1) / at.parts);

  const int wr0 = r0 + wave * 64;
  const Seen wfirst = seen_by(p.mask, shift + min(wr0, nrows - 1) / p.group, sq.keys);
  const Seen wlast = seen_by(p.mask, shift + min(wr0 + 63, nrows - 1) / p.group, sq.keys);
  Seen mine[2];
  u32x4 qf[2][NQS];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int row = min(wr0 + 32 * q + col, nrows - 1);   // rows past the last repeat it
    const int token = row / p.group, head = h * p.group + row - token * p.group;
    mine[q] = seen_by(p.mask, shift + token, sq.keys);
    const T* qr = p.q + (int64_t)(sq.row0 + token) * p.ldq + head * DH;
#pragma unroll
    for (int st = 0; st < NQS; ++st) qf[q][st] = *reinterpret_cast<const u32x4*>(qr + (2 * st + g) * VEC);
  }
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int st = 0; st < NQS; ++st) wide::pin_a(qf[q][st]);   // AGPRs from here on
  const Copies copies(kv, sq, s, h, ex);
  // tiles whose keys all rows of the workgroup (of the wave) see
  const Seen gfirst = seen_by(p.mask, shift + r0 / p.group, sq.keys);
  const Seen glast = seen_by(p.mask, shift + rlast / p.group, sq.keys);
  auto clear = [&](int i, const Seen& a, const Seen& b) __attribute__((always_inline)) {
    const int k0 = i * BN, k1 = k0 + BN;
    return k1 <= a.end && (k0 >= b.start || k1 <= sinks);
  };
  // The order of the tiles: clear ones first (of the sinks, then of the window from wa to wb), then the
  // others, so that the two kinds have a loop each.
  const int sc0 = min(ex.nsink, min(sinks, gfirst.end) / BN);
  const int wend = ex.w0 + ex.ntiles - ex.nsink;
  int wa = max(ex.w0, (glast.start + BN - 1) / BN), wb = min(wend, gfirst.end / BN);
  if (wa >= wb) wa = wb = ex.w0;
  const int nclear = sc0 + wb - wa;
  auto number = [&](int t) __attribute__((always_inline)) {
    if (t < nclear) return t < sc0 ? t : wa + t - sc0;
    const int u = t - nclear + sc0;
    if (u < ex.nsink) return u;
    const int w = ex.w0 + u - ex.nsink;
    return w < wa ? w : w + wb - wa;
  };

  // a lane's places in the tiles' rows (attn_rows.h)
  uint32_t kat[4], vat[ND];
#pragma unroll
  for (int st = 0; st < 4; ++st) {
    kat[st] = col * CH * 16 + 16 * k_swz(col, 2 * st + g);
    wide::pin(kat[st]);
  }
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) {
    const int r = 4 * g + ((lane & 15) >> 2), c = 4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    vat[dt] = r * CH * 16 + 16 * v_swz<T, CH>(r, c) + 8 * (lane & 1);
    wide::pin(vat[dt]);
  }

  f32x16 o[2][ND], negm[2], sc[2];
  float l_run[2] = {0.f, 0.f}, m_run[2] = {0.f, 0.f}, limit[2] = {-1.f, -1.f};
  u32x4 kf[NQS], vf[2 * ND], pc[2][2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
#pragma unroll
    for (int r = 0; r < 16; ++r) negm[q][r] = 0.f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
#pragma unroll
      for (int r = 0; r < 16; ++r) o[q][dt][r] = 0.f;
      wide::pin_a(o[q][dt]);
    }
    pc[q][0] = pc[q][1] = u32x4{0u, 0u, 0u, 0u};
  }
#pragma unroll
  for (int i = 0; i < 2 * ND; ++i) vf[i] = u32x4{0u, 0u, 0u, 0u};

  auto read_k = [&](const Tile& ks, int kk, int i) __attribute__((always_inline)) {
    typedef __attribute__((address_space(3))) const volatile u32x4 lds_t;
    kf[i] = *(lds_t*)(reinterpret_cast<const char*>(&ks[kk * 32][0]) + 128 * (i / 4) + kat[i & 3]);
  };
  // fragment i = 4 u + dt: dims 32 dt .., keys 8 u .. of the lane group's 16
  auto read_v = [&](const Tile& vs, int kk, int i) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s4 lds4_t;
    u32x2 part[2];
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const char* a = reinterpret_cast<const char*>(&vs[kk * 32 + 8 * (2 * (i / ND) + hh)][0]) + vat[i % ND];
      part[hh] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t*)a));
    }
    vf[i] = u32x4{part[0][0], part[0][1], part[1][0], part[1][1]};
#endif
  };

  // Softmax of group q's half, in pieces for the slots behind MFMA k (0 .. 15) of a block: the
  // exponentials two a slot in 0 .. 3 and one in 4 .. 11, each bf16 pair and each add of the
  // two chunk sums a slot behind its last input, the half's sum in slot 13.
  const float unit = SC ? 1.f : p.c;   // scores to base-2 exponents
  float pe[2][16], ta[2][2][4], tb[2][2][2], lsum[2][2], lh[2];
  auto soft = [&](int q, int k) __attribute__((always_inline)) {
    auto at_slot = [](int e) { return e < 8 ? e >> 1 : e - 4; };
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (at_slot(e) == k) {
        float x = sc[q][e];
        if constexpr (!SC) x *= unit;
        pe[q][e] = __builtin_amdgcn_exp2f(x);
        wide::pin(pe[q][e]);
      }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (at_slot(2 * j + 1) + 1 == k) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        const bf16x2 two = {(bf16)pe[q][2 * j], (bf16)pe[q][2 * j + 1]};   // (attn_rows.h: why rounded)
        pc[q][j >> 2][j & 3] = __builtin_bit_cast(uint32_t, two);
        wide::pin(pc[q][j >> 2]);
      }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (at_slot(8 * u + j + 4) + 1 == k) {
          ta[q][u][j] = pe[q][8 * u + j] + pe[q][8 * u + j + 4];
          wide::pin(ta[q][u][j]);
        }
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (at_slot(8 * u + 6 + j) + 2 == k) {
          tb[q][u][j] = ta[q][u][j] + ta[q][u][j + 2];
          wide::pin(tb[q][u][j]);
        }
    }
    if (k == 14) {
      lsum[q][0] = tb[q][0][0] + tb[q][0][1];
      lsum[q][1] = tb[q][1][0] + tb[q][1][1];
      lh[q] = lsum[q][0] + lsum[q][1];
      wide::pin(lh[q]);
    }
  };
  // The base moves (rarely, but for a row's first key).  Behind slot 14 of a block, before
  // its last MFMA, which is the other group's.
  auto settle = [&](int q) __attribute__((always_inline)) {
    if (__builtin_expect(__any(!(lh[q] <= limit[q])), 0)) {
      wide::drain();
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[q][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32)) * unit;
      const bool fresh = limit[q] < 0.f, any = mx > -INFINITY;
      // (a fresh row's sums are 0, and its base may be below 0)
      const float d = fresh ? (any ? mx : 0.f) : fmaxf(mx, 0.f);
      const float alpha = fresh ? 1.f : __builtin_amdgcn_exp2f(-d);
      if (any) limit[q] = (float)(1 << (int)kRowsSlack);
      l_run[q] *= alpha;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        wide::pin_a(o[q][dt]);
#pragma unroll
        for (int r = 0; r < 16; ++r) o[q][dt][r] *= alpha;
        wide::pin_a(o[q][dt]);
      }
      m_run[q] += d;
      const float dm = SC ? d : d / unit;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[q][r] -= dm;
        negm[q][r] -= dm;
      }
      float e16[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) e16[e] = __builtin_amdgcn_exp2f(SC ? sc[q][e] : sc[q][e] * unit);
      lh[q] = 0.f;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        pc[q][u] = Chunk<T>::pack(e16 + 8 * u);
#pragma unroll
        for (int e = 0; e < 8; ++e) lh[q] += e16[8 * u + e];
      }
      wide::pin(negm[q]);
      wide::pin(pc[q][0]);
      wide::pin(pc[q][1]);
      wide::valu_to_mfma();
    }
    l_run[q] += lh[q];
  };
  auto mask = [&](int q, int key0) __attribute__((always_inline)) {
    wide::drain();
    int k = key0 + 16 * g;
    wide::pin(k);
    const int start = mine[q].start - k, end = mine[q].end - k, sunk = sinks - k;
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (!(r < end && (r >= start || r < sunk))) sc[q][r] = -INFINITY;
  };

  // a masked tile's V: through registers
  auto copy_checked = [&](int i, Tile& to) __attribute__((always_inline)) {
    bool found = false;
    int key[NI];
    int32_t pg[NI];
    u32x4 v[NI];
    const uint64_t seen = copies.seen(i);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      key[j] = copies.seen_key(i, seen, key_of_row((j * NW + wave) * Copies::RPI + lane / CH));
      pg[j] = PAGED ? copies.table[key[j] >> kv.page_shift] : 0;
    }
#pragma unroll
    for (int j = 0; j < NI; ++j)
      v[j] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(copies.vbase) +
                                             copies.place(pg[j], key[j], kv.v_slot) +
                                             v_swz<T, CH>(lane / CH, lane % CH) * 16);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if ((v[j][w] & 0x7f80u) == 0x7f80u) {
          v[j][w] &= 0xffff0000u;
          found = true;
        }
        if ((v[j][w] & 0x7f800000u) == 0x7f800000u) {
          v[j][w] &= 0xffffu;
          found = true;
        }
      }
      to[(j * NW + wave) * Copies::RPI + lane / CH][lane % CH] = v[j];
    }
    if (found) odd = 1;
  };
  auto copy = [&](int t, Tile& kt, Tile& vt, int32_t (&page)[NI]) __attribute__((always_inline)) {
    if (t >= ntiles) return;
    const int i = number(t);
    copies.template copy<false>(i, page, kt);
    if (clear(i, gfirst, glast)) copies.template copy<true>(i, page, vt);
    else copy_checked(i, vt);
  };
  // instruction j of the copies of a clear tile (K, then V; keys from k0): its address, and itself
  uint64_t from[2 * NI];
  int32_t page[NI];
  [[maybe_unused]] const uint32_t kl = copies.koff + 16 * (k_swz(lane / CH, lane % CH) ^ k_swz(wave * Copies::RPI, 0));
  [[maybe_unused]] const uint32_t vl = copies.voff + 16 * v_swz<T, CH>(lane / CH, lane % CH);
  static_assert(NW * Copies::RPI % 8 == 0, "the swizzle of an instruction's rows is the wave's");
  // Pages of tile t's runs: sent for during Y(t-3,0) with a vector load that the wait before
  // the next barrier covers, taken up behind that barrier.  (While a scalar load is under
  // way, a wait for an LDS read has to be one for all of them: 2.72 against 2.64 ms for
  // 4680 rows over 32760 keys.)
  int32_t pages = 0;
  auto send_pages = [&](int t) __attribute__((always_inline)) {
    if constexpr (PAGED) {
      const int i = number(min(t, ntiles - 1));
      const int k = ex.nearest(i, i * BN + key_of_row(((lane % NI) * NW + wave) * Copies::RPI));
      pages = copies.table[k >> kv.page_shift];
    }
  };
  auto take_pages = [&]() __attribute__((always_inline)) {
    if constexpr (PAGED) {
#pragma unroll
      for (int j = 0; j < NI; ++j) page[j] = __builtin_amdgcn_readlane(pages, j);
    }
  };
  auto address = [&](int k0, int j) __attribute__((always_inline)) {
    const bool v = j >= NI;
    const int run = v ? j - NI : j, k = k0 + copies.run_key(run);
    if (PAGED && v)   // (pages of K and V have the same strides)
      from[j] = from[run] + ((uint64_t)(uintptr_t)copies.vbase - (uint64_t)(uintptr_t)copies.kbase);
    else
      from[j] = (uint64_t)(uintptr_t)(v ? copies.vbase : copies.kbase) +
                copies.place(PAGED ? page[run] : 0, k, v ? kv.v_slot : kv.k_slot);
    asm volatile("" : "+s"(from[j]));
  };
  auto send = [&](Tile& kt, Tile& vt, int j) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) void lds_t;
    typedef __attribute__((address_space(1))) void glb_t;
    const bool v = j >= NI;
    const int r = ((v ? j - NI : j) * NW + wave) * Copies::RPI;
    Tile& to = v ? vt : kt;
    __builtin_amdgcn_global_load_lds((glb_t*)((const char*)(uintptr_t)from[j] + (v ? vl : kl)), (lds_t*)&to[r][0], 16, 0, 0);
#endif
  };

  // HOT: tiles t to t+2 are clear.
  auto block_x = [&](int t, auto hot, auto h_c, const Tile& ks, const Tile& vs, const Tile& kn, Tile& kfree,
                     Tile& vfree) __attribute__((always_inline)) {
    constexpr bool HOT = decltype(hot)::value;
    constexpr int H = decltype(h_c)::value;
    [[maybe_unused]] const int k0 = (t + 2 + (t + 2 < sc0 ? 0 : wa - sc0)) * BN;   // of clear tile t+2
    if constexpr (!HOT) {
      const int n = number(t);
      if (!clear(n, wfirst, wlast)) mask(0, n * BN + 32 * H);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NQS; ++i) {
      if (i == 0) wide::mma_sc(sc[1], kf[0], qf[1][0], negm[1]);
      else wide::mma_s(sc[1], kf[i], qf[1][i]);
      if constexpr (H == 1) {
        if (i == 0) {
          // (the first score MFMA reads no LDS and runs under the barrier)
          __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (0 << 8));   // vmcnt(0) lgkmcnt(0)
          asm volatile("" ::: "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
        }
        read_k(kn, 0, i);
        if constexpr (HOT) send(kfree, vfree, i);
      } else {
        read_k(ks, 1, i);
        if constexpr (HOT) address(k0, i);
      }
      soft(0, 2 * i);
      if (i == 7) settle(0);
      __builtin_amdgcn_sched_barrier(0);
      if (i == 0) wide::mma_o_first(o[1][i % ND], vf[i], pc[1][i / ND]);
      else wide::mma_o(o[1][i % ND], vf[i], pc[1][i / ND]);
      read_v(vs, H, i);
      soft(0, 2 * i + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (H == 1) {
      if constexpr (!HOT) copy(t + 2, kfree, vfree, page);
      take_pages();
    }
  };
  auto block_y = [&](int t, auto hot, auto h_c) __attribute__((always_inline)) {
    constexpr int H = decltype(h_c)::value;
    if constexpr (!decltype(hot)::value) {
      const int n = number(t);
      if (!clear(n, wfirst, wlast)) mask(1, n * BN + 32 * H);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NQS; ++i) {
      if (i == 0) wide::mma_sc(sc[0], kf[0], qf[0][0], negm[0]);
      else wide::mma_s(sc[0], kf[i], qf[0][i]);
      soft(1, 2 * i);
      if (i == 7) settle(1);
      __builtin_amdgcn_sched_barrier(0);
      if (i == 0) wide::mma_o_first(o[0][i % ND], vf[i], pc[0][i / ND]);
      else wide::mma_o(o[0][i % ND], vf[i], pc[0][i / ND]);
      soft(1, 2 * i + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  using No = std::integral_constant<int, 0>;
  using Yes = std::integral_constant<int, 1>;
  auto tile = [&](int t, auto hot, const Tile& ks, const Tile& vs, const Tile& kn, Tile& kfree,
                  Tile& vfree) __attribute__((always_inline)) {
    block_x(t, hot, No{}, ks, vs, kn, kfree, vfree);
    send_pages(t + 3);
    block_y(t, hot, No{});
    block_x(t, hot, Yes{}, ks, vs, kn, kfree, vfree);
    block_y(t, hot, Yes{});
  };

  if (threadIdx.x == 0) odd = 0;
  __syncthreads();
  if (t0 < ntiles) {
    copies.look_up(number(t0), page);
    copy(t0, ks0, vs0, page);
    if (t0 + 1 < ntiles) copies.look_up(number(t0 + 1), page);
    copy(t0 + 1, ks1, vs1, page);
    if (t0 + 2 < ntiles) copies.look_up(number(t0 + 2), page);
    wait_vmcnt<0>();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NQS; ++i) read_k(ks0, 0, i);
    wide::pin(negm[0]);
    wide::pin(negm[1]);
    wide::valu_to_mfma();
    wide::mma_sc(sc[0], kf[0], qf[0][0], negm[0]);
#pragma unroll
    for (int i = 1; i < NQS; ++i) wide::mma_s(sc[0], kf[i], qf[0][i]);
    wide::drain();
  }
  // tiles whose copies are of clear tiles, three at a time with the buffers in the code, then
  // the others (the two in one loop would not fit the registers)
  int t = t0;
  for (const int n = min(nclear, ntiles); t + 4 < n; t += 3) {
    tile(t, Yes{}, ks0, vs0, ks1, ks2, vs2);
    tile(t + 1, Yes{}, ks1, vs1, ks2, ks0, vs0);
    tile(t + 2, Yes{}, ks2, vs2, ks0, ks1, vs1);
  }
  for (int b = 0; t < ntiles; ++t) {
    tile(t, No{}, kbuf(b), vbuf(b), kbuf(b == 2 ? 0 : b + 1), kbuf(b == 0 ? 2 : b - 1), vbuf(b == 0 ? 2 : b - 1));
    b = b == 2 ? 0 : b + 1;
  }
  wide::valu_to_mfma();
#pragma unroll
  for (int i = 0; i < 2 * ND; ++i) wide::mma_o(o[1][i % ND], vf[i], pc[1][i / ND]);
  wide::drain();
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    wide::pin(negm[q]);   // (read by MFMAs until here)
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) wide::pin_a(o[q][dt]);
  }
  wait_vmcnt<0>();
  __syncthreads();   // (the tiles' space is used again)
  if (wr0 >= nrows) return;
  if (odd) {
    // values that are not finite, for the rows that see them (one accumulator at a time)
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        wide::pin_a(o[q][dt]);
        f32x16 x = o[q][dt];
#pragma unroll 1
        for (int u = t0; u < ntiles; ++u) {
          const int n = number(u);
          if (clear(n, gfirst, glast)) continue;
#pragma unroll 1
          for (int kk = 0; kk < BN; ++kk) {
            const int k = n * BN + kk;
            if (!ex.sees(k)) continue;
            int32_t pg = 0;
            if constexpr (PAGED) pg = copies.table[k >> kv.page_shift];
            const T* v = reinterpret_cast<const T*>(reinterpret_cast<const char*>(copies.vbase) + copies.place(pg, k, kv.v_slot)) +
                         32 * dt + 4 * g;
            const bool see = k < mine[q].end && (k >= mine[q].start || k < sinks);
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) {
              const bf16x4 y = *reinterpret_cast<const bf16x4*>(v + 8 * rr);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float f = (float)y[e];
                if (see && !(fabsf(f) < INFINITY)) x[4 * rr + e] += f;
              }
            }
          }
        }
        o[q][dt] = x;
        wide::pin_a(o[q][dt]);
      }
  }
  static_assert(32 * DH * 2 <= (int)sizeof(Tile), "staging");
  char* stage = reinterpret_cast<char*>(wave == 0 ? &ks0 : wave == 1 ? &vs0 : wave == 2 ? &ks1 : &vs1);
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    finish_rows<T, DH>(p, sq, h, o[q], l_run[q], limit[q] < 0.f ? kNoBase : m_run[q], stage, r0, wave * 64 + 32 * q,
                       nrows, BMQ, at.parts > 1, slot, kWideRule.limit);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

// (a template, so that only the unit that calls it holds the kernels)
template <typename T>
hipError_t launch_wide(const RowsParams<T>& p, hipStream_t stream) {
  const KeyView& kv = p.kv;
  int64_t grid = rows_items(kv.rows, p.heads, kv.kv_heads, kv.n_seqs, kWideTile);
  if (p.part) grid = std::max<int64_t>(grid, kWideRule.limit);
  grid = turns(grid, kv.kv_heads);
  auto go = [&](auto sc, auto paged) {
    hipLaunchKernelGGL((attn_wide_kernel<decltype(sc)::value, decltype(paged)::value>), dim3((unsigned)grid), dim3(256), 0,
                       stream, p);
  };
  auto by_kind = [&](auto sc) {
    if (kv.table) go(sc, std::true_type{});
    else go(sc, std::false_type{});
  };
  if (p.c == 1.f) by_kind(std::true_type{});
  else by_kind(std::false_type{});
  return hipGetLastError();
}

}  // namespace dif
