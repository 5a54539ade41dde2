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

#include "stream.h"

namespace dif {

// LDS place of 16-byte piece c in row `row` of a V tile (CH pieces a row).  bf16: a
// transposing read takes 64 bytes of four consecutive rows; float32: 128 bytes of
// rows four apart.  Both then meet different banks.
template <typename T, int CH>
__device__ __forceinline__ int v_swz(int row, int c) {
  if constexpr (sizeof(T) == 4) return c ^ (((row >> 2) & 1) << 3);
  else if constexpr (CH == 16) return c ^ ((row & 3) << 2);
  else return c ^ (((row >> 1) & 1) << 2);
}

// The same for K, whose reads take one 16-byte piece of consecutive rows: eight rows meet
// different banks, and pieces eight apart keep their distance, so that a lane holds
// few addresses.
__device__ __forceinline__ constexpr int k_swz(int row, int c) { return c ^ (row & 7); }

// Key (0..) whose K and V lie in row r of a tile: accumulator register r of lane group g
// is then key 16 g + r of its 32 (a permutation of the row's bits).
__device__ __forceinline__ constexpr int key_of_row(int r) {
  return (r & ~31) + 16 * ((r >> 2) & 1) + 4 * ((r >> 3) & 3) + (r & 3);
}

// PAGED: kv has a table.
template <typename T, int DH, int BN, bool PAGED>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(RowsParams<T> p) {
  constexpr int NW = 4, BMQ = 32 * NW;
  static_assert(BMQ == kRowsTile, "rows of a workgroup");
  constexpr int VEC = Chunk<T>::VEC, ES = (int)sizeof(T);
  constexpr int CH = DH / VEC;             // pieces per K / V row
  constexpr int NQS = DH / Mma<T>::KS;     // MMA steps over head_dim
  constexpr int NPC = 16 / VEC;            // P pieces per 32 keys
  constexpr int NH = BN / 32;
  constexpr int RPI = 64 / CH;             // rows per copy instruction
  constexpr int NI = BN / (RPI * NW);      // copy instructions of a wave
  static_assert(NI * RPI * NW == BN, "tile split");
  // (a variable per buffer, so that the compiler sees that copies into one are not
  // what it reads from the other)
  typedef u32x4 Tile[BN][CH];
  __shared__ Tile ks0, vs0, ks1, vs1;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 5, col = lane & 31;
  const KeyView& kv = p.kv;

  // this workgroup's piece; heads outermost, so that an XCD's workgroups share keys
  const Load first_seq = first_load<BN>(kv, p.mask, p.group, BMQ);
  const Plan plan = make_plan<BN>(kv, p.mask, p.group, BMQ, p.part != nullptr, kRowsRule, first_seq);
  leave_plan(p.part, plan);
  const int64_t all = min((int64_t)plan.pieces * kv.kv_heads, (int64_t)gridDim.x);
  if ((int64_t)blockIdx.x >= all) return;
  const int idx = xcd_remap(blockIdx.x, (int)all);
  const int h = idx / plan.pieces;
  const Place at = find_place<BN, false>(kv, p.mask, p.group, BMQ, plan, first_seq, idx - h * plan.pieces);
  const int s = at.seq;
  const Sequence sq = sequence(kv, s);
  const int nrows = sq.rows * p.group;
  // the last tiles see the most keys: first
  const int r0 = (((nrows + BMQ - 1) / BMQ) - 1 - at.tile) * BMQ;
  if (r0 < 0) return;   // (offsets that are not ascending)
  const int shift = sq.keys - sq.rows;     // position of the first row

  const int rlast = min(r0 + BMQ, nrows) - 1;
  const Extent ex = extent<BN>(p.mask, seen_by(p.mask, shift + r0 / p.group, sq.keys),
                               seen_by(p.mask, shift + rlast / p.group, sq.keys));
  const int lo = ex.lo, hi = ex.hi, sinks = ex.sinks, nsink = ex.nsink;
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

  // Copies: instruction j of a wave fills rows (j NW + wave) RPI .. of K and of V, lane
  // by lane; each lane fetches the piece that the swizzle puts in its place.  Row to
  // key and the swizzles are linear in the row's bits: a lane's part and j's part.
  [[maybe_unused]] const T* kbase = static_cast<const T*>(kv.k) + h * kv.k_head;
  [[maybe_unused]] const T* vbase = static_cast<const T*>(kv.v) + h * kv.v_head;
  // An instruction's rows are keys of one aligned run of 16 (bf16, head_dim 64: of two in
  // an aligned 32), so they lie in one page but for the latter and pages of 16: its
  // address is then the wave's, and a lane's offset in it the same in every tile.
  constexpr int RUN = RPI > 4 ? 32 : 16;
  const bool runs = !PAGED || (1 << kv.page_shift) >= RUN;
  const uint32_t lane_key = key_of_row(lane / CH);
  [[maybe_unused]] const uint32_t kvoff = (uint32_t)((int)lane_key * kv.k_slot * ES);
  [[maybe_unused]] const uint32_t vvoff = (uint32_t)((int)lane_key * kv.v_slot * ES);
  int32_t page[NI];   // of the next tile's instructions
  typedef const __attribute__((address_space(4))) int32_t* table_t;
  [[maybe_unused]] const table_t table = (table_t)(uintptr_t)(kv.table + s * kv.ld_table);
  auto run_key = [&](int j) __attribute__((always_inline)) { return key_of_row((j * NW + wave) * RPI); };
  // tile i whole: every key of it is seen by some row
  auto whole = [&](int i) __attribute__((always_inline)) {
    const int k0 = key_of(i);
    return runs && (i < nsink ? k0 + BN <= sinks : (k0 >= lo || k0 + BN <= sinks) && k0 + BN <= hi);
  };
  auto look_up = [&](int i) __attribute__((always_inline)) {
    if constexpr (PAGED) {
      if (whole(i)) {
        const int k0 = key_of(i);
#pragma unroll
        for (int j = 0; j < NI; ++j) page[j] = table[(k0 + run_key(j)) >> kv.page_shift];
      }
    }
  };
  auto copy = [&](int i, Tile& ks, Tile& vs) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) void lds_t;
    typedef __attribute__((address_space(1))) void glb_t;
    const int k0 = key_of(i);
    if (whole(i)) {
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int r = (j * NW + wave) * RPI;
        int64_t ko, vo;
        if constexpr (PAGED) {
          const int64_t pg = (int64_t)min((uint32_t)page[j], (uint32_t)kv.n_pages - 1) * kv.page_stride;
          const int64_t slot = (k0 + run_key(j)) & ((1 << kv.page_shift) - 1);
          ko = pg + slot * kv.k_slot;
          vo = pg + slot * kv.v_slot;
        } else {
          ko = (int64_t)(sq.key0 + k0 + run_key(j)) * kv.k_slot;
          vo = (int64_t)(sq.key0 + k0 + run_key(j)) * kv.v_slot;
        }
        const uint32_t kl = kvoff + 16 * (k_swz(lane / CH, lane % CH) ^ k_swz(r, 0));
        const uint32_t vl = vvoff + 16 * (v_swz<T, CH>(lane / CH, lane % CH) ^ v_swz<T, CH>(r, 0));
        __builtin_amdgcn_global_load_lds((glb_t*)(reinterpret_cast<const char*>(kbase + ko) + kl), (lds_t*)&ks[r][0], 16, 0, 0);
        __builtin_amdgcn_global_load_lds((glb_t*)(reinterpret_cast<const char*>(vbase + vo) + vl), (lds_t*)&vs[r][0], 16, 0, 0);
      }
    } else {
      // keys that no row sees are read from the nearest one that is seen (all are in the tile)
      int ln = lane;
      asm volatile("" : "+v"(ln));   // (nothing of this is kept in registers through the key loop)
      const int first = i < nsink || k0 < sinks ? k0 : lo, end = i < nsink ? sinks : hi;
#pragma unroll 1
      for (int j = 0; j < NI; ++j) {
        const int r = (j * NW + wave) * RPI;
        int k = k0 + run_key(j) + key_of_row(ln / CH);
        if (i >= nsink && k >= sinks) k = max(k, lo);
        k = min(max(k, first), end - 1);
        int64_t ko, vo;
        if constexpr (PAGED) {
          const uint32_t pid = (uint32_t)kv.table[s * kv.ld_table + (k >> kv.page_shift)];
          const int64_t pg = (int64_t)min(pid, (uint32_t)kv.n_pages - 1) * kv.page_stride;
          const int64_t slot = k & ((1 << kv.page_shift) - 1);
          ko = pg + slot * kv.k_slot;
          vo = pg + slot * kv.v_slot;
        } else {
          ko = (int64_t)(sq.key0 + k) * kv.k_slot;
          vo = (int64_t)(sq.key0 + k) * kv.v_slot;
        }
        const int kp = (k_swz(ln / CH, ln % CH) ^ k_swz(r, 0)) * VEC;
        const int vp = (v_swz<T, CH>(ln / CH, ln % CH) ^ v_swz<T, CH>(r, 0)) * VEC;
        __builtin_amdgcn_global_load_lds((glb_t*)(kbase + ko + kp), (lds_t*)&ks[r][0], 16, 0, 0);
        __builtin_amdgcn_global_load_lds((glb_t*)(vbase + vo + vp), (lds_t*)&vs[r][0], 16, 0, 0);
      }
    }
#endif
  };

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
    if (i + 1 < ntiles) copy(i + 1, next_ks, next_vs);
    if (i + 2 < ntiles) look_up(i + 2);
    const int k0 = key_of(i), k1 = k0 + BN;
    if (!idle && k0 < wlast.end && (k1 > wfirst.start || k0 < sinks)) {
      if (k1 <= wfirst.end && (k0 >= wlast.start || k1 <= sinks)) tile(i, ks, vs, std::false_type{});
      else tile(i, ks, vs, std::true_type{});
    }
    wait_vmcnt<0>();   // this wave's copies have landed
    __syncthreads();   // ... and every other wave's
  };
  if (t0 < ntiles) {
    look_up(t0);
    copy(t0, ks0, vs0);
    if (t0 + 1 < ntiles) look_up(t0 + 1);
    wait_vmcnt<0>();
    __syncthreads();
  }
  for (int i = t0; i < ntiles; i += 2) {
    visit(i, ks0, vs0, ks1, vs1);
    if (i + 1 < ntiles) visit(i + 1, ks1, vs1, ks0, vs0);
  }
  if (idle) return;

  // Output rows through LDS, so that store instructions write whole rows: a lane holds
  // four consecutive dims of its row per register group.  A row that saw nothing is 0.
  const float l = l_run + __shfl_xor(l_run, 32);
  if (at.parts > 1) {
    const int r = wave * 32 + col;
    float* po = part_sums(p.part, idx, r, BMQ, DH);
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = o[dt][4 * rr + e];
        *reinterpret_cast<f32x4*>(po + dt * 32 + 8 * rr + 4 * g) = v;
      }
    if (g == 0) {
      float* ml = part_stats(p.part, kRowsRule.limit, idx, r, BMQ, DH);
      ml[0] = m_run;
      ml[1] = l;
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  constexpr int RB = DH * ES;
  constexpr int SRPI = 64 / CH;
  static_assert(32 * RB <= (int)sizeof(Tile), "staging");
  char* stage = reinterpret_cast<char*>(wave == 0 ? &ks0 : wave == 1 ? &vs0 : wave == 2 ? &ks1 : &vs1);
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) {
      const int byte = (dt * 32 + 8 * rr + 4 * g) * ES;
      char* at = stage + col * RB + 16 * ((byte / 16) ^ (col % CH)) + byte % 16;
      if constexpr (ES == 4) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = o[dt][4 * rr + e] * inv;
        *reinterpret_cast<f32x4*>(at) = v;
      } else {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (bf16)(o[dt][4 * rr + e] * inv);
        *reinterpret_cast<bf16x4*>(at) = v;
      }
    }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
  for (int i = 0; i < 32 / SRPI; ++i) {
    const int r = i * SRPI + lane / CH, c = lane % CH;
    const u32x4 v = *reinterpret_cast<const u32x4*>(stage + r * RB + 16 * (c ^ (r % CH)));
    if (wr0 + r < nrows) {
      const int t = (wr0 + r) / p.group, hd = h * p.group + wr0 + r - t * p.group;
      *reinterpret_cast<u32x4*>(p.out + (int64_t)(sq.row0 + t) * p.ldo + hd * DH + c * VEC) = v;
    }
  }
}

template <typename T>
hipError_t launch_rows(const RowsParams<T>& p, int head_dim, hipStream_t stream) {
  constexpr int BN = sizeof(T) == 2 ? 64 : 32;
  const KeyView& kv = p.kv;
  int64_t grid = rows_items(kv.rows, p.heads, kv.kv_heads, kv.n_seqs, kRowsTile);
  if (p.part) grid = std::max<int64_t>(grid, kRowsRule.limit);
  auto go = [&](auto dh, auto paged) {
    hipLaunchKernelGGL((attn_rows_kernel<T, decltype(dh)::value, BN, decltype(paged)::value>), dim3((unsigned)grid),
                       dim3(256), 0, stream, p);
  };
  auto by_kind = [&](auto dh) {
    if (kv.table) go(dh, std::true_type{});
    else go(dh, std::false_type{});
  };
  if (head_dim == 128) by_kind(std::integral_constant<int, 128>{});
  else if (head_dim == 64) by_kind(std::integral_constant<int, 64>{});
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace dif
