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
#include <cmath>
#include <type_traits>

#include "stream.h"

namespace dif {

constexpr float kRowsSlack = 8.f;      // log2 headroom of the lazy rescale
constexpr float kNoBase = -1e38f;      // base before a row's first key: any key's score moves it
constexpr int kRowsTile = 128;         // rows of a workgroup

template <typename T>
struct RowsParams {
  KeyView kv;
  const T* q;
  T* out;
  int64_t ldq, ldo;
  int heads, group;    // query heads, and how many share a key head
  SeenMask mask;
  float c;             // log2(e) / sqrt(head_dim): scores to base-2 exponents
};

// What the row at position p sees: keys below sinks and from start to end.
struct Seen {
  int start, end;
};
__device__ __forceinline__ Seen seen_by(const SeenMask& m, int p, int length) {
  if (m.block > 0 && p < 0) return {0, 0};
  // (p + block may pass 2^31)
  const int64_t e = m.block > 0 ? ((int64_t)(p / m.block) + 1) * m.block : length;
  const int end = (int)min(e, (int64_t)length);
  const int start = m.window > 0 ? (int)min(max(e - m.window, (int64_t)0), (int64_t)end) : 0;
  return {start, end};
}

// Sequence s: its rows and keys.
struct Sequence {
  int row0, rows, keys, key0;
};
__device__ __forceinline__ Sequence sequence(const KeyView& kv, int s) {
  Sequence q;
  int hi;
  seq_rows(kv, s, &q.row0, &hi);
  q.rows = hi - q.row0;
  q.key0 = 0;
  if (kv.table) {
    q.keys = min(max(kv.lengths[s], 0), kv.max_keys);
  } else {
    q.key0 = min(max(kv.key_off[s], 0), kv.max_keys);
    q.keys = min(max(kv.key_off[s + 1], q.key0), kv.max_keys) - q.key0;
  }
  return q;
}

// Sums over the lanes below, this one included.
__device__ __forceinline__ int wave_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int t = __shfl_up(v, d);
    if (lane >= d) v += t;
  }
  return v;
}

// Finds item i of the list of row tiles, sequence by sequence (each wave for itself):
// its sequence and which of its tiles it is; -1 past the end.  *total: all items.
__device__ __forceinline__ int find_item(const KeyView& kv, int group, int bmq, int i, int* tile, int* total) {
  const int lane = threadIdx.x & 63, n = kv.n_seqs;
  auto tiles = [&](int s) __attribute__((always_inline)) {
    int lo, hi;
    seq_rows(kv, s, &lo, &hi);
    return (int)(((int64_t)(hi - lo) * group + bmq - 1) / bmq);
  };
  // a lane takes `per` sequences; then the lanes take that lane's
  const int per = (n + 63) / 64, s0 = lane * per;
  int mine = 0;
  for (int j = 0; j < per && s0 + j < n; ++j) mine += tiles(s0 + j);
  int upto = wave_scan(mine);
  *total = __shfl(upto, 63);
  if (i >= *total) return -1;
  int at = __ffsll((long long)__ballot(upto > i)) - 1;
  int before = __shfl(upto - mine, at);
  int s = at * per;
  if (per > 1) {   // (per <= 64: n_seqs is limited)
    mine = lane < per && s + lane < n ? tiles(s + lane) : 0;
    upto = before + wave_scan(mine);
    at = __ffsll((long long)__ballot(upto > i)) - 1;
    before = __shfl(upto - mine, at);
    s += at;
  }
  *tile = i - before;
  return __builtin_amdgcn_readfirstlane(s);
}

// LDS place of 16-byte piece c in row `row` of a V tile (CH pieces a row).  bf16: a
// transposing read takes 64 bytes of four consecutive rows; float32: 128 bytes of
// rows four apart.  Both then meet different banks.
template <typename T, int CH>
__device__ __forceinline__ int v_swz(int row, int c) {
  if constexpr (sizeof(T) == 4) return c ^ (((row >> 2) & 1) << 3);
  else if constexpr (CH == 16) return c ^ ((row & 3) << 2);
  else return c ^ (((row >> 1) & 1) << 2);
}

// SC: queries arrive multiplied by log2(e) / sqrt(dh).  PAGED: kv has a table.
template <typename T, int DH, int BN, bool SC, bool PAGED>
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
  __shared__ u32x4 ks[2][BN][CH];
  __shared__ u32x4 vs[2][BN][CH];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 5, col = lane & 31;
  const KeyView& kv = p.kv;

  // this workgroup's item; heads outermost, so that an XCD's workgroups share keys
  int items, tile_of = 0;
  find_item(kv, p.group, BMQ, 0, &tile_of, &items);
  const int64_t all = (int64_t)items * kv.kv_heads;
  if ((int64_t)blockIdx.x >= all) return;
  const int idx = xcd_remap(blockIdx.x, (int)all);
  const int h = idx / items;
  const int s = find_item(kv, p.group, BMQ, idx - h * items, &tile_of, &items);
  const Sequence sq = sequence(kv, s);
  const int nrows = sq.rows * p.group;
  // the last tiles see the most keys: first
  const int r0 = (((nrows + BMQ - 1) / BMQ) - 1 - tile_of) * BMQ;
  const int shift = sq.keys - sq.rows;     // position of the first row

  // keys that some row of the workgroup sees: [0, sinks) and [lo, hi)
  const int rlast = min(r0 + BMQ, nrows) - 1;
  const Seen first = seen_by(p.mask, shift + r0 / p.group, sq.keys);
  const Seen last = seen_by(p.mask, shift + rlast / p.group, sq.keys);
  const int lo = first.start, hi = last.end;
  const int sinks = p.mask.window > 0 ? min(p.mask.sinks, hi) : 0;
  const int w0 = lo < hi ? lo / BN : (hi + BN - 1) / BN;   // the window's tiles, none if it is empty
  const int nsink = min((sinks + BN - 1) / BN, w0);
  const int ntiles = nsink + (hi + BN - 1) / BN - w0;
  auto key_of = [&](int i) __attribute__((always_inline)) { return (i < nsink ? i : w0 + i - nsink) * BN; };

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
  // by lane; each lane fetches the piece that the swizzle puts in its place.
  [[maybe_unused]] const T* kbase = static_cast<const T*>(kv.k) + h * kv.k_head;
  [[maybe_unused]] const T* vbase = static_cast<const T*>(kv.v) + h * kv.v_head;
  int koff[NI], kc[NI], vc[NI];   // key in the tile, piece of K and of V
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const int r = (j * NW + wave) * RPI + lane / CH, i = r & 31;
    koff[j] = (r & ~31) + 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3);
    kc[j] = swz<CH>(r, lane % CH) * VEC;
    vc[j] = v_swz<T, CH>(r, lane % CH) * VEC;
  }
  int key[NI], page[NI];
  auto look_up = [&](int i) __attribute__((always_inline)) {   // places of tile i's keys
    const int k0 = key_of(i);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      int k = k0 + koff[j];
      if (k >= sinks) k = lo < hi ? min(max(k, lo), hi - 1) : sinks - 1;
      key[j] = k;
      if constexpr (PAGED) page[j] = kv.table[s * kv.ld_table + (k >> kv.page_shift)];
    }
  };
  auto copy = [&](int buf) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) void lds_t;
    typedef __attribute__((address_space(1))) void glb_t;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      int64_t ko, vo;
      if constexpr (PAGED) {
        const int64_t pg = (int64_t)min((uint32_t)page[j], (uint32_t)kv.n_pages - 1) * kv.page_stride;
        const int64_t slot = key[j] & ((1 << kv.page_shift) - 1);
        ko = pg + slot * kv.k_slot;
        vo = pg + slot * kv.v_slot;
      } else {
        ko = (int64_t)(sq.key0 + key[j]) * kv.k_slot;
        vo = (int64_t)(sq.key0 + key[j]) * kv.v_slot;
      }
      const int r = (j * NW + wave) * RPI;
      __builtin_amdgcn_global_load_lds((glb_t*)(kbase + ko + kc[j]), (lds_t*)&ks[buf][r][0], 16, 0, 0);
      __builtin_amdgcn_global_load_lds((glb_t*)(vbase + vo + vc[j]), (lds_t*)&vs[buf][r][0], 16, 0, 0);
    }
#endif
  };

  f32x16 o[DH / 32];
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  float l_run = 0.f, m_run = kNoBase;
  bool masked = false;
  f32x16 zero, negm;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    zero[r] = 0.f;
    negm[r] = -kNoBase;
  }

  auto scores = [&](int buf, int kk, const f32x16& c0) __attribute__((always_inline)) {
    constexpr int KB = NQS >= 8 ? NQS / 2 : NQS;
    f32x16 sc = c0;
#pragma unroll
    for (int s0 = 0; s0 < NQS; s0 += KB) {
      u32x4 kf[KB];
#pragma unroll
      for (int st = 0; st < KB; ++st) kf[st] = ks[buf][kk * 32 + col][swz<CH>(col, 2 * (s0 + st) + g)];
#pragma unroll
      for (int st = 0; st < KB; ++st) Mma<T>::step(sc, kf[st], qf[s0 + st]);
    }
    return sc;
  };
  // hidden keys of the 32 from key0 on -> -inf
  auto mask = [&](f32x16& sc, int key0) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int k = key0 + 16 * g + r;
      if (!(k < mine.end && (k >= mine.start || k < sinks))) sc[r] = -INFINITY;
    }
  };
  // V^T piece u of dims 32 dt + col: this lane group's keys 16 g + VEC u .. of half kk
  auto v_piece = [&](int buf, int kk, int u, int dt) __attribute__((always_inline)) {
    u32x4 f;
    if constexpr (ES == 2) {
#if defined(__HIP_DEVICE_COMPILE__)
      typedef short s4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s4 lds4_t;
      const int c = 4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      u32x2 part[2];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int r = kk * 32 + 8 * (2 * u + hh) + 4 * g + ((lane & 15) >> 2);
        const char* at = reinterpret_cast<const char*>(&vs[buf][r][v_swz<T, CH>(r, c)]) + 8 * (lane & 1);
        part[hh] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t*)at));
      }
      f = u32x4{part[0][0], part[0][1], part[1][0], part[1][1]};
#endif
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = kk * 32 + 8 * u + 4 * g + e;
        f[e] = reinterpret_cast<const uint32_t*>(&vs[buf][r][v_swz<T, CH>(r, 8 * dt + (col >> 2))])[col & 3];
      }
    }
    return f;
  };

  auto tile = [&](int i, auto buf, auto masked_c) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked_c)::value;
    const int key0 = key_of(i);
    auto half = [&](int kk) __attribute__((always_inline)) {
      __builtin_amdgcn_sched_barrier(0);
      f32x16 sc = scores(buf, kk, SC ? negm : zero);
      if (MASKED) mask(sc, key0 + 32 * kk);
      constexpr bool EARLY = !MASKED && ES == 2;   // V^T's operands on their way during the softmax
      u32x4 vf[NPC][DH / 32];
      if constexpr (EARLY) {
#pragma unroll
        for (int u = 0; u < NPC; ++u)
#pragma unroll
          for (int dt = 0; dt < DH / 32; ++dt) vf[u][dt] = v_piece(buf, kk, u, dt);
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
            pv[e] = __builtin_amdgcn_exp2f(SC ? x : fmaf(x, scale, -base));
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
      // numbers).  The scores are then taken anew: against a base far off they have lost their
      // digits (the first key of every row).
      if (__any(!(lh <= (float)(1 << (int)kRowsSlack)))) {
        sc = scores(buf, kk, zero);
        if (MASKED) mask(sc, key0 + 32 * kk);
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
        const float m_new = fmaxf(m_run, fmaxf(mx, __shfl_xor(mx, 32)) * (SC ? 1.f : p.c));
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
        m_run = m_new;
        if constexpr (SC) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            sc[r] -= m_new;
            negm[r] = -m_new;
          }
        }
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
          for (int dt = 0; dt < DH / 32; ++dt) Mma<T>::step(z, v_piece(buf, kk, u, dt), u32x4{0u, 0u, 0u, 0u});
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
              u32x4 one = v_piece(buf, kk, u, dt);
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
          else Mma<T>::step(o[dt], v_piece(buf, kk, u, dt), pc[u]);
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
  // (the two buffers of plain tiles are compile-time, so that addresses are immediates)
  auto visit = [&](int i, auto buf_c) __attribute__((always_inline)) {
    constexpr int buf = decltype(buf_c)::value;
    // the next tile's copies (its buffer was last read before the barrier), the places of the one after it
    if (i + 1 < ntiles) copy(buf ^ 1);
    if (i + 2 < ntiles) look_up(i + 2);
    const int k0 = key_of(i), k1 = k0 + BN;
    if (!idle && k0 < wlast.end && (k1 > wfirst.start || k0 < sinks)) {
      if (k1 <= wfirst.end && (k0 >= wlast.start || k1 <= sinks)) tile(i, buf, std::false_type{});
      else masked = true;
    }
  };
  auto landed = [&]() __attribute__((always_inline)) {
    wait_vmcnt<0>();   // this wave's copies have landed
    __syncthreads();   // ... and every other wave's
  };
  if (ntiles > 0) {
    look_up(0);
    copy(0);
    if (ntiles > 1) look_up(1);
    landed();
  }
  for (int i = 0; i < ntiles; ++i) {
    masked = false;
    if (i & 1) visit(i, std::integral_constant<int, 1>{});
    else visit(i, std::integral_constant<int, 0>{});
    if (masked) tile(i, i & 1, std::true_type{});
    landed();
  }
  if (idle) return;

  // Output rows through LDS, so that store instructions write whole rows: a lane holds
  // four consecutive dims of its row per register group.  A row that saw nothing is 0.
  const float l = l_run + __shfl_xor(l_run, 32);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  constexpr int RB = DH * ES;
  constexpr int SRPI = 64 / CH;
  char* stage = (wave < 2 ? reinterpret_cast<char*>(&ks[0][0][0]) : reinterpret_cast<char*>(&vs[0][0][0])) +
                (wave & 1) * 32 * RB;
  static_assert(2 * 32 * RB <= (int)sizeof(ks), "staging");
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
hipError_t launch_attention_rows(const KeyView& kv, int head_dim, const T* q, int64_t ldq, T* out, int64_t ldo,
                                 int heads, const SeenMask& mask, bool q_scaled, float* part, hipStream_t stream) {
  constexpr int BN = sizeof(T) == 2 ? 64 : 32;
  RowsParams<T> p{kv, q, out, ldq, ldo, heads, heads / kv.kv_heads, mask,
                  (float)(1.4426950408889634 / std::sqrt((double)head_dim))};
  (void)part;
  const dim3 grid((unsigned)rows_items(kv.rows, heads, kv.kv_heads, kv.n_seqs, kRowsTile));
  auto go = [&](auto dh, auto sc, auto paged) {
    hipLaunchKernelGGL((attn_rows_kernel<T, decltype(dh)::value, BN, decltype(sc)::value, decltype(paged)::value>), grid,
                       dim3(256), 0, stream, p);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  auto by_kind = [&](auto dh) {
    if constexpr (sizeof(T) == 2) {
      if (q_scaled) {
        kv.table ? go(dh, Yes{}, Yes{}) : go(dh, Yes{}, No{});
        return;
      }
    }
    if (q_scaled) p.c = 1.f;   // (float32: one form, whose products a scale costs nothing beside)
    kv.table ? go(dh, No{}, Yes{}) : go(dh, No{}, No{});
  };
  if (head_dim == 128) by_kind(std::integral_constant<int, 128>{});
  else if (head_dim == 64) by_kind(std::integral_constant<int, 64>{});
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

#define DIF_ROWS_INSTANCE(T)                                                                                     \
  template hipError_t launch_attention_rows<T>(const KeyView&, int, const T*, int64_t, T*, int64_t, int,        \
                                               const SeenMask&, bool, float*, hipStream_t);

}  // namespace dif
