// Key tiles of the chunks' attention kernels in LDS: their layout, and the copies from
// pages or packed rows.
#pragma once
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


// Copies of K and V tiles of BN keys by NW waves, global -> LDS.  Instruction j of a wave
// fills rows (j NW + wave) RPI .. lane by lane; each lane fetches the piece that the
// swizzle puts in its place.  Row to key and the swizzles are linear in the row's
// bits: a lane's part and j's part.
//
// An instruction's rows are keys of one aligned run of 16 (bf16, head_dim 64: of two in
// an aligned 32), so they lie in one page but for the latter and pages of 16: its
// address is then the wave's, looked up with scalar loads a tile ahead, and a lane's
// offset in it the same in every tile.
//
// Keys that no row sees are read from the place of one in the tile that is seen, lane by
// lane.
template <typename T, int DH, int BN, int NW, bool PAGED, bool GAP>
struct TileCopies {
  static constexpr int VEC = Chunk<T>::VEC, ES = (int)sizeof(T), CH = DH / VEC;
  static constexpr int RPI = 64 / CH;             // rows per copy instruction
  static constexpr int NI = BN / (RPI * NW);      // instructions of a wave
  static_assert(NI * RPI * NW == BN, "tile split");
  static constexpr int RUN = RPI > 4 ? 32 : 16;
  typedef u32x4 Tile[BN][CH];
  typedef const __attribute__((address_space(4))) int32_t* table_t;

  const KeyView& kv;
  const Extent<BN, GAP>& ex;
  int key0, lane, wave;
  bool runs;
  const T *kbase, *vbase;
  const int32_t* table;
  uint32_t koff, voff;   // a lane's, in the run (rows of 32 keys span less than 2 GiB)

  __device__ __forceinline__ TileCopies(const KeyView& view, const Sequence& sq, int s, int h, const Extent<BN, GAP>& e)
      : kv(view), ex(e) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    key0 = sq.key0;
    runs = !PAGED || (1 << kv.page_shift) >= RUN;
    kbase = static_cast<const T*>(kv.k) + h * kv.k_head;
    vbase = static_cast<const T*>(kv.v) + h * kv.v_head;
    table = kv.table + s * kv.ld_table;
    const int key = key_of_row(lane / CH);
    koff = (uint32_t)(key * kv.k_slot * ES);
    voff = (uint32_t)(key * kv.v_slot * ES);
  }
  __device__ __forceinline__ int run_key(int j) const { return key_of_row((j * NW + wave) * RPI); }
  // every key of tile i is seen by some row, and its runs lie in pages
  __device__ __forceinline__ bool whole(int i) const { return runs && ex.whole(i); }
  // the pages of tile i's runs
  __device__ __forceinline__ void look_up(int i, int32_t (&page)[NI]) const {
    if constexpr (PAGED) {
      if (whole(i)) {
        const int k0 = i * BN;
#pragma unroll
        for (int j = 0; j < NI; ++j) page[j] = ((table_t)(uintptr_t)table)[(k0 + run_key(j)) >> kv.page_shift];
      }
    }
  }
  // key `key` of tile i, or one that some row sees; seen: (GAP) of the tile's keys, a bit each
  __device__ __forceinline__ uint64_t seen(int i) const { return GAP ? __ballot(ex.sees(i * BN + (lane & (BN - 1)))) : 0; }
  __device__ __forceinline__ int seen_key(int i, uint64_t seen, int key) const {
    if constexpr (!GAP) return ex.nearest(i, i * BN + key);
    const int first = seen ? i * BN + __builtin_ctzll(seen) : ex.before(i);
    return seen >> key & 1 ? i * BN + key : first;
  }
  // bytes from a head's base to key k, in page `page` (a page spans less than 2 GiB, pages
  // lie less than 4 GiB apart, a packed row less than 64 MiB: the host's checks)
  __device__ __forceinline__ uint64_t place(int32_t page, int k, int64_t slot_stride) const {
    const uint32_t slot = (uint32_t)slot_stride * ES;
    if constexpr (PAGED)
      return (uint64_t)min((uint32_t)page, (uint32_t)kv.n_pages - 1) * ((uint32_t)kv.page_stride * ES) +
             (uint32_t)(k & ((1 << kv.page_shift) - 1)) * slot;
    else
      return (uint64_t)(uint32_t)(key0 + k) * slot;
  }
  // tile i of K (or V); page: of look_up
  template <bool IS_V>
  __device__ __forceinline__ void copy(int i, const int32_t (&page)[NI], Tile& to) const {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) void lds_t;
    typedef __attribute__((address_space(1))) void glb_t;
    const int k0 = i * BN;
    const T* base = IS_V ? vbase : kbase;
    const int64_t stride = IS_V ? kv.v_slot : kv.k_slot;
    auto swizzle = [](int r, int c) __attribute__((always_inline)) { return IS_V ? v_swz<T, CH>(r, c) : k_swz(r, c); };
    if (whole(i)) {
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int r = (j * NW + wave) * RPI;
        const char* run = reinterpret_cast<const char*>(base) + place(PAGED ? page[j] : 0, k0 + run_key(j), stride);
        const uint32_t at = (IS_V ? voff : koff) + 16 * (swizzle(lane / CH, lane % CH) ^ swizzle(r, 0));
        __builtin_amdgcn_global_load_lds((glb_t*)(run + at), (lds_t*)&to[r][0], 16, 0, 0);
      }
    } else {
      int ln = lane;
      asm volatile("" : "+v"(ln));   // (nothing of this is kept in registers through the key loop)
      int key[NI];
      int32_t pg[NI];
      const uint64_t seen = this->seen(i);
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        key[j] = seen_key(i, seen, run_key(j) + key_of_row(ln / CH));
        pg[j] = PAGED ? table[key[j] >> kv.page_shift] : 0;
      }
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int r = (j * NW + wave) * RPI;
        const char* at = reinterpret_cast<const char*>(base) + place(pg[j], key[j], stride) +
                         (swizzle(ln / CH, ln % CH) ^ swizzle(r, 0)) * 16;
        __builtin_amdgcn_global_load_lds((glb_t*)at, (lds_t*)&to[r][0], 16, 0, 0);
      }
    }
#endif
  }
};

// Ends a wave's 32 rows, r .. of the row tile at r0: O^T in o (lane % 32 a row; register 4 rr +
// e of o[dt] is dim 32 dt + 8 rr + 4 (lane / 32) + e), this lane's share of the row's
// sum, its base.  A piece leaves them in the workspace; whole rows go out normalised,
// through LDS (32 rows of the type), so that store instructions write whole rows.  A row
// that saw nothing is 0.
template <typename T, int DH>
__device__ __forceinline__ void finish_rows(const RowsParams<T>& p, const Sequence& sq, int h,
                                            const f32x16 (&o)[DH / 32], float l_lane, float m, char* stage, int r0,
                                            int r, int nrows, int bmq, bool piece, int slot, int limit) {
  constexpr int ES = (int)sizeof(T), VEC = 16 / ES, CH = DH / VEC, RB = DH * ES, RPI = 64 / CH;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));   // (no address of this is kept through the key loop)
  const int g = lane >> 5, col = lane & 31;
  const float l = l_lane + __shfl_xor(l_lane, 32);
  if (piece) {
    float* po = part_sums(p.part, slot, r + col, bmq, DH);
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
      float* ml = part_stats(p.part, limit, slot, r + col, bmq, DH);
      ml[0] = m;
      ml[1] = l;
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
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
  for (int i = 0; i < 32 / RPI; ++i) {
    const int q = i * RPI + lane / CH, c = lane % CH;
    const u32x4 v = *reinterpret_cast<const u32x4*>(stage + q * RB + 16 * (c ^ (q % CH)));
    if (r0 + r + q < nrows) {
      const int t = (r0 + r + q) / p.group, hd = h * p.group + r0 + r + q - t * p.group;
      *reinterpret_cast<u32x4*>(p.out + (int64_t)(sq.row0 + t) * p.ldo + hd * DH + c * VEC) = v;
    }
  }
}

}  // namespace dif
