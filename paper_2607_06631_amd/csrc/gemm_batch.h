// The products of a mixed batch, inside the ring kernel (gemm_ring.h, GA_BATCH):
//
//   rows of group i:  C[r, n] = epi(sum_{k < k_w} A[r, k] B_w[n, k]
//                                   + scale_a sum_{j < r_a} low[r, j] up_a[n, j] + bias_w[n]),  n < n_w
//
// with w the group's matrix and a the adapter of the request that row r belongs
// to; low[r, j] = sum_k A[r, k] down_a[j, k] is itself such a launch (groups =
// requests, matrices = down matrices), so both operators are this one kernel.
//
// The lengths of groups and requests are in device memory, so that a captured
// graph serves any split: the grid covers every split of M rows into the given
// number of groups, each workgroup finds its tile in the table, and those past
// the last tile end.
//
// Bound: the matrix units from about 250 rows a matrix on (65520 x 5120 x 4608 in two
// groups: 1.36 PFLOP/s, as one plain product), the matrices' bytes below (24 rows on 16
// matrices of 8960 x 1536: 62 us, 5.8 TB/s), with adapters for few rows the two launches
// (16 rows of 5120 x 5120, rank 16: 4.8 + 16.6 us).
#pragma once
#include <type_traits>

#include "gemm.h"

namespace dif {

// Where one workgroup works: rows m0 .. (below m_end), columns n0 .. of matrix w,
// whose widths are n and k.
struct BatchTile {
  int m0, m_end, w, n0, n, k;
};

// The running kernel's (first) argument, read anew from where it was passed: what
// only the end of a kernel uses then takes no registers through its k-loop (kept
// there, a 256 x 256 tile spills inside the loop).
template <typename P>
__device__ __forceinline__ const P& kernel_args() {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef const P __attribute__((address_space(4))) args_t;
  args_t* a = (args_t*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(a));
  return *(const P*)a;
#else
  __builtin_unreachable();
#endif
}

__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return min(max(v, lo), hi); }

// Sums over the lanes up to each lane: rows of 16 by shifts, then row 0 into row 1 and
// 2 into 3, then rows 0-1 into 2-3 (see wave_sum).
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ int dpp_add(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROW_MASK, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int v) {
  v = dpp_add<0x111, 0xf>(v);   // row_shr:1
  v = dpp_add<0x112, 0xf>(v);   // row_shr:2
  v = dpp_add<0x114, 0xf>(v);   // row_shr:4
  v = dpp_add<0x118, 0xf>(v);   // row_shr:8
  v = dpp_add<0x142, 0xa>(v);   // row_bcast:15
  return dpp_add<0x143, 0xc>(v);   // row_bcast:31
}

// Rows lo .. hi of entry i of an offset table (whatever it holds: inside 0 .. rows).
__device__ __forceinline__ void table_rows(const int32_t* off, int i, int rows, int& lo, int& hi) {
  lo = clamp_to(off[i], 0, rows);
  hi = clamp_to(off[i + 1], lo, rows);
}

// Tile t of nbm x nbn: groups of GM row tiles that walk the column tiles together.
__device__ __forceinline__ void tile_in_group(int t, int nbm, int nbn, int& mt, int& nt) {
  constexpr int GM = 8;
  const int walk = t / (GM * nbn), first = walk * GM, rows = min(nbm - first, GM), in = t - walk * GM * nbn;
  mt = first + in % rows;
  nt = in / rows;
}

// The tile of workgroup `block`, false if it has none.  Only tiles with something
// to compute count, in the order of the groups.  p.spread: every group's tiles are
// dealt to the eight XCDs in contiguous eighths, so that each XCD gets its share of
// every group whatever the groups' widths; what is left of a group, up to seven
// tiles, goes on from the XCD where the group before stopped, so that the XCDs'
// totals differ by one tile at most (five groups of 77 to 126 tiles, 511 in all:
// 83 us; in eighths rounded up, 42 to 67 tiles an XCD, 113).  Else all tiles together
// are dealt in eighths.
// Each wave takes 64 groups at a time, a lane a group: tiles before a group by a
// prefix sum over the lanes.  (Without the deal the total of all groups is needed
// first.)  0.35 us of a launch for up to 64 groups, most of it the tables' loads.
template <int BM, int BN, typename T, typename OutT>
__device__ __forceinline__ bool batch_tile(const BatchParams<T, OutT>& p, int block, int lane, BatchTile& t) {
  // rows of no request are not computed
  int first = 0, last = p.M;
  if (p.request_off) {
    first = clamp_to(p.request_off[0], 0, p.M);
    last = clamp_to(p.request_off[p.n_requests], first, p.M);
  }
  int lo = 0, hi = 0, w = 0, n = 0;   // of this lane's group
  auto tiles = [&](int i) __attribute__((always_inline)) {
    if (i >= p.n_groups) return 0;
    lo = first, hi = last, w = 0;
    if (p.group_off) {
      table_rows(p.group_off, i, p.M, lo, hi);
      lo = max(lo, first);
      hi = min(hi, last);
      w = p.w_index ? p.w_index[i] : i;
    }
    if (hi <= lo || w < 0 || w >= p.n_weights) return 0;
    n = p.n_kept ? clamp_to(p.n_kept[w], 0, p.N) : p.N;
    return ((hi - lo + BM - 1) / BM) * ((n + BN - 1) / BN);
  };
  const int xcd = block % kXcds;
  int at = p.spread ? block / kXcds : block;   // place among the tiles (spread: this XCD's)
  int v = tiles(lane), upto = wave_scan(v);    // inclusive
  if (!p.spread) {
    int total = __builtin_amdgcn_readlane(upto, kWave - 1);
    if (p.n_groups > kWave) {
      for (int base = kWave; base < p.n_groups; base += kWave)
        total += __builtin_amdgcn_readlane(wave_scan(tiles(base + lane)), kWave - 1);
      tiles(lane);   // (lo, hi, w, n of the first 64 again)
    }
    if (block >= total) return false;
    at = xcd_remap(block, total);
  }
  for (int base = 0, before = 0;;) {
    int unit = v, sum = upto;
    if (p.spread) {
      unit = v / kXcds + ((uint32_t)(xcd - (before + upto - v)) % kXcds < v % kXcds);
      sum = wave_scan(unit);
    }
    const uint64_t behind = __ballot(sum > at);
    if (behind) {
      const int l = __builtin_ctzll(behind);
      int i = at - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(unit, l));
      const int count = __builtin_amdgcn_readlane(v, l);
      if (p.spread) {
        const int part = (uint32_t)(xcd - (before + __builtin_amdgcn_readlane(upto, l) - count)) % kXcds;
        i += part * (count / kXcds) + min(part, count % kXcds);
      }
      // (unsigned: tables whose groups overlap can count past 31 bits)
      if ((uint32_t)i >= (uint32_t)count) return false;
      const int row0 = __builtin_amdgcn_readlane(lo, l);
      t.m_end = __builtin_amdgcn_readlane(hi, l);
      t.w = __builtin_amdgcn_readlane(w, l);
      t.n = __builtin_amdgcn_readlane(n, l);
      t.k = p.k_kept ? clamp_to(__builtin_amdgcn_readfirstlane(p.k_kept[t.w]), 0, p.K) : p.K;
      int mt, nt;
      tile_in_group(i, (t.m_end - row0 + BM - 1) / BM, (t.n + BN - 1) / BN, mt, nt);
      t.m0 = row0 + mt * BM;
      t.n0 = nt * BN;
      return true;
    }
    at -= __builtin_amdgcn_readlane(sum, kWave - 1);
    before += __builtin_amdgcn_readlane(upto, kWave - 1);
    base += kWave;
    if (base >= p.n_groups) return false;
    v = tiles(base + lane);
    upto = wave_scan(v);
  }
}

// The start of a workgroup: finds its tile and leaves the tile's own extents, matrix
// and vectors in p and the references.  False: nothing to do.
template <int BM, int BN, typename T, typename OutT>
__device__ __forceinline__ bool enter_tile(BatchParams<T, OutT>& p, int lane, int& m0, int& n0, const T*& b,
                                           const float*& bias) {
  BatchTile t;
  if (!batch_tile<BM, BN>(p, blockIdx.x, lane, t)) return false;
  m0 = t.m0, n0 = t.n0;
  p.M = t.m_end, p.N = t.n, p.K = t.k;
  b = p.Bs[0] + t.w * p.b_stride;
  bias = p.biases[0] ? p.biases[0] + t.w * p.bias_stride : nullptr;
  if (p.gate1) p.gate1 += t.w * p.gate_stride;
  if (p.k_part) {
    const int k0 = blockIdx.y * p.k_part;
    p.K = clamp_to(p.K - k0, 0, p.k_part);
    p.A += k0;
    b += k0;
    p.C += blockIdx.y * p.c_part;
  }
  return true;
}

// The thread's place again, from the thread number alone: kept through the k-loop,
// these spill beside a 256 x 256 tile.
__device__ __forceinline__ void renew_thread(int& tid, int& lane, int& wave) {
  tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
}

// Elements k .. k + VEC of a row, those from kend on zero and not read.
template <typename T>
__device__ __forceinline__ u32x4 load_chunk_below(const T* row, int k, int kend) {
  constexpr int VEC = Chunk<T>::VEC;
  if (k + VEC <= kend) return *reinterpret_cast<const u32x4*>(row + k);
  typedef T vec_t __attribute__((ext_vector_type(VEC)));
  vec_t v;
#pragma unroll
  for (int e = 0; e < VEC; ++e) v[e] = k + e < kend ? row[k + e] : from_f32<T>(0.f);
  return __builtin_bit_cast(u32x4, v);
}

// Entries j .. j + 4 of a row of low, its parts summed in order (eight in flight).
// Rows are whole chunks of 8 long.
template <typename P>
__device__ __forceinline__ f32x4 load_low4(const P& p, int row, int j) {
  const float* src = p.low + (int64_t)row * p.ld_low + j;
  f32x4 x = *reinterpret_cast<const f32x4*>(src);
  constexpr int PU = 8;
  for (int s = 1; s < p.low_parts; s += PU) {
    f32x4 y[PU];
#pragma unroll
    for (int i = 0; i < PU; ++i)   // (past the last part: the last again, not added)
      y[i] = *reinterpret_cast<const f32x4*>(src + min(s + i, p.low_parts - 1) * p.low_stride);
#pragma unroll
    for (int i = 0; i < PU; ++i)
      if (s + i < p.low_parts) x += y[i];
  }
  return x;
}

// bf16 terms whose sum enters the matrix cores for a 32-bit low: its first bits, then
// those of what the terms before leave.  Two keep 16 bits, which an output of 8 cannot
// tell from all, three 24 for float32 outputs.  All but the last, which is rounded, are
// cut towards zero, so that they have low's sign and none overflows, and a term with
// nothing left for it is 2^-26 of the first instead of zero: an infinite entry of up then
// gives the infinity that it gives with low itself, where terms of both signs or zeros
// would make it NaN.  (Below 2^-100 such a term may be too small for bf16.)
template <typename T, typename OutT>
__host__ __device__ constexpr int low_terms() {
  return sizeof(T) == 4 ? 1 : sizeof(OutT) == 4 ? 3 : 2;
}

// The runs of rows with one adapter among rows first .. end, one after the other
// (neighbouring requests with the same adapter are one run; none for requests
// without), with the adapter's rank and scale.  Every wave of a workgroup walks the
// same runs.
struct AdapterRuns {
  int first, end, lane;
  int at = 0, l = 0, count = 0;   // request at + l is next of `count` that the lanes hold
  int lo_l = 0, hi_l = 0, a_l = -1, rank_l = 0;
  float scale_l = 1.f;
  // the run
  int lo, hi, a, rank;
  float scale;

  template <typename P>
  __device__ __forceinline__ AdapterRuns(const P& p, int first_, int end_, int lane_)
      : first(first_), end(end_), lane(lane_) {
    // past the first 64, the first request that ends behind row `first`
    if (p.n_requests > kWave)
      for (int base = 0; base < p.n_requests; base += kWave) {
        const int q = base + lane;
        at += __builtin_popcountll(__ballot(q < p.n_requests && p.request_off[q + 1] <= first));
      }
    load(p);
  }

  template <typename P>
  __device__ __forceinline__ void load(const P& p) {   // requests at .. , one per lane
    count = clamp_to(p.n_requests - at, 0, kWave);
    l = 0;
    lo_l = hi_l = rank_l = 0, a_l = -1, scale_l = 1.f;
    if (lane < count) {
      table_rows(p.request_off, at + lane, end, lo_l, hi_l);
      a_l = p.adapter[at + lane];
      if (a_l < 0 || a_l >= p.n_adapters || hi_l <= first) a_l = -1;
      if (a_l >= 0) {
        rank_l = p.ranks ? clamp_to(p.ranks[a_l], 0, p.rank) : p.rank;
        if (p.scales) scale_l = p.scales[a_l];
      }
    }
  }

  // the requests behind those at hand, if they can reach the rows
  template <typename P>
  __device__ __forceinline__ bool more(const P& p) {
    at += count;
    if (count == 0 || at >= p.n_requests || __builtin_amdgcn_readlane(lo_l, count - 1) >= end) {
      count = l = 0;   // (the same again if asked again)
      a_l = -1;
      at = p.n_requests;
      return false;
    }
    load(p);
    return true;
  }

  // Row first + lane's adapter, rank and scale from the requests at hand, if one of
  // them holds it (their ends are searched); returns the number of runs that begin
  // among them.
  __device__ __forceinline__ int rows(int& row_a, int& row_rank, float& row_scale) const {
    const bool here = a_l >= 0 && hi_l > lo_l && lo_l < end;
    const int before = __shfl_up(here ? a_l : -1, 1);
    const int row = first + lane, ends = lane < count ? hi_l : INT32_MAX;
    int q = 0;   // requests that end at or before the row
#pragma unroll
    for (int step = kWave / 2; step > 0; step /= 2)
      if (__shfl(ends, q + step - 1) <= row) q += step;
    const int lo_q = __shfl(lo_l, q), hi_q = __shfl(hi_l, q), a_q = __shfl(a_l, q), rank_q = __shfl(rank_l, q);
    const float scale_q = __shfl(scale_l, q);
    if (lo_q <= row && row < hi_q && a_q >= 0) row_a = a_q, row_rank = rank_q, row_scale = scale_q;
    return __builtin_popcountll(__ballot(here && (lane == 0 || before != a_l)));
  }

  template <typename P>
  __device__ __forceinline__ bool next(const P& p) {
    for (;;) {
      // the next request of those at hand that has an adapter and rows here
      const uint64_t some = __ballot(lane >= l && a_l >= 0 && lo_l < end);
      if (some) {
        l = __builtin_ctzll(some);
        a = __builtin_amdgcn_readlane(a_l, l);
        // and those behind it with the same (or no rows)
        const uint64_t others = __ballot(lane > l && lane < count && a_l != a && hi_l > lo_l);
        const int last = (others ? __builtin_ctzll(others) : count) - 1;
        lo = max(__builtin_amdgcn_readlane(lo_l, l), first);
        hi = __builtin_amdgcn_readlane(hi_l, last);
        rank = __builtin_amdgcn_readlane(rank_l, l);
        scale = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scale_l), l));
        l = last + 1;
        if (hi > lo) return true;
        continue;
      }
      if (!more(p)) return false;
    }
  }
};

// What the k-loop leaves of the reduction, elements k0 .. kend of every row (k0 a
// multiple of a chunk, at most CH chunks): through registers into one slot of operand
// rows (BM of A, BN of B), whole chunks where the operands have them, elements at
// their very end, else zeros.  Every tile shape takes the whole chunks in the k-loop's
// places and a last part of one in a step of its own, so that all give the same bits.
template <typename T, typename OutT, int BM, int BN, int AM, int AN, int NW, int CH>
__device__ __forceinline__ void batch_tail(const BatchParams<T, OutT>& p, const T* b_base, int k0, int kend,
                                           f32x4 (&acc)[AM][AN], u32x4 (*s0)[G_BKC], int m0, int n0, int wm, int wn,
                                           int tid) {
  if (k0 >= kend) return;
  constexpr int VEC = Chunk<T>::VEC, ES = sizeof(T), NT = 64 * NW, U = ((BM + BN) * CH + NT - 1) / NT;
  constexpr uint32_t kRsrcWord3 = 0x00020000u;
  const int col = tid & 15, g = (tid & 63) >> 4;
  const T* a_base = p.A + (int64_t)m0 * p.lda;
  const int a_rows = min(BM, p.M - m0), b_rows = min(BN, p.N - n0);
  const __amdgpu_buffer_rsrc_t a_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<T*>(a_base), (short)0, (uint32_t)(a_rows * p.lda * ES), kRsrcWord3);
  const __amdgpu_buffer_rsrc_t b_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<T*>(b_base), (short)0, (uint32_t)(b_rows * p.ldb * ES), kRsrcWord3);
  u32x4 v[U];   // (A's chunks, then B's; whole waves of either)
  static_assert(BM * CH % 64 == 0 && BN * CH % 64 == 0, "one operand per wave and load");
  auto place = [&](int u, bool& is_a, int& r, int& k) __attribute__((always_inline)) {
    const int i = tid + u * NT;
    is_a = __builtin_amdgcn_readfirstlane(i) < BM * CH;
    r = (is_a ? i : i - BM * CH) / CH;
    k = k0 + i % CH * VEC;
    return i < (BM + BN) * CH;
  };
#pragma unroll
  for (int u = 0; u < U; ++u) {
    bool is_a;
    int r, k;
    if (!place(u, is_a, r, k)) continue;
    const bool whole = k + VEC <= kend;
    if (is_a) v[u] = __builtin_amdgcn_raw_buffer_load_b128(a_rsrc, whole ? (uint32_t)((r * p.lda + k) * ES) : kMasked, 0, 0);
    else v[u] = __builtin_amdgcn_raw_buffer_load_b128(b_rsrc, whole ? (uint32_t)((r * p.ldb + k) * ES) : kMasked, 0, 0);
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    bool is_a;
    int r, k;
    if (!place(u, is_a, r, k)) continue;
    if (k < kend && k + VEC > kend && r < (is_a ? a_rows : b_rows))
      v[u] = load_chunk_below(is_a ? a_base + r * p.lda : b_base + r * p.ldb, k, kend);
    s0[is_a ? r : BM + r][swz<G_BKC>(r, (tid + u * NT) % CH)] = v[u];
  }
  __syncthreads();
#pragma unroll
  for (int ks = 0; ks < CH / 4; ++ks) {
    if (k0 + ks * 4 * VEC >= kend) break;
    const int c = swz<G_BKC>(col, 4 * ks + g);
    u32x4 xb[AN];
#pragma unroll
    for (int n = 0; n < AN; ++n) xb[n] = s0[BM + (wn * AN + n) * 16 + col][c];
#pragma unroll
    for (int i = 0; i < AM; ++i) {
      const u32x4 xa = s0[(wm * AM + i) * 16 + col][c];
#pragma unroll
      for (int n = 0; n < AN; ++n) mma16<T>(acc[i][n], xa, xb[n]);
    }
  }
}

// Two floats' upper halves per word: the bf16 numbers next to them towards zero.
template <int N>
__device__ __forceinline__ u32x4 pack_cut(const float (&v)[N]) {
  u32x4 y{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < N / 2; ++w)
    y[w] = __builtin_bit_cast(uint32_t, v[2 * w]) >> 16 | (__builtin_bit_cast(uint32_t, v[2 * w + 1]) & 0xffff0000u);
  return y;
}

// Adds the low-rank terms of the requests that meet the workgroup's tile (rows m0 ..
// m0 + BM below p.M, columns n0 .. n0 + BN below p.N) to its accumulators: wave (wm,
// wn)'s AM x AN tiles of 16 x 16.  s0, s1: two LDS slots of operand rows (BM of A, BN
// of B).  PASSES: what a thread stages is cut in as many, for its registers.
//
// Run after run of rows with one adapter: low's rows as bf16 terms into the A rows of
// the two slots, up's into the B rows of the first, fragments as in the k-loop.  Rows
// and columns outside a run keep what the slots hold: a product's row depends on that
// row of its operands alone, and is added by a select, so that an infinity or NaN of
// one adapter stays with its requests.
template <typename T, typename OutT, int BM, int BN, int AM, int AN, int NW, int PASSES>
__device__ __forceinline__ void add_adapters(const BatchParams<T, OutT>& p, f32x4 (&acc)[AM][AN], u32x4 (*s0)[G_BKC],
                                             u32x4 (*s1)[G_BKC], int m0, int n0, int wm, int wn, int tid) {
  constexpr int VEC = Chunk<T>::VEC, BK = G_BKC * VEC, ES = sizeof(T), NT = 64 * NW;
  constexpr int TERMS = low_terms<T, OutT>();
  static_assert(TERMS < 3 || BN >= BM, "room for three terms");
  constexpr uint32_t kRsrcWord3 = 0x00020000u;
  const int lane = tid & 63, col = lane & 15, g = lane >> 4;
  const BatchParams<T, OutT>& q = kernel_args<BatchParams<T, OutT>>();
  const int m_end = min(m0 + BM, p.M), n_rows = min(BN, p.N - n0);
  auto term_row = [&](int s, int r) __attribute__((always_inline)) -> u32x4* {
    return s == 0 ? s0[r] : s1[s == 1 ? r : BM + r];
  };

  AdapterRuns run(q, m0, m_end, lane);
  constexpr bool SMALL = BM <= 64 && AM * AN <= 4;
  if constexpr (SMALL) {
    // Many short requests (single rows of a batch): run after run would wait for
    // memory once each, about 2 us per 64 of the rank.  Every accumulator's own dot
    // product instead, all adapters' loads in flight together; low's block of the rank
    // waits in the slot.  Its time grows with rank and tile, not with the runs (5120 x
    // 5120, whole calls; run after run second: two rows, rank 16, 20.1 us and 22.4, rank
    // 256 37.3 and 33.1; 8 requests of 4 rows, rank 64, 25.3 and 36.8; on 64 x 64 tiles 4
    // of 20 rows, rank 8, 32.1 and 38.0, rank 64, 47.2 and 39.9; 80 of one row 49 and 161).
    const int few = AM * AN == 1 ? (q.rank <= 32 ? 1 : 2) : clamp_to(q.rank / 10, 2, 10);
    int a_l = -1, rank_l = 0, count = 0;   // of row m0 + lane
    float scale_l = 1.f;
    AdapterRuns all = run;
    do count += all.rows(a_l, rank_l, scale_l);
    while (all.more(q));
    if (count > few) {
      int ra[AM][4];            // of this lane's rows
      const T* up_row[AM][4];
      int64_t up_col[AN];       // (the last column's again past it)
#pragma unroll
      for (int i = 0; i < AM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = (wm * AM + i) * 16 + 4 * g + e;
          ra[i][e] = __shfl(rank_l, r);
          up_row[i][e] = q.up + max(__shfl(a_l, r), 0) * q.up_stride;
        }
#pragma unroll
      for (int n = 0; n < AN; ++n) up_col[n] = min(n0 + (wn * AN + n) * 16 + col, p.N - 1) * q.ld_up;
      // whole chunks everywhere: loads need no branches, chunks from a row's rank on
      // are replaced by zeros
      const bool whole = q.rank % VEC == 0 && !__any(rank_l % VEC);
      static_assert((BM + BN) * G_BKC * sizeof(u32x4) >= (size_t)BM * BK * sizeof(float), "room for low");
      float(*low)[BK] = reinterpret_cast<float(*)[BK]>(&s0[0][0]);
      u32x4 x[AM][4][AN];   // a chunk of every row's and column's up
      auto fetch = [&](int j, auto whole_c) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < AM; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int n = 0; n < AN; ++n) {
              const T* src = up_row[i][e] + up_col[n];
              if constexpr (decltype(whole_c)::value) x[i][e][n] = *reinterpret_cast<const u32x4*>(src + j);
              else x[i][e][n] = load_chunk_below(src, j, ra[i][e]);
            }
      };
      auto blocks = [&](auto whole_c) __attribute__((always_inline)) {
        constexpr bool AHEAD = AM * AN == 1;   // the next chunk one ahead where its registers are few
        fetch(0, whole_c);
        for (int j0 = 0; j0 < q.rank; j0 += BK) {
          const int width = min(q.rank - j0, BK);
          __syncthreads();
          for (int i = tid; i < BM * (BK / 4); i += NT) {   // (whole waves)
            const int r = i / (BK / 4), c = i % (BK / 4) * 4;
            const int rank = __shfl(rank_l, r) - j0 - c;
            const float scale = __shfl(scale_l, r);
            f32x4 v{0.f, 0.f, 0.f, 0.f};
            if (rank > 0) v = load_low4(q, m0 + r, j0 + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = e < rank ? v[e] * scale : 0.f;
            *reinterpret_cast<f32x4*>(&low[r][c]) = v;
          }
          __syncthreads();
          for (int c = 0; c < width; c += VEC) {
            if (!AHEAD && j0 + c > 0) fetch(j0 + c, whole_c);
            u32x4 now[AM][4][AN];
#pragma unroll
            for (int i = 0; i < AM; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int n = 0; n < AN; ++n) now[i][e][n] = x[i][e][n];
            if (AHEAD && j0 + c + VEC < q.rank) fetch(j0 + c + VEC, whole_c);
#pragma unroll
            for (int i = 0; i < AM; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float* lr = &low[(wm * AM + i) * 16 + 4 * g + e][c];
                const bool in = j0 + c < ra[i][e];
#pragma unroll
                for (int n = 0; n < AN; ++n) {
                  float u[VEC];
                  Chunk<T>::unpack(in ? now[i][e][n] : u32x4{0, 0, 0, 0}, u);
#pragma unroll
                  for (int k = 0; k < VEC; ++k) acc[i][n][e] += lr[k] * u[k];
                }
              }
          }
        }
      };
      if (whole) blocks(std::true_type{});
      else blocks(std::false_type{});
      return;
    }
  }

  while (run.next(q)) {
    const int lo = run.lo, hi = run.hi, rank = run.rank;
    const float scale = run.scale;
    const T* up = q.up + run.a * q.up_stride + (int64_t)n0 * q.ld_up;
    // (chunks that are not wholly used get an offset past the descriptors: zeros)
    const __amdgpu_buffer_rsrc_t up_rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<T*>(up), (short)0, (uint32_t)(n_rows * q.ld_up * ES), kRsrcWord3);
    // the run's rows of every part, 32 MiB apart at most in all
    const __amdgpu_buffer_rsrc_t low_rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<float*>(q.low + (int64_t)lo * q.ld_low), (short)0,
        (uint32_t)((q.low_parts - 1) * (int)q.low_stride + (hi - lo) * q.ld_low) * 4u, kRsrcWord3);
    for (int j0 = 0; j0 < rank; j0 += BK) {
      const bool wide = rank - j0 > BK / 2;
      const int lg = wide ? 3 : 2, nc = 1 << lg;   // chunks of the k-steps in use
      // a thread's chunks, UB of up and UA of low at a time: all loads, then all stores
      constexpr int UB = (BN * G_BKC + NT * PASSES - 1) / (NT * PASSES);
      constexpr int UA = (BM * G_BKC + NT * PASSES - 1) / (NT * PASSES);
      const int na = (hi - lo) << lg, nb = n_rows << lg;
      for (int pass = 0; pass < PASSES; ++pass) {
        const int ib = tid + pass * UB * NT, ia = tid + pass * UA * NT;
        u32x4 ub[UB];
        f32x4 ua[UA][VEC / 4];
#pragma unroll
        for (int u = 0; u < UB; ++u) {
          const int i = ib + u * NT, r = i >> lg, j = j0 + (i & (nc - 1)) * VEC;
          ub[u] = __builtin_amdgcn_raw_buffer_load_b128(
              up_rsrc, i < nb && j + VEC <= rank ? (uint32_t)((r * q.ld_up + j) * ES) : kMasked, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < UA; ++u)
#pragma unroll
          for (int k = 0; k < VEC / 4; ++k) ua[u][k] = f32x4{0.f, 0.f, 0.f, 0.f};
        // parts in flight (larger tiles meet at most four: 0.98 to 1.04 of the time)
        constexpr int PU = SMALL && UA * VEC <= 16 ? 16 / (UA * VEC / 4) : 1;
        for (int s = 0; s < q.low_parts; s += PU) {
          f32x4 y[PU][UA][VEC / 4];
#pragma unroll
          for (int t = 0; t < PU; ++t) {
            const uint32_t part = s + t < q.low_parts ? (uint32_t)((s + t) * (int)q.low_stride) * 4u : kMasked;
#pragma unroll
            for (int u = 0; u < UA; ++u) {
              const int i = ia + u * NT, r = i >> lg, j = j0 + (i & (nc - 1)) * VEC;
#pragma unroll
              for (int k = 0; k < VEC / 4; ++k)
                y[t][u][k] = __builtin_bit_cast(
                    f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                               low_rsrc,
                               i < na && j + 4 * k < rank ? part + (uint32_t)(r * q.ld_low + j + 4 * k) * 4u : kMasked, 0,
                               0));
            }
          }
#pragma unroll
          for (int t = 0; t < PU; ++t)
#pragma unroll
            for (int u = 0; u < UA; ++u)
#pragma unroll
              for (int k = 0; k < VEC / 4; ++k) ua[u][k] += y[t][u][k];
        }
        if (pass == 0) __syncthreads();   // the slots are free
#pragma unroll
        for (int u = 0; u < UB; ++u) {
          const int i = ib + u * NT, r = i >> lg, c = i & (nc - 1), j = j0 + c * VEC;
          if (i >= nb) continue;
          if (j < rank && j + VEC > rank) ub[u] = load_chunk_below(up + r * q.ld_up, j, rank);
          s0[BM + r][swz<G_BKC>(r, c)] = ub[u];
        }
#pragma unroll
        for (int u = 0; u < UA; ++u) {
          const int i = ia + u * NT, row = lo + (i >> lg) - m0, c = i & (nc - 1), j = j0 + c * VEC;
          if (i >= na) continue;
          float v[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) v[e] = j + e < rank ? ua[u][e / 4][e % 4] * scale : 0.f;
          const int pc = swz<G_BKC>(row, c);
          float least[VEC];   // what stands for nothing left
#pragma unroll
          for (int s = 0; s < TERMS; ++s) {
            const bool last = s + 1 == TERMS;
            const u32x4 y = last ? Chunk<T>::pack(v) : pack_cut(v);
            term_row(s, row)[pc] = y;
            if (!last) {
              float back[VEC];
              Chunk<T>::unpack(y, back);
#pragma unroll
              for (int e = 0; e < VEC; ++e) {
                if (s == 0) least[e] = back[e] * 0x1p-26f;
                const float left = v[e] - back[e];   // (NaN of an infinity)
                v[e] = __builtin_fabsf(left) > 0.f ? left : least[e];
              }
            }
          }
        }
      }
      __syncthreads();
      for (int ks = 0; ks < nc / 4; ++ks) {
        const int c = swz<G_BKC>(col, 4 * ks + g);
        u32x4 xb[AN];
#pragma unroll
        for (int n = 0; n < AN; ++n) xb[n] = s0[BM + (wn * AN + n) * 16 + col][c];
#pragma unroll
        for (int i = 0; i < AM; ++i) {
          const int tr = (wm * AM + i) * 16, r0 = m0 + tr;
          if (r0 >= hi || r0 + 16 <= lo) continue;
          // (formed here for each i, not kept in registers beside acc)
          int quad = 4 * g;
          asm volatile("" : "+v"(quad));
          u32x4 xa[TERMS];
#pragma unroll
          for (int s = 0; s < TERMS; ++s) xa[s] = term_row(s, tr + col)[c];
#pragma unroll
          for (int n = 0; n < AN; ++n) {
            f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = TERMS - 1; s >= 0; --s) mma16<T>(v, xa[s], xb[n]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int row = r0 + quad + e;
              acc[i][n][e] += row >= lo && row < hi ? v[e] : 0.f;
            }
          }
        }
      }
    }
  }
}

// Workgroups of a launch in BM x BN tiles, as many as any split of the rows makes,
// and how they are dealt out.  Groups of few tiles (less than 64 in the mean) are not
// dealt each: an XCD reads whole matrices then, where the deal has all eight read each
// (9 groups, 847 x 196 x 6860: 16.3 us, dealt 18.5; 13 groups, 13012 x 651 x 1805: 61.2
// and 65.1); from 64 on it is even or the deal better, up to the case above.
template <int BM, int BN, typename P>
dim3 batch_grid(P& p) {
  const int64_t g = p.n_groups < p.M ? p.n_groups : p.M;
  int64_t tiles = (p.M + g * (BM - 1)) / BM * ((p.N + BN - 1) / BN);
  p.spread = tiles >= 64 * g;
  if (p.spread) tiles = (tiles + kXcds - 1) / kXcds * kXcds;
  return dim3((unsigned)tiles, p.k_part ? p.parts : 1);
}

// gemm.hip's 256 x 256 kernel over a mixed batch of bf16 operands
template <typename OutT>
hipError_t launch_gemm_batch_256(const BatchParams<bf16, OutT>& p, int epi, hipStream_t s);

}  // namespace dif
