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
#pragma once
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
// every group whatever the groups' widths; else all tiles together are (for groups
// of few tiles, which would leave most of a deal empty).
// Each wave takes 64 groups at a time, a lane a group: tiles before a group by a
// prefix sum over the lanes, once for the total and once more, from the L1, to find
// the group.
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
  int at = block;   // place among the tiles (spread: among the eighths)
  if (!p.spread) {
    int total = 0;
    for (int base = 0; base < p.n_groups; base += kWave) {
      int v = tiles(base + lane);
#pragma unroll
      for (int s = 1; s < kWave; s *= 2) v += __shfl_xor(v, s);
      total += v;
    }
    total = __builtin_amdgcn_readfirstlane(total);
    if (block >= total) return false;
    at = xcd_remap(block, total);
  } else {
    at = block / kXcds;
  }
  for (int base = 0; base < p.n_groups; base += kWave) {
    const int v = tiles(base + lane), unit = p.spread ? (v + kXcds - 1) / kXcds : v;
    int sum = unit;   // inclusive
#pragma unroll
    for (int s = 1; s < kWave; s *= 2) {
      const int o = __shfl_up(sum, s);
      if (lane >= s) sum += o;
    }
    const uint64_t behind = __ballot(sum > at);
    if (behind) {
      const int l = __builtin_ctzll(behind);
      int i = at - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(unit, l));
      const int count = __builtin_amdgcn_readlane(v, l);
      if (p.spread) i += block % kXcds * __builtin_amdgcn_readlane(unit, l);
      if (i >= count) return false;
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
  }
  return false;
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

// Entries j .. j + N (N a multiple of 4) of a row of low, its parts (one, or a
// multiple of four) summed in order, times its adapter's scale; zero from the rank
// on (rows are whole chunks long).
template <int N, typename P>
__device__ __forceinline__ void load_low(const P& p, int row, int j, int rank, float scale, float* v) {
  const float* src = p.low + (int64_t)row * p.ld_low + j;
#pragma unroll
  for (int q = 0; q < N; q += 4) {
    f32x4 x{0.f, 0.f, 0.f, 0.f};
    if (j + q < rank) {
      x = *reinterpret_cast<const f32x4*>(src + q);
      if (p.low_parts > 1) {
        const float* part = src + q;
        f32x4 y[3];
#pragma unroll
        for (int s = 0; s < 3; ++s) y[s] = *reinterpret_cast<const f32x4*>(part + (s + 1) * p.low_stride);
        x += y[0];
        x += y[1];
        x += y[2];
        for (int s = 4; s < p.low_parts; s += 4) {   // (four loads in flight)
          part += 4 * p.low_stride;
          f32x4 z[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) z[i] = *reinterpret_cast<const f32x4*>(part + i * p.low_stride);
#pragma unroll
          for (int i = 0; i < 4; ++i) x += z[i];
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[q + e] = j + q + e < rank ? x[e] * scale : 0.f;
  }
}

// bf16 terms whose sum enters the matrix cores for a 32-bit low: each is the
// rounding of what the ones before leave, so two keep 16 bits, which an output of 8
// cannot tell from all, and three 24 for float32 outputs.
template <typename T, typename OutT>
__host__ __device__ constexpr int low_terms() {
  return sizeof(T) == 4 ? 1 : sizeof(OutT) == 4 ? 3 : 2;
}

// A small tile takes its adapters run by run (about 1.6 us each) up to this many.
constexpr int kFewRuns = 2;

// Calls f(lo, hi, adapter) for the runs of rows with one adapter among rows first ..
// end (neighbouring requests with the same adapter are one run; none for requests
// without).  Every wave of a workgroup walks the same runs.
template <typename T, typename OutT, typename F>
__device__ __forceinline__ void for_adapters(const BatchParams<T, OutT>& p, int first, int end, int lane, F f) {
  // the first request that ends behind row `first`, then 64 at a time
  int q0 = 0;
  for (int base = 0; base < p.n_requests; base += kWave) {
    const int q = base + lane;
    q0 += __builtin_popcountll(__ballot(q < p.n_requests && p.request_off[q + 1] <= first));
  }
  int lo_l = 0, hi_l = 0, a_l = -1, at = -kWave, l = kWave, count = kWave;
  for (;;) {
    if (l == count) {   // the next requests, one per lane
      at += l;
      if (q0 + at >= p.n_requests) return;
      count = min(kWave, p.n_requests - q0 - at);
      l = 0;
      lo_l = hi_l = 0, a_l = -1;
      if (lane < count) {
        table_rows(p.request_off, q0 + at + lane, end, lo_l, hi_l);
        a_l = p.adapter[q0 + at + lane];
        if (a_l < 0 || a_l >= p.n_adapters) a_l = -1;
      }
    }
    const int lo = __builtin_amdgcn_readlane(lo_l, l), a = __builtin_amdgcn_readlane(a_l, l);
    if (lo >= end) return;
    int hi = __builtin_amdgcn_readlane(hi_l, l);
    for (++l; l < count && __builtin_amdgcn_readlane(a_l, l) == a; ++l) hi = __builtin_amdgcn_readlane(hi_l, l);
    if (a >= 0 && hi > max(lo, first)) f(max(lo, first), hi, a);
  }
}

}  // namespace dif
