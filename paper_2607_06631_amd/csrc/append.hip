// Appending new tokens to a paged cache (dif_cache_append): queries and keys
// normalised, rotated and scaled on the way, keys and values written to their pages.
//
//   y = x / sqrt(sum(x^2) / norm_dim + eps) * gain,   pairs turned by position * freq
//
// HBM-bound: every row of q, k and v is read and written once.  A wave takes one row
// of one of the three and holds it in registers, 16-byte pieces, so the norm's sum
// and the rotation cost no second read.  A lane's pieces are 64 pieces apart, a whole
// number of heads, so it meets the same pairs in all of them: it computes one set
// of angles a row.  Rows and results are read and written once, past the caches' use
// (nontemporal), which leaves L2 to the gains: 4680 rows of q, k and v of 5120 bf16, 288 MB
// in other memory every time, take 57 us (5.05 TB/s; a copy of as much 58), 71 without;
// all rows of one of the three before the next, 57 against 59 with a row's three together.
//
// Angles without a table and without 64-bit floats: a pair's turns per position is
// a fraction of 2^64, and position * freq mod 2^64 is the fraction of a turn, exact to
// the host's rounding of freq (2^-64 of a turn per position).  Its nearest quarter is
// taken off as an integer, the rest (within an eighth of a turn) goes through the
// Taylor series of sine and cosine, both good to 2^-24.
#include <algorithm>

#include "stream.h"

namespace dif {

namespace {

__device__ __forceinline__ void turn(uint64_t phase, float* cs, float* sn) {
  const uint32_t top = (uint32_t)(phase >> 32);
  const uint32_t quarter = (top + 0x20000000u) >> 30;
  const float y = (float)(int32_t)(top - (quarter << 30)) * 1.4629180792671596e-9f;   // pi 2^-31
  const float z = y * y;
  float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);   // 1/9!, -1/7!
  s = fmaf(z, s, 8.3333333e-3f);
  s = fmaf(z, s, -1.6666667e-1f);
  s = fmaf(y * z, s, y);
  float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);   // -1/10!, 1/8!
  c = fmaf(z, c, -1.3888889e-3f);
  c = fmaf(z, c, 4.1666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.f);
  const bool swap = quarter & 1;
  const float a = swap ? s : c, b = swap ? c : s;
  *cs = (quarter + 1) & 2 ? -a : a;   // quarters 1 and 2
  *sn = quarter & 2 ? -b : b;         // quarters 2 and 3
}

enum Part { PART_K = 0, PART_V, PART_Q };

// The row's pieces are held whole when they are normalised (MAXC of them a lane);
// other rows of any width take turns of MAXC.
template <typename T, int DH, int MAXC>
__global__ __launch_bounds__(256) void append_kernel(KeyView kv, const T* k, int64_t ldk, const T* v, int64_t ldv,
                                                     const T* q, int64_t ldq, T* q_out, int64_t ldo, int heads,
                                                     AppendDesc d, int parts) {
  constexpr int VEC = Chunk<T>::VEC, NP = VEC / 2, CPH = DH / VEC;   // pieces per head
  static_assert(64 % CPH == 0, "a lane's pieces lie whole heads apart");
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int part = (int)(w / kv.rows), row = (int)(w % kv.rows);
  if (part >= parts) return;   // (the last workgroup's spare waves)

  const T* src = part == PART_K ? k + row * ldk : part == PART_V ? v + row * ldv : q + row * ldq;
  const int nch = (part == PART_Q ? heads : kv.kv_heads) * CPH;
  u32x4 x[MAXC];
  auto load = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = c0 + lane + 64 * i;
      if (c < nch) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + c * VEC));
    }
  };
  load(0);   // (on its way during the lookups)

  const int s = __builtin_amdgcn_readfirstlane(seq_of_row(kv, row));
  int lo, hi;
  seq_rows(kv, s, &lo, &hi);
  if (row < lo || row >= hi) return;   // a row of no sequence
  const int64_t at = (int64_t)kv.lengths[s] - (hi - row);   // its token's index in the sequence
  T* dst;          // of head 0
  int64_t dst_head;
  if (part == PART_Q) {
    dst = q_out + row * ldo;
    dst_head = DH;
  } else {
    if (at < 0 || at >= kv.max_keys) return;
    const int page = kv.table[s * kv.ld_table + (at >> kv.page_shift)];
    if ((uint32_t)page >= (uint32_t)kv.n_pages) return;
    const int64_t slot = at & ((1 << kv.page_shift) - 1);
    dst = static_cast<T*>(part == PART_K ? kv.k : kv.v) + page * kv.page_stride +
          slot * (part == PART_K ? kv.k_slot : kv.v_slot);
    dst_head = part == PART_K ? kv.k_head : kv.v_head;
  }

  const bool turned = part != PART_V && d.axes > 0;
  float cs[NP], sn[NP];
  if (turned) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int pair = (lane % CPH) * NP + j;
      const int axis = d.axes == 1 ? 0 : (pair >= d.axis1) + (pair >= d.axis2);
      const int64_t pos = d.positions ? (int64_t)d.positions[(int64_t)row * d.axes + axis] : at;
      turn((uint64_t)pos * d.freq[pair], &cs[j], &sn[j]);
    }
  }
  const float* gain = part == PART_Q ? d.gain_q : part == PART_K ? d.gain_k : nullptr;
  const float scale = part == PART_Q ? d.q_scale : 1.f;
  float inv = 1.f;
  if (gain) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      if (lane + 64 * i >= nch) continue;
      float e[VEC];
      Chunk<T>::unpack(x[i], e);
#pragma unroll
      for (int j = 0; j < VEC; ++j) ss = fmaf(e[j], e[j], ss);
    }
    inv = 1.f / sqrtf(wave_sum(ss) * (part == PART_Q ? d.inv_dim_q : d.inv_dim_k) + d.eps);
  }
  inv *= scale;
  const bool plain = !turned && !gain && scale == 1.f;
  for (int c0 = 0;;) {
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
      const int c = c0 + lane + 64 * i;
      if (c >= nch) continue;
      u32x4 y = x[i];
      if (!plain) {
        float e[VEC];
        Chunk<T>::unpack(y, e);
#pragma unroll
        for (int j = 0; j < VEC; j += 4) {
          const f32x4 gn = gain ? *reinterpret_cast<const f32x4*>(gain + c * VEC + j) : f32x4{1.f, 1.f, 1.f, 1.f};
#pragma unroll
          for (int h = 0; h < 4; ++h) e[j + h] *= inv * gn[h];
        }
        if (turned) {
#pragma unroll
          for (int j = 0; j < NP; ++j) {
            const float a = e[2 * j], b = e[2 * j + 1];
            e[2 * j] = a * cs[j] - b * sn[j];
            e[2 * j + 1] = a * sn[j] + b * cs[j];
          }
        }
        y = Chunk<T>::pack(e);
      }
      __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(dst + (c / CPH) * dst_head + (c % CPH) * VEC));
    }
    c0 += 64 * MAXC;
    if (c0 >= nch) break;
    load(c0);
  }
}

}  // namespace

template <typename T>
hipError_t launch_append(const KeyView& kv, int head_dim, const T* k, int64_t ldk, const T* v, int64_t ldv,
                         const T* q, int64_t ldq, T* q_out, int64_t ldo, int heads, const AppendDesc& d,
                         hipStream_t stream) {
  const int parts = q ? 3 : 2;
  const int wide = std::max(q ? heads : 0, kv.kv_heads) * head_dim;
  const int per = (wide / Chunk<T>::VEC + 63) / 64;   // pieces a lane
  const dim3 grid((unsigned)(((int64_t)kv.rows * parts + 3) / 4));
  auto go = [&](auto dh, auto maxc) {
    hipLaunchKernelGGL((append_kernel<T, decltype(dh)::value, decltype(maxc)::value>), grid, dim3(256), 0, stream, kv, k,
                       ldk, v, ldv, q, ldq, q_out, ldo, heads, d, parts);
  };
  auto by_width = [&](auto dh) {
    if (per <= 2) go(dh, std::integral_constant<int, 2>{});
    else if (per <= 6) go(dh, std::integral_constant<int, 6>{});
    else if (per <= 10) go(dh, std::integral_constant<int, 10>{});
    else go(dh, std::integral_constant<int, 16>{});
  };
  if (head_dim == 128) by_width(std::integral_constant<int, 128>{});
  else if (head_dim == 64) by_width(std::integral_constant<int, 64>{});
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

template hipError_t launch_append<float>(const KeyView&, int, const float*, int64_t, const float*, int64_t,
                                         const float*, int64_t, float*, int64_t, int, const AppendDesc&, hipStream_t);
template hipError_t launch_append<bf16>(const KeyView&, int, const bf16*, int64_t, const bf16*, int64_t, const bf16*,
                                        int64_t, bf16*, int64_t, int, const AppendDesc&, hipStream_t);

}  // namespace dif
