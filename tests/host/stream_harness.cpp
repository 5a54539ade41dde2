// The streamed-generation entry points (csrc/stream.cpp) on the host under
// AddressSanitizer and UndefinedBehaviorSanitizer: the kernels' launches are stand-ins that
// read the tables (host memory here) and touch the places of every token that the kernels
// address, so that a size that the checks let through or pass on wrongly becomes an
// out-of-bounds access.  Test infrastructure only.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../include/dif.h"
#include "../../paper_2607_06631_amd/csrc/kernels.h"

hipError_t hipEventCreate(hipEvent_t*) { return hipErrorInvalidValue; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipErrorInvalidValue; }
const char* hipGetErrorString(hipError_t) { return "stub error"; }

static long g_launches = 0;
static hipError_t g_result = hipSuccess;
static volatile unsigned char g_sink;

template <typename T>
static void touch(const T* p, int64_t n, bool write = false) {
  for (int64_t i : {int64_t(0), n - 1}) {
    if (write) ((volatile unsigned char*)(p + i))[0] = 1;
    else g_sink = ((const unsigned char*)(p + i))[sizeof(T) - 1];
  }
}

namespace dif {
template <typename T>
static void rows(const T* p, const KeyView& kv, int64_t ld, int64_t wide, bool write = false) {
  for (int r : {0, kv.rows - 1}) touch(p + r * ld, wide, write);
}
// every token that the tables name
template <typename T>
static void tokens(const KeyView& kv, int dh, bool write) {
  for (int s = 0; s < kv.n_seqs; ++s) {
    const int lo = std::min(std::max(kv.row_off[s], 0), kv.rows), hi = std::min(std::max(kv.row_off[s + 1], lo), kv.rows);
    g_sink = (unsigned char)(hi - lo);
    int k0 = 0, n;
    if (kv.table) {
      n = std::min(std::max(kv.lengths[s], 0), kv.max_keys);
    } else {
      k0 = std::min(std::max(kv.key_off[s], 0), kv.max_keys);
      n = std::min(std::max(kv.key_off[s + 1], k0), kv.max_keys) - k0;
    }
    for (int j = 0; j < n; ++j)
      for (int h = 0; h < kv.kv_heads; ++h) {
        int64_t page = 0, slot = k0 + j;
        if (kv.table) {
          page = std::min<uint32_t>(kv.table[s * kv.ld_table + (j >> kv.page_shift)], kv.n_pages - 1);
          slot = j & ((1 << kv.page_shift) - 1);
        }
        touch((T*)kv.k + page * kv.page_stride + h * kv.k_head + slot * kv.k_slot, dh, write);
        touch((T*)kv.v + page * kv.page_stride + h * kv.v_head + slot * kv.v_slot, dh, write);
      }
  }
}
template <typename T>
hipError_t launch_append(const KeyView& kv, int dh, const T* k, int64_t ldk, const T* v, int64_t ldv, const T* q,
                         int64_t ldq, T* q_out, int64_t ldo, int heads, const AppendDesc& d, hipStream_t) {
  ++g_launches;
  rows(k, kv, ldk, (int64_t)kv.kv_heads * dh);
  rows(v, kv, ldv, (int64_t)kv.kv_heads * dh);
  if (q) {
    rows(q, kv, ldq, (int64_t)heads * dh);
    rows(q_out, kv, ldo, (int64_t)heads * dh, true);
  }
  if (d.gain_k) touch(d.gain_k, kv.kv_heads * dh);
  if (d.gain_q) touch(d.gain_q, heads * dh);
  if (d.positions) touch(d.positions, (int64_t)kv.rows * d.axes);
  if (d.axes && (d.axis1 > dh / 2 || d.axis2 > dh / 2 || d.freq[0] == 0 || d.freq[dh / 2 - 1] == 0)) std::abort();
  tokens<T>(kv, dh, true);
  return g_result;
}
size_t attention_rows_bytes(int head_dim) { return 256 * (head_dim + 2); }
template <typename T>
hipError_t launch_attention_rows(const KeyView& kv, int dh, const T* q, int64_t ldq, T* out, int64_t ldo, int heads,
                                 const SeenMask& m, bool, float* part, hipStream_t) {
  ++g_launches;
  rows(q, kv, ldq, (int64_t)heads * dh);
  rows(out, kv, ldo, (int64_t)heads * dh, true);
  if (part) touch(part, attention_rows_bytes(dh) / 4, true);
  if (m.block < 0 || m.window < 0 || m.sinks < 0) std::abort();
  tokens<T>(kv, dh, false);
  return g_result;
}
#define INST(T)                                                                                                      \
  template hipError_t launch_append<T>(const KeyView&, int, const T*, int64_t, const T*, int64_t, const T*, int64_t, \
                                       T*, int64_t, int, const AppendDesc&, hipStream_t);                            \
  template hipError_t launch_attention_rows<T>(const KeyView&, int, const T*, int64_t, T*, int64_t, int,             \
                                               const SeenMask&, bool, float*, hipStream_t);
INST(__bf16)
INST(float)
}  // namespace dif

static void expect(dif_status got, dif_status want, const char* what) {
  if (got != want) {
    std::fprintf(stderr, "%s: status %d, expected %d (%s)\n", what, got, want, dif_last_error());
    std::exit(1);
  }
}
extern "C" const char* dif_last_error(void) { return ""; }

// exactly sized, 256-byte aligned memory
template <typename T>
struct Mem {
  T* p;
  explicit Mem(size_t n) {
    void* v = nullptr;
    if (posix_memalign(&v, 256, n ? n * sizeof(T) : 1)) std::abort();
    p = (T*)v;
    for (size_t i = 0; i < n; ++i) p[i] = T();
  }
  Mem(const Mem&) = delete;
  ~Mem() { std::free(p); }
};

template <typename T>
static void sizes(int dt) {
  for (int dh : {64, 128})
    for (int kv : {1, 3})
      for (int group : {1, 4})
        for (int page : {16, 64})
          for (int seqs : {1, 3})
            for (bool nhd : {false, true}) {
              const int heads = kv * group, M = 2 * seqs, pages = 2 * seqs;
              // (every buffer ends with its last element)
              Mem<T> k((size_t)pages * kv * page * dh), v((size_t)pages * kv * page * dh), q((size_t)M * heads * dh),
                  nk((size_t)M * kv * dh), out((size_t)M * heads * dh);
              Mem<float> gq(heads * dh), gk(kv * dh);
              Mem<int32_t> table(seqs * 2), lengths(seqs), off(seqs + 1), pos(M * 3);
              for (int s = 0; s < seqs; ++s) {
                table.p[2 * s] = s ? s : -5;
                table.p[2 * s + 1] = s ? 1 << 30 : pages - 1;
                lengths.p[s] = s == 1 ? 1 << 30 : s == 2 ? -7 : 2 * page;
                off.p[s + 1] = s == 1 ? 1 << 30 : 2 * s + 2;
              }
              dif_kv_cache c{k.p, v.p, (int64_t)kv * page * dh, nhd ? dh : (int64_t)page * dh,
                             nhd ? (int64_t)kv * dh : dh, pages, page, kv, dh, seqs, 2, table.p, 2, lengths.p, off.p};
              for (int axes : {0, 1, 3}) {
                dif_append a{axes ? gq.p : nullptr, gk.p, 0, 1e-6f, axes == 1 ? 0.5f : 1e6f, axes,
                             axes == 3 ? pos.p : nullptr, 0.1f};
                expect(dif_cache_append(dt, &c, nk.p, kv * dh, nk.p, kv * dh, q.p, heads * dh, out.p, heads * dh, M, heads,
                                        &a, nullptr), DIF_OK, "append");
                a.gain_q = nullptr;
                expect(dif_cache_append(dt, &c, nk.p, kv * dh, nk.p, kv * dh, nullptr, 0, nullptr, 0, M, 0, &a, nullptr),
                       DIF_OK, "append, no queries");
              }
              size_t need = 0;
              expect(dif_attention_paged_bytes(dh, &need), DIF_OK, "bytes");
              Mem<char> ws(need);
              dif_seen m{1, 30, 4};
              expect(dif_attention_paged(dt, 0, q.p, heads * dh, &c, out.p, heads * dh, M, heads, &m, ws.p, need, nullptr),
                     DIF_OK, "paged");
              expect(dif_attention_paged(dt, 1, q.p, heads * dh, &c, out.p, heads * dh, M, heads, &m, nullptr, 0, nullptr),
                     DIF_OK, "paged, no workspace");
              expect(dif_attention_paged(dt, 1, q.p, heads * dh, &c, out.p, heads * dh, M, heads, &m, ws.p, need - 1,
                                         nullptr), DIF_E_WORKSPACE, "small workspace");
              expect(dif_attention_window(dt, dh, 0, q.p, heads * dh, nk.p, kv * dh, nk.p, kv * dh, out.p, heads * dh, M, M,
                                          heads, kv, seqs, off.p, nullptr, &m, ws.p, need, nullptr), DIF_OK, "window");
              expect(dif_attention_window(dt, dh, 0, q.p, heads * dh, nullptr, 0, nullptr, 0, out.p, heads * dh, M, 0,
                                          heads, kv, seqs, off.p, off.p, &m, nullptr, 0, nullptr), DIF_OK, "no keys");
            }
}

int main() {
  sizes<__bf16>(DIF_BF16);
  sizes<float>(DIF_F32);
  g_result = hipErrorInvalidValue;
  Mem<float> x(64 * 16);
  Mem<int32_t> off(2), one(1);
  off.p[1] = 1;
  dif_kv_cache c{x.p, x.p, 64 * 16, 64 * 16, 64, 1, 16, 1, 64, 1, 1, one.p, 1, one.p, off.p};
  dif_append a{nullptr, nullptr, 0, 1e-6f, 1e4f, 1, nullptr, 1.f};
  dif_seen m{1, 0, 0};
  expect(dif_cache_append(DIF_F32, &c, x.p, 64, x.p, 64, x.p, 64, x.p, 64, 1, 1, &a, nullptr), DIF_E_HIP, "a failing launch");
  expect(dif_attention_paged(DIF_F32, 0, x.p, 64, &c, x.p, 64, 1, 1, &m, nullptr, 0, nullptr), DIF_E_HIP, "a failing launch");
  std::printf("harness: %ld launches, all cases passed\n", g_launches);
  return 0;
}
