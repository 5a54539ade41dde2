// Host runtime shared by the C ABI's sources: the last error, status macros,
// the guard that keeps exceptions inside an entry point, kernel timing.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <exception>
#include <mutex>
#include <string>
#include <vector>

#include "../../include/dif.h"

namespace dif {

inline thread_local std::string g_err;   // dif_last_error of this thread

inline dif_status fail(dif_status code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_err = buf;
  return code;
}

#define HIP_TRY(expr)                                                                   \
  do {                                                                                  \
    hipError_t e_ = (expr);                                                             \
    if (e_ != hipSuccess) return fail(DIF_E_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

#define DIF_TRY(expr)                 \
  do {                                \
    dif_status s_ = (expr);           \
    if (s_ != DIF_OK) return s_;      \
  } while (0)

#define GUARD_BEGIN try {
#define GUARD_END                                                  \
  }                                                                \
  catch (const std::exception& ex) {                               \
    return fail(DIF_E_ARG, "internal error: %s", ex.what());       \
  }                                                                \
  catch (...) {                                                    \
    return fail(DIF_E_ARG, "internal error");                      \
  }

inline size_t align256(size_t n) { return (n + 255) & ~size_t(255); }
inline int64_t round_up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
inline size_t esize(int dtype) { return dtype == DIF_BF16 ? 2 : 4; }

// ---------------------------------------------------------------------------
// kernel timing
// ---------------------------------------------------------------------------
enum ProfKind {
  PK_GEMM_QKV = 0, PK_ATTN_SELF, PK_GEMM_SELF_OUT, PK_GEMM_CROSS_Q, PK_GEMM_CROSS_KV,
  PK_ATTN_CROSS, PK_GEMM_CROSS_OUT, PK_GEMM_FFN1, PK_GEMM_FFN2, PK_NORM, PK_QK_NORM,
  PK_TRANSPOSE,   // (no launch: the projections write V transposed; kept for the kinds' numbers)
  PK_TIME_EMBED, PK_GEMM_IO, PK_GATHER, PK_ELEMENTWISE
};
inline const char* const kKindNames[DIF_PROF_KINDS] = {
    "gemm_qkv", "attn_self", "gemm_self_out", "gemm_cross_q", "gemm_cross_kv", "attn_cross",
    "gemm_cross_out", "gemm_ffn1", "gemm_ffn2", "norm", "qk_norm_rope", "transpose_v",
    "time_embed", "gemm_io", "gather", "elementwise"};

struct ProfRec {
  int kind;
  hipEvent_t a, b;
  double flops, bytes;
};
struct Profiler {
  std::mutex mu;
  bool on = false;
  std::vector<ProfRec> recs;
  std::vector<hipEvent_t> pool;
  size_t used = 0;
  hipEvent_t take() {
    if (used < pool.size()) return pool[used++];
    hipEvent_t e = nullptr;
    if (hipEventCreate(&e) != hipSuccess) return nullptr;
    pool.push_back(e);
    ++used;
    return e;
  }
};
inline Profiler g_prof;

// Brackets the launches issued in its scope with events on `stream`.
class ProfScope {
 public:
  ProfScope(int kind, hipStream_t s, double flops, double bytes)
      : kind_(kind), s_(s), flops_(flops), bytes_(bytes) {
    if (!g_prof.on) return;
    std::lock_guard<std::mutex> lk(g_prof.mu);
    a_ = g_prof.take();
    // a launch whose start event cannot be recorded is left out of the timing
    if (a_ && hipEventRecord(a_, s_) != hipSuccess) a_ = nullptr;
  }
  ~ProfScope() {
    if (!a_) return;
    std::lock_guard<std::mutex> lk(g_prof.mu);
    hipEvent_t b = g_prof.take();
    if (!b || hipEventRecord(b, s_) != hipSuccess) return;
    g_prof.recs.push_back({kind_, a_, b, flops_, bytes_});
  }

 private:
  int kind_;
  hipStream_t s_;
  double flops_, bytes_;
  hipEvent_t a_ = nullptr;
};

}  // namespace dif
