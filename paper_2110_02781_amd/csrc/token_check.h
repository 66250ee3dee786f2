// What the C ABI of the token operators checks: sizes, strides, alignment; errors of a launch.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/ftp.h"
#include "token.h"

void ftp_set_error(const char* fmt, ...);

namespace ftp {

// Refusals: the caller's outputs are untouched, nothing has been launched.
#define NEED(cond, status, ...)       \
  do {                                \
    if (!(cond)) {                    \
      ftp_set_error(__VA_ARGS__);     \
      return status;                  \
    }                                 \
  } while (0)

// Offsets inside a tile are 31-bit byte offsets: 256 rows of up to 2^20 elements.
enum { kMaxDim = 1 << 20 };
const int64_t kMaxRows = (int64_t)1 << 30, kMaxLd = (int64_t)1 << 20;
inline size_t esize(int dt) { return dt == FTP_BF16 ? 2 : 4; }
inline int64_t up_to(int64_t v, int64_t a) { return (v + a - 1) / a * a; }
inline bool at_element(const void* p, int dt) { return (uintptr_t)p % esize(dt) == 0; }
#define TRY(x)                       \
  do {                               \
    const int rc_ = (x);             \
    if (rc_) return rc_;             \
  } while (0)

static inline int check_common(const char* who, int64_t rows, int dt, int act) {
  NEED(dt == FTP_F32 || dt == FTP_BF16, FTP_ERR_ARG, "%s: unknown dtype %d", who, dt);
  NEED(act >= FTP_ACT_NONE && act <= FTP_ACT_GELU, FTP_ERR_ARG, "%s: unknown activation %d", who, act);
  NEED(rows >= 0 && rows <= kMaxRows, FTP_ERR_ARG, "%s: rows must be 0 .. 2^30", who);
  return FTP_OK;
}
// one matrix: there (unless it has no rows), aligned to its elements, rows at least `cols` apart
enum { kBytes = -1 };                    // in place of a dtype: a matrix in 8 bits
static inline int check_mat(const char* who, const char* what, const void* p, int64_t ld, int64_t rows, int64_t cols, int dt, bool optional = false) {
  if (!p && (optional || rows == 0)) return FTP_OK;
  NEED(p, FTP_ERR_ARG, "%s: %s is NULL", who, what);
  NEED(dt == kBytes || at_element(p, dt), FTP_ERR_ARG, "%s: %s is not aligned to its elements", who, what);
  NEED(ld >= cols && ld <= kMaxLd, FTP_ERR_ARG, "%s: %s has rows %lld apart (at least %lld, at most 2^20)", who, what, (long long)ld, (long long)cols);
  return FTP_OK;
}
static inline int launched(const char* who) {
  const hipError_t e = hipGetLastError();
  NEED(e == hipSuccess, FTP_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  if (const char* why = launch_plan_failure_take()) { ftp_set_error("%s", why); return FTP_ERR_UNSUPPORTED; }
  return FTP_OK;
}

}  // namespace ftp
