// Launch interface of what stands between a token stage's products: dropout, joins with norms, the gated recurrence, log probabilities.
// Arguments are checked before (between.cpp); nothing here allocates.
#pragma once
#include "../../include/ftp.h"
#include "token.h"

namespace ftp {

// a mask as the kernels take it: kept are the values with 16 bits of at least `least`, multiplied by `up`
struct DropMask {
  uint32_t least, site;
  float up;
  uint64_t seed;
  const uint64_t* seed_dev;
  int64_t row0;
};
// of p in [0, 1): a larger one may be past what 32 bits hold
static inline uint32_t drop_least(float p) { return (uint32_t)((double)p * 65536.0 + 0.5); }

void bt_dropout(hipStream_t st, int dt, int64_t rows, int cols, const DropMask& m, const void* x, int64_t ldx, const void* r, int64_t ldr, void* y, int64_t ldy);

void bt_join(hipStream_t st, const ftp_join_args& a, const DropMask& m);
size_t bt_join_bwd_bytes(const ftp_join_args& a);
void bt_join_bwd(hipStream_t st, const ftp_join_args& a, const DropMask& m);

size_t bt_scan_bytes(const ftp_scan_args& a, bool backward);
void bt_scan(hipStream_t st, const ftp_scan_args& a);
void bt_scan_bwd(hipStream_t st, const ftp_scan_args& a);

size_t bt_logp_bytes(const ftp_logp_args& a);
void bt_logp(hipStream_t st, const ftp_logp_args& a);
void bt_logp_bwd(hipStream_t st, const ftp_logp_args& a);

}  // namespace ftp
