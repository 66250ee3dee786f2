// C ABI of what stands between a token stage's products: dropout, joins with norms, the gated recurrence, log probabilities.  Argument checks only.
#include <hip/hip_runtime.h>

#include <cmath>

#include "between.h"
#include "token_check.h"

using namespace ftp;

namespace {

int check_floats(const char* who, const char* what, const void* p) {
  NEED((uintptr_t)p % 4 == 0, FTP_ERR_ARG, "%s: %s is not aligned to its elements", who, what);
  return FTP_OK;
}
int check_space(const char* who, const void* ws, size_t have, size_t need) {
  NEED(need == 0 || (ws && have >= need), FTP_ERR_ARG, "%s: workspace of %zu bytes, needs %zu", who, ws ? have : (size_t)0, need);
  NEED(need == 0 || (uintptr_t)ws % 16 == 0, FTP_ERR_ARG, "%s: the workspace must start on 16 bytes", who);
  return FTP_OK;
}
// a result in an operand's buffer: element for element
int check_same(const char* who, const char* out, const void* o, int64_t ldo, const char* in, const void* i, int64_t ldi) {
  NEED(!o || o != i || ldo == ldi, FTP_ERR_ARG, "%s: %s in the buffer of %s has to have its row distance", who, out, in);
  return FTP_OK;
}
template <typename A>
int check_mask(const char* who, const A* a) {
  NEED(a->p >= 0.f && a->p < 1.f && drop_least(a->p) < 65536, FTP_ERR_VALUE, "%s: p must be in [0, 1), with some of 2^-16 left", who);
  NEED(a->row0 >= 0 && a->row0 <= INT64_MAX - a->rows, FTP_ERR_ARG, "%s: row0 must not be negative or too large", who);
  NEED((uintptr_t)a->seed_dev % 8 == 0, FTP_ERR_ARG, "%s: seed_dev is not aligned to its element", who);
  return FTP_OK;
}
template <typename A>
DropMask mask_of(const A& a) {
  const uint32_t least = drop_least(a.p);
  return DropMask{least, a.site, 65536.f / (float)(65536 - least), a.seed, a.seed_dev, a.row0};
}

int check_dropout(const char* who, const ftp_dropout_args* a, bool backward) {
  NEED(a, FTP_ERR_ARG, "%s: NULL argument", who);
  TRY(check_common(who, a->rows, a->dtype, FTP_ACT_NONE));
  NEED(a->cols >= 1 && a->cols <= kMaxDim, FTP_ERR_ARG, "%s: cols must be 1 .. 2^20", who);
  TRY(check_mask(who, a));
  if (!backward) {
    TRY(check_mat(who, "x", a->x, a->ldx, a->rows, a->cols, a->dtype));
    TRY(check_mat(who, "residual", a->residual, a->ldr, a->rows, a->cols, a->dtype, true));
    TRY(check_mat(who, "y", a->y, a->ldy, a->rows, a->cols, a->dtype));
    TRY(check_same(who, "y", a->y, a->ldy, "x", a->x, a->ldx));
    TRY(check_same(who, "y", a->y, a->ldy, "residual", a->residual, a->ldr));
  } else {
    TRY(check_mat(who, "dy", a->dy, a->lddy, a->rows, a->cols, a->dtype));
    TRY(check_mat(who, "dx", a->dx, a->lddx, a->rows, a->cols, a->dtype));
    TRY(check_same(who, "dx", a->dx, a->lddx, "dy", a->dy, a->lddy));
  }
  return FTP_OK;
}

int check_join(const char* who, const ftp_join_args* a, bool backward) {
  NEED(a, FTP_ERR_ARG, "%s: NULL argument", who);
  TRY(check_common(who, a->rows, a->dtype, FTP_ACT_NONE));
  NEED(a->width >= 1 && a->width <= kMaxDim, FTP_ERR_ARG, "%s: width must be 1 .. 2^20", who);
  NEED(a->norm == FTP_NORM_RMS || a->norm == FTP_NORM_LAYER, FTP_ERR_ARG, "%s: unknown norm %d", who, a->norm);
  NEED(std::isfinite(a->eps) && a->eps > 0.f, FTP_ERR_VALUE, "%s: eps must be positive and finite", who);
  NEED(std::isfinite(a->scale), FTP_ERR_VALUE, "%s: scale must be finite", who);
  TRY(check_mask(who, a));
  NEED(a->rows == 0 || a->x || a->b, FTP_ERR_ARG, "%s: x and b are NULL", who);
  TRY(check_mat(who, "x", a->x, a->ldx, a->rows, a->width, a->dtype, true));
  TRY(check_mat(who, "b", a->b, a->ldb, a->rows, a->width, a->dtype, true));
  TRY(check_floats(who, "post_w", a->post_w));
  TRY(check_floats(who, "post_bias", a->post_bias));
  TRY(check_floats(who, "pre_w", a->pre_w));
  TRY(check_floats(who, "pre_bias", a->pre_bias));
  if (a->gate) {
    NEED(a->gate_dtype == FTP_F32 || a->gate_dtype == a->dtype, FTP_ERR_ARG, "%s: the gate is fp32 or of the call's type", who);
    NEED(a->gate_rows >= 1, FTP_ERR_ARG, "%s: gate_rows must be positive", who);
    TRY(check_mat(who, "gate", a->gate, a->ldg, a->rows, a->width, a->gate_dtype));
  }
  if (!backward) {
    NEED(a->rows == 0 || a->y || a->n, FTP_ERR_ARG, "%s: neither y nor n is wanted", who);
    TRY(check_mat(who, "y", a->y, a->ldy, a->rows, a->width, a->dtype, true));
    TRY(check_mat(who, "n", a->n, a->ldn, a->rows, a->width, a->dtype, true));
    TRY(check_same(who, "y", a->y, a->ldy, "x", a->x, a->ldx));
    TRY(check_same(who, "y", a->y, a->ldy, "b", a->b, a->ldb));
    return FTP_OK;
  }
  NEED(a->dx || a->db || a->dgate || a->dpost_w || a->dpost_bias || a->dpre_w || a->dpre_bias, FTP_ERR_ARG, "%s: no gradient is asked for", who);
  NEED(a->rows == 0 || a->dy || a->dn, FTP_ERR_ARG, "%s: dy and dn are NULL", who);
  TRY(check_mat(who, "dy", a->dy, a->lddy, a->rows, a->width, a->dtype, true));
  TRY(check_mat(who, "dn", a->dn, a->lddn, a->rows, a->width, a->dtype, true));
  TRY(check_mat(who, "dx", a->dx, a->lddx, a->rows, a->width, a->dtype, true));
  TRY(check_mat(who, "db", a->db, a->lddb, a->rows, a->width, a->dtype, true));
  TRY(check_same(who, "dx", a->dx, a->lddx, "dy", a->dy, a->lddy));
  NEED(a->rows == 0 || a->b || !(a->db || a->dgate || a->dpost_w || a->dpost_bias), FTP_ERR_ARG, "%s: a gradient of the block's side without b", who);
  NEED(a->post || !(a->dpost_w || a->dpost_bias), FTP_ERR_ARG, "%s: gradients of the weights behind the block without post", who);
  NEED(a->rows == 0 || a->dn || !(a->dpre_w || a->dpre_bias), FTP_ERR_ARG, "%s: dpre_w and dpre_bias need dn", who);
  TRY(check_floats(who, "dpost_w", a->dpost_w));
  TRY(check_floats(who, "dpost_bias", a->dpost_bias));
  TRY(check_floats(who, "dpre_w", a->dpre_w));
  TRY(check_floats(who, "dpre_bias", a->dpre_bias));
  if (a->dgate) {
    NEED(a->gate || a->rows == 0, FTP_ERR_ARG, "%s: dgate without a gate", who);
    NEED(!a->gate_accumulate || a->gate_dtype == FTP_F32, FTP_ERR_UNSUPPORTED, "%s: only fp32 gradients accumulate", who);
    TRY(check_mat(who, "dgate", a->dgate, a->lddg, a->rows, a->width, a->gate_dtype));
  }
  return FTP_OK;
}

int check_scan(const char* who, const ftp_scan_args* a, bool backward) {
  NEED(a, FTP_ERR_ARG, "%s: NULL argument", who);
  TRY(check_common(who, a->rows, a->dtype, a->act));
  NEED(a->width >= 1 && a->width <= kMaxDim, FTP_ERR_ARG, "%s: width must be 1 .. 2^20", who);
  NEED(a->form >= FTP_SCAN_ADD && a->form <= FTP_SCAN_UNIT, FTP_ERR_ARG, "%s: unknown form %d", who, a->form);
  NEED(a->seqs >= 0 && a->seqs <= (1 << 30), FTP_ERR_ARG, "%s: seqs must be 0 .. 2^30", who);
  if (a->starts) {
    NEED((uintptr_t)a->starts % 4 == 0, FTP_ERR_ARG, "%s: starts is not aligned to its elements", who);
  } else {
    NEED(a->length >= 0 && a->length <= kMaxRows && a->rows == a->length * a->seqs, FTP_ERR_ARG, "%s: rows must be seqs * length where there are no starts", who);
  }
  TRY(check_mat(who, "f", a->f, a->ldf, a->rows, a->width, a->dtype));
  TRY(check_mat(who, "x", a->x, a->ldx, a->rows, a->width, a->dtype));
  TRY(check_mat(who, "g", a->g, a->ldg, a->rows, a->width, a->dtype, true));
  TRY(check_mat(who, "h0", a->h0, a->ldh0, a->seqs, a->width, FTP_F32, true));
  if (!backward) {
    NEED(a->rows == 0 || a->y || a->h_end, FTP_ERR_ARG, "%s: neither y nor h_end is wanted", who);
    TRY(check_mat(who, "y", a->y, a->ldy, a->rows, a->width, a->dtype, true));
    TRY(check_mat(who, "h_end", a->h_end, a->ldhe, a->seqs, a->width, FTP_F32, true));
    TRY(check_same(who, "h_end", a->h_end, a->ldhe, "h0", a->h0, a->ldh0));
    return FTP_OK;
  }
  NEED(a->df || a->dx || a->dg || a->dh0, FTP_ERR_ARG, "%s: no gradient is asked for", who);
  NEED(a->g || !a->dg || a->rows == 0, FTP_ERR_ARG, "%s: dg without g", who);
  TRY(check_mat(who, "dy", a->dy, a->lddy, a->rows, a->width, a->dtype));
  TRY(check_mat(who, "dh_end", a->dh_end, a->lddhe, a->seqs, a->width, FTP_F32, true));
  TRY(check_mat(who, "df", a->df, a->lddf, a->rows, a->width, a->dtype, true));
  TRY(check_mat(who, "dx", a->dx, a->lddx, a->rows, a->width, a->dtype, true));
  TRY(check_mat(who, "dg", a->dg, a->lddg, a->rows, a->width, a->dtype, true));
  TRY(check_mat(who, "dh0", a->dh0, a->lddh0, a->seqs, a->width, FTP_F32, true));
  TRY(check_same(who, "dh0", a->dh0, a->lddh0, "dh_end", a->dh_end, a->lddhe));
  return FTP_OK;
}

int check_logp(const char* who, const ftp_logp_args* a, bool backward) {
  NEED(a, FTP_ERR_ARG, "%s: NULL argument", who);
  TRY(check_common(who, a->rows, a->dtype, FTP_ACT_NONE));
  NEED(a->vocab >= 1 && a->vocab <= kMaxDim, FTP_ERR_ARG, "%s: vocab must be 1 .. 2^20", who);
  NEED(std::isfinite(a->scale) && a->scale > 0.f, FTP_ERR_VALUE, "%s: scale must be positive and finite", who);
  TRY(check_mat(who, "logits", a->logits, a->ldl, a->rows, a->vocab, a->dtype));
  const bool ids = backward ? a->dlogp != nullptr : a->logp != nullptr;
  NEED(a->rows == 0 || !ids || a->ids, FTP_ERR_ARG, "%s: ids is NULL", who);
  NEED((uintptr_t)a->ids % (a->ids64 ? 8 : 4) == 0, FTP_ERR_ARG, "%s: ids is not aligned to its elements", who);
  TRY(check_floats(who, "stats", a->stats));
  TRY(check_floats(who, "entropy", a->entropy));
  if (!backward) {
    NEED(a->top >= 0 && a->top <= 64, FTP_ERR_ARG, "%s: top must be 0 .. 64", who);
    NEED(a->rows == 0 || a->logp || a->entropy || a->lse || a->stats || a->top, FTP_ERR_ARG, "%s: nothing is wanted", who);
    NEED(a->rows == 0 || a->top == 0 || (a->top_ids && a->top_logp), FTP_ERR_ARG, "%s: top_ids and top_logp must not be NULL with top", who);
    TRY(check_floats(who, "logp", a->logp));
    TRY(check_floats(who, "lse", a->lse));
    TRY(check_floats(who, "top_ids", a->top_ids));
    TRY(check_floats(who, "top_logp", a->top_logp));
    return FTP_OK;
  }
  NEED(a->rows == 0 || a->stats, FTP_ERR_ARG, "%s: needs the stats that the forward kept", who);
  NEED(a->rows == 0 || a->dlogp || a->dentropy, FTP_ERR_ARG, "%s: dlogp and dentropy are NULL", who);
  NEED(a->rows == 0 || !a->dentropy || a->entropy, FTP_ERR_ARG, "%s: dentropy needs the entropy", who);
  TRY(check_floats(who, "dlogp", a->dlogp));
  TRY(check_floats(who, "dentropy", a->dentropy));
  TRY(check_mat(who, "dlogits", a->dlogits, a->lddl, a->rows, a->vocab, a->dtype));
  TRY(check_same(who, "dlogits", a->dlogits, a->lddl, "logits", a->logits, a->ldl));
  return FTP_OK;
}

}  // namespace

extern "C" int ftp_dropout_forward(const ftp_dropout_args* a, void* stream) {
  TRY(check_dropout("dropout_forward", a, false));
  if (!a->rows) return FTP_OK;
  bt_dropout((hipStream_t)stream, a->dtype, a->rows, a->cols, mask_of(*a), a->x, a->ldx, a->residual, a->ldr, a->y, a->ldy);
  return launched("dropout_forward");
}
extern "C" int ftp_dropout_backward(const ftp_dropout_args* a, void* stream) {
  TRY(check_dropout("dropout_backward", a, true));
  if (!a->rows) return FTP_OK;
  bt_dropout((hipStream_t)stream, a->dtype, a->rows, a->cols, mask_of(*a), a->dy, a->lddy, nullptr, 0, a->dx, a->lddx);
  return launched("dropout_backward");
}

extern "C" int ftp_join_forward(const ftp_join_args* a, void* stream) {
  TRY(check_join("join_forward", a, false));
  if (!a->rows) return FTP_OK;
  bt_join((hipStream_t)stream, *a, mask_of(*a));
  return launched("join_forward");
}
extern "C" int ftp_join_workspace(const ftp_join_args* a, size_t* bytes) {
  NEED(bytes, FTP_ERR_ARG, "join_workspace: NULL argument");
  TRY(check_join("join_workspace", a, true));
  *bytes = a->rows ? bt_join_bwd_bytes(*a) : 0;
  return FTP_OK;
}
extern "C" int ftp_join_backward(const ftp_join_args* a, void* stream) {
  TRY(check_join("join_backward", a, true));
  TRY(check_space("join_backward", a->ws, a->ws_bytes, a->rows ? bt_join_bwd_bytes(*a) : 0));
  bt_join_bwd((hipStream_t)stream, *a, mask_of(*a));
  return launched("join_backward");
}

extern "C" int ftp_scan_workspace(const ftp_scan_args* a, int backward, size_t* bytes) {
  NEED(bytes, FTP_ERR_ARG, "scan_workspace: NULL argument");
  TRY(check_scan("scan_workspace", a, backward != 0));
  *bytes = bt_scan_bytes(*a, backward != 0);
  return FTP_OK;
}
extern "C" int ftp_scan_forward(const ftp_scan_args* a, void* stream) {
  TRY(check_scan("scan_forward", a, false));
  TRY(check_space("scan_forward", a->ws, a->ws_bytes, bt_scan_bytes(*a, false)));
  if (!a->seqs) return FTP_OK;
  bt_scan((hipStream_t)stream, *a);
  return launched("scan_forward");
}
extern "C" int ftp_scan_backward(const ftp_scan_args* a, void* stream) {
  TRY(check_scan("scan_backward", a, true));
  TRY(check_space("scan_backward", a->ws, a->ws_bytes, bt_scan_bytes(*a, true)));
  if (!a->seqs) return FTP_OK;
  bt_scan_bwd((hipStream_t)stream, *a);
  return launched("scan_backward");
}

extern "C" int ftp_logp_workspace(const ftp_logp_args* a, size_t* bytes) {
  NEED(bytes, FTP_ERR_ARG, "logp_workspace: NULL argument");
  TRY(check_logp("logp_workspace", a, false));
  *bytes = a->rows ? bt_logp_bytes(*a) : 0;
  return FTP_OK;
}
extern "C" int ftp_logp_forward(const ftp_logp_args* a, void* stream) {
  TRY(check_logp("logp_forward", a, false));
  TRY(check_space("logp_forward", a->ws, a->ws_bytes, a->rows ? bt_logp_bytes(*a) : 0));
  if (!a->rows) return FTP_OK;
  bt_logp((hipStream_t)stream, *a);
  return launched("logp_forward");
}
extern "C" int ftp_logp_backward(const ftp_logp_args* a, void* stream) {
  TRY(check_logp("logp_backward", a, true));
  if (!a->rows) return FTP_OK;
  bt_logp_bwd((hipStream_t)stream, *a);
  return launched("logp_backward");
}
