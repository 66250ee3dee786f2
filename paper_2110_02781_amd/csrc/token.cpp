// C ABI of the token operators: argument checks, workspace layout, order of the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "token_check.h"

using namespace ftp;

namespace {

// what partial sums of a split reduction may take of the workspace (one product's, all of a call's share it)
const size_t kPartBytes = (size_t)256 << 20;

// fours of columns of a row are aligned
inline bool fours(const void* p, int64_t ld, size_t es) { return (uintptr_t)p % (4 * es) == 0 && ld % 4 == 0; }

// Workspace in the order of use; with no base it only measures.
struct Space {
  char* base;
  size_t used = 0;
  void* take(size_t bytes) {
    void* p = base ? base + used : nullptr;
    used += (size_t)up_to((int64_t)bytes, 256);
    return p;
  }
};
struct Mat { const void* p; int64_t ld; };

struct Call {
  int dt;
  hipStream_t st;
  Space ws;
  bool dry() const { return !ws.base; }
  int64_t wide(int64_t cols) const { return up_to(cols, dt == FTP_BF16 ? 8 : 4); }
  // The products load 16 bytes at a time, from any multiple of 4: an operand whose rows have another length, or start elsewhere, is copied into rows
  // that do (a pass over it; a product reads it several times), one in 8 bits is read back into such rows.  Rows off the 16 bytes are better read where
  // they lie, also by large products: x [8192][4096 of 4098], bfloat16, against 4096 weight rows 268 us, copied 276, on 16 bytes 251; against 512
  // weight rows 62 and 98.  `any`: for the kernel of few rows, which reads rows as they are.  copied() launches the copies that the operands so far need, all at once.
  bool as_is(const void* p, int64_t ld, int cols) const { return wide(cols) == cols && (uintptr_t)p % 4 == 0 && ld * (int64_t)esize(dt) % 4 == 0; }
  TkCopy copies[kCopies];
  int ncopies = 0;
  Mat operand(const void* p, int64_t ld, const uint8_t* scales, int64_t lds, int rows, int cols, bool any = false) {
    const int64_t w = wide(cols);
    if (!scales && (any || as_is(p, ld, cols))) return Mat{p, ld};
    void* q = ws.take((size_t)rows * w * esize(dt));
    if (scales) {
      if (!dry()) tk_act8_unpack(dt, st, (const uint8_t*)p, ld, scales, lds, rows, cols, (int)w, q, w);
    } else {
      copies[ncopies++] = TkCopy{p, ld, q, w, rows, cols};
    }
    return Mat{q, w};
  }
  void copied() {
    if (ncopies && !dry()) tk_align(dt, st, copies, ncopies);
    ncopies = 0;
  }
  // Whether the kernel of few rows takes a product of `mats` weight matrices [n][k] (aligned: a tile could read them as they are).  Up to eight rows always.
  // Beyond them its reads of x, 16 rows for every 16 weight rows, cost more than the empty rows of a tile where the weights are bfloat16 and many: 16 rows, 4096 x 4096
  // 11.4 us, a tile split by four 14.3; 14336 x 4096 33.4 and 28.0; gate and up of 2048 x 5632 and down 25.3, 21.9; fp32 64 and 69, 20 and 28.  Weights that
  // a tile needs copied first are streamed: 4096 x 4100 with one row 6 us, with copies some 20.
  bool few(int rows, int n, int k, int mats, bool aligned) const {
    if (rows > kSkinnyRows) return false;
    return rows <= 8 || dt == FTP_F32 || !aligned || (double)n * k * mats * 2 <= 40e6;
  }
  // the partial sums' room is the same for all products of a call, which follow one another
  void* part = nullptr;
  size_t part_most = 0;
  void product(int lay, int epi, TgJob* jobs, int n) {
    TgPlan plan{128, 1};
    size_t room = 0;
    // the plan of the largest job; all of them have to fit the room with it
    int big = 0;
    for (int i = 1; i < n; ++i)
      if ((double)jobs[i].M * jobs[i].N > (double)jobs[big].M * jobs[big].N) big = i;
    plan = tg_plan(dt, epi, jobs[big].M, jobs[big].N * n, jobs[big].K * jobs[big].nseg, kPartBytes);
    for (int i = 0; i < n; ++i) room += (size_t)up_to((int64_t)tg_part_bytes(epi, jobs[i].M, jobs[i].N, plan.splits), 256);
    part_most = std::max(part_most, room);
    if (dry()) return;
    char* at = (char*)part;
    for (int i = 0; i < n; ++i) {
      jobs[i].part = (float*)at;
      at += up_to((int64_t)tg_part_bytes(epi, jobs[i].M, jobs[i].N, plan.splits), 256);
    }
    tg_launch(dt, st, lay, epi, jobs, n, plan);
  }
};

// Runs `f(call)` once to measure and, where there is a base, once to launch; the partial sums lie in front.
template <typename F>
size_t measure(int dt, F f) {
  Call c{dt, nullptr, Space{nullptr}};
  f(c);
  return (size_t)up_to((int64_t)c.part_most, 256) + c.ws.used;
}
template <typename F>
int run(const char* who, int dt, void* ws, size_t ws_bytes, void* stream, F f) {
  Call m{dt, nullptr, Space{nullptr}};
  f(m);
  const size_t need = (size_t)up_to((int64_t)m.part_most, 256) + m.ws.used;
  NEED(need == 0 || ws, FTP_ERR_ARG, "%s: needs a workspace of %zu bytes", who, need);
  NEED(ws_bytes >= need, FTP_ERR_ARG, "%s: workspace of %zu bytes, needs %zu", who, ws_bytes, need);
  NEED((uintptr_t)ws % 16 == 0, FTP_ERR_ARG, "%s: the workspace must start on 16 bytes", who);
  static char nowhere[1];
  Call c{dt, (hipStream_t)stream, Space{need ? (char*)ws : nowhere}};
  c.part = c.ws.take(m.part_most);
  f(c);
  const hipError_t e = hipGetLastError();
  NEED(e == hipSuccess, FTP_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  if (const char* why = launch_plan_failure_take()) { ftp_set_error("%s", why); return FTP_ERR_UNSUPPORTED; }
  return FTP_OK;
}

int check_grad(const char* who, int dt, int grad_dtype, int accumulate) {
  NEED(grad_dtype == FTP_F32 || grad_dtype == dt, FTP_ERR_ARG, "%s: gradients of the weights are fp32 or of the call's type", who);
  NEED(!accumulate || grad_dtype == FTP_F32, FTP_ERR_UNSUPPORTED, "%s: only fp32 gradients accumulate", who);
  return FTP_OK;
}
int check_linear(const char* who, const ftp_linear_args* a, bool backward) {
  NEED(a, FTP_ERR_ARG, "%s: NULL argument", who);
  TRY(check_common(who, a->rows, a->dtype, a->act));
  NEED(a->n_in >= 1 && a->n_in <= kMaxDim && a->n_out >= 1 && a->n_out <= kMaxDim, FTP_ERR_ARG, "%s: n_in and n_out must be 1 .. 2^20", who);
  const bool x8 = a->x_scales != nullptr;
  if (!backward || a->dw) {
    TRY(check_mat(who, "x", a->x, a->ldx, a->rows, a->n_in, x8 ? kBytes : a->dtype));
    NEED(!x8 || a->ldxs >= act8_groups(a->n_in), FTP_ERR_ARG, "%s: scales of x have rows %lld apart (%d groups)", who, (long long)a->ldxs, act8_groups(a->n_in));
  }
  if (!backward || a->dx) TRY(check_mat(who, "w", a->w, a->ldw, 1, a->n_in, a->dtype));
  if (!backward) {
    NEED((uintptr_t)a->bias % 4 == 0, FTP_ERR_ARG, "%s: bias is not aligned to its elements", who);
    TRY(check_mat(who, "residual", a->residual, a->ldr, a->rows, a->n_out, a->dtype, true));
    TRY(check_mat(who, "y", a->y, a->ldy, a->rows, a->n_out, a->dtype));
    TRY(check_mat(who, "z", a->z, a->ldz, a->rows, a->n_out, a->dtype, true));
  } else {
    NEED(a->dx || a->dw || a->dbias, FTP_ERR_ARG, "%s: no gradient is asked for", who);
    TRY(check_mat(who, "dy", a->dy, a->lddy, a->rows, a->n_out, a->dtype));
    if (a->act != FTP_ACT_NONE) TRY(check_mat(who, "z", a->z, a->ldz, a->rows, a->n_out, a->dtype));
    TRY(check_mat(who, "dx", a->dx, a->lddx, a->rows, a->n_in, a->dtype, true));
    TRY(check_grad(who, a->dtype, a->grad_dtype, a->accumulate));
    NEED(at_element(a->dw, a->grad_dtype) && at_element(a->dbias, a->grad_dtype), FTP_ERR_ARG, "%s: a gradient is not aligned to its elements", who);
  }
  return FTP_OK;
}

void linear_forward(Call& c, const ftp_linear_args& a) {
  const int rows = (int)a.rows;
  if (rows == 0) return;
  const bool few = c.few(rows, a.n_out, a.n_in, 1, c.as_is(a.w, a.ldw, a.n_in));
  const Mat x = c.operand(a.x, a.ldx, a.x_scales, a.ldxs, rows, a.n_in, few), w = c.operand(a.w, a.ldw, nullptr, 0, a.n_out, a.n_in, few);
  c.copied();
  const size_t es = esize(a.dtype);
  TgJob j{};
  j.a[0] = x.p; j.lda = x.ld;
  j.b[0] = w.p; j.ldb[0] = w.ld;
  j.M = rows; j.N = a.n_out; j.K = few ? a.n_in : (int)c.wide(a.n_in); j.nseg = 1;
  j.act = a.act;
  j.bias = a.bias;
  j.res = a.residual; j.ldr = a.ldr;
  j.out = a.y; j.ldo = a.ldy;
  j.z = a.z; j.ldz = a.ldz;
  j.flags = (fours(a.y, a.ldy, es) ? TG_VEC_OUT : 0) | (fours(a.residual, a.ldr, es) ? TG_VEC_RES : 0) | (fours(a.z, a.ldz, es) ? TG_VEC_Z : 0) |
            ((uintptr_t)a.bias % 16 == 0 ? TG_VEC_BIAS : 0);
  if (few) {
    if (!c.dry()) tg_skinny(a.dtype, c.st, TG_LINEAR, j);
  } else {
    c.product(TG_NT, TG_LINEAR, &j, 1);
  }
}

// zero weight gradients of a call without rows
void no_rows(Call& c, void* dw, int64_t n, int64_t m, int dt, int accumulate) {
  if (dw && !accumulate && !c.dry()) tk_fill(c.st, dw, n, m * (int64_t)esize(dt), m * (int64_t)esize(dt));
}

void linear_backward(Call& c, const ftp_linear_args& a) {
  const int rows = (int)a.rows, k = a.n_in, n = a.n_out;
  const size_t es = esize(a.dtype);
  if (rows == 0) {
    no_rows(c, a.dw, n, k, a.grad_dtype, a.accumulate);
    no_rows(c, a.dbias, 1, n, a.grad_dtype, a.accumulate);
    return;
  }
  const int chunks = tk_dz_chunks(rows);
  float* sums = a.dbias ? (float*)c.ws.take((size_t)chunks * n * 4) : nullptr;
  Mat dz{a.dy, a.lddy};
  if (a.act != FTP_ACT_NONE && (a.dx || a.dw)) {
    void* q = c.ws.take((size_t)rows * c.wide(n) * es);
    dz = Mat{q, c.wide(n)};
    if (!c.dry()) tk_dz(a.dtype, c.st, a.dy, a.lddy, a.z, a.ldz, a.act, rows, n, q, dz.ld, sums);
  } else {
    if (a.dbias && !c.dry()) tk_dz(a.dtype, c.st, a.dy, a.lddy, a.z, a.ldz, a.act, rows, n, nullptr, 0, sums);
    if (a.dx || a.dw) dz = c.operand(a.dy, a.lddy, nullptr, 0, rows, n);
  }
  Mat w{}, x{};
  if (a.dx) w = c.operand(a.w, a.ldw, nullptr, 0, n, k);
  if (a.dw) x = c.operand(a.x, a.ldx, a.x_scales, a.ldxs, rows, k);
  c.copied();
  if (a.dbias && !c.dry()) tk_colsum_join(c.st, sums, chunks, n, a.dbias, a.grad_dtype, a.accumulate);
  if (a.dx) {
    TgJob j{};
    j.a[0] = dz.p; j.lda = dz.ld;
    j.b[0] = w.p; j.ldb[0] = w.ld;
    j.M = rows; j.N = k; j.K = n; j.nseg = 1;
    j.out = a.dx; j.ldo = a.lddx;
    j.flags = fours(a.dx, a.lddx, es) ? TG_VEC_OUT : 0;
    c.product(TG_NN, TG_LINEAR, &j, 1);
  }
  if (a.dw) {
    TgJob j{};
    j.a[0] = dz.p; j.lda = dz.ld;
    j.b[0] = x.p; j.ldb[0] = x.ld;
    j.M = n; j.N = k; j.K = rows; j.nseg = 1;
    j.out = a.dw; j.ldo = k;
    j.out_f32 = a.grad_dtype == FTP_F32; j.accumulate = a.accumulate;
    j.flags = fours(a.dw, k, esize(a.grad_dtype)) ? TG_VEC_OUT : 0;
    c.product(TG_TN, TG_GRAD, &j, 1);
  }
}

int check_ffn(const char* who, const ftp_ffn_args* a, bool backward) {
  NEED(a, FTP_ERR_ARG, "%s: NULL argument", who);
  TRY(check_common(who, a->rows, a->dtype, a->act));
  NEED(a->width >= 1 && a->width <= kMaxDim && a->hidden >= 1 && a->hidden <= kMaxDim, FTP_ERR_ARG, "%s: width and hidden must be 1 .. 2^20", who);
  NEED(a->save >= FTP_SAVE_NONE && a->save <= FTP_SAVE_ACT8, FTP_ERR_ARG, "%s: unknown save %d", who, a->save);
  const bool x8 = a->x_scales != nullptr;
  const bool grads = a->dw_gate || a->dw_up || a->dw_down;
  if (!backward || grads) {
    TRY(check_mat(who, "x", a->x, a->ldx, a->rows, a->width, x8 ? kBytes : a->dtype));
    NEED(!x8 || a->ldxs >= act8_groups(a->width), FTP_ERR_ARG, "%s: scales of x have rows %lld apart (%d groups)", who, (long long)a->ldxs, act8_groups(a->width));
  }
  TRY(check_mat(who, "w_gate", a->w_gate, a->ldwg, 1, a->width, a->dtype));
  TRY(check_mat(who, "w_up", a->w_up, a->ldwu, 1, a->width, a->dtype));
  TRY(check_mat(who, "w_down", a->w_down, a->ldwd, 1, a->hidden, a->dtype));
  if (backward) NEED(a->save != FTP_SAVE_NONE, FTP_ERR_ARG, "%s: needs the gate and up values that the forward kept", who);
  if (a->save != FTP_SAVE_NONE && a->rows > 0) {
    NEED(a->gate && a->up, FTP_ERR_ARG, "%s: gate and up must not be NULL with save %d", who, a->save);
    NEED(a->save != FTP_SAVE_ACT8 || (a->gate_scales && a->up_scales), FTP_ERR_ARG, "%s: scales must not be NULL with 8-bit gate and up", who);
    NEED(a->save != FTP_SAVE_FULL || (at_element(a->gate, a->dtype) && at_element(a->up, a->dtype)), FTP_ERR_ARG, "%s: gate or up is not aligned to its elements", who);
  }
  if (!backward) {
    TRY(check_mat(who, "residual", a->residual, a->ldr, a->rows, a->width, a->dtype, true));
    TRY(check_mat(who, "y", a->y, a->ldy, a->rows, a->width, a->dtype));
  } else {
    NEED(a->dx || grads, FTP_ERR_ARG, "%s: no gradient is asked for", who);
    NEED((a->dw_gate && a->dw_up && a->dw_down) || !grads, FTP_ERR_ARG, "%s: the three weight gradients go together", who);
    TRY(check_mat(who, "dy", a->dy, a->lddy, a->rows, a->width, a->dtype));
    TRY(check_mat(who, "dx", a->dx, a->lddx, a->rows, a->width, a->dtype, true));
    TRY(check_grad(who, a->dtype, a->grad_dtype, a->accumulate));
    NEED(at_element(a->dw_gate, a->grad_dtype) && at_element(a->dw_up, a->grad_dtype) && at_element(a->dw_down, a->grad_dtype), FTP_ERR_ARG,
         "%s: a gradient is not aligned to its elements", who);
  }
  return FTP_OK;
}

// gate and up as kept: rows one behind the other
void kept(TgJob& j, const ftp_ffn_args& a) {
  j.save = a.save;
  j.z = a.gate; j.ldz = a.hidden;
  j.up = a.up; j.ldu = a.hidden;
  j.zs = a.gate_scales; j.us = a.up_scales; j.lds = act8_groups(a.hidden);
  const size_t es = a.save == FTP_SAVE_ACT8 ? 1 : esize(a.dtype);
  if (fours(a.gate, a.hidden, es) && fours(a.up, a.hidden, es)) j.flags |= TG_VEC_Z;
}

void ffn_forward(Call& c, const ftp_ffn_args& a) {
  const int rows = (int)a.rows, d = a.width, f = a.hidden;
  if (rows == 0) return;
  const size_t es = esize(a.dtype);
  const int64_t fw = c.wide(f);
  void* h = c.ws.take((size_t)rows * fw * es);
  // few rows: the weights are streamed as they lie (gate and up kept in 8 bits need a tile, which has whole groups of a row)
  const bool few = c.few(rows, d, f, 1, c.as_is(a.w_down, a.ldwd, f));
  const bool few_up = a.save != FTP_SAVE_ACT8 && c.few(rows, f, d, 2, c.as_is(a.w_gate, a.ldwg, d) && c.as_is(a.w_up, a.ldwu, d));
  const Mat x = c.operand(a.x, a.ldx, a.x_scales, a.ldxs, rows, d, few_up);
  const Mat wg = c.operand(a.w_gate, a.ldwg, nullptr, 0, f, d, few_up), wu = c.operand(a.w_up, a.ldwu, nullptr, 0, f, d, few_up);
  const Mat wd = c.operand(a.w_down, a.ldwd, nullptr, 0, d, f, few);
  c.copied();
  TgJob j{};
  j.a[0] = x.p; j.lda = x.ld;
  j.b[0] = wg.p; j.ldb[0] = wg.ld;
  j.b[1] = wu.p; j.ldb[1] = wu.ld;
  j.M = rows; j.N = f; j.K = few_up ? d : (int)c.wide(d); j.nseg = 1;
  j.act = a.act;
  j.out = h; j.ldo = fw;
  kept(j, a);
  if (!few_up) c.product(TG_NT, TG_GLU, &j, 1);
  else if (!c.dry()) tg_skinny(a.dtype, c.st, TG_GLU, j);
  TgJob k{};
  k.a[0] = h; k.lda = fw;
  k.b[0] = wd.p; k.ldb[0] = wd.ld;
  k.M = rows; k.N = d; k.K = few ? f : (int)fw; k.nseg = 1;
  k.res = a.residual; k.ldr = a.ldr;
  k.out = a.y; k.ldo = a.ldy;
  k.flags = (fours(a.y, a.ldy, es) ? TG_VEC_OUT : 0) | (fours(a.residual, a.ldr, es) ? TG_VEC_RES : 0);
  if (!few) c.product(TG_NT, TG_LINEAR, &k, 1);
  else if (!c.dry()) tg_skinny(a.dtype, c.st, TG_LINEAR, k);
}

void ffn_backward(Call& c, const ftp_ffn_args& a) {
  const int rows = (int)a.rows, d = a.width, f = a.hidden;
  const size_t es = esize(a.dtype), gs = esize(a.grad_dtype);
  if (rows == 0) {
    no_rows(c, a.dw_gate, f, d, a.grad_dtype, a.accumulate);
    no_rows(c, a.dw_up, f, d, a.grad_dtype, a.accumulate);
    no_rows(c, a.dw_down, d, f, a.grad_dtype, a.accumulate);
    return;
  }
  const int64_t fw = c.wide(f);
  void *dg = c.ws.take((size_t)rows * fw * es), *du = c.ws.take((size_t)rows * fw * es), *h = c.ws.take((size_t)rows * fw * es);
  const Mat dy = c.operand(a.dy, a.lddy, nullptr, 0, rows, d), wd = c.operand(a.w_down, a.ldwd, nullptr, 0, d, f);
  Mat wg{}, wu{}, x{};
  if (a.dx) {
    wg = c.operand(a.w_gate, a.ldwg, nullptr, 0, f, d);
    wu = c.operand(a.w_up, a.ldwu, nullptr, 0, f, d);
  }
  if (a.dw_gate) x = c.operand(a.x, a.ldx, a.x_scales, a.ldxs, rows, d);
  c.copied();
  TgJob j{};
  j.a[0] = dy.p; j.lda = dy.ld;
  j.b[0] = wd.p; j.ldb[0] = wd.ld;
  j.M = rows; j.N = f; j.K = d; j.nseg = 1;
  j.act = a.act;
  kept(j, a);
  j.out = h; j.ldo = fw;
  j.dgate = dg; j.dup = du; j.ldd = fw;
  c.product(TG_NN, TG_GLUBWD, &j, 1);
  if (a.dx) {
    TgJob k{};
    k.a[0] = dg; k.a[1] = du; k.lda = fw;
    k.b[0] = wg.p; k.ldb[0] = wg.ld;
    k.b[1] = wu.p; k.ldb[1] = wu.ld;
    k.M = rows; k.N = d; k.K = f; k.nseg = 2;
    if (a.dx_residual) { k.res = a.dy; k.ldr = a.lddy; }
    k.out = a.dx; k.ldo = a.lddx;
    k.flags = (fours(a.dx, a.lddx, es) ? TG_VEC_OUT : 0) | (fours(a.dy, a.lddy, es) ? TG_VEC_RES : 0);
    c.product(TG_NN, TG_LINEAR, &k, 1);
  }
  if (a.dw_gate) {
    TgJob k[3] = {};
    const void* left[3] = {dg, du, dy.p};
    const Mat right[3] = {x, x, Mat{h, fw}};
    void* out[3] = {a.dw_gate, a.dw_up, a.dw_down};
    for (int i = 0; i < 3; ++i) {
      k[i].a[0] = left[i]; k[i].lda = i < 2 ? fw : dy.ld;
      k[i].b[0] = right[i].p; k[i].ldb[0] = right[i].ld;
      k[i].M = i < 2 ? f : d; k[i].N = i < 2 ? d : f; k[i].K = rows; k[i].nseg = 1;
      k[i].out = out[i]; k[i].ldo = k[i].N;
      k[i].out_f32 = a.grad_dtype == FTP_F32; k[i].accumulate = a.accumulate;
      k[i].flags = fours(out[i], k[i].ldo, gs) ? TG_VEC_OUT : 0;
    }
    c.product(TG_TN, TG_GRAD, k, 3);
  }
}

int check_act8(const char* who, const ftp_act8_args* a, bool unpack) {
  NEED(a, FTP_ERR_ARG, "%s: NULL argument", who);
  TRY(check_common(who, a->rows, a->dtype, FTP_ACT_NONE));
  NEED(a->cols >= 1 && a->cols <= kMaxDim, FTP_ERR_ARG, "%s: cols must be 1 .. 2^20", who);
  if (unpack) TRY(check_mat(who, "y", a->y, a->ldy, a->rows, a->cols, a->dtype));
  else TRY(check_mat(who, "x", a->x, a->ldx, a->rows, a->cols, a->dtype));
  NEED(a->rows == 0 || (a->q && a->scales), FTP_ERR_ARG, "%s: q and scales must not be NULL", who);
  NEED(a->ldq >= a->cols && a->lds >= act8_groups(a->cols), FTP_ERR_ARG, "%s: rows of q or scales are too close (%d groups)", who, act8_groups(a->cols));
  return FTP_OK;
}

int check_embed(const char* who, const ftp_embed_args* a, bool backward) {
  NEED(a, FTP_ERR_ARG, "%s: NULL argument", who);
  TRY(check_common(who, a->rows, a->dtype, FTP_ACT_NONE));
  NEED(a->vocab >= 1, FTP_ERR_ARG, "%s: vocab must be positive", who);
  NEED(a->width >= 1 && a->width <= kMaxDim, FTP_ERR_ARG, "%s: width must be 1 .. 2^20", who);
  NEED(a->rows == 0 || a->ids, FTP_ERR_ARG, "%s: ids is NULL", who);
  NEED((uintptr_t)a->ids % (a->ids64 ? 8 : 4) == 0, FTP_ERR_ARG, "%s: ids is not aligned to its elements", who);
  NEED(std::isfinite(a->scale), FTP_ERR_VALUE, "%s: scale must be finite", who);
  if (!backward) {
    TRY(check_mat(who, "table", a->table, a->ldt, 1, a->width, a->dtype));
    TRY(check_mat(who, "out", a->out, a->ldo, a->rows, a->width, a->dtype));
  } else {
    TRY(check_mat(who, "dy", a->dy, a->lddy, a->rows, a->width, a->dtype));
    TRY(check_mat(who, "dtable", a->dtable, a->lddt, 1, a->width, FTP_F32));
  }
  return FTP_OK;
}

}  // namespace

extern "C" int ftp_linear_workspace(const ftp_linear_args* a, int backward, size_t* bytes) {
  NEED(bytes, FTP_ERR_ARG, "linear_workspace: NULL argument");
  TRY(check_linear("linear_workspace", a, backward != 0));
  *bytes = measure(a->dtype, [&](Call& c) { backward ? linear_backward(c, *a) : linear_forward(c, *a); });
  return FTP_OK;
}
extern "C" int ftp_linear_forward(const ftp_linear_args* a, void* stream) {
  TRY(check_linear("linear_forward", a, false));
  return run("linear_forward", a->dtype, a->ws, a->ws_bytes, stream, [&](Call& c) { linear_forward(c, *a); });
}
extern "C" int ftp_linear_backward(const ftp_linear_args* a, void* stream) {
  TRY(check_linear("linear_backward", a, true));
  return run("linear_backward", a->dtype, a->ws, a->ws_bytes, stream, [&](Call& c) { linear_backward(c, *a); });
}

extern "C" int ftp_ffn_workspace(const ftp_ffn_args* a, int backward, size_t* bytes) {
  NEED(bytes, FTP_ERR_ARG, "ffn_workspace: NULL argument");
  TRY(check_ffn("ffn_workspace", a, backward != 0));
  *bytes = measure(a->dtype, [&](Call& c) { backward ? ffn_backward(c, *a) : ffn_forward(c, *a); });
  return FTP_OK;
}
extern "C" int ftp_ffn_forward(const ftp_ffn_args* a, void* stream) {
  TRY(check_ffn("ffn_forward", a, false));
  return run("ffn_forward", a->dtype, a->ws, a->ws_bytes, stream, [&](Call& c) { ffn_forward(c, *a); });
}
extern "C" int ftp_ffn_backward(const ftp_ffn_args* a, void* stream) {
  TRY(check_ffn("ffn_backward", a, true));
  return run("ffn_backward", a->dtype, a->ws, a->ws_bytes, stream, [&](Call& c) { ffn_backward(c, *a); });
}

extern "C" int ftp_act8_pack(const ftp_act8_args* a, void* stream) {
  TRY(check_act8("act8_pack", a, false));
  if (a->rows) tk_act8_pack(a->dtype, (hipStream_t)stream, a->x, a->ldx, a->rows, a->cols, a->q, a->ldq, a->scales, a->lds);
  return launched("act8_pack");
}
extern "C" int ftp_act8_unpack(const ftp_act8_args* a, void* stream) {
  TRY(check_act8("act8_unpack", a, true));
  if (a->rows) tk_act8_unpack(a->dtype, (hipStream_t)stream, a->q, a->ldq, a->scales, a->lds, a->rows, a->cols, a->cols, a->y, a->ldy);
  return launched("act8_unpack");
}

extern "C" int ftp_embed_forward(const ftp_embed_args* a, void* stream) {
  TRY(check_embed("embed_forward", a, false));
  if (a->rows) tk_embed(a->dtype, (hipStream_t)stream, a->ids, a->ids64, a->rows, a->vocab, a->width, a->scale, a->table, a->ldt, a->out, a->ldo);
  return launched("embed_forward");
}
extern "C" int ftp_embed_backward_workspace(const ftp_embed_args* a, size_t* bytes) {
  NEED(bytes, FTP_ERR_ARG, "embed_backward_workspace: NULL argument");
  TRY(check_embed("embed_backward_workspace", a, true));
  *bytes = tk_embed_bwd_bytes(a->rows, a->vocab, a->width);
  return FTP_OK;
}
extern "C" int ftp_embed_backward(const ftp_embed_args* a, void* stream) {
  TRY(check_embed("embed_backward", a, true));
  const size_t need = tk_embed_bwd_bytes(a->rows, a->vocab, a->width);
  NEED(a->rows == 0 || (a->ws && a->ws_bytes >= need), FTP_ERR_ARG, "embed_backward: workspace of %zu bytes, needs %zu", a->ws ? a->ws_bytes : (size_t)0, need);
  NEED((uintptr_t)a->ws % 16 == 0, FTP_ERR_ARG, "embed_backward: the workspace must start on 16 bytes");
  tk_embed_bwd(a->dtype, (hipStream_t)stream, a->ids, a->ids64, a->rows, a->vocab, a->width, a->scale, a->pad_id, a->dy, a->lddy, a->dtable,
               a->lddt, a->accumulate, a->ws);
  return launched("embed_backward");
}
