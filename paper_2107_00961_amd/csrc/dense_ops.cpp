// C entry points of the operators of a dense residual block (resist_ops.h): argument checks, then the kernels.
#include <math.h>

#include "internal.h"

using namespace resist;

namespace {
constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int32_t kMaxCols = 1 << 24, kMaxLinear = 1 << 20;

int check_dtype(int32_t dtype) {
  return dtype == DT_F32 || dtype == DT_BF16 ? RESIST_OK : set_error(RESIST_EINVAL, "dtype %d", dtype);
}
int check_size(int64_t M, int32_t N) {
  if (M < 0 || M > kMaxRows) return set_error(RESIST_ESHAPE, "%lld rows", (long long)M);
  if (N < 1 || N > kMaxCols) return set_error(RESIST_ESHAPE, "rows of %d elements", N);
  return RESIST_OK;
}
// a device tensor that has to be there, and aligned
int check_ptr(const void *p, const char *what, bool needed = true) {
  if (!p) return needed ? set_error(RESIST_EINVAL, "%s is NULL", what) : RESIST_OK;
  return (uintptr_t)p & 15 ? set_error(RESIST_EINVAL, "%s is not 16-byte aligned", what) : RESIST_OK;
}
// a row stride: 0 is the row's length
int check_ld(int64_t *ld, int64_t n, const char *what, int64_t most = (int64_t)1 << 40) {
  if (*ld == 0) *ld = n;
  return *ld < n || *ld > most ? set_error(RESIST_ESHAPE, "row stride %lld of %s for rows of %lld", (long long)*ld, what, (long long)n) : RESIST_OK;
}
// one row, or none, has no next one: its stride says nothing, and is not looked at beyond this
int check_rows(const void *p, int64_t *ld, int64_t M, int64_t n, const char *what, bool needed = true, int64_t most = (int64_t)1 << 40) {
  if (M > 0) RESIST_TRY(check_ptr(p, what, needed));
  return p ? check_ld(ld, n, what, most) : RESIST_OK;
}
int check_drop(double p, const uint64_t *rng) {
  if (!(p >= 0. && p < 1.) || p * 4294967296. >= 4294967295.5) return set_error(RESIST_EINVAL, "dropout probability %g", p);
  if (p > 0. && !rng) return set_error(RESIST_EINVAL, "rng is NULL");
  return (uintptr_t)rng & 7 ? set_error(RESIST_EINVAL, "rng is not 8-byte aligned") : RESIST_OK;
}
int check_act(int32_t act) {
  return act < RESIST_ACT_NONE || act > RESIST_ACT_SILU ? set_error(RESIST_EINVAL, "act %d", act) : RESIST_OK;
}
int check_vec(const float *p, const char *what) { return check_ptr(p, what, false); }
}  // namespace

extern "C" int resist_layernorm_workspace_bytes(int64_t M, int32_t N, int64_t *bytes) {
  RESIST_TRY(check_size(M, N));
  if (!bytes) return set_error(RESIST_EINVAL, "bytes is NULL");
  *bytes = layernorm_workspace_floats(M, N) * 4;
  return RESIST_OK;
}

extern "C" int resist_layernorm_forward(int64_t M, int32_t N, int32_t dtype, const void *x, int64_t ldx, const float *gamma, const float *beta,
                                        float eps, void *y, int64_t ldy, float *mean, float *rstd, void *hip_stream) {
  RESIST_TRY(check_dtype(dtype));
  RESIST_TRY(check_size(M, N));
  if (!(eps >= 0.f)) return set_error(RESIST_EINVAL, "eps %g", eps);
  RESIST_TRY(check_rows(x, &ldx, M, N, "x"));
  RESIST_TRY(check_rows(y, &ldy, M, N, "y"));
  RESIST_TRY(check_vec(gamma, "gamma"));
  RESIST_TRY(check_vec(beta, "beta"));
  RESIST_TRY(check_vec(mean, "mean"));
  RESIST_TRY(check_vec(rstd, "rstd"));
  return layernorm_fwd(dtype, LayerNorm{M, N, x, ldx, gamma, beta, mean, rstd, eps}, y, ldy, (hipStream_t)hip_stream);
}

extern "C" int resist_layernorm_backward(int64_t M, int32_t N, int32_t dtype, const void *dy, int64_t lddy, const void *x, int64_t ldx,
                                         const float *gamma, const float *mean, const float *rstd, const void *addend, int64_t ldadd, void *dx,
                                         int64_t lddx, float *dgamma, float *dbeta, void *workspace, int64_t workspace_bytes, void *hip_stream) {
  RESIST_TRY(check_dtype(dtype));
  RESIST_TRY(check_size(M, N));
  RESIST_TRY(check_rows(dy, &lddy, M, N, "dy"));
  RESIST_TRY(check_rows(x, &ldx, M, N, "x"));
  RESIST_TRY(check_rows(addend, &ldadd, M, N, "addend", false));
  RESIST_TRY(check_rows(dx, &lddx, M, N, "dx"));
  RESIST_TRY(check_vec(gamma, "gamma"));
  if (M > 0) {
    RESIST_TRY(check_ptr(mean, "mean"));
    RESIST_TRY(check_ptr(rstd, "rstd"));
    RESIST_TRY(check_ptr(workspace, "workspace"));
    if (workspace_bytes < layernorm_workspace_floats(M, N) * 4) return set_error(RESIST_EWORKSPACE, "workspace too small for the partial sums");
  }
  RESIST_TRY(check_vec(dgamma, "dgamma"));
  RESIST_TRY(check_vec(dbeta, "dbeta"));
  return layernorm_bwd(dtype, LayerNorm{M, N, x, ldx, gamma, nullptr, const_cast<float *>(mean), const_cast<float *>(rstd), 0.f}, dy, lddy, addend, ldadd,
                       dx, lddx, dgamma, dbeta, (float *)workspace, (hipStream_t)hip_stream);
}

extern "C" int resist_dropout_forward(int64_t M, int32_t N, int32_t dtype, const void *x, int64_t ldx, double p, const uint64_t *rng,
                                      const void *residual, int64_t ldr, void *y, int64_t ldy, void *hip_stream) {
  RESIST_TRY(check_dtype(dtype));
  RESIST_TRY(check_size(M, N));
  RESIST_TRY(check_drop(p, rng));
  RESIST_TRY(check_rows(x, &ldx, M, N, "x"));
  RESIST_TRY(check_rows(residual, &ldr, M, N, "residual", false));
  RESIST_TRY(check_rows(y, &ldy, M, N, "y"));
  return dropout(dtype, M, N, x, ldx, residual, ldr, RESIST_ACT_NONE, nullptr, 0, DropSpec{p, rng}, y, ldy, (hipStream_t)hip_stream);
}

extern "C" int resist_dropout_backward(int64_t M, int32_t N, int32_t dtype, const void *dy, int64_t lddy, double p, const uint64_t *rng, int32_t act,
                                       const void *z, int64_t ldz, void *dx, int64_t lddx, void *hip_stream) {
  RESIST_TRY(check_dtype(dtype));
  RESIST_TRY(check_size(M, N));
  RESIST_TRY(check_drop(p, rng));
  RESIST_TRY(check_act(act));
  RESIST_TRY(check_rows(dy, &lddy, M, N, "dy"));
  if (act != RESIST_ACT_NONE) RESIST_TRY(check_rows(z, &ldz, M, N, "z"));
  RESIST_TRY(check_rows(dx, &lddx, M, N, "dx"));
  return dropout(dtype, M, N, dy, lddy, nullptr, 0, act, z, ldz, DropSpec{p, rng}, dx, lddx, (hipStream_t)hip_stream);
}

namespace {
int to_linear(const resist_linear_shape *s, LinearShape *o) {
  if (!s) return set_error(RESIST_EINVAL, "shape is NULL");
  RESIST_TRY(check_dtype(s->dtype));
  if (s->M < 0 || s->M > kMaxRows) return set_error(RESIST_ESHAPE, "%lld rows", (long long)s->M);
  if (s->K < 1 || s->N < 1 || s->K > kMaxLinear || s->N > kMaxLinear) return set_error(RESIST_ESHAPE, "dense layer of %d inputs and %d outputs", s->K, s->N);
  *o = LinearShape{s->M, s->K, s->N, s->ldx, s->ldy};
  RESIST_TRY(check_ld(&o->ldx, s->K, "x", kMaxLinear));
  return check_ld(&o->ldy, s->N, "y", kMaxLinear);
}
int work_of(const LinearShape &s, int dt, int op, int64_t *need) {
  *need = linear_workspace(s, dt, op);
  return *need < 0 ? set_error(RESIST_ESHAPE, "dense layer of %lld rows, %d inputs and %d outputs", (long long)s.M, s.K, s.N) : RESIST_OK;
}
int check_work(const LinearShape &s, int dt, int op, const void *workspace, int64_t bytes) {
  int64_t need;
  RESIST_TRY(work_of(s, dt, op, &need));
  if (need == 0) return RESIST_OK;
  RESIST_TRY(check_ptr(workspace, "workspace"));
  return bytes < need ? set_error(RESIST_EWORKSPACE, "workspace of %lld bytes where %lld are needed", (long long)bytes, (long long)need) : RESIST_OK;
}
}  // namespace

extern "C" int resist_linear_workspace_bytes(const resist_linear_shape *s, int32_t op, int64_t *bytes) {
  LinearShape l;
  RESIST_TRY(to_linear(s, &l));
  if (op < 0 || op > 2) return set_error(RESIST_EINVAL, "op %d", op);
  if (!bytes) return set_error(RESIST_EINVAL, "bytes is NULL");
  return work_of(l, s->dtype, op, bytes);
}

extern "C" int resist_linear_forward(const resist_linear_shape *s, const void *x, const void *w, const resist_linear_epilogue *epilogue, void *y,
                                     void *workspace, int64_t workspace_bytes, void *hip_stream) {
  LinearShape l;
  RESIST_TRY(to_linear(s, &l));
  LinearEpilogue e{};
  if (epilogue) e = LinearEpilogue{epilogue->bias, epilogue->act, DropSpec{epilogue->p, epilogue->rng}, epilogue->residual, epilogue->ldr, epilogue->z, epilogue->ldz};
  RESIST_TRY(check_act(e.act));
  RESIST_TRY(check_drop(e.drop.p, e.drop.rng));
  RESIST_TRY(check_vec(e.bias, "bias"));
  RESIST_TRY(check_rows(e.residual, &e.ldr, l.M, l.N, "residual", false, kMaxLinear));
  RESIST_TRY(check_rows(e.z, &e.ldz, l.M, l.N, "z", false, kMaxLinear));
  if (l.M == 0) return RESIST_OK;
  RESIST_TRY(check_ptr(x, "x"));
  RESIST_TRY(check_ptr(w, "w"));
  RESIST_TRY(check_ptr(y, "y"));
  RESIST_TRY(check_work(l, s->dtype, 0, workspace, workspace_bytes));
  return linear_fwd(l, s->dtype, x, w, e, y, workspace, (hipStream_t)hip_stream);
}

extern "C" int resist_linear_dgrad(const resist_linear_shape *s, const void *dz, const void *w, const resist_linear_through *through, void *dx,
                                   void *workspace, int64_t workspace_bytes, void *hip_stream) {
  LinearShape l;
  RESIST_TRY(to_linear(s, &l));
  LinearThrough t{};
  if (through) t = LinearThrough{through->act, through->z, through->ldz, DropSpec{through->p, through->rng}};
  RESIST_TRY(check_act(t.act));
  RESIST_TRY(check_drop(t.drop.p, t.drop.rng));
  if (t.act != RESIST_ACT_NONE) RESIST_TRY(check_rows(t.z, &t.ldz, l.M, l.K, "z", true, kMaxLinear));
  if (l.M == 0) return RESIST_OK;
  RESIST_TRY(check_ptr(dz, "dz"));
  RESIST_TRY(check_ptr(w, "w"));
  RESIST_TRY(check_ptr(dx, "dx"));
  RESIST_TRY(check_work(l, s->dtype, 1, workspace, workspace_bytes));
  return linear_dgrad(l, s->dtype, dz, w, t, dx, workspace, (hipStream_t)hip_stream);
}

extern "C" int resist_linear_wgrad(const resist_linear_shape *s, const void *dz, const void *x, float *dw, float *db, void *workspace,
                                   int64_t workspace_bytes, void *hip_stream) {
  LinearShape l;
  RESIST_TRY(to_linear(s, &l));
  RESIST_TRY(check_ptr(dw, "dw"));
  RESIST_TRY(check_ptr(db, "db", false));
  if (l.M == 0) {   // no rows: the gradients are there, and zero
    RESIST_TRY(fill_zero_f32(dw, (int64_t)l.N * l.K, (hipStream_t)hip_stream));
    return db ? fill_zero_f32(db, l.N, (hipStream_t)hip_stream) : RESIST_OK;
  }
  RESIST_TRY(check_ptr(dz, "dz"));
  RESIST_TRY(check_ptr(x, "x"));
  RESIST_TRY(check_work(l, s->dtype, 2, workspace, workspace_bytes));
  return linear_wgrad(l, s->dtype, dz, x, dw, db, workspace, (hipStream_t)hip_stream);
}
