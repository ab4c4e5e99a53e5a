// C ABI of dropout and the residual norm: argument checks and entry points.
#include "abi_check.h"
#include "norm.h"

#include <cmath>

using namespace lat;

static const int64_t MAX_ROWS = (int64_t)1 << 30;
// blocks of 256 threads whose global thread number fits 32 bits
static const int64_t MAX_BLOCKS = ((int64_t)1 << 24) - 1;

#define TRY(expr)                          \
  do {                                     \
    lattice_status st__ = (expr);          \
    if (st__ != LATTICE_OK) return st__;   \
  } while (0)

static lattice_status drop_args(const lattice_dropout_desc* d, DropArgs* a) {
  if (!d) return LATTICE_OK;
  REQUIRE(d->p >= 0 && d->p < 1, "p outside 0 .. 1");
  const double t = std::floor(d->p * 65536 + 0.5);
  REQUIRE(t < 65536, "p rounds to 1");
  a->t = (uint32_t)t;
  a->factor = (float)(65536.0 / (65536.0 - t));
  a->site = d->site;
  a->rng = d->rng;
  if (a->t) REQUIRE(d->rng && (uintptr_t)d->rng % 8 == 0, "rng is null or not 8-byte aligned");
  return LATTICE_OK;
}

static lattice_status check_rows(const char* name, const void* p, int64_t stride, int cols, lattice_dtype dt) {
  REQUIRE(p, "null %s", name);
  REQUIRE((uintptr_t)p % esize(dt) == 0, "%s is not aligned to its elements", name);
  REQUIRE(stride >= cols, "%s: row stride %lld < %d columns", name, (long long)stride, cols);
  return LATTICE_OK;
}

// Where a result takes the place of an input, row by row.
static lattice_status check_same(const char* name, const void* out, int64_t out_stride, const void* in, int64_t in_stride) {
  REQUIRE(!out || out != in || out_stride == in_stride, "%s is an input's memory with another row stride", name);
  return LATTICE_OK;
}

static lattice_status check_norm(const lattice_add_rmsnorm_desc* d, int64_t rows, DropArgs* drop) {
  REQUIRE(d, "null norm descriptor");
  REQUIRE(d->dtype == LATTICE_F32 || d->dtype == LATTICE_BF16, "bad dtype");
  REQUIRE(d->cols >= 1, "cols must be at least 1");
  REQUIRE(d->eps >= 0 && std::isfinite(d->eps), "eps must not be negative");
  REQUIRE(rows >= 0, "negative rows");
  TRY(drop_args(d->dropout, drop));
  if (d->cols > NORM_MAX_COLS) FAIL(LATTICE_ERR_UNSUPPORTED, "cols above %d", NORM_MAX_COLS);
  if (rows >= MAX_ROWS) FAIL(LATTICE_ERR_UNSUPPORTED, "rows must be < 2^30");
  return LATTICE_OK;
}

static RowTensor tensor(const void* p, int64_t ld) { return {const_cast<void*>(p), ld}; }

static NormArgs norm_args(const lattice_add_rmsnorm_desc* d, int64_t rows, const DropArgs& drop) {
  NormArgs a;
  a.dt = dt_of(d->dtype);
  a.rows = rows;
  a.cols = d->cols;
  a.eps = d->eps;
  a.gain = d->gain;
  a.drop = drop;
  return a;
}

extern "C" {

lattice_status lattice_dropout(const lattice_dropout_desc* d, lattice_dtype dtype, int64_t rows, int32_t cols,
                               const void* x, int64_t x_stride, void* out, int64_t out_stride, void* stream) {
  REQUIRE(d, "null dropout descriptor");
  DropArgs drop;
  TRY(drop_args(d, &drop));
  REQUIRE(dtype == LATTICE_F32 || dtype == LATTICE_BF16, "bad dtype");
  REQUIRE(rows >= 0 && cols >= 0, "negative sizes");
  if (rows == 0 || cols == 0) return LATTICE_OK;
  if (rows >= MAX_ROWS || cols >= MAX_ROWS) FAIL(LATTICE_ERR_UNSUPPORTED, "rows and cols must be < 2^30");
  TRY(check_rows("x", x, x_stride, cols, dtype));
  TRY(check_rows("out", out, out_stride, cols, dtype));
  TRY(check_same("out", out, out_stride, x, x_stride));
  if (rows * (((int64_t)cols + 7) / 8) > MAX_BLOCKS * 1024)
    FAIL(LATTICE_ERR_UNSUPPORTED, "rows x cols too many for one launch");
  HIPRET(dropout(dt_of(dtype), rows, cols, drop, tensor(x, x_stride), tensor(out, out_stride), strm(stream)));
  return LATTICE_OK;
}

lattice_status lattice_add_rmsnorm_fwd(const lattice_add_rmsnorm_desc* d, int64_t rows, const void* x,
                                       int64_t x_stride, const void* residual, int64_t residual_stride, void* h,
                                       int64_t h_stride, void* y, int64_t y_stride, uint8_t* q, int64_t ldq,
                                       float* scales, void* stream) {
  DropArgs drop;
  TRY(check_norm(d, rows, &drop));
  if (rows == 0) return LATTICE_OK;
  TRY(check_rows("x", x, x_stride, d->cols, d->dtype));
  if (residual) TRY(check_rows("residual", residual, residual_stride, d->cols, d->dtype));
  if (h) TRY(check_rows("h", h, h_stride, d->cols, d->dtype));
  if (y) TRY(check_rows("y", y, y_stride, d->cols, d->dtype));
  REQUIRE(y || q, "neither y nor q");
  REQUIRE(!h || h != y, "h and y are the same memory");
  TRY(check_same("h", h, h_stride, x, x_stride));
  TRY(check_same("h", h, h_stride, residual, residual_stride));
  TRY(check_same("y", y, y_stride, x, x_stride));
  TRY(check_same("y", y, y_stride, residual, residual_stride));
  if (q) {
    REQUIRE(scales, "q without scales");
    REQUIRE(ldq >= d->cols && ldq % 16 == 0, "ldq %lld is no multiple of 16 that holds a row", (long long)ldq);
    REQUIRE((uintptr_t)q % 16 == 0, "q is not 16-byte aligned");
  }
  NormArgs a = norm_args(d, rows, drop);
  a.x = tensor(x, x_stride);
  a.r = tensor(residual, residual_stride);
  a.h = tensor(h, h_stride);
  a.y = tensor(y, y_stride);
  a.q = q;
  a.ldq = ldq;
  a.scales = scales;
  HIPRET(add_rmsnorm_fwd(a, strm(stream)));
  return LATTICE_OK;
}

size_t lattice_add_rmsnorm_bwd_workspace(const lattice_add_rmsnorm_desc* d, int64_t rows) {
  DropArgs drop;
  if (check_norm(d, rows, &drop) != LATTICE_OK) return 0;
  return add_rmsnorm_bwd_workspace(rows, d->cols);
}

lattice_status lattice_add_rmsnorm_bwd(const lattice_add_rmsnorm_desc* d, int64_t rows, const void* h,
                                       int64_t h_stride, const void* dy, int64_t dy_stride, const void* dh,
                                       int64_t dh_stride, void* d_residual, int64_t d_residual_stride, void* dx,
                                       int64_t dx_stride, float* dgain, void* ws, size_t ws_bytes, void* stream) {
  DropArgs drop;
  TRY(check_norm(d, rows, &drop));
  if (rows > 0) {
    TRY(check_rows("h", h, h_stride, d->cols, d->dtype));
    TRY(check_rows("dy", dy, dy_stride, d->cols, d->dtype));
    if (dh) TRY(check_rows("dh", dh, dh_stride, d->cols, d->dtype));
    if (d_residual) TRY(check_rows("d_residual", d_residual, d_residual_stride, d->cols, d->dtype));
    if (dx) TRY(check_rows("dx", dx, dx_stride, d->cols, d->dtype));
    REQUIRE(!dx || dx != d_residual, "d_residual and dx are the same memory");
    const struct { const void* p; int64_t stride; } in[] = {{h, h_stride}, {dy, dy_stride}, {dh, dh_stride}};
    for (const auto& t : in) {
      TRY(check_same("d_residual", d_residual, d_residual_stride, t.p, t.stride));
      TRY(check_same("dx", dx, dx_stride, t.p, t.stride));
    }
    if (dgain) {
      const size_t need = add_rmsnorm_bwd_workspace(rows, d->cols);
      if (!ws || ws_bytes < need) FAIL(LATTICE_ERR_WORKSPACE, "workspace %zu < %zu", ws_bytes, need);
      REQUIRE((uintptr_t)ws % 16 == 0, "workspace is not 16-byte aligned");
    }
  }
  NormArgs a = norm_args(d, rows, drop);
  a.h = tensor(h, h_stride);
  a.dy = tensor(dy, dy_stride);
  a.dh = tensor(dh, dh_stride);
  a.dr = tensor(d_residual, d_residual_stride);
  a.dx = tensor(dx, dx_stride);
  a.dgain = dgain;
  HIPRET(add_rmsnorm_bwd(a, ws, strm(stream)));
  return LATTICE_OK;
}

}  // extern "C"
