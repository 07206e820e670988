// Host side of the training operators: argument checks, scratch and the
// launches of gnn_layer_norm*, gnn_gated* and gnn_clip_grads.  Like the row
// operators they allocate nothing and wait for nothing.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <vector>

#include "../../include/gnn.h"
#include "gnn_internal.h"

using namespace gnn;

namespace {

constexpr int MAX_WIDTH = 16384;
constexpr int64_t MAX_ROWS = (int64_t)1 << 28;
constexpr int64_t MAX_STRIDE = (int64_t)1 << 31;
constexpr int64_t DIRECT_STRIDE = (int64_t)1 << 21;  // most that a product's offsets hold

int bad(int code, const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return set_error(code, buf);
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
int64_t up8(int64_t n) { return (n + 7) & ~(int64_t)7; }

int launched(hipError_t e, const char *what) {
  if (e == hipSuccess) return GNN_OK;
  (void)hipGetLastError();
  return bad(GNN_E_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
}

bool float_type(int t) { return t == GNN_FP32 || t == GNN_BF16 || t == GNN_F16; }

int check_rows(int64_t n_rows) {
  if (n_rows < 0) return bad(GNN_E_INVALID_ARG, "negative row count");
  if (n_rows > MAX_ROWS) return bad(GNN_E_UNSUPPORTED, "more than 2^28 rows");
  return GNN_OK;
}

int check_width(const char *what, int64_t w) {
  if (w < 1) return bad(GNN_E_INVALID_ARG, "%s must be positive", what);
  if (w > MAX_WIDTH) return bad(GNN_E_UNSUPPORTED, "%s above %d is not supported", what, MAX_WIDTH);
  return GNN_OK;
}

// A table of rows: pointer, element type, stride in elements.
int check_table(const char *what, const void *p, int type, int64_t stride, int64_t width) {
  if (!p) return bad(GNN_E_INVALID_ARG, "%s is NULL", what);
  if ((uintptr_t)p % type_bytes(type))
    return bad(GNN_E_INVALID_ARG, "%s is not aligned to its elements", what);
  if (stride < width || stride > MAX_STRIDE)
    return bad(GNN_E_INVALID_ARG, "%s stride %lld outside %lld..2^31", what, (long long)stride,
               (long long)width);
  return GNN_OK;
}

int check_vector(const char *what, const void *p, int type) { return check_table(what, p, type, 1, 1); }

int check_scratch(const void *ws, int64_t have, size_t need) {
  if (need == 0) return GNN_OK;
  if (!ws || have < 0 || (size_t)have < need)
    return bad(GNN_E_INVALID_ARG, "workspace of %lld bytes, %zu needed", (long long)(ws ? have : 0),
               need);
  if ((uintptr_t)ws % 256) return bad(GNN_E_INVALID_ARG, "workspace is not aligned to 256 bytes");
  return GNN_OK;
}

int current_device(int *dev) {
  int n = 0;
  if (hipGetDeviceCount(&n) != hipSuccess || n <= 0 || hipGetDevice(dev) != hipSuccess) {
    (void)hipGetLastError();
    return bad(GNN_E_NO_DEVICE, "no HIP device visible");
  }
  return GNN_OK;
}

struct Carve {
  size_t total = 0;
  size_t take(size_t bytes) {
    const size_t at = total;
    total += up256(bytes);
    return at;
  }
};

int sum_columns(SumArgs s, unsigned char *scratch, const char *what, hipStream_t stream) {
  s.part = (float *)scratch;
  return launched(launch_colsum(s, stream), what);
}

}  // namespace

// ----------------------------------------------------------- layer norm ---

namespace {

int check_norm(int64_t n_rows, int32_t width, int type, float eps) {
  int rc = check_rows(n_rows);
  if (rc || (rc = check_width("width", width))) return rc;
  if (!float_type(type)) return bad(GNN_E_INVALID_ARG, "type %d is not a float type", type);
  if (!(eps > 0.f) || !(eps < 1.f)) return bad(GNN_E_INVALID_ARG, "eps outside (0, 1)");
  return GNN_OK;
}

}  // namespace

extern "C" {

int gnn_layer_norm(const void *x, int32_t type, int64_t x_stride, int64_t n_rows, int32_t width,
                   const float *gamma, const float *beta, float eps, void *y, int64_t y_stride,
                   float *mean, float *rstd, hipStream_t stream) {
  int rc = check_norm(n_rows, width, type, eps);
  if (rc) return rc;
  if (n_rows == 0) return GNN_OK;
  if ((rc = check_table("x", x, type, x_stride, width)) ||
      (rc = check_table("y", y, type, y_stride, width)) ||
      (rc = check_vector("gamma", gamma, GNN_FP32)) || (rc = check_vector("beta", beta, GNN_FP32)))
    return rc;
  if (y == x && y_stride != x_stride)
    return bad(GNN_E_INVALID_ARG, "y overlaps x: in place, the strides have to be equal");
  if (!mean != !rstd) return bad(GNN_E_INVALID_ARG, "mean and rstd go together");
  if (mean && ((rc = check_vector("mean", mean, GNN_FP32)) ||
               (rc = check_vector("rstd", rstd, GNN_FP32))))
    return rc;
  LayerNormArgs a;
  a.x = x;
  a.type = type;
  a.x_stride = x_stride;
  a.y_stride = y_stride;
  a.n = n_rows;
  a.width = width;
  a.eps = eps;
  a.gamma = gamma;
  a.beta = beta;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  return launched(launch_layer_norm(a, stream), "layer norm");
}

size_t gnn_layer_norm_workspace(int64_t n_rows, int32_t width) {
  if (n_rows < 0 || n_rows > MAX_ROWS || width < 1 || width > MAX_WIDTH) return 0;
  const int64_t parts = layer_norm_parts(n_rows, width);
  return up256((size_t)parts * 2 * width * 4) + up256(colsum_scratch(parts, 2 * width, true));
}

int gnn_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                            int32_t type, int64_t n_rows, int32_t width, const float *gamma,
                            const float *mean, const float *rstd, void *dx, int64_t dx_stride,
                            float *dgamma, float *dbeta, void *workspace, int64_t workspace_bytes,
                            hipStream_t stream) {
  int rc = check_norm(n_rows, width, type, 0.5f);
  if (rc) return rc;
  if ((rc = check_vector("dgamma", dgamma, GNN_FP32)) ||
      (rc = check_vector("dbeta", dbeta, GNN_FP32)))
    return rc;
  if (n_rows > 0 && ((rc = check_table("dy", dy, type, dy_stride, width)) ||
                     (rc = check_table("x", x, type, x_stride, width)) ||
                     (rc = check_table("dx", dx, type, dx_stride, width)) ||
                     (rc = check_vector("gamma", gamma, GNN_FP32)) ||
                     (rc = check_vector("mean", mean, GNN_FP32)) ||
                     (rc = check_vector("rstd", rstd, GNN_FP32))))
    return rc;
  if (n_rows > 0 && (dx == x || (dx == dy && dx_stride != dy_stride)))
    return bad(GNN_E_INVALID_ARG, "dx overlaps x, or dy with another stride");
  if ((rc = check_scratch(workspace, workspace_bytes, gnn_layer_norm_workspace(n_rows, width))))
    return rc;
  unsigned char *ws = (unsigned char *)workspace;
  SumArgs s;
  s.x = ws;
  s.x_type = GNN_FP32;
  s.x_stride = s.width = 2 * width;
  s.y[0] = dgamma;
  s.y[1] = dbeta;
  s.y_type = GNN_FP32;
  s.split = s.skip = width;
  if (n_rows > 0) {
    LayerNormArgs a;
    a.dy = dy;
    a.dy_stride = dy_stride;
    a.x = x;
    a.x_stride = x_stride;
    a.type = type;
    a.n = n_rows;
    a.width = width;
    a.gamma = gamma;
    a.mean = (float *)mean;
    a.rstd = (float *)rstd;
    a.dx = dx;
    a.dx_stride = dx_stride;
    a.part = (float *)ws;
    if ((rc = launched(launch_layer_norm_backward(a, stream), "layer norm gradient"))) return rc;
    s.n = layer_norm_parts(n_rows, width);
  }
  return sum_columns(s, ws + up256((size_t)s.n * 2 * width * 4), "parameter gradients", stream);
}

}  // extern "C"

// ---------------------------------------------------------- gated block ---

namespace {

int check_gated_dims(const gnn_gated_dims *d) {
  if (!d) return bad(GNN_E_INVALID_ARG, "dims is NULL");
  if (d->struct_size != sizeof(gnn_gated_dims))
    return bad(GNN_E_INVALID_ARG, "gnn_gated_dims.struct_size mismatch");
  int rc = check_width("in_features", d->in_features);
  if (rc || (rc = check_width("hidden", d->hidden)) ||
      (rc = check_width("out_features", d->out_features)))
    return rc;
  if (d->dtype != GNN_BF16 && d->dtype != GNN_F16)
    return bad(float_type(d->dtype) || d->dtype == GNN_INT8 ? GNN_E_UNSUPPORTED : GNN_E_INVALID_ARG,
               "dtype is GNN_BF16 or GNN_F16");
  if (d->activation < GNN_SILU || d->activation > GNN_RELU)
    return bad(GNN_E_INVALID_ARG, "activation %d unknown", d->activation);
  return GNN_OK;
}

int check_gated_weights(const gnn_gated_weights *w, const char *what) {
  if (!w) return bad(GNN_E_INVALID_ARG, "%s is NULL", what);
  if (w->struct_size != sizeof(gnn_gated_weights))
    return bad(GNN_E_INVALID_ARG, "gnn_gated_weights.struct_size mismatch");
  const struct {
    const char *name;
    const void *p;
    bool need;
  } all[] = {{"gate", w->gate, true},          {"up", w->up, true},
             {"down", w->down, true},          {"gate_bias", w->gate_bias, false},
             {"up_bias", w->up_bias, false},   {"down_bias", w->down_bias, false}};
  for (const auto &t : all) {
    if (!t.p && t.need) return bad(GNN_E_INVALID_ARG, "%s: %s is NULL", what, t.name);
    if ((uintptr_t)t.p % 2)
      return bad(GNN_E_INVALID_ARG, "%s: %s is not aligned to its elements", what, t.name);
  }
  return GNN_OK;
}

// A table that a product reads: as it lies, or copied to aligned rows that zeros
// fill up to a multiple of eight elements.
struct Operand {
  const void *p = nullptr;
  int64_t stride = 0, rows = 0;
  int32_t width = 0;
  bool copy = false;
  size_t at = 0;

  Operand(const void *ptr, int64_t ld, int64_t n, int32_t w, bool aligned) {
    p = ptr;
    stride = ld;
    rows = n;
    width = w;
    copy = !aligned || w % 8 != 0;
  }
  void place(Carve &c) {
    if (copy) at = c.take((size_t)rows * up8(width) * 2);
  }
  // What the products read from here on, and (a) what has to be copied for it.
  void fetch(unsigned char *ws, PackArgs *a) {
    if (!copy) return;
    if (a) {
      a->x[a->count] = p;
      a->y[a->count] = ws + at;
      a->stride[a->count] = stride;
      a->rows[a->count] = rows;
      a->width[a->count++] = width;
    }
    p = ws + at;
    stride = up8(width);
  }
};

bool lies_aligned(const void *p, int64_t stride) {
  return (uintptr_t)p % 16 == 0 && stride % 8 == 0 && stride <= DIRECT_STRIDE;
}

struct GatedForward {
  bool few = false, thin = false;
  Operand x, gate, up, down;
  size_t h = 0, part = 0;
  int splits = 1;
  int gate_tile = 0, down_tile = 0;
  Carve c;
  GatedForward(const gnn_gated_dims &d, int64_t n, int n_cu, const void *xp, int64_t ld, bool x_in,
               const gnn_gated_weights *w, bool w_in)
      : x(xp, ld, n, d.in_features, x_in),
        gate(w ? w->gate : nullptr, d.in_features, d.hidden, d.in_features, w_in),
        up(w ? w->up : nullptr, d.in_features, d.hidden, d.in_features, w_in),
        down(w ? w->down : nullptr, d.hidden, d.out_features, d.hidden, w_in) {
    few = n <= FEW_ROWS;
    if (few && n > 0) {
      splits = few_splits(n, d.out_features, d.hidden, n_cu);
      part = c.take(few_part_bytes(n, d.out_features, splits));
    } else if ((thin = thin_fits(n, d.in_features, d.hidden, d.out_features, n_cu))) {
      for (Operand *o : {&gate, &up, &down}) o->place(c);
      return;
    } else {
      for (Operand *o : {&x, &gate, &up, &down}) o->place(c);
      gate_tile = product_plan(PRODUCT_GATE, n, d.hidden, d.in_features, n_cu).tile;
      down_tile = product_plan(PRODUCT_DOWN, n, d.out_features, d.hidden, n_cu).tile;
    }
    h = c.take((size_t)n * up8(d.hidden) * (n <= TWO_ROWS ? 4 : 2));
  }
};

struct GatedBackward {
  Operand x, dy, gate, up, down;
  ProductPlan grad, dx, dgu, dd;
  // two: h, dg and du in two 16-bit numbers (few rows, as gated_few)
  // dy_sums: dy's sums over rows come with the down projection's gradient
  bool thin = false, two = false, dy_sums = false;
  // half: fp16, whose h, dg and du are multiplied by powers of two
  bool half = false;
  size_t h = 0, g = 0, part = 0, sums = 0, dy_sum = 0, colsum = 0, sizes = 0, scales = 0;
  int64_t sum_rows = 0;
  Carve c;
  GatedBackward(const gnn_gated_dims &d, int64_t n, int n_cu, const void *xp, int64_t x_ld,
                const void *dp, int64_t d_ld, bool rows_in, const gnn_gated_weights *w, bool w_in)
      : x(xp, x_ld, n, d.in_features, rows_in),
        dy(dp, d_ld, n, d.out_features, rows_in),
        gate(w ? w->gate : nullptr, d.in_features, d.hidden, d.in_features, w_in),
        up(w ? w->up : nullptr, d.in_features, d.hidden, d.in_features, w_in),
        down(w ? w->down : nullptr, d.hidden, d.out_features, d.hidden, w_in) {
    const int64_t hp = up8(d.hidden), kp = up8(d.in_features);
    for (Operand *o : {&x, &dy, &gate, &up, &down}) o->place(c);
    grad = product_plan(PRODUCT_GRAD, n, d.hidden, d.in_features, n_cu);
    dx = product_plan(PRODUCT_ROWS, n, d.in_features, 2 * hp, n_cu);
    dgu = product_plan(PRODUCT_WEIGHTS, 2 * hp, d.in_features, n, n_cu);
    dd = product_plan(PRODUCT_WEIGHTS, d.out_features, d.hidden, n, n_cu);
    two = n > 0 && n <= TWO_ROWS;
    if (two) grad.tile = TILE_128_DEEP;
    h = c.take((size_t)n * hp * (two ? 4 : 2));
    g = c.take((size_t)n * hp * (two ? 8 : 4));
    // the parts of one product are joined before the next one's are written
    size_t most = 0;
    if (dgu.splits > 1) most = (size_t)dgu.splits * 2 * hp * kp * 4;
    if (dd.splits > 1) most = std::max(most, (size_t)dd.splits * d.out_features * hp * 4);
    part = c.take(most);
    thin = thin_fits(n, d.in_features, d.hidden, d.out_features, n_cu);
    // sums of dg and du over rows
    sum_rows = thin ? thin_sum_rows(n) : product_sum_rows(grad.tile, n);
    sums = c.take((size_t)sum_rows * 2 * hp * 4);
    dy_sum = c.take((size_t)dd.splits * d.out_features * 4);
    dy_sums = product_sums(dd.tile) && !two;  // which goes through dy twice
    colsum = c.take(std::max(colsum_scratch(sum_rows, (int32_t)(2 * hp), true),
                             dy_sums ? colsum_scratch(dd.splits, d.out_features, true)
                                     : colsum_scratch(n, d.out_features, false)));
    if ((half = d.dtype == GNN_F16 && n > 0)) {
      sizes = c.take(SIZES * SIZE_PARTS * 4);
      scales = c.take(2 * 4);
    }
  }
};

// Where no device is visible, sizes are those of one with 256 compute units.
int devices_cu(int *n_cu) {
  int dev = 0;
  const int rc = current_device(&dev);
  *n_cu = rc ? 256 : cu_count(dev);
  return rc;
}

bool weights_aligned(const gnn_gated_dims &d, const gnn_gated_weights &w) {
  return lies_aligned(w.gate, up8(d.in_features)) && lies_aligned(w.up, up8(d.in_features)) &&
         lies_aligned(w.down, up8(d.hidden));
}

}  // namespace

extern "C" {

size_t gnn_gated_workspace(const gnn_gated_dims *d, int64_t n_rows, int32_t backward,
                           int32_t aligned) {
  if (check_gated_dims(d) || check_rows(n_rows)) return 0;
  if (n_rows == 0 && !backward) return 0;
  int n_cu = 0;
  (void)devices_cu(&n_cu);
  if (!backward) return GatedForward(*d, n_rows, n_cu, nullptr, 0, aligned, nullptr, aligned).c.total;
  return GatedBackward(*d, n_rows, n_cu, nullptr, 0, nullptr, 0, aligned, nullptr, aligned).c.total;
}

int gnn_gated(const gnn_gated_dims *d, const gnn_gated_weights *w, const void *x, int64_t x_stride,
              int64_t n_rows, void *y, int64_t y_stride, void *workspace, int64_t workspace_bytes,
              hipStream_t stream) {
  int rc = check_gated_dims(d);
  if (rc || (rc = check_gated_weights(w, "weights")) || (rc = check_rows(n_rows))) return rc;
  if (n_rows == 0) return GNN_OK;
  if ((rc = check_table("x", x, d->dtype, x_stride, d->in_features)) ||
      (rc = check_table("y", y, d->dtype, y_stride, d->out_features)))
    return rc;
  if (y == x) return bad(GNN_E_INVALID_ARG, "y overlaps x");
  int n_cu = 0;
  const int none = devices_cu(&n_cu);
  GatedForward f(*d, n_rows, n_cu, x, x_stride, lies_aligned(x, x_stride), w,
                 weights_aligned(*d, *w));
  if ((rc = check_scratch(workspace, workspace_bytes, f.c.total))) return rc;
  if (none) return none;
  unsigned char *ws = (unsigned char *)workspace;
  const int t = d->dtype;
  const int64_t hp = up8(d->hidden);
  PackArgs pack;
  if (!f.few && !f.thin) f.x.fetch(ws, &pack);
  if (!f.few)
    for (Operand *o : {&f.gate, &f.up, &f.down}) o->fetch(ws, &pack);
  if ((rc = launched(launch_pack(pack, t, stream), "row copy"))) return rc;
  ProductArgs a;
  a.a[0] = f.x.p;
  a.lda = f.x.stride;
  a.b[0] = f.gate.p;
  a.b[1] = f.up.p;
  a.ldb = f.gate.stride;
  a.M = n_rows;
  a.N = d->hidden;
  a.K = d->in_features;
  a.bias[0] = w->gate_bias;
  a.bias[1] = w->up_bias;
  a.act = d->activation;
  if (f.thin) {
    a.b2 = f.down.p;
    a.ldb2 = f.down.stride;
    a.K2 = d->out_features;
    a.bias2 = w->down_bias;
    a.c = y;
    a.ldc = y_stride;
    return launched(launch_thin(a, false, t, stream), "gated block");
  }
  a.c = ws + f.h;
  a.ldc = n_rows <= TWO_ROWS ? 2 * hp : hp;
  a.lo = n_rows <= TWO_ROWS ? (int32_t)hp : 0;
  rc = launched(f.few ? launch_few(a, true, t, 1, stream)
                      : launch_product(a, PRODUCT_GATE, t, f.gate_tile, stream),
                "gate");
  if (rc) return rc;
  ProductArgs b;
  b.a[0] = ws + f.h;
  b.lda = a.ldc;
  b.lo = a.lo;
  b.b[0] = f.down.p;
  b.ldb = f.down.stride;
  b.M = n_rows;
  b.N = d->out_features;
  b.K = d->hidden;
  b.bias[0] = w->down_bias;
  b.c = y;
  b.ldc = y_stride;
  b.part = (float *)(ws + f.part);
  return launched(f.few ? launch_few(b, false, t, f.splits, stream)
                        : launch_product(b, PRODUCT_DOWN, t, f.down_tile, stream),
                  "down projection");
}

int gnn_gated_backward(const gnn_gated_dims *d, const gnn_gated_weights *w, const void *dy,
                       int64_t dy_stride, const void *x, int64_t x_stride, int64_t n_rows,
                       void *dx, int64_t dx_stride, const gnn_gated_weights *dw, void *workspace,
                       int64_t workspace_bytes, hipStream_t stream) {
  int rc = check_gated_dims(d);
  if (rc || (rc = check_gated_weights(w, "weights")) ||
      (rc = check_gated_weights(dw, "gradients")) || (rc = check_rows(n_rows)))
    return rc;
  if (n_rows > 0 && ((rc = check_table("dy", dy, d->dtype, dy_stride, d->out_features)) ||
                     (rc = check_table("x", x, d->dtype, x_stride, d->in_features)) ||
                     (rc = check_table("dx", dx, d->dtype, dx_stride, d->in_features))))
    return rc;
  if (n_rows > 0 && (dx == x || dx == dy))
    return bad(GNN_E_INVALID_ARG, "dx overlaps an input");
  for (const void *in : {w->gate, w->up, w->down})
    for (const void *out : {dw->gate, dw->up, dw->down})
      if (in == out) return bad(GNN_E_INVALID_ARG, "a gradient overlaps a weight");
  if (dw->gate == dw->up || dw->gate == dw->down || dw->up == dw->down)
    return bad(GNN_E_INVALID_ARG, "gradients overlap");
  int n_cu = 0;
  const int none = devices_cu(&n_cu);
  GatedBackward f(*d, n_rows, n_cu, x, x_stride, dy, dy_stride,
                  n_rows == 0 || (lies_aligned(x, x_stride) && lies_aligned(dy, dy_stride)), w,
                  weights_aligned(*d, *w));
  if ((rc = check_scratch(workspace, workspace_bytes, f.c.total))) return rc;
  if (none) return none;
  unsigned char *ws = (unsigned char *)workspace;
  const int t = d->dtype;
  const int64_t hp = up8(d->hidden);
  Operand *const tables[] = {&f.x, &f.dy, &f.gate, &f.up, &f.down};
  if (f.half) {
    SizeArgs z;
    for (int i = 0; i < SIZES; ++i) {
      const void *bias = i == 5 ? w->gate_bias : i == 6 ? w->up_bias : nullptr;
      const Operand *o = i < 5 ? tables[i] : nullptr;
      z.x[i] = o ? o->p : bias;
      z.y[i] = o && o->copy ? ws + o->at : nullptr;
      z.stride[i] = o ? o->stride : 1;
      z.rows[i] = o ? o->rows : bias ? d->hidden : 0;
      z.width[i] = o ? o->width : 1;
    }
    z.part = (float *)(ws + f.sizes);
    if ((rc = launched(launch_sizes(z, stream), "sizes"))) return rc;
    for (Operand *o : tables) o->fetch(ws, nullptr);
  } else {
    PackArgs pack;
    for (Operand *o : tables) o->fetch(ws, &pack);
    if ((rc = launched(launch_pack(pack, t, stream), "row copy"))) return rc;
  }
  void *h = ws + f.h, *g = ws + f.g;
  float *scales = f.half ? (float *)(ws + f.scales) : nullptr;
  if (n_rows > 0) {
    // g and u again, and dh; from them h, dg and du
    ProductArgs b;
    b.a[0] = f.x.p;
    b.a[1] = f.dy.p;
    b.lda = f.x.stride;
    b.lda2 = f.dy.stride;
    b.b2 = f.down.p;
    b.ldb2 = f.down.stride;
    b.K2 = d->out_features;
    b.b[0] = f.gate.p;
    b.b[1] = f.up.p;
    b.ldb = f.gate.stride;
    b.M = n_rows;
    b.N = d->hidden;
    b.K = d->in_features;
    b.bias[0] = w->gate_bias;
    b.bias[1] = w->up_bias;
    b.c = h;
    b.c2 = g;
    b.ldc = hp;
    b.sums = dw->gate_bias || dw->up_bias ? (float *)(ws + f.sums) : nullptr;
    b.act = d->activation;
    b.lo = f.two;
    b.sizes = f.half ? (const float *)(ws + f.sizes) : nullptr;
    b.scales = scales;
    if (f.thin) {
      b.c = dx;
      b.ldc = dx_stride;
      b.c2 = h;
      b.c3 = g;
      b.ldc2 = hp;
      rc = launched(launch_thin(b, true, t, stream), "gated block's gradients");
      if (rc) return rc;
    }
    if (!f.thin && (rc = launched(launch_product(b, PRODUCT_GRAD, t, f.grad.tile, stream), "gate gradient")))
      return rc;
    // dx = dg Wg + du Wu
    ProductArgs e;
    e.segs = f.two ? 4 : 2;
    for (int i = 0; i < e.segs; ++i) {
      e.a[i] = (unsigned char *)g + i * hp * 2;
      e.b[i] = i % 2 ? f.up.p : f.gate.p;
    }
    e.lda = e.segs * hp;
    e.ldb = f.gate.stride;
    e.M = n_rows;
    e.N = d->in_features;
    e.K = d->hidden;
    e.c = dx;
    e.ldc = dx_stride;
    e.scale = scales;
    if (!f.thin && (rc = launched(launch_product(e, PRODUCT_ROWS, t, f.dx.tile, stream), "gradient of x")))
      return rc;
  }
  // The weights' gradients: the rows are the k.
  auto weights = [&](const void *pa, const void *pa2, int64_t lda, int64_t m, const void *pb,
                     const void *pb2, int64_t ldb, int32_t n,
                     const ProductPlan &plan, void *c, void *c2, int64_t c_rows, int64_t valid,
                     bool sums, const float *scale, const char *what) {
    ProductArgs a;
    a.a[0] = pa;
    a.a[1] = pa2;
    a.lda = lda;
    a.b[0] = pb;
    a.b[1] = pb2;
    a.ldb = ldb;
    a.segs = f.two ? 2 : 1;
    a.M = m;
    a.N = n;
    a.K = (int32_t)n_rows;
    a.splits = plan.splits;
    a.split_steps = plan.splits > 1 ? plan.split_steps : INT32_MAX;
    a.c_rows = c_rows;
    a.c_valid = valid;
    a.c = c;
    a.c2 = c2;
    a.ldc = n;
    a.scale = scale;
    if (sums) a.sums = (float *)(ws + f.dy_sum);
    if (plan.splits == 1)
      return launched(launch_product(a, PRODUCT_WEIGHTS, t, plan.tile, stream), what);
    a.c = ws + f.part;
    a.ldc = up8(n);
    const int e = launched(launch_product(a, PRODUCT_WEIGHTS, t, plan.tile, stream), what);
    if (e) return e;
    JoinArgs j;
    j.part = (const float *)a.c;
    j.splits = plan.splits;
    j.M = m;
    j.ldp = a.ldc;
    j.N = n;
    j.c = c;
    j.c2 = c2;
    j.ldc = n;
    j.c_rows = c_rows;
    j.c_valid = valid;
    return launched(launch_join(j, t, stream), what);
  };
  const unsigned char *g2 = (unsigned char *)g + 2 * hp * 2, *h2 = (unsigned char *)h + hp * 2;
  const int64_t times = f.two ? 2 : 1;
  if ((rc = weights(g, g2, 2 * hp * times, 2 * hp, f.x.p, f.x.p, f.x.stride, d->in_features, f.dgu,
                    (void *)dw->gate, (void *)dw->up, hp, d->hidden, false,
                    scales, "gradients of gate and up")) ||
      (rc = weights(f.dy.p, f.dy.p, f.dy.stride, d->out_features, h, h2, hp * times, d->hidden,
                    f.dd, (void *)dw->down, (void *)dw->down, d->out_features, d->out_features,
                    dw->down_bias && f.dy_sums, scales ? scales + 1 : nullptr, "gradient of down")))
    return rc;
  SumArgs s;
  s.y_type = t;
  if (dw->gate_bias || dw->up_bias) {
    s.x = ws + f.sums;
    s.x_type = GNN_FP32;
    s.x_stride = s.width = (int32_t)(2 * hp);
    s.n = n_rows ? f.sum_rows : 0;
    s.y[0] = (void *)dw->gate_bias;
    s.y[1] = (void *)dw->up_bias;
    s.split = d->hidden;
    s.skip = (int32_t)hp;
    if ((rc = sum_columns(s, ws + f.colsum, "bias gradients", stream))) return rc;
  }
  if (dw->down_bias) {
    const bool there = f.dy_sums;  // dy itself otherwise
    s.x = there ? ws + f.dy_sum : dy;
    s.x_type = there ? GNN_FP32 : t;
    s.x_stride = there ? d->out_features : dy_stride;
    s.n = there ? f.dd.splits : n_rows;
    s.width = s.split = s.skip = d->out_features;
    s.y[0] = (void *)dw->down_bias;
    s.y[1] = nullptr;
    return sum_columns(s, ws + f.colsum, "bias gradients", stream);
  }
  return GNN_OK;
}

int gnn_debug_gated(const gnn_gated_dims *d, int32_t n_cu, int64_t n_rows, int32_t backward,
                    int32_t kernel[7]) {
  int rc = check_gated_dims(d);
  if (rc || (rc = check_rows(n_rows))) return rc;
  if (n_rows == 0 || n_cu < 1 || !kernel) return bad(GNN_E_INVALID_ARG, "bad arguments");
  for (int i = 0; i < 7; ++i) kernel[i] = 0;
  if (!backward) {
    const GatedForward f(*d, n_rows, n_cu, nullptr, 0, true, nullptr, true);
    kernel[0] = f.few ? 1 : f.thin ? 2 : 0;
    kernel[1] = f.few || f.thin ? -1 : f.gate_tile;
    kernel[2] = f.few ? f.splits : f.thin ? -1 : f.down_tile;
    return GNN_OK;
  }
  const GatedBackward f(*d, n_rows, n_cu, nullptr, 0, nullptr, 0, true, nullptr, true);
  kernel[0] = f.thin ? 2 : 0;
  kernel[1] = f.thin ? -1 : f.grad.tile;
  kernel[2] = f.thin ? -1 : f.dx.tile;
  kernel[3] = f.dgu.tile;
  kernel[4] = f.dgu.splits;
  kernel[5] = f.dd.tile;
  kernel[6] = f.dd.splits;
  return GNN_OK;
}

}  // extern "C"

// ------------------------------------------------------------- clipping ---

namespace {

int64_t clip_tiles(const gnn_grad &g) { return (g.count + CLIP_TILE - 1) / CLIP_TILE; }

int check_grads(const gnn_grad *g, int32_t n) {
  if (n < 0) return bad(GNN_E_INVALID_ARG, "negative tensor count");
  if (n > 0 && !g) return bad(GNN_E_INVALID_ARG, "grads is NULL");
  int64_t tiles = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (!float_type(g[i].type))
      return bad(GNN_E_INVALID_ARG, "tensor %d: type %d is not a float type", i, g[i].type);
    if (g[i].count < 0) return bad(GNN_E_INVALID_ARG, "tensor %d: negative count", i);
    if (g[i].count > (int64_t)1 << 40)
      return bad(GNN_E_UNSUPPORTED, "tensor %d: more than 2^40 elements", i);
    tiles += clip_tiles(g[i]);
    if (tiles > (int64_t)1 << 23)
      return bad(GNN_E_UNSUPPORTED, "more than 2^37 elements in all are not supported");
    if (g[i].count == 0) continue;
    const int rc = check_vector("gradient", g[i].grad, g[i].type);
    if (rc) return rc;
    const int ro = check_vector("output", g[i].out, g[i].type);
    if (ro) return ro;
  }
  return GNN_OK;
}

// Every output, the norm among them, has to lie apart from the others and from the
// gradients, but for its own where it takes its place.
int check_apart(const gnn_grad *g, int32_t n, const float *norm) {
  struct Span {
    uintptr_t lo, hi;
    bool out;
  };
  std::vector<Span> spans;
  spans.reserve(2 * (size_t)n + 1);
  spans.push_back({(uintptr_t)norm, (uintptr_t)(norm + 1), true});
  for (int32_t i = 0; i < n; ++i) {
    if (g[i].count == 0) continue;
    const uintptr_t bytes = (uintptr_t)g[i].count * type_bytes(g[i].type);
    spans.push_back({(uintptr_t)g[i].out, (uintptr_t)g[i].out + bytes, true});
    if (g[i].grad != g[i].out)
      spans.push_back({(uintptr_t)g[i].grad, (uintptr_t)g[i].grad + bytes, false});
  }
  std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.lo < b.lo; });
  uintptr_t any = 0, outs = 0;
  for (const Span &s : spans) {
    if (s.lo < (s.out ? any : outs))
      return bad(GNN_E_INVALID_ARG, "an output overlaps another tensor");
    any = std::max(any, s.hi);
    if (s.out) outs = std::max(outs, s.hi);
  }
  return GNN_OK;
}

}  // namespace

extern "C" {

size_t gnn_clip_workspace(const gnn_grad *grads, int32_t n_grads) {
  if (check_grads(grads, n_grads)) return 0;
  int64_t tiles = 0;
  for (int32_t i = 0; i < n_grads; ++i) tiles += clip_tiles(grads[i]);
  return 256 + up256((size_t)tiles * 8);
}

int gnn_clip_grads(const gnn_grad *grads, int32_t n_grads, float max_norm, float *norm,
                   void *workspace, int64_t workspace_bytes, hipStream_t stream) {
  int rc = check_grads(grads, n_grads);
  if (rc) return rc;
  if (!(max_norm > 0.f)) return bad(GNN_E_INVALID_ARG, "max_norm must be positive");
  if ((rc = check_vector("norm", norm, GNN_FP32))) return rc;
  if ((rc = check_scratch(workspace, workspace_bytes, gnn_clip_workspace(grads, n_grads))))
    return rc;
  try {
    if ((rc = check_apart(grads, n_grads, norm))) return rc;
    std::vector<ClipList> lists;
    for (int32_t i = 0; i < n_grads; ++i) {
      if (grads[i].count == 0) continue;
      if (lists.empty() || lists.back().count == CLIP_LIST) {
        lists.emplace_back();
        lists.back().count = 0;
        lists.back().tile[0] = 0;
      }
      ClipList &l = lists.back();
      const int at = l.count++;
      l.x[at] = grads[i].grad;
      l.y[at] = grads[i].out;
      l.n[at] = grads[i].count;
      l.type[at] = (uint8_t)grads[i].type;
      l.tile[at + 1] = l.tile[at] + (int32_t)clip_tiles(grads[i]);
    }
    float *scale = (float *)workspace;
    double *part = (double *)((unsigned char *)workspace + 256);
    int64_t tiles = 0;
    for (const ClipList &l : lists) {
      if ((rc = launched(launch_squares(l, part + tiles, stream), "sum of squares"))) return rc;
      tiles += l.tile[l.count];
    }
    if ((rc = launched(launch_norm_scale(part, tiles, max_norm, norm, scale, stream), "norm")))
      return rc;
    for (size_t i = lists.size(); i-- > 0;)
      if ((rc = launched(launch_scale(lists[i], scale, stream), "scaling"))) return rc;
  } catch (const std::bad_alloc &) {
    return bad(GNN_E_OOM, "host allocation failed");
  }
  return GNN_OK;
}

}  // extern "C"
