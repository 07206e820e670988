// Host side of the row operators: argument checks, weight layouts and the
// launches of gnn_quantize_rows, gnn_group_rows, gnn_linear_* and gnn_mlp_*.
// None of them allocates device memory after its handle is made or waits for
// the device: scratch comes from the caller, so that calls on different
// streams, and captured calls, share nothing but the weights.
#include <cstdarg>
#include <cstdio>
#include <new>
#include <vector>

#include "../../include/gnn.h"
#include "gnn_internal.h"

using namespace gnn;

namespace {

constexpr int MAX_WIDTH = 16384, MAX_HIDDEN = 4096, MAX_GROUPS = 4096;
constexpr int64_t MAX_ROWS = (int64_t)1 << 28;
constexpr int64_t MAX_STRIDE = (int64_t)1 << 31;

int bad(int code, const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return set_error(code, buf);
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

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

}  // namespace

struct gnn_linear {
  gnn_linear_dims dims;
  int device = 0, n_cu = 0;
  void *dev = nullptr;
  LinearArgs tmpl;  // weights and widths
};

struct gnn_mlp {
  gnn_mlp_dims dims;
  int device = 0;
  gnn_linear *layer[GNN_MLP_MAX_LAYERS] = {};
  float *norm[GNN_MLP_MAX_LAYERS] = {};  // gamma [G][H], then beta [G][H]
};

namespace {

int check_linear_dims(const gnn_linear_dims *d) {
  if (!d) return bad(GNN_E_INVALID_ARG, "dims is NULL");
  if (d->struct_size != sizeof(gnn_linear_dims))
    return bad(GNN_E_INVALID_ARG, "gnn_linear_dims.struct_size mismatch");
  if (d->in_features < 1 || d->out_features < 1)
    return bad(GNN_E_INVALID_ARG, "widths must be positive");
  if (d->in_features > MAX_WIDTH || d->out_features > MAX_WIDTH)
    return bad(GNN_E_UNSUPPORTED, "widths above %d are not supported", MAX_WIDTH);
  if (d->n_groups < 1) return bad(GNN_E_INVALID_ARG, "n_groups must be positive");
  if (d->n_groups > MAX_GROUPS)
    return bad(GNN_E_UNSUPPORTED, "more than %d groups are not supported", MAX_GROUPS);
  if (d->dtype == GNN_FP32) return bad(GNN_E_UNSUPPORTED, "weights are GNN_BF16, GNN_F16 or GNN_INT8");
  if (d->dtype != GNN_BF16 && d->dtype != GNN_F16 && d->dtype != GNN_INT8)
    return bad(GNN_E_INVALID_ARG, "dtype %d unknown", d->dtype);
  return GNN_OK;
}

LinearArgs linear_widths(const gnn_linear_dims &d) {
  LinearArgs a;
  a.K = d.in_features;
  a.N = d.out_features;
  a.G = d.n_groups;
  a.w_type = d.dtype;
  a.NB = (a.N + 31) / 32;
  a.S = linear_steps(a.K, a.w_type);
  return a;
}

// Scratch of a call: its rows in the form that the kernels take, and 8-bit
// rows' scales, where they do not take the caller's.
size_t linear_scratch(const gnn_linear *l, int x_type, int64_t n_rows) {
  if (n_rows == 0) return 0;
  LinearArgs a = l->tmpl;
  a.x_type = x_type;
  a.n = (int32_t)n_rows;
  if (!linear_plan(a, l->n_cu).convert) return 0;
  const bool round8 = l->dims.dtype == GNN_INT8 && x_type != GNN_INT8;
  return up256((size_t)n_rows * l->tmpl.S * 32) + (round8 ? up256((size_t)n_rows * 4) : 0);
}

// The launches of a layer; everything has been checked.
int run_linear(const gnn_linear *l, LinearArgs a, unsigned char *ws, hipStream_t stream) {
  const LinearPlan plan = linear_plan(a, l->n_cu);
  if (plan.convert) {
    hipError_t e;
    const int pad = a.S * 32 / type_bytes(a.w_type);
    if (a.w_type == GNN_INT8 && a.x_type != GNN_INT8) {
      QuantArgs q;
      q.x = a.x;
      q.x_type = a.x_type;
      q.x_stride = a.x_stride;
      q.n = a.n;
      q.K = a.K;
      q.q = (int8_t *)ws;
      q.q_stride = q.pad = pad;
      q.scales = (float *)(ws + up256((size_t)a.n * a.S * 32));
      a.xs = q.scales;
      e = launch_quantize(q, stream);
    } else {
      ConvertArgs c;
      c.x = a.x;
      c.x_type = a.x_type;
      c.y_type = a.w_type;
      c.x_stride = a.x_stride;
      c.n = a.n;
      c.K = a.K;
      c.pad = pad;
      c.y = ws;
      e = launch_convert(c, stream);
    }
    const int rc = launched(e, "row conversion");
    if (rc) return rc;
    a.x = ws;
    a.x_type = a.w_type;
    a.x_stride = pad;
  }
  return launched(launch_linear(a, plan, stream), "linear layer");
}

}  // namespace

extern "C" {

int gnn_quantize_rows(const void *x, int32_t x_type, int64_t x_stride, int64_t n_rows,
                      int32_t width, int8_t *q, int64_t q_stride, float *scales,
                      hipStream_t stream) {
  int rc = check_rows(n_rows);
  if (rc) return rc;
  if (width < 1) return bad(GNN_E_INVALID_ARG, "width must be positive");
  if (!float_type(x_type)) return bad(GNN_E_INVALID_ARG, "x_type %d is not a float type", x_type);
  if (n_rows == 0) return GNN_OK;
  if ((rc = check_table("x", x, x_type, x_stride, width))) return rc;
  if ((rc = check_table("q", q, GNN_INT8, q_stride, width))) return rc;
  if ((rc = check_table("scales", scales, GNN_FP32, 1, 1))) return rc;
  QuantArgs a;
  a.x = x;
  a.x_type = x_type;
  a.x_stride = x_stride;
  a.n = n_rows;
  a.K = width;
  a.q = q;
  a.q_stride = q_stride;
  a.scales = scales;
  return launched(launch_quantize(a, stream), "row rounding");
}

size_t gnn_group_workspace(int64_t n_rows, int32_t n_groups) {
  if (n_rows < 0 || n_rows > MAX_ROWS || n_groups < 1 || n_groups > MAX_GROUPS) return 0;
  return group_scratch_bytes(n_rows, n_groups);
}

int gnn_group_rows(const int32_t *ids, int64_t n_rows, int32_t n_groups, int32_t *offsets,
                   int32_t *order, void *workspace, int64_t workspace_bytes, hipStream_t stream) {
  int rc = check_rows(n_rows);
  if (rc) return rc;
  if (n_groups < 1) return bad(GNN_E_INVALID_ARG, "n_groups must be positive");
  if (n_groups > MAX_GROUPS)
    return bad(GNN_E_UNSUPPORTED, "more than %d groups are not supported", MAX_GROUPS);
  if ((rc = check_table("offsets", offsets, GNN_FP32, 1, 1))) return rc;
  if (n_rows == 0)
    return launched(launch_fill_i32(offsets, n_groups + 1, 0, stream), "row grouping");
  if ((rc = check_table("ids", ids, GNN_FP32, 1, 1))) return rc;
  if ((rc = check_table("order", order, GNN_FP32, 1, 1))) return rc;
  if ((rc = check_scratch(workspace, workspace_bytes, group_scratch_bytes(n_rows, n_groups))))
    return rc;
  GroupArgs a;
  a.ids = ids;
  a.n = n_rows;
  a.G = n_groups;
  a.offsets = offsets;
  a.order = order;
  a.counts = (int32_t *)workspace;
  return launched(launch_group(a, stream), "row grouping");
}

size_t gnn_linear_weight_count(const gnn_linear_dims *d) {
  if (check_linear_dims(d)) return 0;
  return (size_t)d->n_groups * ((size_t)d->in_features * d->out_features + d->out_features);
}

gnn_linear *gnn_linear_create(const float *weights, const gnn_linear_dims *dims) {
  if (check_linear_dims(dims)) return nullptr;
  if (!weights) {
    bad(GNN_E_INVALID_ARG, "weights is NULL");
    return nullptr;
  }
  int dev = 0;
  if (current_device(&dev)) return nullptr;
  gnn_linear *l = new (std::nothrow) gnn_linear();
  if (!l) {
    bad(GNN_E_OOM, "host allocation failed");
    return nullptr;
  }
  l->dims = *dims;
  l->device = dev;
  l->n_cu = cu_count(dev);
  LinearArgs &a = l->tmpl;
  a = linear_widths(*dims);
  const size_t fb = linear_frag_bytes(a.K, a.N, a.G, a.w_type);
  const size_t cb = up256((size_t)a.G * a.NB * 32 * 4);
  const size_t blob = gnn_linear_weight_count(dims) * 4;
  float *tmp = nullptr;
  hipError_t e = hipMalloc(&l->dev, up256(fb) + 2 * cb);
  if (e == hipSuccess) e = hipMalloc((void **)&tmp, blob);
  if (e == hipSuccess) e = hipMemcpy(tmp, weights, blob, hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    if (tmp) (void)hipFree(tmp);
    if (l->dev) (void)hipFree(l->dev);
    delete l;
    bad(GNN_E_OOM, "linear weight upload failed");
    return nullptr;
  }
  unsigned char *base = (unsigned char *)l->dev;
  a.w = base;
  a.ws = (const float *)(base + up256(fb));
  a.bias = (const float *)(base + up256(fb) + cb);
  e = launch_linear_layout(tmp, a, base, (float *)a.ws, (float *)a.bias, nullptr);
  if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
  (void)hipFree(tmp);
  if (e != hipSuccess) {
    launched(e, "weight layout");
    (void)hipFree(l->dev);
    delete l;
    return nullptr;
  }
  return l;
}

void gnn_linear_destroy(gnn_linear *l) {
  if (!l) return;
  {
    DeviceGuard guard(l->device);
    (void)hipDeviceSynchronize();
    (void)hipFree(l->dev);
  }
  delete l;
}

size_t gnn_linear_workspace(const gnn_linear *l, int32_t x_type, int64_t n_rows) {
  if (!l || n_rows < 0 || n_rows > MAX_ROWS) return 0;
  return linear_scratch(l, x_type, n_rows);
}

int gnn_linear_apply(gnn_linear *l, const void *x, int32_t x_type, int64_t x_stride,
                     const float *x_scales, int64_t n_rows, const int32_t *offsets,
                     const int32_t *order, void *y, int32_t y_type, int64_t y_stride,
                     void *workspace, int64_t workspace_bytes, hipStream_t stream) {
  if (!l) return bad(GNN_E_INVALID_ARG, "layer is NULL");
  int rc = check_rows(n_rows);
  if (rc) return rc;
  if (!float_type(x_type) && x_type != GNN_INT8)
    return bad(GNN_E_INVALID_ARG, "x_type %d unknown", x_type);
  if (!float_type(y_type)) return bad(GNN_E_INVALID_ARG, "y_type %d is not a float type", y_type);
  if (x_type == GNN_INT8 && l->dims.dtype != GNN_INT8)
    return bad(GNN_E_INVALID_ARG, "GNN_INT8 rows need a GNN_INT8 layer");
  if (n_rows == 0) return GNN_OK;
  if ((x_type == GNN_INT8) != (x_scales != nullptr))
    return bad(GNN_E_INVALID_ARG, "x_scales goes with GNN_INT8 rows, and only with them");
  if (!offsets && l->dims.n_groups > 1)
    return bad(GNN_E_INVALID_ARG, "offsets is NULL with %d groups", l->dims.n_groups);
  if ((rc = check_table("x", x, x_type, x_stride, l->dims.in_features))) return rc;
  if ((rc = check_table("y", y, y_type, y_stride, l->dims.out_features))) return rc;
  if ((uintptr_t)offsets % 4 || (uintptr_t)order % 4 || (uintptr_t)x_scales % 4)
    return bad(GNN_E_INVALID_ARG, "offsets, order or x_scales is not aligned to its elements");
  if ((rc = check_scratch(workspace, workspace_bytes, linear_scratch(l, x_type, n_rows))))
    return rc;
  DeviceGuard guard(l->device);
  LinearArgs a = l->tmpl;
  a.x = x;
  a.x_type = x_type;
  a.x_stride = x_stride;
  a.xs = x_scales;
  a.n = (int32_t)n_rows;
  a.off = offsets;
  a.order = a.y_order = order;
  a.y = y;
  a.y_type = y_type;
  a.y_stride = y_stride;
  return run_linear(l, a, (unsigned char *)workspace, stream);
}

int gnn_debug_linear(const gnn_linear_dims *dims, int32_t n_cu, int32_t x_type, int64_t n_rows,
                     int32_t grouped, int32_t y_type, int64_t y_stride, int32_t kernel[6]) {
  int rc = check_linear_dims(dims);
  if (rc || (rc = check_rows(n_rows))) return rc;
  if (n_rows == 0 || n_cu < 1 || !kernel || !float_type(y_type) ||
      (!float_type(x_type) && (x_type != GNN_INT8 || dims->dtype != GNN_INT8)))
    return bad(GNN_E_INVALID_ARG, "bad arguments");
  static const int32_t some = 0;
  LinearArgs a = linear_widths(*dims);
  a.x_type = x_type;
  a.n = (int32_t)n_rows;
  a.off = grouped ? &some : nullptr;  // whether there are offsets
  a.y_type = y_type;
  a.y_stride = y_stride;
  const LinearPlan p = linear_plan(a, n_cu);
  kernel[0] = p.convert;
  kernel[1] = p.tile;
  kernel[2] = p.RB;
  kernel[3] = p.NW;
  kernel[4] = p.multi ? 1 : p.narrow ? 2 : 0;
  kernel[5] = p.split;
  return GNN_OK;
}

}  // extern "C"

// ------------------------------------------------------------------ MLP ---

namespace {

int check_mlp_dims(const gnn_mlp_dims *d) {
  if (!d) return bad(GNN_E_INVALID_ARG, "dims is NULL");
  if (d->struct_size != sizeof(gnn_mlp_dims))
    return bad(GNN_E_INVALID_ARG, "gnn_mlp_dims.struct_size mismatch");
  if (d->n_layers < 1 || d->n_layers > GNN_MLP_MAX_LAYERS)
    return bad(GNN_E_INVALID_ARG, "n_layers %d outside 1..%d", d->n_layers, GNN_MLP_MAX_LAYERS);
  if (!(d->ln_eps > 0.f) || !(d->ln_eps < 1.f))
    return bad(GNN_E_INVALID_ARG, "ln_eps outside (0, 1)");
  for (int i = 0; i < d->n_layers; ++i) {
    const gnn_linear_dims l = {sizeof(gnn_linear_dims), d->widths[i], d->widths[i + 1],
                               d->n_groups, d->dtype};
    const int rc = check_linear_dims(&l);
    if (rc) return rc;
    if (i > 0 && d->widths[i] > MAX_HIDDEN)
      return bad(GNN_E_UNSUPPORTED, "hidden widths above %d are not supported", MAX_HIDDEN);
  }
  return GNN_OK;
}

// Floats of layer i's parameters for one group: W, b and, between layers,
// gamma and beta.
size_t mlp_layer_floats(const gnn_mlp_dims &d, int i) {
  const size_t in = d.widths[i], out = d.widths[i + 1];
  return in * out + out + (i + 1 < d.n_layers ? 2 * out : 0);
}

struct MlpScratch {
  size_t offsets = 0, order = 0, group = 0, pre = 0, act = 0, scales = 0, linear = 0, total = 0;
};

MlpScratch mlp_scratch(const gnn_mlp *m, int x_type, int64_t n) {
  const gnn_mlp_dims &d = m->dims;
  MlpScratch s;
  auto take = [&](size_t bytes) {
    const size_t at = s.total;
    s.total += up256(bytes);
    return at;
  };
  if (d.n_groups > 1) {
    s.offsets = take((size_t)(d.n_groups + 1) * 4);
    s.order = take((size_t)n * 4);
    s.group = take(group_scratch_bytes(n, d.n_groups));
  }
  size_t widest = 0;
  for (int i = 1; i < d.n_layers; ++i)
    if ((size_t)d.widths[i] > widest) widest = d.widths[i];
  s.pre = take((size_t)n * widest * 4);
  s.act = take((size_t)n * widest * (d.dtype == GNN_INT8 ? 1 : 2));
  s.scales = take(d.dtype == GNN_INT8 ? (size_t)n * 4 : 0);
  size_t linear = 0;  // the layers take turns
  for (int i = 0; i < d.n_layers; ++i) {
    const size_t b = linear_scratch(m->layer[i], i == 0 ? x_type : d.dtype, n);
    if (b > linear) linear = b;
  }
  s.linear = take(linear);
  return s;
}

}  // namespace

extern "C" {

size_t gnn_mlp_weight_count(const gnn_mlp_dims *d) {
  if (check_mlp_dims(d)) return 0;
  size_t n = 0;
  for (int i = 0; i < d->n_layers; ++i) n += mlp_layer_floats(*d, i);
  return n * d->n_groups;
}

void gnn_mlp_destroy(gnn_mlp *m) {
  if (!m) return;
  {
    DeviceGuard guard(m->device);
    (void)hipDeviceSynchronize();
    for (int i = 0; i < GNN_MLP_MAX_LAYERS; ++i) {
      gnn_linear_destroy(m->layer[i]);
      if (m->norm[i]) (void)hipFree(m->norm[i]);
    }
  }
  delete m;
}

gnn_mlp *gnn_mlp_create(const float *weights, const gnn_mlp_dims *dims) {
  if (check_mlp_dims(dims)) return nullptr;
  if (!weights) {
    bad(GNN_E_INVALID_ARG, "weights is NULL");
    return nullptr;
  }
  int dev = 0;
  if (current_device(&dev)) return nullptr;
  gnn_mlp *m = new (std::nothrow) gnn_mlp();
  if (!m) {
    bad(GNN_E_OOM, "host allocation failed");
    return nullptr;
  }
  m->dims = *dims;
  m->device = dev;
  const int G = dims->n_groups;
  try {
    const float *p = weights;
    for (int i = 0; i < dims->n_layers; ++i) {
      const size_t in = dims->widths[i], out = dims->widths[i + 1], wb = in * out + out;
      const bool hidden = i + 1 < dims->n_layers;
      std::vector<float> lin(G * wb), ln(hidden ? 2 * G * out : 0);
      for (int g = 0; g < G; ++g) {
        std::copy(p, p + wb, lin.begin() + g * wb);
        p += wb;
        if (!hidden) continue;
        std::copy(p, p + out, ln.begin() + g * out);
        std::copy(p + out, p + 2 * out, ln.begin() + (G + g) * out);
        p += 2 * out;
      }
      const gnn_linear_dims l = {sizeof(gnn_linear_dims), (int32_t)in, (int32_t)out, G,
                                 dims->dtype};
      m->layer[i] = gnn_linear_create(lin.data(), &l);
      bool ok = m->layer[i] != nullptr;
      if (ok && hidden &&
          (hipMalloc((void **)&m->norm[i], ln.size() * 4) != hipSuccess ||
           hipMemcpy(m->norm[i], ln.data(), ln.size() * 4, hipMemcpyHostToDevice) != hipSuccess)) {
        (void)hipGetLastError();
        bad(GNN_E_OOM, "MLP weight upload failed");
        ok = false;
      }
      if (!ok) {
        gnn_mlp_destroy(m);
        return nullptr;
      }
    }
  } catch (const std::bad_alloc &) {
    gnn_mlp_destroy(m);
    bad(GNN_E_OOM, "host allocation failed");
    return nullptr;
  }
  return m;
}

size_t gnn_mlp_workspace(const gnn_mlp *m, int32_t x_type, int64_t n_rows) {
  if (!m || n_rows < 0 || n_rows > MAX_ROWS) return 0;
  return mlp_scratch(m, x_type, n_rows).total;
}

int gnn_mlp_apply(gnn_mlp *m, const void *x, int32_t x_type, int64_t x_stride,
                  const int32_t *group_ids, int64_t n_rows, void *y, int32_t y_type,
                  int64_t y_stride, void *workspace, int64_t workspace_bytes,
                  hipStream_t stream) {
  if (!m) return bad(GNN_E_INVALID_ARG, "mlp is NULL");
  const gnn_mlp_dims &d = m->dims;
  int rc = check_rows(n_rows);
  if (rc) return rc;
  if (!float_type(x_type)) return bad(GNN_E_INVALID_ARG, "x_type %d is not a float type", x_type);
  if (!float_type(y_type)) return bad(GNN_E_INVALID_ARG, "y_type %d is not a float type", y_type);
  if (n_rows == 0) return GNN_OK;
  if ((d.n_groups > 1) != (group_ids != nullptr))
    return bad(GNN_E_INVALID_ARG, "group_ids goes with several groups, and only with them");
  if ((rc = check_table("x", x, x_type, x_stride, d.widths[0]))) return rc;
  if ((rc = check_table("y", y, y_type, y_stride, d.widths[d.n_layers]))) return rc;
  const MlpScratch s = mlp_scratch(m, x_type, n_rows);
  if ((rc = check_scratch(workspace, workspace_bytes, s.total))) return rc;
  DeviceGuard guard(m->device);
  unsigned char *ws = (unsigned char *)workspace;
  const int32_t *offsets = nullptr, *order = nullptr;
  if (d.n_groups > 1) {
    rc = gnn_group_rows(group_ids, n_rows, d.n_groups, (int32_t *)(ws + s.offsets),
                        (int32_t *)(ws + s.order), ws + s.group, (int64_t)(s.pre - s.group),
                        stream);
    if (rc) return rc;
    offsets = (const int32_t *)(ws + s.offsets);
    order = (const int32_t *)(ws + s.order);
  }
  // Hidden rows lie in group order; the first layer reads, and the last one
  // writes, rows where the caller has them.
  for (int i = 0; i < d.n_layers; ++i) {
    const bool first = i == 0, last = i + 1 == d.n_layers;
    LinearArgs a = m->layer[i]->tmpl;
    a.n = (int32_t)n_rows;
    a.off = offsets;
    a.order = first ? order : nullptr;
    a.y_order = last ? order : nullptr;
    a.x = first ? x : ws + s.act;
    a.x_type = first ? x_type : d.dtype;
    a.x_stride = first ? x_stride : d.widths[i];
    a.xs = !first && d.dtype == GNN_INT8 ? (const float *)(ws + s.scales) : nullptr;
    a.y = last ? y : ws + s.pre;
    a.y_type = last ? y_type : GNN_FP32;
    a.y_stride = last ? y_stride : d.widths[i + 1];
    if ((rc = run_linear(m->layer[i], a, ws + s.linear, stream))) return rc;
    if (last) break;
    NormArgs b;
    b.x = (const float *)(ws + s.pre);
    b.n = n_rows;
    b.H = d.widths[i + 1];
    b.G = d.n_groups;
    b.gamma = m->norm[i];
    b.beta = m->norm[i] + (size_t)d.n_groups * b.H;
    b.ids = group_ids;
    b.order = order;
    b.n_in = offsets ? offsets + d.n_groups : nullptr;
    b.eps = d.ln_eps;
    b.y = ws + s.act;
    b.y_type = d.dtype;
    b.scales = (float *)(ws + s.scales);
    if ((rc = launched(launch_norm(b, stream), "LayerNorm"))) return rc;
  }
  return GNN_OK;
}

}  // extern "C"
