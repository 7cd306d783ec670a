// C ABI of the layer operators (declared in include/pointid.h): argument checks, the
// choice of kernels, scratch, launch sequencing.  Every call only enqueues work.
#include "layers.h"

#include "layers_call.h"

using namespace pointid;

namespace {

constexpr int64_t kMaxSide = int64_t(1) << 20;         // k and n
constexpr int64_t kMaxPitch = int64_t(1) << 21;        // of an operand that the products read in place

// dz of up to this many values is kept in two 16-bit parts.  Rounded once, it makes the error of
// a 16-bit gradient 1.4 times that of its results' own rounding, whatever the size; the second
// part takes twice the multiplications.  Small calls spend their time on launches and on the
// weights' bytes: with one part and two, silu, bf16, 2048 x 2048 20.5 us and 20.7 up to 32 rows,
// a gated 512 x 512 23.6 and 23.9, a gated 2048 x 2048 23.4 and 23.8, dense 512 x 512 15.3
// and 20.8 (the pair's plan splits and joins), 4096 x 12288 48 and 63 for one row.  Past the
// limit it would cost more: 256 x 2048 x 2048 23.2 and 27.9, gated 29.4 and 40.0, 512 rows of
// 4096 x 12288 147 and 220.
constexpr int64_t kTwoPartValues = int64_t(1) << 16;

// ---- argument checks

int check_call(pointid_layers l, int dtype, int act, int64_t m, int64_t k, int64_t n) {
  if (!l) return set_error(POINTID_EINVAL, "layers is NULL");
  if (dtype != POINTID_FP32 && dtype != POINTID_BF16 && dtype != POINTID_FP16)
    return set_error(POINTID_EUNSUPPORTED, "dtype must be POINTID_FP32, POINTID_BF16 or POINTID_FP16");
  if (act < POINTID_ACT_NONE || act > POINTID_ACT_SIGMOID) return set_error(POINTID_EINVAL, "act is no activation");
  if (m < 0 || m > kMaxRows) return set_error(POINTID_EINVAL, "m must be in [0, 2^28]");
  if (k < 1 || k > kMaxSide || n < 1 || n > kMaxSide)
    return set_error(POINTID_EINVAL, "k and n must be in [1, 2^20]");
  return POINTID_OK;
}

int check_packed(const pointid_checkpoint& c, const char* name) {
  if (!c.codes || !c.exponents) return set_error(POINTID_EINVAL, std::string(name) + ": codes or exponents is NULL");
  return POINTID_OK;
}

int check_kept(const pointid_kept* a, const char* name, int dtype, int64_t rows, int64_t cols, bool may_miss) {
  if (!a) {
    if (may_miss || rows == 0) return POINTID_OK;
    return set_error(POINTID_EINVAL, std::string(name) + " is NULL");
  }
  if (a->full.data) {
    if (a->packed.codes || a->packed.exponents)
      return set_error(POINTID_EINVAL, std::string(name) + " is both a matrix and a checkpoint");
    return check_matrix(&a->full, name, dtype, rows, cols);
  }
  if (rows == 0) return POINTID_OK;
  return check_packed(a->packed, name);
}

Kept kept_of(const pointid_kept* a, int64_t rows, int64_t cols) {
  Kept k;
  std::memset(&k, 0, sizeof(k));
  if (!a) return k;
  const pointid_matrix f = matrix_of(&a->full, rows, cols);
  k.matrix = f.data;
  k.ld = f.ld;
  if (!k.matrix) k.packed = {a->packed.codes, a->packed.exponents};
  return k;
}

// A matrix as the products read it: 16-bit planes with aligned rows, zero past the columns
// up to a whole piece of 8, or fp32 values.
struct Planes {
  const void* base = nullptr;
  int64_t ld = 0, plane = 0;       // elements
  int parts = 1;
  const void* at(int part) const { return static_cast<const uint16_t*>(base) + part * plane; }
};

bool read_in_place(const void* p, int64_t ld, int dtype, int64_t cols) {
  return ld <= kMaxPitch && (dtype == POINTID_FP32 || (cols % 8 == 0 && ld % 8 == 0 && aligned16(p)));
}

// An operand, and whether it is read in place or made by a pass into scratch.
struct Source {
  Kept from;                       // a matrix, or a checkpoint
  int dtype;
  int64_t rows, cols;
  bool in_place = false;
  void* made = nullptr;
  Planes planes;

  void plan(const Kept& k, int type, int64_t r, int64_t c, Call& call, bool copy = false) {
    from = k, dtype = type, rows = r, cols = c;
    in_place = !copy && k.matrix && read_in_place(k.matrix, k.ld, type, c);
    planes.base = k.matrix;
    planes.ld = k.ld;
    if (in_place) return;
    planes.ld = round_up(c, 8);
    call.want(&made, (size_t)size_of(dtype) * r * planes.ld);
  }
  // The operand as it will stand, and the job that makes it so.
  void make(FillJobs* jobs) {
    if (in_place) return;
    planes.base = made;
    FillJob& j = jobs->job[jobs->count++];
    j.kind = from.matrix ? FillJob::kCopy : FillJob::kLoad;
    j.dtype = dtype;
    j.src = from.matrix, j.ld_src = from.ld;
    j.packed = from.packed;
    j.rows = rows, j.cols = cols;
    j.out = made, j.ld = planes.ld;
  }
};

int run_fill(Call& call, const FillJobs& jobs) {
  if (jobs.count == 0) return POINTID_OK;
  return call.run("layers_fill", false, [&] { return launch_layers_fill(jobs, call.stream()); });
}

// The weights of one or both halves: these share a pitch, so that where one is copied, so
// is the other.
void plan_weights(Source* s, const pointid_matrix* w, int halves, int dtype, int64_t k, int64_t n, Call& call) {
  bool copy = false;
  for (int h = 0; h < halves; ++h)
    copy = copy || !read_in_place(w[h].data, w[h].ld, dtype, n) || w[h].ld != w[0].ld;
  for (int h = 0; h < halves; ++h) {
    Kept from;
    std::memset(&from, 0, sizeof(from));
    from.matrix = w[h].data, from.ld = w[h].ld;
    s[h].plan(from, dtype, k, n, call, copy);
  }
}

// The products of the parts of an operand with the other's one, the remainder's first.
int add_terms(ProductArgs* a, const Planes& left, const Planes& right0, const Planes* right1) {
  const int parts = left.parts > right0.parts ? left.parts : right0.parts;
  for (int p = parts - 1; p >= 0; --p) {
    if (a->terms == kMaxTerms) return set_error(POINTID_EHIP, "too many terms");
    const int i = left.parts > 1 ? p : 0, j = right0.parts > 1 ? p : 0;
    a->term[a->terms++] = {left.at(i), right0.at(j), right1 ? right1->at(j) : nullptr};
  }
  return POINTID_OK;
}

size_t part_bytes(int splits, const End& e) {
  return splits > 1 ? sizeof(float) * (size_t)splits * e.halves * e.rows * e.part_ld : 0;
}

// A product and, where its sum is split, the join.
int run_product(Call& call, Form form, const ProductPlan& plan, ProductArgs& a, int dtype, float* part, bool last) {
  const End end = a.end;
  if (plan.splits > 1) {
    a.end.mode = kEndPartial;
    a.end.part = part;
  }
  int rc = call.run("layers_product", last && plan.splits == 1, [&] {
    return dtype == POINTID_FP32   ? launch_product_f32(form, plan, a, call.stream())
           : dtype == POINTID_FP16 ? launch_product_fp16(form, plan, a, call.stream())
                                   : launch_product_bf16(form, plan, a, call.stream());
  });
  if (rc != POINTID_OK || plan.splits == 1) return rc;
  return call.run("layers_join", last,
                  [&] { return launch_layers_join(end, part, end.part_ld, plan.splits, call.stream()); });
}

// Both products of a gradient in one launch, and the joins.
int run_pair(Call& call, const ProductPlan& dx_plan, const ProductPlan& dw_plan, ProductArgs& dx, ProductArgs& dw,
             const SumsJobs& sums, int dtype, float* dx_part, float* dw_part) {
  const End dx_end = dx.end, dw_end = dw.end;
  auto split = [](ProductArgs& a, const ProductPlan& plan, float* part) {
    a.splits = plan.splits;
    if (plan.splits == 1) return;
    a.end.mode = kEndPartial;
    a.end.part = part;
  };
  split(dx, dx_plan, dx_part);
  split(dw, dw_plan, dw_part);
  int rc = call.run("layers_product", dx_plan.splits == 1 && dw_plan.splits == 1, [&] {
    return dtype == POINTID_FP32   ? launch_pair_f32(dx_plan.tile, dx, dw, sums, call.stream())
           : dtype == POINTID_FP16 ? launch_pair_fp16(dx_plan.tile, dx, dw, sums, call.stream())
                                   : launch_pair_bf16(dx_plan.tile, dx, dw, sums, call.stream());
  });
  if (rc == POINTID_OK && dx_plan.splits > 1)
    rc = call.run("layers_join", dw_plan.splits == 1, [&] {
      return launch_layers_join(dx_end, dx_part, dx_end.part_ld, dx_plan.splits, call.stream());
    });
  if (rc == POINTID_OK && dw_plan.splits > 1)
    rc = call.run("layers_join", true, [&] {
      return launch_layers_join(dw_end, dw_part, dw_end.part_ld, dw_plan.splits, call.stream());
    });
  return rc;
}

End end_of(int mode, int act, int dtype, int halves, int64_t rows, int64_t cols, const pointid_matrix& y0,
           const pointid_matrix& y1) {
  End e;
  std::memset(&e, 0, sizeof(e));
  e.mode = mode;
  e.act = act;
  e.dtype = dtype;
  e.halves = halves;
  e.rows = rows;
  e.cols = cols;
  e.part_ld = round_up(cols, 32);
  e.y0 = y0.data, e.ld0 = y0.ld;
  e.y1 = y1.data, e.ld1 = y1.ld;
  return e;
}

// ---- the forward pass of a dense (halves == 1) or gated layer

struct Forward {
  int dtype, act, halves;
  int64_t m, k, n;
  pointid_matrix x, w[2];
  const float* bias[2];
  pointid_matrix residual, y;
  Kept keep[2];
};

// Whether the weights are streamed past the rows.  fp32: up to 8 rows (8192 x 8192, 8 rows:
// 63 us, on the matrix cores 70).  16 bits: on the matrix cores from 2 rows on, and for one
// row of up to 2^27 weights, of a gated layer 2^26.  Streamed against those, bf16, weights
// out of memory: 4096 x 4096 15.7 us against 14.0, 8192 x 8192 34.2 against 33.2, 8192 x 9216
// 37.2 against 34.9, 16384 x 8192 57.0 against 55.3, 12288 x 12288 61.2 against 61.8,
// 16384 x 16384 97.0 against 100.5; gated 4096 x 4096 24.2 against 22.7, 4096 x 8192 34.6
// against 35.6, 12288 x 4096 47.6 against 46.8, 4096 x 12288 46.2 against 51.8, 12288 x
// 12288 114 against 137 (fp16 alike).  But streamed up to 8 rows where they would take a copy
// of the weights first.  A lane reads 16 bytes of a row, so a row has to have them.
bool few_rows(const Forward& f) {
  if (f.m > kFewRows || f.n < (f.dtype == POINTID_FP32 ? 4 : 8)) return false;
  for (int h = 0; h < f.halves; ++h)
    if (f.w[h].ld > kMaxPitch) return false;           // past its 32-bit steps
  if (f.dtype == POINTID_FP32 || (f.m == 1 && f.k * f.n > int64_t(1) << (f.halves == 2 ? 25 : 27))) return true;
  for (int h = 0; h < f.halves; ++h)
    if (!read_in_place(f.w[h].data, f.w[h].ld, f.dtype, f.n) || f.w[h].ld != f.w[0].ld) return true;
  return false;
}

int run_forward(pointid_layers l, const Forward& f, hipStream_t stream) {
  DeviceScope dev(l->device);
  if (dev.error() != hipSuccess) return hip_fail(dev.error(), "hipSetDevice");
  Call call(l, stream);
  const pointid_matrix none = {nullptr, 0};
  End e = end_of(f.halves == 2 ? kEndGated : kEndDense, f.act, f.dtype, f.halves, f.m, f.n, f.y, none);
  e.bias0 = f.bias[0];
  e.bias1 = f.bias[1];
  e.residual = f.residual.data;
  e.ld_residual = f.residual.ld;
  e.keep0 = f.keep[0];
  e.keep1 = f.keep[1];
  const Strided x = {f.x.data, f.x.ld, 1, f.dtype};
  Strided w[2];
  for (int h = 0; h < 2; ++h) w[h] = {f.w[h].data, 1, f.w[h].ld, f.dtype};

  if (few_rows(f)) {
    const int splits = few_rows_splits(f.k, f.n, f.halves, l->cus);
    float* part = nullptr;
    call.want(&part, part_bytes(splits, e));
    int rc = call.reserve();
    if (rc != POINTID_OK) return rc;
    End rows_end = e;
    if (splits > 1) {
      rows_end.mode = kEndPartial;
      rows_end.part = part;
    }
    rc = call.run("layers_rows", splits == 1,
                  [&] { return launch_layers_rows(x, w, f.k, rows_end, splits, stream); });
    if (rc != POINTID_OK || splits == 1) return rc;
    return call.run("layers_join", true, [&] { return launch_layers_join(e, part, e.part_ld, splits, stream); });
  }
  Source sx, sw[2];
  Kept from;
  std::memset(&from, 0, sizeof(from));
  from.matrix = f.x.data, from.ld = f.x.ld;
  sx.plan(from, f.dtype, f.m, f.k, call);
  plan_weights(sw, f.w, f.halves, f.dtype, f.k, f.n, call);
  const ProductPlan plan = plan_product(f.dtype == POINTID_FP32, f.m, f.n, f.halves, f.k, 1, l->cus);
  float* part = nullptr;
  call.want(&part, part_bytes(plan.splits, e));
  int rc = call.reserve();
  if (rc != POINTID_OK) return rc;
  FillJobs jobs;
  std::memset(&jobs, 0, sizeof(jobs));
  sx.make(&jobs);
  for (int h = 0; h < f.halves; ++h) sw[h].make(&jobs);
  rc = run_fill(call, jobs);
  if (rc != POINTID_OK) return rc;
  ProductArgs a;
  std::memset(&a, 0, sizeof(a));
  rc = add_terms(&a, sx.planes, sw[0].planes, f.halves == 2 ? &sw[1].planes : nullptr);
  if (rc != POINTID_OK) return rc;
  a.inner = (int32_t)f.k;
  a.ld_left = sx.planes.ld;
  a.ld_right = sw[0].planes.ld;
  a.end = e;
  return run_product(call, kForward, plan, a, f.dtype, part, true);
}

// ---- the backward pass of a dense (halves == 1) or gated layer

struct Backward {
  int dtype, act, halves;
  int64_t m, k, n;
  pointid_matrix dy;
  Kept x, z[2];
  pointid_matrix w[2], dx, dw[2];
  float* db[2];
};

int run_backward(pointid_layers l, const Backward& b, hipStream_t stream) {
  DeviceScope dev(l->device);
  if (dev.error() != hipSuccess) return hip_fail(dev.error(), "hipSetDevice");
  Call call(l, stream);
  const bool want_dx = b.dx.data, want_dw = b.dw[0].data, want_db = b.db[0] || b.db[1];
  if (!want_dx && !want_dw && !want_db) return POINTID_OK;
  const pointid_matrix none = {nullptr, 0};
  if (b.m == 0) {
    int rc = POINTID_OK;
    for (int h = 0; h < b.halves && rc == POINTID_OK; ++h) {
      if (want_dw)
        rc = call.run("layers_zero", false,
                      [&] { return launch_layers_zero(b.dw[h].data, b.dw[h].ld, b.dtype, b.k, b.n, stream); });
      if (rc == POINTID_OK && b.db[h])
        rc = call.run("layers_zero", false,
                      [&] { return launch_layers_zero(b.db[h], b.n, POINTID_FP32, 1, b.n, stream); });
    }
    return rc;
  }
  const bool products = want_dx || want_dw;
  // dz is dy itself where no activation changes it and the products can read it
  const bool plain = b.halves == 1 && b.act == POINTID_ACT_NONE;
  const bool read_dy = plain && read_in_place(b.dy.data, b.dy.ld, b.dtype, b.n);
  const bool exact16 = b.halves == 1 && (b.act == POINTID_ACT_NONE || b.act == POINTID_ACT_RELU);

  GradArgs g;
  std::memset(&g, 0, sizeof(g));
  g.dy = b.dy.data;
  g.ld_dy = b.dy.ld;
  g.dtype = b.dtype;
  g.act = b.act;
  g.halves = b.halves;
  g.rows = b.m;
  g.cols = b.n;
  for (int h = 0; h < b.halves; ++h) g.z[h] = b.z[h];
  g.parts = !products || read_dy                      ? 0
            : b.dtype == POINTID_FP32                 ? -1
            : !exact16 && b.m * b.n <= kTwoPartValues ? 2
                                                      : 1;
  g.ld = round_up(b.n, 8);
  g.plane = b.m * g.ld;
  const size_t dz_bytes = g.parts < 0 ? 4 * (size_t)g.plane : 2 * (size_t)g.plane * g.parts;
  for (int h = 0; h < b.halves && g.parts != 0; ++h) call.want(&g.out[h], dz_bytes);
  const int block_rows = grad_rows(b.m, b.n, l->cus);
  const int64_t grad_blocks = (b.m + block_rows - 1) / block_rows;
  if (want_db) call.want(&g.col_part, sizeof(float) * (size_t)(grad_blocks * b.halves * b.n));
  // what is not dy itself can leave fp16's range
  const bool scaled = b.dtype == POINTID_FP16 && products && !exact16;
  if (scaled) {
    g.maxima_count = grad_max_blocks(b.m, b.n);
    call.want(&g.maxima, sizeof(uint32_t) * g.maxima_count);
    call.want(&g.unscale, sizeof(float));
  }

  // x for dW, the weights for dx
  Source sx, sw[2];
  if (want_dw) sx.plan(b.x, b.dtype, b.m, b.k, call);
  if (want_dx) plan_weights(sw, b.w, b.halves, b.dtype, b.k, b.n, call);
  End dx_end = end_of(kEndStore, POINTID_ACT_NONE, b.dtype, 1, b.m, b.k, b.dx, none);
  End dw_end = end_of(kEndStore, POINTID_ACT_NONE, b.dtype, b.halves, b.k, b.n, b.dw[0], b.dw[1]);
  Planes dz[2];
  for (int h = 0; h < 2; ++h) {
    dz[h].ld = read_dy ? b.dy.ld : g.ld;
    dz[h].plane = g.plane;
    dz[h].parts = read_dy || g.parts < 1 ? 1 : g.parts;
  }
  ProductPlan dx_plan = {0, 1}, dw_plan = {0, 1};
  const bool f32 = b.dtype == POINTID_FP32;
  bool pair = false;
  if (want_dx && want_dw) {
    const PairPlan plan = plan_pair(f32, b.m, b.k, b.n, b.halves, dz[0].parts, l->cus);
    pair = plan.tile >= 0;
    dx_plan = {plan.tile, plan.dx_splits};
    dw_plan = {plan.tile, plan.dw_splits};
  }
  if (want_dx && !pair) dx_plan = plan_product(f32, b.m, b.k, 1, b.n, b.halves * dz[0].parts, l->cus);
  if (want_dw && !pair) dw_plan = plan_product(f32, b.k, b.n, b.halves, b.m, dz[0].parts, l->cus);
  float *part = nullptr, *dw_part = nullptr;
  const size_t dx_bytes = part_bytes(dx_plan.splits, dx_end), dw_bytes = part_bytes(dw_plan.splits, dw_end);
  if (pair) {
    call.want(&part, dx_bytes);
    call.want(&dw_part, dw_bytes);
  } else {
    call.want(&part, dx_bytes > dw_bytes ? dx_bytes : dw_bytes);       // one after the other
  }
  int rc = call.reserve();
  if (rc != POINTID_OK) return rc;

  FillJobs jobs;
  std::memset(&jobs, 0, sizeof(jobs));
  for (int h = 0; h < b.halves && want_dx; ++h) sw[h].make(&jobs);
  if (want_dw) sx.make(&jobs);
  if (scaled) {
    rc = call.run("layers_grad_max", false, [&] { return launch_layers_grad_max(g, stream); });
    if (rc != POINTID_OK) return rc;
    dx_end.unscale = dw_end.unscale = g.unscale;
  }
  if (g.parts != 0 || want_db)
    rc = call.run("layers_grad", false, [&] { return launch_layers_grad(g, block_rows, jobs, stream); });
  else
    rc = run_fill(call, jobs);
  if (rc != POINTID_OK) return rc;
  SumsJobs sums;
  std::memset(&sums, 0, sizeof(sums));
  if (want_db) {
    sums = {g.col_part, grad_blocks, b.n, b.halves, {b.db[0], b.db[1]}};
    if (!pair) {
      rc = call.run("layers_sums", !products, [&] { return launch_layers_sums(sums, stream); });
      if (rc != POINTID_OK) return rc;
    }
  }
  for (int h = 0; h < 2; ++h) dz[h].base = read_dy ? b.dy.data : g.out[h];

  if (!pair) dw_part = part;
  ProductArgs dx, dw;
  std::memset(&dx, 0, sizeof(dx));
  std::memset(&dw, 0, sizeof(dw));
  if (want_dx) {
    for (int h = 0; h < b.halves && rc == POINTID_OK; ++h) rc = add_terms(&dx, dz[h], sw[h].planes, nullptr);
    if (rc != POINTID_OK) return rc;
    dx.inner = (int32_t)b.n;
    dx.ld_left = dz[0].ld;
    dx.ld_right = sw[0].planes.ld;
    dx.end = dx_end;
  }
  if (want_dw) {
    rc = add_terms(&dw, sx.planes, dz[0], b.halves == 2 ? &dz[1] : nullptr);
    if (rc != POINTID_OK) return rc;
    dw.inner = (int32_t)b.m;
    dw.ld_left = sx.planes.ld;
    dw.ld_right = dz[0].ld;
    dw.end = dw_end;
  }
  if (pair) return run_pair(call, dx_plan, dw_plan, dx, dw, sums, b.dtype, part, dw_part);
  if (want_dx) {
    rc = run_product(call, kDx, dx_plan, dx, b.dtype, part, !want_dw);
    if (rc != POINTID_OK) return rc;
  }
  return want_dw ? run_product(call, kDw, dw_plan, dw, b.dtype, dw_part, true) : POINTID_OK;
}

int check_checkpoint_call(int dtype, int64_t rows, int64_t cols, const pointid_matrix* a, const pointid_checkpoint* c) {
  if (dtype != POINTID_FP32 && dtype != POINTID_BF16 && dtype != POINTID_FP16)
    return set_error(POINTID_EUNSUPPORTED, "dtype must be POINTID_FP32, POINTID_BF16 or POINTID_FP16");
  if (rows < 0 || rows > INT32_MAX) return set_error(POINTID_EINVAL, "rows must be in [0, 2^31)");
  if (cols < 1 || cols > kMaxSide) return set_error(POINTID_EINVAL, "cols must be in [1, 2^20]");
  if (rows == 0) return POINTID_OK;
  const int rc = check_matrix(a, "the matrix", dtype, rows, cols);
  if (rc != POINTID_OK) return rc;
  if (!c) return set_error(POINTID_EINVAL, "the checkpoint is NULL");
  return check_packed(*c, "the checkpoint");
}

}  // namespace

extern "C" {

int pointid_layers_create(int device, pointid_layers* out) {
  if (!out) return set_error(POINTID_EINVAL, "out is NULL");
  *out = nullptr;
  return guarded([&] {
    int count = 0;
    if (hipGetDeviceCount(&count) != hipSuccess || count <= 0) return set_error(POINTID_ENODEV, "no HIP device visible");
    if (device < 0 || device >= count) return set_error(POINTID_ENODEV, "device ordinal out of range");
    hipDeviceProp_t prop;
    hipError_t e = hipGetDeviceProperties(&prop, device);
    if (e != hipSuccess) return hip_fail(e, "hipGetDeviceProperties");
    if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0)
      return set_error(POINTID_ENODEV,
                       std::string("device is ") + prop.gcnArchName + ", library is built for gfx950");
    auto* l = new (std::nothrow) pointid_layers_s();
    if (!l) return set_error(POINTID_ENOMEM, "host allocation failed");
    l->device = device;
    l->cus = prop.multiProcessorCount;
    *out = l;
    return (int)POINTID_OK;
  });
}

int pointid_layers_destroy(pointid_layers l) {
  if (!l) return POINTID_OK;
  {
    DeviceScope dev(l->device);
    (void)hipDeviceSynchronize();
    free_scratch(&l->scratch);
  }
  delete l;
  return POINTID_OK;
}

int pointid_layers_trim(pointid_layers l, uint64_t keep_bytes, uint64_t* cached_bytes) {
  if (!l) return set_error(POINTID_EINVAL, "layers is NULL");
  return guarded([&] {
    DeviceScope dev(l->device);
    if (dev.error() != hipSuccess) return hip_fail(dev.error(), "hipSetDevice");
    return trim_scratch(&l->scratch, keep_bytes, cached_bytes);
  });
}

int pointid_dense(pointid_layers l, int dtype, int act, int64_t m, int64_t k, int64_t n, const pointid_matrix* x,
                  const pointid_matrix* w, const float* bias, const pointid_matrix* residual, const pointid_matrix* y,
                  const pointid_kept* keep_z, void* stream) {
  return guarded([&] {
    TRY(check_call(l, dtype, act, m, k, n));
    if (m == 0) return (int)POINTID_OK;
    TRY(check_matrix(x, "x", dtype, m, k));
    TRY(check_matrix(w, "w", dtype, k, n));
    TRY(check_floats(bias, "bias"));
    TRY(check_matrix(residual, "residual", dtype, m, n, true));
    TRY(check_matrix(y, "y", dtype, m, n));
    TRY(check_kept(keep_z, "keep_z", dtype, m, n, true));
    Forward f;
    std::memset(&f, 0, sizeof(f));
    f.dtype = dtype, f.act = act, f.halves = 1, f.m = m, f.k = k, f.n = n;
    f.x = matrix_of(x, m, k);
    f.w[0] = f.w[1] = matrix_of(w, k, n);
    f.bias[0] = bias;
    f.residual = matrix_of(residual, m, n);
    f.y = matrix_of(y, m, n);
    f.keep[0] = kept_of(keep_z, m, n);
    return run_forward(l, f, static_cast<hipStream_t>(stream));
  });
}

int pointid_gated(pointid_layers l, int dtype, int act, int64_t m, int64_t k, int64_t n, const pointid_matrix* x,
                  const pointid_matrix* wg, const pointid_matrix* wu, const float* bias_g, const float* bias_u,
                  const pointid_matrix* h, const pointid_kept* keep_g, const pointid_kept* keep_u, void* stream) {
  return guarded([&] {
    TRY(check_call(l, dtype, act, m, k, n));
    if (m == 0) return (int)POINTID_OK;
    TRY(check_matrix(x, "x", dtype, m, k));
    TRY(check_matrix(wg, "wg", dtype, k, n));
    TRY(check_matrix(wu, "wu", dtype, k, n));
    TRY(check_floats(bias_g, "bias_g"));
    TRY(check_floats(bias_u, "bias_u"));
    TRY(check_matrix(h, "h", dtype, m, n));
    TRY(check_kept(keep_g, "keep_g", dtype, m, n, true));
    TRY(check_kept(keep_u, "keep_u", dtype, m, n, true));
    Forward f;
    std::memset(&f, 0, sizeof(f));
    f.dtype = dtype, f.act = act, f.halves = 2, f.m = m, f.k = k, f.n = n;
    f.x = matrix_of(x, m, k);
    f.w[0] = matrix_of(wg, k, n);
    f.w[1] = matrix_of(wu, k, n);
    f.bias[0] = bias_g;
    f.bias[1] = bias_u;
    f.y = matrix_of(h, m, n);
    f.keep[0] = kept_of(keep_g, m, n);
    f.keep[1] = kept_of(keep_u, m, n);
    return run_forward(l, f, static_cast<hipStream_t>(stream));
  });
}

int pointid_dense_backward(pointid_layers l, int dtype, int act, int64_t m, int64_t k, int64_t n,
                           const pointid_matrix* dy, const pointid_kept* x, const pointid_matrix* w,
                           const pointid_kept* z, const pointid_matrix* dx, const pointid_matrix* dw, float* db,
                           void* stream) {
  return guarded([&] {
    TRY(check_call(l, dtype, act, m, k, n));
    const bool want_dx = dx && dx->data && m > 0, want_dw = dw && dw->data;
    TRY(check_matrix(dy, "dy", dtype, m, n));
    TRY(check_kept(x, "x", dtype, m, k, !want_dw));
    TRY(check_matrix(w, "w", dtype, k, n, !want_dx));
    TRY(check_kept(z, "z", dtype, m, n, act == POINTID_ACT_NONE));
    TRY(check_matrix(dx, "dx", dtype, m, k, true));
    TRY(check_matrix(dw, "dw", dtype, k, n, true));
    TRY(check_floats(db, "db"));
    Backward b;
    std::memset(&b, 0, sizeof(b));
    b.dtype = dtype, b.act = act, b.halves = 1, b.m = m, b.k = k, b.n = n;
    b.dy = matrix_of(dy, m, n);
    b.x = kept_of(x, m, k);
    b.w[0] = matrix_of(w, k, n);
    if (act != POINTID_ACT_NONE) b.z[0] = kept_of(z, m, n);
    if (want_dx) b.dx = matrix_of(dx, m, k);
    if (want_dw) b.dw[0] = matrix_of(dw, k, n);
    b.db[0] = db;
    return run_backward(l, b, static_cast<hipStream_t>(stream));
  });
}

int pointid_gated_backward(pointid_layers l, int dtype, int act, int64_t m, int64_t k, int64_t n,
                           const pointid_matrix* dh, const pointid_kept* x, const pointid_matrix* wg,
                           const pointid_matrix* wu, const pointid_kept* g, const pointid_kept* u,
                           const pointid_matrix* dx, const pointid_matrix* dwg, const pointid_matrix* dwu, float* dbg,
                           float* dbu, void* stream) {
  return guarded([&] {
    TRY(check_call(l, dtype, act, m, k, n));
    const bool want_dx = dx && dx->data && m > 0, want_dw = dwg && dwg->data;
    if (want_dw != (dwu && dwu->data)) return set_error(POINTID_EINVAL, "dwg and dwu are given both or neither");
    TRY(check_matrix(dh, "dh", dtype, m, n));
    TRY(check_kept(x, "x", dtype, m, k, !want_dw));
    TRY(check_matrix(wg, "wg", dtype, k, n, !want_dx));
    TRY(check_matrix(wu, "wu", dtype, k, n, !want_dx));
    TRY(check_kept(g, "g", dtype, m, n, false));
    TRY(check_kept(u, "u", dtype, m, n, false));
    if (m > 0 && !g->full.data != !u->full.data)
      return set_error(POINTID_EINVAL, "g and u are kept alike: two matrices or two checkpoints");
    TRY(check_matrix(dx, "dx", dtype, m, k, true));
    TRY(check_matrix(dwg, "dwg", dtype, k, n, true));
    TRY(check_matrix(dwu, "dwu", dtype, k, n, true));
    TRY(check_floats(dbg, "dbg"));
    TRY(check_floats(dbu, "dbu"));
    Backward b;
    std::memset(&b, 0, sizeof(b));
    b.dtype = dtype, b.act = act, b.halves = 2, b.m = m, b.k = k, b.n = n;
    b.dy = matrix_of(dh, m, n);
    b.x = kept_of(x, m, k);
    b.w[0] = matrix_of(wg, k, n);
    b.w[1] = matrix_of(wu, k, n);
    b.z[0] = kept_of(g, m, n);
    b.z[1] = kept_of(u, m, n);
    if (want_dx) b.dx = matrix_of(dx, m, k);
    if (want_dw) {
      b.dw[0] = matrix_of(dwg, k, n);
      b.dw[1] = matrix_of(dwu, k, n);
    }
    b.db[0] = dbg;
    b.db[1] = dbu;
    return run_backward(l, b, static_cast<hipStream_t>(stream));
  });
}

int pointid_checkpoint_save(int dtype, int64_t rows, int64_t cols, const pointid_matrix* x,
                            const pointid_checkpoint* out, void* stream) {
  return guarded([&] {
    TRY(check_checkpoint_call(dtype, rows, cols, x, out));
    if (rows == 0) return (int)POINTID_OK;
    const pointid_matrix a = matrix_of(x, rows, cols);
    const hipError_t e = launch_checkpoint_save(a.data, a.ld, dtype, rows, cols, {out->codes, out->exponents},
                                                static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)POINTID_OK : hip_fail(e, "checkpoint save launch");
  });
}

int pointid_checkpoint_load(int dtype, int64_t rows, int64_t cols, const pointid_checkpoint* in,
                            const pointid_matrix* out, void* stream) {
  return guarded([&] {
    TRY(check_checkpoint_call(dtype, rows, cols, out, in));
    if (rows == 0) return (int)POINTID_OK;
    const pointid_matrix a = matrix_of(out, rows, cols);
    const hipError_t e = launch_checkpoint_load({in->codes, in->exponents}, rows, cols, dtype, a.data, a.ld,
                                                static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)POINTID_OK : hip_fail(e, "checkpoint load launch");
  });
}

}  // extern "C"
