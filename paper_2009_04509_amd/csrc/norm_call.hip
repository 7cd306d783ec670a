// C ABI of dropout, the norms at a residual joint and log probabilities (declared in
// include/pointid.h): argument checks, scratch, launch sequencing.  Every call only enqueues work.
#include <cmath>

#include "layers_call.h"
#include "norm.h"

using namespace pointid;

namespace {

constexpr int64_t kMaxCols = int64_t(1) << 20;

int check_call(pointid_layers l, int dtype, int64_t m, int64_t n) {
  if (!l) return set_error(POINTID_EINVAL, "layers is NULL");
  if (dtype != POINTID_FP32 && dtype != POINTID_BF16 && dtype != POINTID_FP16)
    return set_error(POINTID_EUNSUPPORTED, "dtype must be POINTID_FP32, POINTID_BF16 or POINTID_FP16");
  if (m < 0 || m > kMaxRows) return set_error(POINTID_EINVAL, "m must be in [0, 2^28]");
  if (n < 1 || n > kMaxCols) return set_error(POINTID_EINVAL, "n must be in [1, 2^20]");
  return POINTID_OK;
}
int check_drop(const pointid_drop& d) {
  if (!(d.p >= 0.0 && d.p <= 1.0)) return set_error(POINTID_EINVAL, "p must be in [0, 1]");
  if (reinterpret_cast<uintptr_t>(d.step) % 8) return set_error(POINTID_EINVAL, "step is not aligned to 8 bytes");
  return POINTID_OK;
}
int check_norm(const pointid_norm_of& n, const char* name) {
  if (n.kind == POINTID_NORM_NONE) return POINTID_OK;
  if (n.kind != POINTID_NORM_RMS && n.kind != POINTID_NORM_LAYER)
    return set_error(POINTID_EINVAL, std::string(name) + ": no kind of norm");
  if (!(n.eps >= 0.f) || std::isinf(n.eps))
    return set_error(POINTID_EINVAL, std::string(name) + ": eps must be finite and not negative");
  TRY(check_floats(n.weight, name));
  return check_floats(n.bias, name);
}
int check_block(const pointid_block& b) {
  TRY(check_norm(b.norm, "the norm after the block"));
  TRY(check_floats(b.gate, "gate"));
  if (!std::isfinite(b.scale)) return set_error(POINTID_EINVAL, "scale must be finite");
  return check_drop(b.drop);
}
int check_scale(float scale) {
  if (!(scale >= 0x1p-64f && scale <= 0x1p64f)) return set_error(POINTID_EINVAL, "scale must be in [2^-64, 2^64]");
  return POINTID_OK;
}
int check_scratch(const void* scratch) {
  if (reinterpret_cast<uintptr_t>(scratch) % 256) return set_error(POINTID_EINVAL, "scratch is not aligned to 256 bytes");
  return POINTID_OK;
}

Drop drop_of(const pointid_drop& d) {
  Drop r;
  r.threshold = (uint32_t)std::floor(d.p * 65536.0 + 0.5);
  r.scale = r.threshold < 65536 ? (float)(65536.0 / (65536 - r.threshold)) : 0.f;
  r.seed = d.seed, r.offset = d.offset, r.step = r.threshold ? d.step : nullptr;
  return r;
}
NormOf norm_of(const pointid_norm_of* n) {
  NormOf r;
  std::memset(&r, 0, sizeof(r));
  if (n && n->kind) r.kind = n->kind, r.eps = n->eps, r.weight = n->weight, r.bias = n->bias;
  return r;
}
Rows rows_of(const pointid_matrix* a, int64_t rows, int64_t cols) {
  const pointid_matrix r = matrix_of(a, rows, cols);
  return {static_cast<char*>(r.data), r.ld};
}
bool has(const pointid_norm_of* n) { return n && n->kind != POINTID_NORM_NONE; }

// What the forward and the backward call have alike.
template <class Args>
void set_block(Args* a, const pointid_norm_of* norm, const pointid_block* block, int64_t m, int64_t n, int dtype) {
  std::memset(static_cast<void*>(a), 0, sizeof(*a));
  a->before = norm_of(norm);
  a->scale = 1.f;
  a->rows = m, a->cols = n, a->dtype = dtype;
  if (!block) return;
  a->after = norm_of(&block->norm);
  a->gate = block->gate;
  a->scale = block->scale;
  a->drop = drop_of(block->drop);
}

size_t means_bytes(int64_t m) { return sizeof(float) * 4 * (size_t)m; }
size_t sums_bytes(int blocks, int wanted, int64_t n) { return sizeof(float) * (size_t)blocks * wanted * n; }

}  // namespace

extern "C" {

int pointid_dropout(pointid_layers l, int dtype, int64_t m, int64_t n, const pointid_matrix* x,
                    const pointid_drop* drop, const pointid_matrix* residual, const pointid_matrix* y, void* stream) {
  return guarded([&] {
    TRY(check_call(l, dtype, m, n));
    if (!drop) return set_error(POINTID_EINVAL, "drop is NULL");
    TRY(check_drop(*drop));
    if (m == 0) return (int)POINTID_OK;
    TRY(check_matrix(x, "x", dtype, m, n));
    TRY(check_matrix(residual, "residual", dtype, m, n, true));
    TRY(check_matrix(y, "y", dtype, m, n));
    DropoutArgs a;
    std::memset(static_cast<void*>(&a), 0, sizeof(a));
    const Rows rx = rows_of(x, m, n), rr = rows_of(residual, m, n), ry = rows_of(y, m, n);
    a.x = rx.p, a.ld_x = rx.ld;
    a.residual = rr.p, a.ld_residual = rr.ld;
    a.y = ry.p, a.ld_y = ry.ld;
    a.rows = m, a.cols = n, a.dtype = dtype;
    a.drop = drop_of(*drop);
    DeviceScope dev(l->device);
    if (dev.error() != hipSuccess) return hip_fail(dev.error(), "hipSetDevice");
    Call call(l, static_cast<hipStream_t>(stream));
    return call.run("dropout", true, [&] { return launch_dropout(a, call.stream()); });
  });
}

int pointid_norm(pointid_layers l, int dtype, int64_t m, int64_t n, const pointid_matrix* x,
                 const pointid_norm_of* norm, const pointid_block* block, const pointid_matrix* total,
                 const pointid_matrix* h, float* stats, void* stream) {
  return guarded([&] {
    TRY(check_call(l, dtype, m, n));
    if (norm) TRY(check_norm(*norm, "norm"));
    if (block) TRY(check_block(*block));
    if (m == 0) return (int)POINTID_OK;
    const bool want_total = total && total->data, want_h = h && h->data;
    if (!want_total && !want_h) return set_error(POINTID_EINVAL, "neither total nor h is given");
    if (want_h != has(norm)) return set_error(POINTID_EINVAL, "norm and h are given both or neither");
    if (want_total && !block) return set_error(POINTID_EINVAL, "total without a block is x itself");
    TRY(check_matrix(x, "x", dtype, m, n));
    if (block) TRY(check_matrix(&block->out, "out", dtype, m, n));
    TRY(check_matrix(total, "total", dtype, m, n, true));
    TRY(check_matrix(h, "h", dtype, m, n, true));
    if (!aligned16(stats)) return set_error(POINTID_EINVAL, "stats is not aligned to 16 bytes");
    NormArgs a;
    set_block(&a, norm, block, m, n, dtype);
    a.x = rows_of(x, m, n);
    if (block) a.o = rows_of(&block->out, m, n);
    a.t = rows_of(total, m, n);
    a.h = rows_of(h, m, n);
    a.stats = stats;
    DeviceScope dev(l->device);
    if (dev.error() != hipSuccess) return hip_fail(dev.error(), "hipSetDevice");
    Call call(l, static_cast<hipStream_t>(stream));
    return call.run("norm", true, [&] { return launch_norm(a, call.stream()); });
  });
}

uint64_t pointid_norm_backward_scratch(pointid_layers l, int64_t m, int64_t n) {
  if (!l || m < 0 || m > kMaxRows || n < 1 || n > kMaxCols) return 0;
  // the most blocks that any such call has
  NormBackArgs a;
  std::memset(static_cast<void*>(&a), 0, sizeof(a));
  a.rows = m, a.cols = n, a.dtype = POINTID_FP32;
  const NormBackPlan plan = plan_norm_back(a, l->cus);
  if (plan.held && plan.blocks <= 1) return 0;
  return (plan.held ? 0 : pad256(means_bytes(m))) + pad256(sums_bytes(plan.blocks, kNormSums, n));
}

int pointid_norm_backward(pointid_layers l, int dtype, int64_t m, int64_t n, const pointid_matrix* dh,
                          const pointid_matrix* total, const float* stats, const pointid_norm_of* norm,
                          const pointid_block* block, const pointid_matrix* dtotal, const pointid_norm_grads* grads,
                          void* scratch, uint64_t scratch_bytes, void* stream) {
  return guarded([&] {
    TRY(check_call(l, dtype, m, n));
    if (!grads) return set_error(POINTID_EINVAL, "grads is NULL");
    if (norm) TRY(check_norm(*norm, "norm"));
    if (block) TRY(check_block(*block));
    const bool after = block && block->norm.kind != POINTID_NORM_NONE;
    const pointid_norm_grads& g = *grads;
    if ((g.dweight || g.dbias) && !has(norm)) return set_error(POINTID_EINVAL, "dweight or dbias without norm");
    if (!block && (g.dout.data || g.dgate)) return set_error(POINTID_EINVAL, "dout or dgate without a block");
    if ((g.dblock_weight || g.dblock_bias) && !after)
      return set_error(POINTID_EINVAL, "dblock_weight or dblock_bias without a norm after the block");
    for (const float* p : {g.dweight, g.dbias, g.dblock_weight, g.dblock_bias, g.dgate}) TRY(check_floats(p, "a parameter's gradient"));
    TRY(check_scratch(scratch));
    if (has(norm)) {
      TRY(check_matrix(dh, "dh", dtype, m, n));
      TRY(check_matrix(total, "total", dtype, m, n));
    }
    const bool need_out = after || g.dgate;
    if (need_out) TRY(check_matrix(&block->out, "out", dtype, m, n));
    TRY(check_matrix(dtotal, "dtotal", dtype, m, n, true));
    if (!has(norm) && m > 0 && !(dtotal && dtotal->data)) return set_error(POINTID_EINVAL, "neither norm nor dtotal is given");
    TRY(check_matrix(&g.dx, "dx", dtype, m, n, true));
    TRY(check_matrix(&g.dout, "dout", dtype, m, n, true));
    if (m > 0 && (has(norm) || after) && (!stats || !aligned16(stats)))
      return set_error(POINTID_EINVAL, "stats is NULL or not aligned to 16 bytes");
    NormBackArgs a;
    set_block(&a, norm, block, m, n, dtype);
    if (has(norm)) {
      a.dh = rows_of(dh, m, n);
      a.t = rows_of(total, m, n);
    }
    a.dt = rows_of(dtotal, m, n);
    if (need_out) a.o = rows_of(&block->out, m, n);
    a.dx = rows_of(&g.dx, m, n);
    a.dout = rows_of(&g.dout, m, n);
    a.stats = has(norm) || after ? stats : nullptr;
    float* const out[kNormSums] = {g.dweight, g.dbias, g.dblock_weight, g.dblock_bias, g.dgate};
    int wanted = 0;
    for (int s = 0; s < kNormSums; ++s) wanted += (a.out[s] = out[s]) != nullptr;
    if (!a.dx.p && !a.dout.p && !wanted) return (int)POINTID_OK;
    if (m == 0 && !wanted) return (int)POINTID_OK;

    DeviceScope dev(l->device);
    if (dev.error() != hipSuccess) return hip_fail(dev.error(), "hipSetDevice");
    Call call(l, static_cast<hipStream_t>(stream), scratch, scratch_bytes);
    const NormBackPlan plan = plan_norm_back(a, l->cus);
    a.blocks = plan.blocks;
    const bool means = !plan.held && (has(norm) || after);
    if (means) call.want(&a.means, means_bytes(m));
    const bool alone = plan.held && plan.blocks == 1;        // its sums are the sums
    if (wanted && !alone) call.want(&a.part, sums_bytes(plan.blocks, wanted, n));
    TRY(call.reserve());
    if (m > 0) {
      if (means) TRY(call.run("norm_means", false, [&] { return launch_norm_means(a, call.stream()); }));
      TRY(call.run("norm_back", !wanted || alone, [&] { return launch_norm_back(a, plan.held, call.stream()); }));
    }
    if (!wanted || alone) return (int)POINTID_OK;
    return call.run("norm_sums", true, [&] { return launch_norm_sums(a, call.stream()); });
  });
}

uint64_t pointid_logprobs_scratch(pointid_layers l, int64_t m, int64_t n, int32_t top) {
  if (!l || m < 1 || m > kMaxRows || n < 1 || n > kMaxCols || top < 0 || top > kMaxTop) return 0;
  const int32_t splits = scan_splits(m, n, l->cus);
  if (splits == 1) return 0;
  return pad256(sizeof(float) * 4 * (size_t)m * splits) + pad256(sizeof(uint64_t) * (size_t)m * splits * top);
}

int pointid_logprobs(pointid_layers l, int dtype, int64_t m, int64_t n, const pointid_matrix* logits, float scale,
                     const int32_t* targets, float* logp, float* lse, float* entropy, int32_t top, int32_t* top_ids,
                     float* top_logp, void* scratch, uint64_t scratch_bytes, void* stream) {
  return guarded([&] {
    TRY(check_call(l, dtype, m, n));
    TRY(check_scale(scale));
    if (top < 0 || top > kMaxTop || top > n) return set_error(POINTID_EINVAL, "top must be in [0, 64] and at most n");
    TRY(check_scratch(scratch));
    if (m == 0) return (int)POINTID_OK;
    TRY(check_matrix(logits, "logits", dtype, m, n));
    if (logp && !targets) return set_error(POINTID_EINVAL, "logp needs targets");
    if (top > 0 && (!top_ids || !top_logp)) return set_error(POINTID_EINVAL, "top_ids or top_logp is NULL");
    if (!logp && !lse && !entropy && top == 0) return set_error(POINTID_EINVAL, "no output is given");
    for (const float* p : {logp, lse, entropy, top_logp}) TRY(check_floats(p, "an output"));
    for (const int32_t* p : {targets, (const int32_t*)top_ids})
      TRY(check_floats(reinterpret_cast<const float*>(p), p == targets ? "targets" : "top_ids"));
    ScanArgs a;
    std::memset(static_cast<void*>(&a), 0, sizeof(a));
    a.x = rows_of(logits, m, n);
    a.rows = m, a.cols = n, a.dtype = dtype;
    a.scale = scale;
    a.targets = targets;
    a.logp = logp, a.lse = lse, a.entropy = entropy;
    a.top = top, a.top_ids = top_ids, a.top_logp = top_logp;
    a.splits = scan_splits(m, n, l->cus);
    a.split_cols = round_up((n + a.splits - 1) / a.splits, 8);
    DeviceScope dev(l->device);
    if (dev.error() != hipSuccess) return hip_fail(dev.error(), "hipSetDevice");
    Call call(l, static_cast<hipStream_t>(stream), scratch, scratch_bytes);
    if (a.splits > 1) {
      call.want(&a.part, sizeof(float) * 4 * (size_t)m * a.splits);
      call.want(&a.part_top, sizeof(uint64_t) * (size_t)m * a.splits * top);
    }
    TRY(call.reserve());
    TRY(call.run("logprobs", a.splits == 1, [&] { return launch_logprobs(a, call.stream()); }));
    if (a.splits == 1) return (int)POINTID_OK;
    return call.run("logprobs_join", true, [&] { return launch_logprobs_join(a, call.stream()); });
  });
}

int pointid_logprobs_backward(pointid_layers l, int dtype, int64_t m, int64_t n, const pointid_matrix* logits,
                              float scale, const float* lse, const int32_t* targets, const float* dlogp,
                              const float* entropy, const float* dentropy, const float* dlse,
                              const pointid_matrix* dlogits, void* stream) {
  return guarded([&] {
    TRY(check_call(l, dtype, m, n));
    TRY(check_scale(scale));
    if (m == 0) return (int)POINTID_OK;
    TRY(check_matrix(logits, "logits", dtype, m, n));
    TRY(check_matrix(dlogits, "dlogits", dtype, m, n));
    if (!lse) return set_error(POINTID_EINVAL, "lse is NULL");
    if (!dlogp && !dentropy && !dlse) return set_error(POINTID_EINVAL, "no gradient is given");
    if (dlogp && !targets) return set_error(POINTID_EINVAL, "dlogp needs targets");
    if (dentropy && !entropy) return set_error(POINTID_EINVAL, "dentropy needs entropy");
    for (const float* p : {lse, dlogp, entropy, dentropy, dlse}) TRY(check_floats(p, "lse, entropy or a gradient"));
    TRY(check_floats(reinterpret_cast<const float*>(targets), "targets"));
    ScanBackArgs a;
    std::memset(static_cast<void*>(&a), 0, sizeof(a));
    a.x = rows_of(logits, m, n);
    a.dx = rows_of(dlogits, m, n);
    a.rows = m, a.cols = n, a.dtype = dtype;
    a.scale = scale;
    a.targets = dlogp ? targets : nullptr;
    a.lse = lse, a.entropy = entropy, a.dlogp = dlogp, a.dentropy = dentropy, a.dlse = dlse;
    DeviceScope dev(l->device);
    if (dev.error() != hipSuccess) return hip_fail(dev.error(), "hipSetDevice");
    Call call(l, static_cast<hipStream_t>(stream));
    return call.run("logprobs_backward", true, [&] { return launch_logprobs_back(a, call.stream()); });
  });
}

}  // extern "C"
