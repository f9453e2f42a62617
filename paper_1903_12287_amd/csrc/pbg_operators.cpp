// Host side of the operators on a caller's own tensors (include/pbg_operators.h): argument checks, workspace and
// launch sequence.  A call checks on the host what the host can see; what lies in device arrays (offsets, labels) is
// checked by a kernel ahead of the work, whose word every workgroup behind it reads before it writes anything, or, where
// there is little of it, by every workgroup itself.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "operators.h"
#include "pbg_operators.h"
#include "runtime_internal.h"

namespace {

// A matrix of rows in memory, for the overlap checks.
struct Rows {
  const void* p;
  int64_t n, width, ld;   // in elements
  int es;
  uintptr_t begin() const { return (uintptr_t)p; }
  uintptr_t end() const { return (uintptr_t)p + ((size_t)(n - 1) * ld + width) * es; }
  bool empty() const { return !p || n <= 0 || width <= 0; }
};

bool overlap(const Rows& a, const Rows& b) {
  if (a.empty() || b.empty() || a.end() <= b.begin() || b.end() <= a.begin()) return false;
  if (a.ld != b.ld || a.es != b.es) return true;
  // rows of one stride: column ranges apart do not meet
  const int64_t pitch = a.ld * a.es;
  const int64_t off = (int64_t)(b.begin() - a.begin());   // signed
  const int64_t at = ((off % pitch) + pitch) % pitch;     // b's first column in a's rows
  return at < a.width * a.es || at + b.width * b.es > pitch;
}

pbg_status begin_call(pbg_ctx* ctx, const char* name) {
  if (!ctx) return PBG_ERR_INVALID_ARG;
  if (ctx->invalid) return set_err(ctx, PBG_ERR_STATE, "context failed to initialise");
  ctx->err.clear();
  // an error that is pending in the runtime ends the call before it has launched anything
  const hipError_t pending = hipGetLastError();
  if (pending != hipSuccess) return set_err(ctx, PBG_ERR_DEVICE, "pending ahead of %s: %s", name, hipGetErrorString(pending));
  int cur = -1;
  if (hipGetDevice(&cur) != hipSuccess || cur != ctx->device)
    return set_err(ctx, PBG_ERR_STATE, "the context's device %d must be current (current: %d)", ctx->device, cur);
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  const hipError_t e = hipStreamIsCapturing(ctx->cs, &cap);
  if (e == hipErrorStreamCaptureImplicit || (e == hipSuccess && cap != hipStreamCaptureStatusNone)) {
    if (e != hipSuccess) (void)hipGetLastError();
    return set_err(ctx, PBG_ERR_STATE, "%s waits for its work and cannot be recorded into a graph", name);
  }
  if (e != hipSuccess) return hip_fail(ctx, e, "hipStreamIsCapturing");
  return PBG_OK;
}

pbg_status workspace(pbg_ctx* ctx, size_t bytes) {
  if (ctx->ops_ws_bytes >= bytes) return PBG_OK;
  if (ctx->ops_ws) (void)hipFree(ctx->ops_ws);   // calls wait for their work: nothing uses it
  ctx->ops_ws = nullptr;
  ctx->ops_ws_bytes = 0;
  const size_t want = (bytes + 0xFFFFF) & ~(size_t)0xFFFFF;
  if (hipMalloc(&ctx->ops_ws, want) != hipSuccess) {
    (void)hipGetLastError();
    ctx->ops_ws = nullptr;
    return set_err(ctx, PBG_ERR_OUT_OF_MEMORY, "workspace allocation failed (%zu bytes)", want);
  }
  ctx->ops_ws_bytes = want;
  return PBG_OK;
}

// Waits for the call's work, whatever e says (what was launched reads the caller's arrays), and turns the device's
// verdict on the arguments into a status.
pbg_status end_call(pbg_ctx* ctx, hipError_t e, const char* name) {
  const hipError_t es = hipStreamSynchronize(ctx->cs);
  if (e == hipSuccess) e = es;
  if (e != hipSuccess) return hip_fail(ctx, e, name);
  const uint32_t flag = *(volatile uint32_t*)ctx->edge_hflag;
  if (flag & OPS_BAD_OFFSETS)
    return set_err(ctx, PBG_ERR_INVALID_ARG, "%s: offsets must be nondecreasing and within [0, n]", name);
  if (flag & OPS_BAD_LABEL)
    return set_err(ctx, PBG_ERR_INVALID_ARG, "%s: a label is not below the number of candidates", name);
  ctx->edge_dirty = false;   // else the next call clears the flags
  return PBG_OK;
}

bool aligned(const void* p, int es) { return ((uintptr_t)p & (uintptr_t)(es - 1)) == 0; }

bool bad_ld(int64_t ld, int64_t width) { return ld < width || ld > PBG_OPS_MAX_LD; }

// The operands of a grouped product as the matrix kernels read them: rows at multiples of 16 bytes, whole 16 bytes
// of values.  Others are copied into the workspace (behind `front` bytes of it), zeros behind their rows.
struct Operands {
  int64_t es, ev;
  int count = 0;
  GroupPack op[3];
  size_t bytes = 0;
  size_t at[3];
  const void** p[3];
  int64_t* out_ld[3];
  explicit Operands(int type) : es(type_bytes(type)), ev(16 / type_bytes(type)) {}
  int padded(int w) const { return (int)((w + ev - 1) / ev * ev); }
  // *ptr (n rows of *row_ld, `matrix` of them a matrix) is used as it is or replaced by its copy; true: copied
  bool add(const void** ptr, int64_t* row_ld, int64_t n, int w, int matrix = 0) {
    if (!*ptr || n <= 0) return false;
    if (((uintptr_t)*ptr & 15) == 0 && *row_ld % ev == 0 && w % ev == 0) return false;
    op[count] = {*ptr, nullptr, *row_ld, n, matrix, w, padded(w)};
    at[count] = bytes;
    bytes += ((size_t)n * padded(w) * es + 255) & ~(size_t)255;
    p[count] = ptr;
    out_ld[count] = row_ld;
    ++count;
    return true;
  }
  // the matrices: no more places than there are rows
  void add_matrices(GroupArgs* g) {
    const int64_t places = std::min<int64_t>(g->groups, g->n);
    g->a_by_row = add(&g->a, &g->lda, places * g->m, g->k, g->m) && places < g->groups;
  }
  void place(char* ws) {
    for (int i = 0; i < count; ++i) {
      op[i].dst = ws + at[i];
      *p[i] = op[i].dst;
      *out_ld[i] = op[i].wp;
    }
  }
};

// the plan's tables and partial sums in the workspace from p (a multiple of 256 bytes) on
void place_plan(GroupPlan* plan, char* p, int64_t m, int64_t k) {
  plan->partial = (float*)p;
  p += (size_t)plan->partial_slots * m * k * 4;
  p = (char*)(((uintptr_t)p + 15) & ~(uintptr_t)15);
  if (!plan->tables) return;
  plan->rows.at = (int4*)p;
  plan->da.at = plan->rows.at + plan->rows.count;
  plan->join = plan->da.at + plan->da.count;
}

pbg_status check_group(pbg_ctx* ctx, int32_t dtype, const int64_t* offsets, int32_t groups, int64_t n, int32_t in_dim,
                       int32_t out_dim) {
  if (dtype < PBG_TYPE_F32 || dtype > PBG_TYPE_F16) return set_err(ctx, PBG_ERR_INVALID_ARG, "unknown type %d", dtype);
  if (groups < 1 || groups > PBG_OPS_MAX_GROUPS) return set_err(ctx, PBG_ERR_INVALID_ARG, "groups out of range");
  if (n < 0 || n > 0x7FFFFFFFll) return set_err(ctx, PBG_ERR_INVALID_ARG, "n out of range");
  if (in_dim < 1 || in_dim > PBG_OPS_MAX_DIM || out_dim < 1 || out_dim > PBG_OPS_MAX_DIM)
    return set_err(ctx, PBG_ERR_INVALID_ARG, "in_dim and out_dim must be in [1, %d]", PBG_OPS_MAX_DIM);
  if (!offsets || !aligned(offsets, 8)) return set_err(ctx, PBG_ERR_INVALID_ARG, "NULL or misaligned offsets");
  return PBG_OK;
}

}  // namespace

extern "C" pbg_status pbg_group_linear(pbg_ctx* ctx, int32_t dtype, const void* x, int64_t ldx, const void* a,
                                       const int64_t* offsets, int32_t groups, int64_t n, int32_t in_dim,
                                       int32_t out_dim, void* y, int64_t ldy) {
  pbg_status st = begin_call(ctx, "pbg_group_linear");
  if (st != PBG_OK) return st;
  st = check_group(ctx, dtype, offsets, groups, n, in_dim, out_dim);
  if (st != PBG_OK) return st;
  const int es = type_bytes(dtype);
  if (bad_ld(ldx, in_dim) || bad_ld(ldy, out_dim))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "a row stride is below its width or above %d", PBG_OPS_MAX_LD);
  if (n > 0 && (!x || !a || !y)) return set_err(ctx, PBG_ERR_INVALID_ARG, "NULL array");
  if (!aligned(x, es) || !aligned(a, es) || !aligned(y, es))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "an array is not aligned to its elements");
  const Rows rx{x, n, in_dim, ldx, es}, ry{y, n, out_dim, ldy, es}, ra{a, (int64_t)groups * out_dim, in_dim, in_dim, es};
  const Rows ro{offsets, 1, groups + 1, groups + 1, 8};
  if (overlap(ry, rx) || overlap(ry, ra) || overlap(ry, ro))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "y overlaps an input");
  st = ensure_edge_flags(ctx);
  if (st != PBG_OK) return st;
  GroupArgs g{x, a, nullptr, y, ldx, in_dim, 0, ldy, 0, offsets, groups, n, in_dim, out_dim, in_dim, out_dim, false,
              ctx->edge_flag, ctx->edge_hflag};
  Operands ops(dtype);
  if (n > 0) {
    ops.add(&g.x, &g.ldx, n, in_dim);
    ops.add_matrices(&g);
  }
  GroupPlan plan = plan_group(dtype, GP_FORWARD, n, groups, out_dim, in_dim, false);
  st = workspace(ctx, ops.bytes + plan.bytes());
  if (st != PBG_OK) return st;
  ops.place((char*)ctx->ops_ws);
  place_plan(&plan, (char*)ctx->ops_ws + ops.bytes, out_dim, in_dim);
  g.kd = ops.padded(in_dim);
  g.a_group = (int64_t)out_dim * g.lda;
  ctx->edge_dirty = true;
  launch_group_plan(plan, offsets, groups, n, ctx->edge_flag, ctx->cs);
  launch_group_pack(dtype, ops.count, ops.op, offsets, groups, ctx->cs);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) {
    launch_group_product(g, dtype, GP_FORWARD, plan, ctx->cs);
    e = hipGetLastError();
  }
  return end_call(ctx, e, "pbg_group_linear");
}

extern "C" pbg_status pbg_group_linear_backward(pbg_ctx* ctx, int32_t dtype, const void* x, int64_t ldx, const void* a,
                                                const void* dy, int64_t lddy, const int64_t* offsets, int32_t groups,
                                                int64_t n, int32_t in_dim, int32_t out_dim, void* dx, int64_t lddx,
                                                void* da) {
  pbg_status st = begin_call(ctx, "pbg_group_linear_backward");
  if (st != PBG_OK) return st;
  st = check_group(ctx, dtype, offsets, groups, n, in_dim, out_dim);
  if (st != PBG_OK) return st;
  const int es = type_bytes(dtype);
  if (bad_ld(lddy, out_dim) || ((da || x) && bad_ld(ldx, in_dim)) || (dx && bad_ld(lddx, in_dim)))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "a row stride is below its width or above %d", PBG_OPS_MAX_LD);
  if (n > 0 && (!dy || (da && !x) || (dx && !a))) return set_err(ctx, PBG_ERR_INVALID_ARG, "NULL array");
  if (!aligned(x, es) || !aligned(a, es) || !aligned(dy, es) || !aligned(dx, es) || !aligned(da, es))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "an array is not aligned to its elements");
  const int64_t gm = (int64_t)groups * out_dim;
  const Rows rx{x, n, in_dim, ldx, es}, ra{a, gm, in_dim, in_dim, es};
  const Rows rdy{dy, n, out_dim, lddy, es}, rdx{dx, n, in_dim, lddx, es}, rda{da, gm, in_dim, in_dim, es};
  const Rows ro{offsets, 1, groups + 1, groups + 1, 8};
  for (const Rows* in : {&rx, &ra, &rdy, &ro})
    if (overlap(rdx, *in) || overlap(rda, *in)) return set_err(ctx, PBG_ERR_INVALID_ARG, "an output overlaps an input");
  if (overlap(rdx, rda)) return set_err(ctx, PBG_ERR_INVALID_ARG, "dx and da overlap");
  if (!dx && !da) return PBG_OK;
  st = ensure_edge_flags(ctx);
  if (st != PBG_OK) return st;
  GroupArgs g{x, a, dy, nullptr, ldx, in_dim, lddy, 0, 0, offsets, groups, n, in_dim, out_dim, in_dim, out_dim, false,
              ctx->edge_flag, ctx->edge_hflag};
  Operands ops(dtype);
  GroupPlan plan = plan_group(dtype, dx ? GP_DX : GP_DA, n, groups, out_dim, in_dim, da != nullptr);
  if (n > 0) {
    ops.add(&g.dy, &g.lddy, n, out_dim);
    if (da) ops.add(&g.x, &g.ldx, n, in_dim);
    if (dx) ops.add_matrices(&g);
  }
  st = workspace(ctx, ops.bytes + plan.bytes() + 16 + (size_t)plan.partial_slots * out_dim * in_dim * 4);
  if (st != PBG_OK) return st;
  ops.place((char*)ctx->ops_ws);
  place_plan(&plan, (char*)ctx->ops_ws + ops.bytes, out_dim, in_dim);
  g.kd = ops.padded(in_dim);
  g.md = ops.padded(out_dim);
  g.a_group = (int64_t)out_dim * g.lda;
  ctx->edge_dirty = true;
  launch_group_plan(plan, offsets, groups, n, ctx->edge_flag, ctx->cs);
  launch_group_pack(dtype, ops.count, ops.op, offsets, groups, ctx->cs);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && dx) {
    g.out = dx;
    g.ldo = lddx;
    launch_group_product(g, dtype, GP_DX, plan, ctx->cs);
    e = hipGetLastError();
  }
  if (e == hipSuccess && da) {
    g.out = da;
    g.ldo = in_dim;
    launch_group_product(g, dtype, GP_DA, plan, ctx->cs);
    e = hipGetLastError();
  }
  return end_call(ctx, e, "pbg_group_linear_backward");
}

namespace {

pbg_status check_pref(pbg_ctx* ctx, int32_t dtype, const void* logits, int64_t ld, const int32_t* labels,
                      const int64_t* offsets, int32_t pairs, int64_t n, int32_t candidates) {
  if (dtype < PBG_TYPE_F32 || dtype > PBG_TYPE_F16) return set_err(ctx, PBG_ERR_INVALID_ARG, "unknown type %d", dtype);
  if (pairs < 1 || pairs > PBG_OPS_MAX_GROUPS / 2) return set_err(ctx, PBG_ERR_INVALID_ARG, "pairs out of range");
  if (n < 0 || n > (1ll << 32) / 256 - 1) return set_err(ctx, PBG_ERR_INVALID_ARG, "n out of range");
  if (candidates < 1 || candidates > PBG_OPS_MAX_LD)
    return set_err(ctx, PBG_ERR_INVALID_ARG, "candidates must be in [1, %d]", PBG_OPS_MAX_LD);
  if (bad_ld(ld, candidates))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "a row stride is below its width or above %d", PBG_OPS_MAX_LD);
  if (!offsets || !aligned(offsets, 8)) return set_err(ctx, PBG_ERR_INVALID_ARG, "NULL or misaligned offsets");
  if (n > 0 && (!logits || !labels)) return set_err(ctx, PBG_ERR_INVALID_ARG, "NULL array");
  if (!aligned(logits, type_bytes(dtype)) || !aligned(labels, 4))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "an array is not aligned to its elements");
  return PBG_OK;
}

}  // namespace

extern "C" pbg_status pbg_preference_loss(pbg_ctx* ctx, int32_t dtype, const void* logits, int64_t ld,
                                          const int32_t* labels, const int64_t* offsets, int32_t pairs, int64_t n,
                                          int32_t candidates, const float* ref_logp, float beta, float smoothing,
                                          float* loss, float* logp, float* dlogp, float* row_stats) {
  pbg_status st = begin_call(ctx, "pbg_preference_loss");
  if (st != PBG_OK) return st;
  st = check_pref(ctx, dtype, logits, ld, labels, offsets, pairs, n, candidates);
  if (st != PBG_OK) return st;
  if (!std::isfinite(beta)) return set_err(ctx, PBG_ERR_INVALID_ARG, "beta must be finite");
  if (!(smoothing >= 0.0f && smoothing < 1.0f)) return set_err(ctx, PBG_ERR_INVALID_ARG, "smoothing must be in [0, 1)");
  if (!logp || (n > 0 && !row_stats)) return set_err(ctx, PBG_ERR_INVALID_ARG, "NULL array");
  if (!aligned(ref_logp, 4) || !aligned(loss, 4) || !aligned(logp, 4) || !aligned(dlogp, 4) || !aligned(row_stats, 4))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "an array is not aligned to its elements");
  const int64_t Q = 2 * (int64_t)pairs;
  const Rows in[] = {{logits, n, candidates, ld, type_bytes(dtype)}, {labels, 1, n, n, 4}, {offsets, 1, Q + 1, Q + 1, 8},
                     {ref_logp, 1, Q, Q, 4}};
  const Rows out[] = {{loss, 1, pairs, pairs, 4}, {logp, 1, Q, Q, 4}, {dlogp, 1, Q, Q, 4}, {row_stats, 1, 2 * n, 2 * n, 4}};
  for (int i = 0; i < 4; ++i) {
    for (const Rows& r : in)
      if (overlap(out[i], r)) return set_err(ctx, PBG_ERR_INVALID_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return set_err(ctx, PBG_ERR_INVALID_ARG, "two outputs overlap");
  }
  st = ensure_edge_flags(ctx);
  const int splits = preference_splits(n, candidates);
  if (st == PBG_OK) st = workspace(ctx, (size_t)std::max<int64_t>(n, 1) * 8 * std::max(splits, 1));
  if (st != PBG_OK) return st;
  ctx->edge_dirty = true;
  PrefArgs p{};
  p.logits = logits;
  p.ld = ld;
  p.labels = labels;
  p.offsets = offsets;
  p.pairs = pairs;
  p.n = n;
  p.V = candidates;
  p.ref = ref_logp;
  p.beta = beta;
  p.smoothing = smoothing;
  p.loss = loss;
  p.logp = logp;
  p.dlogp = dlogp;
  p.stats = row_stats;
  p.picked = (double*)ctx->ops_ws;
  p.parts = (float2*)ctx->ops_ws;
  p.splits = splits;
  p.bad = ctx->edge_flag;
  p.host_bad = ctx->edge_hflag;
  launch_preference_loss(p, dtype, ctx->cs);
  return end_call(ctx, hipGetLastError(), "pbg_preference_loss");
}

extern "C" pbg_status pbg_preference_loss_backward(pbg_ctx* ctx, int32_t dtype, const void* logits, int64_t ld,
                                                   const int32_t* labels, const int64_t* offsets, int32_t pairs,
                                                   int64_t n, int32_t candidates, const float* row_stats,
                                                   const float* dlogp, void* dlogits, int64_t lddl) {
  pbg_status st = begin_call(ctx, "pbg_preference_loss_backward");
  if (st != PBG_OK) return st;
  st = check_pref(ctx, dtype, logits, ld, labels, offsets, pairs, n, candidates);
  if (st != PBG_OK) return st;
  const int es = type_bytes(dtype);
  if (bad_ld(lddl, candidates))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "a row stride is below its width or above %d", PBG_OPS_MAX_LD);
  if (!dlogp || (n > 0 && (!row_stats || !dlogits))) return set_err(ctx, PBG_ERR_INVALID_ARG, "NULL array");
  if (!aligned(row_stats, 4) || !aligned(dlogp, 4) || !aligned(dlogits, es))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "an array is not aligned to its elements");
  const int64_t Q = 2 * (int64_t)pairs;
  const Rows z{logits, n, candidates, ld, es}, dz{dlogits, n, candidates, lddl, es};
  if (!(dlogits == logits && lddl == ld) && overlap(dz, z))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "dlogits overlaps logits without being logits");
  const Rows in[] = {{labels, 1, n, n, 4}, {offsets, 1, Q + 1, Q + 1, 8}, {row_stats, 1, 2 * n, 2 * n, 4}, {dlogp, 1, Q, Q, 4}};
  for (const Rows& r : in)
    if (overlap(dz, r)) return set_err(ctx, PBG_ERR_INVALID_ARG, "an output overlaps an input");
  st = ensure_edge_flags(ctx);
  if (st != PBG_OK) return st;
  ctx->edge_dirty = true;
  PrefArgs p{};
  p.logits = logits;
  p.ld = ld;
  p.labels = labels;
  p.offsets = offsets;
  p.pairs = pairs;
  p.n = n;
  p.V = candidates;
  p.dlogp = const_cast<float*>(dlogp);
  p.stats = const_cast<float*>(row_stats);
  p.dlogits = dlogits;
  p.lddl = lddl;
  p.bad = ctx->edge_flag;
  p.host_bad = ctx->edge_hflag;
  p.splits = 1;
  launch_preference_backward(p, dtype, ctx->cs);
  return end_call(ctx, hipGetLastError(), "pbg_preference_loss_backward");
}

extern "C" pbg_status pbg_clip_gradients(pbg_ctx* ctx, int32_t num_tensors, const int32_t* dtypes_host,
                                         const int64_t* counts_host, const void* const* grads_host,
                                         void* const* outs_host, double max_norm, double* norm_host) {
  pbg_status st = begin_call(ctx, "pbg_clip_gradients");
  if (st != PBG_OK) return st;
  if (num_tensors < 0) return set_err(ctx, PBG_ERR_INVALID_ARG, "num_tensors must be >= 0");
  if (!(max_norm > 0.0)) return set_err(ctx, PBG_ERR_INVALID_ARG, "max_norm must be above 0");
  if (num_tensors > 0 && (!dtypes_host || !counts_host || !grads_host))
    return set_err(ctx, PBG_ERR_INVALID_ARG, "NULL array");
  constexpr int64_t kMaxValues = 1ll << 38;   // of all tensors together, more than the memory holds
  try {
    struct Range {
      uintptr_t begin, end;
      bool out;
    };
    std::vector<Range> ranges;
    std::vector<ClipBatch> batches;
    ranges.reserve((size_t)num_tensors * 2);
    int64_t blocks = 0, values = 0;
    for (int32_t i = 0; i < num_tensors; ++i) {
      if (counts_host[i] < 0 || counts_host[i] > kMaxValues - values)
        return set_err(ctx, PBG_ERR_INVALID_ARG, "count %d out of range", i);
      values += counts_host[i];
    }
    // one workgroup's sum adds all parts: at most about 16,384 of them (75,700 parts of 8,192 values took it 24 us)
    int64_t span = kClipBlock;
    while (values / span > 16384) span *= 2;
    for (int32_t i = 0; i < num_tensors; ++i) {
      const int64_t c = counts_host[i];
      const int32_t ty = dtypes_host[i];
      if (ty < PBG_TYPE_F32 || ty > PBG_TYPE_F16) return set_err(ctx, PBG_ERR_INVALID_ARG, "unknown type %d", ty);
      if (c == 0) continue;
      const int es = type_bytes(ty);
      const void* g = grads_host[i];
      void* o = outs_host ? outs_host[i] : const_cast<void*>(g);
      if (!g || !o) return set_err(ctx, PBG_ERR_INVALID_ARG, "tensor %d is NULL", i);
      if (!aligned(g, es) || !aligned(o, es))
        return set_err(ctx, PBG_ERR_INVALID_ARG, "tensor %d is not aligned to its elements", i);
      ranges.push_back({(uintptr_t)o, (uintptr_t)o + (size_t)c * es, true});
      if (o != g) ranges.push_back({(uintptr_t)g, (uintptr_t)g + (size_t)c * es, false});
      const int64_t nb = (c + span - 1) / span;
      if (batches.empty() || batches.back().n == kClipBatch || batches.back().first[batches.back().n] + nb > (1 << 24) - 1) {
        batches.emplace_back();
        batches.back().n = 0;
        batches.back().span = span;
        batches.back().first[0] = 0;
      }
      ClipBatch& b = batches.back();
      b.g[b.n] = g;
      b.o[b.n] = o;
      b.count[b.n] = c;
      b.type[b.n] = (uint8_t)ty;
      b.first[b.n + 1] = b.first[b.n] + (uint32_t)nb;
      ++b.n;
      blocks += nb;
    }
    // no written range may meet another range
    std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    uintptr_t out_end = 0, any_end = 0;
    for (const Range& r : ranges) {
      if (r.begin < out_end || (r.out && r.begin < any_end))
        return set_err(ctx, PBG_ERR_INVALID_ARG, "an output overlaps another tensor");
      any_end = std::max(any_end, r.end);
      if (r.out) out_end = std::max(out_end, r.end);
    }
    if (!ctx->ops_host && hipHostMalloc((void**)&ctx->ops_host, 64) != hipSuccess) {
      (void)hipGetLastError();
      ctx->ops_host = nullptr;
      return set_err(ctx, PBG_ERR_OUT_OF_MEMORY, "page-locked memory allocation failed");
    }
    st = workspace(ctx, (size_t)(blocks + 1) * 8);
    if (st != PBG_OK) return st;
    double* scale = (double*)ctx->ops_ws;
    launch_clip(batches.data(), (int)batches.size(), blocks, max_norm, scale, scale + 1, ctx->ops_host, ctx->cs);
    hipError_t e = hipGetLastError();
    const hipError_t es = hipStreamSynchronize(ctx->cs);
    if (e == hipSuccess) e = es;
    if (e != hipSuccess) return hip_fail(ctx, e, "pbg_clip_gradients");
    if (norm_host) *norm_host = *(volatile double*)ctx->ops_host;
    return PBG_OK;
  } catch (const std::bad_alloc&) {
    return set_err(ctx, PBG_ERR_OUT_OF_MEMORY, "host memory for the tensors' descriptors");
  }
}
