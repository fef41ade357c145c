// Host side of the EasySpec C ABI (include/easyspec.h): argument checks, the per-sequence
// precise / fuzzy length state machine, weight repacking, and the launch sequence of one
// forward pass.  All arithmetic of the method runs in the kernels of the .hip files.
#include "../../include/easyspec.h"
#include "../../include/easyspec_instrument.h"

#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <unistd.h>

#include <algorithm>
#include <initializer_list>
#include <string>
#include <vector>

#include "kernels.h"
#include "tile_index.hpp"

using namespace es;

struct easyspec_ctx {
  easyspec_config cfg;
  Shape s;
  Buffers b;
  Buffers b2;      // a second set of per-pass workspaces (same weights and caches): the second of two passes run together
  bool has_b2;
  WideBuffers w;   // wide passes (bf16 models whose calibrations can exceed one pass); w.cols == 0: none
  Resident r;      // small models: whole passes in one launch; r.ctl == null: separate launches
  const float* last_H;  // residual rows of the most recent pass
  hipStream_t stream;
  bool weights_loaded;
  std::vector<int32_t> precise, fuzzy;
  // token tree of each sequence (nodes = its fuzzy slots, node t in slot precise + t)
  struct Tree {
    int32_t n = 0;
    int32_t depth[EASYSPEC_MAX_TREE_NODES];
    uint64_t line[EASYSPEC_MAX_TREE_NODES];  // bit a set: node a is the node itself or an ancestor
  };
  std::vector<Tree> tree;
  // bounded caches: what easyspec_track_attention allocated (weights == null: nothing is tracked)
  struct Tracked {
    float* weights = nullptr;   // [L][B][Hkv][max_ctx]
    int32_t* kept = nullptr;    // the same shape: an eviction's list of slots
    float2* stats = nullptr;    // workspace of launch_weigh
    size_t stats_bytes = 0;
    int32_t max_positions = 0;  // rows of the rotary table
    std::vector<int32_t> gone;  // slots evicted so far: slot s of sequence b is at rotary position s + gone[b] from firm[b] on;
    std::vector<int32_t> firm;  // the slots below come from anywhere before
  } track;
  std::vector<int32_t> bounds;  // current layer-parallel strategy
  std::vector<int32_t> single;  // every layer alone (Alg. 1 order)
  std::vector<void*> allocs;
  std::vector<std::pair<void*, size_t>> work;  // the per-pass workspaces (easyspec_poison_workspaces)
  int32_t deny_alloc = -1;  // allocations from here to the one that asks for too much (easyspec_deny_allocation); -1: none does
  int32_t last_rows;
  int32_t parallel_mode;  // EASYSPEC_PARALLEL_*
  // per-kernel timing (easyspec_profile_*)
  int32_t prof_op;
  std::vector<hipEvent_t> prof_ev;  // start/stop pairs
  std::vector<int8_t> prof_op_of;   // kernel class of the launch that took pair i
  LaunchTimer timer;                // the pairs handed to the launches of the profiled kernel class
  std::string err;
};

static thread_local std::string g_err;
thread_local es::LaunchTimer* es::g_launch_timer = nullptr;

static int fail(easyspec_ctx* ctx, int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  if (ctx) ctx->err = buf;
  else g_err = buf;
  return code;
}

#define HIPCHK(ctx, call)                                                                           \
  do {                                                                                              \
    hipError_t e_ = (call);                                                                         \
    if (e_ != hipSuccess) return fail(ctx, EASYSPEC_EHIP, "%s: %s", #call, hipGetErrorString(e_)); \
  } while (0)

// A resident pass that gave up waiting (resident.hip) left wrong results and cache entries behind and lengths that count them:
// every entry point that uses or hands out that state looks here first, those that synchronise once more afterwards.
static int check_passes(const easyspec_ctx* ctx) {
  if (!ctx->r.failed || !*(volatile uint32_t*)ctx->r.failed) return EASYSPEC_OK;
  return fail(const_cast<easyspec_ctx*>(ctx), EASYSPEC_EHIP, "a forward pass of this context gave up waiting for its own values; its results and cache are void: destroy the context");
}
#define CHECK_PASSES(ctx)                                      \
  do {                                                         \
    const int rc_ = check_passes(ctx);                         \
    if (rc_ != EASYSPEC_OK) return rc_;                        \
  } while (0)

static size_t esize(const Shape& s) { return s.dtype == EASYSPEC_DTYPE_BF16 ? 2 : 4; }
static size_t packed_bytes(const Shape& s, int rows, int K, int R = 16) { return es::packed_bytes(s.dtype, rows, K, R); }

static int dev_alloc(easyspec_ctx* ctx, void** p, size_t bytes) {
  *p = nullptr;
  if (bytes == 0) bytes = 16;
  if (ctx->deny_alloc >= 0 && ctx->deny_alloc-- == 0) bytes = (size_t)1 << 60;
  HIPCHK(ctx, hipMalloc(p, bytes));
  ctx->allocs.push_back(*p);
  return EASYSPEC_OK;
}

#define ALLOC(ctx, ptr, bytes)                                       \
  do {                                                               \
    int rc_ = dev_alloc(ctx, (void**)&(ptr), (size_t)(bytes));       \
    if (rc_ != EASYSPEC_OK) return rc_;                              \
  } while (0)
// a workspace that every forward pass writes before it reads it
#define ALLOC_WORK(ctx, ptr, bytes)                                  \
  do {                                                               \
    ALLOC(ctx, ptr, bytes);                                          \
    (ctx)->work.emplace_back((void*)(ptr), (size_t)(bytes));         \
  } while (0)

static int check_config(const easyspec_config* c) {
  if (!c) return fail(nullptr, EASYSPEC_EINVAL, "config is NULL");
  if (c->n_layers < 1 || c->d_model < 32 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->d_ffn < 32 || c->vocab < 1)
    return fail(nullptr, EASYSPEC_EINVAL, "non-positive model dimension");
  if (c->dtype != EASYSPEC_DTYPE_F32 && c->dtype != EASYSPEC_DTYPE_BF16) return fail(nullptr, EASYSPEC_EINVAL, "unknown dtype %d", c->dtype);
  if (c->head_dim != 64 && c->head_dim != 128) return fail(nullptr, EASYSPEC_EINVAL, "head_dim must be 64 or 128, got %d", c->head_dim);
  if (c->d_model % 32 || c->d_ffn % 32 || (c->n_q_heads * c->head_dim) % 32)
    return fail(nullptr, EASYSPEC_EINVAL, "d_model, d_ffn and n_q_heads*head_dim must be multiples of 32");
  if (c->n_q_heads % c->n_kv_heads) return fail(nullptr, EASYSPEC_EINVAL, "n_q_heads must be a multiple of n_kv_heads");
  const int g = c->n_q_heads / c->n_kv_heads;
  if (g != 1 && g != 2 && g != 4 && g != 7 && g != 8)
    return fail(nullptr, EASYSPEC_EINVAL, "n_q_heads/n_kv_heads = %d is not one of 1, 2, 4, 7, 8", g);
  if (c->max_batch < 1 || c->max_batch > EASYSPEC_MAX_BATCH) return fail(nullptr, EASYSPEC_EINVAL, "max_batch must be 1..%d", EASYSPEC_MAX_BATCH);
  if (c->max_calib_tokens < 1 || c->max_calib_tokens > EASYSPEC_MAX_CALIB_TOKENS)
    return fail(nullptr, EASYSPEC_EINVAL, "max_calib_tokens must be 1..%d", EASYSPEC_MAX_CALIB_TOKENS);
  if (c->max_ctx < 1 || c->max_ctx > kMaxChunks * 1024) return fail(nullptr, EASYSPEC_EINVAL, "max_ctx must be 1..%d", kMaxChunks * 1024);
  if (!(c->rms_eps >= 0.f) || !(c->rope_theta > 0.f)) return fail(nullptr, EASYSPEC_EINVAL, "bad rms_eps or rope_theta");
  return EASYSPEC_OK;
}

static void shape_of(const easyspec_config* cfg, Shape& s) {
  memset(&s, 0, sizeof s);
  s.dtype = cfg->dtype; s.L = cfg->n_layers; s.d = cfg->d_model; s.Hq = cfg->n_q_heads; s.Hkv = cfg->n_kv_heads;
  s.hd = cfg->head_dim; s.F = cfg->d_ffn; s.V = cfg->vocab; s.HQ = s.Hq * s.hd; s.RQKV = (s.Hq + 2 * s.Hkv) * s.hd;
  s.B = cfg->max_batch; s.max_ctx = cfg->max_ctx; s.eps = cfg->rms_eps; s.has_bias = cfg->qkv_bias ? 1 : 0;
  s.R_ffn = tile_rows(s.F);
  s.R_qkv = qkv_tile_rows(s.RQKV / 2);
}

// rotary table in double precision: angle(pos, i) = pos * theta^(-2 i / hd), a few thousand positions at a time
static hipError_t fill_rope(const easyspec_config& cfg, float2* rope, int n_pos) {
  const int half = cfg.head_dim / 2, most = std::min(n_pos, 4096);
  std::vector<float2> tab((size_t)most * half);
  std::vector<double> freq(half);
  for (int i = 0; i < half; ++i) freq[i] = pow((double)cfg.rope_theta, -2.0 * (double)i / (double)cfg.head_dim);
  for (int p0 = 0; p0 < n_pos; p0 += most) {
    const int n = std::min(most, n_pos - p0);
    for (int p = 0; p < n; ++p)
      for (int i = 0; i < half; ++i) {
        const double ang = (double)(p0 + p) * freq[i];
        tab[(size_t)p * half + i] = make_float2((float)cos(ang), (float)sin(ang));
      }
    const hipError_t e = hipMemcpy(rope + (size_t)p0 * half, tab.data(), (size_t)n * half * sizeof(float2), hipMemcpyHostToDevice);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

extern "C" int easyspec_create(const easyspec_config* cfg, void* hip_stream, easyspec_ctx** out) {
  if (!out) return fail(nullptr, EASYSPEC_EINVAL, "out is NULL");
  *out = nullptr;
  int rc = check_config(cfg);
  if (rc != EASYSPEC_OK) return rc;
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1)
    return fail(nullptr, EASYSPEC_EHIP, "no HIP device available (this library has no CPU path)");

  easyspec_ctx* ctx = new easyspec_ctx();
  ctx->cfg = *cfg;
  ctx->stream = (hipStream_t)hip_stream;
  ctx->weights_loaded = false;
  ctx->last_rows = 0;
  ctx->last_H = nullptr;
  ctx->has_b2 = false;
  memset(&ctx->w, 0, sizeof ctx->w);
  memset(&ctx->r, 0, sizeof ctx->r);
  ctx->prof_op = -1;
  ctx->timer = LaunchTimer{nullptr, nullptr, 0, 0, 0};
  ctx->parallel_mode = EASYSPEC_PARALLEL_ATTENTION;
  Shape& s = ctx->s;
  shape_of(cfg, s);
  ctx->precise.assign(s.B, 0);
  ctx->fuzzy.assign(s.B, 0);
  ctx->tree.assign(s.B, easyspec_ctx::Tree());
  ctx->track.max_positions = s.max_ctx;
  ctx->track.gone.assign(s.B, 0);
  ctx->track.firm.assign(s.B, 0);
  for (int i = 0; i <= s.L; ++i) ctx->single.push_back(i);
  ctx->bounds = ctx->single;

  auto body = [&]() -> int {
    Buffers& b = ctx->b;
    memset(&b, 0, sizeof b);
    const size_t es_ = esize(s);
    const size_t act_ = es_ * (s.dtype == EASYSPEC_DTYPE_BF16 ? 2 : 1);  // bf16 activations: hi and lo arrays
    ALLOC(ctx, b.wqkv, (size_t)s.L * 2 * packed_bytes(s, s.RQKV / 2, s.d, s.R_qkv));
    ALLOC(ctx, b.wo, (size_t)s.L * packed_bytes(s, s.d, s.HQ));
    ALLOC(ctx, b.wg, (size_t)s.L * packed_bytes(s, s.F, s.d, s.R_ffn));
    ALLOC(ctx, b.wu, (size_t)s.L * packed_bytes(s, s.F, s.d, s.R_ffn));
    ALLOC(ctx, b.wd, (size_t)s.L * packed_bytes(s, s.d, s.F));
    ALLOC(ctx, b.wlm, packed_bytes(s, s.V, s.d));
    ALLOC(ctx, b.embed, (size_t)s.V * s.d * es_);
    if (s.has_bias) ALLOC(ctx, b.bqkv, (size_t)s.L * s.RQKV * sizeof(float));
    ALLOC(ctx, b.g_attn, (size_t)s.L * s.d * sizeof(float));
    ALLOC(ctx, b.g_mlp, (size_t)s.L * s.d * sizeof(float));
    ALLOC(ctx, b.g_final, (size_t)s.d * sizeof(float));
    ALLOC(ctx, b.rope, (size_t)s.max_ctx * (s.hd / 2) * sizeof(float2));
    const size_t kv_bytes = (size_t)s.L * s.B * s.Hkv * s.max_ctx * s.hd * es_;
    ALLOC(ctx, b.kc, kv_bytes);
    ALLOC(ctx, b.vc, kv_bytes);
    ALLOC_WORK(ctx, b.H, (size_t)kMaxCols * s.d * sizeof(float));
    ALLOC_WORK(ctx, b.ssp, (size_t)kMaxCols * (s.d / 16) * sizeof(float));
    ALLOC_WORK(ctx, b.XA, (size_t)EASYSPEC_MAX_SET * kMaxCols * s.d * act_);
    ALLOC_WORK(ctx, b.ssp_set, (size_t)EASYSPEC_MAX_SET * kMaxCols * (s.d / 16) * sizeof(float));
    ALLOC_WORK(ctx, b.XM, (size_t)EASYSPEC_MAX_SET * kMaxCols * s.d * act_);
    ALLOC_WORK(ctx, b.Q, (size_t)EASYSPEC_MAX_SET * kMaxCols * s.HQ * sizeof(float));
    ALLOC_WORK(ctx, b.AO, (size_t)EASYSPEC_MAX_SET * kMaxCols * s.HQ * act_);
    ALLOC_WORK(ctx, b.A, (size_t)EASYSPEC_MAX_SET * kMaxCols * s.d * sizeof(float));
    ALLOC_WORK(ctx, b.ACT, (size_t)EASYSPEC_MAX_SET * kMaxCols * s.F * act_);
    const size_t prow = (size_t)EASYSPEC_MAX_SET * kMaxCols * s.Hq;
    ALLOC_WORK(ctx, b.PO, prow * kMaxChunks * s.hd * sizeof(float));
    ALLOC_WORK(ctx, b.PM, prow * kMaxChunks * sizeof(float));
    ALLOC_WORK(ctx, b.PL, prow * kMaxChunks * sizeof(float));
    const size_t nblk = (size_t)(s.V + 15) / 16;
    ALLOC_WORK(ctx, b.amax_val, kMaxCols * nblk * sizeof(float));
    ALLOC_WORK(ctx, b.amax_idx, kMaxCols * nblk * sizeof(int32_t));
    // A calibration of more columns than one pass holds runs its passes two at a time (the weight kernels serve
    // both from one read of the weights): the second pass of a pair works in a workspace set of its own.  bf16 models
    // run such a calibration as one wide pass and get that set only where pairs are asked for (tests).
    const bool many = (long)s.B * cfg->max_calib_tokens > kMaxCols;
    const char* pair_env = getenv("EASYSPEC_PAIR_PASSES");
    Buffers& b2 = ctx->b2;
    b2 = b;
    ctx->has_b2 = many && (s.dtype != EASYSPEC_DTYPE_BF16 || (pair_env && atoi(pair_env) != 0));
    if (ctx->has_b2) {
      ALLOC_WORK(ctx, b2.H, (size_t)kMaxCols * s.d * sizeof(float));
      ALLOC_WORK(ctx, b2.ssp, (size_t)kMaxCols * (s.d / 16) * sizeof(float));
      ALLOC_WORK(ctx, b2.XA, (size_t)kMaxCols * s.d * act_);
      ALLOC_WORK(ctx, b2.XM, (size_t)kMaxCols * s.d * act_);
      ALLOC_WORK(ctx, b2.Q, (size_t)kMaxCols * s.HQ * sizeof(float));
      ALLOC_WORK(ctx, b2.AO, (size_t)kMaxCols * s.HQ * act_);
      ALLOC_WORK(ctx, b2.A, (size_t)kMaxCols * s.d * sizeof(float));
      ALLOC_WORK(ctx, b2.ACT, (size_t)kMaxCols * s.F * act_);
      const size_t prow2 = (size_t)kMaxCols * s.Hq;  // calibrations go layer by layer: one layer's worth of each
      ALLOC_WORK(ctx, b2.PO, prow2 * kMaxChunks * s.hd * sizeof(float));
      ALLOC_WORK(ctx, b2.PM, prow2 * kMaxChunks * sizeof(float));
      ALLOC_WORK(ctx, b2.PL, prow2 * kMaxChunks * sizeof(float));
      ALLOC_WORK(ctx, b2.amax_val, kMaxCols * nblk * sizeof(float));
      ALLOC_WORK(ctx, b2.amax_idx, kMaxCols * nblk * sizeof(int32_t));
      b2.ssp_set = nullptr;  // full-layer mode never runs two passes together
    }
    WideBuffers& w = ctx->w;
    if (many && s.dtype == EASYSPEC_DTYPE_BF16) {
      w.cols = std::min((s.B * cfg->max_calib_tokens + 15) / 16 * 16, kWideCols);
      ALLOC_WORK(ctx, w.H, (size_t)w.cols * s.d * sizeof(float));
      ALLOC_WORK(ctx, w.rs, (size_t)w.cols * sizeof(float));
      ALLOC_WORK(ctx, w.X, wide_operand_bytes(w.cols, s.d));
      ALLOC_WORK(ctx, w.Q, (size_t)w.cols * s.HQ * sizeof(float));
      ALLOC_WORK(ctx, w.AO, wide_operand_bytes(w.cols, s.HQ));
      ALLOC_WORK(ctx, w.ACT, wide_operand_bytes(w.cols, s.F));
      ALLOC_WORK(ctx, w.P, wide_partial_bytes(s));
    }
    if (s.dtype == EASYSPEC_DTYPE_BF16) HIPCHK(ctx, weight_kernels_prepare());
    if (resident_model(s)) {
      Resident& r = ctx->r;
      ALLOC(ctx, r.ctl, sizeof(ResidentCtl));
      ALLOC_WORK(ctx, r.granules, resident_granule_bytes(s));
      HIPCHK(ctx, hipHostMalloc((void**)&r.failed, sizeof(uint32_t), hipHostMallocDefault));
      *r.failed = 0;
      ResidentCtl ctl;
      memset(&ctl, 0, sizeof ctl);
      ctl.epoch = 1;  // cleared granules are of no pass
      HIPCHK(ctx, hipMemcpy(r.ctl, &ctl, sizeof ctl, hipMemcpyHostToDevice));
      HIPCHK(ctx, hipMemsetAsync(r.granules, 0, resident_granule_bytes(s), ctx->stream));
      HIPCHK(ctx, resident_prepare(s));
    }
    HIPCHK(ctx, hipMemsetAsync(b.kc, 0, kv_bytes, ctx->stream));
    HIPCHK(ctx, hipMemsetAsync(b.vc, 0, kv_bytes, ctx->stream));

    HIPCHK(ctx, fill_rope(ctx->cfg, b.rope, s.max_ctx));
    HIPCHK(ctx, hipStreamSynchronize(ctx->stream));
    return EASYSPEC_OK;
  };
  rc = body();
  if (rc != EASYSPEC_OK) {
    g_err = ctx->err;
    for (void* p : ctx->allocs) (void)hipFree(p);
    if (ctx->r.failed) (void)hipHostFree(ctx->r.failed);
    delete ctx;
    return rc;
  }
  *out = ctx;
  return EASYSPEC_OK;
}

extern "C" void easyspec_destroy(easyspec_ctx* ctx) {
  if (!ctx) return;
  (void)hipStreamSynchronize(ctx->stream);
  for (hipEvent_t e : ctx->prof_ev) (void)hipEventDestroy(e);
  for (void* p : ctx->allocs) (void)hipFree(p);
  if (ctx->r.failed) (void)hipHostFree(ctx->r.failed);
  delete ctx;
}

extern "C" const char* easyspec_last_error(const easyspec_ctx* ctx) { return ctx ? ctx->err.c_str() : g_err.c_str(); }

// ---------------------------------------------------------------------------------------------
// weights
// ---------------------------------------------------------------------------------------------

extern "C" int easyspec_load_weights(easyspec_ctx* ctx, const easyspec_weights* w) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  if (!w || !w->layers || !w->embed || !w->lm_head || !w->g_final) return fail(ctx, EASYSPEC_EINVAL, "weights: NULL pointer");
  const Shape& s = ctx->s;
  for (int l = 0; l < s.L; ++l) {
    const easyspec_layer_weights& lw = w->layers[l];
    if (!lw.wq || !lw.wk || !lw.wv || !lw.wo || !lw.wg || !lw.wu || !lw.wd || !lw.g_attn || !lw.g_mlp)
      return fail(ctx, EASYSPEC_EINVAL, "weights: NULL pointer in layer %d", l);
    if (s.has_bias && (!lw.bq || !lw.bk || !lw.bv)) return fail(ctx, EASYSPEC_EINVAL, "weights: missing bias in layer %d", l);
  }
  const size_t es_ = esize(s);
  const Buffers& b = ctx->b;
  // staging for one row-major matrix (largest: LM head, gate/up, or stacked QKV)
  size_t stage_elems = (size_t)s.V * s.d;
  if ((size_t)s.F * s.d > stage_elems) stage_elems = (size_t)s.F * s.d;
  if ((size_t)s.RQKV * s.d > stage_elems) stage_elems = (size_t)s.RQKV * s.d;
  void* stage = nullptr;
  HIPCHK(ctx, hipMalloc(&stage, stage_elems * es_));
  auto body = [&]() -> int {
    hipStream_t st = ctx->stream;
    auto put = [&](const void* src, size_t elems, size_t off_elems) -> hipError_t {
      return hipMemcpyAsync((char*)stage + off_elems * es_, src, elems * es_, hipMemcpyDefault, st);
    };
    auto pack = [&](void* dst_base, size_t layer, int rows, int K, int R = 16) -> hipError_t {
      launch_repack(s.dtype, stage, (char*)dst_base + layer * packed_bytes(s, rows, K, R), rows, K, R, 0, 0, st);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      return hipStreamSynchronize(st);  // staging is reused
    };
    // stacked [Wq; Wk; Wv]: the first halves of all heads, then the second halves (the rotation pairs)
    auto pack_qkv = [&](size_t layer) -> hipError_t {
      const size_t half_bytes = packed_bytes(s, s.RQKV / 2, s.d, s.R_qkv);
      char* dst = (char*)b.wqkv + layer * 2 * half_bytes;
      launch_repack(s.dtype, stage, dst, s.RQKV / 2, s.d, s.R_qkv, s.hd / 2, 0, st);
      launch_repack(s.dtype, stage, dst + half_bytes, s.RQKV / 2, s.d, s.R_qkv, s.hd / 2, s.hd / 2, st);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      return hipStreamSynchronize(st);
    };
    for (int l = 0; l < s.L; ++l) {
      const easyspec_layer_weights& lw = w->layers[l];
      HIPCHK(ctx, put(lw.wq, (size_t)s.HQ * s.d, 0));
      HIPCHK(ctx, put(lw.wk, (size_t)s.Hkv * s.hd * s.d, (size_t)s.HQ * s.d));
      HIPCHK(ctx, put(lw.wv, (size_t)s.Hkv * s.hd * s.d, (size_t)(s.HQ + s.Hkv * s.hd) * s.d));
      HIPCHK(ctx, pack_qkv(l));
      HIPCHK(ctx, put(lw.wo, (size_t)s.d * s.HQ, 0));
      HIPCHK(ctx, pack(b.wo, l, s.d, s.HQ));
      HIPCHK(ctx, put(lw.wg, (size_t)s.F * s.d, 0));
      HIPCHK(ctx, pack(b.wg, l, s.F, s.d, s.R_ffn));
      HIPCHK(ctx, put(lw.wu, (size_t)s.F * s.d, 0));
      HIPCHK(ctx, pack(b.wu, l, s.F, s.d, s.R_ffn));
      HIPCHK(ctx, put(lw.wd, (size_t)s.d * s.F, 0));
      HIPCHK(ctx, pack(b.wd, l, s.d, s.F));
      if (s.has_bias) {
        float* dst = b.bqkv + (size_t)l * s.RQKV;
        HIPCHK(ctx, hipMemcpyAsync(dst, lw.bq, (size_t)s.HQ * 4, hipMemcpyDefault, st));
        HIPCHK(ctx, hipMemcpyAsync(dst + s.HQ, lw.bk, (size_t)s.Hkv * s.hd * 4, hipMemcpyDefault, st));
        HIPCHK(ctx, hipMemcpyAsync(dst + s.HQ + s.Hkv * s.hd, lw.bv, (size_t)s.Hkv * s.hd * 4, hipMemcpyDefault, st));
      }
      HIPCHK(ctx, hipMemcpyAsync(b.g_attn + (size_t)l * s.d, lw.g_attn, (size_t)s.d * 4, hipMemcpyDefault, st));
      HIPCHK(ctx, hipMemcpyAsync(b.g_mlp + (size_t)l * s.d, lw.g_mlp, (size_t)s.d * 4, hipMemcpyDefault, st));
    }
    HIPCHK(ctx, put(w->lm_head, (size_t)s.V * s.d, 0));
    HIPCHK(ctx, pack(b.wlm, 0, s.V, s.d));
    HIPCHK(ctx, hipMemcpyAsync(b.embed, w->embed, (size_t)s.V * s.d * es_, hipMemcpyDefault, st));
    HIPCHK(ctx, hipMemcpyAsync(b.g_final, w->g_final, (size_t)s.d * 4, hipMemcpyDefault, st));
    HIPCHK(ctx, hipStreamSynchronize(st));
    return EASYSPEC_OK;
  };
  const int rc = body();
  (void)hipFree(stage);
  if (rc == EASYSPEC_OK) ctx->weights_loaded = true;
  return rc;
}

// ---------------------------------------------------------------------------------------------
// layer-parallel strategy
// ---------------------------------------------------------------------------------------------

extern "C" int easyspec_default_groups(int32_t L, int32_t N, int32_t policy, int32_t* bounds, int32_t* n_sets) {
  if (L < 1 || N < 1 || !bounds || !n_sets) return fail(nullptr, EASYSPEC_EINVAL, "default_groups: bad arguments");
  if (policy != EASYSPEC_POLICY_ALIGNED && policy != EASYSPEC_POLICY_PACKED) return fail(nullptr, EASYSPEC_EINVAL, "default_groups: unknown policy %d", policy);
  std::vector<int32_t> b;
  b.push_back(0);
  if (L >= 2) {
    // layers 1 .. L-2 are cut into N-sets; layer 0 and layer L-1 stay alone
    const int32_t stop = L - 1;
    int32_t lo = 1;
    b.push_back(lo);
    while (lo < stop) {
      int32_t hi = policy == EASYSPEC_POLICY_ALIGNED ? (lo / N + 1) * N : lo + N;
      if (hi > stop) hi = stop;
      b.push_back(hi);
      lo = hi;
    }
  }
  b.push_back(L);
  for (size_t i = 0; i < b.size(); ++i) bounds[i] = b[i];
  *n_sets = (int32_t)b.size() - 1;
  return EASYSPEC_OK;
}

extern "C" int easyspec_set_groups(easyspec_ctx* ctx, const int32_t* bounds, int32_t n_sets) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  if (!bounds || n_sets < 1 || n_sets > ctx->s.L) return fail(ctx, EASYSPEC_EINVAL, "set_groups: bad n_sets");
  if (bounds[0] != 0 || bounds[n_sets] != ctx->s.L) return fail(ctx, EASYSPEC_EINVAL, "set_groups: bounds must run from 0 to n_layers");
  for (int j = 0; j < n_sets; ++j) {
    const int k = bounds[j + 1] - bounds[j];
    if (k < 1) return fail(ctx, EASYSPEC_EINVAL, "set_groups: bounds must increase");
    if (k > EASYSPEC_MAX_SET) return fail(ctx, EASYSPEC_EINVAL, "set_groups: set of %d layers exceeds %d", k, EASYSPEC_MAX_SET);
  }
  ctx->bounds.assign(bounds, bounds + n_sets + 1);
  return EASYSPEC_OK;
}

// ---------------------------------------------------------------------------------------------
// one forward pass over the columns `c` (launch sequence of Alg. 1 / Alg. 2)
// ---------------------------------------------------------------------------------------------

// While profiling is on, the launches of one kernel class made inside the scope take event pairs.
struct ProfScope {
  ProfScope(easyspec_ctx* c, int op) {
    g_launch_timer = (c->prof_op == op || c->prof_op == EASYSPEC_OP_ALL) ? &c->timer : nullptr;
    c->timer.cur_op = op;
  }
  ~ProfScope() { g_launch_timer = nullptr; }
};

// Do the switches that force a kernel or the cut of a launch leave room for a resident pass, which has neither?
static bool launches_forced() {
  for (char** e = environ; e && *e; ++e) {
    if (strncmp(*e, "EASYSPEC_", 9) != 0) continue;
    const char* v = *e + 9;
    if (strcmp(v, "RESIDENT=0") == 0) return true;
    if (strcmp(v, "ATTN_MFMA=1") == 0) continue;  // what it is without the switch
    for (const char* p : {"ATTN_", "NW_", "TILE_ROWS", "QKV_TILE_ROWS", "PAIR_"})
      if (strncmp(v, p, strlen(p)) == 0) return true;
  }
  return false;
}

// Does this pass run in one launch (resident.hip)?  Not while launches are timed one by one.
static bool resident_takes(const easyspec_ctx* ctx, const Cols& c, const std::vector<int32_t>& bounds) {
  return ctx->r.ctl && ctx->prof_op < 0 && resident_pass(ctx->s, c, bounds.data(), (int)bounds.size() - 1) && !launches_forced();
}

static float weigh_scale(int hd) { return (float)(1.4426950408889634 / sqrt((double)hd)); }

// The entries of a calibration's columns (those of a sequence lie together) and of a wide pass's, for launch_weigh; false: the
// workspace is too small for them.
static void weigh_begin(const easyspec_ctx* ctx, const float* q, WeighArgs& a) {
  const Shape& s = ctx->s;
  memset(&a, 0, sizeof a);
  a.q = q;
  a.stats = ctx->track.stats;
  a.n_seqs = s.B; a.heads = s.Hkv; a.Hq = s.Hq; a.group = s.Hq / s.Hkv; a.max_slots = s.max_ctx;
  a.scale = weigh_scale(s.hd);
}
static bool weigh_columns(const easyspec_ctx* ctx, const Cols& c, const float* q, WeighArgs& a) {
  const Shape& s = ctx->s;
  weigh_begin(ctx, q, a);
  for (int i = 0; i < c.n; ++i) {
    if (i == 0 || c.seq[i] != c.seq[i - 1]) {
      WeighEntry& e = a.entry[a.n_entries++];
      e.seq = c.seq[i];
      e.q_first = i;
    }
    WeighEntry& e = a.entry[a.n_entries - 1];
    e.n += 1;
    e.len = c.pos[i] + 1;
  }
  weigh_plan(a, 1, s.dtype);
  return weigh_workspace_bytes(a, 1) <= ctx->track.stats_bytes;
}
static bool weigh_spans(const easyspec_ctx* ctx, const Spans& sp, const float* q, WeighArgs& a) {
  const Shape& s = ctx->s;
  weigh_begin(ctx, q, a);
  for (int i = 0; i < sp.n_seq; ++i) {
    WeighEntry& e = a.entry[a.n_entries++];
    e.seq = sp.seq[i];
    e.q_first = sp.first[i];
    e.n = sp.first[i + 1] - sp.first[i];
    e.len = sp.pos0[i] + e.n;
  }
  weigh_plan(a, 1, s.dtype);
  return weigh_workspace_bytes(a, 1) <= ctx->track.stats_bytes;
}
static void weigh_layer(const easyspec_ctx* ctx, WeighArgs& a, int layer) {
  const Shape& s = ctx->s;
  const size_t slots = (size_t)layer * s.B * s.Hkv * s.max_ctx;
  a.k = (const char*)ctx->b.kc + slots * s.hd * esize(s);
  a.w_out = ctx->track.weights + slots;
  a.w_in = a.w_out;
  launch_weigh(a, 1, s.dtype, s.hd, ctx->stream);
}

// c2: a second pass of as many columns run together with the first (sets of one layer only: a calibration); the
// weight kernels then serve both passes in one launch each, embedding, attention and argmax run per pass.
// weigh: the attention weights of the pass's queries are added to the context's (a calibration of a context that tracks them).
static int forward(easyspec_ctx* ctx, const Cols& c, const int32_t* tokens, const std::vector<int32_t>& bounds,
                   bool full_layer, float* logits_out, int32_t* tokens_out, const Cols* c2 = nullptr, bool weigh = false) {
  const Shape& s = ctx->s;
  const Buffers& b = ctx->b;
  const Buffers* b2 = c2 ? &ctx->b2 : nullptr;
  hipStream_t st = ctx->stream;
  const int n_sets = (int)bounds.size() - 1;
  if (c2 && (full_layer || !ctx->has_b2 || c2->n != c.n || n_sets != s.L))
    return fail(ctx, EASYSPEC_EINVAL, "internal: two passes together need equal column counts and sets of one layer");
  WeighArgs wa, wa2;
  if ((weigh && !weigh_columns(ctx, c, b.Q, wa)) || (weigh && c2 && !weigh_columns(ctx, *c2, b2->Q, wa2)))
    return fail(ctx, EASYSPEC_EINVAL, "internal: attention weights need more workspace than there is");
  if (!c2 && !full_layer && !weigh && resident_takes(ctx, c, bounds)) {
    launch_resident(s, b, ctx->r, c, tokens, bounds.data(), n_sets, logits_out, tokens_out, st);
    HIPCHK(ctx, hipGetLastError());
    ctx->last_rows = c.n;
    ctx->last_H = b.H;
    return EASYSPEC_OK;
  }
  { ProfScope p(ctx, EASYSPEC_OP_ALL); launch_embed(s, b, c, tokens, 0, bounds[1] - bounds[0], st); }
  if (c2) { ProfScope p(ctx, EASYSPEC_OP_ALL); launch_embed(s, *b2, *c2, tokens, 0, 1, st); }
  for (int j = 0; j < n_sets; ++j) {
    const int lo = bounds[j], hi = bounds[j + 1], k = hi - lo;
    const AttnCut cut = attn_cut(s, c, k);
    // every attention layer of the set reads the hidden state that enters the set
    { ProfScope p(ctx, EASYSPEC_OP_QKV); launch_qkv(s, b, c, lo, k, st, b2, c2); }
    { ProfScope p(ctx, EASYSPEC_OP_ATTN); launch_attn(s, b, c, lo, k, cut, st); }
    if (c2) { ProfScope p(ctx, EASYSPEC_OP_ATTN); launch_attn(s, *b2, *c2, lo, k, attn_cut(s, *c2, k), st); }
    if (weigh) { ProfScope p(ctx, EASYSPEC_OP_ALL); weigh_layer(ctx, wa, lo); }
    if (weigh && c2) { ProfScope p(ctx, EASYSPEC_OP_ALL); weigh_layer(ctx, wa2, lo); }
    if (full_layer && k > 1) {
      // App. B ablation: the MLPs of the set also work from the set's input, each behind its own
      // layer's attention; one launch per operation for the whole set
      { ProfScope p(ctx, EASYSPEC_OP_OPROJ); launch_oproj_full(s, b, c, lo, k, st); }
      { ProfScope p(ctx, EASYSPEC_OP_GATEUP); launch_gateup(s, b, c, lo, k, b.ssp_set, st); }
      ProfScope p(ctx, EASYSPEC_OP_DOWN);
      if (hi < s.L) launch_down_full(s, b, c, lo, k, b.g_attn + (size_t)hi * s.d, bounds[j + 2] - hi, b.XA, st);
      else launch_down_full(s, b, c, lo, k, b.g_final, 1, b.XA, st);
      continue;
    }
    { ProfScope p(ctx, EASYSPEC_OP_OPROJ); launch_oproj(s, b, c, lo, k, st, b2, c2); }
    // the MLPs run in layer order on the running residual
    for (int i = lo; i < hi; ++i) {
      { ProfScope p(ctx, EASYSPEC_OP_GATEUP); launch_gateup(s, b, c, i, 1, b.ssp, st, b2, c2, c2 ? b2->ssp : nullptr); }
      ProfScope p(ctx, EASYSPEC_OP_DOWN);
      if (i + 1 < hi) {
        launch_down(s, b, c, i, i + 1 - lo, b.g_mlp + (size_t)(i + 1) * s.d, 1, b.XM, st, b2, c2, c2 ? b2->XM : nullptr);
      } else if (hi < s.L) {
        launch_down(s, b, c, i, -1, b.g_attn + (size_t)hi * s.d, bounds[j + 2] - hi, b.XA, st, b2, c2, c2 ? b2->XA : nullptr);
      } else {
        launch_down(s, b, c, i, -1, b.g_final, 1, b.XA, st, b2, c2, c2 ? b2->XA : nullptr);
      }
    }
  }
  { ProfScope p(ctx, EASYSPEC_OP_HEAD); launch_head(s, b, c, logits_out, tokens_out, st, b2, c2); }
  HIPCHK(ctx, hipGetLastError());
  ctx->last_rows = c2 ? c2->n : c.n;
  ctx->last_H = c2 ? b2->H : b.H;
  return EASYSPEC_OK;
}

// A calibration of more than kMaxCols columns as one pass (layers in order, as every calibration).
static int wide_forward(easyspec_ctx* ctx, const Spans& sp, const int32_t* tokens, bool all_rows, float* logits_out, int32_t* tokens_out) {
  const Shape& s = ctx->s;
  const Buffers& b = ctx->b;
  const WideBuffers& w = ctx->w;
  hipStream_t st = ctx->stream;
  { ProfScope p(ctx, EASYSPEC_OP_ALL); launch_wide_embed(s, b, w, sp, tokens, st); }
  const bool wide_head = all_rows && logits_out;
  WeighArgs wa;
  if (ctx->track.weights && !weigh_spans(ctx, sp, w.Q, wa)) return fail(ctx, EASYSPEC_EINVAL, "internal: attention weights need more workspace than there is");
  for (int l = 0; l < s.L; ++l) {
    const bool last = l + 1 == s.L;
    { ProfScope p(ctx, EASYSPEC_OP_QKV); launch_wide_qkv(s, b, w, sp, l, st); }
    { ProfScope p(ctx, EASYSPEC_OP_ATTN); launch_wide_attn(s, b, w, sp, l, st); }
    if (ctx->track.weights) { ProfScope p(ctx, EASYSPEC_OP_ALL); weigh_layer(ctx, wa, l); }
    { ProfScope p(ctx, EASYSPEC_OP_OPROJ); launch_wide_proj(s, b, w, sp, l, false, b.g_mlp + (size_t)l * s.d, false, st); }
    { ProfScope p(ctx, EASYSPEC_OP_GATEUP); launch_wide_gateup(s, b, w, sp, l, st); }
    ProfScope p(ctx, EASYSPEC_OP_DOWN);
    launch_wide_proj(s, b, w, sp, l, true, last ? b.g_final : b.g_attn + (size_t)(l + 1) * s.d, last && !wide_head, st);
  }
  {
    ProfScope p(ctx, EASYSPEC_OP_HEAD);
    if (wide_head) {
      launch_wide_head(s, b, w, sp, logits_out, tokens_out, st);
    } else {
      // only the last column of every entry is asked for: a head launch of n_seq columns
      Cols c;
      memset(&c, 0, sizeof c);
      c.n = sp.n_seq;
      for (int e = 0; e < sp.n_seq; ++e) c.logit_row[e] = c.out_idx[e] = sp.seq[e];
      launch_head(s, b, c, logits_out, tokens_out, st);
    }
  }
  HIPCHK(ctx, hipGetLastError());
  return EASYSPEC_OK;
}

extern "C" int easyspec_set_parallel_mode(easyspec_ctx* ctx, int32_t mode) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  if (mode != EASYSPEC_PARALLEL_ATTENTION && mode != EASYSPEC_PARALLEL_FULL_LAYER)
    return fail(ctx, EASYSPEC_EINVAL, "set_parallel_mode: unknown mode %d", mode);
  ctx->parallel_mode = mode;
  return EASYSPEC_OK;
}

extern "C" int easyspec_draft_step(easyspec_ctx* ctx, const int32_t* tokens_in, int32_t* tokens_out, float* logits_out) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  if (!ctx->weights_loaded) return fail(ctx, EASYSPEC_ESTATE, "draft_step: no weights loaded");
  if (!tokens_in || !tokens_out) return fail(ctx, EASYSPEC_EINVAL, "draft_step: NULL token array");
  const Shape& s = ctx->s;
  Cols c;
  memset(&c, 0, sizeof c);
  for (int b = 0; b < s.B; ++b) {
    if (ctx->precise[b] == 0) continue;
    const int pos = ctx->precise[b] + ctx->fuzzy[b];
    if (pos + 1 > s.max_ctx) return fail(ctx, EASYSPEC_ECAPACITY, "draft_step: sequence %d is full (%d slots)", b, s.max_ctx);
    if (pos + ctx->track.gone[b] >= ctx->track.max_positions)
      return fail(ctx, EASYSPEC_ECAPACITY, "draft_step: sequence %d has reached its last position (%d)", b, ctx->track.max_positions);
    if (ctx->tree[b].n > 0) return fail(ctx, EASYSPEC_ESTATE, "draft_step: sequence %d holds a token tree (continue it with easyspec_draft_tree_step)", b);
    c.seq[c.n] = b; c.pos[c.n] = pos; c.tok_idx[c.n] = b; c.logit_row[c.n] = b; c.out_idx[c.n] = b;
    c.rope_pos[c.n] = pos + ctx->track.gone[b]; c.vis_base[c.n] = pos + 1;  // causal: every earlier slot is visible
    ++c.n;
  }
  if (c.n == 0) return fail(ctx, EASYSPEC_ESTATE, "draft_step: no live sequence (calibrate a prompt first)");
  const int rc = forward(ctx, c, tokens_in, ctx->bounds, ctx->parallel_mode == EASYSPEC_PARALLEL_FULL_LAYER, logits_out, tokens_out);
  if (rc != EASYSPEC_OK) return rc;
  for (int i = 0; i < c.n; ++i) ctx->fuzzy[c.seq[i]] += 1;
  return EASYSPEC_OK;
}

extern "C" int easyspec_draft_tree_step(easyspec_ctx* ctx, const int32_t* tokens_in, const int32_t* n_nodes, const int32_t* parents,
                                        int32_t* tokens_out, float* logits_out) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  if (!ctx->weights_loaded) return fail(ctx, EASYSPEC_ESTATE, "draft_tree_step: no weights loaded");
  if (!tokens_in || !n_nodes || !parents || !tokens_out) return fail(ctx, EASYSPEC_EINVAL, "draft_tree_step: NULL argument");
  const Shape& s = ctx->s;
  const int W = EASYSPEC_MAX_TREE_WIDTH;
  Cols c;
  memset(&c, 0, sizeof c);
  for (int b = 0; b < s.B; ++b) {
    const int n = n_nodes[b];
    if (n == 0) continue;
    const easyspec_ctx::Tree& t = ctx->tree[b];
    if (n < 0 || n > W) return fail(ctx, EASYSPEC_EINVAL, "draft_tree_step: n_nodes[%d] = %d outside 0..%d", b, n, W);
    if (ctx->precise[b] == 0) return fail(ctx, EASYSPEC_ESTATE, "draft_tree_step: sequence %d has no context (calibrate a prompt first)", b);
    if (ctx->fuzzy[b] != t.n) return fail(ctx, EASYSPEC_ESTATE, "draft_tree_step: sequence %d holds chain-drafted slots; calibrate first", b);
    if (t.n + n > EASYSPEC_MAX_TREE_NODES) return fail(ctx, EASYSPEC_ECAPACITY, "draft_tree_step: sequence %d would hold %d > %d tree nodes", b, t.n + n, EASYSPEC_MAX_TREE_NODES);
    if (ctx->precise[b] + t.n + n > s.max_ctx) return fail(ctx, EASYSPEC_ECAPACITY, "draft_tree_step: sequence %d is full (%d slots)", b, s.max_ctx);
    if (c.n + n > kMaxCols) return fail(ctx, EASYSPEC_ECAPACITY, "draft_tree_step: more than %d nodes in one call", kMaxCols);
    for (int j = 0; j < n; ++j) {
      const int par = parents[b * W + j];
      if (par < -1 || par >= t.n) return fail(ctx, EASYSPEC_EINVAL, "draft_tree_step: parent %d of node %d of sequence %d is not a node of an earlier level", par, j, b);
      const int node = t.n + j;
      const int depth = par < 0 ? 0 : t.depth[par] + 1;
      c.seq[c.n] = b;
      c.pos[c.n] = ctx->precise[b] + node;
      c.rope_pos[c.n] = ctx->precise[b] + ctx->track.gone[b] + depth;
      if (c.rope_pos[c.n] >= ctx->track.max_positions)
        return fail(ctx, EASYSPEC_ECAPACITY, "draft_tree_step: sequence %d has reached its last position (%d)", b, ctx->track.max_positions);
      c.vis_base[c.n] = ctx->precise[b];
      c.vis_mask[c.n] = (par < 0 ? 0ull : t.line[par]) | (1ull << node);
      c.tok_idx[c.n] = b * W + j; c.logit_row[c.n] = b * W + j; c.out_idx[c.n] = b * W + j;
      ++c.n;
    }
  }
  if (c.n == 0) return fail(ctx, EASYSPEC_EINVAL, "draft_tree_step: no nodes");
  const int rc = forward(ctx, c, tokens_in, ctx->bounds, ctx->parallel_mode == EASYSPEC_PARALLEL_FULL_LAYER, logits_out, tokens_out);
  if (rc != EASYSPEC_OK) return rc;
  for (int i = 0; i < c.n; ++i) {
    easyspec_ctx::Tree& t = ctx->tree[c.seq[i]];
    const int node = c.pos[i] - ctx->precise[c.seq[i]];
    t.depth[node] = c.rope_pos[i] - ctx->track.gone[c.seq[i]] - ctx->precise[c.seq[i]];
    t.line[node] = c.vis_mask[i];
  }
  for (int b = 0; b < s.B; ++b) {
    ctx->tree[b].n += n_nodes[b];
    ctx->fuzzy[b] += n_nodes[b];
  }
  return EASYSPEC_OK;
}

extern "C" int easyspec_calibrate(easyspec_ctx* ctx, const int32_t* tokens, const int32_t* n_tokens, int32_t* next_token_out,
                                  float* logits_out, int32_t logits_rows) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  if (!ctx->weights_loaded) return fail(ctx, EASYSPEC_ESTATE, "calibrate: no weights loaded");
  if (!tokens || !n_tokens || !next_token_out) return fail(ctx, EASYSPEC_EINVAL, "calibrate: NULL argument");
  if (logits_rows != 0 && logits_rows != 1) return fail(ctx, EASYSPEC_EINVAL, "calibrate: logits_rows must be 0 or 1");
  const Shape& s = ctx->s;
  const int mc = ctx->cfg.max_calib_tokens;
  int total = 0;
  for (int b = 0; b < s.B; ++b) {
    const int n = n_tokens[b];
    if (n < 0 || n > mc) return fail(ctx, EASYSPEC_ECAPACITY, "calibrate: n_tokens[%d] = %d outside 0..%d", b, n, mc);
    if (n > 0 && ctx->precise[b] + n > s.max_ctx)
      return fail(ctx, EASYSPEC_ECAPACITY, "calibrate: sequence %d would hold %d > %d slots", b, ctx->precise[b] + n, s.max_ctx);
    if (n > 0 && ctx->precise[b] + n + ctx->track.gone[b] > ctx->track.max_positions)
      return fail(ctx, EASYSPEC_ECAPACITY, "calibrate: sequence %d would pass its last position (%d)", b, ctx->track.max_positions);
    total += n;
  }
  if (total == 0) return fail(ctx, EASYSPEC_EINVAL, "calibrate: no tokens");
  // passes of at most 16 columns; a sequence's tokens stay together.  Two consecutive passes of equal column
  // counts run together, so that the weights are read once for both.
  int b = 0;
  Cols held;  // a pass waiting for a partner
  memset(&held, 0, sizeof held);
  bool holding = false;
  const char* pair_env = getenv("EASYSPEC_PAIR_PASSES");  // tests: 0 = one pass at a time, 1 = pairs (bf16: if set when the context was made); read at every call
  const bool pair_passes = !pair_env || atoi(pair_env) != 0;
  if (!pair_env && total > kMaxCols && total <= ctx->w.cols) {
    // bf16 models: all columns in one wide pass
    Spans sp;
    memset(&sp, 0, sizeof sp);
    sp.tok_pitch = mc;
    int pass_first = 0, pass_cols = 0;  // of the last pass of kMaxCols columns this calibration would be packed into
    for (int q = 0; q < s.B; ++q) {
      const int n = n_tokens[q];
      if (n == 0) continue;
      if (pass_cols + n > kMaxCols) pass_first = sp.n, pass_cols = 0;
      pass_cols += n;
      const int e = sp.n_seq++;
      sp.first[e] = sp.n;
      sp.seq[e] = q;
      sp.pos0[e] = ctx->precise[q];  // fuzzy slots are dropped: positions restart at the precise length
      sp.ahead[e] = ctx->track.gone[q];
      sp.n += n;
    }
    sp.first[sp.n_seq] = sp.n;
    const int rc = wide_forward(ctx, sp, tokens, logits_rows != 0, logits_out, next_token_out);
    if (rc != EASYSPEC_OK) return rc;
    ctx->last_rows = pass_cols;  // easyspec_get_hidden: the rows it has always returned
    ctx->last_H = ctx->w.H + (size_t)pass_first * s.d;
    b = s.B;
  }
  auto run = [&](const Cols& c, const Cols* partner) { return forward(ctx, c, tokens, ctx->single, false, logits_out, next_token_out, partner, ctx->track.weights != nullptr); };
  while (b < s.B) {
    Cols c;
    memset(&c, 0, sizeof c);
    while (b < s.B && c.n + n_tokens[b] <= kMaxCols) {
      const int n = n_tokens[b];
      for (int r = 0; r < n; ++r) {
        const bool last = r == n - 1;
        c.seq[c.n] = b;
        c.pos[c.n] = ctx->precise[b] + r;  // fuzzy slots are dropped: positions restart at the precise length
        c.rope_pos[c.n] = c.pos[c.n] + ctx->track.gone[b];
        c.vis_base[c.n] = c.pos[c.n] + 1;  // causal among the tokens of the pass
        c.tok_idx[c.n] = b * mc + r;
        c.logit_row[c.n] = logits_rows ? b * mc + r : (last ? b : -1);
        c.out_idx[c.n] = last ? b : -1;
        ++c.n;
      }
      ++b;
    }
    if (c.n == 0) continue;
    int rc = EASYSPEC_OK;
    if (holding && held.n == c.n) {
      rc = run(held, &c);
      holding = false;
    } else {
      if (holding) rc = run(held, nullptr);
      const bool more = b < s.B;  // sequences left: a partner may follow
      if (rc == EASYSPEC_OK && more && pair_passes && ctx->has_b2 && twin_passes_fit(s, c.n)) {
        held = c;
        holding = true;
      } else if (rc == EASYSPEC_OK) {
        holding = false;
        rc = run(c, nullptr);
      }
    }
    if (rc != EASYSPEC_OK) return rc;
  }
  if (holding) {
    const int rc = run(held, nullptr);
    if (rc != EASYSPEC_OK) return rc;
  }
  for (int q = 0; q < s.B; ++q)
    if (n_tokens[q] > 0) {
      ctx->fuzzy[q] = 0;
      ctx->tree[q].n = 0;
      ctx->precise[q] += n_tokens[q];
    }
  return EASYSPEC_OK;
}

// ---------------------------------------------------------------------------------------------
// acceptance
// ---------------------------------------------------------------------------------------------

static int check_greedy_args(const int32_t* draft, const int32_t* target, int32_t batch, int32_t gamma, int32_t* accept_len,
                             int32_t* bonus) {
  if (!target || !accept_len || !bonus || (gamma > 0 && !draft)) return fail(nullptr, EASYSPEC_EINVAL, "greedy_accept: NULL argument");
  if (batch < 1 || gamma < 0) return fail(nullptr, EASYSPEC_EINVAL, "greedy_accept: batch must be >= 1 and gamma >= 0");
  return EASYSPEC_OK;
}

extern "C" int easyspec_greedy_accept(const int32_t* draft, const int32_t* target, int32_t batch, int32_t gamma,
                                      int32_t* accept_len, int32_t* bonus, void* hip_stream) {
  const int rc = check_greedy_args(draft, target, batch, gamma, accept_len, bonus);
  if (rc != EASYSPEC_OK) return rc;
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1) return fail(nullptr, EASYSPEC_EHIP, "no HIP device available (this library has no CPU path)");
  // a host array here would be written by the kernel through an address the device does not have
  hipPointerAttribute_t attr;
  if (hipPointerGetAttributes(&attr, accept_len) != hipSuccess || (attr.type != hipMemoryTypeDevice && attr.type != hipMemoryTypeManaged)) {
    (void)hipGetLastError();
    return fail(nullptr, EASYSPEC_EINVAL, "greedy_accept: accept_len is not device memory (host arrays: easyspec_greedy_accept_host)");
  }
  launch_accept(draft, target, batch, gamma, accept_len, bonus, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

extern "C" int easyspec_greedy_accept_host(const int32_t* draft, const int32_t* target, int32_t batch, int32_t gamma,
                                           int32_t* accept_len, int32_t* bonus) {
  const int rc = check_greedy_args(draft, target, batch, gamma, accept_len, bonus);
  if (rc != EASYSPEC_OK) return rc;
  for (int b = 0; b < batch; ++b) {
    const int32_t* d = draft + (size_t)b * gamma;
    const int32_t* t = target + (size_t)b * (gamma + 1);
    int m = 0;
    while (m < gamma && d[m] == t[m]) ++m;
    accept_len[b] = m;
    bonus[b] = t[m];
  }
  return EASYSPEC_OK;
}

extern "C" int64_t easyspec_accept_workspace_bytes(int32_t batch, int32_t gamma, int32_t vocab) {
  if (batch < 1 || gamma < 0 || vocab < 1) return -1;
  return (int64_t)sample_accept_workspace_bytes(batch, gamma, vocab);
}

static int check_accept_args(const int32_t* draft, const float* draft_logits, const float* target_logits, const float* r,
                             const float* u, int32_t batch, int32_t gamma, int32_t vocab, float temperature, int32_t* accept_len,
                             int32_t* bonus) {
  if (!target_logits || !u || !accept_len || !bonus) return fail(nullptr, EASYSPEC_EINVAL, "accept: NULL argument");
  if (gamma > 0 && (!draft || !draft_logits || !r)) return fail(nullptr, EASYSPEC_EINVAL, "accept: NULL draft argument with gamma > 0");
  if (batch < 1 || batch > 65535 || gamma < 0 || gamma > 64 || vocab < 1)
    return fail(nullptr, EASYSPEC_EINVAL, "accept: need 1 <= batch <= 65535, 0 <= gamma <= 64, vocab >= 1");
  if (!(temperature > 0.f) || !(temperature < INFINITY)) return fail(nullptr, EASYSPEC_EINVAL, "accept: temperature must be positive and finite (use easyspec_greedy_accept at 0)");
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1) return fail(nullptr, EASYSPEC_EHIP, "no HIP device available (this library has no CPU path)");
  return EASYSPEC_OK;
}

static int accept_with(const int32_t* draft, const float* draft_logits, const float* target_logits, const float* r,
                       const float* u, int32_t batch, int32_t gamma, int32_t vocab, float temperature,
                       int32_t* accept_len, int32_t* bonus, void* workspace, bool give_up, void* hip_stream) {
  if (!workspace) return fail(nullptr, EASYSPEC_EINVAL, "accept: NULL argument");
  const int rc = check_accept_args(draft, draft_logits, target_logits, r, u, batch, gamma, vocab, temperature, accept_len, bonus);
  if (rc != EASYSPEC_OK) return rc;
  launch_sample_accept(draft, draft_logits, target_logits, r, u, batch, gamma, vocab, (double)temperature, (double*)workspace,
                       accept_len, bonus, give_up, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

extern "C" int easyspec_accept(const int32_t* draft, const float* draft_logits, const float* target_logits, const float* r,
                               const float* u, int32_t batch, int32_t gamma, int32_t vocab, float temperature,
                               int32_t* accept_len, int32_t* bonus, void* workspace, void* hip_stream) {
  return accept_with(draft, draft_logits, target_logits, r, u, batch, gamma, vocab, temperature, accept_len, bonus, workspace, false, hip_stream);
}

extern "C" int easyspec_accept_give_up(const int32_t* draft, const float* draft_logits, const float* target_logits, const float* r,
                                       const float* u, int32_t batch, int32_t gamma, int32_t vocab, float temperature,
                                       int32_t* accept_len, int32_t* bonus, void* workspace, void* hip_stream) {
  return accept_with(draft, draft_logits, target_logits, r, u, batch, gamma, vocab, temperature, accept_len, bonus, workspace, true, hip_stream);
}

extern "C" int64_t easyspec_accept_static_max_bytes(void) { return (int64_t)sample_accept_static_capacity_bytes(); }

extern "C" int easyspec_accept_static(const int32_t* draft, const float* draft_logits, const float* target_logits, const float* r,
                                      const float* u, int32_t batch, int32_t gamma, int32_t vocab, float temperature,
                                      int32_t* accept_len, int32_t* bonus, void* hip_stream) {
  const int rc = check_accept_args(draft, draft_logits, target_logits, r, u, batch, gamma, vocab, temperature, accept_len, bonus);
  if (rc != EASYSPEC_OK) return rc;
  const size_t need = sample_accept_workspace_bytes(batch, gamma, vocab), have = sample_accept_static_capacity_bytes();
  if (need > have)
    return fail(nullptr, EASYSPEC_ECAPACITY, "accept_static: batch %d, gamma %d, vocab %d need %zu workspace bytes, the built-in workspace holds %zu (use easyspec_accept with a workspace of your own)",
                batch, gamma, vocab, need, have);
  double* ws = nullptr;
  HIPCHK(nullptr, sample_accept_static_workspace(&ws));
  // every workspace entry a call reads was written earlier in the same call, so nothing needs clearing
  launch_sample_accept(draft, draft_logits, target_logits, r, u, batch, gamma, vocab, (double)temperature, ws, accept_len, bonus,
                       false, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

// ---------------------------------------------------------------------------------------------
// beams and bounded caches: operators on the caller's arrays
// ---------------------------------------------------------------------------------------------

// The arrays of a launch have to be memory of the current device (those that it only reads may be pinned host memory): anything else,
// a host array or memory of another device, would be reached through an address that the kernel does not have.  NULL is passed over.
static int check_arrays(easyspec_ctx* ctx, const char* what, std::initializer_list<const void*> written, std::initializer_list<const void*> read) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return fail(ctx, EASYSPEC_EHIP, "%s: no HIP device available (this library has no CPU path)", what);
  auto reachable = [&](const void* p, bool only_read) {
    hipPointerAttribute_t attr;
    if (hipPointerGetAttributes(&attr, p) != hipSuccess) {
      (void)hipGetLastError();
      return false;
    }
    return attr.type == hipMemoryTypeManaged || (attr.type == hipMemoryTypeDevice && attr.device == dev) || (only_read && attr.type == hipMemoryTypeHost);
  };
  for (const void* p : written)
    if (p && !reachable(p, false)) return fail(ctx, EASYSPEC_EINVAL, "%s: an output or the workspace is not memory of the current device", what);
  for (const void* p : read)
    if (p && !reachable(p, true)) return fail(ctx, EASYSPEC_EINVAL, "%s: an input is not memory of the current device", what);
  return EASYSPEC_OK;
}

static bool misaligned(std::initializer_list<const void*> ps, uintptr_t to) {
  for (const void* p : ps)
    if ((uintptr_t)p % to) return true;
  return false;
}

static bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}
// Does an array that a call writes reach into one that it reads, or into another that it writes?  NULL and empty ones do not.
struct Extent {
  const void* p;
  size_t bytes;
};
static bool writes_into(std::initializer_list<Extent> written, std::initializer_list<Extent> read) {
  auto meet = [](const Extent& a, const Extent& b) { return a.p && b.p && a.bytes && b.bytes && overlap(a.p, a.bytes, b.p, b.bytes); };
  for (const Extent* w = written.begin(); w != written.end(); ++w) {
    for (const Extent* o = w + 1; o != written.end(); ++o)
      if (meet(*w, *o)) return true;
    for (const Extent& r : read)
      if (meet(*w, r)) return true;
  }
  return false;
}

static bool beam_sizes_ok(int32_t groups, int32_t beams, int32_t vocab, int32_t n_select) {
  return groups >= 1 && beams >= 1 && beams <= EASYSPEC_MAX_BEAMS && (int64_t)groups * beams <= 65535 && vocab >= 1 &&
         vocab <= EASYSPEC_MAX_BEAM_VOCAB && n_select >= 1 && n_select <= EASYSPEC_MAX_SELECT;
}

extern "C" int64_t easyspec_beam_select_workspace_bytes(int32_t groups, int32_t beams, int32_t vocab, int32_t n_select) {
  if (!beam_sizes_ok(groups, beams, vocab, n_select)) return -1;
  return (int64_t)beam_select_workspace_bytes(groups, beams, vocab, n_select);
}

extern "C" int easyspec_beam_select(const float* logits, const float* scores, const int32_t* ended, int32_t groups, int32_t beams, int32_t vocab,
                                    int32_t n_select, float temperature, int32_t end_token, int32_t* tokens_out, int32_t* parents_out,
                                    float* scores_out, void* workspace, void* hip_stream) {
  if (!logits || !scores || !tokens_out || !parents_out || !scores_out || !workspace) return fail(nullptr, EASYSPEC_EINVAL, "beam_select: NULL argument");
  if (!beam_sizes_ok(groups, beams, vocab, n_select))
    return fail(nullptr, EASYSPEC_EINVAL, "beam_select: need groups >= 1, 1 <= beams <= %d, groups * beams <= 65535, 1 <= vocab <= %d, 1 <= n_select <= %d",
                EASYSPEC_MAX_BEAMS, EASYSPEC_MAX_BEAM_VOCAB, EASYSPEC_MAX_SELECT);
  if (!(temperature > 0.f) || !(temperature < INFINITY)) return fail(nullptr, EASYSPEC_EINVAL, "beam_select: temperature must be positive and finite");
  if (ended && (end_token < 0 || end_token >= vocab)) return fail(nullptr, EASYSPEC_EINVAL, "beam_select: end_token %d outside the vocabulary", end_token);
  if (misaligned({workspace}, 16)) return fail(nullptr, EASYSPEC_EINVAL, "beam_select: workspace must be 16-byte aligned");
  const size_t rows = (size_t)groups * beams, picks = (size_t)groups * n_select * sizeof(int32_t);
  const Extent tokens = {tokens_out, picks}, parents = {parents_out, picks}, sums = {scores_out, picks}, cums = {scores, rows * sizeof(float)};
  const Extent ws = {workspace, beam_select_workspace_bytes(groups, beams, vocab, n_select)};
  const Extent rows_in = {logits, rows * vocab * sizeof(float)}, ends = {ended, rows * sizeof(int32_t)};
  if (!(scores_out == scores && n_select == beams) && writes_into({sums}, {cums}))
    return fail(nullptr, EASYSPEC_EINVAL, "beam_select: scores and scores_out overlap (they may be one array if n_select == beams)");
  // a group is picked while others' logits, scores and ends are still read
  if (writes_into({tokens, parents, sums, ws}, {rows_in, ends}) || writes_into({tokens, parents, ws}, {cums}))
    return fail(nullptr, EASYSPEC_EINVAL, "beam_select: an output or the workspace overlaps another array");
  const int rc = check_arrays(nullptr, "beam_select", {tokens_out, parents_out, scores_out, workspace}, {logits, scores, ended});
  if (rc != EASYSPEC_OK) return rc;
  launch_beam_select(logits, scores, ended, groups, beams, vocab, n_select, (double)temperature, end_token, tokens_out, parents_out, scores_out,
                     workspace, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

static int check_layout(const char* what, const easyspec_kv_layout* g) {
  if (!g) return fail(nullptr, EASYSPEC_EINVAL, "%s: layout is NULL", what);
  if (g->n_layers < 1 || g->n_layers > 65535 || g->n_seqs < 1 || g->n_seqs > EASYSPEC_MAX_BATCH || g->n_kv_heads < 1 || g->n_kv_heads > 65535 ||
      (int64_t)g->n_layers * g->n_seqs * g->n_kv_heads >= EASYSPEC_MAX_CACHE_ROWS || g->max_slots < 1 || g->max_slots > kMaxEvictSlots ||
      (g->head_dim != 64 && g->head_dim != 128) || (g->dtype != EASYSPEC_DTYPE_F32 && g->dtype != EASYSPEC_DTYPE_BF16))
    return fail(nullptr, EASYSPEC_EINVAL, "%s: bad cache layout", what);
  return EASYSPEC_OK;
}
static size_t layout_rows(const easyspec_kv_layout* g) { return (size_t)g->n_layers * g->n_seqs * g->n_kv_heads; }
static int slot_bytes(const easyspec_kv_layout* g) { return g->head_dim * (g->dtype == EASYSPEC_DTYPE_BF16 ? 2 : 4); }

// Outputs of `out_bytes` each that may be the inputs of `in_bytes` themselves or lie apart from both inputs and each other.
static int check_in_place(const char* what, const void* k, const void* v, size_t in_bytes, const void* k_out, const void* v_out, size_t out_bytes) {
  const bool same = k_out == k && v_out == v;
  if ((!same && (overlap(k_out, out_bytes, k, in_bytes) || overlap(k_out, out_bytes, v, in_bytes) || overlap(v_out, out_bytes, k, in_bytes) ||
                 overlap(v_out, out_bytes, v, in_bytes))) ||
      overlap(k_out, out_bytes, v_out, out_bytes))
    return fail(nullptr, EASYSPEC_EINVAL, "%s: arrays overlap (in place: k_out == k and v_out == v)", what);
  return EASYSPEC_OK;
}

extern "C" int easyspec_kv_reorder(const void* k, const void* v, const easyspec_kv_layout* layout, const int32_t* parents, int32_t beams,
                                   int32_t from_slot, int32_t to_slot, void* k_out, void* v_out, void* hip_stream) {
  if (!k || !v || !parents || !k_out || !v_out) return fail(nullptr, EASYSPEC_EINVAL, "kv_reorder: NULL argument");
  int rc = check_layout("kv_reorder", layout);
  if (rc != EASYSPEC_OK) return rc;
  if (beams < 1 || layout->n_seqs % beams) return fail(nullptr, EASYSPEC_EINVAL, "kv_reorder: %d sequences are no groups of %d beams", layout->n_seqs, beams);
  if (from_slot < 0 || to_slot < from_slot || to_slot > layout->max_slots)
    return fail(nullptr, EASYSPEC_EINVAL, "kv_reorder: slots %d..%d outside 0..%d", from_slot, to_slot, layout->max_slots);
  if (misaligned({k, v, k_out, v_out}, 16)) return fail(nullptr, EASYSPEC_EINVAL, "kv_reorder: arrays must be 16-byte aligned");
  const size_t bytes = layout_rows(layout) * layout->max_slots * slot_bytes(layout);
  rc = check_in_place("kv_reorder", k, v, bytes, k_out, v_out, bytes);
  if (rc != EASYSPEC_OK) return rc;
  if (writes_into({{k_out, bytes}, {v_out, bytes}}, {{parents, layout->n_seqs * sizeof(int32_t)}}))
    return fail(nullptr, EASYSPEC_EINVAL, "kv_reorder: parents lie in a cache that is written");
  rc = check_arrays(nullptr, "kv_reorder", {k_out, v_out}, {k, v, parents});
  if (rc != EASYSPEC_OK) return rc;
  const KvLayout g = {layout->n_layers, layout->n_seqs, layout->n_kv_heads, layout->max_slots};
  launch_kv_reorder(k, v, k_out, v_out, g, slot_bytes(layout), parents, 0, 0, layout->n_seqs, beams, from_slot, to_slot, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

static int weigh_args(const char* what, const easyspec_kv_layout* g, const int32_t* n_tokens, const int32_t* lens, int32_t n_q_heads, WeighArgs& a) {
  const int rc = check_layout(what, g);
  if (rc != EASYSPEC_OK) return rc;
  if (!n_tokens || !lens) return fail(nullptr, EASYSPEC_EINVAL, "%s: NULL argument", what);
  const int group = n_q_heads > 0 && n_q_heads % g->n_kv_heads == 0 ? n_q_heads / g->n_kv_heads : 0;
  if (group != 1 && group != 2 && group != 4 && group != 7 && group != 8)
    return fail(nullptr, EASYSPEC_EINVAL, "%s: %d query heads on %d KV heads: not 1, 2, 4, 7 or 8 each", what, n_q_heads, g->n_kv_heads);
  memset(&a, 0, sizeof a);
  int q_first = 0;
  for (int b = 0; b < g->n_seqs; ++b) {
    const int n = n_tokens[b];
    if (n < 0 || n > EASYSPEC_MAX_CALIB_TOKENS) return fail(nullptr, EASYSPEC_EINVAL, "%s: n_tokens[%d] = %d outside 0..%d", what, b, n, EASYSPEC_MAX_CALIB_TOKENS);
    if (n == 0) continue;
    if (lens[b] < n || lens[b] > g->max_slots) return fail(nullptr, EASYSPEC_EINVAL, "%s: lens[%d] = %d outside %d..%d", what, b, lens[b], n, g->max_slots);
    WeighEntry& e = a.entry[a.n_entries++];
    e.seq = b; e.n = n; e.len = lens[b]; e.q_first = q_first;
    q_first += n;
  }
  a.n_seqs = g->n_seqs; a.heads = g->n_kv_heads; a.Hq = n_q_heads; a.group = group; a.max_slots = g->max_slots;
  a.q_layer_pitch = (size_t)q_first * n_q_heads * g->head_dim;
  a.scale = weigh_scale(g->head_dim);
  weigh_plan(a, g->n_layers, g->dtype);
  return EASYSPEC_OK;
}

extern "C" int64_t easyspec_attn_weights_workspace_bytes(const easyspec_kv_layout* layout, const int32_t* n_tokens, const int32_t* lens, int32_t n_q_heads) {
  WeighArgs a;
  if (weigh_args("attn_weights_workspace_bytes", layout, n_tokens, lens, n_q_heads, a) != EASYSPEC_OK) return -1;
  return (int64_t)weigh_workspace_bytes(a, layout->n_layers);
}

extern "C" int easyspec_attn_weights(const float* q, const void* k, const easyspec_kv_layout* layout, const int32_t* n_tokens, const int32_t* lens,
                                     int32_t n_q_heads, const float* weights_in, float* weights_out, void* workspace, void* hip_stream) {
  if (!k || !weights_out) return fail(nullptr, EASYSPEC_EINVAL, "attn_weights: NULL argument");
  WeighArgs a;
  int rc = weigh_args("attn_weights", layout, n_tokens, lens, n_q_heads, a);
  if (rc != EASYSPEC_OK) return rc;
  if (a.n_entries == 0) return EASYSPEC_OK;  // no query and no workspace either
  if (!q || !workspace) return fail(nullptr, EASYSPEC_EINVAL, "attn_weights: NULL argument");
  if (misaligned({q, k, workspace}, 16)) return fail(nullptr, EASYSPEC_EINVAL, "attn_weights: q, k and workspace must be 16-byte aligned");
  if (misaligned({weights_in, weights_out}, 4)) return fail(nullptr, EASYSPEC_EINVAL, "attn_weights: weights must be 4-byte aligned");
  const size_t bytes = layout_rows(layout) * layout->max_slots * sizeof(float);
  if (weights_in && weights_in != weights_out && overlap(weights_in, bytes, weights_out, bytes))
    return fail(nullptr, EASYSPEC_EINVAL, "attn_weights: weights_in and weights_out overlap in part");
  // workgroups read queries, keys and statistics while others write weights already
  const Extent out = {weights_out, bytes}, ws = {workspace, weigh_workspace_bytes(a, layout->n_layers)};
  const Extent rows = {q, a.q_layer_pitch * layout->n_layers * sizeof(float)}, keys = {k, layout_rows(layout) * layout->max_slots * slot_bytes(layout)};
  if (writes_into({out, ws}, {rows, keys}) || writes_into({ws}, {{weights_in, bytes}}))
    return fail(nullptr, EASYSPEC_EINVAL, "attn_weights: weights_out or the workspace overlaps another array");
  rc = check_arrays(nullptr, "attn_weights", {weights_out, workspace}, {q, k, weights_in});
  if (rc != EASYSPEC_OK) return rc;
  a.q = q; a.k = k; a.w_in = weights_in; a.w_out = weights_out; a.stats = (float2*)workspace;
  launch_weigh(a, layout->n_layers, layout->dtype, layout->head_dim, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

extern "C" int easyspec_kv_evict(const void* k, const void* v, const float* weights, const easyspec_kv_layout* layout, const int32_t* lens,
                                 const int32_t* keep, int32_t recent, int32_t out_slots, void* k_out, void* v_out, float* weights_out,
                                 int32_t* slots_out, void* hip_stream) {
  if (!k || !v || !weights || !lens || !keep || !k_out || !v_out || !weights_out || !slots_out) return fail(nullptr, EASYSPEC_EINVAL, "kv_evict: NULL argument");
  int rc = check_layout("kv_evict", layout);
  if (rc != EASYSPEC_OK) return rc;
  if (recent < 0 || out_slots < 1 || out_slots > kMaxEvictSlots) return fail(nullptr, EASYSPEC_EINVAL, "kv_evict: bad recent or out_slots");
  EvictArgs a;
  memset(&a, 0, sizeof a);
  a.recent = recent;
  a.out_slots = out_slots;
  for (int b = 0; b < layout->n_seqs; ++b) {
    if (lens[b] < 0 || lens[b] > layout->max_slots || keep[b] < 0)
      return fail(nullptr, EASYSPEC_EINVAL, "kv_evict: sequence %d: %d slots of %d, %d to stay", b, lens[b], layout->max_slots, keep[b]);
    a.len[b] = lens[b];
    a.keep[b] = std::min(keep[b], lens[b]);
    if (a.keep[b] > out_slots) return fail(nullptr, EASYSPEC_EINVAL, "kv_evict: %d slots of sequence %d stay, the results hold %d", a.keep[b], b, out_slots);
  }
  if (misaligned({k, v, k_out, v_out}, 16)) return fail(nullptr, EASYSPEC_EINVAL, "kv_evict: caches must be 16-byte aligned");
  if (misaligned({weights, weights_out, slots_out}, 4)) return fail(nullptr, EASYSPEC_EINVAL, "kv_evict: weights and slots must be 4-byte aligned");
  const size_t rows = layout_rows(layout), in_bytes = rows * layout->max_slots * slot_bytes(layout), out_bytes = rows * out_slots * slot_bytes(layout);
  const size_t w_in = rows * layout->max_slots * sizeof(float), w_out = rows * out_slots * sizeof(float);
  const bool same = k_out == k && v_out == v;
  rc = check_in_place("kv_evict", k, v, in_bytes, k_out, v_out, out_bytes);
  if (rc != EASYSPEC_OK) return rc;
  auto apart = [&](const void* p, std::initializer_list<const void*> caches, size_t bytes) {
    for (const void* c : caches)
      if (overlap(p, w_out, c, bytes)) return false;
    return true;
  };
  if (same != (weights_out == weights) || (same && out_slots != layout->max_slots) || (!same && overlap(weights, w_in, weights_out, w_out)) ||
      overlap(slots_out, w_out, weights, w_in) || overlap(slots_out, w_out, weights_out, w_out) || !apart(slots_out, {k, v}, in_bytes) ||
      !apart(slots_out, {k_out, v_out}, out_bytes) || !apart(weights_out, {k, v}, in_bytes) || !apart(weights_out, {k_out, v_out}, out_bytes) ||
      overlap(weights, w_in, k_out, out_bytes) || overlap(weights, w_in, v_out, out_bytes))
    return fail(nullptr, EASYSPEC_EINVAL, "kv_evict: arrays overlap (in place: all three of them, with out_slots == max_slots)");
  rc = check_arrays(nullptr, "kv_evict", {k_out, v_out, weights_out, slots_out}, {k, v, weights});
  if (rc != EASYSPEC_OK) return rc;
  const KvLayout g = {layout->n_layers, layout->n_seqs, layout->n_kv_heads, layout->max_slots};
  launch_kv_evict(k, v, weights, k_out, v_out, weights_out, slots_out, g, slot_bytes(layout), a, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

// ---------------------------------------------------------------------------------------------
// caches held in 4 bits, sampling
// ---------------------------------------------------------------------------------------------

// The arrays of such a cache for a layout.
struct KvqExtents {
  Extent kc, vc, ks, vs, bounds;
};
static KvqExtents kvq_extents(const easyspec_kvq* c, const easyspec_kv_layout* g) {
  const size_t rows = layout_rows(g), slots = rows * g->max_slots, blocks = rows * ((g->max_slots + kKvqBlock - 1) / kKvqBlock);
  return {{c->k_codes, slots * (g->head_dim / 2)}, {c->v_codes, slots * (g->head_dim / 2)}, {c->k_scales, slots * (g->head_dim / 32)},
          {c->v_scales, slots * (g->head_dim / 32)}, {c->k_bounds, blocks * 2 * g->head_dim * sizeof(uint16_t)}};
}
static Kvq kvq_arrays(const easyspec_kvq* c) {
  return {(uint8_t*)c->k_codes, (uint8_t*)c->v_codes, (uint8_t*)c->k_scales, (uint8_t*)c->v_scales, (uint16_t*)c->k_bounds};
}

// What store and load have in common.  at4: first slots in the cache of 4 bits, at: in the other, of `slots`.
static int kvq_move_args(const char* what, const easyspec_kvq* cache, const easyspec_kv_layout* g, const void* k, const void* v, int32_t slots,
                         const int32_t* n_slots, const int32_t* at4, const int32_t* at, const int32_t* lens, KvqMoveArgs& a) {
  if (!cache || !k || !v || !n_slots || !at4 || !at || !cache->k_codes || !cache->v_codes || !cache->k_scales || !cache->v_scales)
    return fail(nullptr, EASYSPEC_EINVAL, "%s: NULL argument", what);
  const int rc = check_layout(what, g);
  if (rc != EASYSPEC_OK) return rc;
  if (slots < 1 || slots > kMaxEvictSlots) return fail(nullptr, EASYSPEC_EINVAL, "%s: %d slots outside 1..%d", what, slots, kMaxEvictSlots);
  memset(&a, 0, sizeof a);
  for (int b = 0; b < g->n_seqs; ++b) {
    const int len = lens ? lens[b] : g->max_slots;
    if (n_slots[b] == 0) continue;
    if (n_slots[b] < 0 || len < 0 || len > g->max_slots || at4[b] < 0 || at4[b] > len - n_slots[b] || at[b] < 0 || at[b] > slots - n_slots[b])
      return fail(nullptr, EASYSPEC_EINVAL, "%s: sequence %d: %d slots from %d of %d, and %d of %d", what, b, n_slots[b], at4[b], len, at[b], slots);
    KvqMoveEntry& e = a.entry[a.n_entries++];
    e.seq = b; e.n = n_slots[b]; e.at4 = at4[b]; e.at = at[b]; e.len = len;
  }
  if (misaligned({k, v, cache->k_codes, cache->v_codes, cache->k_bounds}, 16)) return fail(nullptr, EASYSPEC_EINVAL, "%s: values, codes and bounds must be 16-byte aligned", what);
  a.k = k; a.v = v; a.c = kvq_arrays(cache);
  a.n_seqs = g->n_seqs; a.heads = g->n_kv_heads; a.max_slots = g->max_slots; a.slots = slots;
  return EASYSPEC_OK;
}

extern "C" int easyspec_kvq_store(const void* k, const void* v, const easyspec_kv_layout* layout, int32_t src_slots, const int32_t* src_from,
                                  const int32_t* n_slots, const int32_t* to, const int32_t* lens, const easyspec_kvq* cache, void* hip_stream) {
  if (!lens) return fail(nullptr, EASYSPEC_EINVAL, "kvq_store: NULL argument");
  KvqMoveArgs a;
  int rc = kvq_move_args("kvq_store", cache, layout, k, v, src_slots, n_slots, to, src_from, lens, a);
  if (rc != EASYSPEC_OK) return rc;
  const KvqExtents x = kvq_extents(cache, layout);
  const size_t bytes = layout_rows(layout) * src_slots * slot_bytes(layout);
  if (writes_into({x.kc, x.vc, x.ks, x.vs, x.bounds}, {{k, bytes}, {v, bytes}})) return fail(nullptr, EASYSPEC_EINVAL, "kvq_store: arrays overlap");
  rc = check_arrays(nullptr, "kvq_store", {x.kc.p, x.vc.p, x.ks.p, x.vs.p, x.bounds.p}, {k, v});
  if (rc != EASYSPEC_OK) return rc;
  launch_kvq_store(a, layout->n_layers, layout->dtype, layout->head_dim, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

extern "C" int easyspec_kvq_load(const easyspec_kvq* cache, const easyspec_kv_layout* layout, const int32_t* from, const int32_t* n_slots, int32_t out_slots,
                                 const int32_t* to, void* k_out, void* v_out, void* hip_stream) {
  KvqMoveArgs a;
  int rc = kvq_move_args("kvq_load", cache, layout, k_out, v_out, out_slots, n_slots, from, to, nullptr, a);
  if (rc != EASYSPEC_OK) return rc;
  const KvqExtents x = kvq_extents(cache, layout);
  const size_t bytes = layout_rows(layout) * out_slots * slot_bytes(layout);
  if (writes_into({{k_out, bytes}, {v_out, bytes}}, {x.kc, x.vc, x.ks, x.vs})) return fail(nullptr, EASYSPEC_EINVAL, "kvq_load: arrays overlap");
  rc = check_arrays(nullptr, "kvq_load", {k_out, v_out}, {x.kc.p, x.vc.p, x.ks.p, x.vs.p});
  if (rc != EASYSPEC_OK) return rc;
  launch_kvq_load(a, layout->n_layers, layout->dtype, layout->head_dim, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

// Query heads of a KV head, or an error (negative).
static int kvq_group(const char* what, const easyspec_kv_layout* g, int32_t n_q_heads) {
  const int group = n_q_heads > 0 && n_q_heads % g->n_kv_heads == 0 ? n_q_heads / g->n_kv_heads : 0;
  if ((group != 1 && group != 2 && group != 4 && group != 7 && group != 8) || n_q_heads > 65535)
    return fail(nullptr, EASYSPEC_EINVAL, "%s: %d query heads on %d KV heads: not 1, 2, 4, 7 or 8 each, or more than 65535", what, n_q_heads, g->n_kv_heads);
  return group;
}

// The sequences with new tokens, for attention and selection: returns their tokens, or an error.
static int kvq_entries(const char* what, const easyspec_kv_layout* g, const int32_t* n_tokens, const int32_t* lens, int32_t n_q_heads, KvqEntry* entry,
                       int* n_entries, int* n_new) {
  const int rc = check_layout(what, g);
  if (rc != EASYSPEC_OK) return rc;
  if (!n_tokens || !lens) return fail(nullptr, EASYSPEC_EINVAL, "%s: NULL argument", what);
  const int group = kvq_group(what, g, n_q_heads);
  if (group < 0) return group;
  *n_entries = *n_new = 0;
  for (int b = 0; b < g->n_seqs; ++b) {
    const int n = n_tokens[b];
    if (n < 0 || n > EASYSPEC_MAX_CALIB_TOKENS) return fail(nullptr, EASYSPEC_EINVAL, "%s: n_tokens[%d] = %d outside 0..%d", what, b, n, EASYSPEC_MAX_CALIB_TOKENS);
    if (n == 0) continue;
    if (lens[b] < n || lens[b] > g->max_slots) return fail(nullptr, EASYSPEC_EINVAL, "%s: lens[%d] = %d outside %d..%d", what, b, lens[b], n, g->max_slots);
    KvqEntry& e = entry[(*n_entries)++];
    e.seq = b; e.n = n; e.len = lens[b]; e.q_first = *n_new;
    *n_new += n;
  }
  return EASYSPEC_OK;
}

static int kvq_attention_args(const char* what, const easyspec_kv_layout* g, const int32_t* n_tokens, const int32_t* lens, int32_t n_q_heads, int32_t n_blocks,
                              KvqArgs& a) {
  memset(&a, 0, sizeof a);
  const int rc = kvq_entries(what, g, n_tokens, lens, n_q_heads, a.entry, &a.n_entries, &a.n_tokens);
  if (rc != EASYSPEC_OK) return rc;
  if (n_blocks < 0 || n_blocks > kMaxKvqSelect) return fail(nullptr, EASYSPEC_EINVAL, "%s: lists of %d blocks, 0..%d are", what, n_blocks, kMaxKvqSelect);
  a.n_seqs = g->n_seqs; a.heads = g->n_kv_heads; a.Hq = n_q_heads; a.group = n_q_heads / g->n_kv_heads; a.max_slots = g->max_slots; a.n_blocks = n_blocks;
  a.scale = weigh_scale(g->head_dim);
  kvq_plan(a, g->n_layers);
  return EASYSPEC_OK;
}

extern "C" int64_t easyspec_kvq_attention_workspace_bytes(const easyspec_kv_layout* layout, const int32_t* n_tokens, const int32_t* lens, int32_t n_q_heads,
                                                          int32_t n_blocks) {
  KvqArgs a;
  if (kvq_attention_args("kvq_attention_workspace_bytes", layout, n_tokens, lens, n_q_heads, n_blocks, a) != EASYSPEC_OK) return -1;
  return (int64_t)kvq_workspace_bytes(a, layout->n_layers, layout->head_dim);
}

extern "C" int64_t easyspec_kvq_attention_workspace_limit(const easyspec_kv_layout* layout, int32_t max_tokens, int32_t n_q_heads, int32_t max_blocks) {
  const char* what = "kvq_attention_workspace_limit";
  if (check_layout(what, layout) != EASYSPEC_OK) return -1;
  const int group = kvq_group(what, layout, n_q_heads);
  if (group < 0) return -1;
  if (max_tokens < 1 || max_tokens > EASYSPEC_MAX_CALIB_TOKENS || max_blocks < 0 || max_blocks > kMaxKvqSelect) {
    fail(nullptr, EASYSPEC_EINVAL, "%s: up to %d tokens (1..%d) and lists of up to %d blocks (0..%d)", what, max_tokens, EASYSPEC_MAX_CALIB_TOKENS, max_blocks, kMaxKvqSelect);
    return -1;
  }
  return (int64_t)kvq_workspace_limit(layout->n_seqs, layout->n_kv_heads, group, layout->n_layers, layout->head_dim, max_tokens, layout->max_slots, max_blocks);
}

extern "C" int easyspec_kvq_attention(const float* q, const easyspec_kvq* cache, const easyspec_kv_layout* layout, const int32_t* n_tokens, const int32_t* lens,
                                      int32_t n_q_heads, const int32_t* blocks, int32_t n_blocks, float* out, void* workspace, void* hip_stream) {
  if (!cache || !cache->k_codes || !cache->v_codes || !cache->k_scales || !cache->v_scales) return fail(nullptr, EASYSPEC_EINVAL, "kvq_attention: NULL argument");
  KvqArgs a;
  int rc = kvq_attention_args("kvq_attention", layout, n_tokens, lens, n_q_heads, n_blocks, a);
  if (rc != EASYSPEC_OK) return rc;
  if (!blocks != !n_blocks) return fail(nullptr, EASYSPEC_EINVAL, "kvq_attention: lists of %d blocks, and %s", n_blocks, blocks ? "an array of them" : "no array");
  if (a.n_entries == 0) return EASYSPEC_OK;
  const KvqExtents x = kvq_extents(cache, layout);
  const size_t bytes = (size_t)layout->n_layers * a.n_tokens * n_q_heads * layout->head_dim * sizeof(float), ws = kvq_bytes_used(a, layout->n_layers, layout->head_dim);
  if (!q || !out || (ws && !workspace)) return fail(nullptr, EASYSPEC_EINVAL, "kvq_attention: NULL argument");
  if (misaligned({q, out, workspace, x.kc.p, x.vc.p}, 16) || misaligned({blocks}, 4))
    return fail(nullptr, EASYSPEC_EINVAL, "kvq_attention: q, out, workspace and codes must be 16-byte aligned, blocks 4-byte");
  if (writes_into({{out, bytes}, {workspace, ws}}, {{q, bytes}, x.kc, x.vc, x.ks, x.vs, {blocks, (size_t)layout->n_layers * a.n_tokens * layout->n_kv_heads * n_blocks * sizeof(int32_t)}}))
    return fail(nullptr, EASYSPEC_EINVAL, "kvq_attention: out or the workspace overlaps another array");
  rc = check_arrays(nullptr, "kvq_attention", {out, ws ? workspace : nullptr}, {q, x.kc.p, x.vc.p, x.ks.p, x.vs.p, blocks});
  if (rc != EASYSPEC_OK) return rc;
  a.q = q; a.c = kvq_arrays(cache); a.blocks = blocks; a.out = out; a.part = (float*)workspace;
  launch_kvq_attention(a, layout->n_layers, layout->head_dim, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

static int kvq_select_args(const char* what, const easyspec_kv_layout* g, const int32_t* n_tokens, const int32_t* lens, int32_t n_q_heads, int32_t n_select,
                           KvqSelectArgs& a) {
  memset(&a, 0, sizeof a);
  const int rc = kvq_entries(what, g, n_tokens, lens, n_q_heads, a.entry, &a.n_entries, &a.n_tokens);
  if (rc != EASYSPEC_OK) return rc;
  if (n_select < 1 || n_select > kMaxKvqSelect) return fail(nullptr, EASYSPEC_EINVAL, "%s: n_select = %d outside 1..%d", what, n_select, kMaxKvqSelect);
  a.n_seqs = g->n_seqs; a.heads = g->n_kv_heads; a.Hq = n_q_heads; a.group = n_q_heads / g->n_kv_heads; a.n_select = n_select;
  a.max_blocks = (g->max_slots + kKvqBlock - 1) / kKvqBlock;
  for (int i = 0; i < a.n_entries; ++i) a.most = std::max(a.most, (a.entry[i].len + kKvqBlock - 1) / kKvqBlock);
  return EASYSPEC_OK;
}

extern "C" int64_t easyspec_kvq_select_workspace_bytes(const easyspec_kv_layout* layout, const int32_t* n_tokens, const int32_t* lens, int32_t n_q_heads,
                                                       int32_t n_select) {
  KvqSelectArgs a;
  if (kvq_select_args("kvq_select_workspace_bytes", layout, n_tokens, lens, n_q_heads, n_select, a) != EASYSPEC_OK) return -1;
  return (int64_t)kvq_select_workspace_bytes(a, layout->n_layers);
}

extern "C" int easyspec_kvq_select(const float* q, const void* k_bounds, const easyspec_kv_layout* layout, const int32_t* n_tokens, const int32_t* lens,
                                   int32_t n_q_heads, int32_t keep_first, int32_t keep_last, int32_t n_select, int32_t* blocks_out, void* workspace,
                                   void* hip_stream) {
  if (!k_bounds) return fail(nullptr, EASYSPEC_EINVAL, "kvq_select: NULL argument");
  KvqSelectArgs a;
  int rc = kvq_select_args("kvq_select", layout, n_tokens, lens, n_q_heads, n_select, a);
  if (rc != EASYSPEC_OK) return rc;
  if (keep_first < 0 || keep_last < 0) return fail(nullptr, EASYSPEC_EINVAL, "kvq_select: the first %d and the last %d blocks", keep_first, keep_last);
  if (a.n_entries == 0) return EASYSPEC_OK;
  if (!q || !blocks_out || !workspace) return fail(nullptr, EASYSPEC_EINVAL, "kvq_select: NULL argument");
  if (misaligned({q, k_bounds, workspace}, 16) || misaligned({blocks_out}, 4)) return fail(nullptr, EASYSPEC_EINVAL, "kvq_select: q, k_bounds and workspace must be 16-byte aligned, blocks_out 4-byte");
  const size_t lists = (size_t)layout->n_layers * a.n_tokens * layout->n_kv_heads;
  if (writes_into({{blocks_out, lists * n_select * sizeof(int32_t)}, {workspace, kvq_select_workspace_bytes(a, layout->n_layers)}},
                  {{q, (size_t)layout->n_layers * a.n_tokens * n_q_heads * layout->head_dim * sizeof(float)},
                   {k_bounds, layout_rows(layout) * a.max_blocks * 2 * layout->head_dim * sizeof(uint16_t)}}))
    return fail(nullptr, EASYSPEC_EINVAL, "kvq_select: blocks_out or the workspace overlaps another array");
  rc = check_arrays(nullptr, "kvq_select", {blocks_out, workspace}, {q, k_bounds});
  if (rc != EASYSPEC_OK) return rc;
  a.q = q; a.bounds = (const uint16_t*)k_bounds; a.out = blocks_out; a.scores = (double*)workspace;
  a.first = keep_first; a.last = keep_last;
  launch_kvq_select(a, layout->n_layers, layout->head_dim, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

static bool sample_sizes_ok(int32_t rows, int32_t vocab) { return rows >= 1 && rows <= 65535 && vocab >= 1 && vocab <= EASYSPEC_MAX_SAMPLE_VOCAB; }

extern "C" int64_t easyspec_sample_workspace_bytes(int32_t rows, int32_t vocab) {
  return sample_sizes_ok(rows, vocab) ? (int64_t)sample_workspace_bytes(rows, vocab) : -1;
}

extern "C" int easyspec_sample(const float* logits, const float* u, int32_t rows, int32_t vocab, float temperature, int32_t top_k, float top_p, float min_p,
                               int32_t* tokens_out, float* logits_out, void* workspace, void* hip_stream) {
  if (!logits || !workspace || (!tokens_out && !logits_out) || (tokens_out && !u)) return fail(nullptr, EASYSPEC_EINVAL, "sample: NULL argument");
  if (!sample_sizes_ok(rows, vocab)) return fail(nullptr, EASYSPEC_EINVAL, "sample: need 1 <= rows <= 65535, 1 <= vocab <= %d", EASYSPEC_MAX_SAMPLE_VOCAB);
  if (!(temperature > 0.f) || !(temperature < INFINITY)) return fail(nullptr, EASYSPEC_EINVAL, "sample: temperature must be positive and finite");
  if (top_k < 0 || !(top_p > 0.f && top_p <= 1.f) || !(min_p >= 0.f && min_p <= 1.f))
    return fail(nullptr, EASYSPEC_EINVAL, "sample: need top_k >= 0, 0 < top_p <= 1, 0 <= min_p <= 1");
  if (misaligned({workspace}, 16) || misaligned({logits, u, tokens_out, logits_out}, 4)) return fail(nullptr, EASYSPEC_EINVAL, "sample: workspace must be 16-byte aligned, the other arrays 4-byte");
  const size_t words = (size_t)rows * vocab * sizeof(float);
  const Extent in = {logits, words}, us = {tokens_out ? u : nullptr, rows * sizeof(float)}, tokens = {tokens_out, rows * sizeof(int32_t)};
  const Extent left = {logits_out, words}, ws = {workspace, sample_bytes_used(rows, vocab)};
  if (writes_into({tokens, left, ws}, {us}) || writes_into({tokens, ws}, {in}) || (logits_out != logits && writes_into({left}, {in})))
    return fail(nullptr, EASYSPEC_EINVAL, "sample: arrays overlap (logits_out may be logits)");
  const int rc = check_arrays(nullptr, "sample", {tokens_out, logits_out, workspace}, {logits, us.p});
  if (rc != EASYSPEC_OK) return rc;
  launch_sample(logits, u, rows, vocab, (double)temperature, top_k, (double)top_p, (double)min_p, tokens_out, logits_out, workspace, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

// ---------------------------------------------------------------------------------------------
// beams and bounded caches: the same operators on a context
// ---------------------------------------------------------------------------------------------

extern "C" int easyspec_beam_fork(easyspec_ctx* ctx, int32_t source, int32_t first, int32_t count) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  const Shape& s = ctx->s;
  if (source < 0 || source >= s.B || first < 0 || count < 1 || count > s.B - first)
    return fail(ctx, EASYSPEC_EINVAL, "beam_fork: sequence %d into %d from %d on: out of range", source, count, first);
  const int len = ctx->precise[source] + ctx->fuzzy[source], slot = s.hd * (int)esize(s);
  if (ctx->precise[source] == 0) return fail(ctx, EASYSPEC_ESTATE, "beam_fork: sequence %d has no context (calibrate a prompt first)", source);
  const KvLayout g = {s.L, s.B, s.Hkv, s.max_ctx};
  launch_kv_reorder(ctx->b.kc, ctx->b.vc, ctx->b.kc, ctx->b.vc, g, slot, nullptr, source, first, count, 1, 0, len, ctx->stream);
  float* w = ctx->track.weights;
  if (w) launch_kv_reorder(w, nullptr, w, nullptr, g, sizeof(float), nullptr, source, first, count, 1, 0, ctx->precise[source], ctx->stream);
  HIPCHK(ctx, hipGetLastError());
  for (int b = first; b < first + count; ++b) {
    ctx->precise[b] = ctx->precise[source];
    ctx->fuzzy[b] = ctx->fuzzy[source];
    ctx->tree[b] = ctx->tree[source];
    ctx->track.gone[b] = ctx->track.gone[source];
    ctx->track.firm[b] = ctx->track.firm[source];
  }
  return EASYSPEC_OK;
}

extern "C" int easyspec_beam_reorder(easyspec_ctx* ctx, int32_t first, int32_t count, const int32_t* parents, int32_t from_slot) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  if (!parents) return fail(ctx, EASYSPEC_EINVAL, "beam_reorder: NULL argument");
  const Shape& s = ctx->s;
  if (first < 0 || count < 1 || count > s.B - first) return fail(ctx, EASYSPEC_EINVAL, "beam_reorder: sequences %d .. %d out of range", first, first + count - 1);
  const int precise = ctx->precise[first], len = precise + ctx->fuzzy[first], slot = s.hd * (int)esize(s);
  for (int b = first; b < first + count; ++b) {
    if (ctx->precise[b] == 0) return fail(ctx, EASYSPEC_ESTATE, "beam_reorder: sequence %d has no context (calibrate a prompt first)", b);
    // which caches move is known to the device alone: the lengths have to be the same whatever it decides
    if (ctx->precise[b] != precise || ctx->fuzzy[b] != ctx->fuzzy[first] || ctx->track.gone[b] != ctx->track.gone[first] || ctx->track.firm[b] != ctx->track.firm[first])
      return fail(ctx, EASYSPEC_ESTATE, "beam_reorder: sequences %d and %d differ in length", first, b);
    if (ctx->tree[b].n > 0) return fail(ctx, EASYSPEC_ESTATE, "beam_reorder: sequence %d holds a token tree", b);
  }
  if (from_slot < 0 || from_slot > len) return fail(ctx, EASYSPEC_EINVAL, "beam_reorder: from_slot %d outside 0..%d", from_slot, len);
  const int rc = check_arrays(ctx, "beam_reorder", {}, {parents});
  if (rc != EASYSPEC_OK) return rc;
  const KvLayout g = {s.L, s.B, s.Hkv, s.max_ctx};
  launch_kv_reorder(ctx->b.kc, ctx->b.vc, ctx->b.kc, ctx->b.vc, g, slot, parents, 0, first, count, count, from_slot, len, ctx->stream);
  float* w = ctx->track.weights;
  if (w) launch_kv_reorder(w, nullptr, w, nullptr, g, sizeof(float), parents, 0, first, count, count, from_slot, precise, ctx->stream);
  HIPCHK(ctx, hipGetLastError());
  return EASYSPEC_OK;
}

extern "C" int easyspec_track_attention(easyspec_ctx* ctx, int32_t max_positions) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  const Shape& s = ctx->s;
  if (max_positions < s.max_ctx || max_positions > EASYSPEC_MAX_POSITIONS)
    return fail(ctx, EASYSPEC_EINVAL, "track_attention: max_positions must be max_ctx (%d) .. %d", s.max_ctx, EASYSPEC_MAX_POSITIONS);
  if (ctx->track.weights) return fail(ctx, EASYSPEC_ESTATE, "track_attention: attention is tracked already");
  const size_t n = (size_t)s.L * s.B * s.Hkv * s.max_ctx, allocs = ctx->allocs.size(), work = ctx->work.size();
  float *weights = nullptr, *rope = nullptr;
  easyspec_ctx::Tracked& t = ctx->track;
  auto body = [&]() -> int {
    ALLOC(ctx, weights, n * sizeof(float));
    ALLOC(ctx, t.kept, n * sizeof(int32_t));
    t.stats_bytes = weigh_workspace_limit(s.B, s.Hkv, s.Hq / s.Hkv, ctx->cfg.max_calib_tokens, s.max_ctx);
    ALLOC_WORK(ctx, t.stats, t.stats_bytes);
    HIPCHK(ctx, hipMemsetAsync(weights, 0, n * sizeof(float), ctx->stream));
    if (max_positions > s.max_ctx) {
      ALLOC(ctx, rope, (size_t)max_positions * (s.hd / 2) * sizeof(float2));
      HIPCHK(ctx, fill_rope(ctx->cfg, (float2*)rope, max_positions));
    }
    HIPCHK(ctx, hipStreamSynchronize(ctx->stream));
    return EASYSPEC_OK;
  };
  const int rc = body();
  if (rc != EASYSPEC_OK) {  // the context is what it was; a pass that follows does not report this error again
    (void)hipStreamSynchronize(ctx->stream);
    for (size_t i = allocs; i < ctx->allocs.size(); ++i) (void)hipFree(ctx->allocs[i]);
    ctx->allocs.resize(allocs);
    ctx->work.resize(work);
    t.kept = nullptr;
    t.stats = nullptr;
    t.stats_bytes = 0;
    (void)hipGetLastError();
    return rc;
  }
  if (rope) ctx->b.rope = ctx->b2.rope = (float2*)rope;  // the shorter table stays: a captured pass may read it
  t.max_positions = max_positions;
  t.weights = weights;
  return EASYSPEC_OK;
}

extern "C" int easyspec_evict(easyspec_ctx* ctx, const int32_t* keep, int32_t recent) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  if (!keep) return fail(ctx, EASYSPEC_EINVAL, "evict: NULL argument");
  if (recent < 0) return fail(ctx, EASYSPEC_EINVAL, "evict: recent must be >= 0");
  if (!ctx->track.weights) return fail(ctx, EASYSPEC_ESTATE, "evict: attention is not tracked (easyspec_track_attention)");
  const Shape& s = ctx->s;
  EvictArgs a;
  memset(&a, 0, sizeof a);
  a.recent = recent;
  a.out_slots = s.max_ctx;
  bool any = false;
  for (int b = 0; b < s.B; ++b) {
    if (keep[b] == 0) return fail(ctx, EASYSPEC_EINVAL, "evict: nothing of sequence %d would stay (easyspec_truncate makes it idle)", b);
    if (keep[b] < 0 || keep[b] >= ctx->precise[b]) continue;
    a.len[b] = ctx->precise[b];
    a.keep[b] = keep[b];
    any = true;
  }
  if (!any) return EASYSPEC_OK;
  const KvLayout g = {s.L, s.B, s.Hkv, s.max_ctx};
  launch_kv_evict(ctx->b.kc, ctx->b.vc, ctx->track.weights, ctx->b.kc, ctx->b.vc, ctx->track.weights, ctx->track.kept, g, s.hd * (int)esize(s), a, ctx->stream);
  HIPCHK(ctx, hipGetLastError());
  for (int b = 0; b < s.B; ++b)
    if (a.keep[b] > 0) {
      // the slots that stay as a run of positions: the last `recent`, as far as they were one before
      const int run = std::min(std::min(recent, a.keep[b]), ctx->precise[b] - ctx->track.firm[b]);
      ctx->track.gone[b] += ctx->precise[b] - a.keep[b];
      ctx->track.firm[b] = a.keep[b] - run;
      ctx->precise[b] = a.keep[b];
      ctx->fuzzy[b] = 0;
      ctx->tree[b].n = 0;
    }
  return EASYSPEC_OK;
}

extern "C" int easyspec_get_evicted(const easyspec_ctx* ctx, int32_t* evicted) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  if (!evicted) return fail(const_cast<easyspec_ctx*>(ctx), EASYSPEC_EINVAL, "get_evicted: NULL argument");
  for (int b = 0; b < ctx->s.B; ++b) evicted[b] = ctx->track.gone[b];
  return EASYSPEC_OK;
}

extern "C" int easyspec_get_attn_weights(easyspec_ctx* ctx, int32_t b, float* out, int32_t n_slots) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  const Shape& s = ctx->s;
  if (!ctx->track.weights) return fail(ctx, EASYSPEC_ESTATE, "get_attn_weights: attention is not tracked (easyspec_track_attention)");
  if (b < 0 || b >= s.B) return fail(ctx, EASYSPEC_EINVAL, "get_attn_weights: sequence %d out of range", b);
  if (n_slots < 0 || n_slots > ctx->precise[b]) return fail(ctx, EASYSPEC_EINVAL, "get_attn_weights: %d slots outside 0..%d", n_slots, ctx->precise[b]);
  if (n_slots == 0) return EASYSPEC_OK;
  if (!out) return fail(ctx, EASYSPEC_EINVAL, "get_attn_weights: NULL argument");
  const size_t width = n_slots * sizeof(float);
  for (int l = 0; l < s.L; ++l)
    HIPCHK(ctx, hipMemcpy2DAsync(out + (size_t)l * s.Hkv * n_slots, width, ctx->track.weights + ((size_t)l * s.B + b) * s.Hkv * s.max_ctx,
                                 s.max_ctx * sizeof(float), width, s.Hkv, hipMemcpyDefault, ctx->stream));
  HIPCHK(ctx, hipStreamSynchronize(ctx->stream));
  return check_passes(ctx);
}

// ---------------------------------------------------------------------------------------------
// lengths, cache access
// ---------------------------------------------------------------------------------------------

extern "C" int easyspec_get_lens(const easyspec_ctx* ctx, int32_t* precise, int32_t* fuzzy) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  for (int b = 0; b < ctx->s.B; ++b) {
    if (precise) precise[b] = ctx->precise[b];
    if (fuzzy) fuzzy[b] = ctx->fuzzy[b];
  }
  return EASYSPEC_OK;
}

extern "C" int easyspec_truncate(easyspec_ctx* ctx, int32_t b, int32_t new_len) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  if (b < 0 || b >= ctx->s.B) return fail(ctx, EASYSPEC_EINVAL, "truncate: sequence %d out of range", b);
  if (new_len < 0 || new_len > ctx->precise[b]) return fail(ctx, EASYSPEC_EINVAL, "truncate: length %d outside 0..%d", new_len, ctx->precise[b]);
  if (new_len > 0 && new_len < ctx->track.firm[b])
    return fail(ctx, EASYSPEC_ESTATE, "truncate: sequence %d was thinned; its first %d slots are not the first of its tokens", b, ctx->track.firm[b]);
  if (new_len == 0) ctx->track.gone[b] = ctx->track.firm[b] = 0;
  ctx->precise[b] = new_len;
  ctx->fuzzy[b] = 0;
  ctx->tree[b].n = 0;
  return EASYSPEC_OK;
}

// May the copy kernel work on the caller's array itself?  Only on device memory of this device whose allocation holds
// all of it and whose address suits 16-byte accesses; anything else (host arrays, memory of another device, managed
// memory, odd addresses) goes through a staging array and hipMemcpy, which also reports what it cannot copy.
static bool device_array(const void* p, size_t bytes) {
  int dev = -1;
  hipPointerAttribute_t attr;
  void* base = nullptr;
  size_t size = 0;
  const bool ok = ((uintptr_t)p & 15) == 0 && hipGetDevice(&dev) == hipSuccess && hipPointerGetAttributes(&attr, p) == hipSuccess &&
                  attr.type == hipMemoryTypeDevice && attr.device == dev &&
                  hipMemGetAddressRange((hipDeviceptr_t*)&base, &size, (hipDeviceptr_t) const_cast<void*>(p)) == hipSuccess &&
                  (const char*)p + bytes <= (const char*)base + size;
  if (!ok) (void)hipGetLastError();
  return ok;
}

static int kv_xfer(easyspec_ctx* ctx, int32_t b, void* k, void* v, int32_t n, int to_cache) {
  const Shape& s = ctx->s;
  const size_t bytes = (size_t)s.L * s.Hkv * n * s.hd * esize(s);
  if (bytes == 0) return EASYSPEC_OK;
  hipStream_t st = ctx->stream;
  const bool apart = (uintptr_t)k + bytes <= (uintptr_t)v || (uintptr_t)v + bytes <= (uintptr_t)k;  // K and V move in one launch
  if ((to_cache || apart) && device_array(k, bytes) && device_array(v, bytes)) {
    // The copy kernel straight on the caller's arrays: one read and one write of every byte.  2048 slots of the 8B shape,
    // import and export together 17.0 ms through staging arrays, 206 us here (1.07 GB of traffic: 5.2 TB/s with both waits).
    launch_kv_copy(s, ctx->b, b, k, v, n, to_cache, st);
    HIPCHK(ctx, hipGetLastError());
    HIPCHK(ctx, hipStreamSynchronize(st));
    return check_passes(ctx);
  }
  void *dk = nullptr, *dv = nullptr;
  HIPCHK(ctx, hipMalloc(&dk, bytes));
  if (hipMalloc(&dv, bytes) != hipSuccess) {
    (void)hipFree(dk);
    return fail(ctx, EASYSPEC_EHIP, "kv transfer: out of device memory");
  }
  auto body = [&]() -> int {
    if (to_cache) {
      HIPCHK(ctx, hipMemcpyAsync(dk, k, bytes, hipMemcpyDefault, st));
      HIPCHK(ctx, hipMemcpyAsync(dv, v, bytes, hipMemcpyDefault, st));
    }
    launch_kv_copy(s, ctx->b, b, dk, dv, n, to_cache, st);
    HIPCHK(ctx, hipGetLastError());
    if (!to_cache) {
      HIPCHK(ctx, hipMemcpyAsync(k, dk, bytes, hipMemcpyDefault, st));
      HIPCHK(ctx, hipMemcpyAsync(v, dv, bytes, hipMemcpyDefault, st));
    }
    HIPCHK(ctx, hipStreamSynchronize(st));
    return check_passes(ctx);
  };
  const int rc = body();
  (void)hipFree(dk);
  (void)hipFree(dv);
  return rc;
}

extern "C" int easyspec_kv_import(easyspec_ctx* ctx, int32_t b, const void* k, const void* v, int32_t n_slots) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  if (b < 0 || b >= ctx->s.B) return fail(ctx, EASYSPEC_EINVAL, "kv_import: sequence %d out of range", b);
  if (n_slots < 0 || n_slots > ctx->s.max_ctx) return fail(ctx, EASYSPEC_ECAPACITY, "kv_import: %d slots exceed max_ctx %d", n_slots, ctx->s.max_ctx);
  if (n_slots > 0 && (!k || !v)) return fail(ctx, EASYSPEC_EINVAL, "kv_import: NULL argument");
  const int rc = kv_xfer(ctx, b, const_cast<void*>(k), const_cast<void*>(v), n_slots, 1);
  if (rc != EASYSPEC_OK) return rc;
  const Shape& s = ctx->s;
  if (ctx->track.weights && n_slots > 0)  // nothing is known of these slots
    for (int l = 0; l < s.L; ++l)
      HIPCHK(ctx, hipMemset2DAsync(ctx->track.weights + ((size_t)l * s.B + b) * s.Hkv * s.max_ctx, (size_t)s.max_ctx * sizeof(float), 0,
                                   n_slots * sizeof(float), s.Hkv, ctx->stream));
  ctx->track.gone[b] = ctx->track.firm[b] = 0;
  ctx->precise[b] = n_slots;
  ctx->fuzzy[b] = 0;
  ctx->tree[b].n = 0;
  return EASYSPEC_OK;
}

extern "C" int easyspec_kv_export(easyspec_ctx* ctx, int32_t b, void* k, void* v, int32_t n_slots) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  if (b < 0 || b >= ctx->s.B) return fail(ctx, EASYSPEC_EINVAL, "kv_export: sequence %d out of range", b);
  if (n_slots < 0 || n_slots > ctx->s.max_ctx) return fail(ctx, EASYSPEC_ECAPACITY, "kv_export: %d slots exceed max_ctx %d", n_slots, ctx->s.max_ctx);
  if (n_slots > 0 && (!k || !v)) return fail(ctx, EASYSPEC_EINVAL, "kv_export: NULL argument");
  return kv_xfer(ctx, b, k, v, n_slots, 0);
}

extern "C" int easyspec_get_hidden(easyspec_ctx* ctx, float* out, int32_t max_rows, int32_t* n_rows) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  CHECK_PASSES(ctx);
  if (!out || !n_rows) return fail(ctx, EASYSPEC_EINVAL, "get_hidden: NULL argument");
  if (ctx->last_rows == 0) return fail(ctx, EASYSPEC_ESTATE, "get_hidden: no forward has run");
  if (max_rows < ctx->last_rows) return fail(ctx, EASYSPEC_ECAPACITY, "get_hidden: %d rows needed", ctx->last_rows);
  HIPCHK(ctx, hipMemcpyAsync(out, ctx->last_H, (size_t)ctx->last_rows * ctx->s.d * sizeof(float), hipMemcpyDeviceToDevice, ctx->stream));
  *n_rows = ctx->last_rows;
  return EASYSPEC_OK;
}

extern "C" int easyspec_poison_workspaces(easyspec_ctx* ctx) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  // all bits set: a NaN in float32 and in bf16, -1 as an index
  for (const auto& w : ctx->work) HIPCHK(ctx, hipMemsetAsync(w.first, 0xFF, w.second, ctx->stream));
  return EASYSPEC_OK;
}

extern "C" int easyspec_deny_allocation(easyspec_ctx* ctx, int32_t n) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  ctx->deny_alloc = std::max(n, -1);
  return EASYSPEC_OK;
}

extern "C" int easyspec_force_give_up(easyspec_ctx* ctx, int32_t on) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  if (!resident_hasty_model(ctx->s)) return fail(ctx, EASYSPEC_EINVAL, "force_give_up: only fp32 models of one-launch passes with two query heads per KV head");
  ctx->r.hasty = on != 0;
  return EASYSPEC_OK;
}

extern "C" int easyspec_profile_begin(easyspec_ctx* ctx, int32_t op, int32_t max_launches) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  if (op < EASYSPEC_OP_QKV || op > EASYSPEC_OP_ALL) return fail(ctx, EASYSPEC_EINVAL, "profile_begin: unknown op %d", op);
  if (max_launches < 1 || max_launches > (1 << 20)) return fail(ctx, EASYSPEC_EINVAL, "profile_begin: bad max_launches");
  if (ctx->prof_op >= 0) return fail(ctx, EASYSPEC_ESTATE, "profile_begin: already profiling");
  while (ctx->prof_ev.size() < (size_t)max_launches * 2) {
    hipEvent_t e;
    HIPCHK(ctx, hipEventCreate(&e));
    ctx->prof_ev.push_back(e);
  }
  if (ctx->prof_op_of.size() < (size_t)max_launches) ctx->prof_op_of.resize((size_t)max_launches);
  ctx->timer = LaunchTimer{ctx->prof_ev.data(), ctx->prof_op_of.data(), (size_t)max_launches * 2, 0, 0};
  ctx->prof_op = op;
  return EASYSPEC_OK;
}

extern "C" int easyspec_profile_end(easyspec_ctx* ctx, int32_t* n_launches, float* total_ms, float* launch_ms, int32_t* launch_op) {
  if (!ctx) return fail(nullptr, EASYSPEC_EINVAL, "ctx is NULL");
  if (!n_launches || !total_ms) return fail(ctx, EASYSPEC_EINVAL, "profile_end: NULL argument");
  if (ctx->prof_op < 0) return fail(ctx, EASYSPEC_ESTATE, "profile_end: not profiling");
  ctx->prof_op = -1;
  HIPCHK(ctx, hipStreamSynchronize(ctx->stream));
  float sum = 0.f;
  for (size_t i = 0; i + 1 < ctx->timer.used; i += 2) {
    float ms = 0.f;
    HIPCHK(ctx, hipEventElapsedTime(&ms, ctx->timer.ev[i], ctx->timer.ev[i + 1]));
    if (launch_ms) launch_ms[i / 2] = ms;
    if (launch_op) launch_op[i / 2] = ctx->timer.op[i / 2];
    sum += ms;
  }
  *n_launches = (int32_t)(ctx->timer.used / 2);
  *total_ms = sum;
  return check_passes(ctx);
}

extern "C" int easyspec_stream_read(const void* buf, int64_t bytes, float* sink, void* hip_stream) {
  if (!buf || !sink) return fail(nullptr, EASYSPEC_EINVAL, "stream_read: NULL argument");
  if (bytes < 16 || bytes % 16 != 0) return fail(nullptr, EASYSPEC_EINVAL, "stream_read: bytes must be a positive multiple of 16");
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1) return fail(nullptr, EASYSPEC_EHIP, "no HIP device available (this library has no CPU path)");
  launch_stream_read(buf, (size_t)bytes, sink, (hipStream_t)hip_stream);
  HIPCHK(nullptr, hipGetLastError());
  return EASYSPEC_OK;
}

extern "C" int32_t easyspec_stream_read_sink_floats(void) { return stream_read_sink_floats(); }

static_assert(EASYSPEC_MAX_BEAMS == kMaxBeams && EASYSPEC_MAX_SELECT == kMaxSelect && EASYSPEC_MAX_BEAM_VOCAB == kMaxBeamVocab,
              "header and kernels disagree on the limits of a beam selection");
static_assert(EASYSPEC_KVQ_BLOCK == kKvqBlock && EASYSPEC_MAX_KVQ_SELECT == kMaxKvqSelect && EASYSPEC_MAX_SAMPLE_VOCAB == kMaxSampleVocab,
              "header and kernels disagree on the limits of caches in 4 bits and of sampling");
static_assert((uint64_t)EASYSPEC_MAX_CACHE_ROWS * 1024 <= 1ull << 32, "a grid holds 2^32 - 1 threads in a row, a workgroup of 1024 to every row of a cache");
static_assert(EASYSPEC_MAX_BATCH == kMaxCols, "per-sequence arrays of the cache operators hold kMaxCols entries");
static_assert(EASYSPEC_MAX_CHUNKS == kMaxChunks, "header and kernels disagree on the chunk limit");

extern "C" int easyspec_attention_route(const easyspec_config* cfg, const int32_t* ctx_lens, const int32_t* seqs, int32_t n_cols,
                                        int32_t n_layers_in_set, int32_t* route) {
  int rc = check_config(cfg);
  if (rc != EASYSPEC_OK) return rc;
  if (!ctx_lens || !seqs || !route) return fail(nullptr, EASYSPEC_EINVAL, "attention_route: NULL argument");
  if (n_cols < 1 || n_cols > kMaxCols) return fail(nullptr, EASYSPEC_EINVAL, "attention_route: n_cols must be 1..%d", kMaxCols);
  if (n_layers_in_set < 1 || n_layers_in_set > EASYSPEC_MAX_SET)
    return fail(nullptr, EASYSPEC_EINVAL, "attention_route: n_layers_in_set must be 1..%d", EASYSPEC_MAX_SET);
  Shape s;
  memset(&s, 0, sizeof s);
  s.dtype = cfg->dtype; s.Hq = cfg->n_q_heads; s.Hkv = cfg->n_kv_heads; s.hd = cfg->head_dim; s.max_ctx = cfg->max_ctx;
  Cols c;
  memset(&c, 0, sizeof c);
  c.n = n_cols;
  for (int i = 0; i < n_cols; ++i) {
    if (ctx_lens[i] < 1 || ctx_lens[i] > cfg->max_ctx || seqs[i] < 0 || seqs[i] >= cfg->max_batch)
      return fail(nullptr, EASYSPEC_EINVAL, "attention_route: column %d of sequence %d attends to %d slots", i, seqs[i], ctx_lens[i]);
    c.pos[i] = ctx_lens[i] - 1;
    c.seq[i] = seqs[i];
    c.vis_base[i] = ctx_lens[i];
  }
  const AttnCut cut = attn_cut(s, c, n_layers_in_set);
  route[0] = cut.mfma ? 1 : 0;
  route[1] = cut.mfma ? (cut.three ? 3 : 2) : 0;
  route[2] = cut.tiles;
  return EASYSPEC_OK;
}

extern "C" int easyspec_attention_cut(const easyspec_config* cfg, const int32_t* ctx_lens, int32_t n_cols, int32_t n_layers_in_set,
                                      int32_t* n_chunks, int32_t* ranges) {
  int rc = check_config(cfg);
  if (rc != EASYSPEC_OK) return rc;
  if (!ctx_lens || !n_chunks) return fail(nullptr, EASYSPEC_EINVAL, "attention_cut: NULL argument");
  if (n_cols < 1 || n_cols > kMaxCols) return fail(nullptr, EASYSPEC_EINVAL, "attention_cut: n_cols must be 1..%d", kMaxCols);
  if (n_layers_in_set < 1 || n_layers_in_set > EASYSPEC_MAX_SET)
    return fail(nullptr, EASYSPEC_EINVAL, "attention_cut: n_layers_in_set must be 1..%d", EASYSPEC_MAX_SET);
  Shape s;
  memset(&s, 0, sizeof s);
  s.dtype = cfg->dtype; s.Hq = cfg->n_q_heads; s.Hkv = cfg->n_kv_heads; s.hd = cfg->head_dim; s.max_ctx = cfg->max_ctx;
  Cols c;
  memset(&c, 0, sizeof c);
  c.n = n_cols;
  for (int i = 0; i < n_cols; ++i) {
    if (ctx_lens[i] < 1 || ctx_lens[i] > cfg->max_ctx)
      return fail(nullptr, EASYSPEC_EINVAL, "attention_cut: ctx_lens[%d] = %d outside 1..%d", i, ctx_lens[i], cfg->max_ctx);
    c.pos[i] = ctx_lens[i] - 1;
  }
  const AttnCut cut = attn_cut_vector(s, c, n_layers_in_set);
  const int nwv = attn_waves(cut);
  if (ranges) memset(ranges, 0, sizeof(int32_t) * (size_t)n_cols * EASYSPEC_MAX_CHUNKS * 8 * 2);
  for (int i = 0; i < n_cols; ++i) {
    int nch = 0, w0 = 0, w1 = 0;
    attn_ranges(s, cut, ctx_lens[i], 0, 0, &nch, &w0, &w1);
    n_chunks[i] = nch;
    if (!ranges) continue;
    for (int ch = 0; ch < nch && ch < EASYSPEC_MAX_CHUNKS; ++ch)
      for (int w = 0; w < nwv; ++w) {
        attn_ranges(s, cut, ctx_lens[i], ch, w, &nch, &w0, &w1);
        int32_t* r = ranges + (((size_t)i * EASYSPEC_MAX_CHUNKS + ch) * 8 + w) * 2;
        r[0] = w0;
        r[1] = w1;
      }
  }
  return nwv;
}

extern "C" int easyspec_attention_stage_walk(int32_t n_loads, int64_t* report) {
  if (!report) return fail(nullptr, EASYSPEC_EINVAL, "attention_stage_walk: NULL report");
  if (n_loads != 2 && n_loads != 8) return fail(nullptr, EASYSPEC_EINVAL, "attention_stage_walk: n_loads must be 2 or 8");
  constexpr int kPlaces = 32 * kStageRowPieces;  // 32 rows of 16 pieces = the 8 KB a wave owns
  int held_slot[kPlaces], held_piece[kPlaces], stores_at[kPlaces];
  for (int i = 0; i < kPlaces; ++i) held_slot[i] = held_piece[i] = -1, stores_at[i] = 0;
  int64_t* r = report;
  for (int i = 0; i < EASYSPEC_STAGE_FIELDS; ++i) r[i] = 0;
  r[3] = kPlaces;
  auto quarter_conflicts = [&](const int (&place)[64]) {
    int64_t n = 0;
    for (int q = 0; q < 4; ++q)
      for (int a = 0; a < 16; ++a)
        for (int b = a + 1; b < 16; ++b) n += (place[16 * q + a] & 15) == (place[16 * q + b] & 15);
    return n;
  };
  for (int j = 0; j < n_loads; ++j) {
    int place[64];
    for (int lane = 0; lane < 64; ++lane) {
      const int at = stage_store_piece(lane, j);
      place[lane] = at;
      ++r[0];
      if (at < 0 || at >= kPlaces) return fail(nullptr, EASYSPEC_EINVAL, "attention_stage_walk: store outside the stage");
      if (stores_at[at]++ == 0) ++r[1];
      held_slot[at] = 4 * j + (lane >> 4);
      held_piece[at] = lane & 15;
      r[2] = std::max<int64_t>(r[2], at + 1);
    }
    r[8] += quarter_conflicts(place);
  }
  const int n_tiles = (n_loads + 3) / 4;
  for (int t = 0; t < n_tiles; ++t)
    for (int kt = 0; kt < 4; ++kt) {
      int place[64];
      for (int lane = 0; lane < 64; ++lane) {
        const int at = stage_fetch_piece(lane, t, kt);
        place[lane] = at;
        if (at < 0 || at >= kPlaces) return fail(nullptr, EASYSPEC_EINVAL, "attention_stage_walk: fetch outside the stage");
        const int want_slot = t * 16 + stage_tile_slot(lane), want_piece = 4 * kt + (lane >> 4);
        if (want_slot >= 4 * n_loads) {
          ++r[6];
          continue;
        }
        ++r[4];
        r[5] += held_slot[at] != want_slot || held_piece[at] != want_piece;
      }
      r[8] += quarter_conflicts(place);
    }
  for (int j = 0; j < n_loads; ++j)
    for (int lane = 0; lane < 64; ++lane) {
      const int t = j / 4, i = j % 4;
      // element i of the lane's MFMA result is A row 4 (lane / 16) + i, fed by the lanes whose lane % 16 is that row
      const int a_row = 4 * (lane >> 4) + i;
      const int slot_of_row = t * 16 + stage_tile_slot(a_row);
      r[7] += slot_of_row != 4 * j + (lane >> 4) || score_slot_in_batch(lane, t, i) != 4 * j + (lane >> 4);
    }
  return EASYSPEC_OK;
}

extern "C" int easyspec_weight_walk(const easyspec_config* cfg, int32_t op, int32_t n_cols, int32_t n_layers_in_set, int32_t full_layer,
                                    int64_t* report) {
  int rc = check_config(cfg);
  if (rc != EASYSPEC_OK) return rc;
  if (!report) return fail(nullptr, EASYSPEC_EINVAL, "weight_walk: NULL argument");
  if (op != EASYSPEC_OP_QKV && op != EASYSPEC_OP_OPROJ && op != EASYSPEC_OP_GATEUP && op != EASYSPEC_OP_DOWN && op != EASYSPEC_OP_HEAD)
    return fail(nullptr, EASYSPEC_EINVAL, "weight_walk: op %d streams no packed matrix", op);
  if (n_cols < 1 || n_cols > kMaxCols) return fail(nullptr, EASYSPEC_EINVAL, "weight_walk: n_cols must be 1..%d", kMaxCols);
  if (n_layers_in_set < 1 || n_layers_in_set > EASYSPEC_MAX_SET || n_layers_in_set > cfg->n_layers)
    return fail(nullptr, EASYSPEC_EINVAL, "weight_walk: n_layers_in_set must be 1..%d and at most n_layers", EASYSPEC_MAX_SET);
  Shape s;
  shape_of(cfg, s);
  const StreamPlan p = stream_plan(s, op, n_cols, n_layers_in_set, full_layer != 0);
  StreamWalk w;
  if (stream_walk(s, p, n_cols, &w) != 0) return fail(nullptr, EASYSPEC_EINVAL, "weight_walk: launch shape not walkable");
  const int64_t out[EASYSPEC_WALK_FIELDS] = {p.grid, p.nw, p.TP, p.R, p.NB, w.w_max, w.w_pieces, w.w_out_of_range, w.x_max,
                                             w.x_slot_elems, w.x_out_of_range, w.tiles, w.missed_tiles, w.repeated_tiles,
                                             w.reread_tiles, w.uncovered_pieces};
  memcpy(report, out, sizeof out);
  return EASYSPEC_OK;
}

extern "C" int easyspec_wide_walk(const easyspec_config* cfg, int32_t op, int32_t n_cols, int64_t* report) {
  const int rc = check_config(cfg);
  if (rc != EASYSPEC_OK) return rc;
  if (!report) return fail(nullptr, EASYSPEC_EINVAL, "wide_walk: NULL argument");
  if (op != EASYSPEC_OP_QKV && op != EASYSPEC_OP_OPROJ && op != EASYSPEC_OP_GATEUP && op != EASYSPEC_OP_DOWN && op != EASYSPEC_OP_HEAD)
    return fail(nullptr, EASYSPEC_EINVAL, "wide_walk: op %d is no matrix product", op);
  if (cfg->dtype != EASYSPEC_DTYPE_BF16) return fail(nullptr, EASYSPEC_EINVAL, "wide_walk: only bf16 models have wide passes");
  if (n_cols <= kMaxCols || n_cols > kWideCols) return fail(nullptr, EASYSPEC_EINVAL, "wide_walk: n_cols must be %d..%d", kMaxCols + 1, kWideCols);
  Shape s;
  shape_of(cfg, s);
  WideWalk w;
  wide_walk(s, op, n_cols, &w);
  static_assert(sizeof w == EASYSPEC_WIDE_FIELDS * sizeof(int64_t), "the report lists every field in order");
  memcpy(report, &w, sizeof w);
  return EASYSPEC_OK;
}

extern "C" int64_t easyspec_step_bytes(const easyspec_ctx* ctx) {
  if (!ctx) return 0;
  const Shape& s = ctx->s;
  const int64_t e = (int64_t)esize(s);
  const int64_t per_layer = ((int64_t)s.RQKV * s.d + (int64_t)s.d * s.HQ + 3ll * s.F * s.d) * e;
  int64_t bytes = per_layer * s.L + (int64_t)s.V * s.d * e;
  for (int b = 0; b < s.B; ++b)
    if (ctx->precise[b] > 0) bytes += (int64_t)(ctx->precise[b] + ctx->fuzzy[b] + 1) * s.L * 2 * s.Hkv * s.hd * e;
  return bytes;
}
