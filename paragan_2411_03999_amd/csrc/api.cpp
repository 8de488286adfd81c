// C ABI of libparagan (include/paragan.h): argument validation, buffer
// planning, and dispatch into the block executors.  Every entry point
// catches all exceptions and turns them into status codes.
#include <cstring>

#include "../../include/paragan.h"
#include "blocks.hpp"
#include "net.hpp"
#include "token.hpp"
#include <cfloat>
#include <cmath>

using namespace pg;

static std::string g_create_err;

namespace {
// binds the context's profiler to the launchers for the duration of a call
struct ProfBind {
  explicit ProfBind(paragan_ctx* c) { pg::t_prof = c ? &c->prof : nullptr; }
  ~ProfBind() { pg::t_prof = nullptr; }
};
}  // namespace

static int fail(paragan_ctx* ctx, int code, const std::string& msg) {
  if (ctx) {
    ctx->err = msg;
    // leave no work of a failed call running on the context's own streams
    // (it may read the caller's buffers)
    if (ctx->side) (void)hipStreamSynchronize(ctx->side);
    if (ctx->wside) (void)hipStreamSynchronize(ctx->wside);
  } else {
    g_create_err = msg;
  }
  return code;
}

#define PG_TRY(ctx, ...)                                   \
  try {                                                    \
    __VA_ARGS__;                                           \
    return PARAGAN_OK;                                     \
  } catch (const ::pg::Error& e) {                         \
    return fail(ctx, e.code, e.msg);                       \
  } catch (const std::exception& e) {                      \
    return fail(ctx, PARAGAN_EINVAL, e.what());            \
  } catch (...) {                                          \
    return fail(ctx, PARAGAN_EINVAL, "unknown error");     \
  }

extern "C" {

int paragan_create(paragan_ctx** out, void* hip_stream) {
  if (!out) return fail(nullptr, PARAGAN_EINVAL, "paragan_create: out is NULL");
  try {
    int dev = 0;
    PG_HIP(hipGetDevice(&dev));
    hipDeviceProp_t p;
    PG_HIP(hipGetDeviceProperties(&p, dev));
    if (std::strncmp(p.gcnArchName, "gfx950", 6) != 0)
      throw Error{PARAGAN_EUNSUPPORTED, std::string("paragan needs gfx950, found ") + p.gcnArchName};
    void* scr = sn_scratch_init(dev);
    auto* c = new paragan_ctx;
    c->stream = (hipStream_t)hip_stream;
    c->device = dev;
    c->n_cu = p.multiProcessorCount;
    c->sn_scratch = scr;
    *out = c;
    return PARAGAN_OK;
  } catch (const Error& e) {
    return fail(nullptr, e.code, e.msg);
  }
}

void paragan_destroy(paragan_ctx* ctx) {
  if (!ctx) return;
  if (ctx->side) {
    (void)hipStreamSynchronize(ctx->side);
    (void)hipStreamDestroy(ctx->side);
  }
  if (ctx->wside) {
    (void)hipStreamSynchronize(ctx->wside);
    (void)hipStreamDestroy(ctx->wside);
  }
  for (hipEvent_t e : ctx->ev)
    if (e) (void)hipEventDestroy(e);
  for (hipEvent_t e : ctx->wev)
    if (e) (void)hipEventDestroy(e);
  delete ctx;
}

const char* paragan_last_error(const paragan_ctx* ctx) {
  return ctx ? ctx->err.c_str() : g_create_err.c_str();
}

int paragan_sync(paragan_ctx* ctx) {
  if (!ctx) return PARAGAN_EINVAL;
  PG_TRY(ctx, PG_HIP(hipStreamSynchronize(ctx->stream)))
}

int paragan_set_overlap_wgrad(paragan_ctx* ctx, int on) {
  if (!ctx) return PARAGAN_EINVAL;
  if (on != 0 && on != 1) return fail(ctx, PARAGAN_EINVAL, "paragan_set_overlap_wgrad: on must be 0 or 1");
  ctx->overlap_wgrad = on == 1;
  return PARAGAN_OK;
}

int paragan_grad_clip_size(size_t* bytes) {
  if (!bytes) return fail(nullptr, PARAGAN_EINVAL, "paragan_grad_clip_size: bytes is NULL");
  *bytes = 256 + 2 * kClipFlatBlocks * sizeof(double);
  return PARAGAN_OK;
}
int paragan_set_grad_clip(paragan_ctx* ctx, float max_norm_g, float max_norm_d, void* buf) {
  if (!ctx) return PARAGAN_EINVAL;
  if (!(max_norm_g >= 0.f) || !(max_norm_d >= 0.f))
    return fail(ctx, PARAGAN_EINVAL, "paragan_set_grad_clip: the norms must be >= 0");
  if ((max_norm_g > 0.f || max_norm_d > 0.f) && (!buf || ((uintptr_t)buf & 255)))
    return fail(ctx, PARAGAN_EINVAL, "paragan_set_grad_clip: buf must be a 256-byte aligned device buffer");
  ctx->clip_g = max_norm_g;
  ctx->clip_d = max_norm_d;
  ctx->clip_buf = buf;
  return PARAGAN_OK;
}

int64_t paragan_cpad(int64_t c) { return cpad(c); }

}  // extern "C"

// ------------------------------------------------------------ helpers
static void need(const void* p, const char* what) {
  if (!p) throw Error{PARAGAN_EINVAL, std::string(what) + " is NULL"};
}
static void aligned(const void* p, const char* what) {
  if (((uintptr_t)p & 255) != 0) throw Error{PARAGAN_EINVAL, std::string(what) + " is not 256-byte aligned"};
}

static int export_layout(const Layout& L, paragan_tensor_info* out, int32_t cap, int32_t* count,
                         int64_t* n_params, int64_t* n_u) {
  if (count) *count = (int32_t)L.e.size();
  if (n_params) *n_params = L.n_params;
  if (n_u) *n_u = L.n_u;
  if (out) {
    if (cap < (int32_t)L.e.size()) return PARAGAN_EINVAL;
    for (size_t i = 0; i < L.e.size(); ++i) {
      const Entry& e = L.e[i];
      paragan_tensor_info& t = out[i];
      std::memset(&t, 0, sizeof(t));
      std::strncpy(t.name, e.name.c_str(), sizeof(t.name) - 1);
      t.ndim = (int32_t)e.shape.size();
      for (size_t d = 0; d < e.shape.size() && d < 4; ++d) t.shape[d] = e.shape[d];
      t.offset = e.offset;
      t.u_offset = e.u_offset;
    }
  }
  return PARAGAN_OK;
}

// ------------------------------------------------------------ G block
static void gcheck(const paragan_gblock_desc* d) {
  if (!d) throw Error{PARAGAN_EINVAL, "gblock: desc is NULL"};
  PG_CHECK(d->B >= 1 && d->H >= 1 && d->W >= 1, "gblock: B, H, W must be >= 1");
  PG_CHECK(d->cin >= 1 && d->cout >= 1 && d->dc >= 1, "gblock: cin, cout, dc must be >= 1");
  PG_CHECK(d->dtype == PARAGAN_BF16 || d->dtype == PARAGAN_F32, "gblock: dtype must be PARAGAN_BF16 or PARAGAN_F32");
  PG_CHECK(d->n_power_iter >= 1, "gblock: n_power_iter must be >= 1");
  PG_CHECK(d->bn_eps > 0.f && d->sn_eps > 0.f, "gblock: eps must be > 0");
  PG_CHECK((int64_t)d->B * 4 * d->H * d->W < (1LL << 31), "gblock: too many output pixels");
}

static GBlock make_g(const paragan_gblock_desc* d) {
  GBlock g;
  g.B = d->B; g.H = d->H; g.W = d->W; g.cin = d->cin; g.cout = d->cout; g.dc = d->dc;
  g.npi = d->n_power_iter; g.f32 = d->dtype == PARAGAN_F32; g.bn_eps = d->bn_eps; g.sn_eps = d->sn_eps;
  Arena a(nullptr);
  g.plan_saved(a);
  return g;
}

extern "C" int paragan_gblock_check(const paragan_gblock_desc* d) { PG_TRY(nullptr, gcheck(d)) }

extern "C" int paragan_gblock_layout(const paragan_gblock_desc* d, paragan_tensor_info* out, int32_t cap,
                                     int32_t* count, int64_t* n_params, int64_t* n_u) {
  try {
    gcheck(d);
    return export_layout(gblock_layout(d->cin, d->cout, d->dc), out, cap, count, n_params, n_u);
  } catch (const Error& e) {
    return fail(nullptr, e.code, e.msg);
  }
}

extern "C" int paragan_gblock_sizes(const paragan_gblock_desc* d, size_t* saved, size_t* ws) {
  PG_TRY(nullptr, {
    gcheck(d);
    GBlock g = make_g(d);
    Arena a(nullptr);
    g.plan_saved(a);
    if (saved) *saved = a.off;
    int dev = 0, ncu = 256;
    if (hipGetDevice(&dev) == hipSuccess) {
      hipDeviceProp_t p;
      if (hipGetDeviceProperties(&p, dev) == hipSuccess) ncu = p.multiProcessorCount;
    }
    if (ws) *ws = g.ws_size(ncu);
  })
}

static size_t g_ws_for(paragan_ctx* ctx, const GBlock& g) { return g.ws_size(ctx->n_cu); }

extern "C" int paragan_gblock_fwd(paragan_ctx* ctx, const paragan_gblock_desc* d, const float* params, float* u,
                                  const void* x, const float* cond, void* y, void* saved, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    gcheck(d);
    need(params, "params"); need(u, "u"); need(x, "x"); need(cond, "cond"); need(y, "y");
    need(saved, "saved"); need(ws, "ws");
    aligned(saved, "saved"); aligned(ws, "ws");
    GBlock g = make_g(d);
    Arena a(saved);
    g.plan_saved(a);
    Layout L = gblock_layout(d->cin, d->cout, d->dc);
    Params P{&L, "", params, u, nullptr};
    Exec ex{ctx->stream, ctx->n_cu, ws, g_ws_for(ctx, g)};
    g.fwd(ex, P, x, cond, y);
  })
}

extern "C" int paragan_gblock_bwd(paragan_ctx* ctx, const paragan_gblock_desc* d, const float* params,
                                  const void* x, const float* cond, const void* saved, const void* dy, void* dx,
                                  float* dcond, float* grads, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    gcheck(d);
    need(params, "params"); need(x, "x"); need(cond, "cond"); need(saved, "saved"); need(dy, "dy");
    need(dx, "dx"); need(dcond, "dcond"); need(grads, "grads"); need(ws, "ws");
    aligned(saved, "saved"); aligned(ws, "ws");
    GBlock g = make_g(d);
    Arena a((void*)saved);
    g.plan_saved(a);
    Layout L = gblock_layout(d->cin, d->cout, d->dc);
    Params P{&L, "", params, nullptr, grads};
    Exec ex{ctx->stream, ctx->n_cu, ws, g_ws_for(ctx, g)};
    g.bwd(ex, P, x, cond, dy, dx, dcond, false);
  })
}

// ------------------------------------------------------------ D block
static void dcheck(const paragan_dblock_desc* d) {
  if (!d) throw Error{PARAGAN_EINVAL, "dblock: desc is NULL"};
  PG_CHECK(d->B >= 1 && d->H >= 1 && d->W >= 1, "dblock: B, H, W must be >= 1");
  PG_CHECK(d->cin >= 1 && d->cout >= 1, "dblock: cin, cout must be >= 1");
  PG_CHECK(d->dtype == PARAGAN_BF16 || d->dtype == PARAGAN_F32, "dblock: dtype must be PARAGAN_BF16 or PARAGAN_F32");
  PG_CHECK(d->n_power_iter >= 1, "dblock: n_power_iter must be >= 1");
  PG_CHECK(d->sn_eps > 0.f, "dblock: sn_eps must be > 0");
  PG_CHECK(!d->downsample || (d->H % 2 == 0 && d->W % 2 == 0), "dblock: pooling needs even H and W");
  PG_CHECK(d->learnable_sc || (d->cin == d->cout && !d->downsample),
           "dblock: an identity skip needs cin == cout and no pooling");
  PG_CHECK((int64_t)d->B * d->H * d->W < (1LL << 31), "dblock: too many pixels");
}

static DBlock make_d(const paragan_dblock_desc* d) {
  DBlock b;
  b.B = d->B; b.H = d->H; b.W = d->W; b.cin = d->cin; b.cout = d->cout; b.npi = d->n_power_iter;
  b.preact = d->preact != 0; b.down = d->downsample != 0; b.lsc = d->learnable_sc != 0;
  b.f32 = d->dtype == PARAGAN_F32; b.sn_eps = d->sn_eps;
  Arena a(nullptr);
  b.plan_saved(a);
  return b;
}

extern "C" int paragan_dblock_check(const paragan_dblock_desc* d) { PG_TRY(nullptr, dcheck(d)) }

extern "C" int paragan_dblock_layout(const paragan_dblock_desc* d, paragan_tensor_info* out, int32_t cap,
                                     int32_t* count, int64_t* n_params, int64_t* n_u) {
  try {
    dcheck(d);
    return export_layout(dblock_layout(d->cin, d->cout, d->learnable_sc != 0), out, cap, count, n_params, n_u);
  } catch (const Error& e) {
    return fail(nullptr, e.code, e.msg);
  }
}

static int device_cus() {
  int dev = 0, ncu = 256;
  if (hipGetDevice(&dev) == hipSuccess) {
    hipDeviceProp_t p;
    if (hipGetDeviceProperties(&p, dev) == hipSuccess) ncu = p.multiProcessorCount;
  }
  return ncu;
}

extern "C" int paragan_dblock_sizes(const paragan_dblock_desc* d, size_t* saved, size_t* ws) {
  PG_TRY(nullptr, {
    dcheck(d);
    DBlock b = make_d(d);
    Arena a(nullptr);
    b.plan_saved(a);
    if (saved) *saved = a.off;
    if (ws) *ws = b.ws_size(device_cus());
  })
}

extern "C" int paragan_dblock_fwd(paragan_ctx* ctx, const paragan_dblock_desc* d, const float* params, float* u,
                                  const void* x, void* y, void* saved, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    dcheck(d);
    need(params, "params"); need(u, "u"); need(x, "x"); need(y, "y"); need(saved, "saved"); need(ws, "ws");
    aligned(saved, "saved"); aligned(ws, "ws");
    DBlock b = make_d(d);
    Arena a(saved);
    b.plan_saved(a);
    Layout L = dblock_layout(d->cin, d->cout, d->learnable_sc != 0);
    Params P{&L, "", params, u, nullptr};
    Exec ex{ctx->stream, ctx->n_cu, ws, b.ws_size(ctx->n_cu)};
    b.fwd(ex, P, x, y);
  })
}

extern "C" int paragan_dblock_bwd(paragan_ctx* ctx, const paragan_dblock_desc* d, const float* params,
                                  const void* x, const void* saved, const void* dy, void* dx, float* grads,
                                  void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    dcheck(d);
    need(params, "params"); need(x, "x"); need(saved, "saved"); need(dy, "dy"); need(grads, "grads");
    need(ws, "ws");
    aligned(saved, "saved"); aligned(ws, "ws");
    DBlock b = make_d(d);
    Arena a((void*)saved);
    b.plan_saved(a);
    Layout L = dblock_layout(d->cin, d->cout, d->learnable_sc != 0);
    Params P{&L, "", params, nullptr, grads};
    Exec ex{ctx->stream, ctx->n_cu, ws, b.ws_size(ctx->n_cu)};
    b.bwd(ex, P, x, dy, dx, false);
  })
}

// ------------------------------------------------------------ SN
extern "C" int paragan_sn_ws_size(int64_t rows, int64_t cols, size_t* ws_bytes) {
  PG_TRY(nullptr, {
    PG_CHECK(rows >= 1 && cols >= 1, "sn_ws_size: rows and cols must be >= 1");
    need(ws_bytes, "ws_bytes");
    *ws_bytes = sn_ws_bytes(rows, cols);
  })
}

static void sn_check(int64_t rows, int64_t cols, int n_iter, float eps) {
  PG_CHECK(rows >= 1 && cols >= 1, "sn_power_iter: rows and cols must be >= 1");
  PG_CHECK(n_iter >= 1, "sn_power_iter: n_iter must be >= 1");
  PG_CHECK(eps > 0.f, "sn_power_iter: eps must be > 0");
  PG_CHECK(rows < (1LL << 31) && cols < (1LL << 31), "sn_power_iter: matrix too large");
}

extern "C" int paragan_sn_check(int64_t rows, int64_t cols, int n_iter, float eps) {
  PG_TRY(nullptr, sn_check(rows, cols, n_iter, eps))
}

extern "C" int paragan_sn_power_iter(paragan_ctx* ctx, const float* W, int64_t rows, int64_t cols, float* u,
                                     float* v, float* sigma, int n_iter, float eps, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    need(W, "W"); need(u, "u"); need(v, "v"); need(sigma, "sigma"); need(ws, "ws");
    aligned(ws, "ws");
    sn_check(rows, cols, n_iter, eps);
    sn_power_iter(ctx->stream, W, rows, cols, u, v, sigma, n_iter, eps, ws);
  })
}

extern "C" int paragan_sn_power_iter_noalloc(paragan_ctx* ctx, const float* W, int64_t rows, int64_t cols,
                                             float* u, float* v, float* sigma, int n_iter, float eps) {
  if (!ctx) return PARAGAN_EINVAL;
  PG_TRY(ctx, {
    need(W, "W"); need(u, "u"); need(v, "v"); need(sigma, "sigma");
    sn_check(rows, cols, n_iter, eps);
    const size_t want = sn_ws_bytes(rows, cols);
    PG_CHECK(want <= kSnScratchBytes, "sn_power_iter_noalloc: a " + std::to_string(rows) + " x " +
                                          std::to_string(cols) + " weight needs " + std::to_string(want) +
                                          " bytes of scratch, more than the library's " +
                                          std::to_string(kSnScratchBytes) + " (use paragan_sn_power_iter)");
    PG_CHECK(ctx->sn_scratch != nullptr, "sn_power_iter_noalloc: context has no scratch address");
    sn_power_iter(ctx->stream, W, rows, cols, u, v, sigma, n_iter, eps, ctx->sn_scratch);
  })
}

// ------------------------------------------------------------ attention
static void acheck(const paragan_attn_desc* d) {
  if (!d) throw Error{PARAGAN_EINVAL, "attn: desc is NULL"};
  PG_CHECK(d->B >= 1 && d->H >= 2 && d->W >= 2 && d->H % 2 == 0 && d->W % 2 == 0,
           "attn: B >= 1 and H, W even and >= 2");
  PG_CHECK(d->C >= 8 && d->C % 8 == 0, "attn: C must be a multiple of 8");
  PG_CHECK(d->C / 8 <= 32, "attn: C/8 query width above 32 is not supported");
  const int64_t dv = cpad(d->C / 2);
  PG_CHECK(dv == 32 || dv == 64 || dv == 96 || dv == 128, "attn: C/2 value width must pad to 32, 64, 96 or 128");
  PG_CHECK(d->n_power_iter >= 1 && d->sn_eps > 0.f, "attn: bad n_power_iter / sn_eps");
  PG_CHECK((int64_t)d->B * d->H * d->W < (1LL << 31), "attn: too many pixels");
}

static Attn make_a(const paragan_attn_desc* d) {
  Attn t;
  t.B = d->B; t.H = d->H; t.W = d->W; t.C = d->C; t.npi = d->n_power_iter; t.sn_eps = d->sn_eps;
  Arena a(nullptr);
  t.plan_saved(a);
  return t;
}

extern "C" int paragan_attn_check(const paragan_attn_desc* d) { PG_TRY(nullptr, acheck(d)) }

extern "C" int paragan_attn_layout(const paragan_attn_desc* d, paragan_tensor_info* out, int32_t cap,
                                   int32_t* count, int64_t* n_params, int64_t* n_u) {
  try {
    acheck(d);
    return export_layout(attn_layout(d->C), out, cap, count, n_params, n_u);
  } catch (const Error& e) {
    return fail(nullptr, e.code, e.msg);
  }
}

extern "C" int paragan_attn_sizes(const paragan_attn_desc* d, size_t* saved, size_t* ws) {
  PG_TRY(nullptr, {
    acheck(d);
    Attn t = make_a(d);
    Arena a(nullptr);
    t.plan_saved(a);
    if (saved) *saved = a.off;
    if (ws) *ws = t.ws_size(device_cus());
  })
}

extern "C" int paragan_attn_fwd(paragan_ctx* ctx, const paragan_attn_desc* d, const float* params, float* u,
                                const void* x, void* y, void* saved, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    acheck(d);
    need(params, "params"); need(u, "u"); need(x, "x"); need(y, "y"); need(saved, "saved"); need(ws, "ws");
    aligned(saved, "saved"); aligned(ws, "ws");
    Attn t = make_a(d);
    Arena a(saved);
    t.plan_saved(a);
    Layout L = attn_layout(d->C);
    Params P{&L, "", params, u, nullptr};
    Exec ex{ctx->stream, ctx->n_cu, ws, t.ws_size(ctx->n_cu)};
    t.fwd(ex, P, x, y);
  })
}

extern "C" int paragan_attn_bwd(paragan_ctx* ctx, const paragan_attn_desc* d, const float* params, const void* x,
                                const void* saved, const void* dy, void* dx, float* grads, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    acheck(d);
    need(params, "params"); need(x, "x"); need(saved, "saved"); need(dy, "dy"); need(dx, "dx");
    need(grads, "grads"); need(ws, "ws");
    aligned(saved, "saved"); aligned(ws, "ws");
    Attn t = make_a(d);
    Arena a((void*)saved);
    t.plan_saved(a);
    Layout L = attn_layout(d->C);
    Params P{&L, "", params, nullptr, grads};
    Exec ex{ctx->stream, ctx->n_cu, ws, t.ws_size(ctx->n_cu)};
    t.bwd(ex, P, x, dy, dx, true);
  })
}

// ------------------------------------------------------------ token attention operators
static void on_device(const paragan_ctx* ctx, const char* what) {
  int dev = -1;
  PG_HIP(hipGetDevice(&dev));
  PG_CHECK(dev == ctx->device, std::string(what) + ": the context's device is not the current one");
}
static void need16(const void* p, const char* what) {
  need(p, what);
  if (((uintptr_t)p & 15) != 0) throw Error{PARAGAN_EINVAL, std::string(what) + " is not 16-byte aligned"};
}

static QkNorm make_qk(const paragan_qknorm_desc* d) {
  if (!d) throw Error{PARAGAN_EINVAL, "qknorm: desc is NULL"};
  PG_CHECK(d->T >= 1 && d->T < (1LL << 31), "qknorm: T must be 1 .. 2^31 - 1");
  PG_CHECK(d->Hq >= 1 && d->Hk >= 1 && (int64_t)d->Hq + d->Hk <= (1 << 20), "qknorm: Hq, Hk must be >= 1 (and at most 2^20 together)");
  PG_CHECK(d->d >= 8 && d->d <= 256 && d->d % 8 == 0, "qknorm: d must be a multiple of 8 up to 256");
  PG_CHECK(d->rot >= 0 && d->rot <= d->d && d->rot % 16 == 0, "qknorm: rot must be a multiple of 16 up to d");
  PG_CHECK(d->interleaved == 0 || d->interleaved == 1, "qknorm: interleaved must be 0 or 1");
  PG_CHECK(d->n_pos >= 1, "qknorm: n_pos must be >= 1");
  PG_CHECK(d->dtype == PARAGAN_BF16 || d->dtype == PARAGAN_F32, "qknorm: dtype must be PARAGAN_BF16 or PARAGAN_F32");
  // a smaller one is zero to the reciprocal root: infinity, and NaN where a row is zero or padding
  PG_CHECK(d->eps >= FLT_MIN && std::isfinite(d->eps), "qknorm: eps must be > 0 and no smaller than the least normal float");
  const int64_t wq = (int64_t)d->Hq * d->d, wk = (int64_t)d->Hk * d->d;
  PG_CHECK(d->ldq >= wq && d->ldqo >= wq && d->ldk >= wk && d->ldko >= wk, "qknorm: a token stride is below heads * d");
  PG_CHECK(d->ldq % 8 == 0 && d->ldqo % 8 == 0 && d->ldk % 8 == 0 && d->ldko % 8 == 0,
           "qknorm: token strides must be multiples of 8");
  for (int64_t ld : {d->ldq, d->ldqo, d->ldk, d->ldko})
    PG_CHECK(ld < (1LL << 60) / d->T, "qknorm: a token stride is too large");
  QkNorm a;
  a.T = d->T; a.Hq = d->Hq; a.Hk = d->Hk; a.d = d->d; a.rot = d->rot; a.n_pos = d->n_pos;
  a.inter = d->interleaved == 1; a.f32 = d->dtype == PARAGAN_F32; a.eps = d->eps;
  a.ldq = d->ldq; a.ldk = d->ldk; a.ldqo = d->ldqo; a.ldko = d->ldko;
  return a;
}

extern "C" int paragan_qknorm_check(const paragan_qknorm_desc* d) { PG_TRY(nullptr, make_qk(d)) }

extern "C" int paragan_qknorm_ws_size(const paragan_qknorm_desc* d, size_t* ws_bytes) {
  PG_TRY(nullptr, {
    need(ws_bytes, "ws_bytes");
    *ws_bytes = qknorm_ws_bytes(make_qk(d));
  })
}

extern "C" int paragan_qknorm_fwd(paragan_ctx* ctx, const paragan_qknorm_desc* d, const void* q, const void* k,
                                  const float* gain_q, const float* gain_k, const float* table, const int32_t* pos,
                                  void* qo, void* ko) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    const QkNorm a = make_qk(d);
    need16(q, "q"); need16(k, "k"); need(gain_q, "gain_q"); need(gain_k, "gain_k");
    if (a.rot) need16(table, "table");
    need16(qo, "qo"); need16(ko, "ko");
    on_device(ctx, "qknorm_fwd");
    qknorm_fwd(ctx->stream, a, q, k, gain_q, gain_k, table, pos, qo, ko);
  })
}

extern "C" int paragan_qknorm_bwd(paragan_ctx* ctx, const paragan_qknorm_desc* d, const void* q, const void* k,
                                  const float* gain_q, const float* gain_k, const float* table, const int32_t* pos,
                                  const void* dqo, const void* dko, void* dq, void* dk, float* dgain_q,
                                  float* dgain_k, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    const QkNorm a = make_qk(d);
    need16(q, "q"); need16(k, "k"); need(gain_q, "gain_q"); need(gain_k, "gain_k");
    if (a.rot) need16(table, "table");
    need16(dqo, "dqo"); need16(dko, "dko"); need16(dq, "dq"); need16(dk, "dk");
    need(dgain_q, "dgain_q"); need(dgain_k, "dgain_k"); need(ws, "ws");
    aligned(ws, "ws");
    on_device(ctx, "qknorm_bwd");
    qknorm_bwd(ctx->stream, a, q, k, gain_q, gain_k, table, pos, dqo, dko, dq, dk, dgain_q, dgain_k, ws);
  })
}

// Does (b, s, h, c) -> address hit every element of a tensor once?  Strides in
// ascending order each have to step over all that lies inside.
static bool distinct(const int64_t* stride, int64_t B, int64_t S, int64_t H, int64_t d) {
  std::pair<int64_t, int64_t> e[3] = {{stride[0], B}, {stride[1], S}, {stride[2], H}};
  std::sort(e, e + 3);
  __int128 inner = d;
  for (const auto& x : e) {
    if (x.second == 1) continue;
    if (x.first < inner) return false;
    inner += (__int128)x.first * (x.second - 1);
  }
  return true;
}

static Mha make_mha(const paragan_mha_desc* d) {
  if (!d) throw Error{PARAGAN_EINVAL, "mha: desc is NULL"};
  const int32_t big = 1 << 29;   // sums of three positions stay in 32 bits
  PG_CHECK(d->B >= 1 && d->Sq >= 1 && d->Sk >= 1 && d->Sq <= big && d->Sk <= big, "mha: B, Sq, Sk must be >= 1 and Sq, Sk <= 2^29");
  PG_CHECK(d->Hq >= 1 && d->Hk >= 1 && d->Hq % d->Hk == 0, "mha: Hq must be a multiple of Hk >= 1");
  PG_CHECK(d->d >= 8 && d->d <= 128 && d->d % 8 == 0, "mha: d must be a multiple of 8 up to 128");
  PG_CHECK(d->causal == 0 || d->causal == 1, "mha: causal must be 0 or 1");
  PG_CHECK(d->window >= 0 && d->window <= big && d->n_sink >= 0 && d->n_sink <= big, "mha: window, n_sink must be 0 .. 2^29");
  if (d->n_buckets != 0) {
    const int side = d->causal ? d->n_buckets : d->n_buckets / 2;
    PG_CHECK(d->n_buckets > 0 && d->n_buckets <= 256 && side >= 2 && (d->causal || d->n_buckets % 2 == 0),
             "mha: n_buckets must be 2 .. 256 (not causal: even, 4 .. 256)");
    PG_CHECK(d->max_distance > side / 2 && d->max_distance <= kMhaMaxDist,
             "mha: max_distance must be above half of a side's buckets and at most 512");
  }
  PG_CHECK(d->scale >= 1e-30f && d->scale <= 1e30f, "mha: scale must be 1e-30 .. 1e30");
  // a launch has fewer than 2^32 threads: blocks of 256 threads, at least 128 rows of one head in each
  PG_CHECK((int64_t)d->B * d->Hq < (1 << 24) && (int64_t)d->B * d->Hq * cdiv(d->Sq, 128) < (1 << 24) &&
               (int64_t)d->B * d->Hk * cdiv(d->Sk, 128) < (1 << 24),
           "mha: too many rows (B * heads * S / 128 must stay below 2^24)");
  Mha m;
  m.B = d->B; m.Sq = d->Sq; m.Sk = d->Sk; m.Hq = d->Hq; m.Hk = d->Hk; m.d = d->d; m.causal = d->causal == 1;
  m.window = d->window; m.n_sink = d->n_sink; m.n_buckets = d->n_buckets; m.max_distance = d->max_distance;
  m.scale = d->scale;
  for (int i = 0; i < 3; ++i) {
    m.qs[i] = d->q_stride[i]; m.ks[i] = d->k_stride[i]; m.vs[i] = d->v_stride[i]; m.os[i] = d->o_stride[i];
    const int64_t n[4][3] = {{m.B, m.Sq, m.Hq}, {m.B, m.Sk, m.Hk}, {m.B, m.Sk, m.Hk}, {m.B, m.Sq, m.Hq}};
    const int64_t st[4] = {m.qs[i], m.ks[i], m.vs[i], m.os[i]};
    for (int t = 0; t < 4; ++t) {
      PG_CHECK(st[t] >= 0 && st[t] % 8 == 0, "mha: strides must be >= 0 and multiples of 8");
      PG_CHECK((__int128)st[t] * (n[t][i] - 1) < ((__int128)1 << 60), "mha: a stride is too large");
    }
  }
  for (int64_t t : {m.qs[1], m.ks[1], m.vs[1], m.os[1]})   // a tile of 64 tokens is addressed in 32 bits
    PG_CHECK(t < (1LL << 24), "mha: a token stride is 2^24 or more");
  PG_CHECK(distinct(m.os, m.B, m.Sq, m.Hq, m.d), "mha: o overlaps itself");
  return m;
}

extern "C" int paragan_mha_check(const paragan_mha_desc* d) { PG_TRY(nullptr, make_mha(d)) }

extern "C" int paragan_mha_sizes(const paragan_mha_desc* d, size_t* saved, size_t* ws) {
  PG_TRY(nullptr, {
    const Mha m = make_mha(d);
    if (saved) *saved = mha_saved_bytes(m);
    if (ws) *ws = mha_ws_bytes(m);
  })
}

extern "C" int paragan_mha_fwd(paragan_ctx* ctx, const paragan_mha_desc* d, const void* q, const void* k,
                               const void* v, const float* table, const int32_t* len_q, const int32_t* len_k,
                               void* o, void* saved, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    const Mha m = make_mha(d);
    need16(q, "q"); need16(k, "k"); need16(v, "v"); need16(o, "o"); need(ws, "ws");
    if (m.n_buckets) need(table, "table");
    aligned(ws, "ws");
    if (saved) aligned(saved, "saved");
    on_device(ctx, "mha_fwd");
    mha_fwd(ctx->stream, m, q, k, v, table, len_q, len_k, o, saved, ws);
  })
}

extern "C" int paragan_mha_bwd(paragan_ctx* ctx, const paragan_mha_desc* d, const void* q, const void* k,
                               const void* v, const float* table, const int32_t* len_q, const int32_t* len_k,
                               const void* o, const void* saved, const void* dout, void* dq, void* dk, void* dv,
                               float* dtable, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    const Mha m = make_mha(d);
    PG_CHECK(distinct(m.qs, m.B, m.Sq, m.Hq, m.d) && distinct(m.ks, m.B, m.Sk, m.Hk, m.d) &&
                 distinct(m.vs, m.B, m.Sk, m.Hk, m.d),
             "mha_bwd: q, k or v overlaps itself (dq, dk, dv share their strides)");
    need16(q, "q"); need16(k, "k"); need16(v, "v"); need16(o, "o"); need(saved, "saved"); need16(dout, "dout");
    need16(dq, "dq"); need16(dk, "dk"); need16(dv, "dv"); need(ws, "ws");
    if (m.n_buckets) { need(table, "table"); need(dtable, "dtable"); }
    aligned(saved, "saved"); aligned(ws, "ws");
    on_device(ctx, "mha_bwd");
    mha_bwd(ctx->stream, m, q, k, v, table, len_q, len_k, o, saved, dout, dq, dk, dv, dtable, ws);
  })
}

// ------------------------------------------------------------ token block: norms with modulation, recurrence, clipping
// (b, s) strides of a tensor of B x S rows of D elements
static void token_strides(const int64_t* st, int64_t* out, int64_t B, int64_t S, const char* what) {
  for (int i = 0; i < 2; ++i) {
    if (st[i] < 0 || st[i] % 8 != 0)
      throw Error{PARAGAN_EINVAL, std::string(what) + ": strides must be >= 0 and multiples of 8"};
    if ((__int128)st[i] * (i ? S : B) >= ((__int128)1 << 60))
      throw Error{PARAGAN_EINVAL, std::string(what) + ": a stride is too large"};
    out[i] = st[i];
  }
}
static bool rows_distinct(const int64_t* st, int64_t B, int64_t S, int64_t D) {
  const int64_t s[3] = {st[0], st[1], 0};
  return distinct(s, B, S, 1, D);
}

static BlockNorm make_bn(const paragan_blocknorm_desc* d) {
  if (!d) throw Error{PARAGAN_EINVAL, "blocknorm: desc is NULL"};
  PG_CHECK(d->B >= 1 && d->S >= 1 && (int64_t)d->B * d->S <= (1LL << 30), "blocknorm: B, S must be >= 1 and B * S at most 2^30");
  PG_CHECK(d->B <= (1 << 20), "blocknorm: B is more than 2^20");   // a block of up to 1024 threads each
  PG_CHECK(d->D >= 8 && d->D <= 8192 && d->D % 8 == 0, "blocknorm: D must be a multiple of 8 up to 8192");
  PG_CHECK(d->dtype == PARAGAN_BF16 || d->dtype == PARAGAN_F32, "blocknorm: dtype must be PARAGAN_BF16 or PARAGAN_F32");
  PG_CHECK(d->stream_dtype == PARAGAN_F32 || d->stream_dtype == d->dtype,
           "blocknorm: stream_dtype must be dtype or PARAGAN_F32");
  PG_CHECK(d->kind == PARAGAN_NORM_RMS || d->kind == PARAGAN_NORM_LAYER,
           "blocknorm: kind must be PARAGAN_NORM_RMS or PARAGAN_NORM_LAYER");
  for (int32_t f : {d->branch, d->post, d->pre}) PG_CHECK(f == 0 || f == 1, "blocknorm: branch, post, pre must be 0 or 1");
  PG_CHECK(d->branch || d->pre, "blocknorm: neither branch nor pre leaves nothing to do");
  PG_CHECK(d->branch || !d->post, "blocknorm: post needs a branch");
  PG_CHECK(d->eps >= FLT_MIN && std::isfinite(d->eps), "blocknorm: eps must be > 0 and no smaller than the least normal float");
  PG_CHECK(std::isfinite(d->res_scale), "blocknorm: res_scale must be finite");
  PG_CHECK(d->mod_stride == 0 || (d->mod_stride >= d->D && d->mod_stride % 8 == 0 && d->mod_stride < (1LL << 60) / d->B),
           "blocknorm: mod_stride must be 0, or >= D and a multiple of 8");
  BlockNorm a;
  a.B = d->B; a.S = d->S; a.D = d->D; a.f32 = d->dtype == PARAGAN_F32; a.res32 = d->stream_dtype == PARAGAN_F32;
  a.layer = d->kind == PARAGAN_NORM_LAYER; a.branch = d->branch; a.post = d->post; a.pre = d->pre;
  a.eps = d->eps; a.res_scale = d->res_scale; a.mod = d->mod_stride;
  token_strides(d->x_stride, a.xs, a.B, a.S, "blocknorm: x");
  token_strides(d->h_stride, a.hs, a.B, a.S, "blocknorm: h");
  token_strides(a.branch ? d->z_stride : d->x_stride, a.zs, a.B, a.S, "blocknorm: z");
  token_strides(d->y_stride, a.ys, a.B, a.S, "blocknorm: y");
  PG_CHECK(!a.branch || rows_distinct(a.zs, a.B, a.S, a.D), "blocknorm: z overlaps itself");
  PG_CHECK(!a.pre || rows_distinct(a.ys, a.B, a.S, a.D), "blocknorm: y overlaps itself");
  return a;
}
// The rows that the descriptor uses: the others are not read, nor do they enter any gradient
static BlockNormRows bn_rows(const BlockNorm& a, const float* gain_post, const float* gate, const float* gain_pre,
                             const float* scale, const float* shift) {
  const float* p[5] = {gain_post, gate, gain_pre, scale, shift};
  const char* n[5] = {"gain_post", "gate", "gain_pre", "scale", "shift"};
  for (int i = 0; i < 5; ++i)
    if (p[i]) need16(p[i], n[i]);
  return BlockNormRows{a.post ? gain_post : nullptr, a.branch ? gate : nullptr, a.pre ? gain_pre : nullptr,
                       a.pre ? scale : nullptr, a.pre ? shift : nullptr};
}

extern "C" int paragan_blocknorm_check(const paragan_blocknorm_desc* d) { PG_TRY(nullptr, make_bn(d)) }

extern "C" int paragan_blocknorm_sizes(const paragan_blocknorm_desc* d, size_t* saved, size_t* ws) {
  PG_TRY(nullptr, {
    const BlockNorm a = make_bn(d);
    if (saved) *saved = blocknorm_saved_bytes(a);
    if (ws) *ws = blocknorm_ws_bytes(a);
  })
}

extern "C" int paragan_blocknorm_fwd(paragan_ctx* ctx, const paragan_blocknorm_desc* d, const void* x, const void* h,
                                     const float* gain_post, const float* gate, const float* gain_pre,
                                     const float* scale, const float* shift, const int32_t* len, void* z, void* y,
                                     void* saved) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    const BlockNorm a = make_bn(d);
    const BlockNormRows w = bn_rows(a, gain_post, gate, gain_pre, scale, shift);
    need16(x, "x");
    if (a.branch) { need16(h, "h"); need16(z, "z"); }
    if (a.pre) need16(y, "y");
    if (saved) aligned(saved, "saved");
    on_device(ctx, "blocknorm_fwd");
    blocknorm_fwd(ctx->stream, a, w, x, h, len, z, y, saved);
  })
}

extern "C" int paragan_blocknorm_bwd(paragan_ctx* ctx, const paragan_blocknorm_desc* d, const void* x, const void* h,
                                     const float* gain_post, const float* gate, const float* gain_pre,
                                     const float* scale, const float* shift, const int32_t* len, const void* saved,
                                     const void* dz, const void* dy, void* dx, void* dh, float* dgain_post,
                                     float* dgate, float* dgain_pre, float* dscale, float* dshift, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    const BlockNorm a = make_bn(d);
    const BlockNormRows w = bn_rows(a, gain_post, gate, gain_pre, scale, shift);
    PG_CHECK(rows_distinct(a.xs, a.B, a.S, a.D) && (!a.branch || rows_distinct(a.hs, a.B, a.S, a.D)),
             "blocknorm_bwd: x or h overlaps itself (dx and dh share their strides)");
    need16(x, "x"); need16(dx, "dx");
    if (a.branch) { need16(h, "h"); need16(dh, "dh"); }
    if (a.pre) need16(dy, "dy");
    PG_CHECK(a.pre || dz, "blocknorm_bwd: dz is NULL and there is no y");
    if (dz) need16(dz, "dz");
    PG_CHECK(a.branch || (!dgate && !dgain_post), "blocknorm_bwd: dgate, dgain_post need a branch");
    PG_CHECK(a.post || !dgain_post, "blocknorm_bwd: dgain_post needs post");
    PG_CHECK(a.pre || (!dgain_pre && !dscale && !dshift), "blocknorm_bwd: dgain_pre, dscale, dshift need pre");
    need(saved, "saved"); need(ws, "ws");
    aligned(saved, "saved"); aligned(ws, "ws");
    on_device(ctx, "blocknorm_bwd");
    blocknorm_bwd(ctx->stream, a, w, x, h, len, saved, dz, dy, dx, dh,
                  BlockNormGrads{dgain_post, dgate, dgain_pre, dscale, dshift}, ws);
  })
}

static Scan make_scan(const paragan_scan_desc* d) {
  if (!d) throw Error{PARAGAN_EINVAL, "scan: desc is NULL"};
  PG_CHECK(d->B >= 1 && d->S >= 1 && (int64_t)d->B * d->S <= (1LL << 30), "scan: B, S must be >= 1 and B * S at most 2^30");
  PG_CHECK(d->D >= 8 && d->D <= (1 << 20) && d->D % 8 == 0 && (int64_t)d->B * d->D < (1LL << 31),
           "scan: D must be a multiple of 8 up to 2^20 and B * D below 2^31");
  PG_CHECK(d->B * cdiv(d->D, 64) <= (1 << 22), "scan: more than 2^22 sequences of 64 channels");   // a block of up to 512 threads each
  PG_CHECK(d->dtype == PARAGAN_BF16 || d->dtype == PARAGAN_F32, "scan: dtype must be PARAGAN_BF16 or PARAGAN_F32");
  PG_CHECK(d->reverse == 0 || d->reverse == 1, "scan: reverse must be 0 or 1");
  PG_CHECK(d->sharp > 0.f && std::isfinite(d->sharp), "scan: sharp must be > 0 and finite");
  Scan a;
  a.B = d->B; a.S = d->S; a.D = d->D; a.f32 = d->dtype == PARAGAN_F32; a.reverse = d->reverse == 1; a.sharp = d->sharp;
  token_strides(d->x_stride, a.xs, a.B, a.S, "scan: x");
  token_strides(d->r_stride, a.rs, a.B, a.S, "scan: r");
  token_strides(d->g_stride, a.gs, a.B, a.S, "scan: g");
  token_strides(d->y_stride, a.ys, a.B, a.S, "scan: y");
  for (int64_t t : {a.xs[1], a.rs[1], a.gs[1], a.ys[1]})   // a tile of up to 128 tokens is addressed in 32 bits
    PG_CHECK(t < (1LL << 20), "scan: a token stride is 2^20 or more");
  PG_CHECK(rows_distinct(a.ys, a.B, a.S, a.D), "scan: y overlaps itself");
  return a;
}

extern "C" int paragan_scan_check(const paragan_scan_desc* d) { PG_TRY(nullptr, make_scan(d)) }

extern "C" int paragan_scan_sizes(const paragan_scan_desc* d, size_t* saved, size_t* ws) {
  PG_TRY(nullptr, {
    const Scan a = make_scan(d);
    if (saved) *saved = scan_saved_bytes(a);
    if (ws) *ws = scan_ws_bytes(a);
  })
}

extern "C" int paragan_scan_fwd(paragan_ctx* ctx, const paragan_scan_desc* d, const void* x, const void* r,
                                const void* g, const float* decay, const int32_t* len, const float* h0, void* y,
                                float* ht, void* saved, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    const Scan a = make_scan(d);
    need16(x, "x"); need16(r, "r"); need16(g, "g"); need16(decay, "decay"); need16(y, "y"); need(ws, "ws");
    if (h0) need16(h0, "h0");
    if (ht) need16(ht, "ht");
    aligned(ws, "ws");
    if (saved) aligned(saved, "saved");
    on_device(ctx, "scan_fwd");
    scan_fwd(ctx->stream, a, x, r, g, decay, len, h0, y, ht, saved, ws);
  })
}

extern "C" int paragan_scan_bwd(paragan_ctx* ctx, const paragan_scan_desc* d, const void* x, const void* r,
                                const void* g, const float* decay, const int32_t* len, const void* saved,
                                const void* dy, const float* dht, void* dx, void* dr, void* dg, float* ddecay,
                                float* dh0, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    const Scan a = make_scan(d);
    PG_CHECK(rows_distinct(a.xs, a.B, a.S, a.D) && rows_distinct(a.rs, a.B, a.S, a.D) && rows_distinct(a.gs, a.B, a.S, a.D),
             "scan_bwd: x, r or g overlaps itself (dx, dr, dg share their strides)");
    need16(x, "x"); need16(r, "r"); need16(g, "g"); need16(decay, "decay"); need16(dy, "dy");
    need16(dx, "dx"); need16(dr, "dr"); need16(dg, "dg"); need(ddecay, "ddecay");
    if (dht) need16(dht, "dht");
    if (dh0) need16(dh0, "dh0");
    need(saved, "saved"); need(ws, "ws");
    aligned(saved, "saved"); aligned(ws, "ws");
    on_device(ctx, "scan_bwd");
    scan_bwd(ctx->stream, a, x, r, g, decay, len, saved, dy, dht, dx, dr, dg, ddecay, dh0, ws);
  })
}

// The pieces of all tensors, and what is wrong with the list
static paragan_clip_desc clip_desc(const paragan_clip_tensor* t, int32_t n) {
  if (!t) throw Error{PARAGAN_EINVAL, "clip: the tensors are NULL"};
  PG_CHECK(n >= 1, "clip: n_tensors must be >= 1");
  paragan_clip_desc d{};
  d.n_tensors = n;
  d.in_place = 1;
  struct Span { uint64_t at, end; };
  std::vector<Span> spans;
  for (int32_t i = 0; i < n; ++i) {
    PG_CHECK(t[i].dtype == PARAGAN_BF16 || t[i].dtype == PARAGAN_F32, "clip: dtype must be PARAGAN_BF16 or PARAGAN_F32");
    PG_CHECK(t[i].reserved == 0, "clip: reserved must be 0");
    PG_CHECK(t[i].n >= 0 && t[i].n <= (1LL << 40), "clip: n must be 0 .. 2^40");
    if (t[i].n == 0) continue;
    const uint64_t el = t[i].dtype == PARAGAN_BF16 ? 2 : 4, g = (uint64_t)(uintptr_t)t[i].grad, o = (uint64_t)(uintptr_t)t[i].out;
    PG_CHECK(g && o, "clip: a gradient or output is NULL");
    PG_CHECK(g % el == 0 && o % el == 0, "clip: a gradient or output is not aligned to its type");
    spans.push_back({g, g + el * (uint64_t)t[i].n});
    if (o != g) {
      spans.push_back({o, o + el * (uint64_t)t[i].n});
      d.in_place = 0;
    }
    d.n_elements += t[i].n;
    d.bytes += (int64_t)el * t[i].n;
    d.n_pieces += cdiv(t[i].n, kClipPiece / (int64_t)el);
    PG_CHECK(d.n_pieces < (1LL << 31), "clip: too many elements");
  }
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.at < b.at; });
  for (size_t i = 1; i < spans.size(); ++i)
    PG_CHECK(spans[i].at >= spans[i - 1].end, "clip: two tensors overlap (a gradient named twice, or an output on another)");
  return d;
}

extern "C" int paragan_clip_sizes(const paragan_clip_tensor* t, int32_t n, size_t* plan_bytes, size_t* ws_bytes) {
  PG_TRY(nullptr, {
    const paragan_clip_desc d = clip_desc(t, n);
    if (plan_bytes) *plan_bytes = (size_t)d.n_pieces * sizeof(ClipPiece);
    if (ws_bytes) *ws_bytes = clip_ws_bytes();
  })
}

extern "C" int paragan_clip_plan(const paragan_clip_tensor* t, int32_t n, paragan_clip_desc* desc, void* plan_host) {
  PG_TRY(nullptr, {
    need(desc, "desc");
    const paragan_clip_desc d = clip_desc(t, n);
    if (d.n_pieces) need(plan_host, "plan_host");
    ClipPiece* out = (ClipPiece*)plan_host;
    for (int32_t i = 0; i < n; ++i) {
      const uint64_t el = t[i].dtype == PARAGAN_BF16 ? 2 : 4;
      const int64_t per = kClipPiece / (int64_t)el;
      for (int64_t at = 0; at < t[i].n; at += per) {
        const ClipPiece p{(uint64_t)(uintptr_t)t[i].grad + el * at, (uint64_t)(uintptr_t)t[i].out + el * at,
                          (int32_t)std::min<int64_t>(per, t[i].n - at), (int32_t)(t[i].dtype == PARAGAN_BF16)};
        std::memcpy(out++, &p, sizeof(p));
      }
    }
    *desc = d;
  })
}

extern "C" int paragan_clip(paragan_ctx* ctx, const paragan_clip_desc* d, const void* plan, float max_norm,
                            float grad_scale, float* norm, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    if (!d) throw Error{PARAGAN_EINVAL, "clip: desc is NULL"};
    PG_CHECK(d->n_tensors >= 1 && d->n_pieces >= 0 && d->n_pieces < (1LL << 31) && (d->in_place == 0 || d->in_place == 1),
             "clip: desc is not one of paragan_clip_plan");
    if (d->n_pieces) need(plan, "plan");
    PG_CHECK(((uintptr_t)plan & 7) == 0, "clip: plan is not 8-byte aligned");
    PG_CHECK(max_norm > 0.f, "clip: max_norm must be > 0");
    PG_CHECK(grad_scale > 0.f && std::isfinite(grad_scale), "clip: grad_scale must be > 0 and finite");
    need(norm, "norm"); need(ws, "ws");
    aligned(ws, "ws");
    on_device(ctx, "clip");
    clip(ctx->stream, d->n_pieces, (double)d->bytes, d->in_place == 1, plan, max_norm, grad_scale, norm, ws);
  })
}

// ------------------------------------------------------------ generator output layer
static void ocheck(const paragan_gout_desc* d) {
  if (!d) throw Error{PARAGAN_EINVAL, "gout: desc is NULL"};
  PG_CHECK(d->B >= 1 && d->H >= 1 && d->W >= 1 && d->C >= 1, "gout: B, H, W, C >= 1");
  PG_CHECK(ghead_shape_ok(d->W, d->C), "gout: needs cpad(C) <= 128, W a multiple of 4 and W small enough for the "
                                       "weight-gradient tile");
  PG_CHECK(d->n_power_iter >= 1 && d->bn_eps > 0.f && d->sn_eps > 0.f, "gout: bad n_power_iter / eps");
  PG_CHECK((int64_t)d->B * d->H * d->W < (1LL << 31), "gout: too many pixels");
}

static GOut make_o(const paragan_gout_desc* d) {
  GOut g;
  g.B = d->B; g.H = d->H; g.W = d->W; g.C = d->C; g.npi = d->n_power_iter;
  g.bn_eps = d->bn_eps; g.sn_eps = d->sn_eps;
  return g;
}

extern "C" int paragan_gout_check(const paragan_gout_desc* d) { PG_TRY(nullptr, ocheck(d)) }

extern "C" int paragan_gout_layout(const paragan_gout_desc* d, paragan_tensor_info* out, int32_t cap,
                                   int32_t* count, int64_t* n_params, int64_t* n_u) {
  try {
    ocheck(d);
    return export_layout(gout_layout(d->C), out, cap, count, n_params, n_u);
  } catch (const Error& e) {
    return fail(nullptr, e.code, e.msg);
  }
}

extern "C" int paragan_gout_sizes(const paragan_gout_desc* d, size_t* saved, size_t* ws) {
  PG_TRY(nullptr, {
    ocheck(d);
    GOut g = make_o(d);
    Arena a(nullptr);
    g.plan_saved(a);
    if (saved) *saved = a.off;
    if (ws) *ws = g.ws_size();
  })
}

extern "C" int paragan_gout_fwd(paragan_ctx* ctx, const paragan_gout_desc* d, const float* params, float* u,
                                const void* x, float* img, void* saved, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    ocheck(d);
    need(params, "params"); need(u, "u"); need(x, "x"); need(img, "img"); need(saved, "saved"); need(ws, "ws");
    aligned(saved, "saved"); aligned(ws, "ws");
    GOut g = make_o(d);
    Arena a(saved);
    g.plan_saved(a);
    Layout L = gout_layout(d->C);
    Params P{&L, "", params, u, nullptr};
    g.fwd(Exec{ctx->stream, ctx->n_cu, ws, g.ws_size()}, P, x, img);
  })
}

extern "C" int paragan_gout_bwd(paragan_ctx* ctx, const paragan_gout_desc* d, const float* params, const void* x,
                                const float* img, const void* saved, const float* dimg, void* dx, float* grads,
                                void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    ocheck(d);
    need(params, "params"); need(x, "x"); need(img, "img"); need(saved, "saved"); need(dimg, "dimg");
    need(dx, "dx"); need(grads, "grads"); need(ws, "ws");
    aligned(saved, "saved"); aligned(ws, "ws");
    GOut g = make_o(d);
    Arena a((void*)saved);
    g.plan_saved(a);
    Layout L = gout_layout(d->C);
    Params P{&L, "", params, nullptr, grads};
    g.bwd(Exec{ctx->stream, ctx->n_cu, ws, g.ws_size()}, P, x, img, dimg, 3, dx);
  })
}

// ------------------------------------------------------------ networks, step
extern "C" int paragan_biggan_check(const paragan_biggan_desc* d) { PG_TRY(nullptr, check_arch(d)) }

extern "C" int paragan_net_layout(const paragan_biggan_desc* d, int32_t which, paragan_tensor_info* out,
                                  int32_t cap, int32_t* count, int64_t* n_params, int64_t* n_u) {
  try {
    check_arch(d);
    PG_CHECK(which == 0 || which == 1, "net_layout: which must be 0 (G) or 1 (D)");
    const Arch a = arch_from(d);
    return export_layout(which == 0 ? g_layout(a) : d_layout(a), out, cap, count, n_params, n_u);
  } catch (const Error& e) {
    return fail(nullptr, e.code, e.msg);
  }
}

extern "C" int paragan_train_step_ws_size(const paragan_biggan_desc* d, size_t* ws_bytes) {
  PG_TRY(nullptr, {
    check_arch(d);
    need(ws_bytes, "ws_bytes");
    *ws_bytes = train_step_ws(d, device_cus());
  })
}

static void need_state(const paragan_net_state* s, const char* who) {
  need(s, who);
  need(s->params, "params"); need(s->u, "u"); need(s->grads, "grads");
  need(s->opt_m, "opt_m"); need(s->opt_v, "opt_v");
  PG_CHECK(s->opt_t >= 0, "opt_t must be >= 0");
}

static int finish_losses(paragan_ctx* ctx, const float* losses, int n, const char* who) {
  for (int k = 0; k < n; ++k)
    if (!std::isfinite(losses[k])) return fail(ctx, PARAGAN_ENONFINITE, std::string(who) + ": non-finite loss");
  return PARAGAN_OK;
}

#define PG_STEP_TRY(ctx, ...)                              \
  try {                                                    \
    __VA_ARGS__;                                           \
  } catch (const ::pg::Error& e) {                         \
    return fail(ctx, e.code, e.msg);                       \
  } catch (const std::exception& e) {                      \
    return fail(ctx, PARAGAN_EINVAL, e.what());            \
  }

extern "C" int paragan_g_sample(paragan_ctx* ctx, const paragan_biggan_desc* d, paragan_net_state* G,
                                const float* z, const int32_t* y, float* img, void* ws) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_TRY(ctx, {
    check_arch(d);
    need_state(G, "G");
    need(z, "z"); need(y, "y"); need(img, "img"); need(ws, "ws");
    aligned(ws, "ws");
    g_sample(ctx, d, G, z, y, img, ws);
  })
}

extern "C" int paragan_d_step(paragan_ctx* ctx, const paragan_biggan_desc* d, paragan_net_state* D,
                              const float* x_real, const int32_t* y_real, const float* x_fake,
                              const int32_t* y_fake, void* ws, float* loss_host) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_STEP_TRY(ctx, {
    check_arch(d);
    need_state(D, "D");
    need(x_real, "x_real"); need(y_real, "y_real"); need(x_fake, "x_fake"); need(y_fake, "y_fake");
    need(ws, "ws"); need(loss_host, "loss_host");
    aligned(ws, "ws");
    d_step(ctx, d, D, x_real, y_real, x_fake, y_fake, ws, loss_host);
  })
  return finish_losses(ctx, loss_host, 1, "d_step");
}

extern "C" int paragan_g_step(paragan_ctx* ctx, const paragan_biggan_desc* d, paragan_net_state* G,
                              paragan_net_state* D, const float* z, const int32_t* y, void* ws, float* loss_host) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_STEP_TRY(ctx, {
    check_arch(d);
    need_state(G, "G");
    need_state(D, "D");
    need(z, "z"); need(y, "y"); need(ws, "ws"); need(loss_host, "loss_host");
    aligned(ws, "ws");
    g_step(ctx, d, G, D, z, y, ws, loss_host);
  })
  return finish_losses(ctx, loss_host, 1, "g_step");
}

extern "C" int paragan_train_step(paragan_ctx* ctx, const paragan_biggan_desc* d, paragan_net_state* G,
                                  paragan_net_state* D, const paragan_step_inputs* in, int32_t n_D, void* ws,
                                  float* losses_host) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_STEP_TRY(ctx, {
    check_arch(d);
    need_state(G, "G");
    need_state(D, "D");
    need(in, "inputs"); need(ws, "ws"); need(losses_host, "losses_host");
    aligned(ws, "ws");
    PG_CHECK(n_D >= 1 && n_D <= 63, "train_step: n_D must be in [1, 63]");
    need(in->x_real, "x_real"); need(in->y_real, "y_real"); need(in->z_fake, "z_fake"); need(in->y_fake, "y_fake");
    for (int k = 0; k < n_D; ++k) {
      need(in->x_real[k], "x_real[k]"); need(in->y_real[k], "y_real[k]");
      need(in->z_fake[k], "z_fake[k]"); need(in->y_fake[k], "y_fake[k]");
    }
    need(in->z_g, "z_g"); need(in->y_g, "y_g");
    train_step(ctx, d, G, D, in, n_D, ws, losses_host);
  })
  return finish_losses(ctx, losses_host, n_D + 1, "train_step");
}

extern "C" int paragan_async_ws_size(const paragan_biggan_desc* d, int32_t n_D, size_t* ws_bytes) {
  PG_TRY(nullptr, {
    check_arch(d);
    need(ws_bytes, "ws_bytes");
    PG_CHECK(n_D >= 1 && n_D <= 63, "async_ws_size: n_D must be in [1, 63]");
    *ws_bytes = async_step_ws(d, n_D, device_cus());
  })
}

extern "C" int paragan_async_step(paragan_ctx* ctx, const paragan_biggan_desc* d, paragan_net_state* G,
                                  paragan_net_state* D, const paragan_async_inputs* in, int32_t n_D, void* ws,
                                  float* losses_host) {
  if (!ctx) return PARAGAN_EINVAL;
  ProfBind pb(ctx);
  PG_STEP_TRY(ctx, {
    check_arch(d);
    need_state(G, "G");
    need_state(D, "D");
    need(in, "inputs"); need(ws, "ws"); need(losses_host, "losses_host");
    aligned(ws, "ws");
    PG_CHECK(n_D >= 1 && n_D <= 63, "async_step: n_D must be in [1, 63]");
    PG_CHECK((int64_t)n_D * d->B * d->img * d->img < (1LL << 31), "async_step: generator batch n_D * B too large");
    need(in->x_real, "x_real"); need(in->y_real, "y_real");
    for (int k = 0; k < n_D; ++k) { need(in->x_real[k], "x_real[k]"); need(in->y_real[k], "y_real[k]"); }
    need(in->z, "z"); need(in->y, "y");
    need(in->img_buff, "img_buff"); need(in->lab_buff, "lab_buff"); need(in->pred_buff, "pred_buff");
    async_step(ctx, d, G, D, in, n_D, ws, losses_host);
  })
  return finish_losses(ctx, losses_host, n_D + 1, "async_step");
}

// ------------------------------------------------------------ profiler
extern "C" int paragan_profile(paragan_ctx* ctx, int enable) {
  if (!ctx) return PARAGAN_EINVAL;
  ctx->prof.on = enable != 0;
  ctx->prof.detail = enable == 2;
  return PARAGAN_OK;
}

extern "C" int paragan_profile_read(paragan_ctx* ctx, paragan_kernel_stat* out, int32_t cap, int32_t* count) {
  if (!ctx) return PARAGAN_EINVAL;
  PG_TRY(ctx, {
    need(count, "count");
    PG_HIP(hipStreamSynchronize(ctx->stream));
    std::vector<paragan_kernel_stat> agg;
    for (auto& r : ctx->prof.recs) {
      float ms = 0.f;
      PG_HIP(hipEventElapsedTime(&ms, r.a, r.b));
      paragan_kernel_stat* k = nullptr;
      for (auto& x : agg)
        if (r.name == x.name) k = &x;
      if (!k) {
        agg.push_back(paragan_kernel_stat{});
        k = &agg.back();
        std::strncpy(k->name, r.name.c_str(), sizeof(k->name) - 1);
      }
      k->launches += 1;
      k->total_ms += ms;
      k->flops += r.flops;
      k->bytes += r.bytes;
      ctx->prof.pool.push_back(r.a);
      ctx->prof.pool.push_back(r.b);
    }
    ctx->prof.recs.clear();
    *count = (int32_t)agg.size();
    if (out)
      for (int32_t i = 0; i < *count && i < cap; ++i) out[i] = agg[i];
  })
}
