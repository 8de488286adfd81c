// Gated linear recurrence over the tokens of a sequence, every channel by
// itself, forward and backward.
//
//   la = -sharp softplus(decay) s,  s = sigmoid(r);   a = exp(la),  w = (1 - a^2)^1/2,
//   h_t = a_t h_{t-1} + u_t,  u = w sg x,  sg = sigmoid(g);   y = h.
// Backward, with E_t = dy_t + a_{t+1} E_{t+1} (the last also dht):
//   dla = E (a h_{t-1} - u a^2 / w^2);  dr = dla la (1 - s);
//   dg = E u (1 - sg);  dx = E w sg;
//   ddecay = -sharp sigmoid(decay) sum dla s;  dh0 = a_1 E_1.
#include "token.hpp"

namespace pg {

namespace {

constexpr int kStep = 16;          // tokens between two states that a forward keeps

struct ScArgs {
  const void *x, *r, *g, *dy;
  const float* decay;
  const int32_t* len;
  const float* h0;                 // backward: dht
  float* ht;                       // backward: dh0
  void *y, *dr, *dg;               // y; backward: dx in y
  float* saved;                    // [B][ceil(S / kStep)][D]: the state ahead of every kStep tokens
  double* part;                    // [B][D]: sums of dla s
  int64_t xs[2], rs[2], gs[2], ys[2];
  int S, D, reverse;
  float sharp;
};

// two channels as they lie in memory, and as floats
template <typename T> struct Two;
template <> struct Two<bf16_t> {
  uint32_t v;
  PG_DEV void load(const bf16_t* p) { v = *reinterpret_cast<const uint32_t*>(p); }
  PG_DEV float2 get() const { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
};
template <> struct Two<float> {
  float2 v;
  PG_DEV void load(const float* p) { v = *reinterpret_cast<const float2*>(p); }
  PG_DEV float2 get() const { return v; }
};
PG_DEV void st2f(bf16_t* p, float a, float b) { *reinterpret_cast<uint32_t*>(p) = f2bf2(a, b); }
PG_DEV void st2f(float* p, float a, float b) { *reinterpret_cast<float2*>(p) = make_float2(a, b); }

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// sigmoid(v) and 1 - sigmoid(v), both to the last digits
PG_DEV void sigmoid(float v, float& s, float& c) {
  const float e = __builtin_amdgcn_exp2f(-fabsf(v) * kLog2e), q = __builtin_amdgcn_rcpf(1.f + e), t = e * q;
  s = v >= 0.f ? q : t;
  c = v >= 0.f ? t : q;
}
// softplus(v) = log(1 + e^v)
PG_DEV float softplus(float v) { return log1pf(expf(-fabsf(v))) + fmaxf(v, 0.f); }

// a = 2^l2 and p = 1 - a^2 for l2 <= 0: a series where the difference would
// cancel.  p is held above zero, so that w = p p^-1/2 and 1 / p are finite.
PG_DEV void decay_of(float l2, float& a, float& p) {
  a = __builtin_amdgcn_exp2f(l2);
  const float t = l2 * (2.f * kLn2);
  float q = fmaf(t, 1.f / 720.f, 1.f / 120.f);
  q = fmaf(t, q, 1.f / 24.f);
  q = fmaf(t, q, 1.f / 6.f);
  q = fmaf(t, q, 0.5f);
  q = fmaf(t, q, 1.f);
  p = fmaxf(t > -0.25f ? -t * q : fmaf(-a, a, 1.f), 1.17549435e-38f);
}

// One thread takes two channels of one sequence through all its tokens.
template <typename T>
__global__ __launch_bounds__(64) void k_scan_seq_fwd(ScArgs a) {
  const int c = (blockIdx.y * 64 + threadIdx.x) * 2, b = blockIdx.x;
  if (c >= a.D) return;
  const int len = a.len ? min(max(a.len[b], 0), a.S) : a.S;
  const T* x = (const T*)a.x + b * a.xs[0] + c;
  const T* r = (const T*)a.r + b * a.rs[0] + c;
  const T* g = (const T*)a.g + b * a.gs[0] + c;
  T* y = (T*)a.y + b * a.ys[0] + c;
  const int64_t o = (int64_t)b * a.D + c;
  const float k0 = -a.sharp * softplus(a.decay[c]) * kLog2e, k1 = -a.sharp * softplus(a.decay[c + 1]) * kLog2e;
  float2 h = a.h0 ? *reinterpret_cast<const float2*>(a.h0 + o) : make_float2(0.f, 0.f);
  float* keep = a.saved ? a.saved + (int64_t)b * cdiv(a.S, kStep) * a.D + c : nullptr;
  for (int i0 = 0; i0 < len; i0 += kStep) {
    if (keep) *reinterpret_cast<float2*>(keep + (int64_t)(i0 / kStep) * a.D) = h;
    Two<T> xv[kStep], rv[kStep], gv[kStep];
#pragma unroll
    for (int i = 0; i < kStep; ++i) {
      const int j = min(i0 + i, len - 1), t = a.reverse ? len - 1 - j : j;
      xv[i].load(x + t * a.xs[1]);
      rv[i].load(r + t * a.rs[1]);
      gv[i].load(g + t * a.gs[1]);
    }
#pragma unroll
    for (int i = 0; i < kStep; ++i) {
      if (i0 + i >= len) break;
      const float2 xx = xv[i].get(), rr = rv[i].get(), gg = gv[i].get();
      float s, c1, sg, a0, p;
      sigmoid(rr.x, s, c1);
      sigmoid(gg.x, sg, c1);
      decay_of(k0 * s, a0, p);
      h.x = fmaf(a0, h.x, p * __builtin_amdgcn_rsqf(p) * sg * xx.x);
      sigmoid(rr.y, s, c1);
      sigmoid(gg.y, sg, c1);
      decay_of(k1 * s, a0, p);
      h.y = fmaf(a0, h.y, p * __builtin_amdgcn_rsqf(p) * sg * xx.y);
      const int t = a.reverse ? len - 1 - i0 - i : i0 + i;
      st2f(y + t * a.ys[1], h.x, h.y);
    }
  }
  for (int t = len; t < a.S; ++t) st2f(y + t * a.ys[1], 0.f, 0.f);
  if (a.ht) *reinterpret_cast<float2*>(a.ht + o) = h;
}

template <typename T>
__global__ __launch_bounds__(64) void k_scan_seq_bwd(ScArgs a) {
  const int c = (blockIdx.y * 64 + threadIdx.x) * 2, b = blockIdx.x;
  if (c >= a.D) return;
  const int len = a.len ? min(max(a.len[b], 0), a.S) : a.S;
  const T* x = (const T*)a.x + b * a.xs[0] + c;
  const T* r = (const T*)a.r + b * a.rs[0] + c;
  const T* g = (const T*)a.g + b * a.gs[0] + c;
  const T* dy = (const T*)a.dy + b * a.ys[0] + c;
  T* dx = (T*)a.y + b * a.xs[0] + c;
  T* dr = (T*)a.dr + b * a.rs[0] + c;
  T* dg = (T*)a.dg + b * a.gs[0] + c;
  const int64_t o = (int64_t)b * a.D + c;
  const float k[2] = {-a.sharp * softplus(a.decay[c]) * kLog2e, -a.sharp * softplus(a.decay[c + 1]) * kLog2e};
  float E[2] = {a.h0 ? a.h0[o] : 0.f, a.h0 ? a.h0[o + 1] : 0.f};     // a_{t+1} E_{t+1}
  double sum[2] = {0.0, 0.0};
  const float* keep = a.saved + (int64_t)b * cdiv(a.S, kStep) * a.D + c;
  for (int i0 = (len - 1) / kStep * kStep; len > 0 && i0 >= 0; i0 -= kStep) {
    Two<T> xv[kStep], rv[kStep], gv[kStep], dv[kStep];
#pragma unroll
    for (int i = 0; i < kStep; ++i) {
      const int j = min(i0 + i, len - 1), t = a.reverse ? len - 1 - j : j;
      xv[i].load(x + t * a.xs[1]);
      rv[i].load(r + t * a.rs[1]);
      gv[i].load(g + t * a.gs[1]);
      dv[i].load(dy + t * a.ys[1]);
    }
    const float2 first = *reinterpret_cast<const float2*>(keep + (int64_t)(i0 / kStep) * a.D);
    float h[2] = {first.x, first.y}, before[kStep][2];
#pragma unroll
    for (int i = 0; i < kStep; ++i) {
      const float xx[2] = {xv[i].get().x, xv[i].get().y}, rr[2] = {rv[i].get().x, rv[i].get().y};
      const float gg[2] = {gv[i].get().x, gv[i].get().y};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float s, c1, sg, a0, p;
        before[i][e] = h[e];
        sigmoid(rr[e], s, c1);
        sigmoid(gg[e], sg, c1);
        decay_of(k[e] * s, a0, p);
        h[e] = fmaf(a0, h[e], p * __builtin_amdgcn_rsqf(p) * sg * xx[e]);
      }
    }
    float part[2] = {0.f, 0.f};
#pragma unroll
    for (int i = kStep - 1; i >= 0; --i) {
      if (i0 + i >= len) continue;
      const float xx[2] = {xv[i].get().x, xv[i].get().y}, rr[2] = {rv[i].get().x, rv[i].get().y};
      const float gg[2] = {gv[i].get().x, gv[i].get().y}, dd[2] = {dv[i].get().x, dv[i].get().y};
      float ox[2], orr[2], og[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float s, cs, sg, cg, a0, p;
        sigmoid(rr[e], s, cs);
        sigmoid(gg[e], sg, cg);
        decay_of(k[e] * s, a0, p);
        const float q = __builtin_amdgcn_rsqf(p), wsg = p * q * sg, u = wsg * xx[e];
        const float Et = dd[e] + E[e];
        const float dla = Et * (a0 * before[i][e] - u * a0 * a0 * q * q);
        ox[e] = Et * wsg;
        og[e] = Et * u * cg;
        orr[e] = dla * (k[e] * kLn2 * s) * cs;
        part[e] = fmaf(dla, s, part[e]);
        E[e] = a0 * Et;
      }
      const int t = a.reverse ? len - 1 - i0 - i : i0 + i;
      st2f(dx + t * a.xs[1], ox[0], ox[1]);
      st2f(dr + t * a.rs[1], orr[0], orr[1]);
      st2f(dg + t * a.gs[1], og[0], og[1]);
    }
    sum[0] += part[0];
    sum[1] += part[1];
  }
  for (int t = len; t < a.S; ++t) {
    st2f(dx + t * a.xs[1], 0.f, 0.f);
    st2f(dr + t * a.rs[1], 0.f, 0.f);
    st2f(dg + t * a.gs[1], 0.f, 0.f);
  }
  if (a.ht) *reinterpret_cast<float2*>(a.ht + o) = make_float2(E[0], E[1]);
  a.part[o] = sum[0];
  a.part[o + 1] = sum[1];
}

// ddecay = -sharp sigmoid(decay) times the sum over the sequences, in order
__global__ __launch_bounds__(256) void k_scan_decay(const double* part, const float* decay, int B, int D, float sharp,
                                                    float* ddecay) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= D) return;
  double s = 0.0;
#pragma unroll 8
  for (int b = 0; b < B; ++b) s += part[(int64_t)b * D + c];
  ddecay[c] = (float)(-(double)sharp / (1.0 + exp(-(double)decay[c])) * s);
}

ScArgs make_args(const Scan& a, const void* x, const void* r, const void* g, const float* decay, const int32_t* len) {
  ScArgs k{};
  k.x = x; k.r = r; k.g = g; k.decay = decay; k.len = len;
  for (int i = 0; i < 2; ++i) { k.xs[i] = a.xs[i]; k.rs[i] = a.rs[i]; k.gs[i] = a.gs[i]; k.ys[i] = a.ys[i]; }
  k.S = a.S; k.D = a.D; k.reverse = a.reverse; k.sharp = a.sharp;
  return k;
}

}  // namespace

size_t scan_saved_bytes(const Scan& a) { return align256((size_t)a.B * cdiv(a.S, kStep) * a.D * sizeof(float)); }
size_t scan_ws_bytes(const Scan& a) { return align256((size_t)a.B * a.D * sizeof(double)); }

void scan_fwd(hipStream_t st, const Scan& a, const void* x, const void* r, const void* g, const float* decay,
              const int32_t* len, const float* h0, void* y, float* ht, void* saved, void* ws) {
  ScArgs k = make_args(a, x, r, g, decay, len);
  k.h0 = h0; k.y = y; k.ht = ht; k.saved = (float*)saved;
  const dim3 grid((unsigned)a.B, (unsigned)cdiv(a.D, 128));
  ProfScope prof(st);
  if (a.f32) hipLaunchKernelGGL(k_scan_seq_fwd<float>, grid, dim3(64), 0, st, k);
  else hipLaunchKernelGGL(k_scan_seq_fwd<bf16_t>, grid, dim3(64), 0, st, k);
  PG_LAUNCH_CHECK();
  prof.done_bytes("k_scan_fwd", (a.f32 ? 16.0 : 8.0) * a.B * a.S * a.D);
}

void scan_bwd(hipStream_t st, const Scan& a, const void* x, const void* r, const void* g, const float* decay,
              const int32_t* len, const void* saved, const void* dy, const float* dht, void* dx, void* dr, void* dg,
              float* ddecay, float* dh0, void* ws) {
  ScArgs k = make_args(a, x, r, g, decay, len);
  k.dy = dy; k.h0 = dht; k.ht = dh0; k.y = dx; k.dr = dr; k.dg = dg; k.saved = (float*)const_cast<void*>(saved);
  k.part = (double*)ws;
  const dim3 grid((unsigned)a.B, (unsigned)cdiv(a.D, 128));
  ProfScope prof(st);
  if (a.f32) hipLaunchKernelGGL(k_scan_seq_bwd<float>, grid, dim3(64), 0, st, k);
  else hipLaunchKernelGGL(k_scan_seq_bwd<bf16_t>, grid, dim3(64), 0, st, k);
  PG_LAUNCH_CHECK();
  hipLaunchKernelGGL(k_scan_decay, dim3((unsigned)cdiv(a.D, 256)), dim3(256), 0, st, k.part, decay, a.B, a.D, a.sharp,
                     ddecay);
  PG_LAUNCH_CHECK();
  prof.done_bytes("k_scan_bwd", (a.f32 ? 28.0 : 14.0) * a.B * a.S * a.D);
}

}  // namespace pg
