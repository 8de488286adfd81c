// Gated linear recurrence over the tokens of a sequence, every channel by
// itself, forward and backward.
//
//   la = -sharp softplus(decay) s,  s = sigmoid(r);   a = exp(la),  w = (1 - a^2)^1/2,
//   h_t = a_t h_{t-1} + u_t,  u = w sg x,  sg = sigmoid(g);   y = h.
// Backward, with E_t = dy_t + a_{t+1} E_{t+1} (the last also dht):
//   dla = E (a h_{t-1} - u a^2 / w^2);  dr = dla la (1 - s);
//   dg = E u (1 - sg);  dx = E w sg;
//   ddecay = -sharp sigmoid(decay) sum dla s;  dh0 = a_1 E_1.
//
// Bound by memory with the vector units close behind: forward 8 bytes and
// about 35 vector instructions an element in bf16 (five of them
// transcendental), backward 14 bytes and 60.  Every input is read once: a tile
// of tokens lies in a block's registers while its tokens' maps of the state
// are joined, so the sequence is not walked token after token, and only a
// state every 64 tokens is kept for the backward.  Few sequences of few
// channels leave the card idle; then chunks of them go side by side and the
// inputs are read twice.
// Measured, bf16: forward of 8 x 4096 x 2048 that keeps states 131 us (4.1
// TB/s; a copy reaches 5.2), of 16 x 4096 x 1536 219 us (3.7: 384 blocks on
// 256 CUs), of 1 x 32768 x 1280 in chunks 53 and 73 us (4.8 and 4.6), backward
// of 8 x 4096 x 2048 202 us (4.7).  Slabs of 32 channels (64-byte rows) were
// slower when the backward of 64 took 265 us: 402, and the forward 156 for 121.
#include "token.hpp"

#include <cfloat>

namespace pg {

namespace {

constexpr int kStep = 16, kKeep = 64;   // tokens between two states that a forward keeps: a thread a sequence, tiles

struct ScArgs {
  const void *x, *r, *g, *dy;
  const float* decay;
  const int32_t* len;
  const float* h0;                 // backward: dht
  float* ht;                       // backward: dh0
  void *y, *dr, *dg;               // y; backward: dx in y
  float* saved;                    // [B][ceil(S / kStep or kKeep)][D]: the state ahead of that many tokens
  float* maps;                     // [B][chunks][D][2]: A, H of every chunk; in the one nobody needs, the state from outside
  double* part;                    // [B][chunks][D]: sums of dla s
  int64_t xs[2], rs[2], gs[2], ys[2];
  int B, S, D, reverse;
  int slabs, nc, chunk;            // slabs of channels; chunks of a sequence, tokens of one
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

// sigmoid(v) and 1 - sigmoid(v), both to the last digits (e^-v may be infinite)
PG_DEV void sigmoid(float v, float& s, float& c) {
  const float e = __builtin_amdgcn_exp2f(v * -kLog2e);
  s = __builtin_amdgcn_rcpf(1.f + e);
  c = e < 1e30f ? e * s : 1.f;
}
PG_DEV float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -kLog2e)); }
// softplus(v) = log(1 + e^v)
PG_DEV float softplus(float v) { return log1pf(expf(-fabsf(v))) + fmaxf(v, 0.f); }
// -sharp softplus(decay) / ln 2 of two channels; past the largest float that
// one, since an infinity times a closed gate's zero would be NaN (a NaN stays)
PG_DEV float rate(float sharp, float decay) {
  const float k = -sharp * softplus(decay) * kLog2e;
  return k < -FLT_MAX ? -FLT_MAX : k;
}
PG_DEV float2 rates(const ScArgs& a, int c) {
  const float2 d = *reinterpret_cast<const float2*>(a.decay + c);
  return make_float2(rate(a.sharp, d.x), rate(a.sharp, d.y));
}

// a = 2^l and p = 1 - a^2 for l = la / ln 2 <= 0.  Where the difference would
// cancel, p is -l Q(l) with a polynomial Q of degree 4 for (4^l - 1) / l on
// la in [-0.2, 0] (least largest relative error, 6.9e-8 with rounded
// coefficients).
PG_DEV void decay_of(float l, float& a, float& p) {
  a = __builtin_amdgcn_exp2f(l);
  float q = fmaf(l, 0.036133427172899246f, 0.15227515995502472f);
  q = fmaf(l, q, 0.4438667893409729f);
  q = fmaf(l, q, 0.9608999490737915f);
  q = fmaf(l, q, 1.3862943649291992f);
  p = l > -0.2f * kLog2e ? -l * q : fmaf(-a, a, 1.f);
}

// a and u of one element
PG_DEV void gate(float x, float r, float g, float k, float& a, float& u) {
  float p;
  decay_of(k * sigmoid(r), a, p);
  u = __builtin_amdgcn_sqrtf(p) * sigmoid(g) * x;
}
// What one element needs after its gates are known: dx = E fx, dg = E fg,
// dr = E M fr, ddecay += E M s, with M = a h_{t-1} - v.
struct Grad {
  float a, u, v, fx, fg, fr, s;
};
PG_DEV void grad_gate(float x, float r, float g, float k, Grad& e) {
  float cs, sg, cg, p;
  sigmoid(r, e.s, cs);
  sigmoid(g, sg, cg);
  const float l = k * e.s;
  decay_of(l, e.a, p);
  p = fmaxf(p, 1.17549435e-38f);   // so that w = p p^-1/2 and 1 / p are finite
  const float q = __builtin_amdgcn_rsqf(p), aq = e.a * q;
  e.fx = p * q * sg;
  e.u = e.fx * x;
  e.v = e.u * aq * aq;
  e.fg = e.u * cg;
  e.fr = l * kLn2 * cs;
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
  const float2 k = rates(a, c);
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
      float a0, u;
      gate(xx.x, rr.x, gg.x, k.x, a0, u);
      h.x = fmaf(a0, h.x, u);
      gate(xx.y, rr.y, gg.y, k.y, a0, u);
      h.y = fmaf(a0, h.y, u);
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
  const float2 kk = rates(a, c);
  const float k[2] = {kk.x, kk.y};
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
        float a0, u;
        before[i][e] = h[e];
        gate(xx[e], rr[e], gg[e], k[e], a0, u);
        h[e] = fmaf(a0, h[e], u);
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
        Grad q;
        grad_gate(xx[e], rr[e], gg[e], k[e], q);
        const float Et = dd[e] + E[e], EM = Et * fmaf(q.a, before[i][e], -q.v);
        ox[e] = Et * q.fx;
        og[e] = Et * q.fg;
        orr[e] = EM * q.fr;
        part[e] = fmaf(EM, q.s, part[e]);
        E[e] = q.a * Et;
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

// ------------------------------------------------------------- tiles of tokens
// A block takes a slab of 2 CL channels through tiles of TT tokens that lie
// one behind the other in memory: lane (cl, tl) of wave w holds TOK tokens of
// segment w TL + tl in order, two channels of each.  A segment is a linear map
// of the state ahead of it, h -> A h + H: the lanes of a wave join theirs by
// exchanges, the waves through LDS (two halves used in turn: one barrier a
// tile), and every thread then runs its own tokens from the state at its
// segment's start.  The next tile's loads are under way meanwhile.  Loads and
// stores go through buffer descriptors that begin at the tile and end at the
// sequence's length: a lane's offset is fixed, a token's is uniform, and what
// is past the length or the last channel reads as zero and is not written.
template <typename T> PG_DEV Two<T> never();   // sigmoid 0: a token that keeps the state and adds nothing
template <> PG_DEV Two<bf16_t> never<bf16_t>() { return Two<bf16_t>{0xff80ff80u}; }
template <> PG_DEV Two<float> never<float>() { return Two<float>{make_float2(-INFINITY, -INFINITY)}; }

template <typename T_, int CL_, int NW_>
struct Form {
  typedef T_ T;
  static constexpr int CL = CL_, NW = NW_, TOK = sizeof(T) == 2 ? 8 : 4, TL = 64 / CL, NSEG = NW * TL, TT = NSEG * TOK;
};

template <typename F>
struct Place {
  int cl, tl, wave, seg, mseg, c, cc;   // mseg: the segment's place in memory; c: first channel, cc: one that exists
  bool ok;
  int b, chunk, len, lo, hi, n;         // tokens [lo, hi) in memory of the chunk, tiles of it that hold tokens
  PG_DEV Place(const ScArgs& a) {
    const int lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    cl = lane % F::CL; tl = lane / F::CL;
    seg = wave * F::TL + tl;
    mseg = a.reverse ? F::NSEG - 1 - seg : seg;
    // neighbouring slabs on one XCD: they share cache lines and pages
    const uint32_t id = blockIdx.x, per = gridDim.x / 8;
    uint32_t l = (id % 8) * per + id / 8;
    chunk = l % a.nc;
    l /= a.nc;
    const int slab = l % a.slabs;
    b = l / a.slabs;
    c = (slab * F::CL + cl) * 2;
    ok = c < a.D;
    cc = ok ? c : 0;
    if (b < a.B) {
      len = __builtin_amdgcn_readfirstlane(a.len ? min(max(a.len[b], 0), a.S) : a.S);
      lo = (a.reverse ? a.nc - 1 - chunk : chunk) * a.chunk;
      hi = min(a.S, lo + a.chunk);
      n = len > lo ? (min(hi, len) - lo + F::TT - 1) / F::TT : 0;
    }
  }
  // where tile k, in order, begins in memory
  PG_DEV int tile(int k, int reverse) const { return lo + (reverse ? n - 1 - k : k) * F::TT; }
};

PG_DEV void buf_load(Two<bf16_t>& v, __amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t so) {
  v.v = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r, (int)off, (int)so, 0);
}
PG_DEV void buf_load(Two<float>& v, __amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t so) {
  v.v = __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(r, (int)off, (int)so, 0));
}
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
template <typename T>
PG_DEV void buf_store(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t so, float2 v) {
  if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b32(f2bf2(v.x, v.y), r, (int)off, (int)so, 0);
  else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), r, (int)off, (int)so, 0);
}

// A tensor's tokens as a lane takes them: `run` tokens in memory from mseg * run on.  OVER: they may overlap or repeat (the
// forward's inputs; where none may, the backward of 8 x 4096 x 2048 is 5 us faster without).
template <typename F, bool OVER = false>
struct Tokens {
  typedef typename F::T T;
  const char* base;                // the sequence
  int64_t st, over = 0;            // bytes between tokens; by how much a token reaches into the next one
  uint32_t lane;
  PG_DEV Tokens(const void* p, const int64_t* s, const Place<F>& q, int D = 0, int run = F::TOK) {
    base = (const char*)p + q.b * s[0] * (int64_t)sizeof(T);
    st = s[1] * (int64_t)sizeof(T);
    if constexpr (OVER) over = max((int64_t)0, D * (int64_t)sizeof(T) - st);
    lane = q.ok ? (uint32_t)q.mseg * (uint32_t)run * (uint32_t)st + (uint32_t)q.c * (uint32_t)sizeof(T) : kOOB;
  }
  // bytes from token m on, to the end of the last one's row where tokens overlap or repeat
  PG_DEV uint32_t bytes(int m, int len) const {
    const int64_t n = (int64_t)(len - m) * st + (OVER && len > m ? over : 0);
    return (uint32_t)(n > kBufMax ? kBufMax : n < 0 ? 0 : n);
  }
  PG_DEV uint32_t place(int j, int reverse) const { return (uint32_t)(reverse ? F::TOK - 1 - j : j) * (uint32_t)st; }
  // The range check takes the uniform offset from the descriptor's bytes, so
  // that offset stops there: at them no lane's is below what is left.
  PG_DEV void load(Two<T>* v, int m, int len, int reverse, uint32_t so = 0) const {
    const uint32_t n = bytes(m, len);
    const __amdgpu_buffer_rsrc_t r = make_rsrc(base + m * st, n);
#pragma unroll
    for (int j = 0; j < F::TOK; ++j) buf_load(v[j], r, lane, min(so + place(j, reverse), n));
  }
  template <typename G> PG_DEV void store(int m, int len, int reverse, G&& get) const {
    const uint32_t n = bytes(m, len);
    const __amdgpu_buffer_rsrc_t r = make_rsrc(base + m * st, n);
#pragma unroll
    for (int j = 0; j < F::TOK; ++j) buf_store<T>(r, lane, min(place(j, reverse), n), get(j));
  }
  // rows [max(lo, len), hi) become zeros
  PG_DEV void zero(const Place<F>& p) const {
    for (int t = max(p.lo, p.len) + p.seg; t < p.hi; t += F::NSEG)
      if (p.ok) st2f((T*)(const_cast<char*>(base) + t * st) + p.c, 0.f, 0.f);
  }
};
// tokens from m on (of this lane) past the length never come in (the others: where tokens overlap or repeat, what real ones
// own was read all the same)
template <typename F, typename... Others>
PG_DEV void past(int m, int len, int reverse, Two<typename F::T>* r, Others... others) {
#pragma unroll
  for (int j = 0; j < F::TOK; ++j)
    if (m + (reverse ? F::TOK - 1 - j : j) >= len) {
      r[j] = never<typename F::T>();
      ((others[j] = Two<typename F::T>{}), ...);
    }
}

// (A, H) of what lies ahead of this lane's segment in its wave (ahead), and of
// the wave's segments up to it (A, H)
template <int CL>
PG_DEV void join_up(float2& A, float2& H, float2& Ae, float2& He) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = CL; d < 64; d *= 2) {
    const float a0 = __shfl_up(A.x, d, 64), a1 = __shfl_up(A.y, d, 64), h0 = __shfl_up(H.x, d, 64), h1 = __shfl_up(H.y, d, 64);
    if (lane >= d) {
      H = make_float2(fmaf(A.x, h0, H.x), fmaf(A.y, h1, H.y));
      A = make_float2(A.x * a0, A.y * a1);
    }
  }
  const float a0 = __shfl_up(A.x, CL, 64), a1 = __shfl_up(A.y, CL, 64), h0 = __shfl_up(H.x, CL, 64), h1 = __shfl_up(H.y, CL, 64);
  const bool first = lane < CL;
  Ae = first ? make_float2(1.f, 1.f) : make_float2(a0, a1);
  He = first ? make_float2(0.f, 0.f) : make_float2(h0, h1);
}
template <int CL>
PG_DEV void join_down(float2& A, float2& H, float2& Ae, float2& He) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = CL; d < 64; d *= 2) {
    const float a0 = __shfl_down(A.x, d, 64), a1 = __shfl_down(A.y, d, 64), h0 = __shfl_down(H.x, d, 64), h1 = __shfl_down(H.y, d, 64);
    if (lane + d < 64) {
      H = make_float2(fmaf(A.x, h0, H.x), fmaf(A.y, h1, H.y));
      A = make_float2(A.x * a0, A.y * a1);
    }
  }
  const float a0 = __shfl_down(A.x, CL, 64), a1 = __shfl_down(A.y, CL, 64), h0 = __shfl_down(H.x, CL, 64), h1 = __shfl_down(H.y, CL, 64);
  const bool last = lane >= 64 - CL;
  Ae = last ? make_float2(1.f, 1.f) : make_float2(a0, a1);
  He = last ? make_float2(0.f, 0.f) : make_float2(h0, h1);
}
PG_DEV float2 fold(float2 A, float2 H, float2 h) { return make_float2(fmaf(A.x, h.x, H.x), fmaf(A.y, h.y, H.y)); }

// SPLIT: the chunks of a sequence start from the folded maps of those ahead
template <typename F, bool SPLIT>
__global__ __launch_bounds__(F::NW * 64, 4) void k_scan_fwd(ScArgs a) {
  constexpr int CL = F::CL, NW = F::NW, TOK = F::TOK;
  typedef typename F::T T;
  __shared__ float4 sh[2][NW][CL];
  const Place<F> p(a);
  if (p.b >= a.B) return;
  const Tokens<F, true> x(a.x, a.xs, p, a.D), r(a.r, a.rs, p, a.D), g(a.g, a.gs, p, a.D);
  const Tokens<F> y(a.y, a.ys, p);
  const int64_t o = (int64_t)p.b * a.D + p.cc;
  const float2 k = rates(a, p.cc);
  float2 h = !SPLIT && a.h0 ? *reinterpret_cast<const float2*>(a.h0 + o) : make_float2(0.f, 0.f);
  Two<T> X[TOK], R[TOK], G[TOK];
  auto load = [&](int m) {
    r.load(R, m, p.len, a.reverse);
    g.load(G, m, p.len, a.reverse);
    x.load(X, m, p.len, a.reverse);
  };
  if (p.n) load(p.tile(0, a.reverse));
  if constexpr (SPLIT) {
    const float* m = a.maps + ((int64_t)p.b * a.nc * a.D + p.cc) * 2;
    const float4 first = *reinterpret_cast<const float4*>(m + (int64_t)(a.nc - 1) * a.D * 2);
    h = make_float2(first.y, first.w);
#pragma unroll 8
    for (int j = 0; j < p.chunk; ++j) {
      const float4 q = *reinterpret_cast<const float4*>(m + (int64_t)j * a.D * 2);
      h = fold(make_float2(q.x, q.z), make_float2(q.y, q.w), h);
    }
  }
  int turn = 0;
  for (int t = 0; t < p.n; ++t, turn ^= 1) {
    const int m0 = p.tile(t, a.reverse), mine = m0 + p.mseg * TOK;
    if (m0 + F::TT > p.len) past<F>(mine, p.len, a.reverse, R, G, X);
    float2 av[TOK], uv[TOK], A = make_float2(1.f, 1.f), H = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < TOK; ++j) {
      const float2 xx = X[j].get(), rr = R[j].get(), gg = G[j].get();
      gate(xx.x, rr.x, gg.x, k.x, av[j].x, uv[j].x);
      gate(xx.y, rr.y, gg.y, k.y, av[j].y, uv[j].y);
      H = fold(av[j], uv[j], H);
      A.x *= av[j].x;
      A.y *= av[j].y;
    }
    if (t + 1 < p.n) load(p.tile(t + 1, a.reverse));
    float2 Ae, He;
    join_up<CL>(A, H, Ae, He);
    if (p.tl == F::TL - 1) sh[turn][p.wave][p.cl] = make_float4(A.x, A.y, H.x, H.y);
    __syncthreads();
    float2 hw = h;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float4 q = sh[turn][w][p.cl];
      if (w == p.wave) hw = h;
      h = fold(make_float2(q.x, q.y), make_float2(q.z, q.w), h);
    }
    hw = fold(Ae, He, hw);
    // the first segment of kKeep tokens keeps the state ahead of them
    const int keep = mine / kKeep;
    if (a.saved && p.ok && (mine + (a.reverse ? TOK : 0)) % kKeep == 0 && keep * kKeep < p.len)
      *reinterpret_cast<float2*>(a.saved + ((int64_t)p.b * cdiv(a.S, kKeep) + keep) * a.D + p.c) = hw;
    y.store(m0, p.len, a.reverse, [&](int j) { return hw = fold(av[j], uv[j], hw); });
  }
  y.zero(p);
  if (a.ht && p.chunk == a.nc - 1 && p.seg == 0 && p.ok) *reinterpret_cast<float2*>(a.ht + o) = h;
}

// The map (A, H) of every chunk: its segments run through it side by side,
// TOK tokens at a time, and are joined once at the end.
template <typename F>
__global__ __launch_bounds__(F::NW * 64, 4) void k_scan_maps(ScArgs a) {
  constexpr int CL = F::CL, NW = F::NW, TOK = F::TOK;
  typedef typename F::T T;
  __shared__ float4 sh[NW][CL];
  const Place<F> p(a);
  if (p.b >= a.B) return;
  if (p.chunk == a.nc - 1) {       // nobody comes after the last one: its place hands on h0, which ht may overwrite
    const float2 h = a.h0 ? *reinterpret_cast<const float2*>(a.h0 + (int64_t)p.b * a.D + p.cc) : make_float2(0.f, 0.f);
    if (p.seg == 0 && p.ok)
      *reinterpret_cast<float4*>(a.maps + (((int64_t)p.b * a.nc + p.chunk) * a.D + p.c) * 2) = make_float4(0.f, h.x, 0.f, h.y);
    return;
  }
  const int run = a.chunk / F::NSEG, m = p.lo + p.mseg * run;   // a chunk is whole tiles
  const Tokens<F, true> x(a.x, a.xs, p, a.D, run), r(a.r, a.rs, p, a.D, run), g(a.g, a.gs, p, a.D, run);
  const float2 k = rates(a, p.cc);
  float2 A = make_float2(1.f, 1.f), H = make_float2(0.f, 0.f);
  Two<T> X[TOK], R[TOK], G[TOK];
  auto load = [&](int i) {         // i: order index in the run
    const int at = a.reverse ? run - TOK - i : i;
    r.load(R, p.lo, p.len, a.reverse, (uint32_t)at * (uint32_t)r.st);
    g.load(G, p.lo, p.len, a.reverse, (uint32_t)at * (uint32_t)g.st);
    x.load(X, p.lo, p.len, a.reverse, (uint32_t)at * (uint32_t)x.st);
  };
  if (p.n) {
    load(0);
    for (int i = 0; i < run; i += TOK) {
      float2 av[TOK], uv[TOK];
      if (p.lo + a.chunk > p.len) past<F>(m + (a.reverse ? run - TOK - i : i), p.len, a.reverse, R, G, X);
#pragma unroll
      for (int j = 0; j < TOK; ++j) {
        const float2 xx = X[j].get(), rr = R[j].get(), gg = G[j].get();
        gate(xx.x, rr.x, gg.x, k.x, av[j].x, uv[j].x);
        gate(xx.y, rr.y, gg.y, k.y, av[j].y, uv[j].y);
      }
      if (i + TOK < run) load(i + TOK);
#pragma unroll
      for (int j = 0; j < TOK; ++j) {
        H = fold(av[j], uv[j], H);
        A.x *= av[j].x;
        A.y *= av[j].y;
      }
    }
  }
  float2 Ae, He;
  join_up<CL>(A, H, Ae, He);
  if (p.tl == F::TL - 1) sh[p.wave][p.cl] = make_float4(A.x, A.y, H.x, H.y);
  __syncthreads();
  if (p.seg == 0 && p.ok) {
    A = make_float2(1.f, 1.f);
    H = make_float2(0.f, 0.f);
    for (int w = 0; w < NW; ++w) {
      const float4 q = sh[w][p.cl];
      H = fold(make_float2(q.x, q.y), make_float2(q.z, q.w), H);
      A.x *= q.x;
      A.y *= q.y;
    }
    *reinterpret_cast<float4*>(a.maps + (((int64_t)p.b * a.nc + p.chunk) * a.D + p.c) * 2) = make_float4(A.x, H.x, A.y, H.y);
  }
}

// Backward of a tile: the states ahead of its segments from the forward's
// kept state, what flows back into them from the tile behind it, both joined
// at the same barrier.
template <typename F, bool SPLIT>
__global__ __launch_bounds__(F::NW * 64, 2) void k_scan_bwd(ScArgs a) {
  constexpr int CL = F::CL, NW = F::NW, TOK = F::TOK;
  typedef typename F::T T;
  static_assert(CL == 32, "the two halves of a wave");
  __shared__ float4 sh[2][2][NW][CL];   // [turn][towards later, earlier tokens]
  __shared__ double sd[NW][64][2];
  const Place<F> p(a);
  if (p.b >= a.B) return;
  const Tokens<F> x(a.x, a.xs, p), r(a.r, a.rs, p), g(a.g, a.gs, p), dy(a.dy, a.ys, p);
  const Tokens<F> dx(a.y, a.xs, p), dr(a.dr, a.rs, p), dg(a.dg, a.gs, p);
  const int64_t o = (int64_t)p.b * a.D + p.cc;
  const float2 k = rates(a, p.cc);
  // what flows back into the tile
  float2 c = !SPLIT && a.h0 ? *reinterpret_cast<const float2*>(a.h0 + o) : make_float2(0.f, 0.f);
  const float* keep = a.saved + (int64_t)p.b * cdiv(a.S, kKeep) * a.D + p.cc;
  Two<T> X[TOK], R[TOK], G[TOK], Y[TOK], Yn[TOK];
  float2 hn = make_float2(0.f, 0.f);
  auto load = [&](int m) {
    r.load(R, m, p.len, a.reverse);
    g.load(G, m, p.len, a.reverse);
    x.load(X, m, p.len, a.reverse);
    dy.load(Yn, m, p.len, a.reverse);
    // ahead of the tile's first tokens (past the length nothing comes in)
    const int i = a.reverse ? min((m + F::TT) / kKeep - 1, (p.len - 1) / kKeep) : m / kKeep;
    hn = *reinterpret_cast<const float2*>(keep + (int64_t)i * a.D);
  };
  if (p.n) load(p.tile(p.n - 1, a.reverse));
  if constexpr (SPLIT) {
    const float* m = a.maps + ((int64_t)p.b * a.nc * a.D + p.cc) * 2;
    const float4 outer = *reinterpret_cast<const float4*>(m);
    c = make_float2(outer.y, outer.w);
#pragma unroll 8
    for (int j = a.nc - 1; j > p.chunk; --j) {
      const float4 q = *reinterpret_cast<const float4*>(m + (int64_t)j * a.D * 2);
      c = fold(make_float2(q.x, q.z), make_float2(q.y, q.w), c);
    }
  }
  int turn = 0;
  const bool up = (threadIdx.x & 63) < 32;
  const int at = up ? p.wave : NW - 1 - p.wave;
  double sum0 = 0.0, sum1 = 0.0;
  for (int t = p.n - 1; t >= 0; --t, turn ^= 1) {
    const int m0 = p.tile(t, a.reverse);
    if (m0 + F::TT > p.len) past<F>(m0 + p.mseg * TOK, p.len, a.reverse, R, X);
    Grad e0[TOK], e1[TOK];
    float2 A = make_float2(1.f, 1.f), H = make_float2(0.f, 0.f), C = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < TOK; ++j) {
      Y[j] = Yn[j];
      const float2 xx = X[j].get(), rr = R[j].get(), gg = G[j].get();
      grad_gate(xx.x, rr.x, gg.x, k.x, e0[j]);
      grad_gate(xx.y, rr.y, gg.y, k.y, e1[j]);
      H = make_float2(fmaf(e0[j].a, H.x, e0[j].u), fmaf(e1[j].a, H.y, e1[j].u));
      A.x *= e0[j].a;
      A.y *= e1[j].a;
      __builtin_amdgcn_sched_barrier(0);
    }
    float2 h = hn;
    if (t > 0) load(p.tile(t - 1, a.reverse));
#pragma unroll
    for (int j = TOK - 1; j >= 0; --j) {
      const float2 d = Y[j].get();
      C = make_float2(e0[j].a * (d.x + C.x), e1[j].a * (d.y + C.y));
    }
    float2 Ad = A, Ae, He, Ce, Ade;
    join_up<CL>(A, H, Ae, He);
    join_down<CL>(Ad, C, Ade, Ce);
    if (p.tl == F::TL - 1) sh[turn][0][p.wave][p.cl] = make_float4(A.x, A.y, H.x, H.y);
    if (p.tl == 0) sh[turn][1][NW - 1 - p.wave][p.cl] = make_float4(Ad.x, Ad.y, C.x, C.y);
    __syncthreads();
    // one half of the lanes runs through the waves forwards with h, the other backwards with c
    float2 v = up ? h : c, mine = v;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float4 q = sh[turn][up ? 0 : 1][w][p.cl];
      if (w == at) mine = v;
      v = fold(make_float2(q.x, q.y), make_float2(q.z, q.w), v);
    }
    h = make_float2(__shfl(mine.x, p.cl, 64), __shfl(mine.y, p.cl, 64));
    float2 cw = make_float2(__shfl(mine.x, p.cl + 32, 64), __shfl(mine.y, p.cl + 32, 64));
    c = make_float2(__shfl(v.x, p.cl + 32, 64), __shfl(v.y, p.cl + 32, 64));
    h = fold(Ae, He, h);
    cw = fold(Ade, Ce, cw);
#pragma unroll
    for (int j = 0; j < TOK; ++j) {   // v becomes M
      e0[j].v = fmaf(e0[j].a, h.x, -e0[j].v);
      e1[j].v = fmaf(e1[j].a, h.y, -e1[j].v);
      h = make_float2(fmaf(e0[j].a, h.x, e0[j].u), fmaf(e1[j].a, h.y, e1[j].u));
    }
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int j = TOK - 1; j >= 0; --j) {   // u becomes E
      const float2 d = Y[j].get();
      const float E0 = d.x + cw.x, E1 = d.y + cw.y;
      cw = make_float2(e0[j].a * E0, e1[j].a * E1);
      e0[j].u = E0;
      e1[j].u = E1;
      e0[j].v *= E0;
      e1[j].v *= E1;
      s0 = fmaf(e0[j].v, e0[j].s, s0);
      s1 = fmaf(e1[j].v, e1[j].s, s1);
    }
    sum0 += s0;
    sum1 += s1;
    dx.store(m0, p.len, a.reverse, [&](int j) { return make_float2(e0[j].u * e0[j].fx, e1[j].u * e1[j].fx); });
    dr.store(m0, p.len, a.reverse, [&](int j) { return make_float2(e0[j].v * e0[j].fr, e1[j].v * e1[j].fr); });
    dg.store(m0, p.len, a.reverse, [&](int j) { return make_float2(e0[j].u * e0[j].fg, e1[j].u * e1[j].fg); });
  }
  dx.zero(p);
  dr.zero(p);
  dg.zero(p);
  if (a.ht && p.chunk == 0 && p.seg == 0 && p.ok) *reinterpret_cast<float2*>(a.ht + o) = c;
  const int lane = threadIdx.x & 63;
  sd[p.wave][lane][0] = sum0;
  sd[p.wave][lane][1] = sum1;
  __syncthreads();
  if (p.seg == 0 && p.ok) {          // the block's segments in order
    sum0 = sum1 = 0.0;
    for (int i = 0; i < F::NSEG; ++i) {
      sum0 += sd[i / F::TL][i % F::TL * CL + p.cl][0];
      sum1 += sd[i / F::TL][i % F::TL * CL + p.cl][1];
    }
    double* q = a.part + ((int64_t)p.b * a.nc + p.chunk) * a.D + p.c;
    q[0] = sum0;
    q[1] = sum1;
  }
}

// The map c -> A c + C by which what flows into a chunk from behind leaves it
// ahead: from the decays and dy alone.
template <typename F>
__global__ __launch_bounds__(F::NW * 64, 4) void k_scan_back_maps(ScArgs a) {
  constexpr int CL = F::CL, NW = F::NW, TOK = F::TOK;
  typedef typename F::T T;
  __shared__ float4 sh[NW][CL];
  const Place<F> p(a);
  if (p.b >= a.B) return;
  if (p.chunk == 0) {              // nobody comes before the first one: its place hands on dht, which dh0 may overwrite
    const float2 h = a.h0 ? *reinterpret_cast<const float2*>(a.h0 + (int64_t)p.b * a.D + p.cc) : make_float2(0.f, 0.f);
    if (p.seg == 0 && p.ok)
      *reinterpret_cast<float4*>(a.maps + ((int64_t)p.b * a.nc * a.D + p.c) * 2) = make_float4(0.f, h.x, 0.f, h.y);
    return;
  }
  const int run = a.chunk / F::NSEG, m = p.lo + p.mseg * run;
  const Tokens<F> r(a.r, a.rs, p, 0, run), dy(a.dy, a.ys, p, 0, run);
  const float2 k = rates(a, p.cc);
  float2 A = make_float2(1.f, 1.f), H = make_float2(0.f, 0.f);
  Two<T> R[TOK], Y[TOK];
  auto load = [&](int i) {
    const int at = a.reverse ? run - TOK - i : i;
    r.load(R, p.lo, p.len, a.reverse, (uint32_t)at * (uint32_t)r.st);
    dy.load(Y, p.lo, p.len, a.reverse, (uint32_t)at * (uint32_t)dy.st);
  };
  if (p.n) {
    load(run - TOK);
    for (int i = run - TOK; i >= 0; i -= TOK) {
      float2 av[TOK], d[TOK];
      if (p.lo + a.chunk > p.len) past<F>(m + (a.reverse ? run - TOK - i : i), p.len, a.reverse, R, Y);
#pragma unroll
      for (int j = 0; j < TOK; ++j) {
        const float2 rr = R[j].get();
        av[j].x = __builtin_amdgcn_exp2f(k.x * sigmoid(rr.x));
        av[j].y = __builtin_amdgcn_exp2f(k.y * sigmoid(rr.y));
        d[j] = Y[j].get();
      }
      if (i > 0) load(i - TOK);
#pragma unroll
      for (int j = TOK - 1; j >= 0; --j) {
        H = make_float2(av[j].x * (d[j].x + H.x), av[j].y * (d[j].y + H.y));
        A.x *= av[j].x;
        A.y *= av[j].y;
      }
    }
  }
  float2 Ae, He;
  join_down<CL>(A, H, Ae, He);
  if (p.tl == 0) sh[p.wave][p.cl] = make_float4(A.x, A.y, H.x, H.y);
  __syncthreads();
  if (p.seg == 0 && p.ok) {
    A = make_float2(1.f, 1.f);
    H = make_float2(0.f, 0.f);
    for (int w = NW - 1; w >= 0; --w) {
      const float4 q = sh[w][p.cl];
      H = fold(make_float2(q.x, q.y), make_float2(q.z, q.w), H);
      A.x *= q.x;
      A.y *= q.y;
    }
    *reinterpret_cast<float4*>(a.maps + (((int64_t)p.b * a.nc + p.chunk) * a.D + p.c) * 2) = make_float4(A.x, H.x, A.y, H.y);
  }
}

// ddecay = -sharp sigmoid(decay) times the sum over the chunks of all
// sequences: 32 channels x 8 lanes a block, in order
__global__ __launch_bounds__(256) void k_scan_decay(const double* part, const float* decay, int64_t n, int D, float sharp,
                                                    float* ddecay) {
  __shared__ double sh[8][33];
  const int j = threadIdx.x & 31, l = threadIdx.x >> 5, c = blockIdx.x * 32 + j;
  double s = 0.0;
  if (c < D) {
#pragma unroll 8
    for (int64_t i = l; i < n; i += 8) s += part[i * D + c];
  }
  sh[l][j] = s;
  __syncthreads();
  if (l > 0 || c >= D) return;
  s = 0.0;
  for (int i = 0; i < 8; ++i) s += sh[i][j];
  ddecay[c] = (float)(-(double)sharp / (1.0 + exp(-(double)decay[c])) * s);
}

// Which form a call takes, from its sizes alone.
struct Plan {
  int cl, nw;                      // 0: a thread a sequence and two channels
  int slabs, nc, chunk;
};
// Few slabs leave the card idle: then chunks of the sequences go side by side,
// at the price of a pass over the inputs ahead and its launch.  Split where
// the modelled time says so, in us: a block walks its sequence at a rate of
// its own, the split form moves bytes at the card's.  Of 18 shapes of up to
// 255 slabs (fp32: 128), each timed in both forms, types and directions, the
// choice costs at most 5 %.  More slabs are not split, whatever that costs: a
// block of eight waves of the backward has a CU to itself, so that 288 slabs
// (9 x 4096 x 2048) take two rounds and 349 us where 256 take 202.
// Whole and split, bf16: forward of 5 x 3000 x 1320 80 and 71, of 6 x 4096 x
// 1536 106 and 117, of 2 x 600 x 5000 19 and 30, of 1 x 20000 x 2048 483 and
// 123; with the backward 215 and 170, 286 and 272, 55 and 68, 1296 and 283.
// fp32, with the backward, of 6 x 4096 x 1536 417 and 602.
bool split_pays(const Scan& a, bool bwd, int64_t rows) {
  const double n = (double)a.B * a.S * a.D;
  const double whole = 5.0 + a.S * (bwd ? a.f32 ? 0.061 : 0.045 : a.f32 ? 0.033 : 0.026);
  const double parts = bwd ? 12.0 + n * (a.f32 ? 6.2e-6 : 4.1e-6) : 8.0 + n * (a.f32 ? 4.3e-6 : 2.8e-6);
  return rows <= (a.f32 ? 128 : 255) && whole > parts;   // a float block of eight waves has a CU to itself
}
Plan plan_of(const Scan& a, bool bwd) {
  Plan p{0, 0, 0, 1, a.S};
  p.cl = 32;
  p.slabs = (int)cdiv(a.D, 2 * p.cl);
  const int64_t rows = (int64_t)a.B * p.slabs;
  // a thread a sequence: few tokens, or some for so many sequences that they fill the card (64 x 48 x 4096 24 us
  // forward, 50 backward, in tiles 30 and 60; 64 x 64 x 4096 30 and 63, 32 and 62; 32 x 24 x 1024 8 and 17, 7 and 14)
  if (a.S <= kStep || (a.S <= 3 * kStep && rows >= 2048)) return Plan{0, 0, 0, 1, a.S};
  const bool split = split_pays(a, bwd, rows);
  // blocks of four waves side by side, for sequences of one tile, and where many have only a few tiles (64 x 256 x
  // 1024 backward 53 us, of eight 64); of eight otherwise (8 x 4096 x 2048 212, of four 241; 16 x 4096 x 2048 402,
  // 451).  A float tile of four would be shorter than kKeep.
  p.nw = !a.f32 && (split || a.S <= kKeep || (rows >= 512 && a.S <= 512)) ? 4 : 8;
  const int tt = p.nw * (64 / p.cl) * (a.f32 ? 4 : 8);
  // two to three blocks of four waves a CU (one of eight); each folds the chunks ahead of it, so no more than 96
  int64_t nc = 1;
  if (split) nc = std::max<int64_t>(2, std::min<int64_t>((a.f32 ? 256 : bwd ? 512 : 768) / rows, std::min<int64_t>(96, cdiv(a.S, tt))));
  // a chunk is addressed in 32 bits (y's stride covers a row, so this holds for inputs whose rows reach into the next ones too)
  const int64_t st = std::max(std::max(a.xs[1], a.rs[1]), std::max(a.gs[1], a.ys[1])) * (a.f32 ? 4 : 2);
  const int64_t most = std::max<int64_t>(1, kBufMax / std::max<int64_t>(st, 1) / tt) * tt;
  p.chunk = (int)std::min(cdiv(cdiv(a.S, nc), tt) * tt, most);
  p.nc = (int)cdiv(a.S, p.chunk);
  return p;
}

ScArgs make_args(const Scan& a, const Plan& p, const void* x, const void* r, const void* g, const float* decay,
                 const int32_t* len) {
  ScArgs k{};
  k.x = x; k.r = r; k.g = g; k.decay = decay; k.len = len;
  for (int i = 0; i < 2; ++i) { k.xs[i] = a.xs[i]; k.rs[i] = a.rs[i]; k.gs[i] = a.gs[i]; k.ys[i] = a.ys[i]; }
  k.B = a.B; k.S = a.S; k.D = a.D; k.reverse = a.reverse; k.sharp = a.sharp;
  k.slabs = p.slabs; k.nc = p.nc; k.chunk = p.chunk;
  return k;
}
size_t maps_bytes(const Scan& a, const Plan& p) { return align256((size_t)a.B * p.nc * a.D * 2 * sizeof(float)); }

enum { kFwd, kFwdSplit, kMaps, kBwd, kBwdSplit, kBackMaps };
template <typename F>
void launch1(int what, hipStream_t st, const ScArgs& k, unsigned blocks) {
  const dim3 g(blocks), b(F::NW * 64);
  switch (what) {
    case kFwd: hipLaunchKernelGGL((k_scan_fwd<F, false>), g, b, 0, st, k); break;
    case kFwdSplit: hipLaunchKernelGGL((k_scan_fwd<F, true>), g, b, 0, st, k); break;
    case kMaps: hipLaunchKernelGGL((k_scan_maps<F>), g, b, 0, st, k); break;
    case kBwd: hipLaunchKernelGGL((k_scan_bwd<F, false>), g, b, 0, st, k); break;
    case kBwdSplit: hipLaunchKernelGGL((k_scan_bwd<F, true>), g, b, 0, st, k); break;
    case kBackMaps: hipLaunchKernelGGL((k_scan_back_maps<F>), g, b, 0, st, k); break;
  }
  PG_LAUNCH_CHECK();
}
void launch(int what, hipStream_t st, const Scan& a, const Plan& p, const ScArgs& k) {
  const unsigned blocks = (unsigned)(cdiv((int64_t)a.B * p.slabs * p.nc, 8) * 8);
#define PG_SC(CL, NW)                                                  \
  if (p.cl == CL && p.nw == NW) {                                      \
    if (!a.f32) return launch1<Form<bf16_t, CL, NW>>(what, st, k, blocks);                      \
    if constexpr (Form<float, CL, NW>::TT % kKeep == 0) return launch1<Form<float, CL, NW>>(what, st, k, blocks); \
  }
  PG_SC(32, 8)
  PG_SC(32, 4)
#undef PG_SC
  throw Error{-2, "scan: no such form"};
}

}  // namespace

size_t scan_saved_bytes(const Scan& a) {
  return align256((size_t)a.B * cdiv(a.S, plan_of(a, false).cl ? kKeep : kStep) * a.D * sizeof(float));
}
size_t scan_ws_bytes(const Scan& a) {
  const Plan f = plan_of(a, false), b = plan_of(a, true);
  return std::max(maps_bytes(a, f), maps_bytes(a, b) + align256((size_t)a.B * b.nc * a.D * sizeof(double)));
}

void scan_fwd(hipStream_t st, const Scan& a, const void* x, const void* r, const void* g, const float* decay,
              const int32_t* len, const float* h0, void* y, float* ht, void* saved, void* ws) {
  const Plan p = plan_of(a, false);
  ScArgs k = make_args(a, p, x, r, g, decay, len);
  k.h0 = h0; k.y = y; k.ht = ht; k.saved = (float*)saved; k.maps = (float*)ws;
  ProfScope prof(st);
  if (!p.cl) {
    const dim3 grid((unsigned)a.B, (unsigned)cdiv(a.D, 128));
    if (a.f32) hipLaunchKernelGGL(k_scan_seq_fwd<float>, grid, dim3(64), 0, st, k);
    else hipLaunchKernelGGL(k_scan_seq_fwd<bf16_t>, grid, dim3(64), 0, st, k);
    PG_LAUNCH_CHECK();
  } else if (p.nc == 1) {
    launch(kFwd, st, a, p, k);
  } else {
    launch(kMaps, st, a, p, k);
    launch(kFwdSplit, st, a, p, k);
  }
  prof.done_bytes("k_scan_fwd", (a.f32 ? 16.0 : 8.0) * a.B * a.S * a.D);
}

void scan_bwd(hipStream_t st, const Scan& a, const void* x, const void* r, const void* g, const float* decay,
              const int32_t* len, const void* saved, const void* dy, const float* dht, void* dx, void* dr, void* dg,
              float* ddecay, float* dh0, void* ws) {
  const Plan p = plan_of(a, true);
  ScArgs k = make_args(a, p, x, r, g, decay, len);
  k.dy = dy; k.h0 = dht; k.ht = dh0; k.y = dx; k.dr = dr; k.dg = dg; k.saved = (float*)const_cast<void*>(saved);
  k.maps = (float*)ws;
  k.part = (double*)((char*)ws + maps_bytes(a, p));
  ProfScope prof(st);
  if (!p.cl) {
    const dim3 grid((unsigned)a.B, (unsigned)cdiv(a.D, 128));
    if (a.f32) hipLaunchKernelGGL(k_scan_seq_bwd<float>, grid, dim3(64), 0, st, k);
    else hipLaunchKernelGGL(k_scan_seq_bwd<bf16_t>, grid, dim3(64), 0, st, k);
    PG_LAUNCH_CHECK();
  } else if (p.nc == 1) {
    launch(kBwd, st, a, p, k);
  } else {
    launch(kBackMaps, st, a, p, k);
    launch(kBwdSplit, st, a, p, k);
  }
  hipLaunchKernelGGL(k_scan_decay, dim3((unsigned)cdiv(a.D, 32)), dim3(256), 0, st, k.part, decay, (int64_t)a.B * p.nc, a.D,
                     a.sharp, ddecay);
  PG_LAUNCH_CHECK();
  prof.done_bytes("k_scan_bwd", (a.f32 ? 28.0 : 14.0) * a.B * a.S * a.D);
}

}  // namespace pg
