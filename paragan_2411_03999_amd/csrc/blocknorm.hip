// The norms before and after a block with modulation, gate and residual scale
// in one pass over the rows, and the backward.
//
//   v = h or norm(h) g1;   z = x + k v,  k = res_scale gate;   y = norm(z) m + shift,  m = g2 (1 + scale)
// Backward, with n the normed z, nh the normed h (or h) and r, rh the factors:
//   t = dy m;  dZ = dz + r (t - [mean t] - n mean(t n));  dx = dZ;
//   dv = k dZ;  dh = dv, or rh (dv g1 - [mean dv g1] - nh mean(dv g1 nh));
//   over the tokens of a sequence  p = sum dZ nh,  q = sum dy n,  e = sum dy:
//   dgate = res_scale g1 p,  dg1 = res_scale sum_b gate p,  dscale = g2 q,
//   dg2 = sum_b (1 + scale) q,  dshift = e.
// ([...]: with the mean taken off only.)  z is formed again from x and h in
// the backward, so that n is that of the unrounded z in both directions; the
// statistics (four floats a row) are kept by the forward.
//
// Bound by memory: every element is read once and written once, what is
// between stays in registers in fp32.  A lane holds 8 elements of a row (a
// 16-byte access in bf16), a row lies over 8 to 64 lanes of a wave or over
// the waves of a block, whose columns' rows (k, m, shift) stay in registers
// over the tokens of one sequence that the block takes.
#include "rows.hpp"
#include "token.hpp"

namespace pg {

namespace {

constexpr int kMaxRows = 128;      // tokens of one item at most: what a column sums in fp32

struct BnArgs {
  BlockNormRows w;
  const int32_t* len;
  const void *x, *h, *dz, *dy;
  void *z, *y;                     // backward: dx, dh
  float* stats;                    // [B S][4]: mean and factor of h, of z
  float* part;                     // [items][3][D]: e, q, p
  int64_t xs[2], hs[2], zs[2], ys[2], mod;
  int S, D, R, nc;                 // tokens of an item, items of a sequence
  int layer, branch, pre;
  float eps, res_scale, inv_d;
};

PG_DEV void ld8(const float* p, float* f) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

// Sums of two values over the lanes of a row.  P = 0: over the waves of the
// block, through sh[2][16] float2, whose halves are used in turn so that one
// barrier a sum is enough: who writes a half again has passed the barrier
// that everybody reached after reading it.
template <int P>
struct RowSum {
  float2 (*sh)[16];
  int turn, wave, waves;
  PG_DEV float2 operator()(float a, float b) {
    if constexpr (P > 0) {
      return make_float2(group_sum<P>(a), group_sum<P>(b));
    } else {
      a = group_sum<64>(a);
      b = group_sum<64>(b);
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) sh[turn][wave] = make_float2(a, b);
      __syncthreads();
      float2 s = sh[turn][0];
      for (int i = 1; i < waves; ++i) {
        s.x += sh[turn][i].x;
        s.y += sh[turn][i].y;
      }
      return s;
    }
  }
};

// mean and factor of v over the row; v becomes the normed row (zeros outside)
template <int P>
PG_DEV float2 normalise(RowSum<P>& sum, bool layer, bool act, float inv_d, float eps, float* v) {
  float mean = 0.f;
  if (layer) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[e];
    mean = sum(s, 0.f).x * inv_d;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act ? v[e] - mean : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(v[e], v[e], s);
  const float r = __builtin_amdgcn_rsqf(fmaf(sum(s, 0.f).x, inv_d, eps));
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= r;
  return make_float2(mean, r);
}

template <typename TX, typename TH, int P, bool POST>
__global__ __launch_bounds__(P ? 256 : 1024) void k_blocknorm_fwd(BnArgs a) {
  __shared__ float2 sh[2][16];
  constexpr int NG = P ? 256 / P : 1;
  const int tid = threadIdx.x, grp = P ? tid / P : 0, ch = P ? tid % P : tid;
  const bool act = ch * 8 < a.D;
  const int c8 = act ? ch * 8 : 0;
  const int b = blockIdx.x / a.nc, r0 = (blockIdx.x - b * a.nc) * a.R, r1 = min(a.S, r0 + a.R);
  const int len = a.len ? min(max(a.len[b], 0), a.S) : a.S;
  RowSum<P> sum{sh, 0, tid >> 6, (int)blockDim.x >> 6};
  float k[8], m[8], f[8], g1[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { k[e] = a.res_scale; m[e] = 1.f; f[e] = 0.f; g1[e] = 1.f; }
  if (a.branch && a.w.gate) {
    ld8(a.w.gate + b * a.mod + c8, k);
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] *= a.res_scale;
  }
  if (POST && a.w.gain_post) ld8(a.w.gain_post + c8, g1);
  if (a.w.gain_pre) ld8(a.w.gain_pre + c8, m);
  if (a.w.scale) {
    float s[8];
    ld8(a.w.scale + b * a.mod + c8, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] *= 1.f + s[e];
  }
  if (a.w.shift) ld8(a.w.shift + b * a.mod + c8, f);
  const TX* x = (const TX*)a.x + b * a.xs[0] + c8;
  const TH* h = (const TH*)a.h + b * a.hs[0] + c8;
  TX* z = (TX*)a.z + b * a.zs[0] + c8;
  TH* y = (TH*)a.y + b * a.ys[0] + c8;
  for (int rr = r0; rr < r1; rr += NG) {       // as often for every group
    const int r = min(rr + grp, r1 - 1);
    const bool ok = act && rr + grp < r1, real = act && r < len;
    float xv[8] = {}, hv[8] = {};
    if (real) {
      Raw<TX> q;
      q.load(x + r * a.xs[1]);
      q.get(xv);
      if (a.branch) {
        Raw<TH> p;
        p.load(h + r * a.hs[1]);
        p.get(hv);
      }
    }
    float2 sth = make_float2(0.f, 1.f);
    if constexpr (POST) sth = normalise<P>(sum, a.layer, act, a.inv_d, a.eps, hv);
    if (a.branch) {
#pragma unroll
      for (int e = 0; e < 8; ++e) xv[e] = real ? fmaf(k[e], POST ? hv[e] * g1[e] : hv[e], xv[e]) : 0.f;
      if (ok) st8f<TX>(z + r * a.zs[1], xv);
    }
    if (a.pre) {
      const float2 stz = normalise<P>(sum, a.layer, act, a.inv_d, a.eps, xv);
#pragma unroll
      for (int e = 0; e < 8; ++e) xv[e] = real ? fmaf(xv[e], m[e], f[e]) : 0.f;
      if (ok) st8f<TH>(y + r * a.ys[1], xv);
      if (a.stats && ok && ch == 0)
        reinterpret_cast<float4*>(a.stats)[(int64_t)b * a.S + r] = make_float4(sth.x, sth.y, stz.x, stz.y);
    } else if (a.stats && ok && ch == 0) {
      reinterpret_cast<float4*>(a.stats)[(int64_t)b * a.S + r] = make_float4(sth.x, sth.y, 0.f, 0.f);
    }
  }
}

template <typename TX, typename TH, int P, bool POST>
__global__ __launch_bounds__(P ? 256 : 1024) void k_blocknorm_bwd(BnArgs a) {
  __shared__ float2 sh[2][16];
  constexpr int NG = P ? 256 / P : 1;
  const int tid = threadIdx.x, grp = P ? tid / P : 0, ch = P ? tid % P : tid;
  const bool act = ch * 8 < a.D;
  const int c8 = act ? ch * 8 : 0;
  const int b = blockIdx.x / a.nc, r0 = (blockIdx.x - b * a.nc) * a.R, r1 = min(a.S, r0 + a.R);
  const int len = a.len ? min(max(a.len[b], 0), a.S) : a.S;
  RowSum<P> sum{sh, 0, tid >> 6, (int)blockDim.x >> 6};
  float k[8], m[8], se[8] = {}, sq[8] = {}, sp[8] = {};
#pragma unroll
  for (int e = 0; e < 8; ++e) { k[e] = a.res_scale; m[e] = 1.f; }
  if (a.branch && a.w.gate) {
    ld8(a.w.gate + b * a.mod + c8, k);
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] *= a.res_scale;
  }
  if (POST && a.w.gain_post) {
    float g1[8];
    ld8(a.w.gain_post + c8, g1);
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] *= g1[e];
  }
  if (a.w.gain_pre) ld8(a.w.gain_pre + c8, m);
  if (a.w.scale) {
    float s[8];
    ld8(a.w.scale + b * a.mod + c8, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] *= 1.f + s[e];
  }
  const TX* x = (const TX*)a.x + b * a.xs[0] + c8;
  const TH* h = (const TH*)a.h + b * a.hs[0] + c8;
  const TX* dz = (const TX*)a.dz + b * a.zs[0] + c8;
  const TH* dy = (const TH*)a.dy + b * a.ys[0] + c8;
  TX* dx = (TX*)a.z + b * a.xs[0] + c8;
  TH* dh = (TH*)a.y + b * a.hs[0] + c8;
  for (int rr = r0; rr < r1; rr += NG) {
    const int r = min(rr + grp, r1 - 1);
    const bool ok = act && rr + grp < r1, real = ok && r < len;
    float n[8] = {}, hn[8] = {}, dZ[8] = {}, dv[8] = {};
    const float4 st = reinterpret_cast<const float4*>(a.stats)[(int64_t)b * a.S + r];
    if (real) {
      Raw<TX> q;
      Raw<TH> p;
      if (a.branch) {
        p.load(h + r * a.hs[1]);
        p.get(hn);
      }
      if (a.dz) {
        q.load(dz + r * a.zs[1]);
        q.get(dZ);
      }
      if (a.pre) {
        q.load(x + r * a.xs[1]);
        q.get(n);
        p.load(dy + r * a.ys[1]);
        p.get(dv);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (POST) hn[e] = (hn[e] - st.x) * st.y;
        if (a.branch) n[e] = fmaf(k[e], hn[e], n[e]);
        n[e] = (n[e] - st.z) * st.w;
      }
    }
    if (a.pre) {
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        se[e] += dv[e];
        sq[e] = fmaf(dv[e], n[e], sq[e]);
        dv[e] *= m[e];
        s1 += dv[e];
        s2 = fmaf(dv[e], n[e], s2);
      }
      const float2 s = sum(s1, s2);
      const float c1 = a.layer ? s.x * a.inv_d : 0.f, c2 = s.y * a.inv_d;
#pragma unroll
      for (int e = 0; e < 8; ++e) dZ[e] = real ? fmaf(st.w, dv[e] - c1 - n[e] * c2, dZ[e]) : 0.f;
    }
    if (ok) st8f<TX>(dx + r * a.xs[1], dZ);
    if (a.branch) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sp[e] = fmaf(dZ[e], hn[e], sp[e]);
        dv[e] = dZ[e] * k[e];
      }
      if constexpr (POST) {
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s1 += dv[e];
          s2 = fmaf(dv[e], hn[e], s2);
        }
        const float2 s = sum(s1, s2);
        const float c1 = a.layer ? s.x * a.inv_d : 0.f, c2 = s.y * a.inv_d;
#pragma unroll
        for (int e = 0; e < 8; ++e) dv[e] = real ? st.y * (dv[e] - c1 - hn[e] * c2) : 0.f;
      }
      if (ok) st8f<TH>(dh + r * a.hs[1], dv);
    }
  }
  // the item's column sums: the groups' in group order
  float* part = a.part + (int64_t)blockIdx.x * 3 * a.D;
  if constexpr (P == 0) {
    if (act) {
#pragma unroll
      for (int w = 0; w < 3; ++w) st8f<float>(part + (int64_t)w * a.D + c8, w == 0 ? se : w == 1 ? sq : sp);
    }
  } else {
    __shared__ float cols[256 * 8];
#pragma unroll
    for (int w = 0; w < 3; ++w) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) cols[tid * 8 + e] = w == 0 ? se[e] : w == 1 ? sq[e] : sp[e];
      __syncthreads();
      for (int c = tid; c < a.D; c += 256) {
        double s = 0.0;
        for (int j = 0; j < NG; ++j) s += cols[j * P * 8 + c];
        part[(int64_t)w * a.D + c] = (float)s;
      }
    }
  }
}

struct BnJoin {
  BlockNormRows w;
  BlockNormGrads g;
  const float* part;
  double* seq;                     // [B][3][D], sums of every sequence
  int64_t mod;
  int B, D, nc;
  float res_scale;
};

// Sums over the items of one sequence (blockIdx.x): 32 columns x 8 item lanes
// a block, in order, in 64 bits; the sequence's own gradients from them.
__global__ __launch_bounds__(256) void k_blocknorm_seq(BnJoin a) {
  __shared__ double sh[3][8][33];
  const int j = threadIdx.x & 31, l = threadIdx.x >> 5, c = blockIdx.y * 32 + j, b = blockIdx.x;
  double s[3] = {0.0, 0.0, 0.0};
  if (c < a.D) {
    const float* p = a.part + (int64_t)b * a.nc * 3 * a.D + c;
#pragma unroll 4
    for (int i = l; i < a.nc; i += 8)
#pragma unroll
      for (int w = 0; w < 3; ++w) s[w] += p[((int64_t)i * 3 + w) * a.D];
  }
#pragma unroll
  for (int w = 0; w < 3; ++w) sh[w][l][j] = s[w];
  __syncthreads();
  if (l > 0 || c >= a.D) return;
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    s[w] = 0.0;
    for (int i = 0; i < 8; ++i) s[w] += sh[w][i][j];
    if (a.seq) a.seq[((int64_t)b * 3 + w) * a.D + c] = s[w];
  }
  if (a.mod) {
    const int64_t o = b * a.mod + c;
    if (a.g.shift) a.g.shift[o] = (float)s[0];
    if (a.g.scale) a.g.scale[o] = (float)((a.w.gain_pre ? a.w.gain_pre[c] : 1.0) * s[1]);
    if (a.g.gate) a.g.gate[o] = (float)((double)a.res_scale * (a.w.gain_post ? a.w.gain_post[c] : 1.0) * s[2]);
  }
}

// Sums over the sequences: the gains' gradients, and those of shared rows
__global__ __launch_bounds__(256) void k_blocknorm_join(BnJoin a) {
  __shared__ double sh[5][8][33];
  const int j = threadIdx.x & 31, l = threadIdx.x >> 5, c = blockIdx.x * 32 + j;
  double s[5] = {0.0, 0.0, 0.0, 0.0, 0.0};   // e, q, p, (1 + scale) q, gate p
  if (c < a.D) {
#pragma unroll 2
    for (int b = l; b < a.B; b += 8) {
      const double* p = a.seq + (int64_t)b * 3 * a.D + c;
      const double e = p[0], q = p[a.D], pp = p[2 * (int64_t)a.D];
      s[0] += e; s[1] += q; s[2] += pp;
      s[3] += (1.0 + (a.w.scale ? a.w.scale[b * a.mod + c] : 0.0)) * q;
      s[4] += (a.w.gate ? a.w.gate[b * a.mod + c] : 1.0) * pp;
    }
  }
#pragma unroll
  for (int w = 0; w < 5; ++w) sh[w][l][j] = s[w];
  __syncthreads();
  if (l > 0 || c >= a.D) return;
#pragma unroll
  for (int w = 0; w < 5; ++w) {
    s[w] = 0.0;
    for (int i = 0; i < 8; ++i) s[w] += sh[w][i][j];
  }
  if (a.g.gain_pre) a.g.gain_pre[c] = (float)s[3];
  if (a.g.gain_post) a.g.gain_post[c] = (float)((double)a.res_scale * s[4]);
  if (!a.mod) {
    if (a.g.shift) a.g.shift[c] = (float)s[0];
    if (a.g.scale) a.g.scale[c] = (float)((a.w.gain_pre ? a.w.gain_pre[c] : 1.0) * s[1]);
    if (a.g.gate) a.g.gate[c] = (float)((double)a.res_scale * (a.w.gain_post ? a.w.gain_post[c] : 1.0) * s[2]);
  }
}

// lanes of a row inside a wave, or 0 where it lies over a block's waves
int row_lanes(int D) {
  for (int p = 8; p <= 64; p *= 2)
    if (D <= 8 * p) return p;
  return 0;
}

// Items: tokens of one sequence a block takes; enough of them to fill the
// card (`want` blocks) and at most kMaxRows a thread, whole rounds of groups.
void split(const BlockNorm& a, int64_t want, int& R, int& nc) {
  const int p = row_lanes(a.D), ng = p ? 256 / p : 1;
  int64_t r = cdiv((int64_t)a.B * a.S, want);
  r = std::min<int64_t>(cdiv(std::max<int64_t>(r, 1), ng) * ng, (int64_t)kMaxRows * ng);
  R = (int)r;
  nc = (int)cdiv(a.S, r);
}

BnArgs make_args(const BlockNorm& a, const BlockNormRows& w, const int32_t* len, const void* x, const void* h) {
  BnArgs g{};
  g.w = w; g.len = len; g.x = x; g.h = h;
  for (int i = 0; i < 2; ++i) { g.xs[i] = a.xs[i]; g.hs[i] = a.hs[i]; g.zs[i] = a.zs[i]; g.ys[i] = a.ys[i]; }
  g.mod = a.mod; g.S = a.S; g.D = a.D; g.layer = a.layer; g.branch = a.branch; g.pre = a.pre;
  g.eps = a.eps; g.res_scale = a.res_scale; g.inv_d = 1.f / (float)a.D;
  return g;
}

template <bool BWD, typename TX, typename TH, bool POST>
void launch2(hipStream_t st, const BlockNorm& a, const BnArgs& g) {
  const int p = row_lanes(a.D);
  const dim3 grid((unsigned)((int64_t)a.B * g.nc)), blk(p ? 256 : (unsigned)cdiv(a.D, 512) * 64);
#define PG_BN(P)                                                                              \
  case P:                                                                                     \
    if (BWD) hipLaunchKernelGGL((k_blocknorm_bwd<TX, TH, P, POST>), grid, blk, 0, st, g);     \
    else hipLaunchKernelGGL((k_blocknorm_fwd<TX, TH, P, POST>), grid, blk, 0, st, g);         \
    break;
  switch (p) { PG_BN(8) PG_BN(16) PG_BN(32) PG_BN(64) PG_BN(0) }
#undef PG_BN
  PG_LAUNCH_CHECK();
}
template <bool BWD>
void launch(hipStream_t st, const BlockNorm& a, const BnArgs& g) {
#define PG_BN(TX, TH)                                              \
  (a.post ? launch2<BWD, TX, TH, true>(st, a, g) : launch2<BWD, TX, TH, false>(st, a, g))
  if (a.f32) PG_BN(float, float);
  else if (a.res32) PG_BN(float, bf16_t);
  else PG_BN(bf16_t, bf16_t);
#undef PG_BN
}

constexpr int64_t kFwdItems = 4096, kBwdItems = 1024;

}  // namespace

size_t blocknorm_saved_bytes(const BlockNorm& a) { return align256((size_t)a.B * a.S * 16); }

size_t blocknorm_ws_bytes(const BlockNorm& a) {
  int R, nc;
  split(a, kBwdItems, R, nc);
  return align256((size_t)a.B * nc * 3 * a.D * sizeof(float)) + align256((size_t)a.B * 3 * a.D * sizeof(double));
}

void blocknorm_fwd(hipStream_t st, const BlockNorm& a, const BlockNormRows& w, const void* x, const void* h,
                   const int32_t* len, void* z, void* y, void* saved) {
  BnArgs g = make_args(a, w, len, x, h);
  g.z = z; g.y = y; g.stats = (float*)saved;
  split(a, kFwdItems, g.R, g.nc);
  ProfScope prof(st);
  launch<false>(st, a, g);
  const double one = (a.res32 ? 4.0 : 2.0) * (1 + a.branch) + (a.f32 ? 4.0 : 2.0) * (a.branch + a.pre);
  prof.done_bytes("k_blocknorm_fwd", one * a.B * a.S * a.D);
}

void blocknorm_bwd(hipStream_t st, const BlockNorm& a, const BlockNormRows& w, const void* x, const void* h,
                   const int32_t* len, const void* saved, const void* dz, const void* dy, void* dx, void* dh,
                   const BlockNormGrads& gr, void* ws) {
  BnArgs g = make_args(a, w, len, x, h);
  g.dz = dz; g.dy = dy; g.z = dx; g.y = dh; g.stats = (float*)const_cast<void*>(saved); g.part = (float*)ws;
  split(a, kBwdItems, g.R, g.nc);
  ProfScope prof(st);
  launch<true>(st, a, g);
  BnJoin j{w, gr, g.part, nullptr, a.mod, a.B, a.D, g.nc, a.res_scale};
  const bool shared = gr.gain_pre || gr.gain_post || (!a.mod && (gr.gate || gr.scale || gr.shift));
  if (shared) j.seq = (double*)((char*)ws + align256((size_t)a.B * g.nc * 3 * a.D * sizeof(float)));
  if (shared || gr.gate || gr.scale || gr.shift) {
    hipLaunchKernelGGL(k_blocknorm_seq, dim3((unsigned)a.B, (unsigned)cdiv(a.D, 32)), dim3(256), 0, st, j);
    PG_LAUNCH_CHECK();
  }
  if (shared) {
    hipLaunchKernelGGL(k_blocknorm_join, dim3((unsigned)cdiv(a.D, 32)), dim3(256), 0, st, j);
    PG_LAUNCH_CHECK();
  }
  const double one = (a.res32 ? 4.0 : 2.0) * (1 + (dz ? 1 : 0) + a.pre) + (a.f32 ? 4.0 : 2.0) * (2 * a.branch + a.pre);
  prof.done_bytes("k_blocknorm_bwd", one * a.B * a.S * a.D);
}

}  // namespace pg
