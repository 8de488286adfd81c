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
// over the tokens of one sequence that the block takes.  The backward's
// blocks fill a CU with rows side by side, so that few blocks have column sums
// to be joined, and a row's loads are under way while the one before it is
// summed.
// Measured, bf16: forward of 8 x 4096 x 1152 with a normed branch 59 us (5.1
// TB/s; a copy reaches 5.2), backward 92 us (4.9) and 9 us to join the column
// sums; fp32 stream, 3 x 1365 x 1480 padded, 13 and 27 + 8 us.  Before the
// loads ahead and the rows side by side that backward took 165 us.
#include "rows.hpp"
#include "token.hpp"
#include <type_traits>

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
  int branch, pre;
  float eps, res_scale, inv_d;
};

PG_DEV void ld8(const float* p, float* f) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

// Element c of the row at p + row: a uniform address and a lane's 32-bit
// offset where a row lies over a block.
template <typename T>
PG_DEV T* place(T* p, int64_t row, int c) {
  typedef typename std::conditional<std::is_const<T>::value, const char, char>::type B;
  return reinterpret_cast<T*>(reinterpret_cast<B*>(p + row) + (uint32_t)(c * (int)sizeof(T)));
}

// Sums of one or two values over the lanes of a row.  P = 0: over the waves of the
// block, through sh[2][16] float2, whose halves are used in turn so that one
// barrier a sum is enough: who writes a half again has passed the barrier
// that everybody reached after reading it.
template <int P>
struct RowSum {
  float2 (*sh)[16];
  int turn, wave, first, waves;    // this wave; the row's first and how many
  PG_DEV float operator()(float a) {
    if constexpr (P > 0) {
      return group_sum<P>(a);
    } else {
      a = group_sum<64>(a);
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) sh[turn][wave].x = a;
      __syncthreads();
      const int i = threadIdx.x & 15;
      return group_sum<16>(i < waves ? sh[turn][first + i].x : 0.f);
    }
  }
  PG_DEV float2 operator()(float a, float b) {
    if constexpr (P > 0) {
      return make_float2(group_sum<P>(a), group_sum<P>(b));
    } else {
      a = group_sum<64>(a);
      b = group_sum<64>(b);
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) sh[turn][wave] = make_float2(a, b);
      __syncthreads();
      // every 16 lanes sum the waves' once more: one read, and lane moves
      const int i = threadIdx.x & 15;
      const float2 s = i < waves ? sh[turn][first + i] : make_float2(0.f, 0.f);
      return make_float2(group_sum<16>(s.x), group_sum<16>(s.y));
    }
  }
};

// mean and factor of v over the row; v becomes the normed row (zeros outside)
template <int P, bool LAYER>
PG_DEV float2 normalise(RowSum<P>& sum, bool act, float inv_d, float eps, float* v) {
  float mean = 0.f;
  if constexpr (LAYER) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[e];
    mean = sum(s) * inv_d;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act ? v[e] - mean : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(v[e], v[e], s);
  const float r = __builtin_amdgcn_rsqf(fmaf(sum(s), inv_d, eps));
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= r;
  return make_float2(mean, r);
}

template <typename TX, typename TH, int P, bool POST, bool LAYER>
__global__ __launch_bounds__(P ? 256 : 1024) void k_blocknorm_fwd(BnArgs a) {
  __shared__ float2 sh[2][16];
  constexpr int NG = P ? 256 / P : 1;
  const int tid = threadIdx.x, ch = P ? tid % P : tid;
  const int grp = P == 0 ? 0 : P == 64 ? __builtin_amdgcn_readfirstlane(tid / 64) : tid / P;
  const bool act = ch * 8 < a.D;
  const int c8 = act ? ch * 8 : 0;
  const int b = blockIdx.x / a.nc, r0 = (blockIdx.x - b * a.nc) * a.R, r1 = min(a.S, r0 + a.R);
  const int len = __builtin_amdgcn_readfirstlane(a.len ? min(max(a.len[b], 0), a.S) : a.S);
  RowSum<P> sum{sh, 0, tid >> 6, 0, (int)blockDim.x >> 6};
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
  const TX* x = (const TX*)a.x + b * a.xs[0];
  const TH* h = (const TH*)a.h + b * a.hs[0];
  TX* z = (TX*)a.z + b * a.zs[0];
  TH* y = (TH*)a.y + b * a.ys[0];
  for (int rr = r0; rr < r1; rr += NG) {       // as often for every group
    const int r = min(rr + grp, r1 - 1);
    const bool ok = act && rr + grp < r1, real = act && r < len;
    float xv[8] = {}, hv[8] = {};
    if (real) {
      Raw<TX> q;
      q.load(place(x, r * a.xs[1], c8));
      q.get(xv);
      if (a.branch) {
        Raw<TH> p;
        p.load(place(h, r * a.hs[1], c8));
        p.get(hv);
      }
    }
    float2 sth = make_float2(0.f, 1.f);
    if constexpr (POST) sth = normalise<P, LAYER>(sum, act, a.inv_d, a.eps, hv);
    if (a.branch) {
#pragma unroll
      for (int e = 0; e < 8; ++e) xv[e] = real ? fmaf(k[e], POST ? hv[e] * g1[e] : hv[e], xv[e]) : 0.f;
      if (ok) st8f<TX>(place(z, r * a.zs[1], c8), xv);
    }
    if (a.pre) {
      const float2 stz = normalise<P, LAYER>(sum, act, a.inv_d, a.eps, xv);
#pragma unroll
      for (int e = 0; e < 8; ++e) xv[e] = real ? fmaf(xv[e], m[e], f[e]) : 0.f;
      if (ok) st8f<TH>(place(y, r * a.ys[1], c8), xv);
      if (a.stats && ok && ch == 0)
        reinterpret_cast<float4*>(a.stats)[(int64_t)b * a.S + r] = make_float4(sth.x, sth.y, stz.x, stz.y);
    } else if (a.stats && ok && ch == 0) {
      reinterpret_cast<float4*>(a.stats)[(int64_t)b * a.S + r] = make_float4(sth.x, sth.y, 0.f, 0.f);
    }
  }
}

template <typename TX, typename TH, int P, bool POST, bool LAYER, int THREADS>
__global__ __launch_bounds__(THREADS) void k_blocknorm_bwd(BnArgs a) {
  __shared__ float2 sh[2][16];
  // lanes of a row, rows a block takes side by side
  const int tid = threadIdx.x, W = P ? P : (a.D + 511) / 512 * 64, NG = (int)blockDim.x / W;
  const int grp = P == 0 || P == 64 ? __builtin_amdgcn_readfirstlane(tid / W) : tid / W, ch = tid - grp * W;
  const bool act = ch * 8 < a.D;
  const int c8 = act ? ch * 8 : 0;
  const int b = blockIdx.x / a.nc, r0 = (blockIdx.x - b * a.nc) * a.R, r1 = min(a.S, r0 + a.R);
  const int len = __builtin_amdgcn_readfirstlane(a.len ? min(max(a.len[b], 0), a.S) : a.S);
  RowSum<P> sum{sh, 0, tid >> 6, grp * (W >> 6), W >> 6};
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
  const TX* x = (const TX*)a.x + b * a.xs[0];
  const TH* h = (const TH*)a.h + b * a.hs[0];
  const TX* dz = (const TX*)a.dz + b * a.zs[0];
  const TH* dy = (const TH*)a.dy + b * a.ys[0];
  TX* dx = (TX*)a.z + b * a.xs[0];
  TH* dh = (TH*)a.y + b * a.hs[0];
  // the next row's loads are under way while this one is summed; rows that are none read one that is
  Raw<TX> xr{}, zr{};
  Raw<TH> hr{}, yr{};
  float4 sr;
  auto fetch = [&](int r) {
    const int64_t q = min(r, max(len - 1, 0));
    sr = reinterpret_cast<const float4*>(a.stats)[(int64_t)b * a.S + q];
    if (a.branch) hr.load(place(h, q * a.hs[1], c8));
    if (a.dz) zr.load(place(dz, q * a.zs[1], c8));
    if (a.pre) {
      xr.load(place(x, q * a.xs[1], c8));
      yr.load(place(dy, q * a.ys[1], c8));
    }
  };
  fetch(r0 + grp);
  // lanes past the row's end take part with rows of zeros
  if (!act) {
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = m[e] = 0.f;
  }
  const int rl = min(r1, len);
  // mean of t and of t n, and r (t - [mean t] - n mean(t n))
  auto back = [&](const float* t, const float* n, float& c1, float& c2) {
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (LAYER) s1 += t[e];
      s2 = fmaf(t[e], n[e], s2);
    }
    if constexpr (LAYER) {
      const float2 s = sum(s1, s2);
      c1 = s.x * a.inv_d;
      c2 = s.y * a.inv_d;
    } else {
      c1 = 0.f;
      c2 = sum(s2) * a.inv_d;
    }
  };
  for (int rr = r0; rr < r1; rr += NG) {
    const int r = rr + grp;
    const bool ok = act && r < r1;
    float n[8], hn[8], dZ[8], dv[8];
    float4 st = sr;
    xr.get(n);
    hr.get(hn);
    zr.get(dZ);
    yr.get(dv);
    if (rr + NG < r1) fetch(rr + NG + grp);
    if (r >= rl) {                 // no token, nor any after it: zeros throughout, the condition's rows (which may not be finite) too
      st = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int e = 0; e < 8; ++e) n[e] = hn[e] = dZ[e] = dv[e] = k[e] = m[e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (POST) hn[e] = (LAYER ? hn[e] - st.x : hn[e]) * st.y;
      if (a.branch) n[e] = fmaf(k[e], hn[e], n[e]);
      n[e] = (LAYER ? n[e] - st.z : n[e]) * st.w;
    }
    if (a.pre) {
      float c1, c2;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        se[e] += dv[e];
        sq[e] = fmaf(dv[e], n[e], sq[e]);
        dv[e] *= m[e];
      }
      back(dv, n, c1, c2);
#pragma unroll
      for (int e = 0; e < 8; ++e) dZ[e] = fmaf(st.w, fmaf(-n[e], c2, LAYER ? dv[e] - c1 : dv[e]), dZ[e]);
    }
    if (ok) st8f<TX>(place(dx, r * a.xs[1], c8), dZ);
    if (a.branch) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sp[e] = fmaf(dZ[e], hn[e], sp[e]);
        dv[e] = dZ[e] * k[e];
      }
      if constexpr (POST) {
        float c1, c2;
        back(dv, hn, c1, c2);
#pragma unroll
        for (int e = 0; e < 8; ++e) dv[e] = st.y * fmaf(-hn[e], c2, LAYER ? dv[e] - c1 : dv[e]);
      }
      if (ok) st8f<TH>(place(dh, r * a.hs[1], c8), dv);
    }
  }
  // the item's column sums: the groups' in group order
  float* part = a.part + (int64_t)blockIdx.x * 3 * a.D;
  if (NG == 1) {
    if (act) {
      st8f<float>(part + c8, se);
      st8f<float>(part + a.D + c8, sq);
      st8f<float>(part + 2 * (int64_t)a.D + c8, sp);
    }
    return;
  }
  __shared__ float cols[3][THREADS * 8];
  st8f<float>(cols[0] + tid * 8, se);
  st8f<float>(cols[1] + tid * 8, sq);
  st8f<float>(cols[2] + tid * 8, sp);
  __syncthreads();
  const int n = W * 8;             // floats of a group
  for (int i = tid; i < 3 * a.D; i += blockDim.x) {
    const int w = i / a.D, c = i - w * a.D;
    double s = 0.0;
    for (int j = 0; j < NG; ++j) s += cols[w][j * n + c];
    part[i] = (float)s;
  }
}

constexpr int kAhead = 16;         // items of a lane whose loads are under way together

struct BnJoin {
  BlockNormRows w;
  BlockNormGrads g;
  const int32_t* len;
  const float* part;
  int64_t mod;
  int B, D, nc, gs;                // gs: lanes that share a sequence's items, a power of two
  float res_scale;
};

// The rows' gradients from the items' sums, in 64 bits and in order: 16
// columns x 64 lanes a block.  Lanes take sequences; where these are fewer, gs
// lanes share the items of one.  What all sequences share is summed over the
// lanes at the end.  A sequence of no tokens adds nothing, whatever its rows
// hold: zero times what is not finite would be NaN.
template <bool LEN>
__global__ __launch_bounds__(1024) void k_blocknorm_join(BnJoin a) {
  __shared__ double sh[5][64][17];
  const int j = threadIdx.x & 15, l = threadIdx.x >> 4, c = blockIdx.x * 16 + j, cc = min(c, a.D - 1);
  const int grp = l / a.gs, li = l % a.gs, ng = 64 / a.gs;
  const double g1 = a.w.gain_post ? a.w.gain_post[cc] : 1.0, g2 = a.w.gain_pre ? a.w.gain_pre[cc] : 1.0;
  const double rs = a.res_scale;
  double t[5] = {0.0, 0.0, 0.0, 0.0, 0.0};   // over the sequences: e, q, p, (1 + scale) q, gate p
  auto weight = [&](const float* w, int b, double none) { return w ? (double)w[b * a.mod + cc] : none; };
  // (without tokens, n <= 0, the sums are zeros)
  auto done = [&](int b, int n, double e, double q, double p, double scale, double gate) {
    const int64_t o = b * a.mod + cc;
    const bool some = !LEN || n > 0;
    t[0] += e; t[1] += q; t[2] += p;
    t[3] += some ? (1.0 + scale) * q : 0.0;
    t[4] += some ? gate * p : 0.0;
    if (a.mod && c < a.D) {
      if (a.g.shift) a.g.shift[o] = (float)e;
      if (a.g.scale) a.g.scale[o] = some ? (float)(g2 * q) : 0.f;
      if (a.g.gate) a.g.gate[o] = some ? (float)(rs * g1 * p) : 0.f;
    }
  };
  double s[3] = {0.0, 0.0, 0.0}, scale = 0.0, gate = 0.0;
  int n = 1;
  for (int b = grp; b < a.B; b += ng) {
    if (LEN) n = a.len[b];
    scale = weight(a.w.scale, b, 0.0);
    gate = weight(a.w.gate, b, 1.0);
    const float* p = a.part + (int64_t)b * a.nc * 3 * a.D + cc;
    s[0] = s[1] = s[2] = 0.0;
    for (int i0 = li; i0 < a.nc; i0 += kAhead * a.gs) {
      float v[kAhead][3];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int w = 0; w < 3; ++w) v[u][w] = p[((int64_t)min(i0 + u * a.gs, a.nc - 1) * 3 + w) * a.D];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int w = 0; w < 3; ++w) s[w] += i0 + u * a.gs < a.nc ? v[u][w] : 0.f;
    }
    if (a.gs == 1) done(b, n, s[0], s[1], s[2], scale, gate);
  }
  if (a.gs > 1) {                  // then a group of lanes has one sequence or none
#pragma unroll
    for (int w = 0; w < 3; ++w) sh[w][l][j] = s[w];
    __syncthreads();
    if (li == 0 && grp < a.B) {
#pragma unroll
      for (int w = 0; w < 3; ++w) {
        s[w] = 0.0;
        for (int i = 0; i < a.gs; ++i) s[w] += sh[w][l + i][j];
      }
      done(grp, n, s[0], s[1], s[2], scale, gate);
    }
    __syncthreads();
  }
  if (li == 0) {
#pragma unroll
    for (int w = 0; w < 5; ++w) sh[w][grp][j] = t[w];
  }
  __syncthreads();
  if (l >= 5 || c >= a.D) return;
  double v = 0.0;
#pragma unroll 8
  for (int i = 0; i < min(ng, a.B); ++i) v += sh[l][i][j];
  if (l == 3 && a.g.gain_pre) a.g.gain_pre[c] = (float)v;
  if (l == 4 && a.g.gain_post) a.g.gain_post[c] = (float)(rs * v);
  if (a.mod) return;
  if (l == 0 && a.g.shift) a.g.shift[c] = (float)v;
  if (l == 1 && a.g.scale) a.g.scale[c] = (float)(g2 * v);
  if (l == 2 && a.g.gate) a.g.gate[c] = (float)(rs * g1 * v);
}

// lanes of a row inside a wave, or 0 where it lies over a block's waves
int row_lanes(int D) {
  for (int p = 8; p <= 64; p *= 2)
    if (D <= 8 * p) return p;
  return 0;
}

// Threads of a block, and rows it takes side by side
int row_threads(int D) { return row_lanes(D) ? row_lanes(D) : (int)cdiv(D, 512) * 64; }
// A backward's block: rows side by side on up to 12 waves, three a SIMD with
// the registers that takes, or where a row has more than six waves on up to
// 16 with 128 registers and a few of them in memory (8 x 4096 x 1152 post 172
// us against 179 on 16, 8 x 2000 x 1024 fp32 142 against 155).
int bwd_threads(int D) {
  const int t = row_threads(D);
  return (t <= 384 ? 768 : 1024) / t * t;
}

// Items: tokens of one sequence a block takes; enough of them to fill the
// card (`want` blocks) and at most kMaxRows a thread, whole rounds of groups.
// An item does not reach into another sequence, so a few more than `want` may
// come out, which leave CUs idle in a second round (7 x 585 x 1536, 259 items
// of the backward: 24.7 us where the bytes take 15), and many short sequences
// are many small items with a row of column sums each (4096 x 1 x 768 backward
// 80 and join 247 us, 16384 x 4 x 64 185 and 937).
void split(const BlockNorm& a, int threads, int64_t want, int& R, int& nc) {
  const int ng = threads / row_threads(a.D);
  int64_t r = cdiv((int64_t)a.B * a.S, want);
  r = std::min<int64_t>(cdiv(std::max<int64_t>(r, 1), ng) * ng, (int64_t)kMaxRows * ng);
  R = (int)r;
  nc = (int)cdiv(a.S, r);
}

BnArgs make_args(const BlockNorm& a, const BlockNormRows& w, const int32_t* len, const void* x, const void* h) {
  BnArgs g{};
  g.w = w; g.len = len; g.x = x; g.h = h;
  for (int i = 0; i < 2; ++i) { g.xs[i] = a.xs[i]; g.hs[i] = a.hs[i]; g.zs[i] = a.zs[i]; g.ys[i] = a.ys[i]; }
  g.mod = a.mod; g.S = a.S; g.D = a.D; g.branch = a.branch; g.pre = a.pre;
  g.eps = a.eps; g.res_scale = a.res_scale; g.inv_d = 1.f / (float)a.D;
  return g;
}

template <bool BWD, typename TX, typename TH, bool POST, bool LAYER>
void launch3(hipStream_t st, const BlockNorm& a, const BnArgs& g) {
  const int p = row_lanes(a.D);
  const dim3 grid((unsigned)((int64_t)a.B * g.nc)), blk(BWD ? bwd_threads(a.D) : p ? 256 : row_threads(a.D));
#define PG_BN(P)                                                                                                      \
  case P:                                                                                                             \
    if (!BWD) hipLaunchKernelGGL((k_blocknorm_fwd<TX, TH, P, POST, LAYER>), grid, blk, 0, st, g);                     \
    else if (blk.x <= 768) hipLaunchKernelGGL((k_blocknorm_bwd<TX, TH, P, POST, LAYER, 768>), grid, blk, 0, st, g);   \
    else if (P == 0) hipLaunchKernelGGL((k_blocknorm_bwd<TX, TH, 0, POST, LAYER, 1024>), grid, blk, 0, st, g);        \
    break;
  switch (p) { PG_BN(8) PG_BN(16) PG_BN(32) PG_BN(64) PG_BN(0) }
#undef PG_BN
  PG_LAUNCH_CHECK();
}
template <bool BWD, typename TX, typename TH>
void launch2(hipStream_t st, const BlockNorm& a, const BnArgs& g) {
  if (a.post) a.layer ? launch3<BWD, TX, TH, true, true>(st, a, g) : launch3<BWD, TX, TH, true, false>(st, a, g);
  else a.layer ? launch3<BWD, TX, TH, false, true>(st, a, g) : launch3<BWD, TX, TH, false, false>(st, a, g);
}
template <bool BWD>
void launch(hipStream_t st, const BlockNorm& a, const BnArgs& g) {
  if (a.f32) launch2<BWD, float, float>(st, a, g);
  else if (a.res32) launch2<BWD, float, bf16_t>(st, a, g);
  else launch2<BWD, bf16_t, bf16_t>(st, a, g);
}

constexpr int64_t kFwdItems = 4096, kBwdItems = 256;

}  // namespace

size_t blocknorm_saved_bytes(const BlockNorm& a) { return align256((size_t)a.B * a.S * 16); }

size_t blocknorm_ws_bytes(const BlockNorm& a) {
  int R, nc;
  split(a, bwd_threads(a.D), kBwdItems, R, nc);
  return align256((size_t)a.B * nc * 3 * a.D * sizeof(float));
}

void blocknorm_fwd(hipStream_t st, const BlockNorm& a, const BlockNormRows& w, const void* x, const void* h,
                   const int32_t* len, void* z, void* y, void* saved) {
  BnArgs g = make_args(a, w, len, x, h);
  g.z = z; g.y = y; g.stats = (float*)saved;
  split(a, row_lanes(a.D) ? 256 : row_threads(a.D), kFwdItems, g.R, g.nc);
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
  split(a, bwd_threads(a.D), kBwdItems, g.R, g.nc);
  ProfScope prof(st);
  launch<true>(st, a, g);
  if (gr.gain_pre || gr.gain_post || gr.gate || gr.scale || gr.shift) {
    int gs = 64;
    while (gs > 1 && 64 / gs < a.B) gs /= 2;
    hipLaunchKernelGGL(len ? k_blocknorm_join<true> : k_blocknorm_join<false>, dim3((unsigned)cdiv(a.D, 16)), dim3(1024), 0, st,
                       BnJoin{w, gr, len, g.part, a.mod, a.B, a.D, g.nc, gs, a.res_scale});
    PG_LAUNCH_CHECK();
  }
  const double one = (a.res32 ? 4.0 : 2.0) * (1 + (dz ? 1 : 0) + a.pre) + (a.f32 ? 4.0 : 2.0) * (2 * a.branch + a.pre);
  prof.done_bytes("k_blocknorm_bwd", one * a.B * a.S * a.D);
}

}  // namespace pg
