// RMS norm of every query and key head with the position rotation in the
// same pass (forward), and its backward.
//
//   n = x r g,  r = (mean x^2 + eps)^-1/2;  pairs (a, b) of the first `rot`
//   elements -> (a c - b s, a s + b c) with (c, s) = table[pos].
// Backward: dn = the transposed rotation of dy; dg = sum over tokens and
// heads of dn x r;  dx = r (t - x r^2 mean(t x)),  t = dn g.
//
// Bound by memory: each element is read once and written once (backward:
// read twice, written once), everything between stays in registers in fp32.
// A lane holds 8 elements of a head (one 16-byte access in bf16), a group of
// LPH lanes one head; a group keeps its token's rotation row and the gains in
// registers over all the heads it takes.  Sums over a head are butterflies
// inside the group; in the half-split order the pair's other element sits
// rot / 16 lanes away and comes by a lane shuffle.
#include "token.hpp"

namespace pg {

namespace {

constexpr int kGainBlocks = 1024;   // blocks of a backward at most (one row of gain partials each)

struct QkArgs {
  int64_t T;
  int Hq, H, d, rot, n_pos, inter;
  int ns, hc;                       // head splits of a token, heads of one split
  float eps, inv_d;
  int64_t ldx[2], ldy[2];           // token strides of q, k (and dq, dk) and of the outputs (and their gradients)
  const void* x[2];
  const void* dy[2];
  void* y[2];                       // outputs (forward) or input gradients (backward)
  const float* gain[2];
  const float* table;
  const int32_t* pos;
  float* part;
};

template <typename T> PG_DEV void ld8f(const T* p, float* f);
template <> PG_DEV void ld8f<bf16_t>(const bf16_t* p, float* f) { unpack8(*reinterpret_cast<const uint4*>(p), f); }
template <> PG_DEV void ld8f<float>(const float* p, float* f) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <typename T> PG_DEV void st8f(T* p, const float* f);
template <> PG_DEV void st8f<bf16_t>(bf16_t* p, const float* f) { *reinterpret_cast<uint4*>(p) = pack8(f); }
template <> PG_DEV void st8f<float>(float* p, const float* f) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

template <int LPH>
PG_DEV float group_sum(float v) {
#pragma unroll
  for (int o = LPH / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// the rotation row of one token, as this lane's 8 elements need it
struct Turn {
  float c[8], s[8];   // per element; s carries the sign of the partner's term (forward)
  int partner;        // lane of the partner chunk (half-split order)
};

template <int LPH>
PG_DEV void load_turn(Turn& t, const QkArgs& a, bool real, int p, int lane, int ch) {
  const int np = a.rot / 16;
  const bool on = real && ch < 2 * np;
  t.partner = lane;
#pragma unroll
  for (int e = 0; e < 8; ++e) { t.c[e] = 1.f; t.s[e] = 0.f; }
  if (!on) return;
  if (a.inter) {      // pairs (2i, 2i + 1): four pairs in this lane
    const float4* row = reinterpret_cast<const float4*>(a.table + (int64_t)p * a.rot + ch * 8);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 v = row[i];
      t.c[4 * i] = t.c[4 * i + 1] = v.x;
      t.s[4 * i] = -v.y; t.s[4 * i + 1] = v.y;
      t.c[4 * i + 2] = t.c[4 * i + 3] = v.z;
      t.s[4 * i + 2] = -v.w; t.s[4 * i + 3] = v.w;
    }
  } else {            // pairs (i, i + rot / 2): eight pairs shared with the lane np away
    const bool lo = ch < np;
    t.partner = lo ? lane + np : lane - np;
    const float4* row = reinterpret_cast<const float4*>(a.table + (int64_t)p * a.rot + (lo ? ch : ch - np) * 16);
    const float sg = lo ? -1.f : 1.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 v = row[i];
      t.c[2 * i] = v.x; t.s[2 * i] = sg * v.y;
      t.c[2 * i + 1] = v.z; t.s[2 * i + 1] = sg * v.w;
    }
  }
}

// v <- the rotation of v (INV: its transpose).  Every lane of the wave takes part.
template <bool INV>
PG_DEV void turn(const Turn& t, int inter, int rot, float* v) {
  if (rot == 0) return;
  float o[8];
  if (inter) {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = v[e ^ 1];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = __shfl(v[e], t.partner, 64);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = fmaf(INV ? -t.s[e] : t.s[e], o[e], v[e] * t.c[e]);
}

template <typename T, int LPH, bool BWD>
__global__ __launch_bounds__(256) void k_qknorm(QkArgs a) {
  constexpr int GPB = 256 / LPH, U = BWD ? 2 : 4;
  const int tid = threadIdx.x, lane = tid & 63, ch = tid % LPH, grp = tid / LPH;
  const bool act = ch * 8 < a.d;
  float g[2][8], dg[2][8];
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      g[w][e] = act ? a.gain[w][ch * 8 + e] : 0.f;
      dg[w][e] = 0.f;
    }
  // items (token, head split): below 2^31 + 2^19
  const uint32_t items = (uint32_t)a.T * a.ns, step = gridDim.x * GPB;
  // every group of a wave goes round together (the shuffles need all lanes)
  for (uint32_t it0 = blockIdx.x * GPB; it0 < items; it0 += step) {
    const uint32_t it = it0 + grp;
    const bool in = it < items;
    const int64_t t = in ? it / (uint32_t)a.ns : 0;
    const int h0 = in ? (int)(it % (uint32_t)a.ns) * a.hc : 0;
    const int h1 = in ? min(a.H, h0 + a.hc) : 0;
    const int p = a.pos ? a.pos[t] : (int)((uint32_t)t % (uint32_t)a.n_pos);
    const bool real = p >= 0 && p < a.n_pos;          // a position outside the table: padding, zeros
    Turn tn;
    load_turn<LPH>(tn, a, real, p, lane, ch);
    for (int k = 0; k < a.hc; k += U) {
      float x[U][8], dy[U][8];
      bool ok[U];
      int w[U];
      int64_t yo[U], xo[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + k + u;
        w[u] = h >= a.Hq;
        const int hl = w[u] ? h - a.Hq : h;
        ok[u] = h < h1 && k + u < a.hc && act;
        xo[u] = t * a.ldx[w[u]] + (int64_t)hl * a.d + ch * 8;
        yo[u] = t * a.ldy[w[u]] + (int64_t)hl * a.d + ch * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) { x[u][e] = 0.f; dy[u][e] = 0.f; }
        if (ok[u] && real) {
          ld8f<T>((const T*)a.x[w[u]] + xo[u], x[u]);
          if (BWD) ld8f<T>((const T*)a.dy[w[u]] + yo[u], dy[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[u][e], x[u][e], ss);
        const float r = 1.f / sqrtf(fmaf(group_sum<LPH>(ss), a.inv_d, a.eps));
        if (!BWD) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[u][e] = x[u][e] * r * (w[u] ? g[1][e] : g[0][e]);
          turn<false>(tn, a.inter, a.rot, x[u]);
          if (ok[u]) st8f<T>((T*)a.y[w[u]] + yo[u], x[u]);
        } else {
          turn<true>(tn, a.inter, a.rot, dy[u]);
          float tx = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float c = dy[u][e] * (x[u][e] * r);
            if (w[u]) dg[1][e] += c; else dg[0][e] += c;
            dy[u][e] *= w[u] ? g[1][e] : g[0][e];
            tx = fmaf(dy[u][e], x[u][e], tx);
          }
          const float m = group_sum<LPH>(tx) * a.inv_d * r * r;
#pragma unroll
          for (int e = 0; e < 8; ++e) dy[u][e] = r * (dy[u][e] - x[u][e] * m);
          if (ok[u]) st8f<T>((T*)a.y[w[u]] + xo[u], dy[u]);
        }
      }
    }
  }
  if (BWD) {   // gain partials of the block: the groups' sums in group order
    __shared__ float sh[256 * 8];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) sh[tid * 8 + e] = dg[w][e];
      __syncthreads();
      if (tid < a.d) {
        float s = 0.f;
        for (int j = 0; j < GPB; ++j) s += sh[j * LPH * 8 + tid];
        a.part[((int64_t)blockIdx.x * 2 + w) * a.d + tid] = s;
      }
    }
  }
}

// dg[w][c] = sum over blocks of part[block][w][c]: 32 columns x 8 row lanes a block, rows in a fixed order
__global__ __launch_bounds__(256) void k_qknorm_gain(const float* part, int nb, int d, float* dgq, float* dgk) {
  __shared__ float sh[8][32];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), r = threadIdx.x >> 5;
  float s = 0.f;
  if (c < 2 * d)
    for (int b = r; b < nb; b += 8) s += part[(int64_t)b * 2 * d + c];
  sh[r][threadIdx.x & 31] = s;
  __syncthreads();
  if (r == 0 && c < 2 * d) {
    float v = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) v += sh[j][threadIdx.x];
    if (c < d) dgq[c] = v; else dgk[c - d] = v;
  }
}

int lanes_per_head(int d) {
  int l = 1;
  while (l * 8 < d) l *= 2;
  return l;
}

// Heads of a token are split over groups until the groups fill the card's
// 256 x 2048 threads: a few tokens then finish in one round of loads.
QkArgs make_args(const QkNorm& a) {
  QkArgs k{};
  k.T = a.T; k.Hq = a.Hq; k.H = a.Hq + a.Hk; k.d = a.d; k.rot = a.rot; k.n_pos = a.n_pos; k.inter = a.inter;
  k.eps = a.eps; k.inv_d = 1.f / (float)a.d;
  k.ldx[0] = a.ldq; k.ldx[1] = a.ldk; k.ldy[0] = a.ldqo; k.ldy[1] = a.ldko;
  const int64_t want = 524288 / lanes_per_head(a.d);
  const int64_t ns = std::min<int64_t>(k.H, std::max<int64_t>(1, cdiv(want, a.T)));
  k.hc = (int)cdiv(k.H, ns);
  k.ns = (int)cdiv(k.H, k.hc);
  return k;
}

int64_t grid_of(const QkArgs& k, int lph, int64_t most) { return std::min(cdiv(k.T * k.ns, 256 / lph), most); }

template <bool BWD>
void launch(hipStream_t st, const QkNorm& a, const QkArgs& k, int64_t grid) {
  const dim3 g((unsigned)grid), b(256);
#define PG_QK(L)                                                                       \
  case L:                                                                              \
    if (a.f32) hipLaunchKernelGGL((k_qknorm<float, L, BWD>), g, b, 0, st, k);          \
    else hipLaunchKernelGGL((k_qknorm<bf16_t, L, BWD>), g, b, 0, st, k);               \
    break;
  switch (lanes_per_head(a.d)) {
    PG_QK(1) PG_QK(2) PG_QK(4) PG_QK(8) PG_QK(16) PG_QK(32)
    default: throw Error{-2, "qknorm: head width above 256"};
  }
#undef PG_QK
  PG_LAUNCH_CHECK();
}

}  // namespace

size_t qknorm_ws_bytes(const QkNorm& a) { return (size_t)kGainBlocks * 2 * a.d * sizeof(float); }

void qknorm_fwd(hipStream_t st, const QkNorm& a, const void* q, const void* k, const float* gq, const float* gk,
                const float* table, const int32_t* pos, void* qo, void* ko) {
  QkArgs g = make_args(a);
  g.x[0] = q; g.x[1] = k; g.y[0] = qo; g.y[1] = ko;
  g.gain[0] = gq; g.gain[1] = gk; g.table = table; g.pos = pos;
  ProfScope prof(st);
  launch<false>(st, a, g, grid_of(g, lanes_per_head(a.d), 1 << 20));
  prof.done_bytes("k_qknorm_fwd", (double)a.T * (a.Hq + a.Hk) * a.d * (a.f32 ? 8.0 : 4.0));
}

void qknorm_bwd(hipStream_t st, const QkNorm& a, const void* q, const void* k, const float* gq, const float* gk,
                const float* table, const int32_t* pos, const void* dqo, const void* dko, void* dq, void* dk,
                float* dgq, float* dgk, void* ws) {
  QkArgs g = make_args(a);
  g.x[0] = q; g.x[1] = k; g.dy[0] = dqo; g.dy[1] = dko; g.y[0] = dq; g.y[1] = dk;
  g.gain[0] = gq; g.gain[1] = gk; g.table = table; g.pos = pos; g.part = (float*)ws;
  const int64_t grid = grid_of(g, lanes_per_head(a.d), kGainBlocks);
  ProfScope prof(st);
  launch<true>(st, a, g, grid);
  hipLaunchKernelGGL(k_qknorm_gain, dim3((unsigned)cdiv(2 * a.d, 32)), dim3(256), 0, st, (const float*)ws, (int)grid,
                     a.d, dgq, dgk);
  PG_LAUNCH_CHECK();
  prof.done_bytes("k_qknorm_bwd", (double)a.T * (a.Hq + a.Hk) * a.d * (a.f32 ? 12.0 : 6.0));
}

}  // namespace pg
