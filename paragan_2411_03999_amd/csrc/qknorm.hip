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
// registers over the heads it takes, four of which are in flight together.
// Loads are unconditional (a group without work reads a valid row again), so
// nothing waits for a position.  Sums over a head are butterflies inside the
// group (lane moves in the vector unit up to 16 lanes); in the half-split
// order the pair's other element sits rot / 16 lanes away and comes by a lane
// exchange.  Blocks of the grid's second dimension take q or k.
// Measured: forward of 32768 tokens x 16 heads x 64 in bf16 31 us (4.4 TB/s;
// 24 us from cache), in fp32 53 us (5.1 TB/s, partly from cache), backward of
// 15005 x 40 x 128 105 us (4.4 TB/s; a copy reaches 4.8).  Fewer registers for more waves, or two heads in flight, were
// slower (backward 104 to 396 us where this took 100).
#include "rows.hpp"
#include "token.hpp"

namespace pg {

namespace {

constexpr int kGainBlocks = 1024;   // blocks of a backward at most (one row of gain partials each)

struct QkArgs {
  uint32_t T;
  int d, rot, n_pos, inter;
  float eps, inv_d;
  const float* table;
  const int32_t* pos;
  float* part;
  struct Side {                     // q or k
    int H, ns, hc, grid;            // heads; splits of a token's heads, heads of one split; blocks
    int64_t ldx, ldy;               // token strides of the input (and its gradient) and of the output (and its gradient)
    const void *x, *dy;
    void* y;                        // output (forward) or input gradient (backward)
    const float* gain;
  } side[2];
};

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
__global__ __launch_bounds__(256, BWD ? 2 : 4) void k_qknorm(QkArgs a) {
  constexpr int GPB = 256 / LPH, U = 4;
  const auto& sd = a.side[blockIdx.y];
  if ((int)blockIdx.x >= sd.grid) return;
  const int tid = threadIdx.x, lane = tid & 63, ch = tid % LPH, grp = tid / LPH;
  const bool act = ch * 8 < a.d;
  const int c8 = act ? ch * 8 : 0;
  float g[8], dg[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    g[e] = act ? sd.gain[c8 + e] : 0.f;
    dg[e] = 0.f;
  }
  // items (token, head split): below 2^31 + 2^19
  const uint32_t items = a.T * (uint32_t)sd.ns, step = (uint32_t)sd.grid * GPB;
  // every group of a wave goes round together (the lane exchanges need all lanes)
  for (uint32_t it0 = blockIdx.x * GPB; it0 < items; it0 += step) {
    const uint32_t it = min(it0 + grp, items - 1);
    const bool in = it0 + grp < items;
    const uint32_t t = it / (uint32_t)sd.ns;
    const int h0 = (int)(it - t * sd.ns) * sd.hc, h1 = min(sd.H, h0 + sd.hc);
    const T* x0 = (const T*)sd.x + (int64_t)t * sd.ldx + c8;
    const T* dy0 = BWD ? (const T*)sd.dy + (int64_t)t * sd.ldy + c8 : nullptr;
    T* y0 = (T*)sd.y + (int64_t)t * (BWD ? sd.ldx : sd.ldy) + c8;
    const int p = a.pos ? a.pos[t] : (int)(t % (uint32_t)a.n_pos);
    Raw<T> xr[U], dr[U];
    auto fetch = [&](int h) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t o = (int64_t)min(h + u, h1 - 1) * a.d;
        xr[u].load(x0 + o);
        if (BWD) dr[u].load(dy0 + o);
      }
    };
    fetch(h0);
    const bool real = p >= 0 && p < a.n_pos;          // a position outside the table: padding, zeros
    Turn tn;
    load_turn<LPH>(tn, a, real, p, lane, ch);
    for (int h = h0; h < h0 + sd.hc; h += U) {   // as often for every group of the wave
      if (h > h0) fetch(min(h, h1 - 1));
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool ok = in && act && h + u < h1;
        const int64_t o = (int64_t)(h + u) * a.d;
        float x[8], dy[8];
        xr[u].get(x);
        if (BWD) dr[u].get(dy);
        const bool use = act && real && (!BWD || ok);   // nothing of padding, and of a row twice no gain gradient
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = use ? x[e] : 0.f;
          if (BWD) dy[e] = use ? dy[e] : 0.f;
          ss = fmaf(x[e], x[e], ss);
        }
        const float r = __builtin_amdgcn_rsqf(fmaf(group_sum<LPH>(ss), a.inv_d, a.eps));
        if (!BWD) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = x[e] * r * g[e];
          turn<false>(tn, a.inter, a.rot, x);
          if (ok) st8f<T>(y0 + o, x);
        } else {
          turn<true>(tn, a.inter, a.rot, dy);
          float tx = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            dg[e] = fmaf(dy[e], x[e] * r, dg[e]);
            dy[e] *= g[e];
            tx = fmaf(dy[e], x[e], tx);
          }
          const float m = group_sum<LPH>(tx) * a.inv_d * r * r;
#pragma unroll
          for (int e = 0; e < 8; ++e) dy[e] = r * (dy[e] - x[e] * m);
          if (ok) st8f<T>(y0 + o, dy);
        }
      }
    }
  }
  if (BWD) {   // gain partials of the block: the groups' sums in group order, in 64 bits
    __shared__ float sh[256 * 8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sh[tid * 8 + e] = dg[e];
    __syncthreads();
    if (tid < a.d) {
      double s = 0.0;
      for (int j = 0; j < GPB; ++j) s += sh[j * LPH * 8 + tid];
      a.part[((int64_t)(blockIdx.y ? a.side[0].grid : 0) + blockIdx.x) * a.d + tid] = (float)s;
    }
  }
}

// dg[c] = sum over the blocks of q (blockIdx.y = 0) or k of part[block][c]:
// 16 columns x 64 row lanes a block, the rows of a lane and the lanes in
// order, in 64 bits (the sums of a gradient over all tokens and heads mostly
// cancel, and the joins would lose more of them than the sums in the registers do)
__global__ __launch_bounds__(1024) void k_qknorm_gain(const float* part, int nq, int nk, int d, float* dgq, float* dgk) {
  __shared__ double sh[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), r = threadIdx.x >> 4, nb = blockIdx.y ? nk : nq;
  const float* p = part + (blockIdx.y ? (int64_t)nq * d : 0);
  double s = 0.0;
  if (c < d) {
#pragma unroll 8
    for (int b = r; b < nb; b += 64) s += p[(int64_t)b * d + c];
  }
  sh[r][threadIdx.x & 15] = s;
  __syncthreads();
  if (threadIdx.x >= 16 || c >= d) return;
  double v = 0.0;
#pragma unroll
  for (int j = 0; j < 64; ++j) v += sh[j][threadIdx.x];
  (blockIdx.y ? dgk : dgq)[c] = (float)v;
}

int lanes_per_head(int d) {
  int l = 1;
  while (l * 8 < d) l *= 2;
  return l;
}

// Heads of a token are split over groups until the groups fill the card's
// 256 x 2048 threads: a few tokens then finish in one round of loads.  The
// blocks are at most `most`, shared by the sides as their heads are.
QkArgs make_args(const QkNorm& a, int64_t most) {
  QkArgs k{};
  k.T = (uint32_t)a.T; k.d = a.d; k.rot = a.rot; k.n_pos = a.n_pos; k.inter = a.inter;
  k.eps = a.eps; k.inv_d = 1.f / (float)a.d;
  const int H[2] = {a.Hq, a.Hk};
  const int64_t ldx[2] = {a.ldq, a.ldk}, ldy[2] = {a.ldqo, a.ldko};
  const int64_t lph = lanes_per_head(a.d), want = 524288 / lph;
  for (int w = 0; w < 2; ++w) {
    auto& s = k.side[w];
    s.H = H[w]; s.ldx = ldx[w]; s.ldy = ldy[w];
    const int64_t ns = std::min<int64_t>(s.H, std::max<int64_t>(1, cdiv(want * s.H, a.T * (a.Hq + a.Hk))));
    s.hc = (int)cdiv(s.H, ns);
    s.ns = (int)cdiv(s.H, s.hc);
    s.grid = (int)std::min(cdiv(a.T * s.ns, 256 / lph), std::max<int64_t>(1, most * s.H / (a.Hq + a.Hk)));
  }
  return k;
}

template <bool BWD>
void launch(hipStream_t st, const QkNorm& a, const QkArgs& k) {
  const dim3 g((unsigned)std::max(k.side[0].grid, k.side[1].grid), 2), b(256);
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

size_t qknorm_ws_bytes(const QkNorm& a) { return (size_t)(kGainBlocks + 1) * a.d * sizeof(float); }

void qknorm_fwd(hipStream_t st, const QkNorm& a, const void* q, const void* k, const float* gq, const float* gk,
                const float* table, const int32_t* pos, void* qo, void* ko) {
  QkArgs g = make_args(a, 1 << 20);
  g.table = table; g.pos = pos;
  g.side[0].x = q; g.side[0].y = qo; g.side[0].gain = gq;
  g.side[1].x = k; g.side[1].y = ko; g.side[1].gain = gk;
  ProfScope prof(st);
  launch<false>(st, a, g);
  prof.done_bytes("k_qknorm_fwd", (double)a.T * (a.Hq + a.Hk) * a.d * (a.f32 ? 8.0 : 4.0));
}

void qknorm_bwd(hipStream_t st, const QkNorm& a, const void* q, const void* k, const float* gq, const float* gk,
                const float* table, const int32_t* pos, const void* dqo, const void* dko, void* dq, void* dk,
                float* dgq, float* dgk, void* ws) {
  QkArgs g = make_args(a, kGainBlocks);
  g.table = table; g.pos = pos; g.part = (float*)ws;
  g.side[0].x = q; g.side[0].dy = dqo; g.side[0].y = dq; g.side[0].gain = gq;
  g.side[1].x = k; g.side[1].dy = dko; g.side[1].y = dk; g.side[1].gain = gk;
  ProfScope prof(st);
  launch<true>(st, a, g);
  hipLaunchKernelGGL(k_qknorm_gain, dim3((unsigned)cdiv(a.d, 16), 2), dim3(1024), 0, st, (const float*)ws,
                     g.side[0].grid, g.side[1].grid, a.d, dgq, dgk);
  PG_LAUNCH_CHECK();
  prof.done_bytes("k_qknorm_bwd", (double)a.T * (a.Hq + a.Hk) * a.d * (a.f32 ? 12.0 : 6.0));
}

}  // namespace pg
