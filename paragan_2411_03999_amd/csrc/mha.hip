// Multi-head attention on gfx950 (bf16 MFMA 32x32x16, fp32 softmax) with
// shared key heads, ragged lengths, causal order, a sliding window with a few
// first tokens that stay visible, and a learned relative position bias by
// buckets; forward, backward and the form for a few new tokens over a cache.
//
//   S = scale q k^T + bias[h][bucket(j - p)],  P = softmax over visible keys,
//   o = P v;   backward: D = rowsum(do o), dS = P (do v^T - D),
//   dq = scale dS k, dk = scale dS^T q, dv = P^T do,
//   dbias[h][b] = sum of dS over the pairs in bucket b.
//
// S is never stored.  Scores are computed transposed (S^T = K Q^T), so a lane
// owns one query (forward, dq) or one key (dk, dv); probabilities feed the
// next product straight from the accumulator registers.  Softmax statistics,
// all sums and the bias are fp32; the operands of the second products (P, dS)
// are rounded to bf16 because the matrix cores take them so.  Exponentials
// are base 2 and the running maximum is only raised when a tile's maximum
// passes it by 2^8 (the rescale of the accumulators is then rare).
//
// A tile is only visited when some query of the block sees some key of it;
// rows nobody in the block sees are not read (they may hold anything).
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "attn_tiles.hpp"
#include "lds_dma.hpp"
#include "token.hpp"

namespace pg {

namespace {

constexpr int kStepTable = 64;  // buckets up to which a step keeps its rows' bias in LDS (8 KB)
// A bias this large (in log2 units) leaves nothing of a score's fraction in their fp32 sum.  The sum is formed all the same
// then, away from the diagonal too, where a smaller bias goes into the exponent beside the running maximum: taken apart,
// a row of such biases alone would weigh its keys by scores that the sums near the diagonal have lost, up to infinity.
constexpr float kDeep = 0x1p24f;
// From a bias this large on (log2 units; of a head's any finite one) the backward keeps a row's maximum and the logarithm of
// its sum apart: as one number, as exact as 2^-14 up to here, it would lose the sum beside a bias that scores vanish in too.
// (Training 4 x 4096 x 8 heads x 64: 790 us against 780 as one number; 914 where every head has such a bias.)
constexpr float kSteep = 0x1p10f;
constexpr int kMargin = 96;   // distances past max_distance that a 64 x 32 tile can reach, rounded up

struct MhaArgs {
  int B, Sq, Sk, Hq, Hk, G, d, Sqp, nblk;
  int causal, window, n_sink, nb, maxd, half;
  int nsplit, nrt, hset;
  int nks, ns_sink, ns_reg, chunk;   // dk, dv: key blocks with first tokens, splits of these and of the others, steps of a split
  float c, scale;               // c = scale log2(e)
  int64_t qs[3], ks[3], vs[3], os[3];
  const bf16_t *q, *k, *v, *dO;
  bf16_t *o, *dq, *dk, *dv;
  const float* table;
  const int32_t *len_q, *len_k;
  float *top, *lg;              // of a row, in log2 units: its maximum and the log of its sum (no bias: top is both); infinity if it sees nothing
  float *D, *L, *part;          // D: minus do . o of a row; L: what its products start from in the key-owned pass
  uint2* olo;                   // what rounding took off the output, bf16, in register layout: [32-query tile][DT / 8][64 lanes][4]
  uint16_t start[257];          // smallest distance of each bucket of one side
  uint8_t lut[kMhaMaxDist + 8]; // bucket (of one side) of each distance
};

// Block order.  Consecutive block numbers go round the 8 XCDs, each with an L2
// of its own; heads that share keys and values are brought onto one XCD, in
// sets of a.hset heads given to the XCDs in turn (0: left as they come).
// Causal 2 x 8192 x 16 heads x 128: 784 us in plain order, 575 so.
PG_DEV int block_no(const MhaArgs& a, int per_head) {
  const int x = blockIdx.x;
  if (a.hset == 0) return x;
  const int y = x >> 3, per = per_head * a.hset, set = y / per;
  return (set * 8 + (x & 7)) * per + y - set * per;
}

struct Seq { int lq, lk, off; };
PG_DEV Seq seq_of(const MhaArgs& a, int b) {
  Seq s;
  s.lq = a.len_q ? min(max(a.len_q[b], 0), a.Sq) : a.Sq;
  s.lk = a.len_k ? min(max(a.len_k[b], 0), a.Sk) : a.Sk;
  s.lq = __builtin_amdgcn_readfirstlane(s.lq);
  s.lk = __builtin_amdgcn_readfirstlane(s.lk);
  s.off = s.lk - s.lq;
  return s;
}

// Keys that queries at positions p0 .. p1 see: [lo, hi) through the window
// and [0, ns) of the first tokens, as nt tiles of TK: tile n is
// n (n < st) or n - st + ws.
template <int TK>
struct Span {
  int lo, hi, ns, st, ws, nt;
  PG_DEV int key0(int n) const { return TK * (n < st ? n : n - st + ws); }
  PG_DEV bool row(int j) const { return (j >= lo && j < hi) || j < ns; }
  PG_DEV bool tile(int k0) const { return (k0 + TK > lo && k0 < hi) || k0 < ns; }
  PG_DEV bool whole(int k0) const { return (k0 >= lo && k0 + TK <= hi) || k0 + TK <= ns; }
};
template <int TK>
PG_DEV Span<TK> span_of(const MhaArgs& a, int lk, int p0, int p1) {
  Span<TK> s;
  const int top = max(a.causal ? min(lk, p1 + 1) : lk, 0);
  s.lo = a.window ? max(p0 - a.window + 1, 0) : 0;
  s.hi = a.window && !a.causal ? max(min(lk, p1 + a.window), 0) : top;
  s.ns = a.window ? min(a.n_sink, top) : 0;
  const int sink_tiles = (s.ns + TK - 1) / TK, w0 = s.lo / TK, w1 = (s.hi + TK - 1) / TK;
  if (sink_tiles >= w0) {
    s.st = 0;
    s.ws = 0;
    s.nt = max(w1, sink_tiles);
    if (s.lo >= s.hi) s.nt = sink_tiles;
  } else {
    s.st = sink_tiles;
    s.ws = w0;
    s.nt = sink_tiles + max(w1 - w0, 0);
  }
  return s;
}
// Does every query at positions p0 .. p1 see every key of [k0, k0 + TK)?
template <int TK>
PG_DEV bool all_seen(const MhaArgs& a, int lk, int k0, int p0, int p1) {
  if (k0 + TK > lk || (a.causal && k0 + TK - 1 > p0)) return false;
  return !a.window || k0 + TK <= a.n_sink || (p1 - k0 < a.window && k0 + TK - 1 - p0 < a.window);
}
// visible keys of one query: [lo, hi) and [0, ns)
struct Row { int lo, hi, ns; };
PG_DEV Row row_of(const MhaArgs& a, int lk, int p) {
  Row r;
  const int top = a.causal ? min(lk, p + 1) : lk;
  r.lo = a.window ? p - a.window + 1 : 0;
  r.hi = a.window ? min(top, p + a.window) : top;
  r.ns = a.window ? min(a.n_sink, top) : 0;
  return r;
}
PG_DEV bool sees(const Row& r, int j) { return (j >= r.lo && j < r.hi) || j < r.ns; }
// -infinity for the keys k0 + row of a score tile that the row's query does
// not see; one unsigned comparison each away from the first tokens
PG_DEV void hide(f32x16& s, const Row& rw, int k0, int g) {
  if (k0 < rw.ns) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (!sees(rw, k0 + acc_row(r, g))) s[r] = -INFINITY;
  } else {
    const uint32_t at = (uint32_t)(k0 + 4 * g - rw.lo), width = (uint32_t)max(rw.hi - rw.lo, 0);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (at + 8 * (r >> 2) + (r & 3) >= width) s[r] = -INFINITY;
  }
}

// max of three without the quieting moves that fmaxf asks for (a NaN score gives NaN through its exponential)
PG_DEV float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// a bias in log2 units; the lowest and the largest finite values stay finite (a row of nothing else is uniform)
PG_DEV float log2_bias(float t) {
  const float x = t * kL2E;
  return fabsf(t) <= FLT_MAX && fabsf(x) > FLT_MAX ? copysignf(FLT_MAX, t) : x;
}

// bias in log2 units at distance index e = rel + maxd + kMargin; distances past max_distance are its own
PG_DEV float bias2_at(const MhaArgs& a, int h, int e) {
  const int rel = min(max(e - a.maxd - kMargin, -a.maxd), a.causal ? 0 : a.maxd);
  const int b = (int)a.lut[rel < 0 ? -rel : rel] + (rel > 0 ? a.half : 0);
  return log2_bias(a.table[(int64_t)h * a.nb + b]);
}
PG_DEV float uniform(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }
// Is one of head h's biases that large?  (Every wave looks for itself.)
PG_DEV bool steep_bias(const MhaArgs& a, int h, int lane) {
  bool big = false;
  for (int k = lane; k < a.nb; k += 64) {
    const float b = fabsf(log2_bias(a.table[(int64_t)h * a.nb + k]));
    big |= b >= kSteep && b <= FLT_MAX;
  }
  return __any(big);
}
PG_DEV int bias_len(const MhaArgs& a) { return 2 * (a.maxd + kMargin) + 1; }
// where key k0's bias for the query at p0 stands in that array, if the tile is near the diagonal; else the 31st of an
// end's kMargin + 1 equal elements, of which a tile of 64 keys takes those from 31 before to 63 behind
PG_DEV int bias_row(const MhaArgs& a, bool near, int k0, int p0) {
  return near ? k0 - p0 + a.maxd + kMargin : 31 + (k0 < p0 ? 0 : 2 * a.maxd + kMargin);
}

// ROWS rows x NC chunks from memory straight into a swizzled LDS tile by 4
// waves: 16-byte slot i of the tile (lane order) holds chunk (i % NC) ^ swizzle
// of row i / NC.  Chunks at or past d and rows that `ok` refuses read as zeros
// without touching memory.
template <int NC, int ROWS>
struct Ring {
  static constexpr int L = NC * ROWS / 64, N = (L + 3) / 4;   // loads of 64 lanes, of a wave at most
  uint32_t off[N];
  int row[N];
  PG_DEV void init(int64_t ld, int d, int tid) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = (4 * j + (tid >> 6)) * 64 + (tid & 63);
      const int r = i / NC, c = (i - r * NC) ^ swz16<NC>(r);
      row[j] = r;
      off[j] = c * 8 < d ? (uint32_t)(r * (int)ld * 2 + c * 16) : kOOB;
    }
  }
  // base: row 0 of the tile (uniform); rows r0 + r, `all` of which are wanted or those that `ok` says
  template <class F>
  PG_DEV void issue(bf16_t* tile, const bf16_t* base, int64_t ld, int r0, int wave, bool all, F ok) const {
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(base, ((ROWS - 1) * ld + NC * 8) * 2);
    const uint32_t dst = lds_addr(tile) + wave * 1024;
    if (all) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (4 * j + 3 < L || 4 * j + wave < L) lds_load16(dst + j * 4096, off[j], 0, rs);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (4 * j + 3 < L || 4 * j + wave < L) lds_load16(dst + j * 4096, ok(r0 + row[j]) ? off[j] : kOOB, 0, rs);
    }
  }
};

PG_DEV bf16x8 ld_frag(const bf16_t* row, int e, int d, bool ok) { return ok && e < d ? ld8g(row + e) : zero8(); }

// four consecutive channels of a bf16 row; nothing past d
PG_DEV void st4(bf16_t* row, int e, int d, float a, float b, float c, float f) {
  if (e < d) *reinterpret_cast<uint2*>(row + e) = make_uint2(f2bf2(a, b), f2bf2(c, f));
}

// ------------------------------------------------------------- forward
// A wave owns 32 queries of one head, a block of 4 waves 128.  Keys and
// values come in tiles of 64, the next one loading while this one is used.
// Bound by the issue of exponentials and their neighbours beside the matrix
// products: at 128 channels the matrix cores are busy 44 % of the time and
// vector instructions are issued in 39 %, and they overlap little.  Causal
// 2 x 8192 x 16/4 heads x 128: 581 us, 946 TFLOP/s, on new inputs every time,
// 553 on the same (a large library product reaches 1225 TFLOP/s here).
// Tried and slower, where it took 575 then: two query tiles a wave at 128
// channels (2421 us, one wave a SIMD), the next tile's scores formed beside this
// one's exponentials (602), raised wave priority over the products (571 and,
// through a window, 73 for 66).
// At 64 channels four waves a SIMD hide more than the third of the registers
// is worth, though the bias then spills 16 bytes a lane: with it 64 x 256 x 8
// heads 23.5 us against 24.9 with three; without it, 4 x 4099 x 16 heads
// through a window of 512, 56.7 against 57.5 (ragged) and 61.2 against 61.9.
template <int DT, bool BIAS>
__global__ __launch_bounds__(256, DT == 64 ? 4 : 2) void k_mha_fwd(MhaArgs a) {
  constexpr int TK = 64, NC = DT / 8, NT = DT / 32, KF = DT / 16;
  __shared__ __attribute__((aligned(16))) bf16_t Ks[2][TK * DT];
  __shared__ __attribute__((aligned(16))) bf16_t Vs[2][TK * DT];
  extern __shared__ float bs[];
  // the last queries of a causal head see the most keys: they start first
  const int id = block_no(a, a.nblk), qb = a.nblk - 1 - id % a.nblk, bh = id / a.nblk, h = bh % a.Hq, b = bh / a.Hq;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, lq = lane & 31;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Seq sq = seq_of(a, b);
  const int qblk = qb * 128, qw = qblk + wv * 32, q = qw + lq, p0 = qw + sq.off;
  const bf16_t* K = a.k + b * a.ks[0] + (h / a.G) * a.ks[2];
  const bf16_t* V = a.v + b * a.vs[0] + (h / a.G) * a.vs[2];
  if (BIAS)
    for (int e = tid; e < bias_len(a); e += 256) bs[e] = bias2_at(a, h, e);
  const bf16_t* Q = a.q + b * a.qs[0] + q * a.qs[1] + h * a.qs[2];
  bf16x8 qf[KF];
#pragma unroll
  for (int t = 0; t < KF; ++t) qf[t] = ld_frag(Q, 16 * t + 8 * g, a.d, q < sq.lq);
  const Row rw = row_of(a, sq.lk, q + sq.off);
  f32x16 acc[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
  float m2 = -INFINITY, l = 0.f;
  // a block behind the last query visits nothing and writes zeros
  Span<TK> sp = span_of<TK>(a, sq.lk, qblk + sq.off, min(qblk + 128, sq.lq) - 1 + sq.off);
  if (qblk >= sq.lq) sp.nt = 0;
  const Span<TK> sw = span_of<TK>(a, sq.lk, p0, min(qw + 32, sq.lq) - 1 + sq.off);
  const bool mine = qw < sq.lq;
  Ring<NC, TK> rk, rv;
  rk.init(a.ks[1], a.d, tid);
  rv.init(a.vs[1], a.d, tid);
  auto load = [&](int n, int bf) {
    const int k0 = sp.key0(n);
    auto ok = [&](int j) { return sp.row(j); };
    const bool all = sp.whole(k0);
    rk.issue(Ks[bf], K + k0 * a.ks[1], a.ks[1], k0, wv, all, ok);
    rv.issue(Vs[bf], V + k0 * a.vs[1], a.vs[1], k0, wv, all, ok);
  };
  // the buffer is known at compile time, so that LDS addresses need no arithmetic
  auto visit = [&](auto buf_c, int n) {
    constexpr int buf = decltype(buf_c)::value;
    wait_barrier<0>();   // tile n is in LDS, and every wave has left tile n - 1
    const int k0 = sp.key0(n);
    if (n + 1 < sp.nt) load(n + 1, buf ^ 1);
    if (!mine || !sw.tile(k0)) return;
    const bf16_t* ks = Ks[buf];
    const bf16_t* vs = Vs[buf];
    f32x16 s[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] = s[1][r] = 0.f;
#pragma unroll
    for (int t = 0; t < KF; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_row<NC>(ks + 32 * DT * x, lq, 16 * t + 8 * g), qf[t], s[x], 0, 0, 0);
    // a score in log2 units is s cm + off: near the diagonal the bias is added to each, elsewhere it is one number
    float cm = a.c, off = 0.f;
    if (BIAS) {
      const bool near = k0 + TK - 1 - p0 > -a.maxd && k0 - p0 - 31 < a.maxd;
      const float far = k0 < p0 ? bs[0] : bs[bias_len(a) - 1];
      if (near || fabsf(far) >= kDeep) {
        const float* bl = bs + bias_row(a, near, k0, p0) - lq + 4 * g;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[x][r] = fmaf(s[x][r], a.c, bl[32 * x + 8 * (r >> 2) + (r & 3)]);
        cm = 1.f;
      } else {
        off = far;
      }
    }
    if (!all_seen<TK>(a, sq.lk, k0, p0, p0 + 31)) {
      hide(s[0], rw, k0, g);
      hide(s[1], rw, k0 + 32, g);
    }
    float mb = s[0][0], mc = s[1][0];   // two chains
#pragma unroll
    for (int r = 1; r < 15; r += 2) {
      mb = max3(mb, s[0][r], s[0][r + 1]);
      mc = max3(mc, s[1][r], s[1][r + 1]);
    }
    mb = max3(max3(mb, s[0][15], s[1][15]), mc, mc);
    mb = max3(mb, mb, __shfl_xor(mb, 32, 64));
    mb = BIAS ? fmaf(mb, cm, off) : mb * a.c;
    if (mb > m2 + kTau) {
      const float alpha = exp2_(m2 - mb);
      l *= alpha;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][r] *= alpha;
      m2 = mb;
    }
    const float ms = off - (m2 == -INFINITY ? 0.f : m2);   // nothing seen yet: every term is 2^-inf
    float ls[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        s[x][r] = exp2_(fmaf(s[x][r], BIAS ? cm : a.c, ms));
        ls[x] += s[x][r];
      }
    l += ls[0] + ls[1];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bf16x8 pb = pack_regs(s[t >> 1], t & 1);
#pragma unroll
      for (int j = 0; j < NT; ++j)
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_tr<NC>(vs + 32 * DT * (t >> 1), t & 1, 32 * j, lane), pb, acc[j], 0, 0, 0);
    }
  };
  if (sp.nt > 0) load(0, 0);
  for (int n = 0; n < sp.nt; n += 2) {
    visit(std::integral_constant<int, 0>(), n);
    if (n + 1 < sp.nt) visit(std::integral_constant<int, 1>(), n + 1);
  }
  const float lt = l + __shfl_xor(l, 32, 64);
  const bool any = q < sq.lq && lt != 0.f;   // a NaN goes on: only a row that sees nothing is zeros
  const float inv = any ? 1.f / lt : 0.f;
  bf16_t* orow = a.o + b * a.os[0] + q * a.os[1] + h * a.os[2];
  uint2* const lo = a.olo && qw < a.Sqp ? a.olo + ((int64_t)bh * (a.Sqp / 32) + qw / 32) * (DT / 8) * 64 + lane : nullptr;
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = any ? acc[j][4 * i + e] * inv : 0.f;
      if (q < a.Sq) st4(orow, 32 * j + 8 * i + 4 * g, a.d, f[0], f[1], f[2], f[3]);
      if (lo) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] -= rnd<bf16_t>(f[e]);
        lo[(4 * j + i) * 64] = make_uint2(f2bf2(f[0], f[1]), f2bf2(f[2], f[3]));
      }
    }
  if (a.top && g == 0 && q < a.Sqp) {
    const float lg = any ? __log2f(lt) : 0.f;
    a.top[(int64_t)bh * a.Sqp + q] = any ? (BIAS ? m2 : m2 + lg) : INFINITY;
    if (BIAS) a.lg[(int64_t)bh * a.Sqp + q] = lg;
  }
}

// ------------------------------------------------------------- a few new tokens
// The rows (query, query head of the group) of one key head form tiles of 32,
// of neighbouring queries, so that a tile visits no more keys than these see;
// a block's 4 waves take tiles of 32 keys in turn, each with its own running
// softmax, joined at the end; nsplit blocks share a long cache and leave
// partials.  Bound by reading keys and values once: a wave has its next tile
// on the way into a ring of its own in LDS while it works on one, with no
// barrier in the loop.

// 32 rows x NC chunks into a swizzled LDS tile by one wave, as Ring
template <int NC>
struct WaveRing {
  static constexpr int L = NC / 2;   // loads
  uint32_t off[L];
  PG_DEV void init(int64_t ld, int d, int lane) {
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int i = j * 64 + lane, r = i / NC, c = (i - r * NC) ^ swz16<NC>(r);
      off[j] = c * 8 < d ? (uint32_t)(r * (int)ld * 2 + c * 16) : kOOB;
    }
  }
  template <class F>
  PG_DEV void issue(bf16_t* tile, const bf16_t* base, int64_t ld, int r0, int lane, F ok) const {
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(base, (31 * ld + NC * 8) * 2);
    const uint32_t dst = lds_addr(tile);
#pragma unroll
    for (int j = 0; j < L; ++j) lds_load16(dst + j * 1024, ok(r0 + (j * 64 + lane) / NC) ? off[j] : kOOB, 0, rs);
  }
};
// at most N of this wave's loads still on their way
template <int N>
PG_DEV void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <int DT, bool BIAS>
__global__ __launch_bounds__(256, DT <= 64 ? 2 : 1) void k_mha_step(MhaArgs a) {
  constexpr int NC = DT / 8, NT = DT / 32, KF = DT / 16;
  // [wave][buffer][keys, values]; afterwards the waves' outputs
  constexpr int kRing = 4 * 2 * 2 * 32 * DT * 2, kRed = 3 * NT * 16 * 64 * 4;
  __shared__ __attribute__((aligned(16))) char lds[kRing > kRed ? kRing : kRed];
  __shared__ float ml[4][32][2];
  extern __shared__ float dyn[];   // BIAS: the distances' buckets, then (nb <= kStepTable) the rows' bias by bucket
  const int z = blockIdx.x % a.nsplit, rt = (blockIdx.x / a.nsplit) % a.nrt, bh = blockIdx.x / a.nsplit / a.nrt;
  const int hk = bh % a.Hk, b = bh / a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, lq = lane & 31;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Seq sq = seq_of(a, b);
  const int rho = rt * 32 + lq, R = a.G * a.Sq;
  const int i = rho / a.G, h = hk * a.G + rho - i * a.G;
  const bool live = rho < R && i < sq.lq;
  // positions of the tile's queries
  const int i0 = rt * 32 / a.G, p0 = sq.off + i0, p1 = sq.off + min((rt * 32 + 31) / a.G, sq.lq - 1);
  Span<32> sp = span_of<32>(a, sq.lk, p0, p1);
  if (i0 >= sq.lq) sp.nt = 0;
  const int per = (sp.nt + a.nsplit - 1) / a.nsplit, n1 = min(sp.nt, (z + 1) * per);
  const bf16_t* K = a.k + b * a.ks[0] + hk * a.ks[2];
  const bf16_t* V = a.v + b * a.vs[0] + hk * a.vs[2];
  bf16_t* const ring = reinterpret_cast<bf16_t*>(lds) + wv * 4 * 32 * DT;
  WaveRing<NC> rk, rv;
  rk.init(a.ks[1], a.d, lane);
  rv.init(a.vs[1], a.d, lane);
  auto load = [&](int n, int bf) {
    const int k0 = sp.key0(n);
    auto ok = [&](int j) { return sp.row(j); };
    rk.issue(ring + bf * 64 * DT, K + k0 * a.ks[1], a.ks[1], k0, lane, ok);
    rv.issue(ring + bf * 64 * DT + 32 * DT, V + k0 * a.vs[1], a.vs[1], k0, lane, ok);
  };
  int n = z * per + wv, buf = 0;
  if (n < n1) load(n, 0);
  const bf16_t* Q = a.q + b * a.qs[0] + i * a.qs[1] + h * a.qs[2];
  bf16x8 qf[KF];
#pragma unroll
  for (int t = 0; t < KF; ++t) qf[t] = ld_frag(Q, 16 * t + 8 * g, a.d, live);
  const uint8_t* const lut = reinterpret_cast<const uint8_t*>(dyn);
  const float* tab = nullptr;      // this row's bias by bucket
  float cs = a.c, flo = 0.f, fhi = 0.f;
  if (BIAS) {
    uint8_t* lw = reinterpret_cast<uint8_t*>(dyn);
    for (int e = tid; e < bias_len(a); e += 256) {
      const int rel = min(max(e - a.maxd - kMargin, -a.maxd), a.causal ? 0 : a.maxd);
      lw[e] = (uint8_t)(a.lut[rel < 0 ? -rel : rel] + (rel > 0 ? a.half : 0));
    }
    tab = a.table + (int64_t)h * a.nb;
    if (a.nb <= kStepTable) {
      float* tw = dyn + (bias_len(a) + 3) / 4;
      for (int e = tid; e < 32 * a.nb; e += 256)
        tw[e] = a.table[(int64_t)(hk * a.G + (rt * 32 + e / a.nb) % a.G) * a.nb + e % a.nb];
      tab = tw + lq * a.nb;
    }
    __syncthreads();
    flo = log2_bias(tab[lut[0]]);
    fhi = log2_bias(tab[lut[bias_len(a) - 1]]);
  }
  const Row rw = row_of(a, sq.lk, i + sq.off);
  f32x16 acc[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
  float m2 = -INFINITY, l = 0.f;
  for (; n < n1; n += 4, buf ^= 1) {
    const int k0 = sp.key0(n);
    const bf16_t* ks = ring + buf * 64 * DT;
    const bf16_t* vs = ks + 32 * DT;
    if (n + 4 < n1) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the other buffer has been read
      load(n + 4, buf ^ 1);
      wait_loads<2 * WaveRing<NC>::L>();
    } else {
      wait_loads<0>();
    }
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int t = 0; t < KF; ++t) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_row<NC>(ks, lq, 16 * t + 8 * g), qf[t], s, 0, 0, 0);
    float cm = cs, off = 0.f;
    if (BIAS) {
      const float far = k0 < p0 ? flo : fhi;
      if ((k0 + 31 - p0 > -a.maxd && k0 - p1 < a.maxd) || fabsf(far) >= kDeep) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int rel = min(max(k0 + acc_row(r, g) - i - sq.off, -a.maxd), a.maxd);
          s[r] = fmaf(s[r], cs, log2_bias(tab[lut[rel + a.maxd + kMargin]]));
        }
        cm = 1.f;
      } else {
        off = far;
      }
    }
    if (!all_seen<32>(a, sq.lk, k0, p0, p1)) hide(s, rw, k0, g);
    float mb = s[0];
#pragma unroll
    for (int r = 1; r < 15; r += 2) mb = max3(mb, s[r], s[r + 1]);
    mb = max3(mb, mb, s[15]);
    mb = max3(mb, mb, __shfl_xor(mb, 32, 64));
    mb = BIAS ? fmaf(mb, cm, off) : mb * cs;
    if (mb > m2 + kTau) {
      const float alpha = exp2_(m2 - mb);
      l *= alpha;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][r] *= alpha;
      m2 = mb;
    }
    const float ms = off - (m2 == -INFINITY ? 0.f : m2);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = exp2_(fmaf(s[r], BIAS ? cm : cs, ms));
      l += s[r];
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 pb = pack_regs(s, t);
#pragma unroll
      for (int j = 0; j < NT; ++j)
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_tr<NC>(vs, t, 32 * j, lane), pb, acc[j], 0, 0, 0);
    }
  }
  float(*const red)[NT * 16 * 64] = reinterpret_cast<float(*)[NT * 16 * 64]>(lds);
  // join the four waves
  l += __shfl_xor(l, 32, 64);
  if (g == 0) { ml[wv][lq][0] = m2; ml[wv][lq][1] = l; }
  __syncthreads();
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, ml[w][lq][0]);
  const float Ms = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int w = 0; w < 4; ++w) L += ml[w][lq][1] * exp2_(ml[w][lq][0] - Ms);
  const float f = exp2_(m2 - Ms);
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] *= f;
  if (wv > 0)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) red[wv - 1][(j * 16 + r) * 64 + lane] = acc[j][r];
  __syncthreads();
  if (wv > 0) return;
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      acc[j][r] += red[0][(j * 16 + r) * 64 + lane] + red[1][(j * 16 + r) * 64 + lane] + red[2][(j * 16 + r) * 64 + lane];
  if (a.nsplit > 1) {
    float* slot = a.part + (int64_t)blockIdx.x * 32 * (DT + 2);
    if (g == 0) { slot[lq] = M; slot[32 + lq] = L; }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<float4*>(slot + 64 + lq * DT + 32 * j + 8 * e + 4 * g) =
            make_float4(acc[j][4 * e], acc[j][4 * e + 1], acc[j][4 * e + 2], acc[j][4 * e + 3]);
    return;
  }
  if (rho >= R) return;
  const bool any = live && L != 0.f;   // as in the forward
  const float inv = any ? 1.f / L : 0.f;
  bf16_t* orow = a.o + b * a.os[0] + i * a.os[1] + h * a.os[2];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x16& x = acc[j];
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (any) v = make_float4(x[4 * e] * inv, x[4 * e + 1] * inv, x[4 * e + 2] * inv, x[4 * e + 3] * inv);
      st4(orow, 32 * j + 8 * e + 4 * g, a.d, v.x, v.y, v.z, v.w);
    }
}

// Joins the nsplit partials of a row, in split order: a thread holds 4 channels of one row.
template <int DT>
__global__ __launch_bounds__(256) void k_mha_join(MhaArgs a) {
  constexpr int PR = DT / 4;
  const int x = blockIdx.x * 256 + threadIdx.x;
  const int c = 4 * (x % PR), rr = x / PR;               // row of all row tiles
  const int lr = rr % 32, rt = (rr / 32) % a.nrt, bh = rr / 32 / a.nrt;
  const int hk = bh % a.Hk, b = bh / a.Hk, rho = rt * 32 + lr;
  if (b >= a.B || rho >= a.G * a.Sq) return;
  const float* slot = a.part + (int64_t)(bh * a.nrt + rt) * a.nsplit * 32 * (DT + 2);
  float M = -INFINITY, L = 0.f;
#pragma unroll 8
  for (int z = 0; z < a.nsplit; ++z) M = fmaxf(M, slot[(int64_t)z * 32 * (DT + 2) + lr]);
  const float Ms = M == -INFINITY ? 0.f : M;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int z = 0; z < a.nsplit; ++z) {
    const float* p = slot + (int64_t)z * 32 * (DT + 2);
    const float f = exp2_(p[lr] - Ms);
    const float4 v = *reinterpret_cast<const float4*>(p + 64 + lr * DT + c);
    L += p[32 + lr] * f;
    s.x += v.x * f; s.y += v.y * f; s.z += v.z * f; s.w += v.w * f;
  }
  const int i = rho / a.G, h = hk * a.G + rho - i * a.G;
  const Seq sq = seq_of(a, b);
  const bool any = i < sq.lq && L != 0.f;
  const float inv = any ? 1.f / L : 0.f;
  if (!any) s = make_float4(0.f, 0.f, 0.f, 0.f);
  st4(a.o + b * a.os[0] + i * a.os[1] + h * a.os[2], c, a.d, s.x * inv, s.y * inv, s.z * inv, s.w * inv);
}

// ------------------------------------------------------------- dq (query-owned)
// Issue-bound, as the forward: its three products fill the matrix cores 29 %
// of the time and vector instructions are issued in half of it (4 x 4096 x 8 heads
// x 64 with bias: two fifths of the pass's 795 us).  With a bias tiles near the diagonal
// are formed twice (below): all of them where none lies past max_distance.
// Also the row terms D = do . o and the log sums, kept for the key-owned pass
// as it starts its products from them, and the bias gradient: dS of
// the tiles near the diagonal, in a second visit, is summed per distance into
// an array of each wave (an order that is fixed; fp32 atomics in LDS took
// 134 cycles a wave instruction here), tiles past max_distance add into one
// register per side.

// Adds a tile of the accumulator layout (rows: keys, lanes: queries) along its
// diagonals, row - query = -31 .. 31, to arr: lane m of a half collects the
// wrapped diagonal row - query = m (mod 32) of its 16 rows, split where it
// wraps; the halves are joined, one stores each part.
PG_DEV void diag_add(float* arr, const f32x16& v, int lane) {
  const int g = lane >> 5, m = lane & 31;
  float up = 0.f, down = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int row = acc_row(r, g);
    const float x = __int_as_float(__builtin_amdgcn_ds_bpermute((((row - m) & 31) + 32 * g) * 4, __float_as_int(v[r])));
    up += m <= row ? x : 0.f;
    down += m <= row ? 0.f : x;
  }
  up += __shfl_xor(up, 32, 64);
  down += __shfl_xor(down, 32, 64);
  // another lane of this wave may have written the element last: no reordering
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  arr[g ? m - 32 : m] += g ? down : up;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Three waves a SIMD where the registers suffice; with bias they spill 44 bytes
// a lane then, which gains where most tiles are formed once and loses elsewhere
// (training 4 x 4096 x 8 heads x 64 777 us against 783, 16 x 300 with a
// max_distance of 256 85.0 against 83.2, 4 x 1024 with 512 149.7 against 147.0).
template <int DT, bool BIAS>
__global__ __launch_bounds__(256, DT == 64 && !BIAS ? 3 : 2) void k_mha_dq(MhaArgs a) {
  constexpr int TK = 64, NC = DT / 8, NT = DT / 32, KF = DT / 16;
  __shared__ __attribute__((aligned(16))) bf16_t Ks[2][TK * DT];
  __shared__ __attribute__((aligned(16))) bf16_t Vs[2][TK * DT];
  extern __shared__ float bs[];   // bias by distance, then each wave's sums of dS by distance
  const int id = block_no(a, a.nblk), qb = a.nblk - 1 - id % a.nblk, bh = id / a.nblk, h = bh % a.Hq, b = bh / a.Hq;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, lq = lane & 31;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Seq sq = seq_of(a, b);
  const int qblk = qb * 128, qw = qblk + wv * 32, q = qw + lq, p0 = qw + sq.off;
  const bf16_t* K = a.k + b * a.ks[0] + (h / a.G) * a.ks[2];
  const bf16_t* V = a.v + b * a.vs[0] + (h / a.G) * a.vs[2];
  const int bl = BIAS ? bias_len(a) : 0;
  float* const gs = bs + bl + wv * bl;
  if (BIAS) {
    for (int e = tid; e < bl; e += 256) bs[e] = bias2_at(a, h, e);
    for (int e = tid; e < 4 * bl; e += 256) bs[bl + e] = 0.f;
  }
  const bool steep = BIAS && steep_bias(a, h, lane);
  const float far_lo = BIAS ? uniform(bias2_at(a, h, 0)) : 0.f, far_hi = BIAS ? uniform(bias2_at(a, h, bl - 1)) : 0.f;
  const bool valid = q < sq.lq;
  const bf16_t* Q = a.q + b * a.qs[0] + q * a.qs[1] + h * a.qs[2];
  const bf16_t* DO = a.dO + b * a.os[0] + q * a.os[1] + h * a.os[2];
  const bf16_t* O = a.o + b * a.os[0] + q * a.os[1] + h * a.os[2];
  const uint2* const lo = a.olo + ((int64_t)bh * (a.Sqp / 32) + qw / 32) * (DT / 8) * 64;
  bf16x8 qf[KF], df[KF];
  float dd = 0.f;
#pragma unroll
  for (int t = 0; t < KF; ++t) {
    qf[t] = ld_frag(Q, 16 * t + 8 * g, a.d, valid);
    df[t] = ld_frag(DO, 16 * t + 8 * g, a.d, valid);
    // from the output and what its rounding took off (without that D is off by 2^-8 of |do||o|, and dq by half as
    // much again as its own rounding): left is the rounding of P as an operand, averaged over the keys
    float x[8], o[8], e8[8];
    unpack8(__builtin_bit_cast(uint4, df[t]), x);
    unpack8(__builtin_bit_cast(uint4, ld_frag(O, 16 * t + 8 * g, a.d, valid)), o);
    const int ji = 4 * (t / 2) + 2 * (t % 2) + g;
    uint2 e0 = make_uint2(0, 0), e1 = e0;
    if (valid) { e0 = lo[ji * 64 + lq]; e1 = lo[ji * 64 + 32 + lq]; }
    unpack8(make_uint4(e0.x, e0.y, e1.x, e1.y), e8);
#pragma unroll
    for (int e = 0; e < 8; ++e) dd = fmaf(x[e], o[e] + e8[e], dd);
  }
  dd += __shfl_xor(dd, 32, 64);
  // p = 2^(score - top), P = p inv.  Without a bias the log sum is part of top; with one (see kSteep) inv is multiplied
  // into the sums over a row at their end, so that it costs nothing in the loop.
  const float top = valid ? a.top[(int64_t)bh * a.Sqp + q] : INFINITY, lg = BIAS && valid ? a.lg[(int64_t)bh * a.Sqp + q] : 0.f;
  const float inv = BIAS ? exp2_(-lg) : 1.f;
  if (g == 0 && q < a.Sqp) {
    a.D[(int64_t)bh * a.Sqp + q] = valid ? -dd : 0.f;
    a.L[(int64_t)bh * a.Sqp + q] = steep && top != INFINITY ? 0.f : -(top + lg) / a.c;
  }
  const Row rw = row_of(a, sq.lk, q + sq.off);
  f32x16 acc[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
  // BIAS, per row (over inv): dS of the far tiles on either side, sum of dS, P of the far tiles on either side
  float flo = 0.f, fhi = 0.f, rho = 0.f, wlo = 0.f, whi = 0.f;
  Span<TK> sp = span_of<TK>(a, sq.lk, qblk + sq.off, min(qblk + 128, sq.lq) - 1 + sq.off);
  if (qblk >= sq.lq) sp.nt = 0;
  const Span<32> sw = span_of<32>(a, sq.lk, p0, min(qw + 32, sq.lq) - 1 + sq.off);
  const bool mine = qw < sq.lq;
  Ring<NC, TK> rk, rv;
  rk.init(a.ks[1], a.d, tid);
  rv.init(a.vs[1], a.d, tid);
  auto load = [&](int n, int bf) {
    const int k0 = sp.key0(n);
    auto ok = [&](int j) { return sp.row(j); };
    const bool all = sp.whole(k0);
    rk.issue(Ks[bf], K + k0 * a.ks[1], a.ks[1], k0, wv, all, ok);
    rv.issue(Vs[bf], V + k0 * a.vs[1], a.vs[1], k0, wv, all, ok);
  };
  // One pass over the keys.  NEAR (after the other, with a bias): see below.
  auto pass = [&](auto near_c) {
    constexpr bool NEAR = decltype(near_c)::value;
    const int pb0 = qblk + sq.off, pb1 = pb0 + 127;
    auto next = [&](int n) {   // the next tile to visit
      if (NEAR)
        while (n < sp.nt && !(sp.key0(n) + TK - 1 - pb0 > -a.maxd && sp.key0(n) - pb1 < a.maxd)) ++n;
      return n;
    };
    // visits tile n, returns the one after it (the buffer known at compile time, as in the forward)
    auto visit = [&](auto buf_c, int n) {
      constexpr int buf = decltype(buf_c)::value;
      wait_barrier<0>();   // tile n is in LDS, and every wave has left the tile before
      const int n1 = next(n + 1);
      if (n1 < sp.nt) load(n1, buf ^ 1);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int k0 = sp.key0(n) + 32 * x;
        const bool near = BIAS && k0 + 31 - p0 > -a.maxd && k0 - p0 - 31 < a.maxd;
        if (!mine || !sw.tile(k0) || (NEAR && !near)) continue;
        const bf16_t* ks = Ks[buf] + 32 * DT * x;
        const bf16_t* vs = Vs[buf] + 32 * DT * x;
        f32x16 s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) { s[r] = 0.f; dp[r] = 0.f; }
#pragma unroll
        for (int t = 0; t < KF; ++t) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_row<NC>(ks, lq, 16 * t + 8 * g), qf[t], s, 0, 0, 0);
          dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_row<NC>(vs, lq, 16 * t + 8 * g), df[t], dp, 0, 0, 0);
        }
        // scores as the forward forms them
        const float far = k0 < p0 ? far_lo : far_hi;
        if (BIAS && (near || fabsf(far) >= kDeep)) {
          const float* bl4 = bs + bias_row(a, near, k0, p0) - lq + 4 * g;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.c, bl4[8 * (r >> 2) + (r & 3)]) - top;
        } else {
          const float ft = far - top;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.c, ft);
        }
        if (!all_seen<32>(a, sq.lk, k0, p0, p0 + 31)) hide(s, rw, k0, g);
        if constexpr (NEAR) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = exp2_(s[r]) * inv * (dp[r] - (dd + rho));
          diag_add(gs + k0 - p0 + a.maxd + kMargin, s, lane);
          continue;
        }
        float w = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = exp2_(s[r]);
          if (BIAS) w += s[r];
        }
        float t = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] *= dp[r] - dd;
          if (BIAS) t += s[r];
        }
        if (BIAS) {
          rho += t;
          if (!near && k0 < p0) {
            flo += t;
            wlo += w;
          } else if (!near) {
            fhi += t;
            whi += w;
          }
        }
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2) {
          const bf16x8 sb = pack_regs(s, t2);
#pragma unroll
          for (int j = 0; j < NT; ++j)
            acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_tr<NC>(ks, t2, 32 * j, lane), sb, acc[j], 0, 0, 0);
        }
      }
      return n1;
    };
    int n = next(0);
    if (n < sp.nt) load(n, 0);
    while (n < sp.nt) {
      n = visit(std::integral_constant<int, 0>(), n);
      if (n < sp.nt) n = visit(std::integral_constant<int, 1>(), n);
    }
    __syncthreads();   // the tiles are free and the sums whole
  };
  pass(std::integral_constant<bool, false>());
  if (BIAS) {
    // dS sums to zero over a row, but with D from an output of rounded P it sums to
    // rho = (true D) - D, and the bias gradient, many sums of dS with little
    // left over, would show it.  The true dS is dS - rho P: the near tiles are
    // visited again for theirs, the far ones have their P summed a side.
    rho = (rho + __shfl_xor(rho, 32, 64)) * inv;
    pass(std::integral_constant<bool, true>());
    flo = (flo - rho * wlo) * inv;
    fhi = (fhi - rho * whi) * inv;
  }
  if (q < a.Sq) {
    bf16_t* row = a.dq + b * a.qs[0] + q * a.qs[1] + h * a.qs[2];
    const float f = valid ? a.scale * inv : 0.f;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x16& x = acc[j];
        st4(row, 32 * j + 8 * i + 4 * g, a.d, x[4 * i] * f, x[4 * i + 1] * f, x[4 * i + 2] * f, x[4 * i + 3] * f);
      }
  }
  if (BIAS) {
    flo = wave_sum(flo);
    fhi = wave_sum(fhi);
    if (lane == 0) { gs[0] += flo; gs[bl - 1] += fhi; }
    __syncthreads();
    for (int e = tid; e < bl; e += 256) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) t += bs[bl + w * bl + e];
      bs[e] = t;
    }
    __syncthreads();
    // 8 lanes a bucket
    const int mid = a.maxd + kMargin;
    for (int k = tid >> 3; k < (a.nb + 31) / 32 * 32; k += 32) {
      const bool up = k >= a.half;           // later keys (never with causal)
      const int kk = min(up ? k - a.half : k, a.half - 1), n0 = a.start[kk], n1 = kk + 1 < a.half ? a.start[kk + 1] : mid + 1;
      float t = 0.f;
      for (int n = n0 + (tid & 7); n < n1; n += 8)
        if (!(up && n == 0)) t += bs[up ? mid + n : mid - n];
      t += __shfl_xor(t, 1, 64);
      t += __shfl_xor(t, 2, 64);
      t += __shfl_xor(t, 4, 64);
      if ((tid & 7) == 0 && k < a.nb) a.part[((int64_t)bh * a.nblk + qb) * a.nb + k] = t;
    }
  }
}

// dbias[h][k] = sum of the partials of head h's query blocks: a block per
// head, a column and a part of the rows to each thread, the parts added in order.
__global__ __launch_bounds__(256) void k_mha_dbias(const float* part, int B, int Hq, int nblk, int nb, float* out) {
  __shared__ double sh[256];
  const int h = blockIdx.x, parts = 256 / nb, k = threadIdx.x % nb, p = threadIdx.x / nb;
  double t = 0.0;
  if (p < parts)
    for (int i = p; i < B * nblk; i += parts) t += part[(((int64_t)(i / nblk) * Hq + h) * nblk + i % nblk) * nb + k];
  sh[threadIdx.x] = t;
  __syncthreads();
  if (threadIdx.x >= nb) return;
  for (int j = 1; j < parts; ++j) t += sh[j * nb + k];
  out[(int64_t)h * nb + k] = (float)t;
}

// ------------------------------------------------------------- dk, dv (key-owned)
// A wave owns 32 keys of one key head, a block 128; the steps run over the
// query heads of the group and their tiles of queries, so the gradients of a
// shared head are summed in registers.  A key block that many queries see
// (first tokens beside a window; few, long sequences) is split over blocks of
// `chunk` steps, whose fp32 partials k_mha_dkv_join adds in split order.
// Held by dependences between its products and the exponentials at two waves a
// SIMD: matrix cores busy 35 % of the time, vector instructions issued in 32 %,
// waves waiting 46 % of theirs (4 x 4096 x 8 heads x 64 with bias: two fifths of
// the pass's 795 us).  Both
// halves of a query tile in one stretch without branches needed registers that
// cost more (355 -> 362 us a pass, 448 -> 519 at 128 channels); operands read
// ahead changed nothing.

// At head widths past 64 the values of the block's keys stay in LDS and the
// query tiles have 32 rows: two waves fit a SIMD then (with everything in
// registers one does, 240 us where this takes 198; 2 x 4096 x 16 / 4 heads x
// 128, window 1024).
constexpr int dkv_tile(int dt) { return dt > 64 ? 32 : 64; }

// the queries [i0, i1) that see some key of [j0, j1]: none, and no step, where all of these lie behind the last key
PG_DEV void seen_by(const MhaArgs& a, const Seq& sq, int j0, int j1, int& i0, int& i1) {
  j1 = min(j1, sq.lk - 1);
  const bool sink = a.window && j0 < a.n_sink;
  const int lo = a.causal ? j0 : a.window && !sink ? j0 - a.window + 1 : -0x40000000;
  const int hi = a.window && !sink ? j1 + a.window - 1 : 0x40000000;
  i0 = max(lo - sq.off, 0);
  i1 = min(hi - sq.off + 1, sq.lq);
  if (j1 < j0) i0 = i1 = 0;
}
// does some query see key j?  (Others may hold anything: as zeros they give nothing to a product with P = 0.)
PG_DEV bool key_seen(const MhaArgs& a, const Seq& sq, int j) {
  int i0, i1;
  seen_by(a, sq, j, j, i0, i1);
  return i0 < i1;
}

// item of a launch: key block, split, and the slot of its partials
struct KItem { int bh, kb, z; int64_t slot; };
PG_DEV KItem item_of(const MhaArgs& a, int x) {
  const int sinks = a.nks * a.ns_sink, per = sinks + (a.nblk - a.nks) * a.ns_reg;
  KItem it;
  it.bh = x / per;
  const int y = x - it.bh * per;
  if (y < sinks) {
    it.kb = y / a.ns_sink;
    it.z = y - it.kb * a.ns_sink;
  } else {
    it.kb = a.nks + (y - sinks) / a.ns_reg;
    it.z = (y - sinks) % a.ns_reg;
  }
  // slots only for the classes that split
  const int64_t both = (a.ns_sink > 1 ? sinks : 0) + (a.ns_reg > 1 ? per - sinks : 0);
  it.slot = it.bh * both + (y < sinks ? y : y - sinks + (a.ns_sink > 1 ? sinks : 0));
  return it;
}

// Two waves a SIMD: a third at 64 channels spills (the training of 4 x 4096 x 8
// heads with bias 869 us against 783, without bias 4 x 2048 x 16 heads 349
// against 345).
template <int DT, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_mha_dkv(MhaArgs a) {
  constexpr int TQ = dkv_tile(DT), NC = DT / 8, NT = DT / 32, KF = DT / 16;
  __shared__ __attribute__((aligned(16))) bf16_t Qs[2][TQ * DT];
  __shared__ __attribute__((aligned(16))) bf16_t Ds[2][TQ * DT];
  constexpr bool VL = DT > 64;
  __shared__ __attribute__((aligned(16))) bf16_t Vt[VL ? 128 * DT : 8];
  extern __shared__ float ex[];   // rows' L and D of the two tiles, then the current head's bias by query minus key
  float* const bs = ex + 4 * 64;
  bool steep = false;                       // of the current head: has it a bias that large, and
  float far_lo = 0.f, far_hi = 0.f;         // its biases past max_distance, of earlier and later keys
  const KItem it = item_of(a, block_no(a, a.nks * a.ns_sink + (a.nblk - a.nks) * a.ns_reg));
  const int hk = it.bh % a.Hk, b = it.bh / a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, lk = lane & 31;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Seq sq = seq_of(a, b);
  const int kblk = it.kb * 128;
  int i0, i1;
  seen_by(a, sq, kblk, kblk + 127, i0, i1);
  const int t0 = i0 / TQ, nt = max((i1 + TQ - 1) / TQ - t0, 0);
  const int n0 = it.z * a.chunk, n1 = min(n0 + a.chunk, nt * a.G);
  if (it.z > 0 && n0 >= n1) return;
  const int kw = kblk + wv * 32, key = kw + lk;
  const bool kv = key_seen(a, sq, key);
  const int bl = BIAS ? bias_len(a) : 0;
  bf16x8 kf[KF], vf[VL ? 1 : KF];
#pragma unroll
  for (int t = 0; t < KF; ++t) {
    kf[t] = ld_frag(a.k + b * a.ks[0] + key * a.ks[1] + hk * a.ks[2], 16 * t + 8 * g, a.d, kv);
    if (!VL) vf[t] = ld_frag(a.v + b * a.vs[0] + key * a.vs[1] + hk * a.vs[2], 16 * t + 8 * g, a.d, kv);
  }
  f32x16 adk[NT], adv[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) { adk[j][r] = 0.f; adv[j][r] = 0.f; }
  int w0, w1;
  seen_by(a, sq, kw, kw + 31, w0, w1);
  // this lane's key is seen from positions plo .. plo + pspan (none is at 2^31 - 1)
  const bool sink = key < a.n_sink;
  const int plo = !kv ? 0x7fffffff : a.causal ? key : a.window && !sink ? key - a.window + 1 : -0x40000000;
  const uint32_t pspan = !kv ? 0u : (uint32_t)((a.window && !sink ? key + a.window - 1 : 0x7fffffff) - (int64_t)plo);
  Ring<NC, TQ> rq, rd;
  rq.init(a.qs[1], a.d, tid);
  rd.init(a.os[1], a.d, tid);
  if (VL && n0 < n1) {
    Ring<NC, 64> rv;
    rv.init(a.vs[1], a.d, tid);
#pragma unroll
    for (int x = 0; x < 2; ++x)
      rv.issue(Vt + 64 * DT * x, a.v + b * a.vs[0] + (kblk + 64 * x) * a.vs[1] + hk * a.vs[2], a.vs[1], kblk + 64 * x, wv,
               false, [&](int j) { return key_seen(a, sq, j); });
  }
  // step (h, ti): query head of the group, query tile
  auto load = [&](int hg, int ti, int bf) {
    const int h = hk * a.G + hg, q0 = TQ * (t0 + ti);
    auto ok = [&](int i) { return i >= i0 && i < i1; };
    const bool all = q0 >= i0 && q0 + TQ <= i1;
    rq.issue(Qs[bf], a.q + b * a.qs[0] + h * a.qs[2] + q0 * a.qs[1], a.qs[1], q0, wv, all, ok);
    rd.issue(Ds[bf], a.dO + b * a.os[0] + h * a.os[2] + q0 * a.os[1], a.os[1], q0, wv, all, ok);
    // TQ rows of both: the buffers are padded to 64, rows past len_q hold -inf and 0
    const int64_t x = ((int64_t)b * a.Hq + h) * a.Sqp + q0;
    if (wv == 0) lds_load4(lds_addr(ex + bf * 128), lane * 4, make_rsrc(a.L + x, TQ * 4));
    if (wv == 1) lds_load4(lds_addr(ex + bf * 128 + 64), lane * 4, make_rsrc(a.D + x, TQ * 4));
  };
  int hg = 0, ti = 0;
  if (n0 < n1) {
    hg = n0 / nt;
    ti = n0 - hg * nt;
    load(hg, ti, 0);
  }
  auto visit = [&](auto buf_c, int n) {
    const int buf = buf_c;
    wait_barrier<0>();   // tile n is in LDS, and every wave has left tile n - 1
    const int h = hg, qt = TQ * (t0 + ti), pt = qt + sq.off;
    const bool fresh = n == n0 || ti == 0;
    if (++ti == nt) {
      ti = 0;
      ++hg;
    }
    if (n + 1 < n1) load(hg, ti, buf ^ 1);
    if (BIAS && fresh) {   // the next head's bias
      for (int e = tid; e < bl; e += 256) bs[e] = bias2_at(a, hk * a.G + h, bl - 1 - e);
      steep = steep_bias(a, hk * a.G + h, lane);
      far_lo = uniform(bias2_at(a, hk * a.G + h, 0));
      far_hi = uniform(bias2_at(a, hk * a.G + h, bl - 1));
      __syncthreads();
    }
#pragma unroll
    for (int x = 0; x < TQ / 32; ++x) {
      const int q0 = qt + 32 * x, p0 = pt + 32 * x;
      if (q0 + 32 <= w0 || q0 >= w1) continue;
      const bf16_t* qs = Qs[buf] + 32 * DT * x;
      const bf16_t* ds = Ds[buf] + 32 * DT * x;
      const float* Ls = ex + buf * 128 + 32 * x;
      f32x16 s, dp;
      // the products start from the row terms: s comes out as the score less the log sum (over c; with a steep bias as the
      // score alone), dp less D
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 l4 = *reinterpret_cast<const float4*>(Ls + 8 * i + 4 * g);
        const float4 d4 = *reinterpret_cast<const float4*>(Ls + 64 + 8 * i + 4 * g);
        s[4 * i] = l4.x; s[4 * i + 1] = l4.y; s[4 * i + 2] = l4.z; s[4 * i + 3] = l4.w;
        dp[4 * i] = d4.x; dp[4 * i + 1] = d4.y; dp[4 * i + 2] = d4.z; dp[4 * i + 3] = d4.w;
      }
#pragma unroll
      for (int t = 0; t < KF; ++t) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_row<NC>(qs, lk, 16 * t + 8 * g), kf[t], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_row<NC>(ds, lk, 16 * t + 8 * g),
                                                     VL ? ld_row<NC>(Vt + wv * 32 * DT, lk, 16 * t + 8 * g) : vf[VL ? 0 : t], dp, 0, 0, 0);
      }
      float cm = a.c, off = 0.f;   // as in the forward
      if (BIAS) {
        const bool near = kw + 31 - p0 > -a.maxd && kw - p0 - 31 < a.maxd;
        const float far = kw < p0 ? far_lo : far_hi;
        if (near || (steep && fabsf(far) >= kDeep)) {
          // queries are to keys here as keys to queries there
          const float* bn = bs + bias_row(a, near, p0, kw) - lk + 4 * g;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.c, bn[8 * (r >> 2) + (r & 3)]);
          cm = 1.f;
        } else {
          off = far;
        }
        if (steep) {   // rare: the rows' terms from memory
          const int64_t row = ((int64_t)b * a.Hq + hk * a.G + h) * a.Sqp + q0 + 4 * g;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 m4 = *reinterpret_cast<const float4*>(a.top + row + 8 * i);
            const float4 g4 = *reinterpret_cast<const float4*>(a.lg + row + 8 * i);
            s[4 * i] = fmaf(s[4 * i], cm, off - m4.x) - g4.x;
            s[4 * i + 1] = fmaf(s[4 * i + 1], cm, off - m4.y) - g4.y;
            s[4 * i + 2] = fmaf(s[4 * i + 2], cm, off - m4.z) - g4.z;
            s[4 * i + 3] = fmaf(s[4 * i + 3], cm, off - m4.w) - g4.w;
            asm volatile("" ::: "memory");   // few of them in registers at once
          }
          cm = 1.f;
          off = 0.f;
        }
      }
      if (!all_seen<32>(a, sq.lk, kw, p0, p0 + 31)) {
        const uint32_t at = (uint32_t)(p0 + 4 * g - plo);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (at + 8 * (r >> 2) + (r & 3) > pspan) s[r] = -INFINITY;
      }
      f32x16 p;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[r] = exp2_(BIAS ? fmaf(s[r], cm, off) : s[r] * a.c);
        s[r] = p[r] * dp[r];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16x8 pb = pack_regs(p, t), sb = pack_regs(s, t);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          adv[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_tr<NC>(ds, t, 32 * j, lane), pb, adv[j], 0, 0, 0);
          adk[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld_tr<NC>(qs, t, 32 * j, lane), sb, adk[j], 0, 0, 0);
        }
      }
    }
  };
  if constexpr (VL) {   // no registers to spare for two copies of the loop
    for (int n = n0; n < n1; ++n) visit((n - n0) & 1, n);
  } else {
    for (int n = n0; n < n1; n += 2) {
      visit(std::integral_constant<int, 0>(), n);
      if (n + 1 < n1) visit(std::integral_constant<int, 1>(), n + 1);
    }
  }
  if (nt * a.G > a.chunk) {   // one of several splits: partials, key rows of dk then of dv
    float* row = a.part + ((it.slot * 128 + key - kblk) * 2) * DT;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x16 &x = adk[j], &y = adv[j];
        *reinterpret_cast<float4*>(row + 32 * j + 8 * i + 4 * g) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        *reinterpret_cast<float4*>(row + DT + 32 * j + 8 * i + 4 * g) = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
      }
    return;
  }
  if (key >= a.Sk) return;
  bf16_t* dkr = a.dk + b * a.ks[0] + key * a.ks[1] + hk * a.ks[2];
  bf16_t* dvr = a.dv + b * a.vs[0] + key * a.vs[1] + hk * a.vs[2];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x16 &x = adk[j], &y = adv[j];
      st4(dkr, 32 * j + 8 * i + 4 * g, a.d, x[4 * i] * a.scale, x[4 * i + 1] * a.scale, x[4 * i + 2] * a.scale,
          x[4 * i + 3] * a.scale);
      st4(dvr, 32 * j + 8 * i + 4 * g, a.d, y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
    }
}

// Adds the partials of a split key block: a block per (16 keys, key block), a thread per 4 channels of dk or dv.
template <int DT>
__global__ __launch_bounds__(256) void k_mha_dkv_join(MhaArgs a) {
  constexpr int PR = 2 * DT / 4;
  // the key blocks of the classes that split, 8 parts of 16 keys in each
  const int first = a.ns_sink > 1 ? 0 : a.nks, many = (a.ns_reg > 1 ? a.nblk : a.nks) - first;
  const int part = blockIdx.x & 7, kb = first + (blockIdx.x >> 3) % many, bh = (blockIdx.x >> 3) / many;
  const int hk = bh % a.Hk, b = bh / a.Hk;
  const Seq sq = seq_of(a, b);
  int i0, i1;
  seen_by(a, sq, kb * 128, kb * 128 + 127, i0, i1);
  constexpr int TQ = dkv_tile(DT);
  const int steps = max((i1 + TQ - 1) / TQ - i0 / TQ, 0) * a.G, ns = (steps + a.chunk - 1) / a.chunk;
  if (ns <= 1) return;
  const int sinks = a.nks * a.ns_sink, per = sinks + (a.nblk - a.nks) * a.ns_reg;
  const KItem it = item_of(a, bh * per + (kb < a.nks ? kb * a.ns_sink : sinks + (kb - a.nks) * a.ns_reg));
  for (int x = threadIdx.x; x < 16 * PR; x += 256) {
    const int lr = part * 16 + x / PR, c = 4 * (x % PR), key = kb * 128 + lr;
    if (key >= a.Sk) continue;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int z = 0; z < ns; ++z) {
      const float4 v = *reinterpret_cast<const float4*>(a.part + (((it.slot + z) * 128 + lr) * 2) * DT + c);
      t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
    }
    if (c < DT) {
      const float f = a.scale;
      st4(a.dk + b * a.ks[0] + key * a.ks[1] + hk * a.ks[2], c, a.d, t.x * f, t.y * f, t.z * f, t.w * f);
    } else {
      st4(a.dv + b * a.vs[0] + key * a.vs[1] + hk * a.vs[2], c - DT, a.d, t.x, t.y, t.z, t.w);
    }
  }
}

// ------------------------------------------------------------- launchers
// Heads to keep together on an XCD: those of one key head where that deals
// evenly, else an eighth of all.  Sequences of different lengths need several
// sets on each XCD to even out (train 2 x 4096 x 16 / 4 heads x 128 through a
// window, full and three quarters long: 783 us in plain order, 835 so).
int head_set(int64_t heads, int group, bool ragged) {
  if (heads % 8) return 0;
  const int64_t m = heads / group % 8 == 0 ? group : heads / 8;
  return ragged && heads / m < 32 ? 0 : (int)m;
}

int pad_d(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : 128; }

// Smallest distance of each of the `half` buckets of a side: n for the exact
// ones, below half / 2; bucket half / 2 + e starts at the first whole number at
// or above (half / 2) (maxd / (half / 2))^(e / (half - half / 2)).  A boundary
// that is not itself whole is at least 5e-11 of its size from a whole number
// (counted over all half <= 256, maxd <= 512), so rounding cannot move it.
void bucket_starts(int half, int maxd, uint16_t* start) {
  const int first = half / 2;
  for (int k = 0; k <= first; ++k) start[k] = (uint16_t)k;
  const double step = std::log2((double)maxd / first) / (half - first);
  for (int e = 1; first + e < half; ++e) {
    const double x = first * std::exp2(step * e);
    start[first + e] = (uint16_t)std::ceil(x - 1e-12 * x);
  }
}

MhaArgs make_args(const Mha& m) {
  MhaArgs a{};
  a.B = m.B; a.Sq = m.Sq; a.Sk = m.Sk; a.Hq = m.Hq; a.Hk = m.Hk; a.G = m.Hq / m.Hk; a.d = m.d;
  a.Sqp = (int)cdiv(m.Sq, 64) * 64;
  a.causal = m.causal; a.window = m.window; a.n_sink = m.n_sink;
  a.nb = m.n_buckets; a.maxd = m.n_buckets ? m.max_distance : 0;
  a.half = m.causal ? m.n_buckets : m.n_buckets / 2;
  a.scale = m.scale; a.c = m.scale * kL2E;
  for (int i = 0; i < 3; ++i) { a.qs[i] = m.qs[i]; a.ks[i] = m.ks[i]; a.vs[i] = m.vs[i]; a.os[i] = m.os[i]; }
  if (m.n_buckets) {
    bucket_starts(a.half, m.max_distance, a.start);
    for (int k = 0; k < a.half; ++k) {   // a bucket without a distance of its own leaves no mark
      const int end = k + 1 < a.half ? a.start[k + 1] : m.max_distance + 1;
      for (int n = a.start[k]; n < end; ++n) a.lut[n] = (uint8_t)k;
    }
  }
  return a;
}

void set_saved(MhaArgs& a, void* saved) {
  const size_t rows = align256((size_t)a.B * a.Hq * a.Sqp * 4);
  a.top = (float*)saved;
  a.lg = (float*)((char*)saved + rows);
  a.olo = (uint2*)((char*)saved + 2 * rows);
}

int64_t row_tiles(const Mha& m) { return cdiv((int64_t)m.Sq * (m.Hq / m.Hk), 32); }
// Which calls without a backward take the form for a few new tokens: those of
// few queries (the other form leaves three of its four waves idle: 64 x 16
// queries of 32 / 8 heads x 128 over 1024 keys 94 us against 137; 32 queries
// 183 against 142) and those whose row tiles leave CUs without work (128
// queries of 8 heads x 64 over 32768 keys 39 us against 605; 8192 causal queries
// of one head 53 against 128, through a window of 16 5 against 8; 256 tiles, causal
// 2 x 512 x 8 heads x 128, 12.5 against 16.3; 512 of them, 4 x 512, 25 against 17,
// though 16 against 20 at 64 channels over 1024 keys).
bool few_rows(const Mha& m) { return m.Sq <= 16 || (int64_t)m.B * m.Hk * row_tiles(m) <= 256; }

// Splits of the keys: a block for each CU, at least 8 tiles in each (two a
// wave): the caches are read at 5.1 TB/s then, and three blocks a CU lose 15 %
// to the partials they leave.  In whole numbers, so that row tiles past half of
// the CUs or just past all of them leave CUs idle: caches of 8192 x 8 heads x 128
// are read at 5.7 TB/s for 32 sequences, 4.5 for 17 and 3.8 for 33 (same inputs every time).
int step_splits(const Mha& m) {
  const int64_t queries = std::min<int64_t>(m.Sq, cdiv(32, m.Hq / m.Hk) + 1);   // of a row tile
  const int64_t tiles = m.window ? std::min<int64_t>(cdiv(m.Sk, 32), cdiv((m.causal ? 1 : 2) * (int64_t)m.window + queries, 32) + 1 + cdiv(m.n_sink, 32))
                                 : cdiv(m.Sk, 32);
  return (int)std::max<int64_t>(1, std::min(256 / (m.B * m.Hk * row_tiles(m)), cdiv(tiles, 8)));
}

// How the key-owned pass is cut: blocks of 128 keys; a block's steps are
// G x (query tiles that see it).  Blocks with first tokens, which every
// query sees, and all blocks where they are few, are split into pieces of
// `chunk` steps: the number of pieces with the least modelled time, the steps
// over the places on the card plus half the last piece, a piece's partials
// costing about as much as 256 queries to write and add.  The model is not
// exact: swept by hand it was 5 to 7 % off the best number of pieces (2 x 4096 x 16
// / 4 heads x 128 in 1, 2, 3, 6 and 10 pieces: window 1024 491, 389, 435, 452, 513 us
// and its 4 pieces 417; causal 1219, 916, 807, 827, 833 and its own 847).
constexpr int64_t kMaxSlots = 8192;   // partials of at most 1 GB (128 keys x 2 x 128 channels each)
struct KPlan { int nkb, nks, ns_sink, ns_reg, chunk; int64_t items, slots; };
KPlan plan_keys(const Mha& m) {
  const int64_t tq = dkv_tile(pad_d(m.d)), G = m.Hq / m.Hk, all = G * cdiv(m.Sq, tq), bh = (int64_t)m.B * m.Hk, nkb = cdiv(m.Sk, 128);
  const int64_t reg = m.window ? std::min(all, G * (cdiv((m.causal ? 1 : 2) * (int64_t)m.window + 128, tq) + 1)) : all;
  const int64_t nks = m.window && reg < all ? std::min<int64_t>(nkb, cdiv(m.n_sink, 128)) : 0;
  const double places = 512, used = m.causal && !m.window ? 0.5 : 1.0;   // half of a triangle
  const double total = (double)bh * (nks * all + (nkb - nks) * reg * used);
  KPlan best{(int)nkb, (int)nks, 1, 1, (int)std::min<int64_t>(all, 1 << 30), bh * nkb, 0};   // nothing split
  double least = total / places + 0.5 * best.chunk;
  for (int64_t ns = 1; ns <= 16; ++ns) {
    KPlan p{};
    p.nkb = (int)nkb; p.nks = (int)nks;
    p.chunk = (int)std::min<int64_t>(cdiv(reg, ns), 1 << 30);
    p.ns_sink = (int)cdiv(all, p.chunk);
    p.ns_reg = (int)cdiv(reg, p.chunk);
    p.items = bh * (nks * p.ns_sink + (nkb - nks) * p.ns_reg);
    p.slots = bh * ((p.ns_sink > 1 ? nks * p.ns_sink : 0) + (p.ns_reg > 1 ? (nkb - nks) * p.ns_reg : 0));
    const double t = (total + 256.0 / tq * used * p.slots) / places + 0.5 * p.chunk;
    if (p.slots <= kMaxSlots && p.items < (1 << 24) && t < least) { best = p; least = t; }
  }
  return best;
}

size_t bias_bytes(const Mha& m, int arrays) {
  return m.n_buckets ? (size_t)arrays * (2 * (m.max_distance + kMargin) + 1) * 4 : 0;
}

#define PG_DT(d, ...)                                       \
  switch (pad_d(d)) {                                       \
    case 32: { constexpr int DT = 32; __VA_ARGS__; break; } \
    case 64: { constexpr int DT = 64; __VA_ARGS__; break; } \
    case 96: { constexpr int DT = 96; __VA_ARGS__; break; } \
    default: { constexpr int DT = 128; __VA_ARGS__; break; } \
  }

}  // namespace

size_t mha_saved_bytes(const Mha& m) {
  const size_t rows = (size_t)m.B * m.Hq * (size_t)cdiv(m.Sq, 64) * 64;
  return 2 * align256(rows * 4) + align256(rows * pad_d(m.d) * 2);   // the rows' maxima and log2 sums, the output's remainder
}

size_t mha_ws_bytes(const Mha& m) {
  const size_t rows = (size_t)m.B * m.Hq * (size_t)cdiv(m.Sq, 64) * 64;
  // the rows' D and L, then the bias partials or (after these are joined) those of dk and dv
  const size_t bias = (size_t)m.B * m.Hq * cdiv(m.Sq, 128) * m.n_buckets * 4;
  const size_t keys = (size_t)plan_keys(m).slots * 128 * 2 * pad_d(m.d) * 4;
  const size_t bwd = 2 * align256(rows * 4) + align256(std::max(bias, keys));
  size_t step = 0;
  if (few_rows(m) && step_splits(m) > 1) step = (size_t)m.B * m.Hk * row_tiles(m) * step_splits(m) * 32 * (pad_d(m.d) + 2) * 4;
  return std::max<size_t>(std::max(bwd, align256(step)), 256);
}

void mha_fwd(hipStream_t st, const Mha& m, const void* q, const void* k, const void* v, const float* table,
             const int32_t* len_q, const int32_t* len_k, void* o, void* saved, void* ws) {
  MhaArgs a = make_args(m);
  a.q = (const bf16_t*)q; a.k = (const bf16_t*)k; a.v = (const bf16_t*)v; a.o = (bf16_t*)o;
  a.table = table; a.len_q = len_q; a.len_k = len_k;
  const double flops = 4.0 * m.B * m.Hq * (double)m.Sq * m.Sk * m.d;
  if (!saved && few_rows(m)) {
    a.nsplit = step_splits(m);
    a.nrt = (int)row_tiles(m);
    a.part = (float*)ws;
    const dim3 grid((unsigned)((int64_t)m.B * m.Hk * a.nrt * a.nsplit));
    const size_t dyn = m.n_buckets ? align256(2 * (m.max_distance + kMargin) + 4) + (m.n_buckets <= kStepTable ? (size_t)128 * m.n_buckets : 0) : 0;
    ProfScope prof(st);
    PG_DT(m.d, {
      if (m.n_buckets) hipLaunchKernelGGL((k_mha_step<DT, true>), grid, dim3(256), dyn, st, a);
      else hipLaunchKernelGGL((k_mha_step<DT, false>), grid, dim3(256), 0, st, a);
      if (a.nsplit > 1)
        hipLaunchKernelGGL(k_mha_join<DT>, dim3((unsigned)cdiv((int64_t)m.B * m.Hk * a.nrt * 32 * (DT / 4), 256)), dim3(256), 0, st, a);
    });
    PG_LAUNCH_CHECK();
    prof.done("k_mha_step<" + std::to_string(pad_d(m.d)) + ">", flops);
    return;
  }
  if (saved) set_saved(a, saved);
  a.nblk = (int)cdiv(m.Sq, 128);
  a.hset = head_set((int64_t)m.B * m.Hq, a.G, len_k || len_q);
  const dim3 grid((unsigned)((int64_t)m.B * m.Hq * a.nblk));
  ProfScope prof(st);
  PG_DT(m.d, {
    if (m.n_buckets) hipLaunchKernelGGL((k_mha_fwd<DT, true>), grid, dim3(256), bias_bytes(m, 1), st, a);
    else hipLaunchKernelGGL((k_mha_fwd<DT, false>), grid, dim3(256), 0, st, a);
  });
  PG_LAUNCH_CHECK();
  prof.done("k_mha_fwd<" + std::to_string(pad_d(m.d)) + ">", flops);
}

void mha_bwd(hipStream_t st, const Mha& m, const void* q, const void* k, const void* v, const float* table,
             const int32_t* len_q, const int32_t* len_k, const void* o, const void* saved, const void* dO, void* dq,
             void* dk, void* dv, float* dtable, void* ws) {
  MhaArgs a = make_args(m);
  a.q = (const bf16_t*)q; a.k = (const bf16_t*)k; a.v = (const bf16_t*)v; a.o = (bf16_t*)const_cast<void*>(o);
  a.table = table; a.len_q = len_q; a.len_k = len_k;
  a.dO = (const bf16_t*)dO; a.dq = (bf16_t*)dq; a.dk = (bf16_t*)dk; a.dv = (bf16_t*)dv;
  set_saved(a, const_cast<void*>(saved));
  const size_t rows = (size_t)m.B * m.Hq * a.Sqp;
  a.D = (float*)ws;
  a.L = (float*)((char*)ws + align256(rows * 4));
  a.part = (float*)((char*)ws + 2 * align256(rows * 4));
  ProfScope prof(st);
  PG_DT(m.d, {
    a.nblk = (int)cdiv(m.Sq, 128);
    a.hset = head_set((int64_t)m.B * m.Hq, a.G, len_k || len_q);
    const dim3 gq((unsigned)((int64_t)m.B * m.Hq * a.nblk));
    if (m.n_buckets) {
      hipLaunchKernelGGL((k_mha_dq<DT, true>), gq, dim3(256), bias_bytes(m, 5), st, a);
      hipLaunchKernelGGL(k_mha_dbias, dim3((unsigned)m.Hq), dim3(256), 0, st, a.part,
                         m.B, m.Hq, a.nblk, m.n_buckets, dtable);
    } else {
      hipLaunchKernelGGL((k_mha_dq<DT, false>), gq, dim3(256), 0, st, a);
    }
    const KPlan p = plan_keys(m);
    a.nblk = p.nkb; a.nks = p.nks; a.ns_sink = p.ns_sink; a.ns_reg = p.ns_reg; a.chunk = p.chunk;
    a.hset = head_set((int64_t)m.B * m.Hk, 1, len_k || len_q);
    const dim3 gk((unsigned)p.items);
    if (m.n_buckets) hipLaunchKernelGGL((k_mha_dkv<DT, true>), gk, dim3(256), bias_bytes(m, 1) + 1024, st, a);
    else hipLaunchKernelGGL((k_mha_dkv<DT, false>), gk, dim3(256), 1024, st, a);
    if (p.slots) {
      const int many = (p.ns_reg > 1 ? p.nkb : p.nks) - (p.ns_sink > 1 ? 0 : p.nks);
      hipLaunchKernelGGL(k_mha_dkv_join<DT>, dim3((unsigned)((int64_t)m.B * m.Hk * many * 8)), dim3(256), 0, st, a);
    }
  });
  PG_LAUNCH_CHECK();
  prof.done("k_mha_bwd<" + std::to_string(pad_d(m.d)) + ">", 14.0 * m.B * m.Hq * (double)m.Sq * m.Sk * m.d);
}

}  // namespace pg
