// Launchers of the token operators (qknorm.hip, mha.hip, blocknorm.hip, scan.hip, clip.hip).
#pragma once
#include "common.hpp"

namespace pg {

struct QkNorm {
  int64_t T;
  int Hq, Hk, d, rot, n_pos;
  bool inter, f32;
  float eps;
  int64_t ldq, ldk, ldqo, ldko;   // elements between tokens of q, k and of their outputs / output gradients
};
size_t qknorm_ws_bytes(const QkNorm& a);
void qknorm_fwd(hipStream_t st, const QkNorm& a, const void* q, const void* k, const float* gq, const float* gk,
                const float* table, const int32_t* pos, void* qo, void* ko);
void qknorm_bwd(hipStream_t st, const QkNorm& a, const void* q, const void* k, const float* gq, const float* gk,
                const float* table, const int32_t* pos, const void* dqo, const void* dko, void* dq, void* dk,
                float* dgq, float* dgk, void* ws);

constexpr int kMhaMaxDist = 512;   // largest max_distance of a bias
struct Mha {
  int B, Sq, Sk, Hq, Hk, d;
  bool causal;
  int window, n_sink, n_buckets, max_distance;
  float scale;
  int64_t qs[3], ks[3], vs[3], os[3];   // elements between sequences, tokens, heads
};
size_t mha_saved_bytes(const Mha& m);
size_t mha_ws_bytes(const Mha& m);
void mha_fwd(hipStream_t st, const Mha& m, const void* q, const void* k, const void* v, const float* table,
             const int32_t* len_q, const int32_t* len_k, void* o, void* saved, void* ws);
void mha_bwd(hipStream_t st, const Mha& m, const void* q, const void* k, const void* v, const float* table,
             const int32_t* len_q, const int32_t* len_k, const void* o, const void* saved, const void* dO, void* dq,
             void* dk, void* dv, float* dtable, void* ws);

struct BlockNorm {
  int B, S, D;
  bool f32, res32, layer, branch, post, pre;   // f32: h, y; res32: x, z
  float eps, res_scale;
  int64_t mod;                                 // elements between sequences' modulation rows
  int64_t xs[2], hs[2], zs[2], ys[2];          // elements between sequences, tokens
};
struct BlockNormRows {                         // [D] or modulation rows, each may be null
  const float *gain_post, *gate, *gain_pre, *scale, *shift;
};
struct BlockNormGrads {
  float *gain_post, *gate, *gain_pre, *scale, *shift;
};
size_t blocknorm_saved_bytes(const BlockNorm& a);
size_t blocknorm_ws_bytes(const BlockNorm& a);
void blocknorm_fwd(hipStream_t st, const BlockNorm& a, const BlockNormRows& w, const void* x, const void* h,
                   const int32_t* len, void* z, void* y, void* saved);
void blocknorm_bwd(hipStream_t st, const BlockNorm& a, const BlockNormRows& w, const void* x, const void* h,
                   const int32_t* len, const void* saved, const void* dz, const void* dy, void* dx, void* dh,
                   const BlockNormGrads& g, void* ws);

struct Scan {
  int B, S, D;
  bool f32, reverse;
  float sharp;
  int64_t xs[2], rs[2], gs[2], ys[2];          // elements between sequences, tokens
};
size_t scan_saved_bytes(const Scan& a);
size_t scan_ws_bytes(const Scan& a);
void scan_fwd(hipStream_t st, const Scan& a, const void* x, const void* r, const void* g, const float* decay,
              const int32_t* len, const float* h0, void* y, float* ht, void* saved, void* ws);
void scan_bwd(hipStream_t st, const Scan& a, const void* x, const void* r, const void* g, const float* decay,
              const int32_t* len, const void* saved, const void* dy, const float* dht, void* dx, void* dr, void* dg,
              float* ddecay, float* dh0, void* ws);

constexpr int kClipPiece = 16384;              // bytes of a piece of a tensor
struct ClipPiece {                             // one entry of a plan
  uint64_t src, dst;
  int32_t n, bf16;
};
size_t clip_ws_bytes();
void clip(hipStream_t st, int64_t n_pieces, double bytes, bool in_place, const void* plan, float max_norm,
          float grad_scale, float* norm, void* ws);
// Norm and factor of one flat fp32 gradient, for an optimiser that takes the factor along: norm [2], part
// kClipFlatBlocks doubles
constexpr int kClipFlatBlocks = 1024;
void clip_flat(hipStream_t st, const float* g, int64_t n, float max_norm, float* norm, double* part);

}  // namespace pg
