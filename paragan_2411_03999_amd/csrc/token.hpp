// Launchers of the token attention operators (qknorm.hip, mha.hip).
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

}  // namespace pg
