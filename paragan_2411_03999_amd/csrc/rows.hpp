// Eight elements of a row a lane, as the norms over rows (qknorm.hip,
// blocknorm.hip) read, write and sum them.
#pragma once
#include "common.hpp"

namespace pg {

// 8 elements as they lie in memory, and as floats
template <typename T> struct Raw;
template <> struct Raw<bf16_t> {
  uint4 v;
  PG_DEV void load(const bf16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
  PG_DEV void get(float* f) const { unpack8(v, f); }
};
template <> struct Raw<float> {
  float4 a, b;
  PG_DEV void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  PG_DEV void get(float* f) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};
template <typename T> PG_DEV void st8f(T* p, const float* f);
template <> PG_DEV void st8f<bf16_t>(bf16_t* p, const float* f) { *reinterpret_cast<uint4*>(p) = pack8(f); }
template <> PG_DEV void st8f<float>(float* p, const float* f) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

template <int CTRL>
PG_DEV float lane_move(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
// v of this lane and of the lane N away (16 or 32, the bit of the lane's number flipped): the swap leaves one of them in
// either of its results
template <int N>
PG_DEV float half_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  if constexpr (N == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
}
// sum over the LPH lanes of a group, in every lane
template <int LPH>
PG_DEV float group_sum(float v) {
  if (LPH > 1) v += lane_move<0xB1>(v);    // quad lanes 1 0 3 2
  if (LPH > 2) v += lane_move<0x4E>(v);    // quad lanes 2 3 0 1
  if (LPH > 4) v += lane_move<0x141>(v);   // the other quad of 8 (mirrored; a quad is uniform by now)
  if (LPH > 8) v += lane_move<0x140>(v);   // the other half of 16 (mirrored)
  if (LPH > 16) v = half_sum<16>(v);
  if (LPH > 32) v = half_sum<32>(v);
  return v;
}

}  // namespace pg
