// Register and LDS tiles of the attention kernels (bf16 MFMA 32x32x16): the
// score tile's register order, swizzled LDS rows, row-major and transposed
// operand reads.
#pragma once
#include "common.hpp"

namespace pg {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
constexpr float kL2E = 1.4426950408889634f;   // log2(e)
constexpr float kTau = 8.f;                   // lazy-rescale threshold (log2 units)

PG_DEV bf16x8 ld8g(const bf16_t* p) { return *reinterpret_cast<const bf16x8*>(p); }
PG_DEV bf16x8 zero8() {
  uint4 q = make_uint4(0, 0, 0, 0);
  return *reinterpret_cast<bf16x8*>(&q);
}
PG_DEV bf16x8 pack_regs(const f32x16& v, int t) {
  const uint4 q = make_uint4(f2bf2(v[8 * t], v[8 * t + 1]), f2bf2(v[8 * t + 2], v[8 * t + 3]),
                             f2bf2(v[8 * t + 4], v[8 * t + 5]), f2bf2(v[8 * t + 6], v[8 * t + 7]));
  return __builtin_bit_cast(bf16x8, q);
}
// row index (within a 32-tile) held by accumulator register r of lane group g
PG_DEV int acc_row(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }
PG_DEV float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- LDS tiles: rows of NC 16-byte chunks, chunk index XOR-swizzled by row
template <int NC>
PG_DEV int swz16(int r) {
  if (NC == 8) return ((r >> 2) & 3) | (((r >> 1) & 1) << 2);
  if (NC == 16) return 4 * (r & 3) + ((r >> 2) & 3);
  return (r >> 2) & 3;   // NC = 4 or 12
}
template <int NC>
PG_DEV int toff(int r, int e) {
  return r * NC * 8 + ((((e >> 3) ^ swz16<NC>(r))) << 3) + (e & 7);
}
// row-major operand: 8 consecutive elements of row r starting at e (e % 8 == 0)
template <int NC>
PG_DEV bf16x8 ld_row(const bf16_t* t, int r, int e) {
  return *reinterpret_cast<const bf16x8*>(t + toff<NC>(r, e));
}
// transposed operand: column c0 + lane%32 of rows {16kk + 4g + 0..3, 16kk + 8 + 4g + 0..3}
template <int NC>
PG_DEV bf16x8 ld_tr(const bf16_t* t, int kk, int c0, int lane) {
  const int r = 16 * kk + 4 * (lane >> 5) + ((lane & 15) >> 2);
  const int c = c0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(t + toff<NC>(r, c)));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(t + toff<NC>(r + 8, c)));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

}  // namespace

}  // namespace pg
