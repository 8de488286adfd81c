// The norm of many gradients together, and clipping by it.
//
//   norm = grad_scale (sum g^2)^1/2,  factor = grad_scale (norm <= max ? 1 : max / norm),  out = factor g.
//
// Bound by memory: the tensors are read for the sum, and read and written
// for the result.  The tensors come as pieces of up to kClipPiece bytes from a
// table in device memory, so one launch takes all of them; a block takes
// pieces in a fixed order, all loads of one under way together and the next
// one's entry read meanwhile.  Squares are summed in 64 bits, where those
// of the largest and smallest floats are finite and not zero, in a thread,
// over a block's threads and over the blocks in order: the same call gives
// the same bits.
// Measured: 158 M floats in 300 tensors 106 us to read (6.0 TB/s) and 208 us to
// read and write (6.1, part of it from cache), in place 110 and 202, and 5
// where nothing is clipped; 40 M bf16 15 and 30 us; 200 k floats two launches
// of 3 and 4 us.  The norm of one flat gradient of 88 M floats, for an
// optimiser that takes the factor along: 60 us (5.9 TB/s) and 5 to the factor.
#include "token.hpp"

namespace pg {

namespace {

constexpr int kBlocks = 1536;      // at most: blocks of either launch (1024 to 4096 within 4 %)
constexpr double kCache = 256e6;   // bytes that the last cache level holds
PG_DEV void square8(uint4 v, double& s) {
  float f[8];
  unpack8(v, f);
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fma((double)f[e], (double)f[e], s);
}
PG_DEV void square4(float4 v, double& s) {
  s = fma((double)v.x, (double)v.x, s);
  s = fma((double)v.y, (double)v.y, s);
  s = fma((double)v.z, (double)v.z, s);
  s = fma((double)v.w, (double)v.w, s);
}

// elements of p ahead of the next 16-byte place, at most n
template <typename T>
PG_DEV int ahead(const T* p, int n) {
  return min(n, (int)(((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T)));
}

template <typename T>
PG_DEV double piece_sum(const T* p, int n) {
  const int tid = threadIdx.x, h = ahead(p, n), V = 16 / sizeof(T), nv = (n - h) / V;
  double s = 0.0;
  for (int i = tid; i < h; i += 256) {
    const double v = ld<T>(p, i);
    s = fma(v, v, s);
  }
#pragma unroll 4
  for (int i = tid; i < nv; i += 256) {
    if constexpr (sizeof(T) == 2) square8(reinterpret_cast<const uint4*>(p + h)[i], s);
    else square4(reinterpret_cast<const float4*>(p + h)[i], s);
  }
  for (int i = h + nv * V + tid; i < n; i += 256) {
    const double v = ld<T>(p, i);
    s = fma(v, v, s);
  }
  return s;
}

__global__ __launch_bounds__(256) void k_clip_sum(const ClipPiece* plan, int64_t n_pieces, double* part) {
  __shared__ double sh[4];
  double s = 0.0;
  ClipPiece next = (int64_t)blockIdx.x < n_pieces ? plan[blockIdx.x] : ClipPiece{};
  for (int64_t i = blockIdx.x; i < n_pieces; i += gridDim.x) {
    const ClipPiece p = next;
    if (i + gridDim.x < n_pieces) next = plan[i + gridDim.x];
    s += p.bf16 ? piece_sum((const bf16_t*)p.src, p.n) : piece_sum((const float*)p.src, p.n);
  }
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = ((sh[0] + sh[1]) + sh[2]) + sh[3];
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool FAR, typename V>
PG_DEV V ld16(const V* p) {
  if constexpr (FAR) return __builtin_nontemporal_load(p);
  else return *p;
}
// Outputs are marked as not read again, so that the caches keep what the sum
// read last until it is met (158 M floats 371 -> 335 us).  Of more than the
// last cache level holds, what is read is marked too (312 us; 40 M bf16, which
// fit: 54 instead of 45).
template <typename T, bool FAR>
PG_DEV void piece_scale(const T* p, T* o, int n, float k) {
  const int tid = threadIdx.x, V = 16 / sizeof(T);
  // vectors where both lie alike
  const int h = (((uintptr_t)p ^ (uintptr_t)o) & 15) ? n : ahead(p, n), nv = (n - h) / V;
  for (int i = tid; i < h; i += 256) st<T>(o, i, ld<T>(p, i) * k);
#pragma unroll 4
  for (int i = tid; i < nv; i += 256) {
    if constexpr (sizeof(T) == 2) {
      float f[8];
      const u32x4 v = ld16<FAR>(reinterpret_cast<const u32x4*>(p + h) + i);
      unpack8(make_uint4(v.x, v.y, v.z, v.w), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= k;
      const uint4 w = pack8(f);
      __builtin_nontemporal_store((u32x4){w.x, w.y, w.z, w.w}, reinterpret_cast<u32x4*>(o + h) + i);
    } else {
      const f32x4 v = ld16<FAR>(reinterpret_cast<const f32x4*>(p + h) + i);
      __builtin_nontemporal_store((f32x4){v.x * k, v.y * k, v.z * k, v.w * k}, reinterpret_cast<f32x4*>(o + h) + i);
    }
  }
  for (int i = h + nv * V + tid; i < n; i += 256) st<T>(o, i, ld<T>(p, i) * k);
}

template <bool FAR>
__global__ __launch_bounds__(256) void k_clip_scale(const ClipPiece* plan, int64_t n_pieces, const double* part, int n_part,
                                                    float max_norm, float grad_scale, int in_place, float* norm) {
  __shared__ double sh[4];
  double s = 0.0;
  for (int i = threadIdx.x; i < n_part; i += 256) s += part[i];
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  s = (double)grad_scale * sqrt(((sh[0] + sh[1]) + sh[2]) + sh[3]);
  const float k = (float)((double)grad_scale * (s <= (double)max_norm ? 1.0 : (double)max_norm / s));
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    norm[0] = (float)s;
    norm[1] = k;
  }
  if (in_place && k == 1.f) return;
  // backwards: what the sum read last is the nearest
  ClipPiece next = (int64_t)blockIdx.x < n_pieces ? plan[n_pieces - 1 - blockIdx.x] : ClipPiece{};
  for (int64_t i = blockIdx.x; i < n_pieces; i += gridDim.x) {
    const ClipPiece p = next;
    if (i + gridDim.x < n_pieces) next = plan[n_pieces - 1 - i - gridDim.x];
    if (k == 1.f && p.src == p.dst) continue;
    if (p.bf16) piece_scale<bf16_t, FAR>((const bf16_t*)p.src, (bf16_t*)p.dst, p.n, k);
    else piece_scale<float, FAR>((const float*)p.src, (float*)p.dst, p.n, k);
  }
}

__global__ __launch_bounds__(256) void k_clip_flat(const float* g, int64_t n, double* part) {
  __shared__ double sh[4];
  double s = 0.0;
  constexpr int64_t per = kClipPiece / 4;
  for (int64_t i = blockIdx.x * per; i < n; i += gridDim.x * per) s += piece_sum(g + i, (int)min(per, n - i));
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = ((sh[0] + sh[1]) + sh[2]) + sh[3];
}
__global__ __launch_bounds__(256) void k_clip_factor(const double* part, int n, float max_norm, float* norm) {
  __shared__ double sh[4];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) s += part[i];
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x > 0) return;
  s = sqrt(((sh[0] + sh[1]) + sh[2]) + sh[3]);
  norm[0] = (float)s;
  norm[1] = s <= (double)max_norm ? 1.f : (float)((double)max_norm / s);
}

}  // namespace

void clip_flat(hipStream_t st, const float* g, int64_t n, float max_norm, float* norm, double* part) {
  const int grid = (int)std::min<int64_t>(cdiv(n, kClipPiece / 4), kClipFlatBlocks);
  ProfScope prof(st);
  hipLaunchKernelGGL(k_clip_flat, dim3(grid), dim3(256), 0, st, g, n, part);
  PG_LAUNCH_CHECK();
  hipLaunchKernelGGL(k_clip_factor, dim3(1), dim3(256), 0, st, part, grid, max_norm, norm);
  PG_LAUNCH_CHECK();
  prof.done_bytes("k_clip_flat", 4.0 * n);
}

size_t clip_ws_bytes() { return kBlocks * sizeof(double); }

void clip(hipStream_t st, int64_t n_pieces, double bytes, bool in_place, const void* plan, float max_norm,
          float grad_scale, float* norm, void* ws) {
  const int grid = (int)std::min<int64_t>(std::max<int64_t>(n_pieces, 1), kBlocks);
  const ClipPiece* p = (const ClipPiece*)plan;
  ProfScope prof(st);
  hipLaunchKernelGGL(k_clip_sum, dim3(grid), dim3(256), 0, st, p, n_pieces, (double*)ws);
  PG_LAUNCH_CHECK();
  hipLaunchKernelGGL(bytes > kCache ? k_clip_scale<true> : k_clip_scale<false>, dim3(grid), dim3(256), 0, st, p, n_pieces, (const double*)ws, grid, max_norm,
                     grad_scale, (int)in_place, norm);
  PG_LAUNCH_CHECK();
  prof.done_bytes("k_clip", 3.0 * bytes);
}

}  // namespace pg
