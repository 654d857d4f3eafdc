// Global gradient norm and clipping over a table of chunks (gfx950).  The
// first kernel writes one partial sum of squares per block; every block of
// the second adds all partials in the same order, so that all use the same
// factor, and scales its chunks.  Bound by memory: the gradients are read
// twice and written once.
#include "common.hpp"
#include "okernels.hpp"

namespace pulse {
namespace {

__device__ __forceinline__ float get(const float* p, int i) { return p[i]; }
__device__ __forceinline__ float get(const uint16_t* p, int i) { return bf2f(p[i]); }
__device__ __forceinline__ void set(float* p, int i, float v) { p[i] = v; }
__device__ __forceinline__ void set(uint16_t* p, int i, float v) { p[i] = f2bf(v); }

// sum over the 256 threads, the same on every thread
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double w[4];
#pragma unroll
  for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s, 64);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = v;
  __syncthreads();
  return w[0] + w[1] + w[2] + w[3];
}

template <typename T>
__device__ __forceinline__ double squares(const ClipChunk& c) {
  const T* g = static_cast<const T*>(c.g);
  double s = 0.;
  for (int i = threadIdx.x; i < c.n; i += 256) {
    const double v = get(g, i);
    s = fma(v, v, s);
  }
  return s;
}

template <typename T>
__device__ __forceinline__ void scale(const ClipChunk& c, float f) {
  const T* g = static_cast<const T*>(c.g);
  T* o = static_cast<T*>(c.o);
  for (int i = threadIdx.x; i < c.n; i += 256) set(o, i, get(g, i) * f);
}

__global__ __launch_bounds__(256) void k_clip_sum(const ClipChunk* chunks, int count,
                                                  double* part) {
  double s = 0.;
  for (int c = blockIdx.x; c < count; c += gridDim.x) {
    const ClipChunk k = chunks[c];
    s += k.dtype == PULSE_BF16 ? squares<uint16_t>(k) : squares<float>(k);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void k_clip_scale(const ClipChunk* chunks, int count,
                                                    const double* part, int parts, float max_norm,
                                                    float eps, float* norm) {
  double s = 0.;
  for (int i = threadIdx.x; i < parts; i += 256) s += part[i];
  const float n = (float)sqrt(block_sum(s));
  if (blockIdx.x == 0 && threadIdx.x == 0) norm[0] = n;
  const float r = max_norm / (n + eps);
  const float f = r > 1.f ? 1.f : r;  // NaN stays
  for (int c = blockIdx.x; c < count; c += gridDim.x) {
    const ClipChunk k = chunks[c];
    if (f == 1.f && k.g == k.o) continue;
    if (k.dtype == PULSE_BF16)
      scale<uint16_t>(k, f);
    else
      scale<float>(k, f);
  }
}

}  // namespace

hipError_t launch_clip(const ClipChunk* chunks, int count, double* part, float max_norm, float eps,
                       float* norm, hipStream_t st) {
  const int blocks = count < 1 ? 1 : count < CLIP_BLOCKS ? count : CLIP_BLOCKS;
  hipLaunchKernelGGL(k_clip_sum, dim3(blocks), dim3(256), 0, st, chunks, count, part);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_clip_scale, dim3(blocks), dim3(256), 0, st, chunks, count, part, blocks,
                     max_norm, eps, norm);
  return hipGetLastError();
}

}  // namespace pulse
