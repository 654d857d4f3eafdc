// Global gradient norm and clipping over a table of chunks (gfx950).  The
// first kernel writes one partial sum of squares per block; every block of
// the second adds all partials in the same order, so that all use the same
// factor, and scales its chunks, from the last one.  Bound by memory: the
// gradients are read twice, since no factor is known before the last one is
// summed, and written once.  210 tensors of 160 million in fp32 and bf16 (1.07
// GB read once and written): 310 us, the floor of one reading 220; from the
// first chunk again instead of the last, 3 % more.  48 tensors of 11 million
// in fp32: 26 us, the floor 18.
#include "common.hpp"
#include "okernels.hpp"

namespace pulse {
namespace {

// 16 bytes as fp32 and back
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void get(uint4 w, float* v) {
    v[0] = __uint_as_float(w.x), v[1] = __uint_as_float(w.y);
    v[2] = __uint_as_float(w.z), v[3] = __uint_as_float(w.w);
  }
  __device__ static __forceinline__ uint4 put(const float* v) {
    return uint4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                 __float_as_uint(v[3])};
  }
  __device__ static __forceinline__ float one(float x) { return x; }
  __device__ static __forceinline__ float back(float x) { return x; }
};
template <>
struct Vec<uint16_t> {
  static constexpr int N = 8;
  __device__ static __forceinline__ void get(uint4 w, float* v) {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(x[i] << 16);
      v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
    }
  }
  __device__ static __forceinline__ uint4 put(const float* v) {
    return uint4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
  }
  __device__ static __forceinline__ float one(uint16_t x) { return bf2f(x); }
  __device__ static __forceinline__ uint16_t back(float x) { return f2bf(x); }
};

// A chunk is up to `head` elements before the first 16-byte boundary, whole
// 16-byte words, and a tail.
template <typename T>
struct Cut {
  int head, words;
  __device__ __forceinline__ explicit Cut(const ClipChunk& c) {
    const int off = (int)(reinterpret_cast<uintptr_t>(c.g) & 15) / (int)sizeof(T);
    head = min(c.n, off ? Vec<T>::N - off : 0);
    words = (c.n - head) / Vec<T>::N;
  }
  __device__ __forceinline__ int tail() const { return head + words * Vec<T>::N; }
};

// sum over the 256 threads, the same on every thread
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double w[4];
#pragma unroll
  for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s, 64);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = v;
  __syncthreads();
  return w[0] + w[1] + w[2] + w[3];
}

// Words in flight per thread.  48 tensors of 11 million in all: 26.9 us with
// one, 26.3 with two or four; 210 of 160 million: 340, 341 and 351.
constexpr int UN = 2;

// A result is not read here again: written past the caches, it leaves them to
// the gradients, which are (210 tensors of 160 million: 310 us, else 341).
__device__ __forceinline__ void put_past(uint4* p, uint4 w) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(u32x4{w.x, w.y, w.z, w.w}, reinterpret_cast<u32x4*>(p));
}

template <typename T>
__device__ __forceinline__ double squares(const ClipChunk& c) {
  const T* g = static_cast<const T*>(c.g);
  const Cut<T> k(c);
  double s = 0.;
  const auto add = [&](float x) { s = fma((double)x, (double)x, s); };
  if ((int)threadIdx.x < k.head) add(Vec<T>::one(g[threadIdx.x]));
  for (int i = k.tail() + threadIdx.x; i < c.n; i += 256) add(Vec<T>::one(g[i]));
  const uint4* p = reinterpret_cast<const uint4*>(g + k.head);
  int w = threadIdx.x;
  for (; w + 256 * (UN - 1) < k.words; w += 256 * UN) {
    uint4 q[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) q[u] = p[w + 256 * u];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      float v[Vec<T>::N];
      Vec<T>::get(q[u], v);
#pragma unroll
      for (int i = 0; i < Vec<T>::N; ++i) add(v[i]);
    }
  }
  for (; w < k.words; w += 256) {
    float v[Vec<T>::N];
    Vec<T>::get(p[w], v);
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) add(v[i]);
  }
  return s;
}

template <typename T>
__device__ __forceinline__ void scale(const ClipChunk& c, float f) {
  const T* g = static_cast<const T*>(c.g);
  T* o = static_cast<T*>(c.o);
  const Cut<T> k(c);
  if ((int)threadIdx.x < k.head) o[threadIdx.x] = Vec<T>::back(Vec<T>::one(g[threadIdx.x]) * f);
  for (int i = k.tail() + threadIdx.x; i < c.n; i += 256) o[i] = Vec<T>::back(Vec<T>::one(g[i]) * f);
  const uint4* p = reinterpret_cast<const uint4*>(g + k.head);
  const auto turn = [&](uint4 w) {
    float v[Vec<T>::N];
    Vec<T>::get(w, v);
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) v[i] *= f;
    return Vec<T>::put(v);
  };
  T* d = o + k.head;
  if (reinterpret_cast<uintptr_t>(d) & 15) {
    // the output is aligned otherwise: element by element
    for (int i = threadIdx.x; i < k.words * Vec<T>::N; i += 256)
      d[i] = Vec<T>::back(Vec<T>::one(g[k.head + i]) * f);
    return;
  }
  uint4* q = reinterpret_cast<uint4*>(d);
  int w = threadIdx.x;
  for (; w + 256 * (UN - 1) < k.words; w += 256 * UN) {
    uint4 x[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) x[u] = p[w + 256 * u];
#pragma unroll
    for (int u = 0; u < UN; ++u) put_past(q + w + 256 * u, turn(x[u]));
  }
  for (; w < k.words; w += 256) put_past(q + w, turn(p[w]));
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
  // from the last chunk: what the sum read last is still in cache
  for (int c = count - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
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
