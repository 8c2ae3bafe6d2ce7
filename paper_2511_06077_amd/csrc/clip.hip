// The norm of many gradients together, and every one times min(1, max_norm /
// norm).  Squares are added, and the factor is applied, in fp64, so no finite
// gradient is too large or too small, and a result is rounded once, to its own type
// (bf16 below 2^-126: to fp32's smallest numbers before).  Two launches
// a list: sums of squares, one a workgroup, and the scaling, whose workgroups all
// add up the same sums in the same order.  Bound by the bytes: every gradient is
// read twice (the second time from the last-level cache as far as it holds them)
// and written once.
//
// A list travels in the kernel's arguments, kGradsPerLaunch tensors a launch, so a
// call needs no copy to the device and can be captured.
#include "layer_ops.h"

namespace stca {
namespace layers {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int64_t live_of(const Grad& t) {
  if (!t.count) return t.n;
  return min(t.n, static_cast<int64_t>(max(*t.count, 0)) * t.per);
}

__device__ __forceinline__ int tensor_of(const ClipArgs& a, int64_t piece) {
  int lo = 0, hi = a.n_t;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.t[mid].start <= piece) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int o = 32; o > 0; o /= 2) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) v += lds[w];
  return v;
}

// 16 bytes of a gradient.
template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int kN = 4;
  f32x4 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const f32x4*>(p); }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
  }
};
template <> struct Piece<bf16_bits> {
  static constexpr int kN = 8;
  Oct<bf16_bits> v;
  __device__ __forceinline__ void load(const bf16_bits* p) { v.load(p); }
  __device__ __forceinline__ void get(float* x) const { v.get(x); }
};

constexpr int kBatch = 4;  // loads of a thread on their way at a time

template <typename T>
__device__ __forceinline__ double squares(const T* g, int64_t n) {
  constexpr int N = Piece<T>::kN;
  double v[4] = {};
  int64_t done = 0;
  if ((reinterpret_cast<uintptr_t>(g) & 15u) == 0) {
    done = n / N * N;
    for (int64_t i0 = N * threadIdx.x; i0 < done; i0 += kBatch * N * kThreads) {
      Piece<T> p[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (i0 + k * N * kThreads < done) p[k].load(g + i0 + k * N * kThreads);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (i0 + k * N * kThreads >= done) break;
        float x[N];
        p[k].get(x);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e & 3] = fma(static_cast<double>(x[e]), static_cast<double>(x[e]), v[e & 3]);
      }
    }
  }
  for (int64_t i = done + threadIdx.x; i < n; i += kThreads) {
    const double x = to_f32(g[i]);
    v[0] = fma(x, x, v[0]);
  }
  return (v[0] + v[1]) + (v[2] + v[3]);
}

__global__ __launch_bounds__(kThreads) void sum_kernel(const ClipArgs a) {
  __shared__ double lds[kThreads / 64];
  double v = 0.;
  for (int64_t piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) {
    const Grad& t = a.t[tensor_of(a, piece)];
    const int64_t at = (piece - t.start) * kGradPiece, n = min<int64_t>(kGradPiece, live_of(t) - at);
    if (n <= 0) continue;
    v += t.flags & 1 ? squares(static_cast<const bf16_bits*>(t.g) + at, n) : squares(static_cast<const float*>(t.g) + at, n);
  }
  v = block_sum(v, lds);
  if (threadIdx.x == 0) a.part[blockIdx.x] = v;
}

// Past the caches: the next pass over the gradients finds these free of dirty lines
// (243 MB clipped into other buffers: 80 us, 77 so, and the sums of squares before
// them 66 and 44).
template <int N>
__device__ __forceinline__ void store(float* p, const float* x) {
#pragma unroll
  for (int e = 0; e < N; e += 4)
    __builtin_nontemporal_store(f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]}, reinterpret_cast<f32x4*>(p + e));
}
template <int N>
__device__ __forceinline__ void store(bf16_bits* p, const float* x) {
  typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
  words w;
#pragma unroll
  for (int e = 0; e < N / 2; ++e) w[e] = two_bf16(x[2 * e], x[2 * e + 1]);
  __builtin_nontemporal_store(w, reinterpret_cast<words*>(p));
}

// A product in fp64, as a float that rounds to O as the product does: for bf16 what
// fp32 has no bits for is gathered in the last one that it has, since rounded to
// fp32 the product may come to lie in the middle of two bf16 numbers.  (61.7 million
// bf16 elements into others: 41 us with and without.)
template <typename O>
__device__ __forceinline__ float narrow(double x) {
  if constexpr (sizeof(O) == 2) {
    uint64_t w = __builtin_bit_cast(uint64_t, x);
    constexpr uint64_t kLow = (uint64_t(1) << 29) - 1;
    w = (w & ~kLow) | (w & kLow ? kLow + 1 : 0);
    x = __builtin_bit_cast(double, w);
  }
  return static_cast<float>(x);
}

template <typename T, typename O>
__device__ __forceinline__ void scale_piece(const T* g, O* out, int64_t n, double f) {
  constexpr int N = Piece<T>::kN;
  int64_t done = 0;
  if (((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(out)) & 15u) == 0) {
    done = n / N * N;
    for (int64_t i0 = N * threadIdx.x; i0 < done; i0 += kBatch * N * kThreads) {
      Piece<T> p[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (i0 + k * N * kThreads < done) p[k].load(g + i0 + k * N * kThreads);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (i0 + k * N * kThreads >= done) break;
        float x[N];
        p[k].get(x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = narrow<O>(x[e] * f);
        store<N>(out + i0 + k * N * kThreads, x);
      }
    }
  }
  for (int64_t i = done + threadIdx.x; i < n; i += kThreads) out[i] = from_f32<O>(narrow<O>(to_f32(g[i]) * f));
}

__global__ __launch_bounds__(kThreads) void scale_kernel(const ClipArgs a) {
  __shared__ double lds[kThreads / 64];
  double v = 0.;
#pragma unroll 4
  for (int i = threadIdx.x; i < a.n_part; i += kThreads) v += a.part[i];
  const double norm = sqrt(block_sum(v, lds));
  // (a norm that is not finite leaves everything as it is)
  const double f = norm > a.max_norm && norm < INFINITY ? a.max_norm / norm : 1.;
  if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = static_cast<float>(norm);
  for (int64_t piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) {
    const Grad& t = a.t[tensor_of(a, piece)];
    if (!t.out || (f == 1. && t.out == t.g)) continue;
    const int64_t at = (piece - t.start) * kGradPiece, n = min<int64_t>(kGradPiece, live_of(t) - at);
    if (n <= 0) continue;
    if (t.flags & 1) {
      const bf16_bits* g = static_cast<const bf16_bits*>(t.g) + at;
      if (t.flags & 2) scale_piece(g, static_cast<bf16_bits*>(t.out) + at, n, f);
      else scale_piece(g, static_cast<float*>(t.out) + at, n, f);
    } else {
      const float* g = static_cast<const float*>(t.g) + at;
      if (t.flags & 2) scale_piece(g, static_cast<bf16_bits*>(t.out) + at, n, f);
      else scale_piece(g, static_cast<float*>(t.out) + at, n, f);
    }
  }
}

}  // namespace

hipError_t clip_sum(const ClipArgs& a, int grid, hipStream_t st) {
  sum_kernel<<<grid, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t clip_scale(const ClipArgs& a, int grid, hipStream_t st) {
  scale_kernel<<<grid, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace layers
}  // namespace stca
