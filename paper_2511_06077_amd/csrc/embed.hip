// Rows from ids: out_i = scale sum_f T_f[id_f(i)], fp32 sums in the order of the
// fields, rounded once.  Rows of the tables come through L2, which each XCD has for
// itself (a window of 524288 rows of 256 from three fp32 tables, 153 us: 1.6 GB
// through it, 0.38 read past it, some of that from the last-level cache, and 0.27
// written).  A team of lanes takes a row, 16 bytes of a table's row a lane, and
// several rows at once: first the ids of all of them and of up to four fields, then
// their rows, so that one look-up's latency is paid for many rows.
#include "layer_ops.h"

namespace stca {
namespace layers {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 4;  // rows of a team at a time (the window: 2 160 us, 4 153, 8 171)

// 16 bytes of a table's row: kN features.
template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int kN = 4;
  f32x4 v;
  __device__ __forceinline__ void zero() { v = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const f32x4*>(p); }
  __device__ __forceinline__ void add_to(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] += v[i];
  }
};
template <> struct Piece<bf16_bits> {
  static constexpr int kN = 8;
  Oct<bf16_bits> v;
  __device__ __forceinline__ void zero() { v.zero(); }
  __device__ __forceinline__ void load(const bf16_bits* p) { v.load(p); }
  __device__ __forceinline__ void add_to(float* x) const {
    float y[8];
    v.get(y);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] += y[i];
  }
};

// The rows are written past the caches, which keep the tables' rows: 153 us for the
// window, 167 otherwise.
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

// kF: fields whose ids are loaded together; all of them, or four of more.
template <typename T, typename O, int L, int kF>
__global__ __launch_bounds__(kThreads) void embed_kernel(const EmbedArgs a) {
  constexpr int kTeams = kThreads / L, W = Piece<T>::kN;
  const int lane = threadIdx.x % L, team = threadIdx.x / L;
  bool bad = false;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * (kTeams * kRows); base < a.n;
       base += static_cast<int64_t>(gridDim.x) * (kTeams * kRows)) {
    for (int col = W * lane; col < a.d; col += W * L) {
      float acc[kRows][W] = {};
      for (int f0 = 0; f0 < a.n_fields; f0 += kF) {
        int32_t id[kF][kRows];
#pragma unroll
        for (int f = 0; f < kF; ++f)
#pragma unroll
          for (int k = 0; k < kRows; ++k) {
            const int64_t i = base + k * kTeams + team;
            id[f][k] = i < a.n && (kF < 4 || f0 + f < a.n_fields) ? a.ids[f0 + f][i] : -1;
          }
#pragma unroll
        for (int f = 0; f < kF; ++f) {
          if (kF == 4 && f0 + f >= a.n_fields) break;
          const T* table = static_cast<const T*>(a.table[f0 + f]) + col;
          Piece<T> v[kRows];
#pragma unroll
          for (int k = 0; k < kRows; ++k) {
            const bool some = id[f][k] >= 0, have = some && static_cast<uint32_t>(id[f][k]) < a.n_rows[f0 + f];
            bad |= some && !have;
            v[k].zero();
            if (have) v[k].load(table + static_cast<int64_t>(id[f][k]) * a.ld[f0 + f]);
          }
#pragma unroll
          for (int k = 0; k < kRows; ++k) v[k].add_to(acc[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int64_t i = base + k * kTeams + team;
        if (i >= a.n) continue;
#pragma unroll
        for (int e = 0; e < W; ++e) acc[k][e] *= a.scale;
        store<W>(static_cast<O*>(a.out) + i * a.ldo + col, acc[k]);
      }
    }
  }
  if (bad && a.hdr) a.hdr->status = STCA_ERR_INVALID_ARG;  // (every writer writes the same)
}

template <typename T, typename O, int L>
hipError_t launch(const EmbedArgs& a, int n_cu, hipStream_t st) {
  const int64_t per = kThreads / L * kRows;
  const unsigned grid = static_cast<unsigned>(std::min<int64_t>(ceil_div(a.n, per), 32 * static_cast<int64_t>(n_cu)));
  switch (a.n_fields) {
    case 1: embed_kernel<T, O, L, 1><<<grid, kThreads, 0, st>>>(a); break;
    case 2: embed_kernel<T, O, L, 2><<<grid, kThreads, 0, st>>>(a); break;
    case 3: embed_kernel<T, O, L, 3><<<grid, kThreads, 0, st>>>(a); break;
    default: embed_kernel<T, O, L, 4><<<grid, kThreads, 0, st>>>(a);
  }
  return hipGetLastError();
}

template <typename T, typename O>
hipError_t lanes(const EmbedArgs& a, int n_cu, hipStream_t st) {
  const int pieces = a.d / Piece<T>::kN;
  if (pieces <= 8) return launch<T, O, 8>(a, n_cu, st);
  if (pieces <= 16) return launch<T, O, 16>(a, n_cu, st);
  if (pieces <= 32) return launch<T, O, 32>(a, n_cu, st);
  return launch<T, O, 64>(a, n_cu, st);
}

}  // namespace

hipError_t embed_forward(const EmbedArgs& a, int table_dtype, int out_dtype, int n_cu, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  if (table_dtype == STCA_BF16)
    return out_dtype == STCA_BF16 ? lanes<bf16_bits, bf16_bits>(a, n_cu, st) : lanes<bf16_bits, float>(a, n_cu, st);
  return out_dtype == STCA_BF16 ? lanes<float, bf16_bits>(a, n_cu, st) : lanes<float, float>(a, n_cu, st);
}

}  // namespace layers
}  // namespace stca
