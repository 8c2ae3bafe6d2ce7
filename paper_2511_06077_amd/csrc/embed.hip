// Rows from ids: out_i = scale sum_f T_f[id_f(i)], fp32 sums in the order of the
// fields, rounded once.  Bound by the rows' bytes.  A team of lanes takes a row,
// eight features a lane (16 bytes of bf16), and four rows at once, so that four
// rows of every field are on their way together.
#include "layer_ops.h"

namespace stca {
namespace layers {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 4;  // rows of a team at a time

template <typename T, typename O, int L>
__global__ __launch_bounds__(kThreads) void embed_kernel(const EmbedArgs a) {
  constexpr int kTeams = kThreads / L;
  const int lane = threadIdx.x % L, team = threadIdx.x / L, octs = a.d / 8;
  bool bad = false;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * (kTeams * kRows); base < a.n;
       base += static_cast<int64_t>(gridDim.x) * (kTeams * kRows)) {
    for (int c = lane; c < octs; c += L) {
      float acc[kRows][8] = {};
      for (int f = 0; f < a.n_fields; ++f) {
        const T* table = static_cast<const T*>(a.table[f]) + 8 * c;
        Oct<T> v[kRows];
        bool have[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
          const int64_t i = base + k * kTeams + team;
          const int32_t id = i < a.n ? a.ids[f][i] : -1;
          have[k] = id >= 0 && static_cast<uint32_t>(id) < a.n_rows[f];
          bad |= id >= 0 && !have[k];
          v[k].zero();
          if (have[k]) v[k].load(table + static_cast<int64_t>(id) * a.ld[f]);
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
          float x[8];
          v[k].get(x);
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[k][e] += x[e];
        }
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int64_t i = base + k * kTeams + team;
        if (i >= a.n) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[k][e] *= a.scale;
        Oct<O>::store(static_cast<O*>(a.out) + i * a.ldo + 8 * c, acc[k]);
      }
    }
  }
  if (bad && a.hdr) a.hdr->status = STCA_ERR_INVALID_ARG;  // (every writer writes the same)
}

template <typename T, typename O, int L>
hipError_t launch(const EmbedArgs& a, int n_cu, hipStream_t st) {
  const int64_t per = kThreads / L * kRows;
  const int64_t grid = std::min<int64_t>(ceil_div(a.n, per), 32 * static_cast<int64_t>(n_cu));
  embed_kernel<T, O, L><<<static_cast<unsigned>(grid), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T, typename O>
hipError_t lanes(const EmbedArgs& a, int n_cu, hipStream_t st) {
  const int octs = a.d / 8;
  if (octs <= 4) return launch<T, O, 4>(a, n_cu, st);
  if (octs <= 8) return launch<T, O, 8>(a, n_cu, st);
  if (octs <= 16) return launch<T, O, 16>(a, n_cu, st);
  if (octs <= 32) return launch<T, O, 32>(a, n_cu, st);
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
