// Forward over packed rows (see attn_fwd.h), and the joining of the chunks of
// both forwards.
#include "attn_fwd.h"

namespace stca {
namespace ops {

namespace {

// The fewest row tiles that hold a request's rows, up to what the registers
// take beside K and V (the output alone is DH / 16 x 4 registers a tile).
template <typename T, int DH> constexpr int kMaxTiles = Elem<T>::bf16 ? (DH == 128 ? 2 : 4) : (DH == 128 ? 1 : 2);

template <typename T, int DH>
hipError_t forward_dh(const AttnArgs& a, int tiles, hipStream_t st) {
  if constexpr (kMaxTiles<T, DH> >= 4)
    if (tiles == 4) return launch_fwd<T, kRagged, DH, 4>(a, st);
  if constexpr (kMaxTiles<T, DH> >= 2)
    if (tiles == 2) return launch_fwd<T, kRagged, DH, 2>(a, st);
  return launch_fwd<T, kRagged, DH, 1>(a, st);
}

// One row (target, head) per 16 lanes: partials of its request's chunks joined
// in chunk order.
template <typename T, int DH>
__global__ __launch_bounds__(256) void attn_merge_kernel(const AttnArgs a, bool paged) {
  constexpr int NE = DH / 16;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4);
  if (row >= a.n_tgt * a.H) return;
  const int64_t t = row / a.H;
  const int h = static_cast<int>(row % a.H), f0 = (threadIdx.x & 15) * NE;
  int lo = 0, hi = a.R;  // the request of target t
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.tgt_off[mid] <= t) lo = mid;
    else hi = mid;
  }
  int len;
  if (paged) len = min(max(a.lens[lo], 0), a.max_len);
  else len = clamp_off(a.hist_off[lo + 1], a.n_hist) - clamp_off(a.hist_off[lo], a.n_hist);
  if (len <= a.chunk) return;  // written by the attention itself
  const int n = min(a.max_chunks, (len + a.chunk - 1) / a.chunk);
  const int64_t step = a.n_tgt * a.H;
  float M = -INFINITY, L = 0.f, acc[NE] = {};
  for (int c = 0; c < n; ++c) M = fmaxf(M, a.part_ml[2 * (c * step + row)]);
  for (int c = 0; c < n; ++c) {
    const int64_t at = c * step + row;
    const float m = a.part_ml[2 * at], l = a.part_ml[2 * at + 1];
    const float f = m == -INFINITY ? (l != l ? l : 0.f) : exp2_fast(m - M);
    L += f * l;
#pragma unroll
    for (int e = 0; e < NE; ++e) acc[e] += f * a.part_o[at * DH + f0 + e];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int64_t at = (t * a.H + h) * DH + f0;
#pragma unroll
  for (int e = 0; e < NE; ++e) {
    const float y = acc[e] * inv;
    static_cast<T*>(a.out)[at + e] = from_f32<T>(y);
    if (a.sa) a.sa[at + e] = y;
  }
  if (a.sm && f0 == 0) {
    a.sm[row] = M;
    a.sl[row] = L;
  }
}

template <typename T>
hipError_t merge_t(const AttnArgs& a, bool paged, int dh, hipStream_t st) {
  const int64_t grid = ceil_div(a.n_tgt * a.H, 16);
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  if (dh == 32) attn_merge_kernel<T, 32><<<static_cast<unsigned>(grid), 256, 0, st>>>(a, paged);
  else if (dh == 64) attn_merge_kernel<T, 64><<<static_cast<unsigned>(grid), 256, 0, st>>>(a, paged);
  else attn_merge_kernel<T, 128><<<static_cast<unsigned>(grid), 256, 0, st>>>(a, paged);
  return hipGetLastError();
}

}  // namespace

int forward_tiles(int dtype, int dh, int max_rows) {
  const int most = dtype == STCA_BF16 ? (dh == 128 ? 2 : 4) : (dh == 128 ? 1 : 2);
  const int need = static_cast<int>(ceil_div(max_rows, 16));
  return need >= 4 && most == 4 ? 4 : need == 3 && most == 4 ? 4 : need >= 2 && most >= 2 ? 2 : 1;
}

hipError_t attn_forward(const AttnArgs& a, int dtype, int dh, int tiles, hipStream_t st) {
  if (dtype == STCA_BF16) {
    if (dh == 32) return forward_dh<bf16_bits, 32>(a, tiles, st);
    if (dh == 64) return forward_dh<bf16_bits, 64>(a, tiles, st);
    return forward_dh<bf16_bits, 128>(a, tiles, st);
  }
  if (dh == 32) return forward_dh<float, 32>(a, tiles, st);
  if (dh == 64) return forward_dh<float, 64>(a, tiles, st);
  return forward_dh<float, 128>(a, tiles, st);
}

hipError_t attn_merge(const AttnArgs& a, bool bf16, bool paged, int dh, hipStream_t st) {
  return bf16 ? merge_t<bf16_bits>(a, paged, dh, st) : merge_t<float>(a, paged, dh, st);
}

}  // namespace ops
}  // namespace stca
