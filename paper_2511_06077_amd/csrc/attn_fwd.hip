// Forward over packed rows (see attn_fwd.h), and the joining of the chunks of
// both forwards.
#include "attn_fwd.h"

namespace stca {
namespace ops {

namespace {

template <typename T, int DH>
hipError_t forward_dh(const AttnArgs& a, int tiles, hipStream_t st) {
  if constexpr (DH < 128)
    if (tiles == 2) return launch_fwd<T, kRagged, DH, 2>(a, st);
  return launch_fwd<T, kRagged, DH, 1>(a, st);
}

// Partials of a row (target, head) joined, in an order that depends on their
// number and the call's number of rows (see merge_dh) alone: 16 lanes a row, DH / 16 features each, times kSplit lanes that
// take every kSplit-th chunk.
template <typename T, int DH, int kSplit>
__global__ __launch_bounds__(256) void attn_merge_kernel(const AttnArgs a, bool paged) {
  constexpr int NE = DH / 16, kRows = 16 / kSplit;
  __shared__ float part[kSplit > 1 ? 16 : 1][kSplit > 1 ? DH + 2 : 1];
  const int f0 = (threadIdx.x & 15) * NE, s = (threadIdx.x >> 4) % kSplit, slot = threadIdx.x >> 4;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + slot / kSplit;
  const int64_t t = row / a.H;
  int64_t first = 0, step = 0;
  int n = 0;
  if (row < a.n_tgt * a.H) {
    int lo = 0, hi = a.R;  // the request of target t
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.tgt_off[mid] <= t) lo = mid;
      else hi = mid;
    }
    int len;
    if (paged) len = min(max(a.lens[lo], 0), a.max_len);
    else len = clamp_off(a.hist_off[lo + 1], a.n_hist) - clamp_off(a.hist_off[lo], a.n_hist);
    if (len > a.chunk && part_rows(a, lo, t, row, first, step))
      n = min(a.max_chunks, (len + a.chunk - 1) / a.chunk);  // (else written by the attention itself)
  }
  float M = -INFINITY, L = 0.f, acc[NE] = {};
#pragma unroll 4
  for (int c = s; c < n; c += kSplit) {
    const int64_t at = c * step + first;
    const float m = a.part_ml[2 * at], l = a.part_ml[2 * at + 1], mn = fmaxf(M, m);
    const float f = m == -INFINITY ? (l != l ? l : 0.f) : exp2_fast(m - mn), keep = M == -INFINITY ? (L != L ? L : 0.f) : exp2_fast(M - mn);
    L = keep * L + f * l;
#pragma unroll
    for (int e = 0; e < NE; ++e) acc[e] = keep * acc[e] + f * a.part_o[at * DH + f0 + e];
    M = mn;
  }
  if constexpr (kSplit > 1) {
#pragma unroll
    for (int e = 0; e < NE; ++e) part[slot][f0 + e] = acc[e];
    if (f0 == 0) {
      part[slot][DH] = M;
      part[slot][DH + 1] = L;
    }
    __syncthreads();
    if (s != 0 || n == 0) return;
    for (int k = 1; k < kSplit; ++k) M = fmaxf(M, part[slot + k][DH]);
    L = 0.f;
#pragma unroll
    for (int e = 0; e < NE; ++e) acc[e] = 0.f;
    for (int k = 0; k < kSplit; ++k) {
      const float m = part[slot + k][DH], l = part[slot + k][DH + 1];
      const float f = m == -INFINITY ? (l != l ? l : 0.f) : exp2_fast(m - M);
      L += f * l;
#pragma unroll
      for (int e = 0; e < NE; ++e) acc[e] += f * part[slot + k][f0 + e];
    }
  } else if (n == 0) {
    return;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int64_t at = row * DH + f0;
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

// A row's DH features by 16 lanes, its chunks one after the other; where there are
// many chunks and too few rows to fill the card, by 16 times as many lanes, each
// with every 16th chunk (8 rows of 40 chunks 4.2 us for 5.8, 1536 of 10 9.5 for
// 10.6; but 2048 rows of 8 chunks 1.6 us more, 4096 4.6, 32768 40).
template <typename T, int DH>
hipError_t merge_dh(const AttnArgs& a, bool paged, hipStream_t st) {
  const int split = a.max_chunks >= 8 && a.n_tgt * a.H <= 1536 ? 16 : 1;
  const int64_t grid = ceil_div(a.n_tgt * a.H, 16 / split);
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  if (split == 16) attn_merge_kernel<T, DH, 16><<<static_cast<unsigned>(grid), 256, 0, st>>>(a, paged);
  else attn_merge_kernel<T, DH, 1><<<static_cast<unsigned>(grid), 256, 0, st>>>(a, paged);
  return hipGetLastError();
}

template <typename T>
hipError_t merge_t(const AttnArgs& a, bool paged, int dh, hipStream_t st) {
  return dh == 32 ? merge_dh<T, 32>(a, paged, st) : dh == 64 ? merge_dh<T, 64>(a, paged, st) : merge_dh<T, 128>(a, paged, st);
}

}  // namespace

// Row tiles of 16 a wave holds.  More read K and V less often, fewer leave room
// for a second wave on the SIMD: four of them are slower throughout (128 requests
// of 2048 packed rows, 64 targets, 8 heads of 32 features 155 us for 131, of 64 428
// for 183), and of 128 features two are (32 targets, 4 heads 278 for 163), except
// where a page's rows are converted or looked up once for both (one tile: 32 requests
// of 10240 8-bit rows, 32 targets, 4 heads 145 us for 126; 24 of 10240 bf16 rows, 16
// targets, 4 heads to a kv head 252 for 190).
int forward_tiles(int dtype, int dh, int max_rows, bool paged) {
  const int most = dtype == STCA_BF16 ? (dh == 128 && !paged ? 1 : 2) : (dh == 128 ? 1 : 2);
  return max_rows > 16 ? most : 1;
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
