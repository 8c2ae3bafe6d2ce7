// Rows written into a paged K/V cache and read back.
//
// K pages are [page][kv head][slot][dh], V pages [page][kv head][dh][slot]:
// what the attention's matrix operands read in one piece each.  8-bit pages
// hold, per row and kv head, n = x / step rounded to nearest even within
// -127..127, step = 2^max(floor(log2 max|x|) - 6, -126), and the byte
// log2(step) + 127 beside them; a power of two makes every step of this exact
// but the one rounding, so any order of evaluation gives the same bytes.  A row
// with an infinity or a NaN gets the byte 255 and n = 0: it reads as NaN.
//
// One workgroup takes 64 consecutive slots (aligned, so they fill cache lines
// of V) of one request and up to 128 features' worth of kv heads (whole cache
// lines of the packed rows), four threads a row; V turns in LDS.  Both
// directions are bound by their bytes; with one head a workgroup they waited for
// the look-ups of request and pages instead (64 requests of 512 to 4096 8-bit
// rows of 8 heads of 32 features read back, 234 MB out of cold caches: 72 us, now
// 59, of which the bytes take 45).
#include <type_traits>

#include "attn_ops.h"

namespace stca {
namespace ops {

namespace {

constexpr int kSlots = 64;  // slots of a workgroup

struct Span {
  int r, p0, lo, hi;  // positions [lo, hi) of request r's cache, within [p0, p0 + kSlots)
  int64_t row;        // packed row of position 0
};

// Request r owns the units from row_off[r] / 64 + 2 r on: n rows touch at most
// n / 64 + 2 aligned blocks.
__device__ __forceinline__ bool find_span(const CacheArgs& a, int unit, Span& s) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.R;
  while (n > 1) {
    const int stride = (n + 63) / 64, r = lo + lane * stride;
    bool le = false;
    if (lane * stride < n) le = clamp_off(a.row_off[r], a.n_rows) / kSlots + 2 * static_cast<int64_t>(r) <= unit;
    const int c = __popcll(__ballot(le));
    if (c == 0) break;
    lo += (c - 1) * stride;
    n = min(stride, n - (c - 1) * stride);
  }
  s.r = lo;
  const int r0 = clamp_off(a.row_off[lo], a.n_rows), r1 = clamp_off(a.row_off[lo + 1], a.n_rows);
  const int64_t start = a.start[lo], b = unit - (r0 / kSlots + 2 * static_cast<int64_t>(lo));
  if (start < 0 || b < 0) return false;
  const int64_t p0 = (start / kSlots + b) * kSlots, end = start + (r1 - r0);
  if (p0 >= end || p0 + kSlots > 0x7fffffff) return false;
  s.p0 = static_cast<int>(p0);
  s.lo = static_cast<int>(max(p0, start));
  s.hi = static_cast<int>(min(end, p0 + kSlots));
  s.row = r0 - start;
  return s.lo < s.hi;
}

// Page of a position, -1 where the table has none.
__device__ __forceinline__ int page_of(const CacheArgs& a, int r, int pos) {
  const int i = pos >> a.page_shift;
  if (i >= a.table_ld) return -1;
  const int p = a.table[static_cast<int64_t>(r) * a.table_ld + i];
  return p < 0 || p >= a.n_pages ? -1 : p;
}

__device__ void check_rows(const CacheArgs& a) {
  if (!a.hdr) return;
  int bad = 0;
  const int per = max(1, static_cast<int>(blockDim.x) / a.R), sub = threadIdx.x % per;
  for (int r = threadIdx.x / per; r < a.R; r += blockDim.x / per) {
    const int o0 = a.row_off[r], o1 = a.row_off[r + 1];
    const int64_t start = a.start[r], end = start + o1 - o0;
    const bool odd = o1 < o0 || start < 0 || (r == 0 && o0 != 0) || (r == a.R - 1 && o1 != a.n_rows) ||
                     end > 0x7fffffff - kSlots;
    bad |= odd;
    if (odd || o1 == o0) continue;
    const int i0 = static_cast<int>(start >> a.page_shift), i1 = static_cast<int>((end - 1) >> a.page_shift) + 1;
    bad |= i1 > a.table_ld;
    bad |= check_pages(a.table, static_cast<int64_t>(r) * a.table_ld, i0 + sub, min(i1, a.table_ld), per, a.n_pages);
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) set_status(a.hdr, bad);
}

template <typename T, int N>
__device__ __forceinline__ void load_row(const T* p, float* x) {
  if constexpr (Elem<T>::bf16) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      const uint4 w = reinterpret_cast<const uint4*>(p)[i];
      const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[8 * i + 2 * k] = lo_f32(v[k]);
        x[8 * i + 2 * k + 1] = hi_f32(v[k]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const f32x4 v = reinterpret_cast<const f32x4*>(p)[i];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[4 * i + k] = v[k];
    }
  }
}

template <typename T, int N>
__device__ __forceinline__ void store_row(T* p, const float* x) {
  if constexpr (Elem<T>::bf16) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i)
      reinterpret_cast<uint4*>(p)[i] =
          make_uint4(pack_bf16(x[8 * i], x[8 * i + 1]), pack_bf16(x[8 * i + 2], x[8 * i + 3]),
                     pack_bf16(x[8 * i + 4], x[8 * i + 5]), pack_bf16(x[8 * i + 6], x[8 * i + 7]));
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) reinterpret_cast<f32x4*>(p)[i] = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
  }
}

// Step byte of a row spread over four threads.
template <int N>
__device__ __forceinline__ uint32_t step_byte(const float* x) {
  uint32_t top = 0;  // largest magnitude as bits: NaN above infinity above the finite
#pragma unroll
  for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
  if (top >= 0x7f800000u) return 255u;
  return static_cast<uint32_t>(max(static_cast<int>(top >> 23) - 6, 1));
}

__device__ __forceinline__ uint32_t quantise4(const float* x, uint32_t byte) {
  if (byte == 255u) return 0u;
  const float inv = __uint_as_float((254u - byte) << 23);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = static_cast<int>(fminf(fmaxf(rintf(x[i] * inv), -127.f), 127.f));
    w |= (static_cast<uint32_t>(n) & 0xffu) << (8 * i);
  }
  return w;
}

template <typename T, bool kInt8, int DH, int HB>
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheArgs a) {
  constexpr int N = DH / 4;  // elements of a thread and head
  using S = typename std::conditional<kInt8, uint8_t, uint16_t>::type;
  constexpr int kLd = kSlots + 16 / sizeof(S);  // V tile [HB DH][slots], 16-byte rows
  __shared__ __align__(16) S tile[HB * DH * kLd];
  if (blockIdx.x == gridDim.x - 1) {
    check_rows(a);
    return;
  }
  const int groups = a.Hk / HB, unit = static_cast<int>(blockIdx.x) / groups, g0 = static_cast<int>(blockIdx.x) % groups * HB;
  Span s;
  if (!find_span(a, unit, s)) return;
  const int slot = threadIdx.x >> 2, part = threadIdx.x & 3, pos = s.p0 + slot;
  const bool have = pos >= s.lo && pos < s.hi;
  const int page = have ? page_of(a, s.r, pos) : -1;
  const int P = 1 << a.page_shift, at = pos & (P - 1);
  float x[2][HB][N];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv)
#pragma unroll
    for (int h = 0; h < HB; ++h) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[kv][h][i] = 0.f;
      if (have)
        load_row<T, N>(static_cast<const T*>(kv ? a.xv : a.xk) + (s.row + pos) * (kv ? a.ldv : a.ldk) + (g0 + h) * DH +
                           part * N, x[kv][h]);
    }
#pragma unroll
  for (int h = 0; h < HB; ++h) {
    uint32_t byte[2];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      uint32_t w[kInt8 ? N / 4 : N / 2];
      if constexpr (kInt8) {
        byte[kv] = step_byte<N>(x[kv][h]);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) w[i] = quantise4(x[kv][h] + 4 * i, byte[kv]);
      } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) w[i] = pack_bf16(x[kv][h][2 * i], x[kv][h][2 * i + 1]);
      }
      if (kv == 0) {
        if (page >= 0) {
          uint32_t* p = reinterpret_cast<uint32_t*>(static_cast<S*>(a.k) +
                                                    ((static_cast<int64_t>(page) * a.Hk + g0 + h) * P + at) * DH + part * N);
          constexpr int W = sizeof(w) / 4;
#pragma unroll
          for (int i = 0; i < W / 2; ++i) reinterpret_cast<uint2*>(p)[i] = make_uint2(w[2 * i], w[2 * i + 1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          tile[(h * DH + part * N + i) * kLd + slot] = kInt8 ? static_cast<S>(w[i / 4] >> (8 * (i % 4)))
                                                             : static_cast<S>(w[i / 2] >> (16 * (i % 2)));
      }
    }
    if constexpr (kInt8)
      if (page >= 0 && part == 0) {
        const int64_t e = (static_cast<int64_t>(page) * a.Hk + g0 + h) * P + at;
        a.ke[e] = static_cast<uint8_t>(byte[0]);
        a.ve[e] = static_cast<uint8_t>(byte[1]);
      }
  }
  if (page >= 0 && part == 0 && g0 == 0 && a.pos && a.xpos) a.pos[static_cast<int64_t>(page) * P + at] = a.xpos[s.row + pos];
  __syncthreads();
  // V: 16 bytes of one feature's slots at a time (within one page), or the
  // slots that exist one by one
  constexpr int kRun = 16 / sizeof(S);
#pragma unroll 2
  for (int i = threadIdx.x; i < HB * DH * (kSlots / kRun); i += 256) {
    const int d = i / (kSlots / kRun), c = i % (kSlots / kRun) * kRun, p = s.p0 + c;
    const int pg = p < s.hi && p + kRun > s.lo ? page_of(a, s.r, p) : -1;
    if (pg < 0) continue;
    S* out = static_cast<S*>(a.v) + ((static_cast<int64_t>(pg) * a.Hk + g0) * DH + d) * P + (p & (P - 1));
    const S* in = tile + d * kLd + c;
    if (p >= s.lo && p + kRun <= s.hi) {
      *reinterpret_cast<uint4*>(out) = *reinterpret_cast<const uint4*>(in);
    } else {
      for (int k = 0; k < kRun; ++k)
        if (p + k >= s.lo && p + k < s.hi) out[k] = in[k];
    }
  }
}

template <typename T, bool kInt8, int DH, int HB>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheArgs a) {
  constexpr int N = DH / 4;
  using S = typename std::conditional<kInt8, uint8_t, uint16_t>::type;
  constexpr int kLd = kSlots + 16 / sizeof(S), W = N * static_cast<int>(sizeof(S)) / 4;
  __shared__ __align__(16) S tile[HB * DH * kLd];
  if (blockIdx.x == gridDim.x - 1) {
    check_rows(a);
    return;
  }
  const int groups = a.Hk / HB, unit = static_cast<int>(blockIdx.x) / groups, g0 = static_cast<int>(blockIdx.x) % groups * HB;
  Span s;
  if (!find_span(a, unit, s)) return;
  const int P = 1 << a.page_shift;
  constexpr int kRun = 16 / sizeof(S), kPieces = HB * DH * (kSlots / kRun), kMine = (kPieces + 255) / 256;
  // everything on its way first: V's pieces, then this thread's part of K's rows
  uint4 vq[kMine];
#pragma unroll
  for (int n = 0; n < kMine; ++n) {
    const int i = threadIdx.x + 256 * n, d = i / (kSlots / kRun), p = s.p0 + i % (kSlots / kRun) * kRun;
    const int pg = i < kPieces && p < s.hi && p + kRun > s.lo ? page_of(a, s.r, p) : -1;
    vq[n] = uint4{};
    if (pg >= 0)
      vq[n] = *reinterpret_cast<const uint4*>(static_cast<const S*>(a.v) +
                                              ((static_cast<int64_t>(pg) * a.Hk + g0) * DH + d) * P + (p & (P - 1)));
  }
  const int slot = threadIdx.x >> 2, part = threadIdx.x & 3, pos = s.p0 + slot;
  const bool have = pos >= s.lo && pos < s.hi;
  const int page = have ? page_of(a, s.r, pos) : -1;
  const int64_t row = (static_cast<int64_t>(max(page, 0)) * a.Hk + g0) * P + (pos & (P - 1));  // of head g0; others P on
  uint32_t kq[HB][W];
  uint8_t ke[HB], ve[HB];
#pragma unroll
  for (int h = 0; h < HB; ++h) {
    if (page >= 0) {
      const uint2* p = reinterpret_cast<const uint2*>(static_cast<const S*>(a.k) + (row + h * P) * DH + part * N);
#pragma unroll
      for (int i = 0; i < W / 2; ++i) {
        kq[h][2 * i] = p[i].x;
        kq[h][2 * i + 1] = p[i].y;
      }
      if constexpr (kInt8) {
        ke[h] = a.ke[row + h * P];
        ve[h] = a.ve[row + h * P];
      }
    }
  }
#pragma unroll
  for (int n = 0; n < kMine; ++n) {
    const int i = threadIdx.x + 256 * n;
    if (i < kPieces)
      *reinterpret_cast<uint4*>(tile + i / (kSlots / kRun) * kLd + i % (kSlots / kRun) * kRun) = vq[n];
  }
  float x[N];
  if (page >= 0) {
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      const float step = kInt8 ? __uint_as_float(static_cast<uint32_t>(ke[h]) << 23) : 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i)
        x[i] = kInt8 ? static_cast<float>(static_cast<int8_t>(kq[h][i / 4] >> (8 * (i % 4)))) * step
                     : __uint_as_float((kq[h][i / 2] >> (16 * (i % 2))) << 16);
      store_row<T, N>(static_cast<T*>(const_cast<void*>(a.xk)) + (s.row + pos) * a.ldk + (g0 + h) * DH + part * N, x);
    }
    if (a.pos && a.xpos && g0 == 0 && part == 0)
      const_cast<int32_t*>(a.xpos)[s.row + pos] = a.pos[static_cast<int64_t>(page) * P + (pos & (P - 1))];
  }
  __syncthreads();
  if (page >= 0) {
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      const float step = kInt8 ? __uint_as_float(static_cast<uint32_t>(ve[h]) << 23) : 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const S v = tile[(h * DH + part * N + i) * kLd + slot];
        x[i] = kInt8 ? static_cast<float>(static_cast<int8_t>(v)) * step : __uint_as_float(static_cast<uint32_t>(v) << 16);
      }
      store_row<T, N>(static_cast<T*>(const_cast<void*>(a.xv)) + (s.row + pos) * a.ldv + (g0 + h) * DH + part * N, x);
    }
  }
}

template <typename T, bool kInt8, int DH, int HB>
hipError_t launch(const CacheArgs& a, bool write, hipStream_t st) {
  const int64_t grid = (a.n_rows / kSlots + 2 * static_cast<int64_t>(a.R)) * (a.Hk / HB) + 1;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  if (write) cache_write_kernel<T, kInt8, DH, HB><<<static_cast<unsigned>(grid), 256, 0, st>>>(a);
  else cache_read_kernel<T, kInt8, DH, HB><<<static_cast<unsigned>(grid), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T, bool kInt8, int DH>
hipError_t heads(const CacheArgs& a, bool write, hipStream_t st) {
  if constexpr (DH == 32)
    if (a.Hk % 4 == 0) return launch<T, kInt8, DH, 4>(a, write, st);
  if constexpr (DH <= 64)
    if (a.Hk % 2 == 0) return launch<T, kInt8, DH, 2>(a, write, st);
  return launch<T, kInt8, DH, 1>(a, write, st);
}

template <typename T>
hipError_t move(const CacheArgs& a, bool int8, int dh, bool write, hipStream_t st) {
  if (int8) return dh == 32 ? heads<T, true, 32>(a, write, st) : dh == 64 ? heads<T, true, 64>(a, write, st) : heads<T, true, 128>(a, write, st);
  return dh == 32 ? heads<T, false, 32>(a, write, st) : dh == 64 ? heads<T, false, 64>(a, write, st) : heads<T, false, 128>(a, write, st);
}

}  // namespace

hipError_t cache_write(const CacheArgs& a, int dtype, bool int8, int dh, hipStream_t st) {
  return dtype == STCA_BF16 ? move<bf16_bits>(a, int8, dh, true, st) : move<float>(a, int8, dh, true, st);
}
hipError_t cache_read(const CacheArgs& a, int dtype, bool int8, int dh, hipStream_t st) {
  return dtype == STCA_BF16 ? move<bf16_bits>(a, int8, dh, false, st) : move<float>(a, int8, dh, false, st);
}

}  // namespace ops
}  // namespace stca
