// Internal interface of the stand-alone attention operators (stca_attn_*,
// stca_cache_*): kernel arguments, launchers and the device code that the
// forward and the backward share (buckets of distance, the tanh cap, finding a
// workgroup's request).
#pragma once

#include <atomic>

#include "common.h"

namespace stca {
namespace ops {

constexpr int kMaxBuckets = 128;
constexpr int kMaxGroup = 64;     // query heads per kv head
constexpr int kWaves = 4;         // waves per workgroup of the attention kernels
constexpr int kThreads = 64 * kWaves;
constexpr int kChunkStep = 256;   // chunk lengths are multiples of this: a chunk starts on a page
constexpr int kXcds = 8;          // workgroup i runs on XCD i % 8

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Buckets of distance, by value in the kernel arguments.  A distance's cell is
// its octave and next two bits; cell[] holds the bucket of the cell's lowest
// distance, from which the edges above it are walked (none or one, where edges
// are no closer than a quarter octave).
struct Buckets {
  int32_t n;                       // buckets; 0: no bias
  int32_t edges[kMaxBuckets];      // n - 1 ascending, then INT32_MAX
  uint8_t cell[128];
};

struct AttnArgs {
  const void *q, *k, *v;           // ragged: rows of the batch; cache: q rows, K and V pages
  int64_t ldq, ldk, ldv;           // row strides in elements
  const int32_t *hist_off, *tgt_off;
  const int32_t *tgt_pos, *hist_pos;  // hist_pos of a cache: [page][slot]
  const float* bias;               // [H][n]
  // cache
  const uint8_t *ke, *ve;          // exponents [page][kv head][slot]
  const int32_t *table, *lens;
  int32_t table_ld, page_shift, n_pages, max_len;
  int32_t R, H, Hk, G;
  int32_t masked, placed;          // placed: distances are needed
  float scale, cap;
  int64_t n_hist, n_tgt;
  int32_t chunk, max_chunks, units, zgroups;
  // forward
  void* out;
  float *sa, *sm, *sl;             // saved (nullable): normalised output, score maximum, sum
  float *part_o, *part_ml;         // [max_chunks][n_tgt][H][dh], [max_chunks][n_tgt][H][2]
  // backward
  const void* dout;
  const float *fa, *fm, *fl;       // what the forward saved
  void *dq, *dk, *dv;
  int64_t lddq, lddk, lddv;
  float *dbias, *part_dq, *part_db, *acc_kv;
  WsHeader* hdr;
  Buckets b;
};

// ---- launchers (hipGetLastError of the launches)
hipError_t attn_forward(const AttnArgs& a, int dtype, int dh, int tiles, hipStream_t st);
hipError_t cache_attend(const AttnArgs& a, bool int8, int dh, int tiles, hipStream_t st);
hipError_t attn_merge(const AttnArgs& a, bool bf16, bool paged, int dh, hipStream_t st);
hipError_t attn_backward(const AttnArgs& a, int dtype, int dh, int tiles, hipStream_t st);

int forward_tiles(int dtype, int dh, int max_rows);  // row tiles of 16 a wave holds
int backward_tiles(int dtype, int dh, int need);      // ... of the `need` of a request

struct CacheArgs {
  void *k, *v;
  uint8_t *ke, *ve;
  int32_t* pos;                    // [page][slot]
  const void *xk, *xv;             // write: rows; read: destination
  const int32_t* xpos;
  int64_t ldk, ldv;
  const int32_t *row_off, *start, *table;
  int32_t table_ld, page_shift, n_pages, R, Hk;
  int64_t n_rows;
  WsHeader* hdr;                   // nullable
};
hipError_t cache_write(const CacheArgs& a, int dtype, bool int8, int dh, hipStream_t st);
hipError_t cache_read(const CacheArgs& a, int dtype, bool int8, int dh, hipStream_t st);



// Dynamic LDS beyond the default limit of a launch, granted once per kernel and
// device.
template <auto kernel>
hipError_t allow_lds(size_t bytes) {
  static std::atomic<int> granted[64];
  if (bytes <= 65536) return hipSuccess;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev >= 0 && dev < 64 && granted[dev] >= static_cast<int>(bytes)) return hipSuccess;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                          static_cast<int>(bytes));
  if (e == hipSuccess && dev >= 0 && dev < 64) granted[dev] = static_cast<int>(bytes);
  return e;
}

// ---- element types
template <typename T> struct Elem;
template <> struct Elem<bf16_bits> { static constexpr bool bf16 = true; };
template <> struct Elem<float> { static constexpr bool bf16 = false; };

__device__ __forceinline__ f32x4 mfma_bf16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 p = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
  return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Both terms of a two-term bf16 split of (a, b): hi is a rounded to 8
// significant bits, lo the rest rounded likewise, together 16 bits or more.
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = pack_bf16(a, b);
  lo = pack_bf16(a - lo_f32(hi), b - hi_f32(hi));
}

// exp(x) of a difference in natural units: the factor log2 e comes after the
// subtraction, so that scores of the type's lowest value still cancel.
__device__ __forceinline__ float exp_nat(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// tanh(x) to about 1e-7 relative: 1 - 2 / (e^2x + 1) away from zero, the odd
// series up to x^9 near it, where the difference would cancel.
__device__ __forceinline__ float tanh_fast(float x) {
  const float e = __builtin_amdgcn_exp2f(x * (2.f * kLog2e));
  const float far = 1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f);
  const float x2 = x * x;
  float p = fmaf(x2, 62.f / 2835.f, -17.f / 315.f);
  p = fmaf(x2, p, 2.f / 15.f);
  p = fmaf(x2, p, -1.f / 3.f);
  const float near = fmaf(x * x2, p, x);
  return fabsf(x) < 0.3f ? near : far;
}

__device__ __forceinline__ int sub_sat(int a, int b) { return __builtin_elementwise_sub_sat(a, b); }

// Buckets in LDS: edges, cells and the bias rows of a workgroup's heads.
struct BucketLds {
  const int32_t* edges;
  const uint8_t* cell;
  const float* bias;  // [heads of the workgroup][n]
  int n;
};

__device__ __forceinline__ int bucket_of(const BucketLds& b, int dist) {
  const uint32_t d = static_cast<uint32_t>(max(dist, 0));
  const int z = __clz(static_cast<int>(d | 1u));
  const uint32_t top = (d << z) >> 29;                 // 1xx (0 for d = 0)
  const int c = 4 * (31 - z) + static_cast<int>(top & 3u);
  int k = b.cell[c];
  while (static_cast<int>(d) >= b.edges[k] && k < b.n - 1) ++k;
  return k;
}

// The request of unit u: every request r holds the units from hist_off[r] /
// chunk + r on, one per chunk of its history and at least one.  64 candidates
// a step, so two steps for up to 4096 requests.
__device__ __forceinline__ int find_request(const int32_t* off, int R, int64_t n, int chunk, int u) {
  int lo = 0, n_left = R;  // answer in [lo, lo + n_left)
  const int lane = threadIdx.x & 63;
  while (n_left > 1) {
    const int stride = (n_left + 63) / 64;
    const int r = lo + lane * stride;
    bool le = false;
    if (lane * stride < n_left) {
      const uint32_t o = static_cast<uint32_t>(min<int64_t>(max(off[r], 0), n));
      le = o / static_cast<uint32_t>(chunk) + r <= static_cast<uint32_t>(u);
    }
    const int c = __popcll(__ballot(le));
    if (c == 0) return lo;
    lo += (c - 1) * stride;
    n_left = min(stride, n_left - (c - 1) * stride);
  }
  return lo;
}

__device__ __forceinline__ int clamp_off(int32_t v, int64_t n) {
  return static_cast<int>(min<int64_t>(max(v, 0), n));
}

__device__ __forceinline__ void set_status(WsHeader* hdr, int bad) {
  hdr->status = bad ? STCA_ERR_INVALID_ARG : STCA_OK;
  hdr->range = 0;
}

// The whole of a call's device offsets, lengths and pages as its status: one
// workgroup of its own, the only writer of the status word.
__device__ __forceinline__ void check_call(const AttnArgs& a, bool paged) {
  int bad = 0;
  for (int r = threadIdx.x; r < a.R; r += blockDim.x) {
    bad |= a.tgt_off[r + 1] < a.tgt_off[r] || (r == 0 && a.tgt_off[0] != 0) ||
           (r == a.R - 1 && a.tgt_off[a.R] != a.n_tgt);
    if (paged) {
      bad |= a.lens[r] < 0 || a.lens[r] > a.max_len;
    } else {
      bad |= a.hist_off[r + 1] < a.hist_off[r] || (r == 0 && a.hist_off[0] != 0) ||
             (r == a.R - 1 && a.hist_off[a.R] != a.n_hist);
    }
  }
  if (paged) {
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    for (int r = threadIdx.x >> 6; r < a.R; r += waves) {
      const int n = (min(max(a.lens[r], 0), a.max_len) + (1 << a.page_shift) - 1) >> a.page_shift;
      for (int i = lane; i < n; i += 64) {
        const int p = a.table[static_cast<int64_t>(r) * a.table_ld + i];
        bad |= p < 0 || p >= a.n_pages;
      }
    }
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) set_status(a.hdr, bad);
}

}  // namespace ops
}  // namespace stca
