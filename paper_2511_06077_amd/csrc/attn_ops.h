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
constexpr int kPageStep = 256;    // a cache's chunk lengths are multiples of this: a chunk starts on a page
constexpr int kXcds = 8;          // workgroup i runs on XCD i % 8

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Buckets of distance, by value in the kernel arguments.
struct Buckets {
  int32_t n;                       // buckets; 0: no bias
  int32_t multi;                   // a cell of the lookup holds several edges
  int32_t edges[kMaxBuckets];      // n - 1 ascending, then INT32_MAX
  uint8_t cell[512];               // bucket of each cell's lowest x (see below)
};

// The lookup of a bucket: with x = max(D + 1, 0), cell 0..495 is x's octave and
// next four bits (so the cells of up to 32 distances hold one each), and cell
// kHiddenCell is x = 0, a distance below 0.  An entry holds the bucket of the
// cell's lowest x and the first edge above it, which x > edge has passed.
constexpr int kCells = 497, kHiddenCell = 496;
inline __host__ __device__ int64_t cell_low(int c) {  // lowest x of cell c (rounded up)
  const int o = c >> 4;
  return ((static_cast<int64_t>(16 + (c & 15)) << o) + 15) >> 4;
}

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
  int32_t max_tgt;                 // most targets of a request that the launch takes
  int32_t part_tgt;                // partials: see part_row
  int32_t bufs;                    // backward: a workgroup's rows in LDS, 2 where there are several passes
  int32_t hw;                      // kv heads of a workgroup (1, 2 or 4): a wave has one, 4 / hw waves share it
  // forward
  void* out;
  float *sa, *sm, *sl;             // saved (nullable): normalised output, score maximum, sum
  float *part_o, *part_ml;         // [part rows][H][dh], [part rows][H][2]
  // backward
  const void* dout;
  const float *fa, *fm, *fl;       // what the forward saved
  void *dq, *dk, *dv;
  int64_t lddq, lddk, lddv;
  float *dbias, *part_dq, *part_db, *acc_kv;
  float* rows;                     // per target and head: maximum, 1 / sum, D, position (attn_bwd.hip)
  WsHeader* hdr;
  Buckets b;
};

// ---- launchers (hipGetLastError of the launches)
hipError_t attn_forward(const AttnArgs& a, int dtype, int dh, int tiles, hipStream_t st);
hipError_t cache_attend(const AttnArgs& a, bool int8, int dh, int tiles, hipStream_t st);
hipError_t attn_merge(const AttnArgs& a, bool bf16, bool paged, int dh, hipStream_t st);
hipError_t attn_backward(const AttnArgs& a, int dtype, int dh, int tiles, hipStream_t st);

// LDS of a workgroup in bytes, of the kMaxLds that a CU has.  Forward: the join's
// rows and flags, the cells, the edges, the biases of hw kv heads' groups, a chunk's pages.
constexpr size_t kMaxLds = 160 << 10;
inline size_t forward_lds(int dh, int hw, int G, int n, int64_t pages) {
  return 4 * (kWaves * 16 * (dh + 2) + kWaves + 2 * (kCells + 1) + kMaxBuckets +
              static_cast<size_t>(hw) * G * ((n > 1 ? n : 1) + 1) + pages);
}
size_t backward_lds(int dtype, int dh, int tiles, int bufs, int hw, int G, int n);

int forward_tiles(int dtype, int dh, int max_rows, bool paged);  // row tiles of 16 a wave holds
int backward_tiles(int dtype, int dh, int need, int G);  // ... of the `need` of a request's G heads

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

// The high halves of a and b as a pair of bf16.
__device__ __forceinline__ uint32_t high_halves(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
// Splits a and b into bf16 terms by cutting bits off: the first returned, the
// rest left in a and b.  Each term holds 8 significant bits, so three leave
// nothing of an fp32.  Where two are all, the second is rounded (pack_bf16): that
// leaves at most 2^-16 of a value, to either side; cut, it left up to 2^-15, always
// towards zero, and a sum of many weights was low by 2^-17 of it.
__device__ __forceinline__ uint32_t cut_bf16(float& a, float& b) {
  const uint32_t t = high_halves(a, b);
  a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
  b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
  return t;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// tanh(x) as 1 - 2 / (e^2x + 1), within 2e-7; where `fine`, also relative to
// small values: there the odd series up to x^9, since the difference cancels.
// A cap of up to kPlainCap turns 2e-7 into no more than the 2^-16 that two bf16
// terms leave of a weight: where the weights have two, it does without (a third
// of the cost).
constexpr float kPlainCap = 64.f;
__device__ __forceinline__ float tanh_fast(float x, bool fine) {
  const float e = exp2_fast(x * (2.f * kLog2e));
  const float far = fmaf(-2.f, __builtin_amdgcn_rcpf(e + 1.f), 1.f);
  if (!fine) return far;
  const float x2 = x * x;
  float p = fmaf(x2, 62.f / 2835.f, -17.f / 315.f);
  p = fmaf(x2, p, 2.f / 15.f);
  p = fmaf(x2, p, -1.f / 3.f);
  const float near = fmaf(x * x2, p, x);
  return fabsf(x) < 0.3f ? near : far;
}

__device__ __forceinline__ int sub_sat(int a, int b) { return __builtin_elementwise_sub_sat(a, b); }

// A workgroup's bucket tables in LDS: the cells, and per query head (`heads` from
// that of kv head g on) the biases in units of log2 e (a finite one stays finite).  Without a
// bias there is one bucket, of bias 0; the slot after the buckets is for what
// is hidden, minus infinity.
struct BucketLds {
  const int2* cells;  // {next edge, bucket}
  const float* bias;  // [heads][slots + 1]
  const int32_t* edges;
  int slots, multi;
};

__device__ __forceinline__ float scaled_bias(float b) {
  const float x = b * kLog2e;
  constexpr float top = 3.4028234663852886e38f;
  return fabsf(b) <= top ? fminf(fmaxf(x, -top), top) : x;
}

// Fills the tables (threads of the whole workgroup; a barrier follows).
__device__ __forceinline__ void fill_buckets(const AttnArgs& a, int g, int heads, int2* cells, float* bias, int32_t* edges) {
  const int n = a.b.n, slots = max(n, 1);
  for (int i = threadIdx.x; i < kCells; i += blockDim.x) {
    const int k = i == kHiddenCell && a.masked ? slots : a.b.cell[i];
    cells[i] = make_int2(k < slots - 1 ? a.b.edges[k] : 0x7fffffff, k);
  }
  for (int i = threadIdx.x; i < heads * (slots + 1); i += blockDim.x) {
    const int h = i / (slots + 1), k = i % (slots + 1);
    bias[i] = k < n ? scaled_bias(a.bias[(static_cast<int64_t>(g) * a.G + h) * n + k]) : k == slots ? -INFINITY : 0.f;
  }
  for (int i = threadIdx.x; i < slots; i += blockDim.x) edges[i] = a.b.edges[i];
}

// x of a distance and its cell
__device__ __forceinline__ int place_of(int tpos, int pos) {
  return max(__builtin_elementwise_add_sat(sub_sat(tpos, pos), 1), 0);
}
__device__ __forceinline__ int cell_of(int x) {
  const int z = x ? __builtin_clz(static_cast<uint32_t>(x)) : -1;
  return static_cast<int>((static_cast<uint32_t>(x) << (z & 31)) >> 27) - 16 * z + 480;
}
__device__ __forceinline__ int bucket_in(const BucketLds& b, int x, int2 cell) {
  int k = cell.y + (x > cell.x);
  if (b.multi && x > 0)
    while (k < b.slots - 1 && x > b.edges[k]) ++k;
  return k;
}
// A lane's rows may lie in two neighbouring buckets at most: `far` for distances
// from `edge` on, else `near`.  Tells whether they do, from their least and
// greatest x; one look-up each instead of one a row.
struct TwoBuckets {
  int near, far, edge;
};
__device__ __forceinline__ bool two_buckets(const BucketLds& b, int xmin, int xmax, TwoBuckets& t) {
  const int2 cn = b.cells[cell_of(xmin)], cf = b.cells[cell_of(xmax)];
  t.near = bucket_in(b, xmin, cn);
  t.far = bucket_in(b, xmax, cf);
  t.edge = t.far == t.near + 1 && t.near < b.slots ? b.edges[t.near] : -2147483647 - 1;
  // (hidden rows have the bucket after the last: all of them or none)
  return t.far == t.near || (t.far == t.near + 1 && t.far < b.slots);
}
// Distances (as x) of a bucket, for a lane that keeps it: none if it is hidden.
__device__ __forceinline__ void keep_bucket(const BucketLds& b, bool masked, int k, float bias, int& lo, int& hi) {
  lo = k > 0 && k < b.slots ? b.edges[k - 1] + 1 : masked ? 1 : 0;
  hi = k < b.slots - 1 ? b.edges[k] : 0x7fffffff;
  if (bias == -INFINITY) lo = 0x7fffffff, hi = 0;
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

// A value that is the same in every lane, in scalar registers (so that loads
// take it as their base).
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
typedef const __attribute__((address_space(1))) char* gptr;  // global memory
__device__ __forceinline__ gptr uniform(const void* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
  return reinterpret_cast<gptr>(static_cast<uint64_t>(hi) << 32 | lo);
}
template <typename V>
__device__ __forceinline__ V load_at(gptr base, uint32_t at) {
  return *reinterpret_cast<const __attribute__((address_space(1))) V*>(base + at);
}

__device__ __forceinline__ int clamp_off(int32_t v, int64_t n) {
  return static_cast<int>(min<int64_t>(max(v, 0), n));
}

// Partials of target t (of its request's from t0 on) and chunk c, which is unit u:
// a row a chunk and target of the batch, or, where that would be more (a few long
// histories among short ones), a row a unit and target of a request, part_tgt each.
template <typename Args>
__device__ __forceinline__ int64_t part_row(const Args& a, int c, int64_t u, int64_t t0, int64_t t) {
  return a.part_tgt ? u * a.part_tgt + (t - t0) : c * a.n_tgt + t;
}
// ... of the first chunk, for a row (target t, head) of request r, and how far apart
// its chunks' lie; false where offsets that are not the host's leave it none.
__device__ __forceinline__ bool part_rows(const AttnArgs& a, int r, int64_t t, int64_t row, int64_t& at, int64_t& step) {
  at = row;
  step = a.n_tgt * a.H;
  if (a.part_tgt) {
    const int64_t u = clamp_off(a.hist_off[r], a.n_hist) / a.chunk + r, in = t - clamp_off(a.tgt_off[r], a.n_tgt);
    if (in < 0 || in >= a.part_tgt) return false;
    at = (u * a.part_tgt + in - t) * a.H + row;
    step = static_cast<int64_t>(a.part_tgt) * a.H;
  }
  return true;
}

__device__ __forceinline__ void set_status(WsHeader* hdr, int bad) {
  hdr->status = bad ? STCA_ERR_INVALID_ARG : STCA_OK;
  hdr->range = 0;
}

// Entries [i0, i1) of request r's row of a table of pages, for a share of the
// threads: nonzero if one is outside the pages.
__device__ __forceinline__ int check_pages(const int32_t* table, int64_t row, int i0, int i1, int step, int n_pages) {
  int bad = 0;
#pragma unroll 4
  for (int i = i0; i < i1; i += step) {
    const int p = table[row + i];
    bad |= p < 0 || p >= n_pages;
  }
  return bad;
}

// The whole of a call's device offsets, lengths and pages as its status: one
// workgroup of its own, the only writer of the status word.  As many threads a
// request as there are (a wave a request took 0.3 us for each of them).  A
// request of more rows or targets than the host's offsets have, on which chunks,
// passes and the workspace were planned, is not taken whole: an error as well.
__device__ __forceinline__ void check_call(const AttnArgs& a, bool paged) {
  int bad = 0;
  const int per = max(1, static_cast<int>(blockDim.x) / a.R), sub = threadIdx.x % per;
  for (int r = threadIdx.x / per; r < a.R; r += blockDim.x / per) {
    bad |= a.tgt_off[r + 1] < a.tgt_off[r] || (r == 0 && a.tgt_off[0] != 0) ||
           (r == a.R - 1 && a.tgt_off[a.R] != a.n_tgt);
    bad |= static_cast<int64_t>(a.tgt_off[r + 1]) - a.tgt_off[r] > a.max_tgt;
    if (paged) {
      const int len = a.lens[r];
      bad |= len < 0 || len > a.max_len;
      const int n = (min(max(len, 0), a.max_len) + (1 << a.page_shift) - 1) >> a.page_shift;
      bad |= check_pages(a.table, static_cast<int64_t>(r) * a.table_ld, sub, n, per, a.n_pages);
    } else {
      bad |= a.hist_off[r + 1] < a.hist_off[r] || (r == 0 && a.hist_off[0] != 0) ||
             (r == a.R - 1 && a.hist_off[a.R] != a.n_hist);
      bad |= static_cast<int64_t>(a.hist_off[r + 1]) - a.hist_off[r] > static_cast<int64_t>(a.max_chunks) * a.chunk;
    }
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) set_status(a.hdr, bad);
}

}  // namespace ops
}  // namespace stca
