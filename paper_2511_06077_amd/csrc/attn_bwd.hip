// Backward of the stand-alone target-to-history attention.  With w the softmax
// weights of the forward (from its saved maxima and sums), per (target t, head
// h, history row j):
//   dP = dout . v,  D = dout . out,  dx = w (dP - D)       -> dbias[h][bucket]
//   dz = dx (1 - (y / c)^2)                                 (c: the score cap)
//   dv_j += w dout,  dk_j += scale dz q,  dq_t += scale dz k_j
//
// One workgroup takes one chunk of one request's history for hw kv heads; 4 / hw
// of its four waves share a head, each with consecutive steps of 16 history rows
// (see attn_fwd.h).  A wave holds dK^T, dV^T of its step in registers while it
// goes through the pass's MT tiles of 16 targets (of one query head each), whose
// q and dout rows wait in LDS.  dq of a pass stays in registers over the whole
// chunk.  More tiles than MT are further passes over the chunk; a chunk is then
// one step a wave, whose K, V, dK and dV stay in registers from pass to pass
// (or, where that would make too many chunks, dK and dV of the passes so far
// wait in fp32 in the workspace, written and read by the same lanes).  So K, V
// are read and dK, dV written once, nothing is added in order of arrival, and
// gradients repeat bitwise.
//
// Scores are formed as S^T = K Q^T: a lane holds one target, column t = lane %
// 16, and rows j = 4 (lane / 16) + i, so that the target's constants and its
// bucket are a lane's own, and dz is the operand of the sum over j (dQ^T = K^T
// dz) as it stands.  The sums over t (dV^T = dout^T w, dK^T = q^T dz) need the
// other order: w and dz go through LDS, written four rows at a time and read
// with the transposing LDS read; K^T, q^T and dout^T likewise.
//
// w and dz enter the products as two bf16 terms each (16 significant bits, so
// the one rounding that is left is the output's).
//
// dbias: a lane sums the dx of its target in a register as long as its bucket
// (an interval of distances) covers its rows.  When a vote finds a lane outside,
// every score looks its bucket up, and the four of a lane go to LDS sums that
// belong to the lane (or to lanes that take turns), so that the order is fixed:
// in two sums where they lie in the first's and the last's bucket, else one by
// one.  (LDS float atomics in their place take a cycle a lane: 2.3 times the
// kernel's time, window of 256 requests with 32 buckets.)
//
// Of that window (16 targets, 2048 rows, 8 heads of 32) a call takes 290 us
// without bias, 1.4 times what its bytes take at a large copy's rate, and 392 to
// 400 with a mask and 32 buckets: the turns of the bucket sums in LDS.  Several
// passes wait for each other's barriers instead (48 requests, 4 heads of 64 to a kv
// head, 227 us; 3 barriers a pass for 5 and two passes' rows in LDS took 6% off).
#include <type_traits>

#include "attn_ops.h"
#include "ring.h"

namespace stca {
namespace ops {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma16_bf16(s16x4 a, s16x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, 0, 0, 0);
}

// Operand over 16 of the summed axis, 4 per lane (index 4 (lane / 16) + i).
template <typename T> struct Four;
template <> struct Four<bf16_bits> { typedef s16x4 type; };
template <> struct Four<float> { typedef f32x4 type; };

// Eight consecutive features of a row.
template <typename T> struct Eight;
template <> struct Eight<bf16_bits> { bf16x8 v; };
template <> struct Eight<float> { f32x4 a, b; };

__device__ __forceinline__ f32x4 mma32(const Eight<bf16_bits>& a, const Eight<bf16_bits>& b, f32x4 c) {
  return mfma_bf16(a.v, b.v, c);
}
__device__ __forceinline__ f32x4 mma32(const Eight<float>& a, const Eight<float>& b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = mfma_f32(a.a[i], b.a[i], c);
#pragma unroll
  for (int i = 0; i < 4; ++i) c = mfma_f32(a.b[i], b.b[i], c);
  return c;
}
__device__ __forceinline__ f32x4 mma16(s16x4 a, s16x4 b, f32x4 c) { return mfma16_bf16(a, b, c); }
__device__ __forceinline__ f32x4 mma16(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = mfma_f32(a[i], b[i], c);
  return c;
}
template <typename T>
__device__ __forceinline__ Eight<T> load8(const T* p) {
  Eight<T> r;
  if constexpr (Elem<T>::bf16) {
    r.v = *reinterpret_cast<const bf16x8*>(p);
  } else {
    r.a = reinterpret_cast<const f32x4*>(p)[0];
    r.b = reinterpret_cast<const f32x4*>(p)[1];
  }
  return r;
}
template <typename T>
__device__ __forceinline__ Eight<T> load8_at(gptr p, uint32_t at) {
  Eight<T> r;
  if constexpr (Elem<T>::bf16) {
    r.v = load_at<bf16x8>(p, at);
  } else {
    r.a = load_at<f32x4>(p, at);
    r.b = load_at<f32x4>(p + 16, at);
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const Eight<T>& r) {
  if constexpr (Elem<T>::bf16) {
    *reinterpret_cast<bf16x8*>(p) = r.v;
  } else {
    reinterpret_cast<f32x4*>(p)[0] = r.a;
    reinterpret_cast<f32x4*>(p)[1] = r.b;
  }
}
template <typename T>
__device__ __forceinline__ bool odd8(const Eight<T>& r) {  // a value is not finite
  bool odd = false;
  if constexpr (Elem<T>::bf16) {
    const uint4 w = __builtin_bit_cast(uint4, r.v);
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) odd |= (v[i] & 0x7f80u) == 0x7f80u || (v[i] & 0x7f800000u) == 0x7f800000u;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      odd |= (__float_as_uint(r.a[i]) & 0x7f800000u) == 0x7f800000u || (__float_as_uint(r.b[i]) & 0x7f800000u) == 0x7f800000u;
  }
  return odd;
}

// A row-major LDS tile of rows of DH elements of T (rows padded by 16 bytes:
// 16 lanes' 16-byte reads then fall on different banks).
template <typename T, int DH> constexpr int kRowBytes = DH * static_cast<int>(sizeof(T)) + 16;

// Feature e of lane index m (0..15) of operand tile e: with the four features
// of a lane group's result rows consecutive over the tiles, a lane ends up with
// DH / 4 consecutive features.
template <int DH>
__device__ __forceinline__ int tile_feature(int e, int m) { return 4 * ((DH / 16) * (m >> 2) + e) + (m & 3); }

// Operand over the rows 4 g4 .. + 3 of a tile starting at `row0`, feature
// tile_feature(e, c16): column c16 of the 4 x 16 block.
template <typename T, int DH>
__device__ __forceinline__ typename Four<T>::type column4(const unsigned char* tile, int row0, int e, int c16, int g4) {
  if constexpr (Elem<T>::bf16) {
    return __builtin_bit_cast(s16x4, lds_read_tr16(tile + (row0 + 4 * g4 + (c16 >> 2)) * kRowBytes<T, DH> +
                                                   2 * 4 * ((DH / 16) * (c16 & 3) + e)));
  } else {
    f32x4 r;
    const float* p = reinterpret_cast<const float*>(tile + (row0 + 4 * g4) * kRowBytes<T, DH>) + tile_feature<DH>(e, c16);
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = p[i * (kRowBytes<T, DH> / 4)];
    return r;
  }
}

template <typename T>
__device__ __forceinline__ bool odd16(const uint4& w) {  // a value of 16 bytes is not finite
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) odd |= (v[i] & 0x7f800000u) == 0x7f800000u || (Elem<T>::bf16 && (v[i] & 0x7f80u) == 0x7f80u);
  return odd;
}

// Elements of x whose bit in h is set are cleared.
__device__ __forceinline__ s16x4 cleared(s16x4 x, uint32_t h) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = (h >> i) & 1 ? static_cast<short>(0) : x[i];
  return x;
}
__device__ __forceinline__ f32x4 cleared(f32x4 x, uint32_t h) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = (h >> i) & 1 ? 0.f : x[i];
  return x;
}

// Bytes of a target's row in the tiles of w and dz: bf16 4 terms of 16 rows,
// fp32 2 of 16 and a pad.
template <typename T> constexpr int kPRow = Elem<T>::bf16 ? 4 * 32 + 16 : 2 * 64 + 16;

// LDS of a workgroup, in bytes.
template <typename T, int DH, int MT>
struct BwdLds {
  static constexpr int kHead = 16 * MT * (2 * kRowBytes<T, DH> + 16);  // per head of the pass: q rows, dout rows,
  static constexpr int kDo = 16 * MT * kRowBytes<T, DH>;               // and per row maximum, 1 / sum, D, position
  static constexpr int kRow = 2 * kDo;
  static constexpr int kK = 0;                                       // per wave: K rows of the step
  static constexpr int kKWave = 16 * kRowBytes<T, DH>;
  static constexpr int kDz = kK + kWaves * kKWave;                   // per wave: w and dz tiles, both terms
  static constexpr int kDzWave = 16 * kPRow<T>;
  static constexpr int kComb = 0;                                    // dq of the waves, between passes
  static constexpr int kSteps = kDz + kWaves * kDzWave, kJoin = kWaves * 16 * (DH + 4) * 4;
  static constexpr int kTables = kSteps > kJoin ? kSteps : kJoin;    // heads (twice for several passes), flags, cells, edges, biases, bins
  static constexpr int kFlags = 2 * kWaves * 4;  // of a pass (two at a time) and wave: a row is not finite
  static size_t bytes(int bufs, int hw, int G, int n, int copies) {
    const size_t slots = n > 1 ? n : 1, heads = static_cast<size_t>(hw) * G;
    return kTables + bufs * hw * kHead + kFlags + 8 * (kCells + 1) +
           4 * (kMaxBuckets + (heads * (slots + 1) + 3) / 4 * 4 + (n ? kWaves * (slots + 1) * copies : 0));
  }
};

// Lanes of a wave that have dbias sums of their own: all while the four waves'
// sums stay within 36 KB, else every second or fourth, which then take turns.
inline __host__ __device__ int bin_copies(int n) { return n <= 34 ? 64 : n <= 70 ? 32 : 16; }

// Waves a SIMD is to hold: what the registers allow with few spills (128 requests
// of 2048 rows, 48 targets, 8 heads of 64, 4 tiles: two 376 us, one 514), and no more
// than two, since the workgroups of a chunk's heads, which read parts of the same
// DRAM pages, drift apart the more of them run (window of 256 requests, 16
// targets, 2048 rows, 8 heads of 32: one 366 us, two 288, three 327, four 363).
template <typename T, int DH, int MT> constexpr int kBwdWaves = DH == 128 ? 1 : 2;
template <typename T, int DH, int MT> constexpr int kBwdMost = kBwdWaves<T, DH, MT> == 1 ? 8 : 2;

// The kernel's arguments, `kFresh`: as loads that are not moved out of a loop.
// Kept from pass to pass they take more scalar registers than there are (48
// requests, 4 heads of 64 to a kv head: 238 us for 227, without bias 149 for 141, of
// 128 455 for 342); with one pass the loads cost more (the window 400 us for 396).
typedef const __attribute__((address_space(4))) AttnArgs KernelArgs;
template <bool kFresh>
__device__ __forceinline__ decltype(auto) again(const AttnArgs& a) {
  if constexpr (kFresh) {
    uint64_t p = reinterpret_cast<uint64_t>(__builtin_amdgcn_kernarg_segment_ptr());  // (`a` is the only argument)
    asm volatile("" : "+s"(p));
    return *reinterpret_cast<KernelArgs*>(p);
  } else {
    return (a);
  }
}

constexpr int kStep = 16;  // history rows of a wave's step

template <typename T, int DH, int MT, bool kOnePass>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kBwdWaves<T, DH, MT>, kBwdMost<T, DH, MT>))) void attn_bwd_kernel(const AttnArgs a) {
  constexpr bool kBf16 = Elem<T>::bf16;
  constexpr int KS = DH / 32, NE = DH / 16;
  using F4 = typename Four<T>::type;
  using E8 = Eight<T>;
  using Lds = BwdLds<T, DH, MT>;
  extern __shared__ __align__(16) unsigned char smem[];
  const int nb = a.b.n;
  float* s_comb = reinterpret_cast<float*>(smem + Lds::kComb);
  const int slots = max(nb, 1), copies = bin_copies(nb);
  int* s_flags = reinterpret_cast<int*>(smem + Lds::kTables + a.bufs * a.hw * Lds::kHead);
  int2* s_cells = reinterpret_cast<int2*>(s_flags + 2 * kWaves);
  int32_t* s_edges = reinterpret_cast<int32_t*>(s_cells + kCells + 1);
  float* s_bias = reinterpret_cast<float*>(s_edges + kMaxBuckets);
  float* s_bins = s_bias + (a.hw * a.G * (slots + 1) + 3) / 4 * 4;

  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ghs = a.Hk / a.hw;
  const int unit = static_cast<int>(blockIdx.x) / kXcds / ghs * kXcds + static_cast<int>(blockIdx.x) % kXcds;
  if (unit >= a.units) return;
  const int g0 = static_cast<int>(blockIdx.x) / kXcds % ghs * a.hw;
  const int hs = wave % a.hw, part = wave / a.hw, parts = kWaves / a.hw, g = g0 + hs, heads = a.hw * a.G;
  const int r = uniform(find_request(a.hist_off, a.R, a.n_hist, a.chunk, unit));
  const int64_t h0 = uniform(clamp_off(a.hist_off[r], a.n_hist));
  const int len = uniform(max(0, static_cast<int>(clamp_off(a.hist_off[r + 1], a.n_hist) - h0)));
  const int c = unit - static_cast<int>(h0 / a.chunk + r);
  float* part_db = a.part_db + (static_cast<int64_t>(unit) * a.H + g0 * a.G) * nb;
  if (c < 0 || c >= a.max_chunks || (c > 0 && static_cast<int64_t>(c) * a.chunk >= len)) {
    for (int i = tid; i < heads * nb; i += kThreads) part_db[i] = 0.f;
    return;
  }
  const int j0 = c * a.chunk, j1 = j0 + min(len - j0, a.chunk);
  const int t0 = uniform(clamp_off(a.tgt_off[r], a.n_tgt)), m = min(max(0, uniform(clamp_off(a.tgt_off[r + 1], a.n_tgt)) - t0), a.max_tgt);
  const int ttiles = (m + 15) / 16, groups = (ttiles + MT - 1) / MT;  // groups of MT tiles of one head

  const BucketLds bl{s_cells, s_bias, s_edges, slots, a.b.multi};  // (pointers that are known to be LDS)
  if (a.placed) fill_buckets(a, g0, heads, s_cells, s_bias, s_edges);
  if (ttiles == 0)
    for (int i = tid; i < heads * nb; i += kThreads) part_db[i] = 0.f;
  unsigned char* kt = smem + Lds::kK + wave * Lds::kKWave;
  unsigned char* dzt = smem + Lds::kDz + wave * Lds::kDzWave;
  float* bins = s_bins + wave * (slots + 1) * copies;
  const float gain = kLog2e * (a.cap > 0.f ? a.cap : a.scale), cap_in = a.cap > 0.f ? a.scale / a.cap : 0.f;

  const int passes = kOnePass ? 1 : max(1, groups * a.G);
  const bool single = a.chunk <= kStep * parts;  // one step a wave
  f32x4 dk[NE], dv[NE];
  E8 kf[KS], vf[KS];  // the step's rows, or the next one's once they are used
  int pj[4];          // positions of rows 4 g4 + i
  const uint32_t lk = static_cast<uint32_t>(a.ldk * sizeof(T)), lv = static_cast<uint32_t>(a.ldv * sizeof(T));
  auto load = [&](const auto& a, int jb) {
    const int last = len - 1 - jb;
    const gptr kp = uniform(static_cast<const T*>(a.k) + (h0 + jb) * a.ldk + g * DH);
    const gptr vp = uniform(static_cast<const T*>(a.v) + (h0 + jb) * a.ldv + g * DH);
    const int jr = min(c16, last);
    const uint32_t ak = __umul24(jr, lk) + 8 * g4 * sizeof(T), av = __umul24(jr, lv) + 8 * g4 * sizeof(T);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      kf[s] = load8_at<T>(kp + 32 * s * sizeof(T), ak);
      vf[s] = load8_at<T>(vp + 32 * s * sizeof(T), av);
    }
    if (a.hist_pos) {
      const gptr hp = uniform(a.hist_pos + h0 + jb);
#pragma unroll
      for (int i = 0; i < 4; ++i) pj[i] = load_at<int>(hp, 4u * min(4 * g4 + i, last));
    }
  };
  // a pass's rows on their way to LDS, 16 bytes of q and of dout a thread
  constexpr int kPieces = DH * static_cast<int>(sizeof(T)) / 16;
  constexpr int kHeadsMost = MT < 4 ? 2 : 1;  // (heads a workgroup, see the host)
  constexpr int kFetch = (16 * MT * kHeadsMost * kPieces + kThreads - 1) / kThreads;
  uint4 fq[kFetch], fd[kFetch];
  f32x4 frow;
  const uint32_t lq = static_cast<uint32_t>(a.ldq * sizeof(T)), ldo = static_cast<uint32_t>(a.H * DH * sizeof(T));
  auto fetch = [&](const auto& a, int hh, int first) {
    const int64_t row0 = t0 + 16 * static_cast<int64_t>(first), head0 = g0 * a.G + hh;
    const int left = m - 16 * first;
    const gptr qp = uniform(static_cast<const T*>(a.q) + row0 * a.ldq + head0 * DH);
    const gptr dp = uniform(static_cast<const T*>(a.dout) + (row0 * a.H + head0) * DH);
#pragma unroll
    for (int n = 0; n < kFetch; ++n) {
      const int i = tid + n * kThreads, piece = i % kPieces, at = i / kPieces, hd = at / (16 * MT), row = at % (16 * MT);
      fq[n] = fd[n] = uint4{};
      if (hd < a.hw && m > 0) {
        const uint32_t in = hd * a.G * (DH * static_cast<int>(sizeof(T))) + 16 * piece, t = min(row, left - 1);
        fq[n] = __builtin_bit_cast(uint4, load_at<u32x4>(qp, __umul24(t, lq) + in));
        fd[n] = __builtin_bit_cast(uint4, load_at<u32x4>(dp, __umul24(t, ldo) + in));
      }
    }
    const int hd = tid / (16 * MT), row = tid % (16 * MT);
    // a row behind the last target is that target again without weight: of zeros,
    // its product with an infinite K would be NaN where no target's score is
    frow = f32x4{INFINITY, 0.f, 0.f, 0.f};
    if (hd < a.hw && m > 0) {
      const f32x4 x = load_at<f32x4>(uniform(a.rows + 4 * (row0 * a.H + head0)),
                                     16u * (__umul24(min(row, left - 1), a.H) + hd * a.G));
      frow = row < left ? x : f32x4{INFINITY, 0.f, 0.f, x[3]};
    }
  };
  fetch(a, 0, 0);
  if (nb)
    for (int i = 4 * tid; i < kWaves * (slots + 1) * copies; i += 4 * kThreads) *reinterpret_cast<f32x4*>(s_bins + i) = f32x4{};
  int hh = 0, first = 0;  // the pass's query head of the group and first tile
  const AttnArgs& once = a;
  for (int pass = 0; pass < passes; ++pass) {
    const auto& a = again<!kOnePass>(once);
    const int held = min(MT, ttiles - first);
    const bool last_of_head = first + MT >= ttiles;
    // one pass's rows are read while the next one's arrive
    const int buf = pass & (a.bufs - 1);
    unsigned char* rows = smem + Lds::kTables + buf * a.hw * Lds::kHead;
    int odd_rows = 0;
#pragma unroll
    for (int n = 0; n < kFetch; ++n) {
      const int i = tid + n * kThreads, piece = i % kPieces, at = i / kPieces, hd = at / (16 * MT), row = at % (16 * MT);
      if (hd < a.hw) {
        unsigned char* to = rows + hd * Lds::kHead + row * kRowBytes<T, DH> + 16 * piece;
        *reinterpret_cast<uint4*>(to) = fq[n];
        *reinterpret_cast<uint4*>(to + Lds::kDo) = fd[n];
        if (a.placed) odd_rows |= odd16<T>(fq[n]) || odd16<T>(fd[n]);
      }
    }
    if (tid < 16 * MT * a.hw)
      reinterpret_cast<f32x4*>(rows + tid / (16 * MT) * Lds::kHead + Lds::kRow)[tid % (16 * MT)] = frow;
    if (a.placed) {
      odd_rows = __ballot(odd_rows) != 0;
      if (lane == 0) s_flags[buf * kWaves + wave] = odd_rows;
    }
    if (!kOnePass && pass + 1 < passes) fetch(a, last_of_head ? hh + 1 : hh, last_of_head ? 0 : first + MT);
    __syncthreads();
    if (a.placed) {
      const int4 f = *reinterpret_cast<const int4*>(s_flags + buf * kWaves);
      odd_rows = f.x | f.y | f.z | f.w;
    }
    const unsigned char* mine = rows + hs * Lds::kHead;  // q, dout and rows of this wave's head
    const float* s_row = reinterpret_cast<const float*>(mine + Lds::kRow);

    // this lane's target of each tile: its constants, the bucket it keeps
    f32x4 dq[MT][NE];
    float mx[MT], il[MT], D[MT], bias[MT], dsum[MT];
    int tp[MT], blo[MT], bhi[MT], bk[MT];
    int seen_max = -2147483647 - 1;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int e = 0; e < NE; ++e) dq[mt][e] = f32x4{};
      const f32x4 row = *reinterpret_cast<const f32x4*>(s_row + 4 * (16 * mt + c16));
      mx[mt] = row[0];
      il[mt] = row[1];
      D[mt] = row[2];
      tp[mt] = __float_as_int(row[3]);
      bias[mt] = dsum[mt] = 0.f;
      bk[mt] = 0;
      blo[mt] = a.masked ? 1 : 0;
      bhi[mt] = nb ? -1 : 0x7fffffff;  // (a bias: none kept yet)
      if (mt < held) seen_max = max(seen_max, tp[mt]);
    }
    int jend = j1;  // rows from here on are hidden from every target of the pass
    if (a.masked && !a.hist_pos) {
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) seen_max = max(seen_max, __shfl_xor(seen_max, o));
      jend = static_cast<int>(min<int64_t>(jend, static_cast<int64_t>(seen_max) + 1));
      jend = __builtin_amdgcn_readfirstlane(jend);
    }
    if (held <= 0) jend = 0;

    // v to bucket k and u to bucket l of this lane's sums (l = -1: nothing); lanes
    // that share a sum take turns, each of which ends before the next one reads
    auto add_bins = [&](int k, float v, int l, float u) {
      if (l == k) {
        v += u;
        l = -1;
      }
      for (int turn = 0; turn < 64 / copies; ++turn) {
        if (lane / copies == turn) {
          float* p = bins + k * copies + lane % copies;
          float* q = bins + max(l, 0) * copies + lane % copies;
          const float x = *p, y = *q;
          *p = x + v;
          if (l >= 0) *q = y + u;
        }
        if (copies < 64) {
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
          __builtin_amdgcn_wave_barrier();
          __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
      }
    };

    // each wave takes consecutive steps (a lane's bucket changes seldom then)
    const int steps = (j1 - j0 + kStep - 1) / kStep, share = (steps + parts - 1) / parts;
    const int jfirst = j0 + part * share * kStep, jstop = min(j1, jfirst + share * kStep);
    if (jfirst < min(jstop, single ? j1 : jend) && (pass == 0 || !single)) load(a, jfirst);
    for (int jb = jfirst; jb < jstop; jb += kStep) {
      const int64_t acc_at = ((h0 + jb) * a.Hk + g) * DH;  // fp32 sums of the earlier passes: row c16
      const int64_t acc_v = a.n_hist * a.Hk * DH;
      if (pass == 0 || !single) {
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          dk[e] = dv[e] = f32x4{};
          if (pass > 0 && jb + c16 < j1) {
            const float* p = a.acc_kv + acc_at + static_cast<int64_t>(c16) * a.Hk * DH + 4 * (NE * g4 + e);
            dk[e] = *reinterpret_cast<const f32x4*>(p);
            dv[e] = *reinterpret_cast<const f32x4*>(p + acc_v);
          }
        }
      }
      if (jb < jend) {
        // K in the other order: rows of the step along the operand
        bool odd_k = false;
#pragma unroll
        for (int s = 0; s < KS; ++s)
          store8<T>(reinterpret_cast<T*>(kt + c16 * kRowBytes<T, DH>) + 32 * s + 8 * g4, kf[s]);
        f32x4 S[MT], dP[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          S[mt] = dP[mt] = f32x4{};
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            const unsigned char* row = mine + (16 * mt + c16) * kRowBytes<T, DH> + (32 * s + 8 * g4) * sizeof(T);
            const E8 qf = load8<T>(reinterpret_cast<const T*>(row));
            const E8 df = load8<T>(reinterpret_cast<const T*>(row + Lds::kDo));
            S[mt] = mma32(kf[s], qf, S[mt]);
            dP[mt] = mma32(vf[s], df, dP[mt]);
          }
        }
        const bool tail = jb + kStep > jend;
        int pos[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) pos[i] = a.hist_pos ? pj[i] : jb + 4 * g4 + i;
        if (a.placed) {
#pragma unroll
          for (int s = 0; s < KS; ++s) odd_k |= odd8<T>(kf[s]);
        }
        if (!single && jb + kStep < min(jstop, jend)) load(a, jb + kStep);
        F4 kc[NE];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < NE; ++e) kc[e] = column4<T, DH>(kt, 0, e, c16, g4);
        __builtin_amdgcn_wave_barrier();
        int pmin = pos[0], pmax = pos[0];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pmin = min(pmin, pos[i]);
          pmax = max(pmax, pos[i]);
        }

#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          if (mt >= held) break;
          const unsigned char* qt = mine + 16 * mt * kRowBytes<T, DH>;
          const unsigned char* dt = qt + Lds::kDo;
          const bool slow =
              __ballot(tail || (a.placed && (place_of(tp[mt], pmax) < blo[mt] || place_of(tp[mt], pmin) > bhi[mt]))) != 0;
          uint32_t hid = 0;  // bit i
          float w[4], dz[4], dx[4];
          // a lane's rows in two buckets at most, or each in its own
          int kk[4];
          TwoBuckets two{0, 0, 0};
          bool each = false;
          if (slow) {
            const float* hb = bl.bias + (hs * a.G + hh) * (slots + 1);
            if (a.placed) {
              each = __ballot(!two_buckets(bl, place_of(tp[mt], pmax), place_of(tp[mt], pmin), two)) != 0;
              if (!each) {
                const float near = hb[two.near], far = hb[two.far];
#pragma unroll
                for (int i = 0; i < 4; ++i) dx[i] = sub_sat(tp[mt], pos[i]) >= two.edge ? far : near;
              } else {
                int at[4];
                int2 cell[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  at[i] = place_of(tp[mt], pos[i]);
                  cell[i] = bl.cells[cell_of(at[i])];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  kk[i] = bucket_in(bl, at[i], cell[i]);
                  dx[i] = hb[kk[i]];
                }
              }
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) dx[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (tail && jb + 4 * g4 + i >= jend) dx[i] = -INFINITY;
              hid |= dx[i] == -INFINITY ? 1u << i : 0u;
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) dx[i] = bias[mt];
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x = S[mt][i], slope = 1.f;
            if (a.cap > 0.f) {
              x = kBf16 ? tanh_fast(x * cap_in, true) : tanhf(x * cap_in);
              slope = 1.f - x * x;
            }
            x = fmaf(x, gain, dx[i]);
            float p = exp2_fast(x - mx[mt]) * il[mt];
            float d = p * (dP[mt][i] - D[mt]);
            if (slow && ((hid >> i) & 1)) p = d = 0.f;
            w[i] = p;
            dz[i] = d * slope;
            dx[i] = d;
          }
          // a row that has all the weight has no gradient: its dP and D differ by
          // the order of their sums alone (what is not finite stays so)
          if (__ballot(fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3])) >= 1.f)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (w[i] >= 1.f) {
                dz[i] *= 0.f;
                dx[i] *= 0.f;
              }
          }
          if (nb) {
            if (!slow) {
              dsum[mt] += (dx[0] + dx[1]) + (dx[2] + dx[3]);
            } else {
              // what the lane has kept so far goes along where it can
              if (!each) {
                float near = 0.f, far = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const bool is_far = sub_sat(tp[mt], pos[i]) >= two.edge;
                  far += is_far ? dx[i] : 0.f;
                  near += is_far ? 0.f : dx[i];
                }
                if (__ballot(dsum[mt] != 0.f && bk[mt] != two.far) == 0) {
                  far += dsum[mt];
                  dsum[mt] = 0.f;
                }
                add_bins(two.far, far, two.near == two.far ? -1 : two.near, near);
              } else {
                add_bins(kk[0], dx[0], kk[1], dx[1]);
                add_bins(kk[2], dx[2], kk[3], dx[3]);
              }
              if (__ballot(dsum[mt] != 0.f)) add_bins(bk[mt], dsum[mt], -1, 0.f);
              dsum[mt] = 0.f;
              bk[mt] = each ? kk[3] : two.near;
              bias[mt] = bl.bias[(hs * a.G + hh) * (slots + 1) + bk[mt]];
              keep_bucket(bl, a.masked, bk[mt], bias[mt], blo[mt], bhi[mt]);
            }
          }
          if (slow && __ballot(hid != (1u << 4) - 1u) == 0) continue;

          // ---- the terms of w and dz; by target in LDS
          F4 zh, zl;
          unsigned char* row = dzt + c16 * kPRow<T>;
          if constexpr (kBf16) {
            auto cut4 = [](float (&x)[4], bool last) {
              return last ? make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]))
                          : make_uint2(cut_bf16(x[0], x[1]), cut_bf16(x[2], x[3]));
            };
            *reinterpret_cast<uint2*>(row + 8 * g4) = cut4(w, false);
            *reinterpret_cast<uint2*>(row + 32 + 8 * g4) = cut4(w, true);
            const uint2 h = cut4(dz, false), l = cut4(dz, true);
            *reinterpret_cast<uint2*>(row + 64 + 8 * g4) = h;
            *reinterpret_cast<uint2*>(row + 96 + 8 * g4) = l;
            zh = __builtin_bit_cast(s16x4, h);
            zl = __builtin_bit_cast(s16x4, l);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) zh[i] = dz[i];
            *reinterpret_cast<f32x4*>(row + 16 * g4) = f32x4{w[0], w[1], w[2], w[3]};
            *reinterpret_cast<f32x4*>(row + 64 + 16 * g4) = zh;
          }
          __builtin_amdgcn_wave_barrier();
          const bool careful = slow && (odd_rows || __ballot(odd_k)) && __ballot(hid != 0) != 0;
          // ---- sum over the step's rows: dQ^T += K^T dz; sums over targets:
          // dV^T += dout^T w, dK^T += q^T dz
          F4 p[4];  // w, dz (bf16: two terms each) of row c16, targets 4 g4 + i
          if constexpr (kBf16) {
            const unsigned char* at = dzt + (4 * g4 + (c16 >> 2)) * kPRow<T> + 8 * (c16 & 3);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = __builtin_bit_cast(s16x4, lds_read_tr16(at + 32 * i));
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float* at = reinterpret_cast<const float*>(dzt + (4 * g4 + i) * kPRow<T>) + c16;
              p[0][i] = at[0];
              p[2][i] = at[16];
            }
          }
          if (!careful) {
#pragma unroll
            for (int e = 0; e < NE; ++e) {
              const F4 dT = column4<T, DH>(dt, 0, e, c16, g4), qT = column4<T, DH>(qt, 0, e, c16, g4);
              dq[mt][e] = mma16(kc[e], zh, dq[mt][e]);
              dv[e] = mma16(dT, p[0], dv[e]);
              dk[e] = mma16(qT, p[2], dk[e]);
              if constexpr (kBf16) {
                dq[mt][e] = mma16(kc[e], zl, dq[mt][e]);
                dv[e] = mma16(dT, p[1], dv[e]);
                dk[e] = mma16(qT, p[3], dk[e]);
              }
            }
          } else {
            // 0 times an infinite or NaN row is not 0: column by column, with
            // the rows that a column does not see (is hidden from) cleared
#pragma unroll 1
            for (int col = 0; col < 16; ++col) {
              const uint32_t hq = __shfl(hid, col + 16 * g4);
              uint32_t hk = 0;  // targets 4 g4 + i that row `col` is hidden from
#pragma unroll
              for (int i = 0; i < 4; ++i)
                hk |= ((__shfl(hid, 4 * g4 + i + 16 * (col >> 2)) >> (col & 3)) & 1u) << i;
#pragma unroll
              for (int e = 0; e < NE; ++e) {
                const F4 kx = cleared(kc[e], hq), dx = cleared(column4<T, DH>(dt, 0, e, c16, g4), hk),
                         qx = cleared(column4<T, DH>(qt, 0, e, c16, g4), hk);
                f32x4 nq = mma16(kx, zh, dq[mt][e]), nv = mma16(dx, p[0], dv[e]),
                      nk = mma16(qx, p[2], dk[e]);
                if constexpr (kBf16) {
                  nq = mma16(kx, zl, nq);
                  nv = mma16(dx, p[1], nv);
                  nk = mma16(qx, p[3], nk);
                }
                if (c16 == col) {
                  dq[mt][e] = nq;
                  dv[e] = nv;
                  dk[e] = nk;
                }
              }
            }
          }
          __builtin_amdgcn_wave_barrier();
        }
      }
      // ---- this step's dK, dV: a lane holds DH / 4 consecutive features of row c16
      if (jb + c16 >= j1 || (single && pass + 1 < passes)) continue;
      if (pass + 1 < passes) {
        float* p = a.acc_kv + acc_at + static_cast<int64_t>(c16) * a.Hk * DH + 4 * NE * g4;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          reinterpret_cast<f32x4*>(p)[e] = dk[e];
          reinterpret_cast<f32x4*>(p + acc_v)[e] = dv[e];
        }
      } else {
        T* kp = static_cast<T*>(a.dk) + (h0 + jb + c16) * a.lddk + g * DH + 4 * NE * g4;
        T* vp = static_cast<T*>(a.dv) + (h0 + jb + c16) * a.lddv + g * DH + 4 * NE * g4;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          const f32x4 k = dk[e] * a.scale, v = dv[e];
          if constexpr (kBf16) {
            reinterpret_cast<uint2*>(kp)[e] = make_uint2(pack_bf16(k[0], k[1]), pack_bf16(k[2], k[3]));
            reinterpret_cast<uint2*>(vp)[e] = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
          } else {
            reinterpret_cast<f32x4*>(kp)[e] = k;
            reinterpret_cast<f32x4*>(vp)[e] = v;
          }
        }
      }
    }

    // ---- dq of the pass: the waves' sums in wave order
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (mt >= held) break;
      if (nb) add_bins(bk[mt], dsum[mt], -1, 0.f);
      __syncthreads();
#pragma unroll
      for (int e = 0; e < NE; ++e)
        reinterpret_cast<f32x4*>(s_comb + (wave * 16 + c16) * (DH + 4) + 4 * NE * g4)[e] = dq[mt][e];
      __syncthreads();
      const int row = tid >> 4, f = (tid & 15) * NE;
      const int64_t row0 = t0 + 16 * static_cast<int64_t>(first + mt), head0 = g0 * a.G + hh;
      for (int hd = 0; hd < a.hw && 16 * (first + mt) + row < m; ++hd) {
        float v[NE];
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          v[e] = 0.f;
          for (int wv = hd; wv < kWaves; wv += a.hw) v[e] += s_comb[(wv * 16 + row) * (DH + 4) + f + e];
          v[e] *= a.scale;
        }
        if (a.max_chunks > 1) {
          float* p = a.part_dq + (part_row(a, c, unit, t0, row0) * a.H + head0) * DH + (row * a.H + hd * a.G) * DH + f;
#pragma unroll
          for (int e = 0; e < NE; e += 2) *reinterpret_cast<f32x2*>(p + e) = f32x2{v[e], v[e + 1]};
        } else {
          T* p = static_cast<T*>(a.dq) + (row0 + row) * a.lddq + (head0 + hd * a.G) * DH + f;
#pragma unroll
          for (int e = 0; e < NE; ++e) p[e] = from_f32<T>(v[e]);
        }
      }
    }
    // dbias of a head: 4 threads a bucket, one wave's sums each (cleared for the
    // next head), added over the head's waves
    for (int i = tid; last_of_head && ttiles > 0 && i < (4 * nb + 63) / 64 * 64; i += kThreads) {
      const int k = i >> 2, wv = i & 3;
      float v = 0.f;
      if (k < nb) {
        float* p = s_bins + (wv * (slots + 1) + k) * copies;
#pragma unroll 16
        for (int l = 0; l < copies; ++l) v += p[(l + k) & (copies - 1)];
        if (pass + 1 < passes)
#pragma unroll 16
          for (int l = 0; l < copies; ++l) p[(l + k) & (copies - 1)] = 0.f;
      }
      if (a.hw < 4) v += __shfl_xor(v, 2);
      if (a.hw < 2) v += __shfl_xor(v, 1);
      if (k < nb && wv < a.hw) part_db[(wv * a.G + hh) * nb + k] = v;
    }
    first = last_of_head ? 0 : first + MT;
    hh += last_of_head;
  }
}

// Per target and head what every chunk's workgroups need: the forward's maximum,
// 1 / its sum, D = dout . out and the position.  A row that sees nothing has an
// infinite maximum, and so no weight anywhere.
template <typename T, int DH>
__global__ __launch_bounds__(256) void attn_bwd_rows_kernel(const AttnArgs a) {
  constexpr int NE = DH / 16;
  if (blockIdx.x == gridDim.x - 1) {
    check_call(a, false);
    return;
  }
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4);
  if (row >= a.n_tgt * a.H) return;
  const int f = (threadIdx.x & 15) * NE;
  float D = 0.f;
#pragma unroll
  for (int e = 0; e < NE; ++e)
    D += to_f32(static_cast<const T*>(a.dout)[row * DH + f + e]) * a.fa[row * DH + f + e];
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) D += __shfl_xor(D, o);
  if (f == 0) {
    const float mx = a.fm[row], l = a.fl[row];
    const bool none = mx == -INFINITY && l == 0.f;
    reinterpret_cast<f32x4*>(a.rows)[row] = f32x4{none ? INFINITY : mx, none ? 0.f : 1.f / l, none ? 0.f : D,
                                                  __int_as_float(a.placed ? a.tgt_pos[row / a.H] : 0)};
  }
}

// The chunks' dq (one row per 16 lanes) and the units' dbias (one bucket per
// thread column, 16 unit strides), each summed in a fixed order, with several
// loads on their way (8192 requests with 2 heads of 16 buckets 55 us for 279; 256
// of 8 chunks and 8 heads of 32 buckets 11 for 27).
template <typename T, int DH>
__global__ __launch_bounds__(256) void attn_bwd_sum_kernel(const AttnArgs a, int dq_blocks) {
  constexpr int NE = DH / 16;
  if (static_cast<int>(blockIdx.x) < dq_blocks) {
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4);
    if (row >= a.n_tgt * a.H) return;
    const int64_t t = row / a.H;
    const int f0 = (threadIdx.x & 15) * NE;
    int lo = 0, hi = a.R;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.tgt_off[mid] <= t) lo = mid;
      else hi = mid;
    }
    const int len = clamp_off(a.hist_off[lo + 1], a.n_hist) - clamp_off(a.hist_off[lo], a.n_hist);
    const int n = max(1, min(a.max_chunks, (len + a.chunk - 1) / a.chunk));
    int64_t first, step;
    if (!part_rows(a, lo, t, row, first, step)) return;
    float acc[NE] = {};
#pragma unroll 4
    for (int c = 0; c < n; ++c)
#pragma unroll
      for (int e = 0; e < NE; ++e) acc[e] += a.part_dq[(c * step + first) * DH + f0 + e];
    T* p = static_cast<T*>(a.dq) + t * a.lddq + (row % a.H) * DH + f0;
#pragma unroll
    for (int e = 0; e < NE; ++e) p[e] = from_f32<T>(acc[e]);
    return;
  }
  __shared__ double s[256];
  const int b = (static_cast<int>(blockIdx.x) - dq_blocks) * 16 + (threadIdx.x & 15), n = a.H * a.b.n;
  double v = 0.;
  if (b < n) {
#pragma unroll 8
    for (int u = threadIdx.x >> 4; u < a.units; u += 16) v += a.part_db[static_cast<int64_t>(u) * n + b];
  }
  s[threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.x < 16 && b < n) {
    for (int k = 1; k < 16; ++k) v += s[threadIdx.x + 16 * k];
    a.dbias[b] = static_cast<float>(v);
  }
}

template <typename T, int DH, int MT, bool kOnePass>
hipError_t launch_bwd(const AttnArgs& a, hipStream_t st) {
  const size_t lds = BwdLds<T, DH, MT>::bytes(a.bufs, a.hw, a.G, a.b.n, bin_copies(a.b.n));
  const int64_t grid = round_up(a.units, kXcds) * (a.Hk / a.hw), rows = ceil_div(a.n_tgt * a.H, 16) + 1;
  if (grid > 0x7fffffff || rows > 0x7fffffff) return hipErrorInvalidValue;
  hipError_t e = allow_lds<&attn_bwd_kernel<T, DH, MT, kOnePass>>(lds);
  if (e != hipSuccess) return e;
  attn_bwd_rows_kernel<T, DH><<<static_cast<unsigned>(rows), 256, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  attn_bwd_kernel<T, DH, MT, kOnePass><<<static_cast<unsigned>(grid), kThreads, lds, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t dq_blocks = a.max_chunks > 1 ? ceil_div(a.n_tgt * a.H, 16) : 0;
  const int64_t blocks = dq_blocks + ceil_div(static_cast<int64_t>(a.H) * a.b.n, 16);
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  if (blocks) attn_bwd_sum_kernel<T, DH><<<static_cast<unsigned>(blocks), 256, 0, st>>>(a, static_cast<int>(dq_blocks));
  return hipGetLastError();
}

// (A kernel of its own where one pass is all, without the state of the others: 48
// targets of 8 heads of 64 features 379 us for 486, the window 392 for 420; of 4 heads
// of 128, whose four tiles spill either way, 603 for 573.)
template <typename T, int DH>
hipError_t backward_dh(const AttnArgs& a, int tiles, hipStream_t st) {
  const bool one = a.bufs == 1;
  if constexpr (Elem<T>::bf16) {
    if constexpr (DH > 32)
      if (tiles == 4) return launch_bwd<T, DH, 4, true>(a, st);  // (see backward_tiles)
    if constexpr (DH == 32)
      if (tiles == 4) return one ? launch_bwd<T, DH, 4, true>(a, st) : launch_bwd<T, DH, 4, false>(a, st);
  }
  if constexpr (DH < 128 || Elem<T>::bf16)
    if (tiles == 2) return one ? launch_bwd<T, DH, 2, true>(a, st) : launch_bwd<T, DH, 2, false>(a, st);
  return one ? launch_bwd<T, DH, 1, true>(a, st) : launch_bwd<T, DH, 1, false>(a, st);
}

template <typename T>
hipError_t backward_t(const AttnArgs& a, int dh, int tiles, hipStream_t st) {
  if (dh == 32) return backward_dh<T, 32>(a, tiles, st);
  if (dh == 64) return backward_dh<T, 64>(a, tiles, st);
  return backward_dh<T, 128>(a, tiles, st);
}

}  // namespace

size_t backward_lds(int dtype, int dh, int tiles, int bufs, int hw, int G, int n) {
  auto of = [&](auto lds) { return decltype(lds)::bytes(bufs, hw, G, n, bin_copies(n)); };
  auto type = [&](auto t) {
    using T = decltype(t);
    auto width = [&](auto w) {
      constexpr int DH = decltype(w)::value;
      return tiles == 4 ? of(BwdLds<T, DH, 4>{}) : tiles == 2 ? of(BwdLds<T, DH, 2>{}) : of(BwdLds<T, DH, 1>{});
    };
    using std::integral_constant;
    return dh == 32 ? width(integral_constant<int, 32>{}) : dh == 64 ? width(integral_constant<int, 64>{})
                                                                       : width(integral_constant<int, 128>{});
  };
  return dtype == STCA_BF16 ? type(bf16_bits{}) : type(float{});
}

// Row tiles a wave holds: the fewest that take a request's `need` tiles of a head
// in one pass, up to what registers (dq, DH / 16 x 4 a tile) and LDS allow.  In
// bf16 of 64 and 128 features four spill: they pay where one pass then takes the
// chunk (128 requests of 2048 rows, 48 targets, 8 heads of 64: four tiles 379 us, two
// 973; 4 heads of 128: four 603, two 1379, one 1462), but not where the heads that
// share a kv head or more targets make several passes anyway, of chunks of one step a
// wave (48 requests, 4 heads of 64 to a kv head: two 227 us, one 250, four 428; of 128:
// two 342, one 375, four 397; 128 requests, 100 targets, 4 heads of 64: two 889, one
// 1015, four 1302; of 128: two 2496, one 2758, four 2775).
int backward_tiles(int dtype, int dh, int need, int G) {
  if (dtype != STCA_BF16) return dh < 128 && need >= 2 ? 2 : 1;
  if (dh > 32 && (G > 1 || need > 4)) return need > 1 ? 2 : 1;
  return need >= 3 ? 4 : need == 2 ? 2 : 1;
}

hipError_t attn_backward(const AttnArgs& a, int dtype, int dh, int tiles, hipStream_t st) {
  return dtype == STCA_BF16 ? backward_t<bf16_bits>(a, dh, tiles, st) : backward_t<float>(a, dh, tiles, st);
}

}  // namespace ops
}  // namespace stca
