// Forward of the stand-alone target-to-history attention, over packed rows or
// over a paged cache:
//   x = cap(scale q.k) + bias[h][bucket(p_t - p_j)];  out = softmax(x) v.
//
// One workgroup of four waves takes one chunk of one request's history for up to
// 16 MT rows (target, query head of a kv head's group) and hw kv heads; 4 / hw
// waves share a head, each with consecutive blocks of 16 NT history rows and
// softmax statistics and an output of its own, joined in LDS at the end.  Four
// heads a workgroup read packed rows in whole cache lines at one time (256
// requests, 16 targets, 2048 rows, 8 heads of 32 features: 128 us, one 179); one
// head a workgroup spreads a small batch over more of them.  Several chunks
// leave (output, maximum, sum) partials for attn_merge.
//
// Packed rows are bound by their bytes (that window: 541 MB, 104 us at a large
// copy's rate, takes 128 us, with mask and bias 146), pages by the vector
// instructions of a score: 8-bit rows are converted for the matrix cores, and a
// target of few rows fills a quarter of a tile or less.
//
// Everything of a block stays in one wave's registers.  Scores are formed
// transposed, S^T = K Q^T (v_mfma 16x16x32 bf16, or 16x16x4 fp32), so that the
// result registers of a lane (column t = lane % 16, rows 4 (lane / 16) + i)
// are the operand of O^T = V^T P^T as they stand: the history row of S^T's
// tile i, row r, is j = 4 NT (r / 4) + 4 i + r % 4, which gives lane group g
// the 4 NT consecutive rows 4 NT g ..., the ones that its V operand holds.
// V of packed rows is read a row at a time, DH / 16 elements a lane, and pairs
// of rows are merged by byte permutes; V pages hold rows along the fast axis.
// A row's maximum is only raised (and O rescaled) when a score passes it by
// kSlack: a vote per block instead of a reduction across lanes.  (The maximum of rows
// that are taken again, see kLargeSum, lies `above` the scores from the start.)
//
// P enters the matrix cores as bf16 terms: two (one term's rounding would show
// in the output as a second rounding of its size, 1.7e-3 -> 2.4e-3 relative to
// 64 bits on normal inputs), or three, an fp32 whole, where a backward will
// form D = dout . out from what is saved.  The matrix cores have the time.
//
// Where the distances of a block lie in one bucket for every lane (a vote over
// the interval that each lane keeps), its bias is added as it stands; elsewhere
// every score looks its bucket up.
#pragma once

#include <type_traits>

#include "attn_ops.h"

namespace stca {
namespace ops {

constexpr int kRagged = 0, kPagedBf16 = 1, kPagedInt8 = 2;
constexpr float kSlack = 8.f;  // a weight before the division is at most 2^8
// ... and a sum of them times V may leave fp32 where the output does not.  Where one
// of a workgroup's comes to 2^100 (or is not finite), it takes the rows again with
// weights of at most 1 / (the request's rows); below that all joins stay finite.
// (Not from the start: scores far below the maximum lose bits in the subtraction.)
constexpr float kLargeSum = 1.2676506002282294e30f;  // 2^100

template <int DH> constexpr int kCombineFloats = kWaves * 16 * (DH + 2);  // LDS before the tables (see forward_lds)

template <typename T, int KV, int DH, int NT>
struct Block {
  static constexpr bool kF32 = !Elem<T>::bf16;
  static constexpr int KS = DH / 32;   // k steps of 32 features
  static constexpr int NE = DH / 16;   // output tiles; lane c holds features NE c + e
  static constexpr int NJ = 4 * NT;    // history rows of a lane
  // K operand of tile i, step s
  f32x4 kf[kF32 ? NT : 1][kF32 ? 2 * KS : 1];
  bf16x8 kb[KV == kRagged && kF32 ? 1 : (KV == kPagedInt8 ? 1 : NT)][KS];
  uint2 k8[KV == kPagedInt8 ? NT : 1][KV == kPagedInt8 ? KS : 1];
  // V as loaded
  uint32_t vw[KV == kRagged ? NJ : 1][KV == kRagged ? (kF32 ? NE : NE / 2) : 1];
  uint32_t vp[KV == kRagged ? 1 : NE][NJ / (KV == kPagedInt8 ? 4 : 2)];
  uint32_t ke[NJ / 4], ve[NJ / 4];     // exponents
  int pj[NJ];                          // positions, where the rows have some
};

template <int N>
__device__ __forceinline__ void load_words(gptr base, uint32_t at, uint32_t* w) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4 x = load_at<u32x4>(base + 16 * i, at);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[4 * i + k] = x[k];
    }
  } else if constexpr (N == 2) {
    const u32x2 x = load_at<u32x2>(base, at);
    w[0] = x[0];
    w[1] = x[1];
  } else {
    w[0] = load_at<uint32_t>(base, at);
  }
}

// N words (2 or 4, aligned to all of them).
template <int N>
__device__ __forceinline__ void copy_words(const void* p, uint32_t* w) {
  if constexpr (N == 4) {
    const uint4 x = *static_cast<const uint4*>(p);
    w[0] = x.x;
    w[1] = x.y;
    w[2] = x.z;
    w[3] = x.w;
  } else {
    const uint2 x = *static_cast<const uint2*>(p);
    w[0] = x.x;
    w[1] = x.y;
  }
}

// First feature of lane group g's eight of step s.
template <int KV, int DH>
__device__ __forceinline__ int feature(int s, int g) {
  if constexpr (KV == kPagedInt8 && DH >= 64) return 64 * (s / 2) + 16 * g + 8 * (s % 2);
  else return 32 * s + 8 * g;
}

__device__ __forceinline__ float int8_f32(uint32_t w, int k) {
  return static_cast<float>(static_cast<int8_t>(w >> (8 * k)));
}
// Eight int8 of two words as bf16 (exact: 8 significant bits hold 0..127).
__device__ __forceinline__ bf16x8 int8_bf16(uint32_t a, uint32_t b) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? a : b;
    const float x = int8_f32(w, 2 * (i % 2)), y = int8_f32(w, 2 * (i % 2) + 1);
    r[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
  }
  return __builtin_bit_cast(bf16x8, make_uint4(r[0], r[1], r[2], r[3]));
}
// 2^(byte k - 127), byte 255 infinity, in one instruction (the compiler takes a
// shift and a mask).
template <int K>
__device__ __forceinline__ float exp_byte(uint32_t w) {
  uint32_t r;
  const uint32_t n = 23;
  if constexpr (K == 0)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(r) : "v"(n), "v"(w));
  else if constexpr (K == 1)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(r) : "v"(n), "v"(w));
  else if constexpr (K == 2)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(r) : "v"(n), "v"(w));
  else
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(r) : "v"(n), "v"(w));
  return __uint_as_float(r);
}
__device__ __forceinline__ void exp_bytes(const uint32_t (&w)[2], float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    f[4 * i] = exp_byte<0>(w[i]);
    f[4 * i + 1] = exp_byte<1>(w[i]);
    f[4 * i + 2] = exp_byte<2>(w[i]);
    f[4 * i + 3] = exp_byte<3>(w[i]);
  }
}

__device__ __forceinline__ bool odd_bf16(uint32_t w) {  // a half of w is not finite
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

// Two waves a SIMD, where the registers hold a block, the next one on its way,
// the output and the rows.  Of 128 features they do without the next block (one
// wave that has it, two tiles: 32 requests of 10240 8-bit rows, 32 targets, 4 heads
// 172 us for 126; 24 of 10240 bf16 rows, 16 targets, 4 heads to a kv head 231 for 190).
// Three of 8-bit rows of 32 features: left to itself the compiler takes one register
// too many for them (128 requests of 10240 rows, 32 targets 273 us, three 250).
template <int KV, int DH> constexpr int kFwdWaves = KV == kPagedInt8 && DH == 32 ? 3 : 2;
template <int DH> constexpr bool kAhead = DH < 128;

template <typename T, int KV, int DH, int MT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kFwdWaves<KV, DH>))) void attn_fwd_kernel(const AttnArgs a) {
  constexpr bool kF32 = !Elem<T>::bf16;
  constexpr bool kPaged = KV != kRagged;
  constexpr int NT = 2;
  constexpr int BJ = 16 * NT;
  constexpr int KS = DH / 32, NE = DH / 16, NJ = 4 * NT;
  using Blk = Block<T, KV, DH, NT>;
  extern __shared__ __align__(16) unsigned char smem[];
  float* comb = reinterpret_cast<float*>(smem);
  int* s_large = reinterpret_cast<int*>(comb + kCombineFloats<DH>);  // a joining wave has seen a large sum
  int2* s_cells = reinterpret_cast<int2*>(s_large + kWaves);
  int32_t* s_edges = reinterpret_cast<int32_t*>(s_cells + kCells + 1);
  float* s_bias = reinterpret_cast<float*>(s_edges + kMaxBuckets);
  int32_t* s_table = reinterpret_cast<int32_t*>(s_bias + a.hw * a.G * (max(a.b.n, 1) + 1));

  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  if (blockIdx.x == gridDim.x - 1) {
    check_call(a, kPaged);
    return;
  }
  // every kv head and row group of a chunk on one XCD: heads share cache lines
  // of packed rows, row groups share everything
  const int ghs = a.Hk / a.hw, per = ghs * a.zgroups;
  const int unit = static_cast<int>(blockIdx.x) / kXcds / per * kXcds + static_cast<int>(blockIdx.x) % kXcds;
  if (unit >= a.units) return;
  const int rem = static_cast<int>(blockIdx.x) / kXcds % per;
  const int g0 = rem % ghs * a.hw, z = rem / ghs;
  const int hs = wave % a.hw, part = wave / a.hw, parts = kWaves / a.hw, g = g0 + hs;

  int r, c, len;
  int64_t h0 = 0;
  if constexpr (kPaged) {
    r = unit / a.max_chunks;
    c = unit % a.max_chunks;
    len = uniform(min(max(a.lens[r], 0), a.max_len));
  } else {
    r = uniform(find_request(a.hist_off, a.R, a.n_hist, a.chunk, unit));
    h0 = uniform(clamp_off(a.hist_off[r], a.n_hist));
    len = uniform(max(0, static_cast<int>(clamp_off(a.hist_off[r + 1], a.n_hist) - h0)));
    c = unit - static_cast<int>(h0 / a.chunk + r);
  }
  if (c < 0 || c >= a.max_chunks || (c > 0 && static_cast<int64_t>(c) * a.chunk >= len)) return;
  const int j0 = c * a.chunk;
  const int t0 = uniform(clamp_off(a.tgt_off[r], a.n_tgt));
  const int m = min(uniform(clamp_off(a.tgt_off[r + 1], a.n_tgt)) - t0, a.max_tgt), rows = m * a.G;
  if (z * 16 * MT >= rows) return;
  // (one chunk on the host's offsets: there are no partials, whatever the device's say)
  const bool split = a.max_chunks > 1 && len > a.chunk;
  const int j1 = j0 + min(len - j0, a.chunk);

  // tables
  // (pointers that are known to be LDS: set whether used or not)
  const BucketLds bl{s_cells, s_bias, s_edges, max(a.b.n, 1), a.b.multi};
  if (a.placed) fill_buckets(a, g0, a.hw * a.G, s_cells, s_bias, s_edges);
  if (tid < kWaves) s_large[tid] = 0;
  bool holes = false;
  if constexpr (kPaged) {
    const int p0 = j0 >> a.page_shift, p1 = (j1 + (1 << a.page_shift) - 1) >> a.page_shift;
    for (int i = p0 + tid; i < p1; i += kThreads) {
      const int p = a.table[static_cast<int64_t>(r) * a.table_ld + i];
      const bool bad = p < 0 || p >= a.n_pages;
      s_table[i - p0] = bad ? -1 : p;
      holes |= bad;
    }
    holes = __syncthreads_or(holes);
  } else {
    __syncthreads();
  }

  // (a copy of its own for the rows that are taken again: as a turn of this loop it
  // costs the first one registers, a step of 147 requests of 72 fp32 rows 95 us for 89)
  auto take = [&](auto second) {
  const float above = decltype(second)::value ? kSlack + static_cast<float>(32 - __builtin_clz(len)) : 0.f;
  for (int zz = z; zz * 16 * MT < rows; zz += a.zgroups) {
    // ---- this lane's rows: column c16 of each tile
    int tpos[MT], hbias[MT];  // hbias: this row's biases in the table
    int64_t trow[MT];
    bool have[MT];
    bf16x8 qb[kF32 ? 1 : MT][KS];
    f32x4 qf[kF32 ? MT : 1][kF32 ? 2 * KS : 1];
    int seen_max = -2147483647 - 1;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int row = (zz * MT + mt) * 16 + c16;
      have[mt] = row < rows;
      const int t = have[mt] ? row / a.G : 0;
      const int head = have[mt] ? row % a.G : 0;
      hbias[mt] = (hs * a.G + head) * (bl.slots + 1);
      trow[mt] = t0 + t;
      tpos[mt] = a.placed ? a.tgt_pos[trow[mt]] : 0;
      if (have[mt]) seen_max = max(seen_max, tpos[mt]);
      const T* qp = static_cast<const T*>(a.q) + trow[mt] * a.ldq + (static_cast<int64_t>(g) * a.G + head) * DH;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const T* p = qp + feature<KV, DH>(s, g4);
        if constexpr (kF32) {
          qf[mt][2 * s] = have[mt] ? reinterpret_cast<const f32x4*>(p)[0] : f32x4{};
          qf[mt][2 * s + 1] = have[mt] ? reinterpret_cast<const f32x4*>(p)[1] : f32x4{};
        } else {
          qb[mt][s] = have[mt] ? *reinterpret_cast<const bf16x8*>(p) : bf16x8{};
        }
      }
    }
    // rows past every target's own index are hidden from all of them
    int jend = j1;
    if (a.masked && !a.hist_pos) {
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) seen_max = max(seen_max, __shfl_xor(seen_max, o));
      jend = max(j0, static_cast<int>(min<int64_t>(jend, static_cast<int64_t>(seen_max) + 1)));
      jend = __builtin_amdgcn_readfirstlane(jend);
    }

    float mx[MT], sum[MT], bias[MT];
    int blo[MT], bhi[MT];  // the distances that `bias` is for
    f32x4 o[MT][NE];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      mx[mt] = -INFINITY;
      sum[mt] = 0.f;
      bias[mt] = 0.f;
      blo[mt] = a.masked ? 1 : 0;
      bhi[mt] = a.b.n ? -1 : 0x7fffffff;  // (a bias: none kept yet)
#pragma unroll
      for (int e = 0; e < NE; ++e) o[mt][e] = f32x4{};
    }

    // K and V of block jb; a row past the end is the last one again (hidden below)
    const uint32_t lk = static_cast<uint32_t>(a.ldk * sizeof(T)), lv = static_cast<uint32_t>(a.ldv * sizeof(T));
    auto load = [&](Blk& b, int jb) {
      const int last = len - 1 - jb;
      if constexpr (!kPaged) {
        const gptr kp = uniform(static_cast<const char*>(a.k) + ((h0 + jb) * a.ldk + static_cast<int64_t>(g) * DH) * sizeof(T));
        const gptr vp = uniform(static_cast<const char*>(a.v) + ((h0 + jb) * a.ldv + static_cast<int64_t>(g) * DH) * sizeof(T));
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const uint32_t at = __umul24(min(NJ * (c16 >> 2) + 4 * i + (c16 & 3), last), lk) + 8 * g4 * sizeof(T);
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            const gptr p = kp + 32 * s * sizeof(T);
            if constexpr (kF32) {
              b.kf[i][2 * s] = load_at<f32x4>(p, at);
              b.kf[i][2 * s + 1] = load_at<f32x4>(p + 16, at);
            } else {
              b.kb[i][s] = load_at<bf16x8>(p, at);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
          const uint32_t at = __umul24(min(NJ * g4 + i, last), lv) + c16 * NE * static_cast<uint32_t>(sizeof(T));
          load_words<(kF32 ? NE : NE / 2)>(vp, at, b.vw[i]);
        }
        if (a.hist_pos) {
          const gptr hp = uniform(a.hist_pos + h0 + jb);
#pragma unroll
          for (int i = 0; i < NJ; ++i) b.pj[i] = load_at<int>(hp, 4u * min(NJ * g4 + i, last));
        }
      } else {
        // The NJ rows of a lane's V operand lie in one page, and so do those of
        // its K operand's tiles.  Past the end: the last run's, which exists.
        const int P = 1 << a.page_shift, ps = a.page_shift, p0 = j0 >> ps;
        constexpr uint32_t ES = KV == kPagedInt8 ? 1 : 2;
        auto run = [&](int i) { return min(jb + NJ * i, (len - 1) & ~(NJ - 1)); };
        auto page_at = [&](int j) { return static_cast<uint32_t>(max(s_table[(j >> ps) - p0], 0)); };
        const uint32_t head_rows = static_cast<uint32_t>(a.Hk) << ps;  // rows of a page, all heads
        const int jk = run(c16 >> 2), jv = run(g4);
        const char* kp = static_cast<const char*>(a.k) + (static_cast<int64_t>(g) << ps) * (DH * ES) +
                         static_cast<uint64_t>(page_at(jk)) * (head_rows * (DH * ES)) +
                         ((jk & (P - 1)) + (c16 & 3)) * (DH * ES);
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            const char* p = kp + 4 * i * DH * ES + feature<KV, DH>(s, g4) * ES;
            if constexpr (KV == kPagedInt8) b.k8[i][s] = *reinterpret_cast<const uint2*>(p);
            else b.kb[i][s] = *reinterpret_cast<const bf16x8*>(p);
          }
        const uint32_t pv = page_at(jv), slot = jv & (P - 1);
        const char* vp = static_cast<const char*>(a.v) + (static_cast<int64_t>(g) << ps) * (DH * ES) +
                         static_cast<uint64_t>(pv) * (head_rows * (DH * ES)) + (((NE * c16) << ps) + slot) * ES;
#pragma unroll
        for (int e = 0; e < NE; ++e) copy_words<NJ * ES / 4>(vp + ((e * ES) << ps), b.vp[e]);
        if constexpr (KV == kPagedInt8) {
          const uint64_t at = (static_cast<uint64_t>(g) << ps) + static_cast<uint64_t>(pv) * head_rows + slot;
          copy_words<NJ / 4>(a.ke + at, b.ke);
          copy_words<NJ / 4>(a.ve + at, b.ve);
        }
        if (a.hist_pos) {
          const int32_t* hp = a.hist_pos + (static_cast<int64_t>(pv) << ps) + slot;
#pragma unroll
          for (int i = 0; i < NJ; ++i) b.pj[i] = hp[i];
        }
      }
    };

    // scores in units of log2 e: gain (q k) + bias, or with a cap gain tanh(cap_in (q k)) + bias
    const float gain = kLog2e * (a.cap > 0.f ? a.cap : a.scale), cap_in = a.cap > 0.f ? a.scale / a.cap : 0.f;
    const bool whole = !kPaged && a.sa != nullptr;

    auto compute = [&](Blk& b, int jb, bool more) {
      // V operand of O^T: rows NJ g4 + 8 s + 0..7, feature NE c16 + e
      bf16x8 vb[kF32 ? 1 : NT / 2][kF32 ? 1 : NE];
      float vf[kF32 ? NJ : 1][kF32 ? NE : 1];
      if constexpr (KV == kRagged && !kF32) {
#pragma unroll
        for (int s = 0; s < NT / 2; ++s)
#pragma unroll
          for (int e2 = 0; e2 < NE / 2; ++e2) {
            uint32_t lo[4], hi[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              lo[i] = __builtin_amdgcn_perm(b.vw[8 * s + 2 * i + 1][e2], b.vw[8 * s + 2 * i][e2], 0x05040100u);
              hi[i] = __builtin_amdgcn_perm(b.vw[8 * s + 2 * i + 1][e2], b.vw[8 * s + 2 * i][e2], 0x07060302u);
            }
            vb[s][2 * e2] = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
            vb[s][2 * e2 + 1] = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
          }
      } else if constexpr (KV == kRagged) {
#pragma unroll
        for (int i = 0; i < NJ; ++i)
#pragma unroll
          for (int e = 0; e < NE; ++e) vf[i][e] = __uint_as_float(b.vw[i][e]);
      } else if constexpr (KV == kPagedBf16) {
#pragma unroll
        for (int e = 0; e < NE; ++e)
          vb[0][e] = __builtin_bit_cast(bf16x8, make_uint4(b.vp[e][0], b.vp[e][1], b.vp[e][2], b.vp[e][3]));
      } else if constexpr (KV == kPagedInt8) {
#pragma unroll
        for (int e = 0; e < NE; ++e) {
#pragma unroll
          for (int s = 0; s < NT / 2; ++s) vb[s][e] = int8_bf16(b.vp[e][2 * s], b.vp[e][2 * s + 1]);
        }
      }
      f32x4 S[MT][NT];
#pragma unroll
      for (int i = 0; i < NT; ++i) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) S[mt][i] = f32x4{};
        if constexpr (kF32) {
#pragma unroll
          for (int k = 0; k < 2 * KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) S[mt][i] = mfma_f32(b.kf[i][k][e], qf[mt][k][e], S[mt][i]);
        } else {
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            bf16x8 kc;
            if constexpr (KV == kPagedInt8) kc = int8_bf16(b.k8[i][k].x, b.k8[i][k].y);
            else kc = b.kb[i][k];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) S[mt][i] = mfma_bf16(kc, qb[mt][k], S[mt][i]);
          }
        }
      }
      uint32_t kexp[NJ / 4], vexp[NJ / 4];
#pragma unroll
      for (int i = 0; i < NJ / 4; ++i) {
        kexp[i] = b.ke[i];
        vexp[i] = b.ve[i];
      }
      int pj[NJ];
      int pmin = 0, pmax = 0;
      if (a.placed) {
        if (a.hist_pos) {
          pmin = pmax = b.pj[0];
#pragma unroll
          for (int i = 0; i < NJ; ++i) {
            pj[i] = b.pj[i];
            pmin = min(pmin, pj[i]);
            pmax = max(pmax, pj[i]);
          }
        } else {
          pmin = jb + NJ * g4;
          pmax = pmin + NJ - 1;
#pragma unroll
          for (int i = 0; i < NJ; ++i) pj[i] = pmin + i;
        }
      }
      // the block's registers are free: the next one is on its way from here on
      if (more) load(b, jb + BJ);
      const bool tail = jb + BJ > jend || holes;
      // a score's factor before the cap, or its whole gain; an 8-bit row's step in it
      float row_gain[KV == kPagedInt8 ? NJ : 1];
      float vstep[KV == kPagedInt8 ? NJ : 1];
      if constexpr (KV == kPagedInt8) {
        exp_bytes(kexp, row_gain);
        exp_bytes(vexp, vstep);
#pragma unroll
        for (int i = 0; i < NJ; ++i) row_gain[i] *= a.cap > 0.f ? cap_in : gain;
      } else {
        row_gain[0] = a.cap > 0.f ? cap_in : gain;
      }
      auto gain_of = [&](int i) { return a.cap > 0.f ? gain : row_gain[KV == kPagedInt8 ? i : 0]; };
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        // biases, in units of log2 e as the scores
        float x[NJ];
        uint32_t hid = 0;
        const bool slow = __ballot(tail || place_of(tpos[mt], pmax) < blo[mt] || place_of(tpos[mt], pmin) > bhi[mt]) != 0;
        if (a.cap > 0.f) {
#pragma unroll
          for (int i = 0; i < NJ; ++i) {
            const float y = S[mt][i / 4][i % 4] * row_gain[KV == kPagedInt8 ? i : 0];
            S[mt][i / 4][i % 4] = kF32 ? tanhf(y) : tanh_fast(y, whole || a.cap > kPlainCap);
          }
        }
        if (!slow) {
#pragma unroll
          for (int i = 0; i < NJ; ++i) x[i] = fmaf(S[mt][i / 4][i % 4], gain_of(i), bias[mt]);
        } else {
          if (a.placed) {
            TwoBuckets two;
            int k;
            if (__ballot(!two_buckets(bl, place_of(tpos[mt], pmax), place_of(tpos[mt], pmin), two)) == 0) {
              const float near = bl.bias[hbias[mt] + two.near], far = bl.bias[hbias[mt] + two.far];
#pragma unroll
              for (int i = 0; i < NJ; ++i) x[i] = sub_sat(tpos[mt], pj[i]) >= two.edge ? far : near;
              k = two.near;
              bias[mt] = near;
            } else {
#pragma unroll
              for (int i4 = 0; i4 < NJ; i4 += 4) {
                int at[4];
                int2 cell[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  at[i] = place_of(tpos[mt], pj[i4 + i]);
                  cell[i] = bl.cells[cell_of(at[i])];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  k = bucket_in(bl, at[i], cell[i]);
                  x[i4 + i] = bias[mt] = bl.bias[hbias[mt] + k];
                }
              }
            }
            // the lane keeps one of its buckets: its nearest rows', or its last row's
            keep_bucket(bl, a.masked, k, bias[mt], blo[mt], bhi[mt]);
          } else {
#pragma unroll
            for (int i = 0; i < NJ; ++i) x[i] = 0.f;
          }
          if (tail) {
#pragma unroll
            for (int i = 0; i < NJ; ++i) {
              const int j = jb + NJ * g4 + i;
              bool out = j >= jend;
              if constexpr (kPaged)
                if (holes) out |= s_table[(min(j, len - 1) >> a.page_shift) - (j0 >> a.page_shift)] < 0;
              if (out) x[i] = -INFINITY;
            }
          }
          // (a hidden row's score may be NaN)
#pragma unroll
          for (int i = 0; i < NJ; ++i) {
            hid |= x[i] == -INFINITY ? 1u << i : 0u;
            const float y = fmaf(S[mt][i / 4][i % 4], gain_of(i), x[i]);
            x[i] = x[i] == -INFINITY ? x[i] : y;
          }
          if (!__ballot(hid != (1u << NJ) - 1u)) continue;  // nothing of this block is seen
        }
        // running maximum
        float top = x[0];
#pragma unroll
        for (int i = 1; i < NJ; ++i) top = fmaxf(top, x[i]);
        if (__ballot(top > mx[mt] + (kSlack - above))) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float mn = fmaxf(mx[mt], top + above);
          const float f = mx[mt] == -INFINITY ? 0.f : exp2_fast(mx[mt] - mn);
          mx[mt] = mn;
          sum[mt] *= f;
#pragma unroll
          for (int e = 0; e < NE; ++e) o[mt][e] *= f;
        }
        const float base = mx[mt] == -INFINITY ? 0.f : mx[mt];
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
          x[i] = exp2_fast(x[i] - base);
          sum[mt] += x[i];
        }
        if constexpr (KV == kPagedInt8) {
#pragma unroll
          for (int i = 0; i < NJ; ++i) x[i] *= vstep[i];
        }
        // A hidden row's value (or its scale) may be infinite or NaN, and 0
        // times it is not 0: such blocks go column by column, each with the
        // values it may not see cleared.
        bool careful = false;
        if (slow && __ballot(hid != 0)) {
          bool odd = false;
          if constexpr (KV == kPagedInt8) {
#pragma unroll
            for (int i = 0; i < NJ; ++i) x[i] = (hid >> i) & 1 ? 0.f : x[i];
          } else if constexpr (kF32) {
#pragma unroll
            for (int i = 0; i < NJ; ++i)
#pragma unroll
              for (int e = 0; e < NE; ++e) odd |= !(fabsf(vf[i][e]) < INFINITY);
          } else {
#pragma unroll
            for (int s = 0; s < NT / 2; ++s)
#pragma unroll
              for (int e = 0; e < NE; ++e) {
                const uint4 w = __builtin_bit_cast(uint4, vb[s][e]);
                odd |= odd_bf16(w.x) || odd_bf16(w.y) || odd_bf16(w.z) || odd_bf16(w.w);
              }
          }
          careful = __ballot(odd) != 0;
        }
        if constexpr (kF32) {
          if (!careful) {
#pragma unroll
            for (int i = 0; i < NJ; ++i)
#pragma unroll
              for (int e = 0; e < NE; ++e) o[mt][e] = mfma_f32(vf[i][e], x[i], o[mt][e]);
          } else {
            for (int col = 0; col < 16; ++col) {
              const uint32_t h = __shfl(hid, col + 16 * g4);
#pragma unroll
              for (int e = 0; e < NE; ++e) {
                f32x4 n = o[mt][e];
#pragma unroll
                for (int i = 0; i < NJ; ++i) n = mfma_f32((h >> i) & 1 ? 0.f : vf[i][e], x[i], n);
                if (c16 == col) o[mt][e] = n;
              }
            }
          }
        } else {
          // a term at a time: its operands, then its products; the second is rounded,
          // and what that leaves, of either sign, is the third
          auto term = [&](int n) {
            bf16x8 p[NT / 2];
#pragma unroll
            for (int s = 0; s < NT / 2; ++s) {
              uint32_t w[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                float &a0 = x[8 * s + 2 * k], &a1 = x[8 * s + 2 * k + 1];
                w[k] = n == 0 ? cut_bf16(a0, a1) : n == 1 ? pack_bf16(a0, a1) : high_halves(a0, a1);
                if (n == 1 && whole) {
                  a0 -= lo_f32(w[k]);
                  a1 -= hi_f32(w[k]);
                }
              }
              p[s] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
            }
            if (!careful) {
#pragma unroll
              for (int s = 0; s < NT / 2; ++s)
#pragma unroll
                for (int e = 0; e < NE; ++e) o[mt][e] = mfma_bf16(vb[s][e], p[s], o[mt][e]);
            } else {
              for (int col = 0; col < 16; ++col) {
                const uint32_t h = __shfl(hid, col + 16 * g4);
#pragma unroll
                for (int s = 0; s < NT / 2; ++s)
#pragma unroll
                  for (int e = 0; e < NE; ++e) {
                    uint4 w = __builtin_bit_cast(uint4, vb[s][e]);
                    auto keep = [&](uint32_t v, int i) {
                      return v & (((h >> (8 * s + i)) & 1 ? 0u : 0xffffu) | ((h >> (8 * s + i + 1)) & 1 ? 0u : 0xffff0000u));
                    };
                    w = make_uint4(keep(w.x, 0), keep(w.y, 2), keep(w.z, 4), keep(w.w, 6));
                    const f32x4 n = mfma_bf16(__builtin_bit_cast(bf16x8, w), p[s], o[mt][e]);
                    if (c16 == col) o[mt][e] = n;
                  }
              }
            }
          };
          term(0);
          term(1);
          if (whole) term(2);
        }
      }
    };

    // each wave takes consecutive blocks (a lane's bucket changes seldom then)
    const int blocks = (jend - j0 + BJ - 1) / BJ, share = (blocks + parts - 1) / parts;
    int jb = j0 + part * share * BJ;
    const int jstop = min(jend, jb + share * BJ);
    if (jb < jstop) {
      Blk blk;
      if constexpr (kAhead<DH>) load(blk, jb);
      for (; jb < jstop; jb += BJ) {
        if constexpr (!kAhead<DH>) load(blk, jb);
        compute(blk, jb, kAhead<DH> && jb + BJ < jstop);
      }
    }

    // ---- join the waves: lane group g4 of wave w holds features NE (4 g4 + i) + e of column c16
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if ((zz * MT + mt) * 16 >= rows) break;
      float l = sum[mt];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      float* cw = comb + wave * 16 * (DH + 2);
      if (g4 == 0) {
        cw[16 * DH + 2 * c16] = mx[mt];
        cw[16 * DH + 2 * c16 + 1] = l;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < NE; ++e) cw[(NE * (4 * g4 + i) + e) * 16 + c16] = o[mt][e][i];
      __syncthreads();
      // thread: column tid / 16, DH / 16 consecutive features, of each head
      const int col = tid >> 4, f0 = (tid & 15) * NE;
      const int row = (zz * MT + mt) * 16 + col;
      for (int hd = 0; hd < a.hw && row < rows; ++hd) {
        float M = -INFINITY, L = 0.f, acc[NE];
        for (int w = hd; w < kWaves; w += a.hw) M = fmaxf(M, comb[w * 16 * (DH + 2) + 16 * DH + 2 * col]);
#pragma unroll
        for (int e = 0; e < NE; ++e) acc[e] = 0.f;
        for (int w = hd; w < kWaves; w += a.hw) {
          const float* p = comb + w * 16 * (DH + 2);
          const float mw = p[16 * DH + 2 * col], lw = p[16 * DH + 2 * col + 1];
          // (a NaN sum without a maximum is a row of NaN scores)
          const float f = mw == -INFINITY ? (lw != lw ? lw : 0.f) : exp2_fast(mw - M);
          L += f * lw;
#pragma unroll
          for (int e = 0; e < NE; ++e) acc[e] += f * p[(f0 + e) * 16 + col];
        }
        bool large = false;
#pragma unroll
        for (int e = 0; e < NE; ++e) large |= !(fabsf(acc[e]) < kLargeSum);
        if (large) s_large[wave] = 1;
        const int64_t t = t0 + row / a.G;
        const int h = (g0 + hd) * a.G + row % a.G;
        if (split) {
          const int64_t at = part_row(a, c, unit, t0, t) * a.H + h;
#pragma unroll
          for (int e = 0; e < NE; ++e) a.part_o[at * DH + f0 + e] = acc[e];
          if (f0 == 0) {
            a.part_ml[2 * at] = M;
            a.part_ml[2 * at + 1] = L;
          }
        } else {
          const float inv = L == 0.f ? 0.f : 1.f / L;
          T* op = static_cast<T*>(a.out) + (t * a.H + h) * DH + f0;
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            const float y = acc[e] * inv;
            op[e] = from_f32<T>(y);
            if (a.sa) a.sa[(t * a.H + h) * DH + f0 + e] = y;
          }
          if (a.sm && f0 == 0) {
            a.sm[t * a.H + h] = M;
            a.sl[t * a.H + h] = L;
          }
        }
      }
      __syncthreads();
    }
  }
  };
  take(std::false_type{});
  const int4 large = *reinterpret_cast<const int4*>(s_large);
  if (uniform(large.x | large.y | large.z | large.w)) take(std::true_type{});
}

template <typename T, int KV, int DH, int MT>
hipError_t launch_fwd(const AttnArgs& a, hipStream_t st) {
  const int64_t pages = KV == kRagged ? 0 : (a.chunk >> a.page_shift) + 1;
  const size_t lds = forward_lds(DH, a.hw, a.G, a.b.n, pages);
  const int64_t grid = round_up(a.units, kXcds) * (a.Hk / a.hw) * a.zgroups + 1;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const hipError_t e = allow_lds<&attn_fwd_kernel<T, KV, DH, MT>>(lds);
  if (e != hipSuccess) return e;
  attn_fwd_kernel<T, KV, DH, MT><<<static_cast<unsigned>(grid), kThreads, lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace ops
}  // namespace stca
