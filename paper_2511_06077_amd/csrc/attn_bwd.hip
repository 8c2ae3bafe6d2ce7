// Backward of the stand-alone target-to-history attention.  With w the softmax
// weights of the forward (from its saved maxima and sums), per (target t, head
// h, history row j):
//   dP = dout . v,  D = dout . out,  dx = w (dP - D)       -> dbias[h][bucket]
//   dz = dx (1 - (y / c)^2)                                 (c: the score cap)
//   dv_j += w dout,  dk_j += scale dz q,  dq_t += scale dz k_j
//
// One workgroup takes one chunk of one request's history for one kv head; its
// four waves take steps of 16 JT history rows in turn and hold dK^T, dV^T of a
// step in registers while they go through the pass's MT tiles of 16 targets (of
// one query head each), whose q and dout rows wait in LDS.  dq of a pass stays
// in registers over the whole chunk.  More tiles than MT are further passes
// over the chunk, with dK, dV of the passes so far in fp32 in the workspace
// (the same lanes write and read them).  So K, V are read and dK, dV written
// once, nothing is added in order of arrival, and gradients repeat bitwise.
//
// Scores are formed as S = Q K^T: a lane holds column j = lane % 16 and rows
// t = 4 (lane / 16) + i, which is the operand of the sums over t (dV^T =
// dout^T w, dK^T = q^T dz) as it stands.  The sum over j (dQ = dz K) needs the
// other order: dz goes through LDS, written four targets at a time and read
// with the transposing LDS read; K too, and q^T, dout^T likewise.
//
// w and dz are split into two bf16 terms (the products then carry 16
// significant bits, and the one rounding left is the output's).
//
// dbias: a lane sums the dx of its column in a register as long as its bucket
// (an interval of distances) covers all four targets; when a vote finds a lane
// outside, the wave sums bucket by bucket what its lanes hold (the first
// lane's bucket, then the first of those left) into LDS sums of its own.
#include <type_traits>

#include "attn_ops.h"
#include "ring.h"

namespace stca {
namespace ops {

namespace {

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

// LDS of a workgroup, in bytes.
template <typename T, int DH, int MT, int JT>
struct BwdLds {
  static constexpr int kQ = 0;                                       // q rows of the pass
  static constexpr int kDo = kQ + 16 * MT * kRowBytes<T, DH>;        // dout rows
  static constexpr int kRow = kDo + 16 * MT * kRowBytes<T, DH>;      // per row: maximum, 1 / sum, D, position
  static constexpr int kK = kRow + 16 * MT * 16;                     // per wave: K rows of the step
  static constexpr int kKWave = 16 * JT * kRowBytes<T, DH>;
  static constexpr int kDz = kK + kWaves * kKWave;                   // per wave: dz tile, both terms
  static constexpr int kDzWave = 16 * JT * (Elem<T>::bf16 ? 2 * 32 : 80);
  static constexpr int kComb = kDz + kWaves * kDzWave;               // dq of the waves
  static constexpr int kBins = kComb + kWaves * 16 * DH * 4;         // dbias per wave and tile
  static size_t bytes(int G, int n) {
    return kBins + 4 * (kWaves * MT * static_cast<size_t>(n) + kMaxBuckets + 32 + 2 * static_cast<size_t>(G) * n);
  }
};

template <typename T, int DH, int MT, int JT>
__global__ __launch_bounds__(kThreads) void attn_bwd_kernel(const AttnArgs a) {
  constexpr bool kBf16 = Elem<T>::bf16;
  constexpr int KS = DH / 32, NE = DH / 16, BJ = 16 * JT;
  using F4 = typename Four<T>::type;
  using E8 = Eight<T>;
  using Lds = BwdLds<T, DH, MT, JT>;
  extern __shared__ __align__(16) unsigned char smem[];
  const int nb = a.b.n;
  float* s_row = reinterpret_cast<float*>(smem + Lds::kRow);
  float* s_comb = reinterpret_cast<float*>(smem + Lds::kComb);
  float* s_bins = reinterpret_cast<float*>(smem + Lds::kBins);
  int32_t* s_edges = reinterpret_cast<int32_t*>(s_bins + kWaves * MT * nb);
  uint8_t* s_cell = reinterpret_cast<uint8_t*>(s_edges + kMaxBuckets);
  float* s_bias = reinterpret_cast<float*>(s_cell + 128);
  float* s_db = s_bias + a.G * nb;

  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (blockIdx.x == gridDim.x - 1) {
    check_call(a, false);
    return;
  }
  const int unit = static_cast<int>(blockIdx.x) / kXcds / a.Hk * kXcds + static_cast<int>(blockIdx.x) % kXcds;
  if (unit >= a.units) return;
  const int g = static_cast<int>(blockIdx.x) / kXcds % a.Hk;
  const int r = find_request(a.hist_off, a.R, a.n_hist, a.chunk, unit);
  const int64_t h0 = clamp_off(a.hist_off[r], a.n_hist);
  const int len = max(0, static_cast<int>(clamp_off(a.hist_off[r + 1], a.n_hist) - h0));
  const int c = unit - static_cast<int>(h0 / a.chunk + r);
  float* part_db = a.part_db + (static_cast<int64_t>(unit) * a.H + g * a.G) * nb;
  if (c < 0 || c >= a.max_chunks || (c > 0 && static_cast<int64_t>(c) * a.chunk >= len)) {
    for (int i = tid; i < a.G * nb; i += kThreads) part_db[i] = 0.f;
    return;
  }
  const int j0 = c * a.chunk, j1 = min(len, j0 + a.chunk);
  const int t0 = clamp_off(a.tgt_off[r], a.n_tgt), m = max(0, clamp_off(a.tgt_off[r + 1], a.n_tgt) - t0);
  const int ttiles = (m + 15) / 16, tiles = ttiles * a.G;

  for (int i = tid; i < nb; i += kThreads) s_edges[i] = a.b.edges[i];
  if (nb) {
    if (tid < 128) s_cell[tid] = a.b.cell[tid];
    for (int i = tid; i < a.G * nb; i += kThreads) {
      s_bias[i] = a.bias[static_cast<int64_t>(g) * a.G * nb + i];
      s_db[i] = 0.f;
    }
  }
  const BucketLds bl{s_edges, s_cell, s_bias, nb};
  unsigned char* kt = smem + Lds::kK + wave * Lds::kKWave;
  unsigned char* dzt = smem + Lds::kDz + wave * Lds::kDzWave;

  const int passes = max(1, (tiles + MT - 1) / MT);
  for (int pass = 0; pass < passes; ++pass) {
    const int first = pass * MT, held = min(MT, tiles - first);
    __syncthreads();
    // ---- the pass's rows: 16 threads a row, DH / 16 features each
    int odd_rows = 0;
    for (int row = tid >> 4; row < 16 * MT; row += kThreads / 16) {
      const int tile = first + row / 16, hh = tile < tiles ? tile / ttiles : 0;
      const int t = tile < tiles ? tile % ttiles * 16 + row % 16 : m;
      const bool have = t < m;
      const int64_t tr = t0 + min(t, max(m - 1, 0)), h = g * a.G + hh;
      const int f = (tid & 15) * NE;
      T* qs = reinterpret_cast<T*>(smem + Lds::kQ + row * kRowBytes<T, DH>) + f;
      T* ds = reinterpret_cast<T*>(smem + Lds::kDo + row * kRowBytes<T, DH>) + f;
      float D = 0.f;
      bool odd = false;
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        T qv = 0, dv = 0;
        if (have) {
          qv = static_cast<const T*>(a.q)[tr * a.ldq + h * DH + f + e];
          dv = static_cast<const T*>(a.dout)[(tr * a.H + h) * DH + f + e];
          D += to_f32(dv) * a.fa[(tr * a.H + h) * DH + f + e];
          odd |= !(fabsf(to_f32(qv)) < INFINITY) || !(fabsf(to_f32(dv)) < INFINITY);
        }
        qs[e] = qv;
        ds[e] = dv;
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) D += __shfl_xor(D, o);
      odd_rows |= odd;
      if ((tid & 15) == 0) {
        // a row without a target, or that sees nothing, has no weight anywhere
        const float mx = have ? a.fm[tr * a.H + h] : INFINITY, l = have ? a.fl[tr * a.H + h] : 1.f;
        const bool none = mx == -INFINITY && l == 0.f;
        s_row[4 * row] = none ? INFINITY : mx;
        s_row[4 * row + 1] = none ? 0.f : 1.f / l;
        s_row[4 * row + 2] = none ? 0.f : D;
        s_row[4 * row + 3] = __int_as_float(a.placed && m > 0 ? a.tgt_pos[tr] : 0);
      }
    }
    for (int i = tid; i < kWaves * MT * nb; i += kThreads) s_bins[i] = 0.f;
    odd_rows = __syncthreads_or(odd_rows);

    f32x4 dq[MT][NE];
    float bias[MT], dsum[MT];
    int blo[MT], bhi[MT], bk[MT], tmin[MT], tmax[MT], head[MT];
    int seen_max = -2147483647 - 1;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int e = 0; e < NE; ++e) dq[mt][e] = f32x4{};
      bias[mt] = dsum[mt] = 0.f;
      bk[mt] = 0;
      head[mt] = mt < held ? (first + mt) / ttiles : 0;
      blo[mt] = a.masked ? 0 : -2147483647 - 1;
      bhi[mt] = nb ? -2147483647 - 1 : 2147483647;
      tmin[mt] = 2147483647;
      tmax[mt] = -2147483647 - 1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = __float_as_int(s_row[4 * (16 * mt + 4 * g4 + i) + 3]);
        tmin[mt] = min(tmin[mt], p);
        tmax[mt] = max(tmax[mt], p);
      }
      if (mt < held) seen_max = max(seen_max, tmax[mt]);
    }
    int jend = j1;  // rows from here on are hidden from every target of the pass
    if (a.masked && !a.hist_pos) {
      seen_max = max(seen_max, __shfl_xor(seen_max, 16));
      seen_max = max(seen_max, __shfl_xor(seen_max, 32));
      jend = static_cast<int>(min<int64_t>(jend, static_cast<int64_t>(seen_max) + 1));
      jend = __builtin_amdgcn_readfirstlane(jend);
    }
    if (held <= 0) jend = 0;

    // what lanes hold for their buckets, into this wave's sums
    auto add_bins = [&](int mt, const int* kk, const float* vv, int n) {
      uint32_t left = (1u << n) - 1u;
      while (true) {
        const uint64_t some = __ballot(left != 0);
        if (!some) break;
        const int src = static_cast<int>(__builtin_ctzll(some));
        int mine = kk[0];
        for (int i = n - 1; i >= 0; --i)
          if ((left >> i) & 1) mine = kk[i];
        const int k = __builtin_amdgcn_readlane(mine, src);
        float v = 0.f;
        for (int i = 0; i < n; ++i)
          if (((left >> i) & 1) && kk[i] == k) {
            v += vv[i];
            left &= ~(1u << i);
          }
#pragma unroll
        for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
        if (lane == 0) s_bins[(wave * MT + mt) * nb + k] += v;
      }
    };

    for (int jb = j0 + wave * BJ; jb < j1; jb += kWaves * BJ) {
      f32x4 dk[JT][NE], dv[JT][NE];
      const int64_t acc_at = ((h0 + jb) * a.Hk + g) * DH;  // fp32 sums of the earlier passes: row jt 16 + c16
      const int64_t acc_v = a.n_hist * a.Hk * DH;
#pragma unroll
      for (int jt = 0; jt < JT; ++jt)
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          dk[jt][e] = dv[jt][e] = f32x4{};
          const int j = 16 * jt + c16;
          if (pass > 0 && jb + j < j1) {
            const float* p = a.acc_kv + acc_at + static_cast<int64_t>(j) * a.Hk * DH + 4 * (NE * g4 + e);
            dk[jt][e] = *reinterpret_cast<const f32x4*>(p);
            dv[jt][e] = *reinterpret_cast<const f32x4*>(p + acc_v);
          }
        }
      if (jb < jend) {
        E8 kf[JT][KS], vf[JT][KS];
        int pj[JT];
        const int last = len - 1 - jb;
#pragma unroll
        for (int jt = 0; jt < JT; ++jt) {
          const int jr = min(16 * jt + c16, last);
          const T* kp = static_cast<const T*>(a.k) + (h0 + jb + jr) * a.ldk + g * DH + 8 * g4;
          const T* vp = static_cast<const T*>(a.v) + (h0 + jb + jr) * a.ldv + g * DH + 8 * g4;
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            kf[jt][s] = load8<T>(kp + 32 * s);
            vf[jt][s] = load8<T>(vp + 32 * s);
          }
          pj[jt] = !a.placed ? 0 : a.hist_pos ? a.hist_pos[h0 + jb + jr] : jb + 16 * jt + c16;
        }
        // K in the other order: rows of the step along the operand
        F4 kc[JT][NE];
        bool odd_k = false;
#pragma unroll
        for (int jt = 0; jt < JT; ++jt)
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            store8<T>(reinterpret_cast<T*>(kt + (16 * jt + c16) * kRowBytes<T, DH>) + 32 * s + 8 * g4, kf[jt][s]);
            odd_k |= odd8<T>(kf[jt][s]);
          }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int jt = 0; jt < JT; ++jt)
#pragma unroll
          for (int e = 0; e < NE; ++e) kc[jt][e] = column4<T, DH>(kt, 16 * jt, e, c16, g4);
        __builtin_amdgcn_wave_barrier();
        const bool tail = jb + BJ > jend;
        const bool odd_step = odd_rows || __ballot(odd_k) != 0;

#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          if (mt >= held) break;
          const unsigned char* qt = smem + Lds::kQ + 16 * mt * kRowBytes<T, DH>;
          const unsigned char* dt = smem + Lds::kDo + 16 * mt * kRowBytes<T, DH>;
          float mx[4], il[4], D[4];
          int tp[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 row = *reinterpret_cast<const f32x4*>(s_row + 4 * (16 * mt + 4 * g4 + i));
            mx[i] = row[0];
            il[i] = row[1];
            D[i] = row[2];
            tp[i] = __float_as_int(row[3]);
          }
          f32x4 S[JT], dP[JT];
#pragma unroll
          for (int jt = 0; jt < JT; ++jt) S[jt] = dP[jt] = f32x4{};
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            const E8 qf = load8<T>(reinterpret_cast<const T*>(qt + c16 * kRowBytes<T, DH>) + 32 * s + 8 * g4);
            const E8 df = load8<T>(reinterpret_cast<const T*>(dt + c16 * kRowBytes<T, DH>) + 32 * s + 8 * g4);
#pragma unroll
            for (int jt = 0; jt < JT; ++jt) {
              S[jt] = mma32(qf, kf[jt][s], S[jt]);
              dP[jt] = mma32(df, vf[jt][s], dP[jt]);
            }
          }
          bool out = tail;
#pragma unroll
          for (int jt = 0; jt < JT; ++jt)
            out |= sub_sat(tmin[mt], pj[jt]) < blo[mt] || sub_sat(tmax[mt], pj[jt]) > bhi[mt];
          const bool slow = __ballot(out) != 0;
          uint32_t hid = 0;  // bit 4 jt + i
          float w[JT][4], dz[JT][4];
          int kk[4 * JT + 1];
          float xb[JT][4];
          if (!slow) {
#pragma unroll
            for (int jt = 0; jt < JT; ++jt)
#pragma unroll
              for (int i = 0; i < 4; ++i) xb[jt][i] = bias[mt];
          } else {
#pragma unroll
            for (int jt = 0; jt < JT; ++jt)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int d = a.placed ? sub_sat(tp[i], pj[jt]) : 0;
                bool vis = jb + 16 * jt + c16 < jend && !(a.masked && d < 0);
                xb[jt][i] = 0.f;
                kk[4 * jt + i] = 0;
                if (nb) {
                  kk[4 * jt + i] = bucket_of(bl, d);
                  xb[jt][i] = s_bias[head[mt] * nb + kk[4 * jt + i]];
                  vis = vis && xb[jt][i] != -INFINITY;
                }
                if (!vis) hid |= 1u << (4 * jt + i);
              }
          }
          float dx[4 * JT + 1];
#pragma unroll
          for (int jt = 0; jt < JT; ++jt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float x = S[jt][i] * a.scale, slope = 1.f;
              if (a.cap > 0.f) {
                const float th = kBf16 ? tanh_fast(x / a.cap) : tanhf(x / a.cap);
                x = a.cap * th;
                slope = 1.f - th * th;
              }
              x += xb[jt][i];
              float p = exp_nat(x - mx[i]) * il[i];
              float g = p * (dP[jt][i] - D[i]);
              if (slow && ((hid >> (4 * jt + i)) & 1)) p = g = 0.f;
              w[jt][i] = p;
              dx[4 * jt + i] = g;
              dz[jt][i] = g * slope;
            }
          if (nb) {
            if (!slow) {
#pragma unroll
              for (int i = 0; i < 4 * JT; ++i) dsum[mt] += dx[i];
            } else {
              kk[4 * JT] = bk[mt];
              dx[4 * JT] = dsum[mt];
              dsum[mt] = 0.f;
              bk[mt] = kk[4 * JT - 1];
              bias[mt] = xb[JT - 1][3];
              const int edge = bk[mt] ? s_edges[bk[mt] - 1] : (a.masked ? 0 : -2147483647 - 1);
              blo[mt] = bias[mt] == -INFINITY ? 2147483647 : edge;
              bhi[mt] = bk[mt] == nb - 1 ? 2147483647 : s_edges[bk[mt]] - 1;
              add_bins(mt, kk, dx, 4 * JT + 1);
            }
          }
          if (slow && __ballot(hid != (1u << (4 * JT)) - 1u) == 0) continue;

          // ---- sums over targets: dV^T += dout^T w, dK^T += q^T dz
          F4 wh[JT], wl[JT], zh[JT], zl[JT];
#pragma unroll
          for (int jt = 0; jt < JT; ++jt) {
            if constexpr (kBf16) {
              uint2 h, l;
              split_bf16(w[jt][0], w[jt][1], h.x, l.x);
              split_bf16(w[jt][2], w[jt][3], h.y, l.y);
              wh[jt] = __builtin_bit_cast(s16x4, h);
              wl[jt] = __builtin_bit_cast(s16x4, l);
              split_bf16(dz[jt][0], dz[jt][1], h.x, l.x);
              split_bf16(dz[jt][2], dz[jt][3], h.y, l.y);
              zh[jt] = __builtin_bit_cast(s16x4, h);
              zl[jt] = __builtin_bit_cast(s16x4, l);
              *reinterpret_cast<uint2*>(dzt + (16 * jt + c16) * 64 + 8 * g4) = __builtin_bit_cast(uint2, zh[jt]);
              *reinterpret_cast<uint2*>(dzt + (16 * jt + c16) * 64 + 32 + 8 * g4) = __builtin_bit_cast(uint2, zl[jt]);
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                wh[jt][i] = w[jt][i];
                zh[jt][i] = dz[jt][i];
              }
              *reinterpret_cast<f32x4*>(dzt + (16 * jt + c16) * 80 + 16 * g4) = zh[jt];
            }
          }
          __builtin_amdgcn_wave_barrier();
          const bool careful = slow && odd_step && __ballot(hid != 0) != 0;
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            const F4 dT = column4<T, DH>(dt, 0, e, c16, g4), qT = column4<T, DH>(qt, 0, e, c16, g4);
#pragma unroll
            for (int jt = 0; jt < JT; ++jt) {
              if (!careful) {
                dv[jt][e] = mma16(dT, wh[jt], dv[jt][e]);
                dk[jt][e] = mma16(qT, zh[jt], dk[jt][e]);
                if constexpr (kBf16) {
                  dv[jt][e] = mma16(dT, wl[jt], dv[jt][e]);
                  dk[jt][e] = mma16(qT, zl[jt], dk[jt][e]);
                }
              } else {
                // 0 times an infinite or NaN row is not 0: column by column,
                // with the rows that a column is hidden from cleared
                for (int col = 0; col < 16; ++col) {
                  const uint32_t h = __shfl(hid, col + 16 * g4) >> (4 * jt);
                  const F4 dc = cleared(dT, h), qc = cleared(qT, h);
                  f32x4 nv = mma16(dc, wh[jt], dv[jt][e]), nk = mma16(qc, zh[jt], dk[jt][e]);
                  if constexpr (kBf16) {
                    nv = mma16(dc, wl[jt], nv);
                    nk = mma16(qc, zl[jt], nk);
                  }
                  if (c16 == col) {
                    dv[jt][e] = nv;
                    dk[jt][e] = nk;
                  }
                }
              }
            }
          }
          // ---- sum over the step's rows: dQ += dz K
#pragma unroll
          for (int jt = 0; jt < JT; ++jt) {
            F4 ah, al;
            if constexpr (kBf16) {
              const unsigned char* p = dzt + (16 * jt + 4 * g4 + (c16 >> 2)) * 64 + 8 * (c16 & 3);
              ah = __builtin_bit_cast(s16x4, lds_read_tr16(p));
              al = __builtin_bit_cast(s16x4, lds_read_tr16(p + 32));
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                ah[i] = *reinterpret_cast<const float*>(dzt + (16 * jt + 4 * g4 + i) * 80 + 4 * c16);
            }
#pragma unroll
            for (int e = 0; e < NE; ++e) {
              if (!careful) {
                dq[mt][e] = mma16(ah, kc[jt][e], dq[mt][e]);
                if constexpr (kBf16) dq[mt][e] = mma16(al, kc[jt][e], dq[mt][e]);
              } else {
                for (int t = 0; t < 16; ++t) {
                  uint32_t h = 0;
#pragma unroll
                  for (int i = 0; i < 4; ++i)
                    h |= ((__shfl(hid, 4 * g4 + i + 16 * (t >> 2)) >> (4 * jt + (t & 3))) & 1u) << i;
                  const F4 kx = cleared(kc[jt][e], h);
                  f32x4 n = mma16(ah, kx, dq[mt][e]);
                  if constexpr (kBf16) n = mma16(al, kx, n);
                  if (g4 == (t >> 2)) dq[mt][e][t & 3] = n[t & 3];
                }
              }
            }
          }
          __builtin_amdgcn_wave_barrier();
        }
      }
      // ---- this step's dK, dV: a lane holds DH / 4 consecutive features of row 16 jt + c16
#pragma unroll
      for (int jt = 0; jt < JT; ++jt) {
        const int j = 16 * jt + c16;
        if (jb + j >= j1) continue;
        if (pass + 1 < passes) {
          float* p = a.acc_kv + acc_at + static_cast<int64_t>(j) * a.Hk * DH + 4 * NE * g4;
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            reinterpret_cast<f32x4*>(p)[e] = dk[jt][e];
            reinterpret_cast<f32x4*>(p + acc_v)[e] = dv[jt][e];
          }
        } else {
          T* kp = static_cast<T*>(a.dk) + (h0 + jb + j) * a.lddk + g * DH + 4 * NE * g4;
          T* vp = static_cast<T*>(a.dv) + (h0 + jb + j) * a.lddv + g * DH + 4 * NE * g4;
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            const f32x4 k = dk[jt][e] * a.scale, v = dv[jt][e];
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
    }

    // ---- dq of the pass: the waves' sums in wave order
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (mt >= held) break;
      if (nb) {
        const int kk[1] = {bk[mt]};
        const float vv[1] = {dsum[mt]};
        add_bins(mt, kk, vv, 1);
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < NE; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s_comb[(wave * 16 + 4 * g4 + i) * DH + tile_feature<DH>(e, c16)] = dq[mt][e][i];
      __syncthreads();
      const int tile = first + mt, hh = tile / ttiles, row = tid >> 4, t = tile % ttiles * 16 + row;
      if (t < m) {
        const int64_t tr = t0 + t, h = g * a.G + hh;
        const int f = (tid & 15) * NE;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          float v = 0.f;
#pragma unroll
          for (int wv = 0; wv < kWaves; ++wv) v += s_comb[(wv * 16 + row) * DH + f + e];
          v *= a.scale;
          if (a.max_chunks > 1) a.part_dq[((static_cast<int64_t>(c) * a.n_tgt + tr) * a.H + h) * DH + f + e] = v;
          else static_cast<T*>(a.dq)[tr * a.lddq + h * DH + f + e] = from_f32<T>(v);
        }
      }
    }
    __syncthreads();
    for (int k = tid; k < nb; k += kThreads)
      for (int mt = 0; mt < held; ++mt) {
        float v = 0.f;
        for (int wv = 0; wv < kWaves; ++wv) v += s_bins[(wv * MT + mt) * nb + k];
        s_db[(first + mt) / ttiles * nb + k] += v;
      }
  }
  if (nb) {
    __syncthreads();
    for (int i = tid; i < a.G * nb; i += kThreads) part_db[i] = s_db[i];
  }
}

// The chunks' dq (one row per 16 lanes) and the units' dbias (one bucket per
// thread column, 16 unit strides), each summed in a fixed order.
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
    float acc[NE] = {};
    for (int c = 0; c < n; ++c)
#pragma unroll
      for (int e = 0; e < NE; ++e) acc[e] += a.part_dq[(c * a.n_tgt * a.H + row) * DH + f0 + e];
    T* p = static_cast<T*>(a.dq) + t * a.lddq + (row % a.H) * DH + f0;
#pragma unroll
    for (int e = 0; e < NE; ++e) p[e] = from_f32<T>(acc[e]);
    return;
  }
  __shared__ double s[256];
  const int b = (static_cast<int>(blockIdx.x) - dq_blocks) * 16 + (threadIdx.x & 15), n = a.H * a.b.n;
  double v = 0.;
  if (b < n)
    for (int u = threadIdx.x >> 4; u < a.units; u += 16) v += a.part_db[static_cast<int64_t>(u) * n + b];
  s[threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.x < 16 && b < n) {
    for (int k = 1; k < 16; ++k) v += s[threadIdx.x + 16 * k];
    a.dbias[b] = static_cast<float>(v);
  }
}

template <typename T, int DH, int MT>
hipError_t launch_bwd(const AttnArgs& a, hipStream_t st) {
  constexpr int JT = DH == 128 ? 1 : 2;
  const size_t lds = BwdLds<T, DH, MT, JT>::bytes(a.G, a.b.n);
  const int64_t grid = round_up(a.units, kXcds) * a.Hk + 1;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  hipError_t e = allow_lds<&attn_bwd_kernel<T, DH, MT, JT>>(lds);
  if (e != hipSuccess) return e;
  attn_bwd_kernel<T, DH, MT, JT><<<static_cast<unsigned>(grid), kThreads, lds, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t dq_blocks = a.max_chunks > 1 ? ceil_div(a.n_tgt * a.H, 16) : 0;
  const int64_t blocks = dq_blocks + ceil_div(static_cast<int64_t>(a.H) * a.b.n, 16);
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  if (blocks) attn_bwd_sum_kernel<T, DH><<<static_cast<unsigned>(blocks), 256, 0, st>>>(a, static_cast<int>(dq_blocks));
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t backward_dh(const AttnArgs& a, int tiles, hipStream_t st) {
  if constexpr (DH < 128 && Elem<T>::bf16)
    if (tiles == 4) return launch_bwd<T, DH, 4>(a, st);
  if constexpr (DH < 128 || Elem<T>::bf16)
    if (tiles == 2) return launch_bwd<T, DH, 2>(a, st);
  return launch_bwd<T, DH, 1>(a, st);
}

template <typename T>
hipError_t backward_t(const AttnArgs& a, int dh, int tiles, hipStream_t st) {
  if (dh == 32) return backward_dh<T, 32>(a, tiles, st);
  if (dh == 64) return backward_dh<T, 64>(a, tiles, st);
  return backward_dh<T, 128>(a, tiles, st);
}

}  // namespace

// Row tiles a wave holds: the fewest that take a request's tiles in one pass,
// up to what registers (dq, DH / 16 x 4 a tile) and LDS allow.
int backward_tiles(int dtype, int dh, int need) {
  const int most = dtype == STCA_BF16 ? (dh == 128 ? 2 : 4) : (dh == 128 ? 1 : 2);
  return need >= 3 && most == 4 ? 4 : need >= 2 && most >= 2 ? 2 : 1;
}

hipError_t attn_backward(const AttnArgs& a, int dtype, int dh, int tiles, hipStream_t st) {
  return dtype == STCA_BF16 ? backward_t<bf16_bits>(a, dh, tiles, st) : backward_t<float>(a, dh, tiles, st);
}

}  // namespace ops
}  // namespace stca
