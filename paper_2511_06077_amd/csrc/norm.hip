// Norms before and after a block, with its gate and residual scale:
//   t = post(o) act(g);  h = x + scale ls t;  y = pre(h)
// and the gradients of all of it.  A team of lanes takes a row, eight features a
// lane, and holds it in registers from the loads to the stores, so every row is
// read and written once: bound by those bytes (524288 rows of 256 in bf16: the norm
// alone 95 us, 5.6 TB/s; with block and gate 268 forward and 390 backward, 5.0 and
// 5.5 TB/s).  The backward recomputes what it needs from x, o and g, which it has to
// read anyway; nothing is saved.
//
// With u = (v - mean) r the unit row of a layer norm (mean = 0: of an rms norm),
// a = w dy:  dv = r (a - mean(a) - u mean(a u)), without mean(a) for rms.
#include "layer_ops.h"

namespace stca {
namespace layers {

namespace {

constexpr int kThreads = 256;
constexpr int kSums = 5;

template <int L>
struct Team {
  static constexpr int kBlock = L > kThreads ? L : L > 64 ? L : kThreads;  // one team a workgroup beyond a wave
  static constexpr int kRows = kBlock / L;
  static constexpr int kWaves = L > 64 ? L / 64 : 1;
};

// Whether the next row's loads are on their way while a row is computed.  Where a
// row's sums wait at barriers it pays (8191 rows of 2000: 71 -> 63 us backward, 38
// -> 37 forward); where a wave has whole rows, the others hide the loads, and the
// registers cost more (524288 of 256: 387 -> 399 and 267 -> 286).
template <int L>
constexpr bool kAhead = L > 64;

// Sums over a team; of several waves through LDS, two buffers in turn, so that one
// barrier a sum is enough.
template <int L>
struct Reduce {
  float (*lds)[2][16];
  int turn;
  __device__ __forceinline__ void two(float& a, float& b) {
    a = team_sum<(L > 64 ? 64 : L)>(a);
    b = team_sum<(L > 64 ? 64 : L)>(b);
    if constexpr (L > 64) {
      const int wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0) {
        lds[turn][0][wave] = a;
        lds[turn][1][wave] = b;
      }
      __syncthreads();
      a = b = 0.f;
#pragma unroll
      for (int w = 0; w < L / 64; ++w) {
        a += lds[turn][0][w];
        b += lds[turn][1][w];
      }
      turn ^= 1;
    }
  }
  __device__ __forceinline__ float one(float a) {
    a = team_sum<(L > 64 ? 64 : L)>(a);
    if constexpr (L > 64) {
      const int wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0) lds[turn][0][wave] = a;
      __syncthreads();
      a = 0.f;
#pragma unroll
      for (int w = 0; w < L / 64; ++w) a += lds[turn][0][w];
      turn ^= 1;
    }
    return a;
  }
};

// The unit row u of v (zero in lanes behind the row) and r, from values `by` as large.
// False: it has to be taken again with more turns, and `by` may be smaller then.
template <int L, int kTurns>
__device__ __forceinline__ bool unit_of(Reduce<L>& red, const float* v, bool live, int layer, float inv_d, float eps,
                                        float& by, float* u, float& r) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = live ? v[e] * by : 0.f;
  float var;
  bool rough = false;
  if (layer) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += x[e];
    float mean = red.one(s) * inv_d;
    // the differences' own mean corrects for the rounding of the first one, which
    // a row far from zero would see; where that is more than the deviation, as in a
    // row of one value, the variance would be what is left of the rounding: again,
    // each turn with 2^-18 of the mean before or less
#pragma unroll
    for (int turn = 0; turn < kTurns; ++turn) {
      float off = 0.f, sq = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = live ? x[e] - mean : 0.f;
        off += x[e];
        sq = fmaf(x[e], x[e], sq);
      }
      red.two(off, sq);
      mean = off * inv_d;
      var = fmaxf(fmaf(sq, inv_d, -mean * mean), 0.f);
      if (!(sq <= 1e37f)) var = sq;
    }
    rough = mean * mean > var;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = live ? x[e] - mean : 0.f;
  } else {
    float sq = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sq = fmaf(x[e], x[e], sq);
    sq = red.one(sq);
    var = !(sq <= 1e37f) ? sq : sq * inv_d;
  }
  if (kTurns > 1 && by != 1.f && var == 0.f) {  // all values the same
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = 0.f;
    r = __frsqrt_rn(eps);
    return true;
  }
  r = __frsqrt_rn(var + fmaxf(eps * by * by, 1e-37f));
#pragma unroll
  for (int e = 0; e < 8; ++e) u[e] = x[e] * r;
  r *= by;
  if (!(var <= 1e37f)) by = 0x1p-80f;
  return var <= 1e37f && !rough;
}

// Values whose squares leave fp32 are taken 2^-80 as large: eps is nothing beside
// their variance, if they have one.  The second take, for either reason, is out of the
// way of the others without a loop of its own (layer norms backward, 131071 rows of
// 264 in fp32 260 us, in a loop 267; 524288 of 256 in bf16 431 and 440).
template <int L>
__device__ __forceinline__ void unit_row(Reduce<L>& red, const float* v, bool live, int layer, float inv_d, float eps,
                                         float* u, float& r) {
  float by = 1.f;
  if (unit_of<L, 1>(red, v, live, layer, inv_d, eps, by, u, r)) return;  // (the same in the whole team)
  unit_of<L, 6>(red, v, live, layer, inv_d, eps, by, u, r);
}

// Gradient of a unit row, from a = the gradient of u.
template <int L>
__device__ __forceinline__ void unit_grad(Reduce<L>& red, const float* a, const float* u, float r, int layer,
                                          float inv_d, float* g) {
  float s = 0.f, m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    s += a[e];
    m = fmaf(a[e], u[e], m);
  }
  if (layer) {
    red.two(s, m);
    s *= inv_d;
  } else {
    m = red.one(m);
    s = 0.f;
  }
  m *= inv_d;
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] = r * (a[e] - s - u[e] * m);
}

// s(g) and 1 - s(g), the small one of them within 11 halves of a step too: what the
// exponent loses where -|g| log2(e) is rounded, up to |g| 2^-24 of the result, is put
// back as the factor 1 + rest; fp32's ln 2 leaves |g| 2^-28.4 of it.  exp2 gives zero
// below 2^-126, and keeps it where the exponent is not finite (fminf takes the number).
__device__ __forceinline__ void sigmoid(float g, float& s, float& rest) {
  const float x = -fabsf(g), power = x * kLog2e;
  float e = __builtin_amdgcn_exp2f(power);
  e = fmaf(e, fminf(fmaf(power, -kLn2, x), 1.f), e);
  const float p = __builtin_amdgcn_rcpf(1.f + e), q = e * p;
  s = g < 0.f ? q : p;
  rest = g < 0.f ? p : q;
}

struct Vec8 {
  float v[8];
  __device__ __forceinline__ void load(const float* p, int col, bool live, float none) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = live ? none : 0.f;
    if (p && live) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = p[col + e];
    }
  }
};

template <typename T>
__device__ __forceinline__ void row_of(const void* p, int64_t ld, int64_t i, int col, bool have, Oct<T>& o) {
  o.zero();
  if (p && have) o.load(static_cast<const T*>(p) + i * ld + col);
}

template <typename T, int L>
__global__ __launch_bounds__(Team<L>::kBlock) void forward_kernel(const NormArgs a) {
  __shared__ float lds[2][2][16];
  Reduce<L> red{lds, 0};
  const int lane = threadIdx.x % L, team = threadIdx.x / L, col = 8 * lane;
  const bool live = col < a.d;
  const float inv_d = 1.f / static_cast<float>(a.d);
  Vec8 pw, pb, qw, qb, ls;
  pw.load(a.pre_w, col, live, 1.f);
  pb.load(a.pre_b, col, live, 0.f);
  qw.load(a.post_w, col, live, 1.f);
  qb.load(a.post_b, col, live, 0.f);
  ls.load(a.ls, col, live, 1.f);
  const int64_t step = static_cast<int64_t>(gridDim.x) * Team<L>::kRows;
  Oct<T> nx, no, ng;
  auto fetch = [&](int64_t i) {
    const bool have = live && i < a.n;
    row_of(a.x, a.ldx, i, col, have, nx);
    row_of(a.block, a.ldb, i, col, have, no);
    row_of(a.gate, a.ldg, i, col, have, ng);
  };
  if (kAhead<L>) fetch(static_cast<int64_t>(blockIdx.x) * Team<L>::kRows + team);
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * Team<L>::kRows; base < a.n; base += step) {
    const int64_t i = base + team;
    const bool have = live && i < a.n;
    if (!kAhead<L>) fetch(i);
    const Oct<T> ox = nx, oo = no, og = ng;
    if (kAhead<L>) fetch(i + step);
    float h[8], u[8], r;
    ox.get(h);
    if (a.block) {
      float t[8], g[8];
      oo.get(t);
      og.get(g);
      if (a.post) {
        unit_row<L>(red, t, live, a.layer, inv_d, a.eps, u, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = fmaf(u[e], qw.v[e], qb.v[e]);
      }
      if (a.act) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float s, rest;
          sigmoid(g[e], s, rest);
          t[e] *= a.act == 2 ? g[e] * s : s;
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = fmaf(a.scale * ls.v[e], t[e], h[e]);
      if (a.h && have) Oct<T>::store(static_cast<T*>(a.h) + i * a.ldh + col, h);
    }
    if (a.pre) {
      unit_row<L>(red, h, live, a.layer, inv_d, a.eps, u, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = fmaf(u[e], pw.v[e], pb.v[e]);
      if (have) Oct<T>::store(static_cast<T*>(a.y) + i * a.ldy + col, h);
    }
  }
}

template <typename T, int L>
__global__ __launch_bounds__(Team<L>::kBlock) void backward_kernel(const NormArgs a) {
  constexpr int kRows = Team<L>::kRows;
  __shared__ float lds[2][2][16];
  __shared__ float join[kRows > 1 ? kRows : 1][kRows > 1 ? 8 * L : 1];
  Reduce<L> red{lds, 0};
  const int lane = threadIdx.x % L, team = threadIdx.x / L, col = 8 * lane;
  const bool live = col < a.d;
  const float inv_d = 1.f / static_cast<float>(a.d);
  Vec8 pw, qw, qb, ls;
  pw.load(a.pre_w, col, live, 1.f);
  qw.load(a.post_w, col, live, 1.f);
  qb.load(a.post_b, col, live, 0.f);
  ls.load(a.ls, col, live, 1.f);
  float sum[kSums][8] = {};
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
  Oct<T> nx, no, ng, nh, ny;
  auto fetch = [&](int64_t i) {
    const bool have = live && i < a.n;
    row_of(a.x, a.ldx, i, col, have, nx);
    row_of(a.block, a.ldb, i, col, have, no);
    row_of(a.gate, a.ldg, i, col, have, ng);
    row_of(a.dh, a.lddh, i, col, have, nh);
    row_of(a.dy, a.lddy, i, col, have, ny);
  };
  if (kAhead<L>) fetch(static_cast<int64_t>(blockIdx.x) * kRows + team);
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * kRows; base < a.n; base += step) {
    const int64_t i = base + team;
    const bool have = live && i < a.n;
    if (!kAhead<L>) fetch(i);
    const Oct<T> ox = nx, oo = no, og = ng, oh = nh, oy = ny;
    if (kAhead<L>) fetch(i + step);
    float h[8], t[8], n[8], s[8], slope[8], uo[8], ro = 0.f;
    ox.get(h);
    if (a.block) {
      float g[8];
      oo.get(n);
      og.get(g);
      if (a.post) {
        unit_row<L>(red, n, live, a.layer, inv_d, a.eps, uo, ro);
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = fmaf(uo[e], qw.v[e], qb.v[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[e] = 1.f;
        slope[e] = 0.f;
        if (a.act) {
          float p, rest;
          sigmoid(g[e], p, rest);
          s[e] = a.act == 2 ? g[e] * p : p;
          slope[e] = a.act == 2 ? fmaf(g[e] * p, rest, p) : p * rest;
        }
        t[e] = n[e] * s[e];
        h[e] = fmaf(a.scale * ls.v[e], t[e], h[e]);
      }
    }
    float d[8];
    oh.get(d);
    if (a.pre) {
      float u[8], r, y[8], w[8], g[8];
      oy.get(y);
      unit_row<L>(red, h, live, a.layer, inv_d, a.eps, u, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = y[e] * pw.v[e];
        sum[0][e] = fmaf(y[e], u[e], sum[0][e]);
        sum[1][e] += y[e];
      }
      unit_grad<L>(red, w, u, r, a.layer, inv_d, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] += g[e];
    }
    if (have && a.dx) Oct<T>::store(static_cast<T*>(a.dx) + i * a.lddx + col, d);
    if (a.block) {
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum[4][e] = fmaf(d[e], t[e], sum[4][e]);
        d[e] *= a.scale * ls.v[e];
        slope[e] *= d[e] * n[e];
        o[e] = d[e] * s[e];
      }
      if (a.act && a.dgate && have) Oct<T>::store(static_cast<T*>(a.dgate) + i * a.lddg + col, slope);
      if (a.post) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          w[e] = o[e] * qw.v[e];
          sum[2][e] = fmaf(o[e], uo[e], sum[2][e]);
          sum[3][e] += o[e];
        }
        unit_grad<L>(red, w, uo, ro, a.layer, inv_d, o);
      }
      if (have && a.dblock) Oct<T>::store(static_cast<T*>(a.dblock) + i * a.lddb + col, o);
    }
  }
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    if (!a.sums[k]) continue;
    const float by = k == 4 ? a.scale : 1.f;
    float* to = a.part + (static_cast<int64_t>(blockIdx.x) * kSums + k) * a.d;
    if constexpr (kRows > 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) join[team][col + e] = sum[k][e];
      __syncthreads();
      for (int c = threadIdx.x; c < a.d; c += Team<L>::kBlock) {
        float v = 0.f;
#pragma unroll
        for (int m = 0; m < kRows; ++m) v += join[m][c];
        to[c] = v * by;
      }
    } else if (live) {
#pragma unroll
      for (int e = 0; e < 8; ++e) to[col + e] = sum[k][e] * by;
    }
  }
}

// The workgroups' sums added up, in fp64: 32 columns and as many slices of the
// workgroups a workgroup.
constexpr int kCols = 32, kSlices = 32;
__global__ __launch_bounds__(kCols * kSlices) void join_kernel(const NormArgs a, int parts) {
  __shared__ double lds[kSlices][kCols + 1];
  const int c = threadIdx.x % kCols, slice = threadIdx.x / kCols, col = blockIdx.x * kCols + c, k = blockIdx.y;
  float* to = a.sums[k];
  if (!to) return;
  double v = 0.;
  if (col < a.d) {
#pragma unroll 8
    for (int p = slice; p < parts; p += kSlices) v += a.part[(static_cast<int64_t>(p) * kSums + k) * a.d + col];
  }
  lds[slice][c] = v;
  __syncthreads();
  if (slice == 0 && col < a.d) {
    v = 0.;
#pragma unroll
    for (int m = 0; m < kSlices; ++m) v += lds[m][c];
    to[col] = static_cast<float>(v);
  }
}

int team_of(int d) {
  int l = 8;
  while (8 * l < d) l *= 2;
  return l;
}

template <typename T, int L>
hipError_t launch(const NormArgs& a, int grid, bool backward, hipStream_t st) {
  if (backward) backward_kernel<T, L><<<grid, Team<L>::kBlock, 0, st>>>(a);
  else forward_kernel<T, L><<<grid, Team<L>::kBlock, 0, st>>>(a);
  return hipGetLastError();
}

int rows_of(int d) {
  const int l = team_of(d);
  return l > 64 ? 1 : kThreads / l;
}

template <typename T>
hipError_t pick(const NormArgs& a, int grid, bool backward, hipStream_t st) {
  switch (team_of(a.d)) {
    case 8: return launch<T, 8>(a, grid, backward, st);
    case 16: return launch<T, 16>(a, grid, backward, st);
    case 32: return launch<T, 32>(a, grid, backward, st);
    case 64: return launch<T, 64>(a, grid, backward, st);
    case 128: return launch<T, 128>(a, grid, backward, st);
    case 256: return launch<T, 256>(a, grid, backward, st);
    default: return launch<T, 512>(a, grid, backward, st);
  }
}

}  // namespace

// Workgroups of a backward: as many as its registers let run at once, since each
// leaves a row of partial sums (four a CU, with the sums' joining: 407 us for two's
// 402, and 76 for 69 of 8191 rows of 2000).
int norm_partials(int64_t n, int d, int n_cu) {
  return static_cast<int>(std::min<int64_t>(ceil_div(n, rows_of(d)), 2 * static_cast<int64_t>(n_cu)));
}

hipError_t norm_forward(const NormArgs& a, int dtype, int n_cu, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  const int grid = static_cast<int>(std::min<int64_t>(ceil_div(a.n, rows_of(a.d)), 16 * static_cast<int64_t>(n_cu)));
  return dtype == STCA_BF16 ? pick<bf16_bits>(a, grid, false, st) : pick<float>(a, grid, false, st);
}

hipError_t norm_backward(const NormArgs& a, int dtype, int n_cu, hipStream_t st) {
  const int parts = norm_partials(a.n, a.d, n_cu);
  if (parts > 0) {
    const hipError_t e = dtype == STCA_BF16 ? pick<bf16_bits>(a, parts, true, st) : pick<float>(a, parts, true, st);
    if (e != hipSuccess) return e;
  }
  bool any = false;
  for (float* s : a.sums) any |= s != nullptr;
  if (!any) return hipSuccess;
  join_kernel<<<dim3(static_cast<unsigned>(ceil_div(a.d, kCols)), kSums), kCols * kSlices, 0, st>>>(a, parts);
  return hipGetLastError();
}

}  // namespace layers
}  // namespace stca
