// The gradient of an embedding table: dT[v] = scale sum over the tokens i with
// id v of dout_i, the tokens of up to four parts one after the other.
//
// The tokens are sorted by their ids (a stable radix sort of (id, token) pairs,
// so that a row's tokens keep their order), and the rows of dout are added run by
// run.  A workgroup takes a fixed number of sorted tokens, whatever runs they
// belong to, a team of lanes 32 of them; runs that end where they began are
// written at once, the others leave up to two sums a team in LDS (that of the run
// it found begun, its head, and that of the run that it leaves open, its tail)
// and then two a workgroup, which the next level adds the same way.  So the work
// is even, whether every id is another or all are the same, nothing is added
// atomically, and the order of a row's sum depends on the tokens alone.
#include "layer_ops.h"

namespace stca {
namespace layers {

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kDigits = 256;
constexpr int kMaxBlocks = 256;  // workgroups of a sort
constexpr int kItems = 8;        // tokens a thread of a sort's tile
constexpr int kSmall = kThreads * kItems;
constexpr int kTeamTokens = 32;

__device__ __forceinline__ int part_of(const EmbedGradArgs& a, int64_t i) {
  return (i >= a.end[0]) + (i >= a.end[1]) + (i >= a.end[2]);
}

// Id of a token; n_rows, which sorts behind every row, for one without a row.
__device__ __forceinline__ uint32_t id_of(const EmbedGradArgs& a, int64_t i, bool& bad) {
  const int p = part_of(a, i);
  const int32_t id = a.ids[p][i - (p ? a.end[p - 1] : 0)];
  const bool have = id >= 0 && static_cast<uint32_t>(id) < a.n_rows;
  bad |= id >= 0 && !have;
  return have ? static_cast<uint32_t>(id) : a.n_rows;
}

__device__ __forceinline__ uint64_t pair_of(uint32_t id, int64_t i) {
  return static_cast<uint64_t>(id) << 32 | static_cast<uint32_t>(i);
}

// Lanes of the wave whose digit is this lane's, among the valid ones.
__device__ __forceinline__ uint64_t peers(uint32_t digit, int bits, bool valid) {
  uint64_t m = __ballot(valid);
  for (int b = 0; b < bits; ++b) {
    const uint64_t on = __ballot(digit >> b & 1);
    m &= digit >> b & 1 ? on : ~on;
  }
  return m;
}

__device__ __forceinline__ int lanes_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), 0));
}

// Exclusive prefix sums over the kThreads threads (a barrier before and after).
__device__ __forceinline__ int block_prefix(int v, int* waves, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? waves[w] : 0;
    total += waves[w];
  }
  return before + x - v;
}

// ---- sort

// Counts of the digits of a workgroup's tokens.
__global__ __launch_bounds__(kThreads) void count_kernel(const EmbedGradArgs a, const EmbedGradPlan p, int pass) {
  __shared__ int cnt[kDigits];
  for (int i = threadIdx.x; i < kDigits; i += kThreads) cnt[i] = 0;
  __syncthreads();
  const int64_t t0 = blockIdx.x * p.range, t1 = min(a.n, t0 + p.range);
  const int shift = pass * p.bits, mask = (1 << p.bits) - 1;
  bool bad = false;
  for (int64_t i = t0 + threadIdx.x; i < t1; i += kThreads) {
    const uint32_t id = pass == 0 ? id_of(a, i, bad) : static_cast<uint32_t>(a.pairs[(pass - 1) & 1][i] >> 32);
    atomicAdd(&cnt[id >> shift & mask], 1);
  }
  const int any = __syncthreads_or(bad);
  for (int i = threadIdx.x; i < kDigits; i += kThreads) a.counts[blockIdx.x * kDigits + i] = cnt[i];
  if (pass == 0 && threadIdx.x == 0) a.bad[blockIdx.x] = any;
}

struct SortLds {
  int cnt[kWaves][kDigits];  // of a wave's tokens of the tile, then where its first one goes
  int base[kDigits];         // where the next token of a digit goes
  int waves[kWaves];
};

// Ranks a tile's tokens by their digits, in order: `item`(it) gives the wave's
// it-th 64 tokens, `put`(it, place) takes each token's place.
template <typename Digit, typename Put>
__device__ __forceinline__ void place_tile(SortLds& s, int items, int bits, Digit digit_of, Put put) {
  const int wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < kWaves * kDigits; i += kThreads) (&s.cnt[0][0])[i] = 0;
  __syncthreads();
  int rank[kItems];
  uint32_t digit[kItems];
  bool valid[kItems];
#pragma unroll
  for (int it = 0; it < kItems; ++it) {
    valid[it] = false;
    digit[it] = 0;
    if (it < items) valid[it] = digit_of(it, digit[it]);
  }
#pragma unroll
  for (int it = 0; it < kItems; ++it) {
    if (it >= items) continue;
    const uint64_t same = peers(digit[it], bits, valid[it]);
    const int below = lanes_below(same);
    if (valid[it]) rank[it] = s.cnt[wave][digit[it]] + below;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // every lane has read before the first one counts on
    if (valid[it] && below == 0) s.cnt[wave][digit[it]] = rank[it] + __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  __syncthreads();
  for (int d = threadIdx.x; d < kDigits; d += kThreads) {
    int at = s.base[d];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int c = s.cnt[w][d];
      s.cnt[w][d] = at;
      at += c;
    }
    s.base[d] = at;
  }
  __syncthreads();
#pragma unroll
  for (int it = 0; it < kItems; ++it)
    if (it < items && valid[it]) put(it, s.cnt[wave][digit[it]] + rank[it]);
  __syncthreads();
}

__global__ __launch_bounds__(kThreads) void scatter_kernel(const EmbedGradArgs a, const EmbedGradPlan p, int pass) {
  __shared__ SortLds s;
  __shared__ int part[2][kThreads];  // totals of half of the blocks, and of those before this one
  const int shift = pass * p.bits, mask = (1 << p.bits) - 1;
  {
    // threads t and t + 256 add digit t's counts of every other block
    const int d = threadIdx.x % kDigits, half = threadIdx.x / kDigits;
    int all = 0, before = 0;
#pragma unroll 8
    for (int b = half; b < p.blocks; b += kThreads / kDigits) {
      const int c = a.counts[b * kDigits + d];
      all += c;
      before += b < static_cast<int>(blockIdx.x) ? c : 0;
    }
    part[0][threadIdx.x] = all;
    part[1][threadIdx.x] = before;
    __syncthreads();
    int total;
    const int t = threadIdx.x;
    const int mine = t < kDigits ? part[0][t] + part[0][t + kDigits] : 0;
    const int at = block_prefix(mine, s.waves, total);
    if (t < kDigits) s.base[t] = at + part[1][t] + part[1][t + kDigits];
  }
  if (pass == 0 && blockIdx.x == 0 && a.hdr) {
    int bad = 0;
    for (int b = threadIdx.x; b < p.blocks; b += kThreads) bad |= a.bad[b];
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
      a.hdr->status = bad ? STCA_ERR_INVALID_ARG : STCA_OK;
      a.hdr->range = 0;
    }
  }
  __syncthreads();
  const int64_t t0 = blockIdx.x * p.range, t1 = min(a.n, t0 + p.range);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t* from = pass ? a.pairs[(pass - 1) & 1] : nullptr;
  uint64_t* to = a.pairs[pass & 1];
  for (int64_t tile = t0; tile < t1; tile += kSmall) {
    const int left = static_cast<int>(min<int64_t>(kSmall, t1 - tile));
    const int items = (left + kThreads - 1) / kThreads;  // of 64 tokens, a wave
    uint64_t pair[kItems];
    place_tile(
        s, items, p.bits,
        [&](int it, uint32_t& digit) {
          const int64_t i = tile + wave * (items * 64) + it * 64 + lane;
          if (i >= t1) return false;
          bool bad = false;
          pair[it] = from ? from[i] : pair_of(id_of(a, i, bad), i);
          digit = static_cast<uint32_t>(pair[it] >> 32) >> shift & mask;
          return true;
        },
        [&](int it, int place) { to[place] = pair[it]; });
  }
}

// All passes of up to kSmall tokens by one workgroup, in LDS.
__global__ __launch_bounds__(kThreads) void sort_small_kernel(const EmbedGradArgs a, const EmbedGradPlan p) {
  __shared__ SortLds s;
  __shared__ uint64_t buf[kSmall];  // (a pass holds it in registers before it writes)
  const int n = static_cast<int>(a.n), items = (n + kThreads - 1) / kThreads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, mask = (1 << p.bits) - 1;
  bool bad = false;
  for (int i = threadIdx.x; i < n; i += kThreads) buf[i] = pair_of(id_of(a, i, bad), i);
  const int any = __syncthreads_or(bad);
  if (threadIdx.x == 0 && a.hdr) {
    a.hdr->status = any ? STCA_ERR_INVALID_ARG : STCA_OK;
    a.hdr->range = 0;
  }
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.bits;
    for (int i = threadIdx.x; i < kDigits; i += kThreads) s.base[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) atomicAdd(&s.base[static_cast<uint32_t>(buf[i] >> 32) >> shift & mask], 1);
    __syncthreads();
    int total;
    const int t = threadIdx.x;
    const int at = block_prefix(t < kDigits ? s.base[t] : 0, s.waves, total);
    if (t < kDigits) s.base[t] = at;
    __syncthreads();
    uint64_t pair[kItems];
    place_tile(
        s, items, p.bits,
        [&](int it, uint32_t& digit) {
          const int i = wave * (items * 64) + it * 64 + lane;
          if (i >= n) return false;
          pair[it] = buf[i];
          digit = static_cast<uint32_t>(pair[it] >> 32) >> shift & mask;
          return true;
        },
        [&](int it, int place) { buf[place] = pair[it]; });
  }
  for (int i = threadIdx.x; i < n; i += kThreads) a.pairs[(p.passes - 1) & 1][i] = buf[i];
}

// ---- the distinct ids before each summing workgroup's tokens

__device__ __forceinline__ uint32_t key_at(const uint64_t* pairs, int64_t i) {
  return static_cast<uint32_t>(pairs[i] >> 32);
}
// Token i is the first one of a row.
__device__ __forceinline__ bool head_at(const uint64_t* pairs, int64_t i, uint32_t n_rows) {
  const uint32_t k = key_at(pairs, i);
  return k < n_rows && (i == 0 || key_at(pairs, i - 1) != k);
}

__global__ __launch_bounds__(kThreads) void heads_kernel(const EmbedGradArgs a, const EmbedGradPlan p, int64_t per) {
  __shared__ int waves[kWaves];
  const uint64_t* pairs = a.pairs[(p.passes - 1) & 1];
  const int64_t g0 = blockIdx.x * per, g1 = min(p.groups, g0 + per);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t g = g0 + wave; g < g1; g += kWaves) {
    int c = 0;
    const int64_t t1 = min(a.n, (g + 1) * p.tokens);
    for (int64_t i = g * p.tokens + lane; i < t1; i += 64) c += head_at(pairs, i, a.n_rows);
#pragma unroll
    for (int o = 32; o > 0; o /= 2) c += __shfl_xor(c, o);
    if (lane == 0) a.head_off[g] = c;
  }
  __syncthreads();
  int before = 0;
  for (int64_t g = g0; g < g1; g += kThreads) {
    const int64_t at = g + threadIdx.x;
    int total;
    const int x = block_prefix(at < g1 ? a.head_off[at] : 0, waves, total);
    if (at < g1) a.head_off[at] = before + x;
    before += total;
  }
  if (threadIdx.x == 0) a.head_sum[blockIdx.x] = before;
}

// ---- sums

// Features of a lane: 16 bytes of what is added.
template <typename T> struct Part;
template <> struct Part<float> {
  static constexpr int kN = 4;
  f32x4 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const f32x4*>(p); }
  __device__ __forceinline__ void add_to(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] += v[i];
  }
};
template <> struct Part<bf16_bits> {
  static constexpr int kN = 8;
  Oct<bf16_bits> v;
  __device__ __forceinline__ void load(const bf16_bits* p) { v.load(p); }
  __device__ __forceinline__ void add_to(float* x) const {
    float y[8];
    v.get(y);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] += y[i];
  }
};

struct Level {
  int64_t n;        // what is added: tokens, or slots of the level before
  int64_t groups;   // workgroups of this level, each of which leaves two slots
  int in, out;      // buffers of slots
  int blocks;       // of head_sum; 0: every workgroup counts for itself
  int64_t per;      // workgroups of a block
};

// kFirst: the rows of dout in the order of the sorted tokens; else slots.  W:
// features a lane, L: lanes a team.
template <bool kFirst, typename T, int L>
__global__ __launch_bounds__(kThreads) void sum_kernel(const EmbedGradArgs a, const EmbedGradPlan p, const Level lv) {
  constexpr int W = Part<T>::kN, kTeams = kThreads / L, kTokens = kTeams * kTeamTokens;
  constexpr int kBatch = 8;
  __shared__ int row[kTokens];      // run of a token: its row of the result, -1: none
  __shared__ int src[kTokens];      // where its value lies, -1: none
  __shared__ float head[kTeams][L * W], tail[kTeams][L * W];
  __shared__ int state[kTeams];     // of a team's head: 0 none, 1 it ends there, 2 it goes on
  __shared__ int edge[2], waves[kWaves];
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens;
  const int n = static_cast<int>(min<int64_t>(kTokens, lv.n - t0));
  const uint64_t* pairs = kFirst ? a.pairs[(p.passes - 1) & 1] : nullptr;
  const int2* slots = kFirst ? nullptr : a.slot[lv.in];
  const bool sparse = a.dtable == nullptr;

  if constexpr (kFirst) {
    int base = 0;
    if (sparse) {
      // distinct ids before this workgroup's, and of all
      int before = 0, all = 0, part = 0;
      if (lv.blocks > 0) {
        const int b = static_cast<int>(blockIdx.x / lv.per);
        for (int i = threadIdx.x; i < lv.blocks; i += kThreads) {
          const int c = a.head_sum[i];
          before += i < b ? c : 0;
          all += c;
        }
        part = a.head_off[blockIdx.x];
      } else {
        for (int64_t i = threadIdx.x; i < lv.n; i += kThreads) {
          const int c = head_at(pairs, i, a.n_rows);
          before += i < t0 ? c : 0;
          all += c;
        }
      }
      int total;
      block_prefix(before, waves, total);
      base = total + part;
      block_prefix(all, waves, total);
      if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.count = total;
    }
    for (int i0 = 0; i0 < kTokens; i0 += kThreads) {
      const int i = i0 + threadIdx.x;
      uint32_t key = a.n_rows;
      int64_t tok = 0;
      int first = 0;
      if (i < n) {
        const uint64_t w = pairs[t0 + i];
        key = static_cast<uint32_t>(w >> 32);
        tok = static_cast<uint32_t>(w);
        first = sparse && head_at(pairs, t0 + i, a.n_rows);
      }
      int r = key < a.n_rows ? static_cast<int>(key) : -1;
      if (sparse) {
        int total;
        const int x = block_prefix(first, waves, total);
        if (r >= 0) {
          r = base + x + first - 1;
          if (first && blockIdx.y == 0) a.rows[r] = static_cast<int32_t>(key);
        }
        base += total;
      }
      if (i < kTokens) {  // (a workgroup of wide rows has fewer tokens than threads)
        row[i] = r;
        src[i] = r >= 0 ? static_cast<int>(tok) : -1;
      }
    }
    if (threadIdx.x == 0) {
      // rows of the neighbours on both sides, as far as they are those of the outermost tokens
      const int64_t last = t0 + n - 1;
      edge[0] = t0 > 0 && key_at(pairs, t0 - 1) == key_at(pairs, t0);
      edge[1] = last + 1 < lv.n && key_at(pairs, last + 1) == key_at(pairs, last);
    }
  } else {
    for (int i = threadIdx.x; i < kTokens; i += kThreads) {
      int2 s = make_int2(-1, 0);
      if (i < n) s = slots[t0 + i];
      row[i] = s.x;
      src[i] = s.x >= 0 && s.y ? static_cast<int>(t0 + i) : -1;
    }
    if (threadIdx.x == 0) {
      const int64_t last = t0 + n - 1;
      edge[0] = t0 > 0 && slots[t0 - 1].x == slots[t0].x;
      edge[1] = last + 1 < lv.n && slots[last + 1].x == slots[last].x;
    }
  }
  if (threadIdx.x < kTeams) state[threadIdx.x] = 0;
  __syncthreads();

  const int lane = threadIdx.x % L, team = threadIdx.x / L;
  const int col = (static_cast<int>(blockIdx.y) * L + lane) * W;
  const bool live = col < a.d;
  auto load = [&](int at) {
    Part<T> v;
    if constexpr (kFirst) {
      const int64_t i = static_cast<uint32_t>(at);
      const int q = part_of(a, i);
      v.load(static_cast<const T*>(a.dout[q]) + (i - (q ? a.end[q - 1] : 0)) * a.ld[q] + col);
    } else {
      v.load(reinterpret_cast<const T*>(a.slot_val[lv.in]) + static_cast<int64_t>(at) * a.d + col);
    }
    return v;
  };
  auto put = [&](int r, const float* x) {
    if (!live) return;
    float* to = sparse ? a.grads + static_cast<int64_t>(r) * a.d + col : a.dtable + static_cast<int64_t>(r) * a.ldt + col;
#pragma unroll
    for (int e = 0; e < W; e += 4) {
      f32x4 y = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]} * a.scale;
      if (!sparse && a.accumulate) y += *reinterpret_cast<const f32x4*>(to + e);
      *reinterpret_cast<f32x4*>(to + e) = y;
    }
  };

  // the team's tokens
  const int i0 = team * kTeamTokens, i1 = min(n, i0 + kTeamTokens);
  bool open = false;  // the run at the team's end began here and goes on
  if (i0 < n) {
    float acc[W] = {};
    int cur = row[i0];
    bool begun = i0 == 0 ? edge[0] != 0 : row[i0 - 1] == cur;  // before the team's first token
    for (int i = i0; i < i1; i += kBatch) {
      Part<T> v[kBatch];
      bool have[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int s = i + k < i1 ? src[i + k] : -1;
        have[k] = s != -1 && live;
        if (have[k]) v[k] = load(s);
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (i + k >= i1) break;
        const int r = row[i + k];
        if (r != cur) {
          if (cur >= 0) {
            if (begun) {
#pragma unroll
              for (int e = 0; e < W; ++e) head[team][lane * W + e] = acc[e];
              if (lane == 0) state[team] = 1;
            } else {
              put(cur, acc);
            }
          }
          begun = false;
          cur = r;
#pragma unroll
          for (int e = 0; e < W; ++e) acc[e] = 0.f;
        }
        if (have[k]) v[k].add_to(acc);
      }
    }
    if (cur >= 0) {
      const bool on = i1 < n ? row[i1] == cur : edge[1] != 0;
      if (begun || on) {
        float* to = begun ? head[team] : tail[team];
#pragma unroll
        for (int e = 0; e < W; ++e) to[lane * W + e] = acc[e];
        if (begun && lane == 0) state[team] = on ? 2 : 1;
        open = !begun;
      } else {
        put(cur, acc);
      }
    }
  }
  __syncthreads();

  // runs over several teams: the team that began one adds the others' heads; the
  // first team also the run that it found begun
  const int teams = (n + kTeamTokens - 1) / kTeamTokens;
  auto join = [&](float* acc, int at) {  // true: the run ends in this workgroup
    for (; at < teams; ++at) {
#pragma unroll
      for (int e = 0; e < W; ++e) acc[e] += head[at][lane * W + e];
      if (state[at] == 1) return true;
    }
    return false;
  };
  auto leave = [&](int slot, const float* acc) {
    if (!live) return;
    float* to = a.slot_val[lv.out] + (2 * static_cast<int64_t>(blockIdx.x) + slot) * a.d + col;
#pragma unroll
    for (int e = 0; e < W; e += 4) *reinterpret_cast<f32x4*>(to + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
  };
  const bool note = lane == 0 && blockIdx.y == 0 && lv.groups > 1;
  int2* made = lv.groups > 1 ? a.slot[lv.out] + 2 * static_cast<int64_t>(blockIdx.x) : nullptr;
  if (note && team == 0) {
    // the run that goes on behind the last token, of which the tail slot has a value
    // only if it began here
    const int r = edge[1] ? row[n - 1] : -1;
    int through = edge[0] && r >= 0 && row[0] == r;  // it was begun before the first token
    made[0] = make_int2(edge[0] ? row[0] : -1, 1);
    made[1] = make_int2(r, !through);
  }
  if (team == 0 && state[0] != 0) {
    float acc[W];
#pragma unroll
    for (int e = 0; e < W; ++e) acc[e] = head[0][lane * W + e];
    if (state[0] == 2) join(acc, 1);
    leave(0, acc);
  }
  if (open) {
    float acc[W];
#pragma unroll
    for (int e = 0; e < W; ++e) acc[e] = tail[team][lane * W + e];
    if (join(acc, team + 1)) put(row[i1 - 1], acc);
    else leave(1, acc);
  }
}

__global__ __launch_bounds__(256) void clear_kernel(const EmbedGradArgs a) {
  if (a.dtable && !a.accumulate) {
    const int64_t quads = a.d / 4, all = quads * a.n_rows;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < all; i += gridDim.x * 256ll) {
      const int64_t r = i / quads, c = i % quads;
      *reinterpret_cast<f32x4*>(a.dtable + r * a.ldt + 4 * c) = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  if (a.n == 0 && blockIdx.x == 0 && threadIdx.x == 0) {
    if (a.count) *a.count = 0;
    if (a.hdr) a.hdr->status = STCA_OK, a.hdr->range = 0;
  }
}

template <bool kFirst, typename T, int L>
hipError_t launch_sum(const EmbedGradArgs& a, const EmbedGradPlan& p, const Level& lv, int cols, hipStream_t st) {
  sum_kernel<kFirst, T, L><<<dim3(static_cast<unsigned>(lv.groups), cols), kThreads, 0, st>>>(a, p, lv);
  return hipGetLastError();
}

// Lanes of a team of W features each, column blocks, and tokens of a workgroup.
struct Shape {
  int lanes, cols;
  int64_t tokens;
};
Shape shape_of(int d, int W) {
  Shape s{8, 1, 0};
  while (s.lanes < 64 && s.lanes * W < d) s.lanes *= 2;
  s.cols = static_cast<int>(ceil_div(d, s.lanes * W));
  s.tokens = kThreads / s.lanes * kTeamTokens;
  return s;
}

template <bool kFirst, typename T>
hipError_t sum_level(const EmbedGradArgs& a, const EmbedGradPlan& p, const Level& lv, hipStream_t st) {
  const Shape s = shape_of(a.d, Part<T>::kN);
  if (s.lanes == 8) return launch_sum<kFirst, T, 8>(a, p, lv, s.cols, st);
  if (s.lanes == 16) return launch_sum<kFirst, T, 16>(a, p, lv, s.cols, st);
  if (s.lanes == 32) return launch_sum<kFirst, T, 32>(a, p, lv, s.cols, st);
  return launch_sum<kFirst, T, 64>(a, p, lv, s.cols, st);
}

}  // namespace

EmbedGradPlan embed_grad_plan(int64_t n, uint32_t n_rows, int d, int dtype) {
  EmbedGradPlan p{};
  const int bits = 32 - __builtin_clz(n_rows);  // (n_rows itself is a key)
  p.passes = (bits + 7) / 8;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.small = n <= kSmall;
  p.blocks = static_cast<int>(std::min<int64_t>(kMaxBlocks, std::max<int64_t>(1, ceil_div(n, kSmall / 2))));
  p.range = ceil_div(n, p.blocks);
  const Shape s = shape_of(d, dtype == STCA_BF16 ? 8 : 4), up = shape_of(d, 4);
  p.tokens = s.tokens;
  p.groups = ceil_div(n, s.tokens);
  p.next_groups = ceil_div(2 * p.groups, up.tokens);
  p.head_blocks = p.small ? 0 : static_cast<int>(std::min<int64_t>(kMaxBlocks, p.groups));
  return p;
}

hipError_t embed_grad(const EmbedGradArgs& a, int dtype, hipStream_t st) {
  const EmbedGradPlan p = embed_grad_plan(a.n, a.n_rows, a.d, dtype);
  if (a.n == 0 || (a.dtable && !a.accumulate)) {
    const int64_t all = a.dtable && !a.accumulate ? ceil_div(static_cast<int64_t>(a.n_rows) * a.d / 4, 256) : 1;
    clear_kernel<<<static_cast<unsigned>(std::min<int64_t>(all, 8192)), 256, 0, st>>>(a);
    if (a.n == 0) return hipGetLastError();
  }
  if (p.small) {
    sort_small_kernel<<<1, kThreads, 0, st>>>(a, p);
  } else {
    for (int pass = 0; pass < p.passes; ++pass) {
      count_kernel<<<p.blocks, kThreads, 0, st>>>(a, p, pass);
      scatter_kernel<<<p.blocks, kThreads, 0, st>>>(a, p, pass);
    }
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  Level lv{a.n, p.groups, 0, 0, 0, 0};
  if (!a.dtable && p.head_blocks > 0) {
    lv.per = ceil_div(p.groups, p.head_blocks);
    lv.blocks = static_cast<int>(ceil_div(p.groups, lv.per));
    heads_kernel<<<lv.blocks, kThreads, 0, st>>>(a, p, lv.per);
  }
  e = dtype == STCA_BF16 ? sum_level<true, bf16_bits>(a, p, lv, st) : sum_level<true, float>(a, p, lv, st);
  const int64_t up = shape_of(a.d, 4).tokens;
  while (e == hipSuccess && lv.groups > 1) {
    lv.n = 2 * lv.groups;
    lv.groups = ceil_div(lv.n, up);
    lv.in = lv.out;
    lv.out ^= 1;
    e = sum_level<false, float>(a, p, lv, st);
  }
  return e;
}

}  // namespace layers
}  // namespace stca
