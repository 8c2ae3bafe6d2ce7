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
//
// Bound by the bytes of dout and of the distinct rows, which the first level moves
// (528384 tokens of 256 fp32 features, 150 us for
// 691 MB, 4.6 TB/s; 524288 bf16 ones of 16 ids 52 us, 5.2 TB/s); the sort before it
// is latency, 18 us for every 8 bits of the ids, and the levels above 6 to 9 each.
// What the first level measured before its results were written past the caches (us,
// 528384 tokens; 157 then): 512 threads a workgroup and 8 rows on their way 161 for
// 256 and 4 (bf16, 16 ids: 66 for 52, registers for 8 waves a SIMD); the next batch
// fetched before one is added 178.
#include "layer_ops.h"

namespace stca {
namespace layers {

namespace {

constexpr int kThreads = 1024;   // of a sorting workgroup (512: 15 us a pass over 528384 tokens, 1024: 13)
constexpr int kWaves = kThreads / 64;
constexpr int kDigits = 256;
constexpr int kMaxBlocks = 256;  // workgroups of a sort
constexpr int kItems = kEmbedSmall / kThreads;        // tokens a thread of a sort's tile
constexpr int kSmall = kEmbedSmall;
constexpr int kFirstThreads = 256;  // of a summing workgroup of the first level
constexpr int kUpThreads = 1024;    // ... of the levels above: as few of them as may be
constexpr int kNone = -2;        // no row of the result (-1: the last one of the numbering before)

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

// Sum over a wave, in every lane.
__device__ __forceinline__ int wave_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0xb1, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x4e, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x140, 0xf, 0xf, true);
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = r[0] + r[1];
  const auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return q[0] + q[1];
}

// Exclusive prefix sums over a workgroup's threads (a barrier before and after).
template <int kWaves>
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
  for (int i = threadIdx.x; i <= mask; i += kThreads) a.counts[i * kMaxBlocks + blockIdx.x] = cnt[i];
  if (pass == 0 && threadIdx.x == 0) a.bad[blockIdx.x] = any;
}

struct SortLds {
  int cnt[kWaves][kDigits];  // of a wave's tokens of the tile, then of the waves' before it
  int start[kDigits];        // of a digit in the sorted tile
  int waves[kWaves];
  uint64_t buf[kSmall];      // the sorted tile
};

// Sorts a tile of up to kSmall tokens by a digit, in order, into s.buf: get(it, pair)
// gives the wave's it-th 64 tokens.  Returns how many have the digit that is the
// thread's number; s.start says where they begin.
template <typename Get>
__device__ __forceinline__ int sort_tile(SortLds& s, int items, int shift, int bits, Get get) {
  const int wave = threadIdx.x >> 6, mask = (1 << bits) - 1;
  for (int i = threadIdx.x; i < kWaves * kDigits; i += kThreads) (&s.cnt[0][0])[i] = 0;
  __syncthreads();
  uint64_t pair[kItems];
  int rank[kItems], digit[kItems];
  bool valid[kItems];
#pragma unroll
  for (int it = 0; it < kItems; ++it) {
    pair[it] = 0;
    valid[it] = it < items && get(it, pair[it]);
    digit[it] = static_cast<int>(static_cast<uint32_t>(pair[it] >> 32) >> shift) & mask;
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
  const int d = threadIdx.x;
  int all = 0, total;
  if (d < kDigits) {
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int c = s.cnt[w][d];
      s.cnt[w][d] = all;
      all += c;
    }
  }
  const int at = block_prefix<kWaves>(all, s.waves, total);
  if (d < kDigits) s.start[d] = at;
  __syncthreads();
#pragma unroll
  for (int it = 0; it < kItems; ++it)
    if (valid[it]) s.buf[s.start[digit[it]] + s.cnt[wave][digit[it]] + rank[it]] = pair[it];
  __syncthreads();
  return all;
}

__global__ __launch_bounds__(kThreads) void scatter_kernel(const EmbedGradArgs a, const EmbedGradPlan p, int pass) {
  __shared__ SortLds s;
  __shared__ int base[kDigits];    // where the next token of a digit goes
  __shared__ int before[kDigits];  // of the digit, in the workgroups before this one
  const int shift = pass * p.bits, mask = (1 << p.bits) - 1;
  {
    // a wave takes every kWaves-th digit: its counts in all workgroups are one load,
    // four a lane, and all of them are on their way together
    constexpr int kEach = kDigits / kWaves;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = 4 * lane;
    int4 c[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int d = wave + k * kWaves;
      c[k] = make_int4(0, 0, 0, 0);
      if (d <= mask && b < p.blocks) c[k] = *reinterpret_cast<const int4*>(a.counts + d * kMaxBlocks + b);
    }
    const int me = static_cast<int>(blockIdx.x);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int d = wave + k * kWaves;
      if (d > mask) {
        if (lane == 0) base[d] = 0;
        continue;
      }
      const int v[4] = {c[k].x, c[k].y, c[k].z, c[k].w};
      int all = 0, low = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        all += b + e < p.blocks ? v[e] : 0;
        low += b + e < min(me, p.blocks) ? v[e] : 0;
      }
      all = wave_sum(all);
      low = wave_sum(low);
      if (lane == 0) {
        base[d] = all;
        before[d] = low;
      }
    }
    __syncthreads();
    int total;
    const int t = threadIdx.x;
    const int at = block_prefix<kWaves>(t < kDigits ? base[t] : 0, s.waves, total);
    if (t < kDigits) base[t] = at + before[t];
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
    const int all = sort_tile(s, items, shift, p.bits, [&](int it, uint64_t& pair) {
      const int64_t i = tile + wave * (items * 64) + it * 64 + lane;
      bool bad = false;
      if (i < t1) pair = from ? from[i] : pair_of(id_of(a, i, bad), i);
      return i < t1;
    });
    // neighbours in the sorted tile go to neighbouring places (stored one by one from
    // where they were read, 64 places a store, the pass took 15 us for 528384 tokens)
    for (int i = threadIdx.x; i < left; i += kThreads) {
      const uint64_t pair = s.buf[i];
      const int d = static_cast<int>(static_cast<uint32_t>(pair >> 32) >> shift) & mask;
      to[base[d] + i - s.start[d]] = pair;
    }
    __syncthreads();
    if (threadIdx.x < kDigits) base[threadIdx.x] += all;
  }
}

// All passes of up to kSmall tokens by one workgroup, in LDS.
__global__ __launch_bounds__(kThreads) void sort_small_kernel(const EmbedGradArgs a, const EmbedGradPlan p) {
  __shared__ SortLds s;
  const int n = static_cast<int>(a.n), items = (n + kThreads - 1) / kThreads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  bool bad = false;
  for (int pass = 0; pass < p.passes; ++pass)  // (a pass holds its tokens in registers before it writes them)
    sort_tile(s, items, pass * p.bits, p.bits, [&](int it, uint64_t& pair) {
      const int i = wave * (items * 64) + it * 64 + lane;
      if (i < n) pair = pass ? s.buf[i] : pair_of(id_of(a, i, bad), i);
      return i < n;
    });
  const int any = __syncthreads_or(bad);
  if (threadIdx.x == 0 && a.hdr) {
    a.hdr->status = any ? STCA_ERR_INVALID_ARG : STCA_OK;
    a.hdr->range = 0;
  }
  // the rows of the result, and where there are distinct ids their list
  const bool sparse = a.dtable == nullptr;
  int base = 0;
  for (int i0 = 0; i0 < n; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    const uint32_t key = i < n ? static_cast<uint32_t>(s.buf[i] >> 32) : a.n_rows;
    int row = key < a.n_rows ? static_cast<int>(key) : kNone;
    if (sparse) {
      const int first = key < a.n_rows && (i == 0 || static_cast<uint32_t>(s.buf[i - 1] >> 32) != key);
      int total;
      const int x = block_prefix<kWaves>(first, s.waves, total);
      if (row >= 0) row = base + x + first - 1;
      if (first) a.rows[row] = static_cast<int32_t>(key);
      base += total;
    }
    if (i < n) a.tokens[i] = make_int2(row, static_cast<int>(static_cast<uint32_t>(s.buf[i])));
  }
  if (sparse && threadIdx.x == 0) *a.count = base;
}

// ---- rows of the result

// A dense result's rows are the ids.  Of distinct ids, a workgroup numbers those
// that begin among its tokens (of which it takes kThreads at a time) from 0, so
// that a run begun before them has the number -1; head_sum holds how many begin.
__global__ __launch_bounds__(kThreads) void rows_kernel(const EmbedGradArgs a, const EmbedGradPlan p) {
  __shared__ int waves[kWaves];
  const uint64_t* pairs = a.pairs[(p.passes - 1) & 1];
  const int64_t t0 = blockIdx.x * p.head_range, t1 = min(a.n, t0 + p.head_range);
  int base = 0;
  uint64_t next = t0 + threadIdx.x < t1 ? pairs[t0 + threadIdx.x] : 0, next_low = 0;
  if (t0 + threadIdx.x < t1 && t0 + threadIdx.x > 0) next_low = pairs[t0 + threadIdx.x - 1];
  for (int64_t i0 = t0; i0 < t1; i0 += kThreads) {
    const int64_t i = i0 + threadIdx.x;
    const uint64_t w = next, low = next_low;
    if (i + kThreads < t1) {
      next = pairs[i + kThreads];
      next_low = pairs[i + kThreads - 1];
    }
    const uint32_t key = i < t1 ? static_cast<uint32_t>(w >> 32) : a.n_rows;
    const int first = key < a.n_rows && (i == 0 || static_cast<uint32_t>(low >> 32) != key);
    int total;
    const int x = block_prefix<kWaves>(first, waves, total);
    if (i < t1) a.tokens[i] = make_int2(key < a.n_rows ? base + x + first - 1 : kNone, static_cast<int>(static_cast<uint32_t>(w)));
    base += total;
  }
  if (threadIdx.x == 0) a.head_sum[blockIdx.x] = base;
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

// Token i's row of dout.  (Looked up once a token, by one thread: by the lanes that
// load it, the look-up's own loads were three of the four of a row.)
template <typename T>
__device__ __forceinline__ const T* dout_row(const EmbedGradArgs& a, int64_t i) {
  const int q = part_of(a, i);
  return static_cast<const T*>(a.dout[q]) + (i - (q ? a.end[q - 1] : 0)) * a.ld[q];
}

struct Level {
  int64_t n;        // what is added: tokens, or slots of the level before
  int64_t groups;   // workgroups of this level, each of which leaves two slots
  int in, out;      // buffers of slots
  int heads;        // workgroups that numbered distinct ids; 0: rows are known
};

// kFirst: the rows of dout in the order of the sorted tokens; else slots.  W:
// features a lane, L: lanes a team, kTeam: tokens of a team.
template <bool kFirst, typename T, int L, int kTeam>
__global__ __launch_bounds__(kFirst ? kFirstThreads : kUpThreads) void sum_kernel(const EmbedGradArgs a, const EmbedGradPlan p, const Level lv) {
  constexpr int kSumThreads = kFirst ? kFirstThreads : kUpThreads, kSumWaves = kSumThreads / 64;
  constexpr int W = Part<T>::kN, kTeams = kSumThreads / L, kTokens = kTeams * kTeam;
  constexpr int kBatch = kFirst ? 4 : 16;  // rows of a team on their way at a time
  __shared__ int row[kTokens];      // run of a token: its row of the result, -1: none
  __shared__ const T* src[kTokens]; // its value's row, null: none
  __shared__ float head[kTeams][L * W];
  __shared__ int state[kTeams];     // of a team's head: 0 none, 1 it ends there, 2 it goes on
  __shared__ int edge[2], waves[kSumWaves];
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens;
  const int n = static_cast<int>(min<int64_t>(kTokens, lv.n - t0));
  const bool sparse = a.dtable == nullptr;

  if constexpr (kFirst) {
    // (row, token) of the workgroup's tokens, which one workgroup numbered
    const bool numbered = lv.heads > 0, keyed = !p.small && !numbered;
    const uint64_t* pairs = a.pairs[(p.passes - 1) & 1];
    int base = 0;
    if (numbered) {
      const int b = static_cast<int>(t0 / p.head_range);
      int low = 0, all = 0;
      for (int i = threadIdx.x; i < lv.heads; i += kSumThreads) {
        const int c = a.head_sum[i];
        all += c;
        low += i < b ? c : 0;
      }
      block_prefix<kSumWaves>(low, waves, base);
      if (blockIdx.x == 0 && blockIdx.y == 0) {
        int total;
        block_prefix<kSumWaves>(all, waves, total);
        if (threadIdx.x == 0) *a.count = total;
      }
    }
    auto at = [&](int64_t i) {
      if (!keyed) return a.tokens[i];
      const uint64_t w = pairs[i];
      const uint32_t key = static_cast<uint32_t>(w >> 32);
      return make_int2(key < a.n_rows ? static_cast<int>(key) : kNone, static_cast<int>(static_cast<uint32_t>(w)));
    };
    for (int i = threadIdx.x; i < kTokens; i += kSumThreads) {
      int2 w = make_int2(kNone, -1);
      if (i < n) w = at(t0 + i);
      row[i] = w.x == kNone ? -1 : base + w.x;
      src[i] = w.x == kNone ? nullptr : dout_row<T>(a, static_cast<uint32_t>(w.y));
    }
    if (threadIdx.x == 0) {
      // whether the runs of the outermost tokens reach over the workgroup's borders
      const int64_t after = t0 + n;
      auto same = [&](int64_t i) {  // tokens i - 1 and i
        const int r = at(i).x;
        return numbered && i % p.head_range == 0 ? r == -1 : r == at(i - 1).x;
      };
      edge[0] = t0 > 0 && same(t0);
      edge[1] = after < lv.n && same(after);
    }
  } else {
    const int2* slots = a.slot[lv.in];
    for (int i = threadIdx.x; i < kTokens; i += kSumThreads) {
      int2 s = make_int2(-1, 0);
      if (i < n) s = slots[t0 + i];
      row[i] = s.x;
      src[i] = s.x >= 0 && s.y ? reinterpret_cast<const T*>(a.slot_val[lv.in]) + (t0 + i) * a.d : nullptr;
    }
    if (threadIdx.x == 0) {
      const int64_t last = t0 + n - 1;
      edge[0] = t0 > 0 && slots[t0 - 1].x == slots[t0].x;
      edge[1] = last + 1 < lv.n && slots[last + 1].x == slots[last].x;
    }
  }
  if (threadIdx.x < kTeams) state[threadIdx.x] = 0;
  __syncthreads();
  if constexpr (kFirst) {
    if (lv.heads > 0 && blockIdx.y == 0) {  // the list of the distinct ids
      const uint64_t* pairs = a.pairs[(p.passes - 1) & 1];
      for (int i = threadIdx.x; i < n; i += kSumThreads)
        if (row[i] >= 0 && (i ? row[i - 1] != row[i] : !edge[0])) a.rows[row[i]] = static_cast<int32_t>(pairs[t0 + i] >> 32);
    }
  }
  const int lane = threadIdx.x % L, team = threadIdx.x / L;
  const int col = (static_cast<int>(blockIdx.y) * L + lane) * W;
  const bool live = col < a.d;
  auto put = [&](int r, const float* x) {
    if (!live) return;
    float* to = sparse ? a.grads + static_cast<int64_t>(r) * a.d + col : a.dtable + static_cast<int64_t>(r) * a.ldt + col;
#pragma unroll
    for (int e = 0; e < W; e += 4) {
      f32x4 y = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]} * a.scale;
      if (!sparse && a.accumulate) y += *reinterpret_cast<const f32x4*>(to + e);
      __builtin_nontemporal_store(y, reinterpret_cast<f32x4*>(to + e));
    }
  };

  // the team's tokens
  const int i0 = team * kTeam, i1 = min(n, i0 + kTeam);
  bool open = false;  // the run at the team's end began here and goes on
  float acc[W] = {};  // ... and its sum
  if (i0 < n) {
    int cur = row[i0];
    bool begun = i0 == 0 ? edge[0] != 0 : row[i0 - 1] == cur;  // before the team's first token
    auto fetch = [&](Part<T>* v, bool* have, int i) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const T* s = i + k < i1 ? src[i + k] : nullptr;
        have[k] = s && live;
        if (have[k]) v[k].load(s + col);
      }
    };
    auto take = [&](const Part<T>* v, const bool* have, int i) {
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
    };
    for (int i = i0; i < i1; i += kBatch) {
      Part<T> v[kBatch];
      bool have[kBatch];
      fetch(v, have, i);
      take(v, have, i);
    }
    if (cur >= 0) {
      const bool on = i1 < n ? row[i1] == cur : edge[1] != 0;
      if (begun) {
#pragma unroll
        for (int e = 0; e < W; ++e) head[team][lane * W + e] = acc[e];
        if (lane == 0) state[team] = on ? 2 : 1;
      } else if (on) {
        open = true;
      } else {
        put(cur, acc);
      }
    }
  }
  __syncthreads();

  // runs over several teams: the team that began one adds the others' heads; the
  // first team also the run that it found begun
  const int teams = (n + kTeam - 1) / kTeam;
  auto join = [&](float* sum, int at) {  // true: the run ends in this workgroup
    for (; at < teams; ++at) {
#pragma unroll
      for (int e = 0; e < W; ++e) sum[e] += head[at][lane * W + e];
      if (state[at] == 1) return true;
    }
    return false;
  };
  auto leave = [&](int slot, const float* x) {
    if (!live) return;
    float* to = a.slot_val[lv.out] + (2 * static_cast<int64_t>(blockIdx.x) + slot) * a.d + col;
#pragma unroll
    for (int e = 0; e < W; e += 4) *reinterpret_cast<f32x4*>(to + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
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
    float sum[W];
#pragma unroll
    for (int e = 0; e < W; ++e) sum[e] = head[0][lane * W + e];
    if (state[0] == 2) join(sum, 1);
    leave(0, sum);
  }
  if (open) {
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

// Tokens of a team: enough that few runs cross a border and the teams' own cost
// is spread, few where there are few, and where the levels above add sums.
constexpr int kTeamFirst = 32, kTeamSmall = 8, kTeamUp = 16;

template <bool kFirst, typename T, int L>
hipError_t launch_sum(const EmbedGradArgs& a, const EmbedGradPlan& p, const Level& lv, int cols, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(lv.groups), cols);
  if constexpr (!kFirst) sum_kernel<kFirst, T, L, kTeamUp><<<grid, kUpThreads, 0, st>>>(a, p, lv);
  else if (p.small) sum_kernel<kFirst, T, L, kTeamSmall><<<grid, kFirstThreads, 0, st>>>(a, p, lv);
  else sum_kernel<kFirst, T, L, kTeamFirst><<<grid, kFirstThreads, 0, st>>>(a, p, lv);
  return hipGetLastError();
}

// Lanes of a team of W features each, column blocks, and tokens of a workgroup.
struct Shape {
  int lanes, cols;
  int64_t tokens;
};
Shape shape_of(int d, int W, int threads, int team) {
  Shape s{8, 1, 0};
  while (s.lanes < 64 && s.lanes * W < d) s.lanes *= 2;
  s.cols = static_cast<int>(ceil_div(d, s.lanes * W));
  s.tokens = threads / s.lanes * team;
  return s;
}

template <bool kFirst, typename T>
hipError_t sum_level(const EmbedGradArgs& a, const EmbedGradPlan& p, const Level& lv, hipStream_t st) {
  const Shape s = shape_of(a.d, Part<T>::kN, 1, 1);
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
  const int64_t tokens = shape_of(d, dtype == STCA_BF16 ? 8 : 4, kFirstThreads, p.small ? kTeamSmall : kTeamFirst).tokens;
  p.groups = ceil_div(n, tokens);
  p.next_groups = ceil_div(2 * p.groups, shape_of(d, 4, kUpThreads, kTeamUp).tokens);
  p.head_range = std::max<int64_t>(tokens, round_up(ceil_div(n, kMaxBlocks), tokens));
  p.heads = p.small ? 0 : static_cast<int>(ceil_div(n, p.head_range));
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
  Level lv{a.n, p.groups, 0, 0, 0};
  if (!a.dtable && !p.small) {
    lv.heads = p.heads;
    rows_kernel<<<p.heads, kThreads, 0, st>>>(a, p);
  }
  e = dtype == STCA_BF16 ? sum_level<true, bf16_bits>(a, p, lv, st) : sum_level<true, float>(a, p, lv, st);
  const int64_t up = shape_of(a.d, 4, kUpThreads, kTeamUp).tokens;
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
