// Internal interface of the operators between ids, rows and gradients
// (stca_embed_*, stca_norm_*, stca_clip): kernel arguments, launchers and the
// device code that they share (wide loads, sums over a team of lanes).
#pragma once

#include <algorithm>

#include "common.h"

namespace stca {
namespace layers {

constexpr int kMaxFields = 8;
constexpr int kMaxParts = 4;

// ---- embedding rows
struct EmbedArgs {
  const void* table[kMaxFields];
  const int32_t* ids[kMaxFields];
  int64_t ld[kMaxFields];       // row strides in elements
  uint32_t n_rows[kMaxFields];
  int32_t n_fields, d;
  int64_t n, ldo;
  float scale;
  void* out;
  WsHeader* hdr;                // nullable
};
hipError_t embed_forward(const EmbedArgs& a, int table_dtype, int out_dtype, int n_cu, hipStream_t st);

// ---- the gradient of a table
struct EmbedGradArgs {
  const int32_t* ids[kMaxParts];
  const void* dout[kMaxParts];
  int64_t ld[kMaxParts];
  int64_t end[kMaxParts];       // tokens of the parts up to this one; the last ones hold n
  int64_t n;                    // tokens of all parts
  int32_t d;
  uint32_t n_rows;
  float scale;
  // dense: [n_rows][ldt], added to where `accumulate`
  float* dtable;
  int64_t ldt;
  int32_t accumulate;
  // sparse (dtable null)
  int32_t* rows;
  float* grads;
  int32_t* count;
  // workspace
  WsHeader* hdr;
  int32_t* counts;              // [digits][256 blocks]
  int32_t* bad;                 // [blocks]
  uint64_t* pairs[2];           // id in the high half, token in the low one
  int2* tokens;                 // row of the result and token, in sorted order (not of a long list for a dense result)
  int32_t* head_sum;            // distinct ids that each numbering workgroup found
  int2* slot[2];                // per workgroup of a level two: run's row, whether there is a value
  float* slot_val[2];
};
constexpr int kEmbedSmall = 4096;  // up to so many tokens are sorted by one workgroup
// Sizes that the workspace and the launches agree on.
struct EmbedGradPlan {
  int blocks, passes, bits;     // sort: workgroups, digits and bits a digit
  int64_t range;                // tokens of a workgroup
  bool small;                   // sorted by one workgroup
  int64_t groups, next_groups;  // summing workgroups of the first level and the next
  int64_t head_range;           // tokens of a numbering workgroup: whole summing workgroups'
  int heads;                    // numbering workgroups
};
EmbedGradPlan embed_grad_plan(int64_t n, uint32_t n_rows, int d, int dtype);
hipError_t embed_grad(const EmbedGradArgs& a, int dtype, hipStream_t st);

// ---- norms around a block
struct NormArgs {
  const void *x, *block, *gate, *dh, *dy;
  int64_t ldx, ldb, ldg, lddh, lddy;
  void *h, *y, *dx, *dblock, *dgate;
  int64_t ldh, ldy, lddx, lddb, lddg;
  const float *pre_w, *pre_b, *post_w, *post_b, *ls;  // nullable: ones, zeros
  int64_t n;
  int32_t d, layer, act, post, pre;                   // act: 0 none, 1 sigmoid, 2 silu
  float scale, eps;
  float* part;                                        // [workgroups][sums][d]
  float* sums[5];                                     // gradients of pre_w, pre_b, post_w, post_b, ls; nullable
};
int norm_partials(int64_t n, int d, int n_cu);        // workgroups of a backward
hipError_t norm_forward(const NormArgs& a, int dtype, int n_cu, hipStream_t st);
hipError_t norm_backward(const NormArgs& a, int dtype, int n_cu, hipStream_t st);

// ---- the norm of many gradients
struct Grad {
  const void* g;
  void* out;
  const int32_t* count;         // nullable: rows in use
  int64_t n;                    // elements
  int32_t per;                  // elements of a row, with a count
  int32_t flags;                // 1: bf16, 2: out is bf16
  int64_t start;                // pieces of the tensors before this one
};
constexpr int kGradsPerLaunch = 64;
constexpr int kGradPiece = 8192;    // elements of a piece
constexpr int kGradGroups = 2048;   // workgroups of a launch
struct ClipArgs {
  Grad t[kGradsPerLaunch];
  int32_t n_t;
  int64_t pieces;
  double max_norm;
  double* part;                 // partial sums of this launch on; of all in the scaling
  int32_t n_part;
  float* norm;                  // nullable: written by another launch
};
hipError_t clip_sum(const ClipArgs& a, int grid, hipStream_t st);
hipError_t clip_scale(const ClipArgs& a, int grid, hipStream_t st);

// ---- device code

__device__ __forceinline__ float lo_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 p = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
  return __builtin_bit_cast(uint32_t, p);
}

// Eight features as they lie in memory (16-byte aligned), and as floats.
template <typename T> struct Oct;
template <> struct Oct<bf16_bits> {
  uint4 w;
  __device__ __forceinline__ void load(const bf16_bits* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { w = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = lo_of(w.x), x[1] = hi_of(w.x), x[2] = lo_of(w.y), x[3] = hi_of(w.y);
    x[4] = lo_of(w.z), x[5] = hi_of(w.z), x[6] = lo_of(w.w), x[7] = hi_of(w.w);
  }
  static __device__ __forceinline__ void store(bf16_bits* p, const float* x) {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    const words w = {two_bf16(x[0], x[1]), two_bf16(x[2], x[3]), two_bf16(x[4], x[5]), two_bf16(x[6], x[7])};
    __builtin_nontemporal_store(w, reinterpret_cast<words*>(p));
  }
};
template <> struct Oct<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const f32x4*>(p)[0];
    b = reinterpret_cast<const f32x4*>(p)[1];
  }
  __device__ __forceinline__ void zero() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  }
  static __device__ __forceinline__ void store(float* p, const float* x) {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{x[0], x[1], x[2], x[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{x[4], x[5], x[6], x[7]};
  }
};

template <int kCtrl>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, 0xf, 0xf, true));
}

// Sum over aligned teams of L lanes (a power of two up to 64), in every lane and
// in the same order in each: neighbours, pairs, then mirrored halves of 8 and 16
// lanes, which by then hold one value each, then the rows of 16 and the halves.
template <int L>
__device__ __forceinline__ float team_sum(float x) {
  if constexpr (L >= 2) x += dpp<0xb1>(x);    // quad_perm 1 0 3 2
  if constexpr (L >= 4) x += dpp<0x4e>(x);    // quad_perm 2 3 0 1
  if constexpr (L >= 8) x += dpp<0x141>(x);   // row_half_mirror
  if constexpr (L >= 16) x += dpp<0x140>(x);  // row_mirror
  if constexpr (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

}  // namespace layers
}  // namespace stca
