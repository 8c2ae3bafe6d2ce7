// Attention of a request's new tokens over its rows of a paged cache, bf16 or
// 8-bit pages (see attn_fwd.h).
#include "attn_fwd.h"

namespace stca {
namespace ops {

namespace {

template <int KV, int DH>
hipError_t attend_dh(const AttnArgs& a, int tiles, hipStream_t st) {
  if (tiles == 2) return launch_fwd<bf16_bits, KV, DH, 2>(a, st);
  return launch_fwd<bf16_bits, KV, DH, 1>(a, st);
}

template <int KV>
hipError_t attend(const AttnArgs& a, int dh, int tiles, hipStream_t st) {
  if (dh == 32) return attend_dh<KV, 32>(a, tiles, st);
  if (dh == 64) return attend_dh<KV, 64>(a, tiles, st);
  return attend_dh<KV, 128>(a, tiles, st);
}

}  // namespace

hipError_t cache_attend(const AttnArgs& a, bool int8, int dh, int tiles, hipStream_t st) {
  return int8 ? attend<kPagedInt8>(a, dh, tiles, st) : attend<kPagedBf16>(a, dh, tiles, st);
}

}  // namespace ops
}  // namespace stca
