// The compiled instances of the multi-head attention kernels of 16-bit types,
// each type and direction in a source file of its own (they take the longest
// to compile).
#pragma once

#include <cmath>

#include "sm_heads.hpp"

namespace smx {

// Where the keys lie (kPacked, kBlocks, kSmallBlocks of sm_heads_mfma.hpp).
const void* heads_fwd_f16(const HeadsArgs& a, int where);
const void* heads_fwd_bf16(const HeadsArgs& a, int where);
const void* heads_dq_f16(const HeadsArgs& a);
const void* heads_dq_bf16(const HeadsArgs& a);
const void* heads_dkv_f16(const HeadsArgs& a);
const void* heads_dkv_bf16(const HeadsArgs& a);

#define SMX_FN(...) reinterpret_cast<const void*>(&__VA_ARGS__)

// The instance of a head width: its columns padded to 64, 128 or 256.
#define SMX_BY_WIDTH(d, K, T, ...)                                                    \
  ((d) <= 64 ? SMX_FN(K<T, 64, __VA_ARGS__>)                                          \
             : (d) <= 128 ? SMX_FN(K<T, 128, __VA_ARGS__>) : SMX_FN(K<T, 256, __VA_ARGS__>))

// How the call's scores are formed (kPlain, kBias, kCap, kCapBias).  A scale
// of no ordinary size goes with the bias, whose scores are formed before the
// mask.
inline int score_mode(const HeadsArgs& a) {
  if (a.cap > 0.0f) return a.slopes != nullptr ? 3 : 2;
  return a.slopes != nullptr || !(std::fabs(a.scale) > 1e-20f) ? 1 : 0;
}

}  // namespace smx
