// Instances of the attention forward kernel for bf16.
#include "sm_heads_launch.hpp"
#include "sm_heads_mfma.hpp"

namespace smx {

template <int WHERE>
static const void* fwd(const HeadsArgs& a) {
  switch (score_mode(a)) {
    case kPlain: return SMX_BY_WIDTH(a.d, k_heads_fwd, bf16, WHERE, kPlain);
    case kBias: return SMX_BY_WIDTH(a.d, k_heads_fwd, bf16, WHERE, kBias);
    case kCap: return SMX_BY_WIDTH(a.d, k_heads_fwd, bf16, WHERE, kCap);
    default: return SMX_BY_WIDTH(a.d, k_heads_fwd, bf16, WHERE, kCapBias);
  }
}

const void* heads_fwd_bf16(const HeadsArgs& a, int where) {
  return where == kPacked ? fwd<kPacked>(a) : where == kBlocks ? fwd<kBlocks>(a) : fwd<kSmallBlocks>(a);
}

}  // namespace smx
