// Instances of the attention gradient kernels for bf16.
#include "sm_heads_bwd.hpp"
#include "sm_heads_launch.hpp"

namespace smx {

const void* heads_dq_bf16(const HeadsArgs& a) {
  switch (score_mode(a)) {
    case kPlain: return SMX_BY_WIDTH(a.d, k_heads_dq, bf16, kPlain);
    case kBias: return SMX_BY_WIDTH(a.d, k_heads_dq, bf16, kBias);
    case kCap: return SMX_BY_WIDTH(a.d, k_heads_dq, bf16, kCap);
    default: return SMX_BY_WIDTH(a.d, k_heads_dq, bf16, kCapBias);
  }
}

const void* heads_dkv_bf16(const HeadsArgs& a) {
  switch (score_mode(a)) {
    case kPlain: return SMX_BY_WIDTH(a.d, k_heads_dkv, bf16, kPlain);
    case kBias: return SMX_BY_WIDTH(a.d, k_heads_dkv, bf16, kBias);
    case kCap: return SMX_BY_WIDTH(a.d, k_heads_dkv, bf16, kCap);
    default: return SMX_BY_WIDTH(a.d, k_heads_dkv, bf16, kCapBias);
  }
}

}  // namespace smx
