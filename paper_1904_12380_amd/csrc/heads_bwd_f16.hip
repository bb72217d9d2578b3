// Instances of the attention gradient kernels for f16.
#include "sm_heads_bwd.hpp"
#include "sm_heads_launch.hpp"

namespace smx {

const void* heads_dq_f16(const HeadsArgs& a) {
  switch (score_mode(a)) {
    case kPlain: return SMX_BY_WIDTH(a.d, k_heads_dq, f16, kPlain);
    case kBias: return SMX_BY_WIDTH(a.d, k_heads_dq, f16, kBias);
    case kCap: return SMX_BY_WIDTH(a.d, k_heads_dq, f16, kCap);
    default: return SMX_BY_WIDTH(a.d, k_heads_dq, f16, kCapBias);
  }
}

const void* heads_dkv_f16(const HeadsArgs& a) {
  switch (score_mode(a)) {
    case kPlain: return SMX_BY_WIDTH(a.d, k_heads_dkv, f16, kPlain);
    case kBias: return SMX_BY_WIDTH(a.d, k_heads_dkv, f16, kBias);
    case kCap: return SMX_BY_WIDTH(a.d, k_heads_dkv, f16, kCap);
    default: return SMX_BY_WIDTH(a.d, k_heads_dkv, f16, kCapBias);
  }
}

}  // namespace smx
