// The attention's backward passes at head dimension 128.
#include "attn_bwd_sm100.cuh"

namespace focus {

template int launch_bwd_d<128>(const AttnBwdArgs& a, const BwdParams& kv, const BwdParams& q, cudaStream_t st);

}  // namespace focus
