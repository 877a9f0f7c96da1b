// The attention kernels of bfloat16; a source of its own, so that the types
// are compiled side by side.
#include "attention_kernels.hpp"

template void attention::launch_attention<__bf16>(const AttentionArgs &, const ForwardPlan &, hipStream_t);
template void attention::launch_attention_backward<__bf16>(AttentionArgs, int32_t, hipStream_t);
