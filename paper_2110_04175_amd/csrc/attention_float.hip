// The attention kernels of binary32; a source of its own, so that the types
// are compiled side by side.
#include "attention_kernels.hpp"

template void attention::launch_attention<float>(const AttentionArgs &, const ForwardPlan &, hipStream_t);
template void attention::launch_attention_backward<float>(AttentionArgs, int32_t, hipStream_t);
