// The attention kernels of binary16; a source of its own, so that the types
// are compiled side by side.
#include "attention_kernels.hpp"

template void attention::launch_attention<_Float16>(const AttentionArgs &, const ForwardPlan &, hipStream_t);
template void attention::launch_attention_backward<_Float16>(AttentionArgs, int32_t, hipStream_t);
