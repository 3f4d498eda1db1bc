// The attention kernels of one storage type (attention_device.h).
#include "attention_device.h"

void ppipe::launch_attention_bf16(const AttentionArgs& a, const AttentionPlan& p,
                                 const AttentionChoice& c, hipStream_t s)
{
    launch_type<__bf16>(a, p, c, s);
}
