// The attention kernels of one storage type (attention_device.h).
#include "attention_device.h"

void ppipe::launch_attention_f32(const AttentionArgs& a, const AttentionPlan& p,
                                 const AttentionChoice& c, hipStream_t s)
{
    launch_type<float>(a, p, c, s);
}
