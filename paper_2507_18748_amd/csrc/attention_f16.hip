// The attention kernels of one storage type (attention_device.h).
#include "attention_device.h"

void ppipe::launch_attention_f16(const AttentionArgs& a, const AttentionPlan& p,
                                 const AttentionChoice& c, hipStream_t s)
{
    launch_type<_Float16>(a, p, c, s);
}
