// Argument checks and argument structs of the operators on device tensors,
// shared by their C entries and the partition runtime.
#pragma once
#include "kernels.h"
#include "ppipe.h"

#include <string>

namespace ppipe {

constexpr int HEAD_DIM_MAX = 256;
constexpr int MAX_HEADS = 65536;
constexpr int GROUP_NORM_MAX_C = 65536;
constexpr int ATTENTION_MAX_LEN = 1 << 28;
constexpr int64_t ROW_STRIDE_LIMIT = 1 << 22;

// Compute units of the current device (256 when it cannot be queried).
int device_cus();

// The checks that need no pointer; a ppipe_status, with the message recorded.
int check_group_norm(int dt, int64_t batch, int64_t pixels, int C, int G, float eps, int act,
                     const std::string& who);
int check_rotary(const ppipe_rotary_desc& r, const std::string& who);
int check_attention(const ppipe_attention_desc& t, const std::string& who);

RotaryArgs rotary_args(const ppipe_rotary_desc& r, const void* x, const int* pos, void* y);
AttentionArgs attention_args(const ppipe_attention_desc& t, const void* q, const void* k,
                             const void* v, void* out, const float* slopes, const int* qpos,
                             const int* kpos, const int* spans);

}  // namespace ppipe
