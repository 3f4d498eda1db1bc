// Group norm with an activation over NHWC maps.
//
//   y = act( (x - mean) / sqrt(var + eps) * gamma + beta )
//
// with mean and biased variance over the pixels and consecutive channels of
// each image's group.  One block takes one group of one image: a sum, a sum of
// squared differences from the mean, then the outputs.
#include "kernels.h"

namespace ppipe {
namespace {

__device__ __forceinline__ float norm_act(float z, int act)
{
    if (act == ACT_RELU) return z < 0.0f ? 0.0f : z;      // a NaN stays one
    if (act == ACT_RELU6) return z < 0.0f ? 0.0f : z > 6.0f ? 6.0f : z;
    if (act == ACT_SILU) return z / (1.0f + expf(-z));
    if (act == ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    return z;
}

__device__ float block_sum(float v, float* lds)
{
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) s += lds[w];
    return s;
}

template <typename T>
__global__ void __launch_bounds__(256) group_norm_kernel(GroupNormArgs a)
{
    __shared__ float lds[4];
    const int n = blockIdx.x / a.G, g = blockIdx.x % a.G, cg = a.C / a.G;
    const int64_t base = (int64_t)n * a.P * a.C + g * cg;
    const T* x = (const T*)a.x + base;
    T* y = (T*)a.y + base;
    const int64_t total = (int64_t)a.P * cg;
    auto at = [&](int64_t i) { return i / cg * a.C + i % cg; };
    float s = 0.0f;
    for (int64_t i = threadIdx.x; i < total; i += 256) s += (float)x[at(i)];
    const float mean = block_sum(s, lds) / (float)total;
    s = 0.0f;
    for (int64_t i = threadIdx.x; i < total; i += 256) {
        const float d = (float)x[at(i)] - mean;
        s += d * d;
    }
    const float rstd = 1.0f / sqrtf(block_sum(s, lds) / (float)total + a.eps);
    for (int64_t i = threadIdx.x; i < total; i += 256) {
        const int c = g * cg + (int)(i % cg);
        const float z = ((float)x[at(i)] - mean) * rstd * (a.gamma ? a.gamma[c] : 1.0f) +
                        (a.beta ? a.beta[c] : 0.0f);
        y[at(i)] = (T)norm_act(z, a.act);
    }
}

}  // namespace

size_t group_norm_workspace(int, int, int, int, int, int) { return 0; }
int group_norm_launches(int, int, int, int, int, int) { return 1; }
const char* group_norm_name(int dt, int, int, int, int, int, int)
{
    return dt == DT_F32 ? "group_norm<f32>" : dt == DT_F16 ? "group_norm<f16>" : "group_norm<bf16>";
}

hipError_t launch_group_norm(int dt, const GroupNormArgs& a, void*, int, int, hipStream_t s)
{
    const dim3 grid((uint32_t)((int64_t)a.N * a.G)), block(256);
    if (dt == DT_F32)
        PPIPE_LAUNCH(group_norm_kernel<float>, grid, block, 0, s, a);
    else if (dt == DT_F16)
        PPIPE_LAUNCH(group_norm_kernel<_Float16>, grid, block, 0, s, a);
    else
        PPIPE_LAUNCH(group_norm_kernel<__bf16>, grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace ppipe
