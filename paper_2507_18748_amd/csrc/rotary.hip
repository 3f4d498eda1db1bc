// Rotary positions with one to three axes (see ppipe_rotary_desc).
//
// The angle position * base^-e is reduced in 64 bits to a fraction of a turn
// (positions are 32-bit integers, so 2^-21 of a turn is the worst error), and
// the sine and cosine of that fraction are taken in 32 bits.
#include "kernels.h"

namespace ppipe {
namespace {

template <typename T>
__global__ void __launch_bounds__(256) rotary_kernel(RotaryArgs a, int P, int64_t total)
{
    const int items = a.d - P;               // pairs, then copied elements
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const int e = (int)(i % items);
    const int64_t r = i / items;
    const int h = (int)(r % a.H);
    const int64_t token = r / a.H;
    const int n = (int)(token / a.L), l = (int)(token % a.L);
    const T* x = (const T*)a.x + n * a.xs[0] + l * a.xs[1] + h * a.xs[2];
    T* y = (T*)a.y + n * a.ys[0] + l * a.ys[1] + h * a.ys[2];
    if (e >= P) {
        y[e + P] = x[e + P];
        return;
    }
    int axis = 0, k = e;
    while (k >= a.pairs[axis]) k -= a.pairs[axis++];
    const double ex = a.shared ? (double)e / P : (double)k / a.pairs[axis];
    const double turns = (double)a.pos[n * a.ps + (int64_t)l * a.A + axis] *
                         (pow(a.base, -ex) * 0.15915494309189535);
    const float f = (float)(turns - rint(turns));
    const float c = cospif(2.0f * f), sn = sinpif(2.0f * f);
    const int e0 = a.adjacent ? 2 * e : e, e1 = a.adjacent ? 2 * e + 1 : e + P;
    const float u = (float)x[e0], w = (float)x[e1];
    y[e0] = (T)(u * c - w * sn);
    y[e1] = (T)(u * sn + w * c);
}

}  // namespace

const char* rotary_name(int dt)
{
    return dt == DT_F32 ? "rotary<f32>" : dt == DT_F16 ? "rotary<f16>" : "rotary<bf16>";
}

hipError_t launch_rotary(int dt, const RotaryArgs& a, hipStream_t s)
{
    const int P = a.pairs[0] + a.pairs[1] + a.pairs[2];
    const int64_t total = (int64_t)a.N * a.L * a.H * (a.d - P);
    const dim3 grid((uint32_t)((total + 255) / 256)), block(256);
    if (dt == DT_F32)
        PPIPE_LAUNCH(rotary_kernel<float>, grid, block, 0, s, a, P, total);
    else if (dt == DT_F16)
        PPIPE_LAUNCH(rotary_kernel<_Float16>, grid, block, 0, s, a, P, total);
    else
        PPIPE_LAUNCH(rotary_kernel<__bf16>, grid, block, 0, s, a, P, total);
    return hipGetLastError();
}

}  // namespace ppipe
