// Attention over [batch][token][head][dim] tensors by strides (see
// ppipe_attention_desc), and the spans of keys that its queries see.
//
// One wave takes one query of one head and walks its visible keys 64 at a
// time with a running maximum and sum: a lane scores one key, then each lane
// adds the values of its elements of the head.
#include "kernels.h"

namespace ppipe {
namespace {

__global__ void __launch_bounds__(256) attention_spans_kernel(SpansArgs a)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)a.N * a.Lq) return;
    const int b = (int)(i / a.Lq);
    const int64_t pos = (int64_t)(a.start ? a.start[b] : 0) + i % a.Lq;
    auto off = [&](int d) {
        return !a.offsets ? (d ? a.Lk : 0)
                          : min(max(a.offsets[(int64_t)b * (a.docs + 1) + d], 0), a.Lk);
    };
    int lo = 0, hi = a.docs + 1;         // first d with offset > pos
    while (lo < hi) {
        const int m = (lo + hi) / 2;
        if (off(m) > pos) hi = m;
        else lo = m + 1;
    }
    int first = 0, end = 0;
    if (lo > 0 && lo <= a.docs) {
        first = off(lo - 1);
        end = off(lo);
        if (a.causal) {
            const int64_t pre = a.prefix ? (int64_t)a.prefix[(int64_t)b * a.docs + lo - 1] : 0;
            end = (int)min((int64_t)end, max(pos + 1, first + pre));
        }
    }
    a.spans[2 * i] = first;
    a.spans[2 * i + 1] = end;
}

template <typename T>
__global__ void __launch_bounds__(256) attention_kernel(AttentionArgs a)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    const int lane = threadIdx.x % 64;
    if (row >= (int64_t)a.N * a.Lq * a.H) return;
    const int h = (int)(row % a.H);
    const int64_t t = row / a.H;
    const int n = (int)(t / a.Lq), i = (int)(t % a.Lq), hk = h / (a.H / a.Hk);
    const T* q = (const T*)a.q + n * a.qs[0] + i * a.qs[1] + h * a.qs[2];
    const T* k = (const T*)a.k + n * a.ks[0] + hk * a.ks[2];
    const T* v = (const T*)a.v + n * a.vs[0] + hk * a.vs[2];
    T* out = (T*)a.out + n * a.os[0] + i * a.os[1] + h * a.os[2];
    int lo = 0, hi = a.Lk;
    if (a.spans) {
        lo = max(0, a.spans[n * a.sps + 2 * (int64_t)i]);
        hi = min(a.Lk, a.spans[n * a.sps + 2 * (int64_t)i + 1]);
    }
    float m = -INFINITY, l = 0.0f, acc[4] = {};
    for (int j0 = lo; j0 < hi; j0 += 64) {
        const int j = j0 + lane;
        float s = -INFINITY;
        if (j < hi) {
            float dot = 0.0f;
            for (int e = 0; e < a.d; ++e) dot += (float)q[e] * (float)k[j * a.ks[1] + e];
            s = dot * a.scale;
            if (a.cap > 0.0f) s = a.cap * tanhf(s / a.cap);
            if (a.slopes) {
                uint32_t dist = 0;
                for (int x = 0; x < a.A; ++x) {
                    const int p = a.qpos[n * a.qps + (int64_t)i * a.A + x];
                    const int r = a.kpos[n * a.kps + (int64_t)j * a.A + x];
                    dist += (uint32_t)max(p, r) - (uint32_t)min(p, r);
                }
                s -= a.slopes[h] * (float)dist;
            }
        }
        float top = s;
        for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float mn = fmaxf(m, top), base = mn == -INFINITY ? 0.0f : mn;
        const float alpha = expf(m - base), p = expf(s - base);
        float sum = p;
        for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
        l = l * alpha + sum;
        m = mn;
        for (int x = 0; x < 4; ++x) acc[x] *= alpha;
        for (int jj = 0; jj < 64 && j0 + jj < hi; ++jj) {
            const float pj = __shfl(p, jj);
            for (int x = 0; x < 4; ++x)
                if (lane + 64 * x < a.d)
                    acc[x] += pj * (float)v[(j0 + jj) * a.vs[1] + lane + 64 * x];
        }
    }
    for (int x = 0; x < 4; ++x)
        if (lane + 64 * x < a.d) out[lane + 64 * x] = (T)(l == 0.0f ? 0.0f : acc[x] / l);
}

}  // namespace

hipError_t launch_attention_spans(const SpansArgs& a, hipStream_t s)
{
    const dim3 grid((uint32_t)(((int64_t)a.N * a.Lq + 255) / 256)), block(256);
    PPIPE_LAUNCH(attention_spans_kernel, grid, block, 0, s, a);
    return hipGetLastError();
}

size_t attention_workspace(int, const AttentionArgs&, int) { return 0; }
int attention_launches(int, const AttentionArgs&, int) { return 1; }
const char* attention_name(int dt, const AttentionArgs&, int, int)
{
    return dt == DT_F32 ? "attention<f32>" : dt == DT_F16 ? "attention<f16>" : "attention<bf16>";
}

hipError_t launch_attention(int dt, const AttentionArgs& a, void*, int, int, hipStream_t s)
{
    const dim3 grid((uint32_t)(((int64_t)a.N * a.Lq * a.H + 3) / 4)), block(256);
    if (dt == DT_F32)
        PPIPE_LAUNCH(attention_kernel<float>, grid, block, 0, s, a);
    else if (dt == DT_F16)
        PPIPE_LAUNCH(attention_kernel<_Float16>, grid, block, 0, s, a);
    else
        PPIPE_LAUNCH(attention_kernel<__bf16>, grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace ppipe
