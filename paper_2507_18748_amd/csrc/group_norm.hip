// Group norm with an activation over NHWC maps.
//
//   y = act( (x - mean) / sqrt(var + eps) * gamma + beta )
//
// with mean and biased variance over the pixels and consecutive channels of
// each image's group.  Bound by memory: the least is one read and one write.
//
// A block holds a slab (pixels x whole groups of one image) in registers, at
// most 256 KB (32 vectors of 16 bytes for each of 512 threads).  Each thread
// takes the mean and the squared differences of its own values, and these are
// joined by the parallel form for sums of squares (Chan, Golub, LeVeque), fp32
// throughout.  Where a slab is all pixels
// it writes the outputs at once: one read, one write, one launch.  Larger maps
// take two launches: slabs leave their mean and sum of squared differences,
// the second launch joins those (Chan's formula) and reads the map again.
//
// 64 maps of 56x56x256 in 32 groups, bf16: 54 us, 3.8 TB/s (a copy of the bytes: 41); one
// of 14x14x256: 4.6 us.
#include "gemm_device.h"

#include <algorithm>

namespace ppipe {
namespace {

template <int act> __device__ __forceinline__ float norm_act(float z)
{
    // (maximum and minimum that keep a NaN)
    if (act == ACT_RELU) return __builtin_elementwise_maximum(z, 0.0f);
    if (act == ACT_RELU6) return __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, 0.0f), 6.0f);
    if (act == ACT_SILU)
        return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
    if (act == ACT_GELU) {
        // Phi(-|z|) = erfc(|z| / sqrt 2) / 2 by Abramowitz and Stegun 7.1.26, off by
        // at most 7.5e-8 (half of its 1.5e-7)
        const float x = fabsf(z) * 0.70710678f;
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, x, 1.0f));
        float q = __builtin_fmaf(1.061405429f, t, -1.453152027f);
        q = __builtin_fmaf(q, t, 1.421413741f);
        q = __builtin_fmaf(q, t, -0.284496736f);
        q = __builtin_fmaf(q, t, 0.254829592f);
        const float h = 0.5f * q * t * __builtin_amdgcn_exp2f(-1.4426950408889634f * x * x);
        return z * (z < 0.0f ? h : 1.0f - h);
    }
    return z;
}

// f(integral_constant) of the activation: one branch for all elements.
template <typename F> __device__ __forceinline__ void with_act(int act, F&& f)
{
    if (act == ACT_NONE) f(std::integral_constant<int, ACT_NONE>{});
    else if (act == ACT_RELU) f(std::integral_constant<int, ACT_RELU>{});
    else if (act == ACT_RELU6) f(std::integral_constant<int, ACT_RELU6>{});
    else if (act == ACT_SILU) f(std::integral_constant<int, ACT_SILU>{});
    else f(std::integral_constant<int, ACT_GELU>{});
}

template <typename T, int V>
__device__ __forceinline__ void unpack(const uint4& u, float* f)
{
    if constexpr (std::is_same<T, __bf16>::value) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
        return;
    }
    T e[V];
    __builtin_memcpy(e, &u, 16);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (float)e[i];
}
template <typename T, int V>
__device__ __forceinline__ uint4 pack(const float* f)
{
    T e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = (T)f[i];
    uint4 u;
    __builtin_memcpy(&u, e, 16);
    return u;
}

// How a call is cut.
struct NormPlan {
    bool single;       // a block takes one group
    bool whole;        // of whole vectors
    int cv;            // vectors of a pixel that a block takes
    int groups;        // groups of a block
    int chunks;        // blocks per image and slab
    int slabs, px;     // slabs of an image, pixels of a slab
    int nt, r;         // threads, vectors each holds
    FastDiv div_cv;
};

constexpr int NORM_R = 32, NORM_SLAB_R = 8, NORM_NT = 512;

enum NormMode {
    MIXED = 0,         // several groups of a pixel, vectors of several groups
    SEVERAL = 1,       // several groups of whole vectors
    ONE = 2,           // one group of whole vectors, a row no longer than the block
    ANY = 3            // one group whose rows begin or end inside a vector, or are longer
};

// One launch or two.  A block alone takes about 4 us and 0.45 us for each vector
// that a thread holds (fp32: 0.3; of several groups 2.2 times that), and blocks beyond one per CU come in turn; two
// launches take about 9 us and three passes at 5 TB/s.  Measured both ways (one /
// two, us): 64 x 56x56x256 bf16 55 / 67, 8 x the same 14.8 / 17.6, 2 x 9.9 / 11.6,
// 64 x 14x14x1024 15.6 / 25, 32 x 40x40x96 17.8 / 21.6, 1 x 112x112x64 in 32
// groups 29.5 / 16.4.  Rows read in pieces of 256 or 1024 bytes where slabs fill
// the chip anyway: 1 x 128x128x320 f16 23 -> 24 and 33 (64 bytes stay).
NormPlan norm_plan(int dt, int N, int P, int C, int G, int cus)
{
    const int esz = dtype_size(dt), V = 16 / esz, cpg = C / G;
    auto pixels = [&](const NormPlan& p, int nt, int r) {    // of a slab, below 2 GiB apart
        const int64_t n = p.cv <= nt ? (int64_t)(nt / p.cv) * r
                          : nt == NORM_NT ? r / ((p.cv + nt - 1) / nt) : 0;
        return std::min<int64_t>(n, 0x7fffffff / ((int64_t)C * esz));
    };
    // Rows of a group from 64 bytes on are read well by themselves.  Smaller
    // groups are taken several to a block: the least number whose channels are
    // whole vectors, then up to 64 bytes while the grid still fills the chip.
    auto cut = [&](int fill) {
        NormPlan p;
        p.single = cpg * esz >= 64;
        p.whole = cpg % V == 0;
        if (p.single) {
            p.cv = p.whole ? cpg / V : cpg / V + 2;
            p.groups = 1;
            p.chunks = G;
        } else {
            int l = cpg;
            while (l % V) l += cpg;                       // least common multiple
            const int all = C / l;
            int m = 1;
            for (int q = 2; q <= all && q * l * esz <= 64; ++q)
                if (all % q == 0 && (int64_t)N * (all / q) >= fill) m = q;
            p.cv = m * l / V;
            p.groups = m * l / cpg;
            p.chunks = all / m;
        }
        p.div_cv = fast_div_of((uint32_t)p.cv);
        return p;
    };
    NormPlan p = cut(cus);
    p.nt = 256;
    for (p.r = 1; p.r < 4 && pixels(p, 256, p.r) < P; p.r *= 2) {}
    if (pixels(p, p.nt, p.r) < P) {
        p.nt = NORM_NT;
        const int most = p.single && !(p.whole && p.cv <= NORM_NT) ? NORM_R / 2 : NORM_R;
        for (p.r = 4; p.r < most && pixels(p, p.nt, p.r) < P; p.r *= 2) {}
    }
    const double rounds = (double)(((int64_t)N * p.chunks + cus - 1) / cus);
    const double each = (esz == 2 ? 0.45 : 0.3) * (p.single || p.whole ? 1.0 : 2.2);
    const double one = 4.0 + each * ((double)P * p.cv / p.nt) * rounds;
    const double two = 9.0 + 3.0 * N * (double)P * C * esz / 5e6;
    p.px = P;
    p.slabs = 1;
    if (pixels(p, p.nt, p.r) >= P && one <= two) return p;
    p = cut(0);
    p.nt = NORM_NT;
    p.r = NORM_SLAB_R;
    while (p.r > 4 && pixels(p, p.nt, p.r / 2) > 0 &&
           (int64_t)N * p.chunks * ((P + pixels(p, p.nt, p.r) - 1) / pixels(p, p.nt, p.r)) < 4 * cus)
        p.r /= 2;
    while (pixels(p, p.nt, p.r) < 1) p.r *= 2;
    p.px = (int)std::min<int64_t>(P, pixels(p, p.nt, p.r));
    p.slabs = (P + p.px - 1) / p.px;
    p.px = (P + p.slabs - 1) / p.slabs;
    return p;
}

template <typename T, int NT, int R, int MODE>
__global__ void __launch_bounds__(NT, NT != NORM_NT ? 1 : R < NORM_R && (MODE == SEVERAL || MODE == ONE) ? 4 : 2)
group_norm_kernel(GroupNormArgs a, NormPlan p, float* part)
{
    constexpr int ESZ = (int)sizeof(T), V = 16 / ESZ, NW = NT / 64;
    constexpr bool SINGLE = MODE >= ONE;
    constexpr int S = MODE == MIXED ? V : 1;       // statistics of a thread's channels
    __shared__ float2 red[SINGLE ? 1 : NT * S];
    __shared__ float4 stat[64];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    // blocks of one image side by side on one XCD: their rows share cache lines
    const uint32_t per = gridDim.x / NUM_XCD, rem = gridDim.x % NUM_XCD, xcd = blockIdx.x % NUM_XCD;
    uint32_t lin = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / NUM_XCD;
    const int chunk = (int)(lin % (uint32_t)p.chunks);
    lin /= (uint32_t)p.chunks;
    const int slab = (int)(lin % (uint32_t)p.slabs), n = (int)(lin / (uint32_t)p.slabs);
    const int cpg = a.C / a.G, p0 = slab * p.px, px = min(p.px, a.P - p0);
    const int g0 = chunk * p.groups, c0 = g0 * cpg;          // first group and channel
    const int v0 = c0 / V;                                   // first vector
    const T* x = (const T*)a.x + ((int64_t)n * a.P + p0) * a.C;
    T* y = (T*)a.y + ((int64_t)n * a.P + p0) * a.C;
    const auto rx = make_rsrc(x, (uint32_t)px * (uint32_t)(a.C * ESZ));

    // ---- the slab into registers ----
    // Vector i of a thread lies in row slot + i slots of the slab, always in one
    // column; where rows are longer than the block: row i / per_row, column col +
    // (i % per_row) NT.
    uint4 u[R];
    const int cvs = SINGLE ? (c0 + cpg - 1) / V - v0 + 1 : p.cv;
    const int per_row = MODE == ANY ? (p.cv + NT - 1) / NT : 1;
    const bool wide = MODE == ANY && per_row > 1;
    const int slots = wide ? 1 : NT / p.cv;
    const int slot = wide ? 0 : fast_div(tid, p.div_cv);
    const int col = tid - slot * p.cv;
    const uint32_t row_bytes = (uint32_t)(a.C * ESZ), step = (uint32_t)slots * row_bytes;
    uint32_t off0 = (uint32_t)slot * row_bytes + (uint32_t)(v0 + col) * 16u;
    // first vector of the thread outside the slab
    int mine = wide || slot >= slots || col >= cvs ? 0 : (px - slot + slots - 1) / slots;
    auto offset = [&](int i) {
        if (wide) {
            const int row = i / per_row, c = (i - row * per_row) * NT;
            return row < px && col + c < cvs ? off0 + (uint32_t)row * row_bytes + (uint32_t)c * 16u : OOB;
        }
        return i < mine ? off0 + (uint32_t)i * step : OOB;
    };
#pragma unroll
    for (int i = 0; i < R; ++i) u[i] = buf_load16(rx, offset(i));
    // scale and shift of the thread's channels, on their way before they are needed
    float ga[V], be[V];
    auto affine = [&](int i) {
        const int c = (v0 + col + (wide ? (i % per_row) * NT : 0)) * V;
        const bool ok = p.slabs == 1 && offset(i) != OOB;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            ga[e] = ok && a.gamma ? a.gamma[c + e] : 1.0f;
            be[e] = ok && a.beta ? a.beta[c + e] : 0.0f;
        }
    };
    affine(0);
    // which channels of vector i belong to the group (SINGLE: the first and
    // last vector of a row may reach beyond it)
    const bool ends = MODE == ANY && cpg % V != 0;
    auto inside = [&](int i, int e) {
        const int c = (v0 + col + (wide ? (i % per_row) * NT : 0)) * V + e;
        return c >= c0 && c < c0 + cpg;
    };

    // ---- statistics of the thread's values, of one group or of each channel's ----
    // Mean and squared differences of a thread's values x by sums of x - k and
    // (x - k)^2, k its first value: a value far off the others counts in the sum of
    // squares itself, so what cancels stays below (values of the thread) 2^-24 of it.
    float k[S], sum[S], sq[S], cnt = 0.0f;
#pragma unroll
    for (int e = 0; e < S; ++e) sum[e] = sq[e] = 0.0f;
    {
        float v[V];
        unpack<T, V>(u[0], v);
#pragma unroll
        for (int e = 0; e < S; ++e) k[e] = v[e];
        if constexpr (MODE == ANY)
#pragma unroll
            for (int e = V - 1; e >= 0; --e)
                if (inside(0, e)) k[0] = v[e];
    }
    // Each pass unpacks a vector and computes its offset when it comes to it: the
    // compiler would do so for all at once, which does not fit the registers.
    auto turn_to = [&](int i) {
        asm volatile("" : "+v"(u[i].x), "+v"(u[i].y), "+v"(u[i].z), "+v"(u[i].w), "+v"(off0), "+v"(mine));
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int i = 0; i < R; ++i) {
        turn_to(i);
        if (offset(i) == OOB) continue;
        float v[V];
        unpack<T, V>(u[i], v);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const bool in = MODE != ANY || inside(i, e);
            const float d = in ? v[e] - k[e % S] : 0.0f;
            sum[e % S] += d;
            sq[e % S] = __builtin_fmaf(d, d, sq[e % S]);
            if constexpr (MODE == ANY) cnt += in ? 1.0f : 0.0f;
        }
    }
    if constexpr (MODE != ANY) cnt = (float)(mine * (V / S));
    const float inv = cnt > 0.0f ? 1.0f / cnt : 0.0f;
    float mean[S], m2[S];
#pragma unroll
    for (int e = 0; e < S; ++e) {
        const float m = sum[e] * inv, s = __builtin_fmaf(-sum[e], m, sq[e]);
        mean[e] = cnt > 0.0f ? k[e] + m : 0.0f;
        m2[e] = s < 0.0f ? 0.0f : s;
    }

    // ---- of the groups: first the means are added, then the differences from the sum ----
    auto wave_sum = [](float v) {
        for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
        return v;
    };
    // partial (count, mean, squared differences) of a wave's part of a group
    int parts, mygroup = 0;
    if constexpr (SINGLE) {
        const float n = wave_sum(cnt), m = n > 0.0f ? wave_sum(cnt * mean[0]) / n : wave_sum(0.0f);
        const float d = mean[0] - m, s = wave_sum(cnt > 0.0f ? m2[0] + cnt * d * d : 0.0f);
        if (lane == 0) stat[wave] = make_float4(n, m, s, 0.0f);
        parts = NW;
        __syncthreads();
    } else {
        if (slot < slots)
#pragma unroll
            for (int e = 0; e < S; ++e) red[tid * S + e] = make_float2(mean[e], m2[e]);
        __syncthreads();
        const int width = p.cv * S, each = S == 1 ? cpg / V : cpg;
        parts = max(NW / p.groups, 1);
        const int full = px / slots, more = px - full * slots;   // pixels of a slot
        for (int w = wave; w < p.groups * parts; w += NW) {
            const int part = w / p.groups, g = w - part * p.groups;
            const int q0 = slots * part / parts, q1 = slots * (part + 1) / parts;
            auto walk = [&](auto&& f) {
                int q = q0 + lane / each, e = lane % each;
                const int dq = 64 / each, de = 64 - dq * each;
                float s = 0.0f;
                while (q < q1) {
                    const float2 v = red[q * width + g * each + e];
                    s += f((float)(full + (q < more ? 1 : 0)), v);
                    q += dq;
                    e += de;
                    if (e >= each) {
                        e -= each;
                        ++q;
                    }
                }
                return wave_sum(s);
            };
            const int rows = max(0, min(q1, more) - min(q0, more)) + full * (q1 - q0);
            const float n = (float)(rows * each);
            const float m = n > 0.0f ? walk([](float c, float2 v) { return c * v.x; }) / n : 0.0f;
            const float s = walk([m](float c, float2 v) {
                const float d = v.x - m;
                return v.y + c * (V / S) * d * d;      // a pixel of a thread: V / S values
            });
            if (lane == 0) stat[part * p.groups + g] = make_float4(n * (V / S), m, s, 0.0f);
        }
        __syncthreads();
    }
    // the parts join; S > 1: of each channel's group
#pragma unroll
    for (int e = 0; e < S; ++e) {
        if constexpr (!SINGLE) mygroup = min((col * V + e) / cpg, p.groups - 1);
        const int stride = SINGLE ? 1 : p.groups;
        float m = 0.0f, n = 0.0f, s = 0.0f;
        for (int q = 0; q < parts; ++q) {
            const float4 v = stat[q * stride + mygroup];
            m += v.x * v.y;
            n += v.x;
        }
        m /= n;
        for (int q = 0; q < parts; ++q) {
            const float4 v = stat[q * stride + mygroup];
            s += v.z + v.x * (v.y - m) * (v.y - m);
        }
        mean[e] = m;
        m2[e] = s;
    }
    const float count = (float)px * (float)cpg;

    if (p.slabs > 1) {
        // mean and sum of squared differences of this slab's groups
        float* out = part + (((int64_t)n * p.slabs + slab) * a.G + g0) * 2;
        if constexpr (SINGLE) {
            if (tid == 0) {
                out[0] = mean[0];
                out[1] = m2[0];
            }
        } else if (slot == 0) {
#pragma unroll
            for (int e = 0; e < S; ++e)
                if ((col * V + e) % cpg == 0) {
                    out[(col * V + e) / cpg * 2] = mean[e];
                    out[(col * V + e) / cpg * 2 + 1] = m2[e];
                }
        }
        return;
    }
    // ---- outputs ----
    float rstd[S];
#pragma unroll
    for (int e = 0; e < S; ++e) rstd[e] = 1.0f / sqrtf(m2[e] / count + a.eps);
    // 16-bit: the mean goes into the shift (its rounding, 2^-24 of mean / deviation,
    // is far below the output's); fp32 subtracts it first
    auto finish_affine = [&] {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            ga[e] *= rstd[e % S];
            if constexpr (ESZ == 2) be[e] = __builtin_fmaf(-mean[e % S], ga[e], be[e]);
        }
    };
    finish_affine();
    with_act(a.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            turn_to(i);
            const uint32_t off = offset(i);
            if (off == OOB) continue;
            if (wide && i > 0) {
                affine(i);
                finish_affine();
            }
            float v[V];
            unpack<T, V>(u[i], v);
#pragma unroll
            for (int e = 0; e < V; ++e)
                v[e] = norm_act<decltype(act)::value>(
                    __builtin_fmaf(ESZ == 2 ? v[e] : v[e] - mean[e % S], ga[e], be[e]));
            T* dst = (T*)((uint8_t*)y + off);
            const uint4 w = pack<T, V>(v);
            if (!ends || (inside(i, 0) && inside(i, V - 1))) {
                *(uint4*)dst = w;
            } else {
                // element by element, not unrolled: the code would outgrow the rest
#pragma unroll 1
                for (int e = 0; e < V; ++e) {
                    if (!inside(i, e)) continue;
                    const int k = e * ESZ / 4;
                    const uint32_t x = k == 0 ? w.x : k == 1 ? w.y : k == 2 ? w.z : w.w;
                    if constexpr (ESZ == 4) ((uint32_t*)dst)[e] = x;
                    else ((uint16_t*)dst)[e] = (uint16_t)(x >> (16 * (e & 1)));
                }
            }
        }
    });
}

// Second launch: a block joins the slabs' statistics of the groups that its
// columns touch and normalises its pixels.
constexpr int APPLY_NT = 256;
template <typename T>
__global__ void __launch_bounds__(APPLY_NT)
group_norm_apply_kernel(GroupNormArgs a, NormPlan p, const float* part, int cols, int col_tiles,
                        int rows, int row_tiles)
{
    constexpr int ESZ = (int)sizeof(T), V = 16 / ESZ;
    __shared__ float stat[2 * APPLY_NT * V];
    const int tid = threadIdx.x;
    const uint32_t per = gridDim.x / NUM_XCD, rem = gridDim.x % NUM_XCD, xcd = blockIdx.x % NUM_XCD;
    uint32_t lin = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / NUM_XCD;
    const int ct = (int)(lin % (uint32_t)col_tiles);
    lin /= (uint32_t)col_tiles;
    const int rt = (int)(lin % (uint32_t)row_tiles), n = (int)(lin / (uint32_t)row_tiles);
    const int cpg = a.C / a.G, CV = a.C / V;
    const int nc = min(cols, CV - ct * cols);                // columns of this block
    const int step = APPLY_NT / cols, slot = tid / cols, col = tid - slot * cols;
    const int first = rt * rows, last = slot >= step || col >= nc ? 0 : min(a.P, first + rows);
    const int64_t at = (int64_t)n * a.P * CV + ct * cols + col;
    const uint4* x = (const uint4*)a.x + at;
    uint4* y = (uint4*)a.y + at;
    // first vectors, scales and shifts on their way while the statistics are joined
    constexpr int B = 4;
    uint4 u[B];
    auto load = [&](int q) {
#pragma unroll
        for (int b = 0; b < B; ++b)
            if (q + b * step < last) u[b] = x[(int64_t)(q + b * step) * CV];
    };
    load(first + slot);
    float mean[V], ga[V], be[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = (ct * cols + min(col, nc - 1)) * V + e;
        ga[e] = a.gamma ? a.gamma[c] : 1.0f;
        be[e] = a.beta ? a.beta[c] : 0.0f;
    }
    const int g0 = ct * cols * V / cpg, g1 = (ct * cols * V + nc * V - 1) / cpg;
    // eight lanes a group: each joins every eighth slab, then they join each other
    // (n = pixels; the differences' sums are of pixels x channels)
    auto join = [&](float& n0, float& mean0, float& m20, float n1, float mean1, float m21) {
        const float both = n0 + n1, d = mean1 - mean0, w = both > 0.0f ? n1 / both : 0.0f;
        m20 += n1 > 0.0f ? m21 + d * d * n0 * w * (float)cpg : 0.0f;
        mean0 += n1 > 0.0f ? d * w : 0.0f;
        n0 = both;
    };
    for (int gb = g0; gb <= g1; gb += APPLY_NT / 8) {
        const int g = min(gb + tid / 8, g1);
        const float* q = part + ((int64_t)n * p.slabs * a.G + g) * 2;
        float cnt = 0.0f, mean = 0.0f, m2 = 0.0f;
#pragma unroll 4
        for (int s = tid % 8; s < p.slabs; s += 8) {
            const float2 v = *(const float2*)(q + (int64_t)s * a.G * 2);
            join(cnt, mean, m2, (float)min(p.px, a.P - s * p.px), v.x, v.y);
        }
#pragma unroll
        for (int m = 1; m < 8; m *= 2)
            join(cnt, mean, m2, __shfl_xor(cnt, m), __shfl_xor(mean, m), __shfl_xor(m2, m));
        if (tid % 8 == 0 && gb + tid / 8 <= g1) {
            stat[2 * (g - g0)] = mean;
            stat[2 * (g - g0) + 1] = 1.0f / sqrtf(m2 / ((float)a.P * (float)cpg) + a.eps);
        }
    }
    __syncthreads();
    if (last == 0) return;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int g = ((ct * cols + col) * V + e) / cpg - g0;
        mean[e] = stat[2 * g];
        ga[e] *= stat[2 * g + 1];
        if constexpr (ESZ == 2) be[e] = __builtin_fmaf(-mean[e], ga[e], be[e]);
    }
    with_act(a.act, [&](auto act) {
        for (int q = first + slot; q < last; q += B * step) {
            if (q > first + slot) load(q);
#pragma unroll
            for (int b = 0; b < B; ++b) {
                if (q + b * step >= last) break;
                float v[V];
                unpack<T, V>(u[b], v);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    v[e] = norm_act<decltype(act)::value>(
                        __builtin_fmaf(ESZ == 2 ? v[e] : v[e] - mean[e], ga[e], be[e]));
                y[(int64_t)(q + b * step) * CV] = pack<T, V>(v);
            }
        }
    });
}

template <typename T, int NT, int R>
void launch_norm(const GroupNormArgs& a, const NormPlan& p, float* part, hipStream_t s)
{
    const dim3 grid((uint32_t)((int64_t)a.N * p.slabs * p.chunks));
    if (!p.single && !p.whole) PPIPE_LAUNCH((group_norm_kernel<T, NT, R, MIXED>), grid, dim3(NT), 0, s, a, p, part);
    else if (!p.single) PPIPE_LAUNCH((group_norm_kernel<T, NT, R, SEVERAL>), grid, dim3(NT), 0, s, a, p, part);
    else if (p.whole && p.cv <= NT) PPIPE_LAUNCH((group_norm_kernel<T, NT, R, ONE>), grid, dim3(NT), 0, s, a, p, part);
    else if constexpr (R < NORM_R || sizeof(T) == 4)     // 16-bit: 65536 channels are 16 vectors a thread
        PPIPE_LAUNCH((group_norm_kernel<T, NT, R, ANY>), grid, dim3(NT), 0, s, a, p, part);
}

template <typename T>
void launch_type(const GroupNormArgs& a, const NormPlan& p, float* part, int cus, int launch,
                 hipStream_t s)
{
    if (launch == 1) {
        // columns of a block: a divisor-free choice, all of them where they fit
        const int V = 16 / (int)sizeof(T), CV = a.C / V, cols = std::min(CV, APPLY_NT);
        const int col_tiles = (CV + cols - 1) / cols, step = APPLY_NT / cols;
        // rows of a block: eight or more vectors a thread, a few blocks per CU
        const int64_t tiles = (int64_t)a.N * col_tiles;
        int rows = 8 * step;
        while (rows < 64 * step && tiles * ((a.P + rows - 1) / rows) > 16 * cus) rows *= 2;
        const int row_tiles = (a.P + rows - 1) / rows;
        PPIPE_LAUNCH(group_norm_apply_kernel<T>, dim3((uint32_t)(tiles * row_tiles)), dim3(APPLY_NT),
                     0, s, a, p, part, cols, col_tiles, rows, row_tiles);
        return;
    }
    if (p.nt != NORM_NT) {
        if (p.r == 1) launch_norm<T, 256, 1>(a, p, part, s);
        else if (p.r == 2) launch_norm<T, 256, 2>(a, p, part, s);
        else launch_norm<T, 256, 4>(a, p, part, s);
    } else {
        if (p.r == 4) launch_norm<T, NORM_NT, 4>(a, p, part, s);
        else if (p.r == 8) launch_norm<T, NORM_NT, 8>(a, p, part, s);
        else if (p.r == 16) launch_norm<T, NORM_NT, 16>(a, p, part, s);
        else launch_norm<T, NORM_NT, 32>(a, p, part, s);
    }
}

}  // namespace

size_t group_norm_workspace(int dt, int N, int P, int C, int G, int cus)
{
    const NormPlan p = norm_plan(dt, N, P, C, G, cus);
    return p.slabs > 1 ? (size_t)N * p.slabs * G * 8 : 0;
}

bool group_norm_fits(int dt, int N, int P, int C, int G, int cus)
{
    const NormPlan p = norm_plan(dt, N, P, C, G, cus);
    // the second launch has fewer blocks than one for each eight rows of vectors
    const int V = 16 / dtype_size(dt), CV = C / V, cols = std::min(CV, APPLY_NT);
    const double apply = p.slabs > 1 ? (double)N * ((CV + cols - 1) / cols) *
                                           (P / (8 * (APPLY_NT / cols)) + 1) * APPLY_NT : 0.0;
    return std::max((double)N * p.slabs * p.chunks * p.nt, apply) < 4294967296.0;
}

int group_norm_launches(int dt, int N, int P, int C, int G, int cus)
{
    return norm_plan(dt, N, P, C, G, cus).slabs > 1 ? 2 : 1;
}

const char* group_norm_name(int dt, int N, int P, int C, int G, int cus, int launch)
{
    static const char* names[3][3] = {
        {"group_norm<f32>", "group_norm<f16>", "group_norm<bf16>"},
        {"group_norm_stats<f32>", "group_norm_stats<f16>", "group_norm_stats<bf16>"},
        {"group_norm_apply<f32>", "group_norm_apply<f16>", "group_norm_apply<bf16>"}};
    return names[norm_plan(dt, N, P, C, G, cus).slabs > 1 ? 1 + launch : 0][dt];
}

hipError_t launch_group_norm(int dt, const GroupNormArgs& a, void* ws, int cus, int launch,
                             hipStream_t s)
{
    const NormPlan p = norm_plan(dt, a.N, a.P, a.C, a.G, cus);
    if (dt == DT_F32) launch_type<float>(a, p, (float*)ws, cus, launch, s);
    else if (dt == DT_F16) launch_type<_Float16>(a, p, (float*)ws, cus, launch, s);
    else launch_type<__bf16>(a, p, (float*)ws, cus, launch, s);
    return hipGetLastError();
}

}  // namespace ppipe
