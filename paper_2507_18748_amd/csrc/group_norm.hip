// Group norm with an activation over NHWC maps.
//
//   y = act( (x - mean) / sqrt(var + eps) * gamma + beta )
//
// with mean and biased variance over the pixels and consecutive channels of
// each image's group.  Bound by memory: the least is one read and one write.
//
// A block holds a slab (pixels x whole groups of one image) in registers, at
// most 256 KB, and takes its mean and then the squared differences from it
// from there (no cancellation, fp32 throughout).  Where a slab is all pixels
// it writes the outputs at once: one read, one write, one launch.  Larger maps
// take two launches: slabs leave their mean and sum of squared differences,
// the second launch joins those (Chan's formula) and reads the map again.
#include "gemm_device.h"

#include <algorithm>

namespace ppipe {
namespace {

__device__ __forceinline__ float norm_act(float z, int act)
{
    if (act == ACT_RELU) return z < 0.0f ? 0.0f : z;      // a NaN stays one
    if (act == ACT_RELU6) return z < 0.0f ? 0.0f : z > 6.0f ? 6.0f : z;
    if (act == ACT_SILU)
        return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
    if (act == ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    return z;
}

template <typename T, int V>
__device__ __forceinline__ void unpack(const uint4& u, float* f)
{
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
    bool single;       // a block takes one group (its vectors may begin and end inside it)
    int cv;            // vectors of a pixel that a block takes
    int groups;        // groups of a block
    int chunks;        // blocks per image and slab
    int slabs, px;     // slabs of an image, pixels of a slab
    int nt, r;         // threads, vectors each holds
    FastDiv div_cv;
};

constexpr int NORM_R = 16, NORM_NT = 1024;

NormPlan norm_plan(int dt, int N, int P, int C, int G, int cus)
{
    const int esz = dtype_size(dt), V = 16 / esz, cpg = C / G;
    NormPlan p;
    // Rows of a group from 64 bytes on are read well by themselves.  Smaller
    // groups are taken several to a block: the least number whose channels are
    // whole vectors, then up to 64 bytes while the grid still fills the chip.
    p.single = cpg * esz >= 64;
    if (p.single) {
        p.cv = cpg % V ? cpg / V + 2 : cpg / V;
        p.groups = 1;
        p.chunks = G;
    } else {
        int l = cpg;
        while (l % V) l += cpg;                       // least common multiple
        const int all = C / l;
        int m = 1;
        for (int q = 2; q <= all && q * l * esz <= 64; ++q)
            if (all % q == 0 && (int64_t)N * (all / q) >= cus) m = q;
        p.cv = m * l / V;
        p.groups = m * l / cpg;
        p.chunks = all / m;
    }
    // pixels of a slab: what the largest block holds, below 2 GiB apart
    auto pixels = [&](int nt, int r) {
        const int64_t n = p.single ? (int64_t)nt * r / p.cv : (int64_t)(nt / p.cv) * r;
        return std::min<int64_t>(n, 0x7fffffff / ((int64_t)C * esz));
    };
    p.nt = 256;
    for (p.r = 1; p.r < 4 && pixels(256, p.r) < P; p.r *= 2) {}
    if (pixels(p.nt, p.r) < P) {
        p.nt = NORM_NT;
        for (p.r = 2; p.r < NORM_R && pixels(p.nt, p.r) < P; p.r *= 2) {}
    }
    p.px = (int)std::min<int64_t>(P, pixels(p.nt, p.r));
    p.slabs = p.px < 1 ? 0 : (P + p.px - 1) / p.px;
    if (p.slabs > 1) p.px = (P + p.slabs - 1) / p.slabs;
    p.div_cv = fast_div_of((uint32_t)p.cv);
    return p;
}

template <typename T, int NT, int R, bool SINGLE>
__global__ void __launch_bounds__(NT)
group_norm_kernel(GroupNormArgs a, NormPlan p, float* part)
{
    constexpr int ESZ = (int)sizeof(T), V = 16 / ESZ, NW = NT / 64;
    __shared__ float red[SINGLE ? NW : NT * V];
    __shared__ float stat[SINGLE ? 1 : 64];
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
    uint4 u[R];
    uint32_t off[R];
    const int cvs = SINGLE ? min(p.cv, (c0 + cpg - 1) / V - v0 + 1) : p.cv;
    const int slots = SINGLE ? 1 : NT / p.cv, slot = SINGLE ? 0 : fast_div(tid, p.div_cv);
    const int col = SINGLE ? 0 : tid - slot * p.cv;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        int q, v;
        bool ok;
        if constexpr (SINGLE) {
            const int idx = tid + NT * i;
            q = fast_div(idx, p.div_cv);
            v = idx - q * p.cv;
            ok = q < px && v < cvs;
        } else {
            q = slot + i * slots;
            v = col;
            ok = slot < slots && q < px;
        }
        off[i] = ok ? (uint32_t)q * (uint32_t)(a.C * ESZ) + (uint32_t)(v0 + v) * 16u : OOB;
        u[i] = buf_load16(rx, off[i]);
    }
    // which channels of vector i belong to the group (SINGLE: ends may not)
    auto inside = [&](int i, int e) {
        if constexpr (!SINGLE) return off[i] != OOB;
        const int c = (int)(off[i] % (uint32_t)(a.C * ESZ)) / ESZ + e;
        return off[i] != OOB && c >= c0 && c < c0 + cpg;
    };
    const bool ends = SINGLE && cpg % V != 0;

    // ---- group sums of V values a thread, or of one where a vector lies in one group ----
    const bool whole = cpg % V == 0;
    auto reduce = [&](const float* f, float* out) {
        if constexpr (SINGLE) {
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < V; ++e) s += f[e];
            for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m);
            __syncthreads();
            if (lane == 0) red[wave] = s;
            __syncthreads();
            s = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) s += red[w];
            *out = s;
        } else {
            __syncthreads();
            const int vp = whole ? 1 : V, width = p.cv * vp, each = whole ? cpg / V : cpg;
            if (slot < slots) {
                if (whole) {
                    float s = 0.0f;
#pragma unroll
                    for (int e = 0; e < V; ++e) s += f[e];
                    red[tid] = s;
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) red[tid * V + e] = f[e];
                }
            }
            __syncthreads();
            for (int g = wave; g < p.groups; g += NW) {
                float s = 0.0f;
                int q = lane / each, e = lane - q * each;
                const int dq = 64 / each, de = 64 - dq * each;
                while (q < slots) {
                    s += red[q * width + g * each + e];
                    q += dq;
                    e += de;
                    if (e >= each) {
                        e -= each;
                        ++q;
                    }
                }
                for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m);
                if (lane == 0) stat[g] = s;
            }
            __syncthreads();
            // of the thread's channels
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = stat[min((col * V + e) / cpg, p.groups - 1)];
        }
    };
    constexpr int S = SINGLE ? 1 : V;
    const float count = (float)px * (float)cpg;
    float f[V], mean[S], m2[S];
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = 0.0f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        float v[V];
        unpack<T, V>(u[i], v);
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] += !ends || inside(i, e) ? v[e] : 0.0f;
    }
    reduce(f, mean);
#pragma unroll
    for (int e = 0; e < S; ++e) mean[e] /= count;
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = 0.0f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        float v[V];
        unpack<T, V>(u[i], v);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float d = v[e] - mean[SINGLE ? 0 : e];
            f[e] += (ends ? inside(i, e) : off[i] != OOB) ? d * d : 0.0f;
        }
    }
    reduce(f, m2);

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
            for (int e = 0; e < V; ++e)
                if ((col * V + e) % cpg == 0) {
                    out[(col * V + e) / cpg * 2] = mean[e];
                    out[(col * V + e) / cpg * 2 + 1] = m2[e];
                }
        }
        return;
    }
    // ---- outputs ----
    float rstd[S], ga[V], be[V];
#pragma unroll
    for (int e = 0; e < S; ++e) rstd[e] = 1.0f / sqrtf(m2[e] / count + a.eps);
    if constexpr (!SINGLE) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = c0 + col * V + e;
            ga[e] = (a.gamma ? a.gamma[c] : 1.0f) * rstd[e];
            be[e] = a.beta ? a.beta[c] : 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (off[i] == OOB) continue;
        float v[V];
        unpack<T, V>(u[i], v);
        if constexpr (SINGLE) {
            const int c = (int)(off[i] % (uint32_t)(a.C * ESZ)) / ESZ;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int cc = min(c + e, a.C - 1);
                ga[e] = (a.gamma ? a.gamma[cc] : 1.0f) * rstd[0];
                be[e] = a.beta ? a.beta[cc] : 0.0f;
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e)
            v[e] = norm_act(__builtin_fmaf(v[e] - mean[SINGLE ? 0 : e], ga[e], be[e]), a.act);
        T* dst = (T*)((uint8_t*)y + off[i]);
        if (!ends || (inside(i, 0) && inside(i, V - 1))) {
            *(uint4*)dst = pack<T, V>(v);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (inside(i, e)) dst[e] = (T)v[e];
        }
    }
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
    const int g0 = ct * cols * V / cpg, g1 = (ct * cols * V + nc * V - 1) / cpg;
    for (int g = g0 + tid; g <= g1; g += APPLY_NT) {
        const float* q = part + ((int64_t)n * p.slabs * a.G + g) * 2;
        float mean = 0.0f, m2 = 0.0f;
        for (int s = 0; s < p.slabs; ++s)
            mean += q[(int64_t)s * a.G * 2] * ((float)min(p.px, a.P - s * p.px) / (float)a.P);
        for (int s = 0; s < p.slabs; ++s) {
            const float d = q[(int64_t)s * a.G * 2] - mean;
            m2 += q[(int64_t)s * a.G * 2 + 1] +
                  (float)min(p.px, a.P - s * p.px) * (float)cpg * d * d;
        }
        stat[2 * (g - g0)] = mean;
        stat[2 * (g - g0) + 1] = 1.0f / sqrtf(m2 / ((float)a.P * (float)cpg) + a.eps);
    }
    __syncthreads();
    const int step = APPLY_NT / cols, slot = tid / cols, col = tid - slot * cols;
    if (slot >= step || col >= nc) return;
    float mean[V], ga[V], be[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = (ct * cols + col) * V + e, g = c / cpg - g0;
        mean[e] = stat[2 * g];
        ga[e] = stat[2 * g + 1] * (a.gamma ? a.gamma[c] : 1.0f);
        be[e] = a.beta ? a.beta[c] : 0.0f;
    }
    const int first = rt * rows, last = min(a.P, first + rows);
    const int64_t at = (int64_t)n * a.P * CV + ct * cols + col;
    const uint4* x = (const uint4*)a.x + at;
    uint4* y = (uint4*)a.y + at;
    constexpr int B = 4;
    for (int q = first + slot; q < last; q += B * step) {
        uint4 u[B];
#pragma unroll
        for (int b = 0; b < B; ++b)
            if (q + b * step < last) u[b] = x[(int64_t)(q + b * step) * CV];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (q + b * step >= last) break;
            float v[V];
            unpack<T, V>(u[b], v);
#pragma unroll
            for (int e = 0; e < V; ++e)
                v[e] = norm_act(__builtin_fmaf(v[e] - mean[e], ga[e], be[e]), a.act);
            y[(int64_t)(q + b * step) * CV] = pack<T, V>(v);
        }
    }
}

template <typename T, int NT, int R>
void launch_norm(const GroupNormArgs& a, const NormPlan& p, float* part, hipStream_t s)
{
    const dim3 grid((uint32_t)((int64_t)a.N * p.slabs * p.chunks));
    if (p.single) PPIPE_LAUNCH((group_norm_kernel<T, NT, R, true>), grid, dim3(NT), 0, s, a, p, part);
    else PPIPE_LAUNCH((group_norm_kernel<T, NT, R, false>), grid, dim3(NT), 0, s, a, p, part);
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
    if (p.nt == 256) {
        if (p.r == 1) launch_norm<T, 256, 1>(a, p, part, s);
        else if (p.r == 2) launch_norm<T, 256, 2>(a, p, part, s);
        else launch_norm<T, 256, 4>(a, p, part, s);
    } else {
        if (p.r == 2) launch_norm<T, NORM_NT, 2>(a, p, part, s);
        else if (p.r == 4) launch_norm<T, NORM_NT, 4>(a, p, part, s);
        else if (p.r == 8) launch_norm<T, NORM_NT, 8>(a, p, part, s);
        else launch_norm<T, NORM_NT, 16>(a, p, part, s);
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
