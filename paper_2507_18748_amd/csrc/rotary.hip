// Rotary positions with one to three axes (see ppipe_rotary_desc).
//
//   (u, w) -> (u cos t - w sin t, u sin t + w cos t),  t = position * f
//
// Bound by memory: one read and one write of the heads.  A block takes a few
// tokens: it computes their sines and cosines once (into LDS) for all heads,
// while its first loads are under way.  The angle is reduced in 64 bits to a
// fraction of a turn (positions are 32-bit integers: position * f keeps 2^-21
// of a turn at the far end), then sine and cosine are taken in 32 bits.
// Two clips of 8x28x28 tokens, 24 heads of 64 of a packed map, bf16: 13.4 us, 5.8 TB/s
// (in part from the caches; element by element with the angle of each: 98 us).
#include "kernels.h"

#include <algorithm>
#include <cmath>

namespace ppipe {
namespace {

constexpr int ROT_NT = 256, ROT_MAX_PAIRS = 128, ROT_K = 4, ROT_TABLE = 2048;

// Turns per position of every pair, by value with the launch.
struct Turns {
    double f[ROT_MAX_PAIRS];
};

struct RotaryPlan {
    int P;                 // rotated pairs
    int first[3];          // first pair of each axis
    int turn, units;       // units of a head that turn, and with those that are copied
    int T;                 // tokens of a block
    FastDiv div_units, div_heads, div_p;
};

enum RotaryMode {
    HALVES = 0,            // pairs (p, p + P), both halves whole vectors
    NEIGHBOURS = 1,        // pairs (2p, 2p + 1)
    SCALAR = 2             // pairs (p, p + P) at any P, element by element
};

template <typename T, int MODE>
__global__ void __launch_bounds__(ROT_NT)
rotary_kernel(RotaryArgs a, RotaryPlan p, Turns turns)
{
    constexpr int ESZ = (int)sizeof(T), V = 16 / ESZ;
    // elements of a unit, and pairs of a unit that turns
    constexpr int E = MODE == SCALAR ? 1 : V, PU = MODE == SCALAR ? 1 : MODE == HALVES ? V : V / 2;
    __shared__ float2 cs[ROT_TABLE];
    const int tid = threadIdx.x;
    const int64_t t0 = (int64_t)blockIdx.x * p.T, tokens = (int64_t)a.N * a.L;
    const int T_ = (int)min((int64_t)p.T, tokens - t0);
    const int total = T_ * a.H * p.units;

    struct Unit {
        const T* x;
        T* y;
        int u, t;          // unit of its head, token of the block
    };
    auto unit = [&](int x) {
        Unit q;
        const int r = fast_div(x, p.div_units);
        q.u = x - r * p.units;
        q.t = fast_div(r, p.div_heads);
        const int h = r - q.t * a.H;
        const int64_t token = t0 + q.t;
        const int n = (int)(token / a.L), l = (int)(token - (int64_t)n * a.L);
        // first element: of the pair's first half, or of the copied rest
        const int e = MODE == NEIGHBOURS || q.u < p.turn ? q.u * E : 2 * p.P + (q.u - p.turn) * E;
        q.x = (const T*)a.x + n * a.xs[0] + l * a.xs[1] + h * a.xs[2] + e;
        q.y = (T*)a.y + n * a.ys[0] + l * a.ys[1] + h * a.ys[2] + e;
        return q;
    };
    struct Data {
        T u[E], w[E];
    };
    auto load = [&](const Unit& q, Data& d) {
        if constexpr (MODE == SCALAR) {
            d.u[0] = q.x[0];
            d.w[0] = q.u < p.turn ? q.x[p.P] : q.x[0];
        } else {
            const uint4 u = *(const uint4*)q.x;
            __builtin_memcpy(d.u, &u, 16);
            if (MODE == HALVES && q.u < p.turn) {
                const uint4 w = *(const uint4*)(q.x + p.P);
                __builtin_memcpy(d.w, &w, 16);
            }
        }
    };
    auto store = [&](T* y, const T* e) {
        if constexpr (MODE == SCALAR) {
            y[0] = e[0];
        } else {
            uint4 u;
            __builtin_memcpy(&u, e, 16);
            *(uint4*)y = u;
        }
    };
    auto finish = [&](const Unit& q, Data& d) {
        if (q.u < p.turn) {
            const float2* c = cs + q.t * p.P + q.u * PU;
            if constexpr (MODE == NEIGHBOURS) {
#pragma unroll
                for (int i = 0; i < PU; ++i) {
                    if (q.u * PU + i >= p.P) break;      // the rest of the last vector is copied
                    const float u = (float)d.u[2 * i], w = (float)d.u[2 * i + 1];
                    d.u[2 * i] = (T)(u * c[i].x - w * c[i].y);
                    d.u[2 * i + 1] = (T)(u * c[i].y + w * c[i].x);
                }
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float u = (float)d.u[i], w = (float)d.w[i];
                    d.u[i] = (T)(u * c[i].x - w * c[i].y);
                    d.w[i] = (T)(u * c[i].y + w * c[i].x);
                }
                store(q.y + p.P, d.w);
            }
        }
        store(q.y, d.u);
    };

    // first units on their way
    Unit q[ROT_K];
    Data d[ROT_K];
#pragma unroll
    for (int k = 0; k < ROT_K; ++k)
        if (tid + k * ROT_NT < total) {
            q[k] = unit(tid + k * ROT_NT);
            load(q[k], d[k]);
        }
    for (int x = tid; x < T_ * p.P; x += ROT_NT) {
        const int t = fast_div(x, p.div_p), i = x - t * p.P;
        const int64_t token = t0 + t;
        const int n = (int)(token / a.L), l = (int)(token - (int64_t)n * a.L);
        const int axis = i >= p.first[2] ? 2 : i >= p.first[1] ? 1 : 0;
        const double turn = (double)a.pos[n * a.ps + (int64_t)l * a.A + axis] * turns.f[i];
        const float f = (float)(turn - rint(turn));
        cs[x] = make_float2(cospif(2.0f * f), sinpif(2.0f * f));
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ROT_K; ++k)
        if (tid + k * ROT_NT < total) finish(q[k], d[k]);
    for (int x = tid + ROT_K * ROT_NT; x < total; x += ROT_NT) {
        const Unit r = unit(x);
        Data e;
        load(r, e);
        finish(r, e);
    }
}

template <typename T>
hipError_t launch_type(const RotaryArgs& a, int cus, hipStream_t s)
{
    const int V = 16 / (int)sizeof(T);
    RotaryPlan p;
    Turns turns;
    p.P = 0;
    // base^-e by products in 64-bit mantissas: the ladder's error stays below a
    // double's rounding
    for (int x = 0; x < 3; ++x) {
        const int n = x < a.A ? a.pairs[x] : 0;
        p.first[x] = n ? p.P : ROT_MAX_PAIRS + 1;
        p.P += n;
    }
    const long double two_pi = 6.283185307179586476925286766559L;
    const int all = p.P;
    long double r = powl((long double)a.base, -1.0L / all), f = 1.0L;
    for (int x = 0, i = 0; x < a.A; ++x) {
        if (!a.shared && a.pairs[x]) {
            r = powl((long double)a.base, -1.0L / a.pairs[x]);
            f = 1.0L;
        }
        for (int k = 0; k < a.pairs[x]; ++k, f *= r) turns.f[i++] = (double)(f / two_pi);
    }
    const int mode = a.adjacent ? NEIGHBOURS : p.P % V ? SCALAR : HALVES;
    p.turn = mode == NEIGHBOURS ? (2 * p.P + V - 1) / V : mode == HALVES ? p.P / V : p.P;
    p.units = p.turn;
    if (a.x != a.y)
        p.units += mode == NEIGHBOURS ? a.d / V - p.turn : (a.d - 2 * p.P) / (mode == HALVES ? V : 1);
    // tokens of a block: as many as its threads take at once, fewer while the
    // chip is not filled
    const int64_t tokens = (int64_t)a.N * a.L;
    int64_t t = std::max<int64_t>(1, ROT_K * ROT_NT / ((int64_t)a.H * p.units));
    t = std::min<int64_t>(t, ROT_TABLE / p.P);
    while (t > 1 && (tokens + t - 1) / t < 4 * cus) t = (t + 1) / 2;
    p.T = (int)t;
    p.div_units = fast_div_of((uint32_t)p.units);
    p.div_heads = fast_div_of((uint32_t)a.H);
    p.div_p = fast_div_of((uint32_t)p.P);
    const dim3 grid((uint32_t)((tokens + t - 1) / t)), block(ROT_NT);
    if (mode == HALVES) PPIPE_LAUNCH((rotary_kernel<T, HALVES>), grid, block, 0, s, a, p, turns);
    else if (mode == NEIGHBOURS) PPIPE_LAUNCH((rotary_kernel<T, NEIGHBOURS>), grid, block, 0, s, a, p, turns);
    else PPIPE_LAUNCH((rotary_kernel<T, SCALAR>), grid, block, 0, s, a, p, turns);
    return hipGetLastError();
}

}  // namespace

const char* rotary_name(int dt)
{
    return dt == DT_F32 ? "rotary<f32>" : dt == DT_F16 ? "rotary<f16>" : "rotary<bf16>";
}

hipError_t launch_rotary(int dt, const RotaryArgs& a, int cus, hipStream_t s)
{
    if (dt == DT_F32) return launch_type<float>(a, cus, s);
    if (dt == DT_F16) return launch_type<_Float16>(a, cus, s);
    return launch_type<__bf16>(a, cus, s);
}

}  // namespace ppipe
