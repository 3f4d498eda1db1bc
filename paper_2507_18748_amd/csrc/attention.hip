// Attention over [batch][token][head][dim] tensors by strides (see
// ppipe_attention_desc), and the spans of keys that its queries see.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c s_ij - M_i)
//
// in one pass over the keys with a running maximum M and sum.  The scores are
// computed transposed, S^T = K Q^T, so that a lane holds one query's scores
// (half of a tile's keys, the other half wave the other half): maximum and sum
// stay in the lane, and the weights are already the right operand of
// O^T = V^T P^T if the keys of V^T come in the same order, which the transposing
// LDS reads give for 16-bit types and plain reads for fp32.
//
// Rows: the queries of all heads that share a key head, (token, head) with the
// head fastest, 32 to a wave, so that few tokens with many heads fill a tile.
#include "attention_device.h"

#include <algorithm>

namespace ppipe {
namespace {

// A thread finds the document of one query by bisection (3.1 us for 8191 queries
// of 9 documents, the launch for the most part).
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

// Parts of the splits brought to one maximum, added in split order and
// normalised; a thread takes four elements of a row and reads four parts at a time
// (one after another they took 8 us instead of 4 for 16 x 32 rows in 4 parts).
template <typename T>
__global__ void __launch_bounds__(64) attention_join_kernel(AttentionArgs a, AttentionPlan p)
{
    const int64_t x = (int64_t)blockIdx.x * 64 + threadIdx.x, all = (int64_t)a.N * a.Hk * p.rows;
    const int quads = a.d / 4;
    const int64_t row = x / quads;
    const int e = 4 * (int)(x - row * quads);
    if (row >= all) return;
    const float2* ml = (const float2*)p.ml + row;
    const float* part = p.part + row * a.d + e;
    float m = -INFINITY, w = 0.0f;
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) m = fmaxf(m, ml[s * all].x);
    float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
        // a part without weight counts nothing; one of NaN scores alone has no
        // maximum but its weight
        const float2 x = ml[s * all];
        const float f = x.y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(x.x - m);
        const float4 v = *(const float4*)(part + s * all * a.d);
        w += x.y * f;
        sum.x += v.x * f; sum.y += v.y * f; sum.z += v.z * f; sum.w += v.w * f;
    }
    const int64_t group = row / p.rows;
    const int r = (int)(row - group * p.rows), G = a.H / a.Hk, i = r / G;
    const int n = (int)(group / a.Hk), h = (int)(group - (int64_t)n * a.Hk) * G + r - i * G;
    T* y = (T*)a.out + n * a.os[0] + i * a.os[1] + h * a.os[2] + e;
    const float inv = w == 0.0f ? 0.0f : 1.0f / w;
    Vec4<T>::store(y, make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
}

// Rows of one key head up to 32, or so few that blocks of 32 rows all run at once
// (two to a CU up to 128 bytes of head, else one, by their LDS): the waves of a
// block split the keys.  Measured, rows split / keys split (8 heads, us): 14x14
// maps f32 of 32 x 3 16.1 / 8.5, bf16 of 64 x 1 9.1 / 7.7, x 4 9.3 / 8.0, 32x32 maps of 64 x 2
// 18.6 / 15.8, f32 of 64 x 1 76 / 36; beyond one round: 32x32 of 128 x 3 27.6 / 45.6,
// 14x14 of 32 x 16 8.0 / 11.6.
// Few blocks: the keys are split further among blocks until the chip is filled;
// each part keeps at least 512 keys of heads of 64, 256 from 128 on, for what the
// join costs (256 and 512: 900 tokens of 2 heads of 64 12.3 / 11.0 us, a token of 8
// heads of 128 against 4000 keys 15.2 / 18.6; fp32, whose tiles take several times
// as long: 256 of heads of 64, 64 of 256; 32 and 512 keys there: 500 tokens of 8
// heads of 128 32.7 / 44.6 / 45.1 us).
AttentionChoice choose(int dt, const AttentionArgs& a, int cus)
{
    AttentionChoice c;
    const int64_t rows = (int64_t)a.Lq * (a.H / a.Hk), groups = (int64_t)a.N * a.Hk;
    c.splitk = rows <= 32 || groups * ((rows + 31) / 32) <=
                                 (int64_t)cus * (a.d * dtype_size(dt) <= 128 ? 2 : 1);
    const int per = c.splitk ? 32 : 128;
    c.tiles = (int)((rows + per - 1) / per);
    c.splits = 1;
    const int part = dt == DT_F32 ? std::max(64, 256 * 64 / a.d)
                                  : std::min(512, std::max(256, 512 * 64 / a.d));
    while (c.splitk && c.splits < 64 && groups * c.tiles * c.splits < 2 * cus &&
           a.Lk / (c.splits * 2) >= part)
        c.splits *= 2;
    c.blocks = groups * c.tiles * c.splits;
    return c;
}

AttentionPlan plan_of(int dt, const AttentionArgs& a, const AttentionChoice& c, void* ws)
{
    AttentionPlan p;
    p.rows = a.Lq * (a.H / a.Hk);
    p.tiles = c.tiles;
    p.splits = c.splits;
    // The scale goes into the exponent where it can: with a bias and no cap the
    // slopes are divided by it (a scale beyond 2^+-40 multiplies the scores instead).
    constexpr double LOG2E = 1.4426950408889634;
    p.sign = a.scale == 0.0f ? 0 : a.scale < 0.0f ? -1 : 1;
    const float scale = a.scale == 0.0f ? 1.0f : fabsf(a.scale);
    const bool fold = scale > 0x1p-40f && scale < 0x1p40f;
    p.capc = a.cap > 0.0f ? (float)(2.0 * LOG2E * scale / a.cap) : 0.0f;
    p.capk = 2.0f * a.cap;
    p.pre = scale;
    p.slope = 1.0f;
    p.c = (float)LOG2E;
    p.cap_mode = a.cap == 0.0f ? CAP_NONE
                 : dt == DT_F32 || a.cap > 1024.0f ? CAP_EXACT : a.slopes ? CAP_SUM : CAP_ALONE;
    if (p.cap_mode == CAP_ALONE) {
        p.c = (float)(LOG2E * p.capk);
    } else if (a.cap == 0.0f && (fold || !a.slopes)) {
        p.pre = 1.0f;
        p.slope = 1.0f / scale;
        p.c = (float)(LOG2E * scale);
    }
    const int64_t groups = (int64_t)a.N * a.Hk;
    p.by_tile = c.splits == 1 && groups % NUM_XCD != 0 && groups <= 64;
    const int64_t all = groups * p.rows;
    p.part = (float*)ws;
    p.ml = ws ? (float*)ws + c.splits * all * a.d : nullptr;
    return p;
}

}  // namespace

hipError_t launch_attention_spans(const SpansArgs& a, hipStream_t s)
{
    const dim3 grid((uint32_t)(((int64_t)a.N * a.Lq + 255) / 256)), block(256);
    PPIPE_LAUNCH(attention_spans_kernel, grid, block, 0, s, a);
    return hipGetLastError();
}

size_t attention_workspace(int dt, const AttentionArgs& a, int cus)
{
    const AttentionChoice c = choose(dt, a, cus);
    return c.splits > 1 ? (size_t)c.splits * a.N * a.Lq * a.H * (a.d + 2) * 4 : 0;
}

bool attention_fits(int dt, const AttentionArgs& a, int cus)
{
    const AttentionChoice c = choose(dt, a, cus);
    return c.blocks < 1 << 24 && (c.splits == 1 || (double)a.N * a.Lq * a.H * (a.d / 4) < 4294967040.0);
}

int attention_launches(int dt, const AttentionArgs& a, int cus)
{
    return choose(dt, a, cus).splits > 1 ? 2 : 1;
}

const char* attention_name(int dt, const AttentionArgs&, int, int launch)
{
    static const char* names[2][3] = {
        {"attention<f32>", "attention<f16>", "attention<bf16>"},
        {"attention_join<f32>", "attention_join<f16>", "attention_join<bf16>"}};
    return names[launch][dt];
}

hipError_t launch_attention(int dt, const AttentionArgs& a, void* ws, int cus, int launch,
                            hipStream_t s)
{
    const AttentionChoice c = choose(dt, a, cus);
    const AttentionPlan p = plan_of(dt, a, c, ws);
    if (launch == 1) {
        const int64_t n = (int64_t)a.N * a.Lq * a.H * (a.d / 4);
        const dim3 grid((uint32_t)((n + 63) / 64)), block(64);
        if (dt == DT_F32) PPIPE_LAUNCH(attention_join_kernel<float>, grid, block, 0, s, a, p);
        else if (dt == DT_F16) PPIPE_LAUNCH(attention_join_kernel<_Float16>, grid, block, 0, s, a, p);
        else PPIPE_LAUNCH(attention_join_kernel<__bf16>, grid, block, 0, s, a, p);
        return hipGetLastError();
    }
    if (dt == DT_F32) launch_attention_f32(a, p, c, s);
    else if (dt == DT_F16) launch_attention_f16(a, p, c, s);
    else launch_attention_bf16(a, p, c, s);
    return hipGetLastError();
}

}  // namespace ppipe
