// Device side of the attention kernels: tile loads, matrix instructions and
// the pass over the keys with a running maximum and sum.
#pragma once
#include "gemm_device.h"

namespace ppipe {

typedef float accx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

// How scores are capped: cap tanh x = cap - 2 cap / (2^(2 x log2 e) + 1).
// Alone, the constant drops out of the softmax and the factor is the
// exponent's.  These two lose 2^-23 of the cap, which 16-bit weights bear up to a
// cap of 1024; fp32 and larger caps take the exact form (16-bit: a series where x is small).
enum CapMode { CAP_NONE = 0, CAP_ALONE = 1, CAP_SUM = 2, CAP_EXACT = 3 };

// What a launch adds to the call's arguments.
struct AttentionPlan {
    int rows;          // query rows of one key head: Lq * (H / Hk)
    int tiles;         // row tiles of one key head
    int splits;        // key ranges per row tile
    int by_tile;       // blocks in the order of row tiles, not key heads
    int cap_mode;
    float capc, capk;  // with a cap: tanh's exponent per unit of q . k; 2 cap
    float c;           // powers of two per unit of the scores as they are kept
    float pre;         // factor of the scores before a bias
    float slope;       // factor of the slopes
    int sign;          // 0: q is read as zeros, -1: with its sign turned
    float* part;       // [splits][N * Hk * rows][d] sums and [..][2] maxima and weights
    float* ml;
};

// How a call is cut into blocks.
struct AttentionChoice {
    bool splitk;       // the waves of a block take keys, not rows
    int tiles, splits;
    int64_t blocks;
};
void launch_attention_f32(const AttentionArgs& a, const AttentionPlan& p, const AttentionChoice& c,
                          hipStream_t s);
void launch_attention_f16(const AttentionArgs& a, const AttentionPlan& p, const AttentionChoice& c,
                          hipStream_t s);
void launch_attention_bf16(const AttentionArgs& a, const AttentionPlan& p, const AttentionChoice& c,
                           hipStream_t s);

// One 32 x 32 block of products over 16 bytes of k per lane (16-bit types:
// 16 of k, half a wave each 8; fp32: 8 of k, half a wave each 4, in four
// instructions).  Lane l gives row or column l % 32; of the result it holds
// column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4 in register i.
template <typename T> struct Mfma32;
template <> struct Mfma32<_Float16> {
    static __device__ __forceinline__ void step(const uint4& a, const uint4& b, accx16& c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a),
                                                   __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
    }
};
template <> struct Mfma32<__bf16> {
    static __device__ __forceinline__ void step(const uint4& a, const uint4& b, accx16& c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                    __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mfma32<float> {
    static __device__ __forceinline__ void step(const uint4& a, const uint4& b, accx16& c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
    }
};

// One 4-byte load per lane into LDS (see dma16).
__device__ __forceinline__ void dma4(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(voff), "s"(r) : "memory");
}

__device__ __forceinline__ uint32_t lds_address(const void* p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// Four 16-bit values of one column: lane l of each 16 names the 8 bytes of row
// l / 4, columns 4 (l % 4) of a 4 x 16 block and receives column l's four rows.
__device__ __forceinline__ uint2 lds_read_columns(uint32_t addr)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) shortx4*)(uintptr_t)addr));
}

// Maximum of the two half waves.
__device__ __forceinline__ float half_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ int wave_min(int v)
{
    for (int m = 32; m; m >>= 1) v = min(v, __shfl_xor(v, m));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_max(int v)
{
    for (int m = 32; m; m >>= 1) v = max(v, __shfl_xor(v, m));
    return __builtin_amdgcn_readfirstlane(v);
}

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 lds_read16(uint32_t addr)
{
    return __builtin_bit_cast(uint4, *(const __attribute__((address_space(3))) uintx4*)(uintptr_t)addr);
}
__device__ __forceinline__ float lds_read_f32(uint32_t addr)
{
    return *(const __attribute__((address_space(3))) float*)(uintptr_t)addr;
}

__device__ __forceinline__ uint32_t word(const uint4& u, int w)
{
    return w == 0 ? u.x : w == 1 ? u.y : w == 2 ? u.z : u.w;
}

// |a - b| + c of integers whose sign bits were turned.
__device__ __forceinline__ uint32_t sad(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("v_sad_u32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// Two values rounded to a 16-bit type, and a + b + c of such a pair: the sum of
// the weights as the products with the values see them.
typedef float floatx2 __attribute__((ext_vector_type(2)));
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b)
{
    typedef T pair __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2){a, b}, pair));
}
template <typename T> __device__ __forceinline__ float add2(uint32_t u, float c)
{
    typedef T pair __attribute__((ext_vector_type(2)));
    if constexpr (std::is_same<T, __bf16>::value)
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair, u),
                                               (pair){(T)1.0f, (T)1.0f}, c, false);
    else
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(pair, u), (pair){(T)1.0f, (T)1.0f}, c, false);
}

// z, or NaN if one of two 16-bit values is not finite.
template <typename T> __device__ __forceinline__ float add_not_finite(uint32_t u, float z)
{
    typedef T pair __attribute__((ext_vector_type(2)));
    if constexpr (std::is_same<T, __bf16>::value)
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair, u), (pair){}, z, false);
    else
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(pair, u), (pair){}, z, false);
}

// SPLITK: the waves of a block share one tile of rows and take key tiles in
// turn, each with LDS of its own and no barrier (few rows, long caches: bound
// by memory; single tokens of 16 streams, 32 heads on 8 of 128, up to 16384 keys, f16:
// 149 us, 5.0 TB/s).  Otherwise they take rows of their own and share
// the key tiles (bound by the matrix cores and, heads of 64 and less or with cap or
// bias, by the vector instructions of a score; 4 x 64x64 maps, 16 heads of 128, bf16:
// 510-535 us, 1.03-1.08 PFLOP/s; 8 x 64x64 maps, 16 heads of 64, f16: 612 us, 0.9 PFLOP/s).
// A key tile is 64 keys, two stages of it 64 KB at heads of 128, so two blocks fit
// a CU; from heads of 136 on 32 keys, whose scores and weights leave the registers room.
template <typename T, int DP, bool SPLITK> struct AttentionTile {
    static constexpr int ESZ = (int)sizeof(T);
    static constexpr int CH = DP * ESZ / 16;                    // 16-byte vectors of a row
    static constexpr int BK = SPLITK || DP * ESZ > 256 * (ESZ / 2) ? 32 : 64;
    static constexpr int KT = BK / 32;
    static constexpr int POS = 64 * 3 * 4;                      // key positions of a tile
    static constexpr int STAGE = 2 * BK * DP * ESZ + POS;
    static constexpr int NW = !SPLITK || 8 * STAGE <= 160 * 1024 ? 4 : 4 * STAGE <= 160 * 1024 ? 2 : 1;
    static constexpr int STAGES = 2 * (SPLITK ? NW : 1);
    static constexpr int JOIN = SPLITK && NW > 1 ? NW * 32 * (DP + 2) * 4 : 0;
    static constexpr int LDS = STAGES * STAGE > JOIN ? STAGES * STAGE : JOIN;
    static constexpr int WAVES = ESZ == 2 && DP <= 128 && !SPLITK ? 2 : 1;   // per SIMD
    static constexpr int ROWS = SPLITK ? 32 : 32 * NW;     // rows of a block
    static constexpr int NI = BK * CH / 64;                     // wave loads of a K or V tile
    static constexpr int NL = SPLITK ? NI : NI / NW;            // of them, one wave's
    // LDS has 64 banks: 16 lanes of a 16-byte read, 32 of an 8-byte one must lie in
    // different 16 or 8 bytes of 256.  Row r keeps vector c of K at c ^ kswz(r), so
    // the 16 rows that a fragment read takes at once do; of V, 16-bit, at
    // c ^ vswz(r): the 4 rows x 64 bytes of two transposing reads do.
    static __device__ __forceinline__ int kswz(int r)
    {
        return CH % 16 == 0 ? r & 15 : CH % 8 == 0 ? (r >> 1) & 7 : (r >> 2) & 3;
    }
    static __device__ __forceinline__ int vswz(int r)
    {
        return ESZ == 4 || CH % 8 ? 0 : CH % 16 == 0 ? (r & 3) << 2 : ((r >> 1) & 1) << 2;
    }
};

template <typename T, int DP, bool SPLITK, bool EXTRA>
__global__ void __launch_bounds__((AttentionTile<T, DP, SPLITK>::NW * 64),
                                  (AttentionTile<T, DP, SPLITK>::WAVES))
attention_kernel(AttentionArgs a, AttentionPlan p)
{
    using TL = AttentionTile<T, DP, SPLITK>;
    constexpr int ESZ = TL::ESZ, CH = TL::CH, BK = TL::BK, KT = TL::KT, NW = TL::NW, NL = TL::NL;
    constexpr int DT = DP / 32, RB = DP * ESZ, KB = BK * RB;
    constexpr int EPV = 16 / ESZ;
    __shared__ __align__(1024) uint8_t lds[TL::LDS];
    __shared__ int range[2 * NW];

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int col = lane % 32, half = lane / 32;
    // Blocks of one key head lie on one XCD, the later rows (more keys under a
    // causal mask) first.  A number of key heads that the XCDs do not divide goes
    // row tile by row tile, or some would get the long rows alone (causal, 4 key
    // heads: 193 -> 132 us).
    const uint32_t xcd = blockIdx.x % NUM_XCD;
    uint32_t lin = blockIdx.x;
    int split = 0, tile, group;                                // group: n * Hk + hk
    if (p.by_tile) {
        const uint32_t groups = (uint32_t)(a.N * a.Hk);
        tile = p.tiles - 1 - (int)(lin / groups);
        group = (int)(lin % groups);
    } else {
        const uint32_t per = gridDim.x / NUM_XCD, rem = gridDim.x % NUM_XCD;
        lin = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / NUM_XCD;
        split = lin % (uint32_t)p.splits;
        lin /= (uint32_t)p.splits;
        tile = p.tiles - 1 - (int)(lin % (uint32_t)p.tiles);
        group = (int)(lin / (uint32_t)p.tiles);
    }
    const int n = group / a.Hk, hk = group - n * a.Hk, G = a.H / a.Hk;

    // ---- this lane's row: query, span, bias ----
    const int row0 = tile * TL::ROWS + (SPLITK ? 0 : wave * 32);
    uint4 q[CH / 2];
    const int r = row0 + col;
    const bool ok = r < p.rows;
    const int i = ok ? r / G : 0, h = hk * G + (ok ? r - i * G : 0);
    const T* qr = (const T*)a.q + n * a.qs[0] + i * a.qs[1] + h * a.qs[2];
#pragma unroll
    for (int c = 0; c < CH / 2; ++c) {
        const int e = (2 * c + half) * EPV;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (ok && e < a.d && p.sign) u = *(const uint4*)(qr + e);
        if (p.sign < 0) {
            const uint32_t m = ESZ == 4 ? 0x80000000u : 0x80008000u;
            u.x ^= m; u.y ^= m; u.z ^= m; u.w ^= m;
        }
        q[c] = u;
    }
    int lo = 0, hi = ok ? a.Lk : 0;
    if (ok && a.spans) {
        const int* sp = a.spans + n * a.sps + 2 * (int64_t)i;
        lo = max(sp[0], 0);
        hi = min(sp[1], a.Lk);
    }
    if (hi <= lo) lo = hi = 0;
    float slope = 0.0f;
    uint32_t qp[3];
    if constexpr (EXTRA) {
        slope = a.slopes && ok ? a.slopes[h] * p.slope : 0.0f;
#pragma unroll
        for (int x = 0; x < 3; ++x)
            qp[x] = a.slopes && ok && x < a.A
                        ? (uint32_t)a.qpos[n * a.qps + (int64_t)i * a.A + x] ^ 0x80000000u : 0u;
    }
    // the wave's rows see keys from wlo to whi, and all of them those from wlo_max to whi_min
    const int wlo = wave_min(hi > lo ? lo : 0x7fffffff), whi = wave_max(hi);
    const int wlo_max = wave_max(lo), whi_min = wave_min(ok ? hi : 0x7fffffff);

    // ---- the block's keys, and this split's part of them in whole tiles ----
    int kbeg = wlo, kend = whi;
    if constexpr (!SPLITK) {
        if (lane == 0) {
            range[wave] = wlo;
            range[NW + wave] = whi;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            kbeg = min(kbeg, range[w]);
            kend = max(kend, range[NW + w]);
        }
        kbeg = __builtin_amdgcn_readfirstlane(kbeg);
        kend = __builtin_amdgcn_readfirstlane(kend);
    }
    int ntiles = kend > kbeg ? (kend - kbeg + BK - 1) / BK : 0;
    if (p.splits > 1) {
        const int each = (ntiles + p.splits - 1) / p.splits;
        const int first = min(split * each, ntiles);
        ntiles = min(each, ntiles - first);
        kbeg += first * BK;
        kend = min(kend, kbeg + ntiles * BK);
    }
    if constexpr (SPLITK) {                    // tiles wave, wave + NW, ... are this wave's
        kbeg += wave * BK;
        ntiles = ntiles > wave ? (ntiles - wave + NW - 1) / NW : 0;
    }
    constexpr int STEP = SPLITK ? NW * BK : BK;

    // ---- tile loads: LDS-direct, each lane its own (swizzled) vector ----
    const int kst = (int)a.ks[1] * ESZ, vst = (int)a.vs[1] * ESZ;
    uint32_t koff[NL], voff[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int vi = ((SPLITK ? 0 : wave * NL) + i) * 64 + lane, r = vi / CH, s = vi - r * CH;
        const int kc = s ^ TL::kswz(r), vc = s ^ TL::vswz(r);
        koff[i] = kc * EPV < a.d ? (uint32_t)(r * kst + kc * 16) : OOB;
        voff[i] = vc * EPV < a.d ? (uint32_t)(r * vst + vc * 16) : OOB;
    }
    const T* kbase = (const T*)a.k + n * a.ks[0] + hk * a.ks[2];
    const T* vbase = (const T*)a.v + n * a.vs[0] + hk * a.vs[2];
    const uint32_t lds0 = lds_address(lds) + (SPLITK ? wave * 2 * TL::STAGE : 0);
    auto load_tile = [&](int k0, int stage) {
        const uint32_t dst = lds0 + stage * TL::STAGE;
        const int valid = min(kend - k0, BK);
        const auto kr = make_rsrc(kbase + (int64_t)k0 * a.ks[1], (uint32_t)((valid - 1) * kst + a.d * ESZ));
        const auto vr = make_rsrc(vbase + (int64_t)k0 * a.vs[1], (uint32_t)((valid - 1) * vst + a.d * ESZ));
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const uint32_t at = dst + ((SPLITK ? 0 : wave * NL) + i) * 1024;
            dma16(kr, koff[i], __builtin_amdgcn_readfirstlane(at));
            dma16(vr, voff[i], __builtin_amdgcn_readfirstlane(at + KB));
        }
        if constexpr (EXTRA)
            if (a.slopes) {
                const auto pr = make_rsrc(a.kpos + n * a.kps + (int64_t)k0 * a.A,
                                          (uint32_t)(valid * a.A * 4));
#pragma unroll
                for (int x = 0; x < 3; ++x)
                    if (x < a.A && (SPLITK || wave == x))
                        dma4(pr, lane < BK ? (uint32_t)((lane * a.A + x) * 4) : OOB,
                             __builtin_amdgcn_readfirstlane(dst + 2 * KB + x * 256));
            }
    };

    // the queries (and their positions) are here before the loop: else every tile
    // would wait for all loads under way, the next tile's among them, before its
    // first product
#pragma unroll
    for (int c = 0; c < CH / 2; ++c)
        asm volatile("" : "+v"(q[c].x), "+v"(q[c].y), "+v"(q[c].z), "+v"(q[c].w));
    if constexpr (EXTRA)
        asm volatile("" : "+v"(slope), "+v"(qp[0]), "+v"(qp[1]), "+v"(qp[2]));

    accx16 o[DT];
    float M = -INFINITY, l = 0.0f;       // running maximum (a power of two) and sum of weights
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = accx16{};
    constexpr int KX = CH % 16 == 0 ? 8 : CH % 8 == 0 ? 4 : 2;    // vector pairs that the swizzle mixes
    const int kswz = TL::kswz(col);
    const uint32_t kread = (uint32_t)(col * RB + ((half ^ kswz) * 16));
    // 16-bit V: this lane's row and column of a transposing read, for four
    // blocks of 32 elements (the swizzle turns their order); fp32: its element
    const int vrow = ESZ == 2 ? 4 * half + (lane % 16) / 4 : 4 * half;
    const int vcol = 2 * ((lane / 16) % 2) + (lane % 4) / 2;
    uint32_t vread[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
        vread[d] = KB + vrow * RB + (ESZ == 2 ? ((4 * d + vcol) ^ TL::vswz(vrow)) * 16 + (lane & 1) * 8
                                              : 32 * d * 4 + col * 4);

    auto tile_pass = [&](int k0, uint32_t src, auto seen_whole) {
        constexpr bool whole = decltype(seen_whole)::value;
        // this stage's read addresses, held apart from the loop (the compiler would
        // keep one for every read of both stages)
        uint32_t kat[KX], vat[4];
#pragma unroll
        for (int c = 0; c < KX; ++c) kat[c] = src + (kread ^ (c * 32));
#pragma unroll
        for (int d = 0; d < 4; ++d) vat[d] = src + vread[d];
#pragma unroll
        for (int c = 0; c < KX; ++c) asm volatile("" : "+v"(kat[c]));
        asm volatile("" : "+v"(vat[0]), "+v"(vat[1]), "+v"(vat[2]), "+v"(vat[3]));

        // ---- scores ----
        accx16 s[KT];
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int c = 0; c < CH / 2; ++c) {
                const uint4 kf = lds_read16(kat[c % KX] + (c / KX) * (32 * KX) + k * 32 * RB);
                if (c == 0) s[k] = accx16{};
                Mfma32<T>::step(kf, q[c], s[k]);
            }
        // six reads ahead of the products (two, the compiler's choice, leave each
        // product waiting for LDS)
        {
            constexpr int N = KT * (CH / 2), PER = ESZ == 4 ? 4 : 1, AHEAD = N < 6 ? N : 6;
            __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
            for (int i = 0; i < N - AHEAD; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, AHEAD * PER, 0);
        }
        if constexpr (EXTRA) {
            // one branch for the tile, not for each score
            auto each = [&](auto&& f) {
#pragma unroll
                for (int k = 0; k < KT; ++k)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[k][i] = f(s[k][i]);
            };
            if (p.cap_mode == CAP_EXACT) {
                if constexpr (ESZ == 4)
                    each([&](float v) { return a.cap * tanhf(v * p.pre / a.cap); });
                else
                    each([&](float v) {
                        const float u = v * p.pre, x = v * (p.pre / a.cap), y = x * x;
                        const float e = __builtin_amdgcn_exp2f(v * p.capc);
                        const float far = __builtin_fmaf(-p.capk, __builtin_amdgcn_rcpf(e + 1.0f), a.cap);
                        float near = __builtin_fmaf(y, -0.053968254f, 0.13333333f);
                        near = __builtin_fmaf(y, near, -0.33333333f);
                        return fabsf(x) < 0.125f ? __builtin_fmaf(u * y, near, u) : far;
                    });
            } else if (p.cap_mode == CAP_ALONE) {
                each([&](float v) {
                    return __builtin_amdgcn_rcpf(-1.0f - __builtin_amdgcn_exp2f(v * p.capc));
                });
            } else if (p.cap_mode == CAP_SUM) {
                each([&](float v) {
                    const float e = __builtin_amdgcn_exp2f(v * p.capc);
                    return __builtin_fmaf(-p.capk, __builtin_amdgcn_rcpf(e + 1.0f), a.cap);
                });
            } else if (p.pre != 1.0f) {
                each([&](float v) { return v * p.pre; });
            }
            auto bias = [&](auto axes) {
                constexpr int A = decltype(axes)::value;
#pragma unroll
                for (int k = 0; k < KT; ++k)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        uint4 kp[A];
#pragma unroll
                        for (int x = 0; x < A; ++x)
                            kp[x] = lds_read16(src + 2 * KB + x * 256 + (32 * k + 8 * g + 4 * half) * 4);
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            uint32_t dist = 0;
#pragma unroll
                            for (int x = 0; x < A; ++x)
                                dist = sad(qp[x], word(kp[x], b) ^ 0x80000000u, dist);
                            s[k][4 * g + b] = __builtin_fmaf(-slope, (float)dist, s[k][4 * g + b]);
                        }
                    }
            };
            if (a.slopes) {
                if (a.A == 1) bias(std::integral_constant<int, 1>{});
                else if (a.A == 2) bias(std::integral_constant<int, 2>{});
                else bias(std::integral_constant<int, 3>{});
            }
        }
        if constexpr (!whole) {
            // a bit for each of 32 keys, spread to a word that takes the score or -inf
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                const int from = min(max(lo - k0 - 32 * k, 0), 32), to = min(max(hi - k0 - 32 * k, 0), 32);
                const uint32_t seen = (uint32_t)((1ull << to) - 1) & ~(uint32_t)((1ull << from) - 1);
                const uint32_t mine = seen >> (4 * half);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t take = (uint32_t)((int)(mine << (31 - 8 * (i / 4) - i % 4)) >> 31);
                    s[k][i] = __uint_as_float((__float_as_uint(s[k][i]) & take) | (0xff800000u & ~take));
                }
            }
        }

        // ---- running maximum and sum, weights ----
        uint4 pf[KT * 2];
        float mx = s[0][0];
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[k][i]);
        mx = half_max(mx) * p.c;
        // the maximum follows only when weights would pass 2^8: they stay
        // within the 16-bit range and the sums within fp32
        if (__any(mx > M + 8.0f)) {
            const float mn = fmaxf(M, mx);
            const float alpha = M == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(M - mn);
            M = mn;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= alpha;
        }
        // weights of f16 are kept 2^6 up (at most 2^14), away from its small end
        constexpr float UP = std::is_same<T, _Float16>::value ? 6.0f : 0.0f;
        const float base = (M == -INFINITY ? 0.0f : M) - UP;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[k][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k][i], p.c, -base));
                if constexpr (ESZ == 4) l += s[k][i];
            }
        if constexpr (ESZ == 2)
#pragma unroll
            for (int k = 0; k < 2 * KT; ++k) {
                auto w = [&](int i) { return s[k / 2][8 * (k % 2) + i]; };
                // one rounding of the weights to the storage type: the matrix
                // instruction takes both operands in it
                pf[k] = make_uint4(pack2<T>(w(0), w(1)), pack2<T>(w(2), w(3)),
                                   pack2<T>(w(4), w(5)), pack2<T>(w(6), w(7)));
                l = add2<T>(pf[k].w, add2<T>(pf[k].z, add2<T>(pf[k].y, add2<T>(pf[k].x, l))));
            }

        // ---- values ----
        // Keys that only some rows see may hold NaN or infinities, and 0 x NaN
        // would reach the others: where a tile is not seen whole, non-finite
        // values are looked for and then added key by key, to their rows alone.
        if constexpr (ESZ == 2) {
            // values of the next 32 elements are read while these are multiplied
            uint4 vf[2][2 * KT];
            auto read_v = [&](int d, uint4* f) {
#pragma unroll
                for (int k = 0; k < 2 * KT; ++k) {
                    const uint32_t at = vat[d & 3] + (d / 4) * 256 + 16 * k * RB;
                    const uint2 x = lds_read_columns(at), y = lds_read_columns(at + 8 * RB);
                    f[k] = make_uint4(x.x, x.y, y.x, y.y);
                }
            };
            read_v(0, vf[0]);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const uint4* f = vf[d & 1];
                __builtin_amdgcn_sched_barrier(0);
                if (d + 1 < DT) read_v(d + 1, vf[(d + 1) & 1]);
                bool clean = true;
                if constexpr (!whole) {
                    float z = 0.0f;
#pragma unroll
                    for (int k = 0; k < 2 * KT; ++k)
#pragma unroll
                        for (int w = 0; w < 4; ++w) z = add_not_finite<T>(word(f[k], w), z);
                    clean = !__any(!(z == 0.0f));
                }
                if (whole || clean) {
#pragma unroll
                    for (int k = 0; k < 2 * KT; ++k) Mfma32<T>::step(f[k], pf[k], o[d]);
                } else {
#pragma unroll
                    for (int k = 0; k < 2 * KT; ++k)
#pragma unroll 1
                        for (int e = 0; e < 16; ++e) {
                            const uint32_t m = half == e / 8 ? (e & 1 ? 0xffff0000u : 0x0000ffffu) : 0u;
                            const int w = (e / 2) & 3;
                            auto only = [&](const uint4& u) {
                                return make_uint4(w == 0 ? u.x & m : 0u, w == 1 ? u.y & m : 0u,
                                                  w == 2 ? u.z & m : 0u, w == 3 ? u.w & m : 0u);
                            };
                            const int j = k0 + 16 * k + 4 * (e / 8) + (e & 3) + 8 * ((e >> 2) & 1);
                            const uint4 vk = only(f[k]);
                            accx16 one = accx16{};
                            Mfma32<T>::step(vk, only(pf[k]), one);
                            const bool sees = j >= lo && j < hi;
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[d][i] += sees ? one[i] : 0.0f;
                        }
                }
            }
        } else {
            // 16 keys and 32 elements at a time
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    float vf[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        vf[i] = lds_read_f32(vat[d & 3] + (d / 4) * 512 + (32 * k + 8 * (i / 4) + i % 4) * RB);
                    bool clean = true;
                    if constexpr (!whole) {
                        float z = 0.0f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) z += vf[i] * 0.0f;
                        clean = !__any(!(z == 0.0f));
                    }
                    if (whole || clean) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[i], s[k][i], o[d], 0, 0, 0);
                    } else {
#pragma unroll 1
                        for (int x = 0; x < 32; ++x) {
                            const int e = x / 16, i = x % 16;
                            const int j = k0 + 32 * k + 8 * (i / 4) + 4 * e + i % 4;
                            float v = 0.0f;
#pragma unroll
                            for (int y = 0; y < 16; ++y) v = y == i ? vf[y] : v;
                            float w = 0.0f;
#pragma unroll
                            for (int y = 0; y < 16; ++y) w = y == i ? s[k][y] : w;
                            const bool sees = j >= lo && j < hi;
                            const accx16 one = __builtin_amdgcn_mfma_f32_32x32x2f32(
                                half == e ? v : 0.0f, half == e ? w : 0.0f, accx16{}, 0, 0, 0);
#pragma unroll
                            for (int y = 0; y < 16; ++y) o[d][y] += sees ? one[y] : 0.0f;
                        }
                    }
                }
        }
    };

    // waits for tile `it`, sends the next one's loads, gives the tile's first key
    auto next_tile = [&](int it) {
        dma_wait<0>();
        lds_read_drain();
        if constexpr (!SPLITK) bare_barrier();
        const int k0 = kbeg + it * STEP;
        if (it + 1 < ntiles) load_tile(k0 + STEP, (it + 1) & 1);
        return k0;
    };
    // A tile that every row sees whole needs no mask and no care for its values.
    // Runs of such tiles have a loop of their own, in which the accumulators stay
    // where they are.
    auto whole = [&](int it) {
        const int k0 = kbeg + it * STEP;
        return k0 >= wlo_max && k0 + BK <= whi_min;
    };
    if (ntiles > 0) load_tile(kbeg, 0);
    for (int it = 0; it < ntiles;) {
        for (; it < ntiles && !whole(it); ++it) {
            const int k0 = next_tile(it);
            if (k0 < whi && k0 + BK > wlo)                     // some row of this wave sees it
                tile_pass(k0, lds0 + (it & 1) * TL::STAGE, std::false_type{});
        }
        for (; it < ntiles && whole(it); ++it) {
            const int k0 = next_tile(it);
            tile_pass(k0, lds0 + (it & 1) * TL::STAGE, std::true_type{});
        }
    }

    l += __shfl_xor(l, 32);
    auto row_of = [&](int r, int& i, int& h) {
        i = r / G;
        h = hk * G + r - i * G;
    };
    // four consecutive elements of a row: normalised, or this split's part
    auto store4 = [&](int r, int e, float w, float x0, float x1, float x2, float x3) {
        if (p.splits > 1) {
            float* part = p.part + (((int64_t)split * a.N * a.Hk + group) * p.rows + r) * a.d + e;
            *(float4*)part = make_float4(x0, x1, x2, x3);
            return;
        }
        int i, h;
        row_of(r, i, h);
        T* y = (T*)a.out + n * a.os[0] + i * a.os[1] + h * a.os[2] + e;
        const float inv = w == 0.0f ? 0.0f : 1.0f / w;
        Vec4<T>::store(y, make_float4(x0 * inv, x1 * inv, x2 * inv, x3 * inv));
    };
    auto store_ml = [&](int r, float m, float w) {
        float* ml = p.ml + (((int64_t)split * a.N * a.Hk + group) * p.rows + r) * 2;
        ml[0] = m;
        ml[1] = w;
    };
    if constexpr (!SPLITK || NW == 1) {
        const int r = row0 + col;
        if (r >= p.rows) return;
        if (p.splits > 1 && half == 0) store_ml(r, M, l);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int e = 32 * d + 8 * g + 4 * half;
                if (e < a.d)
                    store4(r, e, l, o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2],
                           o[d][4 * g + 3]);
            }
    } else {
        // the waves' parts meet in LDS, each brought to the common maximum
        float* f = (float*)lds;
        float* ml = f + NW * 32 * DP;
        dma_wait<0>();
        __syncthreads();
        if (half == 0) {
            ml[(wave * 32 + col) * 2] = M;
            ml[(wave * 32 + col) * 2 + 1] = l;
        }
        __syncthreads();
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) m = fmaxf(m, ml[(w * 32 + col) * 2]);
        const float scale = M == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(M - m);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(float4*)&f[(wave * 32 + col) * DP + 32 * d + 8 * g + 4 * half] =
                    make_float4(o[d][4 * g] * scale, o[d][4 * g + 1] * scale,
                                o[d][4 * g + 2] * scale, o[d][4 * g + 3] * scale);
        __syncthreads();
        const int rows = min(32, p.rows - row0);
        for (int x = threadIdx.x; x < rows * (DP / 4); x += NW * 64) {
            const int rr = x / (DP / 4), e = 4 * (x % (DP / 4));
            if (e >= a.d) continue;
            float top = -INFINITY, w = 0.0f;
            for (int v = 0; v < NW; ++v) top = fmaxf(top, ml[(v * 32 + rr) * 2]);
            float4 sum = make_float4(0, 0, 0, 0);
            for (int v = 0; v < NW; ++v) {
                // a part without weight counts nothing; one of NaN scores alone
                // has no maximum but its weight
                const float wv = ml[(v * 32 + rr) * 2 + 1];
                w += wv == 0.0f ? 0.0f : wv * __builtin_amdgcn_exp2f(ml[(v * 32 + rr) * 2] - top);
                const float4 part = *(const float4*)&f[(v * 32 + rr) * DP + e];
                sum.x += part.x; sum.y += part.y; sum.z += part.z; sum.w += part.w;
            }
            if (p.splits > 1 && e == 0) store_ml(row0 + rr, top, w);
            store4(row0 + rr, e, w, sum.x, sum.y, sum.z, sum.w);
        }
    }
}

template <typename T, int DP>
void launch_tile(const AttentionArgs& a, const AttentionPlan& p, const AttentionChoice& c, hipStream_t s)
{
    const dim3 grid((uint32_t)c.blocks);
    const bool extra = a.cap > 0.0f || a.slopes;
    if (c.splitk) {
        constexpr int NT = 64 * AttentionTile<T, DP, true>::NW;
        if (extra) PPIPE_LAUNCH((attention_kernel<T, DP, true, true>), grid, dim3(NT), 0, s, a, p);
        else PPIPE_LAUNCH((attention_kernel<T, DP, true, false>), grid, dim3(NT), 0, s, a, p);
    } else {
        if (extra) PPIPE_LAUNCH((attention_kernel<T, DP, false, true>), grid, dim3(256), 0, s, a, p);
        else PPIPE_LAUNCH((attention_kernel<T, DP, false, false>), grid, dim3(256), 0, s, a, p);
    }
}

template <typename T>
void launch_type(const AttentionArgs& a, const AttentionPlan& p, const AttentionChoice& c, hipStream_t s)
{
    if (a.d <= 32) launch_tile<T, 32>(a, p, c, s);
    else if (a.d <= 64) launch_tile<T, 64>(a, p, c, s);
    else if (a.d <= 96) launch_tile<T, 96>(a, p, c, s);
    else if (a.d <= 128) launch_tile<T, 128>(a, p, c, s);
    else if (a.d <= 192) launch_tile<T, 192>(a, p, c, s);
    else launch_tile<T, 256>(a, p, c, s);
}

}  // namespace ppipe
