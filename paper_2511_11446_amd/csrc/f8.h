// The layers in 8-bit floating point, routing to experts and the experts' layers: launch interface between the host side (f8_api.hip) and
// the kernels, and device helpers that they share.  Not part of the public ABI.
#pragma once
#include "ql_internal.h"

#include <atomic>

namespace ql {

constexpr int F8_BLOCK = 128;   // channels that share an activation scale, and the side of a weight block
constexpr float F8_MAX = 448.0f;
constexpr int F8_LDS = 160 * 1024;   // of a compute unit
constexpr int F8_UP = 64;       // outputs of an expert's row that share a power of two

inline int f8_blocks(int64_t n) { return (int)((n + F8_BLOCK - 1) / F8_BLOCK); }

struct F8DaqArgs {
    const void *x;       // fp16 [M,K]; [M,2K] with glu; fp32 [M,K] with wide
    void *q;             // e4m3 [M,K]
    float *scales;       // [M, KB]
    int M, K, KB;
    bool glu, wide;
    const int *rows;     // device: rows that there are (at most M), or null: M
};
hipError_t launch_daq_f8(const F8DaqArgs &a, hipStream_t stream);

// Where the rows of (token, choice) lie when they are sorted by expert.  All in device memory, in the call's workspace: whoever reads it holds what it says within the
// arrays (within, below), so that a workspace which other work writes to meanwhile gives wrong numbers and no access elsewhere.
struct ExpertRows {
    int *first;          // [E+1] first row of each expert, and how many rows there are
    int *order;          // [P] row -> token * k + choice
    int *place;          // [P] token * k + choice -> row, -1 without an expert
    int *tiles;          // [1 + 2 * most]: how many tiles of `tile` rows there are, then expert and first row of each; most = expert_tiles_most
    int *counts;         // [chunks][E] scratch
    int P, E, tile;
};
constexpr int EXPERT_CHUNK = 2048;   // rows that a workgroup sorts
inline int expert_chunks(int64_t P) { return (int)((P + EXPERT_CHUNK - 1) / EXPERT_CHUNK); }
inline int64_t expert_tiles_most(int64_t P, int64_t E, int tile) { return P / tile + (P < E ? P : E); }
hipError_t launch_expert_rows(const int *ids, const ExpertRows &r, const F8DaqArgs &x, hipStream_t stream);   // and quantizes x (fp16 rows, not gated)

// y[t] = residual[t] + sum_j weights[t,j] * o[place[t,j]]
struct ExpertSumArgs {
    const void *o;       // fp16 or (wide) fp32 [rows, N]
    const uint8_t *up;   // of fp16 rows: F8Gemm::up
    const int *place;    // [T,k] rows, or (ids) an expert where there is one: row token * k + choice
    bool ids;
    int E;
    const float *weights;
    const void *residual;
    void *y;
    int T, k, N;
    bool wide;
};
hipError_t launch_expert_sum(const ExpertSumArgs &a, hipStream_t stream);

struct RouteArgs {
    const void *logits;
    const float *bias;
    int *ids;
    float *weights;
    int T, E, k, groups, top_groups, group_top;
    bool wide, sigmoid, renorm;
    float scale;
};
hipError_t launch_route(const RouteArgs &a, hipStream_t stream);

struct F8Gemm {
    const uint8_t *q;    // e4m3 [M,K]
    const float *s;      // [M,KB]
    const uint8_t *w;    // e4m3 [N,K]; of experts [E][N,K], with gated [E][2][N,K]
    const float *s_w;    // [NB,KB] of each of these matrices
    int M, N, K, KB, NB;
    // a layer's epilogue
    const void *bias;
    int act;
    const void *residual, *gate;
    int gate_rows;
    void *y;             // fp16 [M,N]; of experts the rows' outputs, fp32 of few rows
    // experts: rows as ExpertRows says, or null
    const int *first, *tiles;
    const int *order;    // row -> token * k + choice where the rows of q are tokens, or null
    int k, tiles_most, tile;
    bool gated;          // the two matrices of an expert's gated layer: h = silu(g) * u, in fp32 [M,N] at y, or quantized at hq and hs
    uint8_t *hq;
    float *hs;
    uint8_t *up;         // of experts' fp16 outputs: [M, ceil(N/64)] powers of two that 64 neighbours are times (0 below 2^15)
    // rows that the launch quantizes itself (qgemm_f8_takes_rows, experts_f8_takes_ids), in the place of q and s
    const void *x;       // fp16 [M,K], [M,2K] with glu; of experts fp16 [M / k, K] gated, else fp32 [M,K]
    bool glu;
    const int *ids;      // of experts: [M] (M up to 16, experts_f8_takes_ids) in the place of first, tiles and order; outputs at row token * k + choice
    int E;
    bool codes;          // the matrix cores' own sums of codes will do (a layer of many rows that is not behind a gated product)
};
hipError_t launch_qgemm_f8(const F8Gemm &a, hipStream_t stream);
// rows of an expert's tile, by the rows that an expert has on average: 16, or F8_TILE_ROWS and more where the tiles quantize the gated product themselves
constexpr int F8_TILE_ROWS = 64;
int f8_expert_tile(int64_t P, int64_t E);
// rows from which on tiles are not of 16: h and o of fewer are fp32
inline int64_t f8_expert_few(int64_t E) { return E < 2 ? 384 * E : 12 * (E > 44 ? E : 44); }
// rows from which on a layer takes the matrix cores' own sums of codes, if it may
constexpr int F8_MANY = 256;
float qgemm_f8_tiles_us(const F8Gemm &a);
bool qgemm_f8_takes_rows(int64_t M, int64_t K, int64_t N, bool glu);
// steps of eight wavefronts that are requested at once, and the LDS that they and the rows take
inline int f8_self_steps(int KB) { return KB <= 8 ? 1 : KB <= 16 ? 2 : 4; }
inline int64_t f8_self_bytes(int64_t rows, int KB, bool gated) { return 8 * f8_self_steps(KB) * (gated ? 2 : 1) * 2048 + KB * rows * (F8_BLOCK + 4) + 2048 + 64; }
inline bool experts_f8_takes_ids(int64_t P, int64_t K, int64_t I, int64_t N)
{
    return P <= 16 && N <= 1 << 26 /* 2^31 threads */ && K <= 4096 && I <= 4096 && f8_self_bytes(P, f8_blocks(K), true) <= F8_LDS && f8_self_bytes(P, f8_blocks(I), false) <= F8_LDS;
}
hipError_t launch_qgemm_f8_tiles(const F8Gemm &a, hipStream_t stream);

// Once for a kernel and device: that it may use F8_LDS bytes of LDS (asked for at every launch it is 1 us of the host's time)
template <auto KERNEL>
hipError_t allow_lds()
{
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, F8_LDS);
    if (e == hipSuccess && dev < 64) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// ---- device helpers -------------------------------------------------------------------------------------------------------------

#ifdef __HIPCC__
typedef int v8i __attribute__((ext_vector_type(8)));

// v where it is one of 0..n-1, else one of them
__device__ __forceinline__ int within(int v, int n) { return (int)min((unsigned)v, (unsigned)n - 1u); }

// The expert's tile `tile` of a plan: its expert and rows [m0, m_end)
struct ExpertTile {
    int e, m0, m_end;
    __device__ __forceinline__ ExpertTile(const int *tiles, const int *first, int tile, int E, int rows)
        : e(within(tiles[1 + 2 * tile], E)), m0(within(tiles[2 + 2 * tile], rows)), m_end(max(m0, within(first[e + 1] - 1, rows)) + 1)
    {
    }
};

// silu(a) = a / (1 + 2^(-a log2 e)).  The exponent is taken in two parts (the product and what its rounding lost), so that the power is
// off by about 2^-22 for every a, not by 2^-24 of the exponent's size; v_exp_f32 and v_rcp_f32 are off by an ulp each.  Below a = -87 the
// result may be 0 where it is less than 2^-118.
__device__ __forceinline__ float silu_dev(float a)
{
    constexpr float L = -1.44269502f, L_REST = -1.92596299e-8f;   // -log2(e) = L + L_REST
    const float h = a * L;
    const float rest = __builtin_fmaf(a, L, -h) + a * L_REST;
    // 2^rest = 1 + rest ln 2, |rest| < 2^-6 even at the end of binary16's range, where the power is infinite or 0; an infinite power stays so
    const float e = __builtin_amdgcn_exp2f(h) * __builtin_fmaf(rest, 0.693147182f, 1.0f);
    return a * __builtin_amdgcn_rcpf(1.0f + e);
}

// The codes of one block: 448 v / amax to the nearest e4m3 value.  With r = fl(1 / amax), q0 = fl(t r) and the remainder t - q0 amax, which an fma gives without
// error, q0 + remainder * r is the quotient with less than one rounding of error and exactly where it is representable.  t = 448 v is exact for binary16 v; a quotient of
// such a t (14 bits) and a binary16 amax (11 bits) that is no tie of e4m3 (5 bits) is at least 2^-16 away from one, so the codes are those of the exact quotient.
// An amax so small that 1 / amax would be infinite, or so large that 448 of it would be (gated values only), is brought nearer to 1 with the values.  (What 2^-64 makes
// subnormal of them is below 2^-120 of amax: its code is 0.)
struct F8Scale {
    float amax, r, up;
    __device__ __forceinline__ explicit F8Scale(float a)
    {
        const float by = a < 0x1p-60f ? 0x1p64f : a > 0x1p60f ? 0x1p-64f : 1.0f;
        up = by * F8_MAX;
        amax = a == 0.0f ? 1.0f : a * by;
        r = 1.0f / amax;
    }
    __device__ __forceinline__ float code(float v) const
    {
        const float t = v * up, q = t * r;
        return __builtin_fmaf(__builtin_fmaf(-q, amax, t), r, q);
    }
    __device__ static __forceinline__ float scale(float a) { return a == 0.0f ? 1.0f : a / F8_MAX; }
};

// The products of a step of 128 channels, 16 x 16 of them, a lane's 32 bytes of either operand.
//
// Wide: the codes are taken to binary16, which holds every e4m3 value, and multiplied by v_mfma_f32_16x16x32_f16, whose sums keep 24 bits.
// Plain codes: v_mfma_f32_16x16x128_f8f6f4.  It lines the products of 8 neighbouring channels up under the largest of them and cuts off what lies
// more than 13 bits below that one's exponent, towards zero (measured: beside 2^16 a product of 15 counts as 8, of 7 as nothing; the eights are then added
// in 24 bits).  From registers it is twice as fast: 3580 against 1680 TFLOP/s with the fold, conversions counted.
// Which one: the second leaves 2e-5 of the result's size on activations as layers have them and 2.6e-4 behind a gated product, whose values in a block are
// further apart (the result's own rounding to binary16 leaves 2.1e-4).  Where codes are made of the result, every error next to the border of two codes
// becomes a whole step: the outputs of the experts' layers were 1.7e-3 off with it, 2e-4 without.  So it is taken for plain layers of many rows only.
typedef _Float16 f8_h2 __attribute__((ext_vector_type(2)));
typedef _Float16 f8_h8 __attribute__((ext_vector_type(8)));
typedef float f8_v4f __attribute__((ext_vector_type(4)));
struct Wide {
    f8_h8 h[4];
    Wide() = default;
    __device__ __forceinline__ explicit Wide(v8i c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f8_h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 * i], 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 * i], 1.0f, true);
            const f8_h2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 * i + 1], 1.0f, false), e = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 * i + 1], 1.0f, true);
            h[i] = f8_h8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
        }
    }
};
__device__ __forceinline__ f8_v4f step_product(const Wide &a, const Wide &b)
{
    f8_v4f d = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h[i], b.h[i], d, 0, 0, 0);
    return d;
}
__device__ __forceinline__ f8_v4f step_product(v8i a, v8i b)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f8_v4f{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
}

// the largest of 16 lanes' values, in all of them
__device__ __forceinline__ float max16(float m)
{
#define QL_ROR(ctrl) m = fmaxf(m, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, m), ctrl, 0xF, 0xF, true)));
    QL_ROR(0x128)
    QL_ROR(0x124)
    QL_ROR(0x122)
    QL_ROR(0x121)
#undef QL_ROR
    return m;
}

// four values to e4m3, round to nearest even; lowest first
__device__ __forceinline__ unsigned f8_pack4(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
#endif

}  // namespace ql
