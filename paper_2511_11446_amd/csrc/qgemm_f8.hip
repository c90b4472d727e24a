// e4m3 x e4m3 -> fp32 products with a scale for every row and 128 channels of the activations and every 128 x 128 block of the weights (gfx950),
// of a layer and of the experts' layers.
//
// A K step is one block of 128 channels: the matrix cores give its 16 x 16 sums from zero (f8.h), one fma a sum takes them into the
// result with the product of the two scales.  The weights are the instruction's first operand: a lane's four sums are then four outputs of one row, and as
// 16 outputs lie in one weight block, all its sums of a step have one scale: s[row] * s_w.
#include "qgemm_f8.h"

namespace ql {

// four neighbouring outputs of row m from column n on
template <bool WIDE>
__device__ __forceinline__ void store4(void *y, long long m, int N, int n, const float (&u)[4])
{
    if constexpr (WIDE) {
        float *at = static_cast<float *>(y) + m * N + n;
        if (N % 4 == 0) {
            if (n < N) *reinterpret_cast<float4 *>(at) = make_float4(u[0], u[1], u[2], u[3]);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (n + r < N) at[r] = u[r];
        }
    } else {
        _Float16 *at = static_cast<_Float16 *>(y) + m * N + n;
        typedef _Float16 h4 __attribute__((ext_vector_type(4), may_alias));
        const h4 h = {(_Float16)u[0], (_Float16)u[1], (_Float16)u[2], (_Float16)u[3]};
        if (N % 4 == 0) {
            if (n < N) *reinterpret_cast<h4 *>(at) = h;
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (n + r < N) at[r] = h[r];
        }
    }
}

// Few rows: 16 MB rows and 16 NB outputs a workgroup, whose wavefronts take every WAVES-th step and add up through LDS.  The weights are read once, by one
// wavefront, straight into the operands' registers: bound by memory, so what counts is how much is under way: AHEAD steps a wavefront.
// Lane group g reads chunks g and 4 + g (of 16 bytes) of a step's 8: the order along K is free, if both operands have it.
// EXPERTS: the rows of a tile of ExpertRows; GATED: NB blocks of the gate and the same NB of the up matrix, y = silu(g) * u.
template <int MB, int NB, int WAVES, int AHEAD, bool EXPERTS, bool GATED>
__global__ __launch_bounds__(64 * WAVES) void qgemm_f8_few(F8Gemm a)
{
    constexpr int COLS = NB * (GATED ? 2 : 1), TOTAL = MB * COLS;
    __shared__ v4f sums[WAVES][TOTAL][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p = lane & 15, g = lane >> 4;
    const int across = (a.N + 16 * NB - 1) / (16 * NB), tile = blockIdx.x / across;
    int m0 = tile * 16 * MB, m_end = a.M;
    const uint8_t *w = a.w;
    const float *s_w = a.s_w;
    if constexpr (EXPERTS) {
        if (tile >= a.tiles[0]) return;
        const int e = a.tiles[1 + 2 * tile];
        m0 = a.tiles[2 + 2 * tile];
        m_end = a.first[e + 1];
        const long long matrix = (long long)e * (GATED ? 2 : 1);
        w += matrix * a.N * a.K;
        s_w += matrix * a.NB * a.KB;
    }
    const int n0 = ((int)blockIdx.x - tile * across) * 16 * NB;
    const auto rows_x = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.q), 0, 0xffffffe0u, 0x00020000);
    const auto rows_w = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(w), 0, (unsigned)a.N * (unsigned)a.K * (GATED ? 2u : 1u), 0x00020000);
    unsigned at_x[MB], at_w[COLS];
    const float *s[MB];
    int sw_row[COLS];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        int m = min(m0 + 16 * i + p, m_end - 1);
        if (EXPERTS && a.order) m = a.order[m] / a.k;
        at_x[i] = (unsigned)m * (unsigned)a.K + 16 * g;
        s[i] = a.s + (long long)m * a.KB;
    }
#pragma unroll
    for (int j = 0; j < COLS; ++j) {
        const int n = n0 + 16 * (j % NB);
        at_w[j] = (unsigned)(min(n + p, a.N - 1) + (j < NB ? 0 : a.N)) * (unsigned)a.K + 16 * g;
        sw_row[j] = ((j < NB ? 0 : a.NB) + min(n, a.N - 1) / F8_BLOCK) * a.KB;
    }
    // chunks behind the end of a row are zero: their offset lies behind the operand
    const int last = a.K - (a.KB - 1) * F8_BLOCK;
    const bool dead_lo = 16 * g >= last, dead_hi = 16 * g + 64 >= last;
    auto load = [&](__amdgpu_buffer_rsrc_t rows, unsigned at, int kb) {
        const unsigned off = at + (unsigned)kb * F8_BLOCK;
        const bool end = kb == a.KB - 1;
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
        const u4 lo = __builtin_amdgcn_raw_buffer_load_b128(rows, end && dead_lo ? 0xfffffff0u : off, 0, 0);
        const u4 hi = __builtin_amdgcn_raw_buffer_load_b128(rows, end && dead_hi ? 0xfffffff0u : off + 64, 0, 0);
        return __builtin_bit_cast(v8i, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    v8i x[AHEAD][MB], f[AHEAD][COLS];
    float sa[AHEAD][MB], sw[AHEAD][COLS];
    auto request = [&](int u, int kb) {
#pragma unroll
        for (int j = 0; j < COLS; ++j) f[u][j] = load(rows_w, at_w[j], kb);
#pragma unroll
        for (int i = 0; i < MB; ++i) x[u][i] = load(rows_x, at_x[i], kb);
#pragma unroll
        for (int i = 0; i < MB; ++i) sa[u][i] = s[i][kb];
#pragma unroll
        for (int j = 0; j < COLS; ++j) sw[u][j] = s_w[sw_row[j] + kb];
    };
    v4f acc[TOTAL];
#pragma unroll
    for (int t = 0; t < TOTAL; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // steps behind the last one are the last one again, with a scale of 0: no branch stands between requests and their use, where the compiler would wait for
    // what is under way
    auto step_of = [&](int n) { return wave + n * WAVES; };
    auto consume = [&](int u, int kb) {
        Wide xw[MB];
#pragma unroll
        for (int i = 0; i < MB; ++i) xw[i] = Wide(x[u][i]);
#pragma unroll
        for (int j = 0; j < COLS; ++j) {
            const Wide fw(f[u][j]);
            const float sj = kb < a.KB ? sw[u][j] : 0.0f;
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const v4f d = step_product(fw, xw[i]);
                const float scale = sa[u][i] * sj;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j * MB + i][r] = __builtin_fmaf(d[r], scale, acc[j * MB + i][r]);
            }
        }
    };
    const int steps = (a.KB + WAVES - 1) / WAVES;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) request(u, min(step_of(u), a.KB - 1));
    int n = 0;
    for (; n + AHEAD < steps; n += AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            consume(u, step_of(n + u));
            request(u, min(step_of(n + u + AHEAD), a.KB - 1));
        }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (n + u < steps) consume(u, step_of(n + u));
#pragma unroll
    for (int t = 0; t < TOTAL; ++t) sums[wave][t][lane] = acc[t];
    __syncthreads();
    auto total = [&](int t) {
        v4f v = sums[0][t][lane];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) v += sums[k][t][lane];
        return v;
    };
    for (int t = wave; t < MB * NB; t += WAVES) {
        const int j = t / MB, i = t % MB, m = m0 + 16 * i + p, n = n0 + 16 * j + 4 * g;
        const v4f d = total(t);
        float u[4] = {d[0], d[1], d[2], d[3]};
        if (m >= m_end || n >= a.N) continue;
        if constexpr (GATED) {
            const v4f up = total(t + MB * NB);
#pragma unroll
            for (int r = 0; r < 4; ++r) u[r] = silu_dev(u[r]) * up[r];
            store4<true>(a.y, m, a.N, n, u);
        } else if constexpr (EXPERTS) {
            if (a.wide) store4<true>(a.y, m, a.N, n, u);
            else store4<false>(a.y, m, a.N, n, u);
        } else {
            finish4(a, m, n, u);
            store4<false>(a.y, m, a.N, n, u);
        }
    }
}

// Workgroups of 32 outputs from which on it is their number that keeps the memory busy
constexpr int64_t FEW_GROUPS = 1024;

int f8_expert_tile(int64_t P, int64_t E) { return P >= 64 * E ? F8_TILE_ROWS : 16; }

template <int MB, int NB, int WAVES, int AHEAD, bool EXPERTS, bool GATED>
static hipError_t run_few(const F8Gemm &a, hipStream_t s)
{
    const unsigned across = (unsigned)((a.N + 16 * NB - 1) / (16 * NB)), down = EXPERTS ? (unsigned)a.tiles_most : (unsigned)((a.M + 16 * MB - 1) / (16 * MB));
    hipLaunchKernelGGL((qgemm_f8_few<MB, NB, WAVES, AHEAD, EXPERTS, GATED>), dim3(across * down), dim3(64 * WAVES), 0, s, a);
    return hipGetLastError();
}

// A wavefront requests as many steps ahead as it has, up to MOST (steps that there are not would be requested for nothing)
template <int MB, int NB, int WAVES, int MOST, bool EXPERTS, bool GATED>
static hipError_t run_ahead(const F8Gemm &a, hipStream_t s)
{
    const int steps = (a.KB + WAVES - 1) / WAVES;
    if constexpr (MOST >= 4) {
        if (steps >= 4) return run_few<MB, NB, WAVES, 4, EXPERTS, GATED>(a, s);
    }
    if (steps >= 2) return run_few<MB, NB, WAVES, 2, EXPERTS, GATED>(a, s);
    return run_few<MB, NB, WAVES, 1, EXPERTS, GATED>(a, s);
}

hipError_t launch_qgemm_f8(const F8Gemm &a, hipStream_t s)
{
    if (a.first) {
        if (a.tile >= F8_TILE_ROWS) return launch_qgemm_f8_tiles(a, s);
        const bool many = (int64_t)a.tiles_most * (a.N / 32) >= FEW_GROUPS;
        if (a.gated) return many ? run_few<1, 2, 4, 1, true, true>(a, s) : run_ahead<1, 1, 8, 2, true, true>(a, s);
        return many ? run_few<1, 2, 4, 1, true, false>(a, s) : run_ahead<1, 1, 4, 2, true, false>(a, s);
    }
    if (a.M > 64) return launch_qgemm_f8_tiles(a, s);
    if (a.M <= 16) return a.N / 32 >= FEW_GROUPS ? run_few<1, 2, 4, 1, false, false>(a, s) : run_ahead<1, 1, 8, 4, false, false>(a, s);
    if (a.M <= 32) return run_ahead<2, 1, 8, 2, false, false>(a, s);
    return run_ahead<4, 1, 8, 2, false, false>(a, s);
}

}  // namespace ql
