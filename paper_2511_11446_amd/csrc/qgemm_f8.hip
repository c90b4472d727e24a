// e4m3 x e4m3 -> fp32 products with a scale for every row and 128 channels of the activations and every 128 x 128 block of the weights (gfx950),
// of a layer and of the experts' layers.
//
// A K step is one block of 128 channels: the matrix cores give its 16 x 16 sums from zero (f8.h), one fma a sum takes them into the
// result with the product of the two scales.  The weights are the instruction's first operand: a lane's four sums are then four outputs of one row, and as
// 16 outputs lie in one weight block, all its sums of a step have one scale: s[row] * s_w.
#include "qgemm_f8.h"

namespace ql {

// chunk c of 16 bytes at a lane's row: lane group g has chunks g and 4 + g of a step (the order along K is free, if both operands have it)
__device__ __forceinline__ v8i load_step(const uint8_t *row, int at, int K)
{
    v4i lo = {0, 0, 0, 0}, hi = lo;
    if (at < K) lo = *reinterpret_cast<const v4i *>(row + at);
    if (at + 64 < K) hi = *reinterpret_cast<const v4i *>(row + at + 64);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

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

// 16 MB rows and 16 NB outputs a workgroup, whose wavefronts share the steps and add up through LDS.  The operands come straight from memory.
// EXPERTS: the rows of expert tiles[2 t + 1]; GATED: NB blocks of the gate and the same NB of the up matrix, y = silu(g) * u.
template <int MB, int NB, int WAVES, bool EXPERTS, bool GATED>
__global__ __launch_bounds__(64 * WAVES) void qgemm_f8_few(F8Gemm a)
{
    constexpr int TOTAL = MB * NB * (GATED ? 2 : 1);
    __shared__ v4f sums[WAVES][TOTAL][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, p = lane & 15, g = lane >> 4;
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
    const uint8_t *row[MB];
    const float *s[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        int m = min(m0 + 16 * i + p, m_end - 1);
        if (EXPERTS && a.order) m = a.order[m] / a.k;
        row[i] = a.q + (long long)m * a.K;
        s[i] = a.s + (long long)m * a.KB;
    }
    v4f acc[TOTAL];
#pragma unroll
    for (int t = 0; t < TOTAL; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int kb = wave; kb < a.KB; kb += WAVES) {
        const int at = kb * F8_BLOCK + 16 * g;
        Wide x[MB];
        float sa[MB];
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            x[i] = Wide(load_step(row[i], at, a.K));
            sa[i] = s[i][kb];
        }
#pragma unroll
        for (int j = 0; j < NB * (GATED ? 2 : 1); ++j) {
            const int nb = n0 + 16 * (j % NB);
            const uint8_t *wm = w + (j < NB ? 0ll : (long long)a.N * a.K);
            const float sw = s_w[(j < NB ? 0 : a.NB * a.KB) + (min(nb, a.N - 1) / F8_BLOCK) * a.KB + kb];
            const Wide f(load_step(wm + (long long)min(nb + p, a.N - 1) * a.K, at, a.K));
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const v4f d = step_product(f, x[i]);
                const float scale = sa[i] * sw;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j * MB + i][r] = __builtin_fmaf(d[r], scale, acc[j * MB + i][r]);
            }
        }
    }
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

int f8_expert_tile(int64_t P, int64_t E) { return P >= 64 * E ? F8_TILE_ROWS : 16; }

hipError_t launch_qgemm_f8(const F8Gemm &a, hipStream_t stream)
{
    if (a.first ? a.tile >= F8_TILE_ROWS : a.M > 256) return launch_qgemm_f8_tiles(a, stream);
    if (a.first) {
        const dim3 grid((unsigned)((a.N + 31) / 32) * (unsigned)a.tiles_most);
        if (a.gated) hipLaunchKernelGGL((qgemm_f8_few<1, 2, 4, true, true>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((qgemm_f8_few<1, 2, 4, true, false>), grid, dim3(256), 0, stream, a);
    } else {
        const dim3 grid((unsigned)((a.N + 31) / 32) * (unsigned)((a.M + 31) / 32));
        hipLaunchKernelGGL((qgemm_f8_few<2, 2, 4, false, false>), grid, dim3(256), 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace ql
