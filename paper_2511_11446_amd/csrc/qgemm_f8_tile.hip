// e4m3 products with block scales on tiles of many rows (gfx950): layers and the experts' layers.  The operands come to LDS by DMA, a K step of 128 channels at a
// time; the scheme of operands, sums and scales is that of qgemm_f8.hip.
#include "qgemm_f8.h"

namespace ql {

// A wavefront holds MT x NT blocks of 16 x 16; WM x WN wavefronts.  WIDE: sums in binary16 products (f8.h)
template <int MT_, int NT_, int WM_, int WN_, int STAGES_, bool WIDE_>
struct TileF8 {
    static constexpr int MT = MT_, NT = NT_, WM = WM_, WN = WN_, STAGES = STAGES_;
    static constexpr bool WIDE = WIDE_;
    static constexpr int NW = WM * WN, NTHR = 64 * NW, BM = 16 * MT * WM, BN = 16 * NT * WN;
    static constexpr int NA = BM / 8 / NW, NB = BN / 8 / NW;             // DMA instructions of 8 rows for each wavefront and step
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, S_AT = A_BYTES + B_BYTES, STAGE = S_AT + BM * 4;
    static constexpr int ISSUED = NA + NB + 1;                           // and one for the rows' scales
    static constexpr int LDS_BYTES = STAGES * STAGE;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && BM % 64 == 0 && NT % 2 == 0 && (16 * NT <= 128), "whole DMA instructions");
    static_assert(LDS_BYTES <= 160 * 1024 && ISSUED * (STAGES - 2) < 64, "LDS, outstanding operations");
};

enum class F8Out { LAYER, GATED, ROWS };   // a layer's y; an expert's gated product, quantized; an expert's output rows

// LDS row 16 b + i of a wavefront's weights is its column 32 (b / 2) + 8 (i / 4) + 4 (b % 2) + i % 4: lane group g then has 8 neighbouring
// outputs of two blocks.  Of GATED the first half of the blocks are the gate's columns, the second half the same ones of the up matrix.
template <class T, F8Out OUT>
__global__ __launch_bounds__(T::NTHR, 2) void qgemm_f8_tile(F8Gemm a, int tiles_m, int tiles_n, int group_m)
{
    constexpr int MT = T::MT, NT = T::NT;
    constexpr bool EXPERTS = OUT != F8Out::LAYER, GATED = OUT == F8Out::GATED;
    constexpr int COLS = GATED ? T::BN / 2 : T::BN;     // outputs of a tile
    extern __shared__ __align__(1024) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / T::WN, wn = wave % T::WN, p = lane & 15, g = lane >> 4;

    // ---- the tile: neighbours in the launch's order share an XCD's L2
    const int tiles = (EXPERTS ? a.tiles[0] : tiles_m) * tiles_n, per_xcd = (tiles + XCDS - 1) / XCDS;
    const int in_xcd = blockIdx.x / XCDS, logical = (blockIdx.x % XCDS) * per_xcd + in_xcd;
    if (in_xcd >= per_xcd || logical >= tiles) return;
    int m0, n0, m_end = a.M;
    const uint8_t *w = a.w;
    const float *s_w = a.s_w;
    if constexpr (EXPERTS) {
        const int t = logical / tiles_n, e = a.tiles[1 + 2 * t];
        m0 = a.tiles[2 + 2 * t];
        n0 = (logical - t * tiles_n) * COLS;
        m_end = a.first[e + 1];
        const long long matrix = (long long)e * (GATED ? 2 : 1);
        w += matrix * a.N * a.K;
        s_w += matrix * a.NB * a.KB;
    } else {
        const int group = group_m * tiles_n, first_m = logical / group * group_m, gm = min(tiles_m - first_m, group_m);
        m0 = (first_m + logical % group % gm) * T::BM;
        n0 = logical % group / gm * COLS;
    }

    // ---- DMA: lane l fills bytes [16 l, 16 l + 16) of 1024 = row l / 8, slot l % 8; chunk c of row r lies at slot c ^ ((r >> 1) & 7)
    unsigned offA[T::NA], offB[T::NB], offS;
    bool dead[2];   // the chunk lies behind the end of a row in the last step (of rows with (row >> 1) & 4 clear, set)
    const unsigned bytesA = EXPERTS && a.order ? 0xffffffe0u : (unsigned)a.M * (unsigned)a.K;
    const unsigned bytesB = (unsigned)a.N * (unsigned)a.K * (GATED ? 2u : 1u);
    auto source_row = [&](int r) {
        int m = min(m0 + r, m_end - 1);
        if (EXPERTS && a.order) m = a.order[m] / a.k;
        return m;
    };
    const int last = a.K - (a.KB - 1) * F8_BLOCK;
#pragma unroll
    for (int i = 0; i < T::NA; ++i) {
        const int r = 8 * (wave + i * T::NW) + (lane >> 3);
        offA[i] = (unsigned)source_row(r) * (unsigned)a.K + 16 * ((lane & 7) ^ ((r >> 1) & 7));
    }
#pragma unroll
    for (int i = 0; i < T::NB; ++i) {
        const int r = 8 * (wave + i * T::NW) + (lane >> 3), of = r / (16 * NT), b = r / 16 % NT, x = r % 16;
        const int half = GATED && b >= NT / 2, bb = GATED ? b % (NT / 2) : b;
        const int c = of * (GATED ? 8 * NT : 16 * NT) + 32 * (bb / 2) + 8 * (x / 4) + 4 * (bb % 2) + x % 4;
        offB[i] = (unsigned)(min(n0 + c, a.N - 1) + half * a.N) * (unsigned)a.K + 16 * ((lane & 7) ^ ((r >> 1) & 7));
    }
    // rows of one DMA instruction begin at a multiple of 8: (r >> 1) & 3 is the lane's, bit 2 that of the instruction's number
#pragma unroll
    for (int h = 0; h < 2; ++h) dead[h] = 16 * ((lane & 7) ^ ((lane >> 4 & 3) + 4 * h)) >= last;
    offS = (unsigned)source_row(64 * (wave % (T::BM / 64)) + lane) * (unsigned)a.KB * 4u;

    auto issue = [&](int kt, int stage) {
        unsigned char *st = smem + stage * T::STAGE;
        const bool tail = kt == a.KB - 1 && last != F8_BLOCK;
#pragma unroll
        for (int i = 0; i < T::NA; ++i) {
            const int at = wave + i * T::NW;
            if (tail) dma16_buf(a.q, bytesA, st + at * 1024, dead[at & 1] ? 0xfffffff0u : offA[i] + (unsigned)kt * 128u, 0);
            else dma16_buf(a.q, bytesA, st + at * 1024, offA[i], kt * 128);
        }
#pragma unroll
        for (int i = 0; i < T::NB; ++i) {
            const int at = wave + i * T::NW;
            if (tail) dma16_buf(w, bytesB, st + T::A_BYTES + at * 1024, dead[at & 1] ? 0xfffffff0u : offB[i] + (unsigned)kt * 128u, 0);
            else dma16_buf(w, bytesB, st + T::A_BYTES + at * 1024, offB[i], kt * 128);
        }
        // (several wavefronts bring the same scales, so that all have as many operations under way)
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(a.s), 0, 0xffffffff, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(st + T::S_AT + wave % (T::BM / 64) * 256), 4, offS, kt * 4, 0, 0);
    };

    // ---- fragments
    const int frag = p * 128, lo = (g ^ ((p >> 1) & 7)) * 16, hi = ((4 + g) ^ ((p >> 1) & 7)) * 16;
    auto read = [&](const unsigned char *rows) {
        const v4i x = *reinterpret_cast<const v4i *>(rows + frag + lo), y = *reinterpret_cast<const v4i *>(rows + frag + hi);
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    typedef typename std::conditional<T::WIDE, Wide, v8i>::type operand;
    v4f acc[NT][MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    // a wavefront's outputs lie in one weight block (of each matrix)
    const int col0 = n0 + wn * (GATED ? 8 * NT : 16 * NT);
    const float *sw_row = s_w + (long long)(min(col0, a.N - 1) / F8_BLOCK) * a.KB, *sw_up = sw_row + (long long)a.NB * a.KB;

#pragma unroll
    for (int s = 0; s < T::STAGES - 1; ++s)
        if (s < a.KB) issue(s, s);
    int stage = 0;
    for (int kt = 0; kt < a.KB; ++kt) {
        // the step has arrived, and everybody is done with the stage in front of it
        if (T::STAGES > 2 && kt + T::STAGES - 2 < a.KB) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(T::ISSUED * (T::STAGES - 2)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (kt + T::STAGES - 1 < a.KB) issue(kt + T::STAGES - 1, stage == 0 ? T::STAGES - 1 : stage - 1);
        const unsigned char *st = smem + stage * T::STAGE;
        const float sw = sw_row[kt], su = GATED ? sw_up[kt] : 0.0f;
        operand x[MT];
        float scale[MT], scale_up[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            x[i] = operand(read(st + (wm * MT + i) * 2048));
            const float s = *reinterpret_cast<const float *>(st + T::S_AT + (wm * MT + i) * 64 + p * 4);
            scale[i] = s * sw;
            scale_up[i] = s * su;
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const operand f(read(st + T::A_BYTES + (wn * NT + j) * 2048));
            v4f d[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) d[i] = step_product(f, x[i]);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const float s = GATED && j >= NT / 2 ? scale_up[i] : scale[i];
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j][i][r] = __builtin_fmaf(d[i][r], s, acc[j][i][r]);
            }
        }
        if (++stage == T::STAGES) stage = 0;
    }

    // ---- epilogue
    typedef _Float16 h8a __attribute__((ext_vector_type(8), may_alias));
    if constexpr (GATED) {
        // h = silu(g) * u of 8 channels and MT rows a lane; the block's maximum over the lanes of a row and the WN wavefronts
        static_assert(8 * NT * T::WN == F8_BLOCK, "a tile is one block of channels");
        float h[MT][8];
        float *most = reinterpret_cast<float *>(smem);   // [BM][WN]
        const int c = col0 + 8 * g;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();                    // the last step has been read everywhere
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            float m = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[i][e] = silu_dev(acc[e / 4][i][e % 4]) * acc[NT / 2 + e / 4][i][e % 4];
                m = fmaxf(m, fabsf(h[i][e]));
            }
            if (c >= a.N) m = 0.0f;
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            if (g == 0) most[((wm * MT + i) * 16 + p) * T::WN + wn] = m;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int r = (wm * MT + i) * 16 + p, m = m0 + r;
            float amax = most[r * T::WN];
#pragma unroll
            for (int k = 1; k < T::WN; ++k) amax = fmaxf(amax, most[r * T::WN + k]);
            if (m >= m_end) continue;
            const F8Scale s(amax);
            if (c < a.N) {
                uint2 out;
                out.x = f8_pack4(s.code(h[i][0]), s.code(h[i][1]), s.code(h[i][2]), s.code(h[i][3]));
                out.y = f8_pack4(s.code(h[i][4]), s.code(h[i][5]), s.code(h[i][6]), s.code(h[i][7]));
                *reinterpret_cast<uint2 *>(a.hq + (long long)m * a.N + c) = out;
            }
            if (wn == 0 && g == 0) a.hs[(long long)m * a.NB + n0 / F8_BLOCK] = F8Scale::scale(amax);
        }
    } else {
        const bool pieces = a.N % 8 == 0;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = m0 + (wm * MT + i) * 16 + p;
            if (m >= m_end) continue;
#pragma unroll
            for (int b = 0; b < NT / 2; ++b) {
                const int n = col0 + 32 * b + 8 * g;
                if (n >= a.N) continue;
                const long long at = (long long)m * a.N + n;
                float u[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = acc[2 * b + e / 4][i][e % 4];
                if constexpr (OUT == F8Out::LAYER) {
                    float v[4] = {u[0], u[1], u[2], u[3]}, x[4] = {u[4], u[5], u[6], u[7]};
                    finish4(a, m, n, v);
                    if (n + 4 < a.N) finish4(a, m, n + 4, x);
#pragma unroll
                    for (int e = 0; e < 4; ++e) u[e] = v[e], u[4 + e] = x[e];
                }
                h8 out;
#pragma unroll
                for (int e = 0; e < 8; ++e) out[e] = (_Float16)u[e];
                _Float16 *y = static_cast<_Float16 *>(a.y) + at;
                if (pieces) *reinterpret_cast<h8a *>(y) = out;
                else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (n + e < a.N) y[e] = out[e];
                }
            }
        }
    }
}

template <class T, F8Out OUT>
static hipError_t run_tile(const F8Gemm &a, hipStream_t s)
{
    const hipError_t opt_in = hipFuncSetAttribute(reinterpret_cast<const void *>(&qgemm_f8_tile<T, OUT>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES);
    if (opt_in != hipSuccess) return opt_in;
    const int cols = OUT == F8Out::GATED ? T::BN / 2 : T::BN;
    const int tiles_m = OUT == F8Out::LAYER ? (a.M + T::BM - 1) / T::BM : a.tiles_most, tiles_n = (a.N + cols - 1) / cols;
    const unsigned grid = (unsigned)((tiles_m * tiles_n + XCDS - 1) / XCDS * XCDS);
    hipLaunchKernelGGL((qgemm_f8_tile<T, OUT>), dim3(grid), dim3(T::NTHR), T::LDS_BYTES, s, a, tiles_m, tiles_n, pick_group_m(T::BM));
    return hipGetLastError();
}

using CoreTile = TileF8<4, 8, 4, 2, 2, false>;    // 256 x 256
using WideTile = TileF8<4, 4, 2, 4, 3, true>;     // 128 x 256
static_assert(WideTile::BM == F8_TILE_ROWS, "what the rows of experts are cut into");

hipError_t launch_qgemm_f8_tiles(const F8Gemm &a, hipStream_t s)
{
    if (a.first) return a.gated ? run_tile<WideTile, F8Out::GATED>(a, s) : run_tile<WideTile, F8Out::ROWS>(a, s);
    return a.codes ? run_tile<CoreTile, F8Out::LAYER>(a, s) : run_tile<WideTile, F8Out::LAYER>(a, s);
}

}  // namespace ql
