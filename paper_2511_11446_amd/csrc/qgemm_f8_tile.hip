// e4m3 products with block scales on tiles of many rows (gfx950): layers and the experts' layers.  The operands come to LDS by DMA, a K step of 128 channels at a
// time; the scheme of operands, sums and scales is that of qgemm_f8.hip.
//
// Two stages in LDS: the next step comes while this one is multiplied.  Side of the tile: 256 x 256 reads the operands' bytes least often (8192^3 478 us with its inputs in a
// cache, 563 in turn with others: 2.3 and 2.0 PFLOP/s; the matrix cores 52 % busy, vector units, that is the folds, 42 %); 128 x 128, two on a CU, hides ends and writing
// under the other's products (16384 x 1152 x 4608 125 us, 134 to 141 with inputs from memory; 256 x 256 136: nine steps, and 151 MB written at their end); 64 x 64, four on a CU, is for layers with few tiles
// (1021 x 2224 x 1001 10.6 us, 14 to 15 with inputs from memory).  tiles_us below chooses.
// In binary16 products (WIDE) a wavefront issues two conversions and one fold for every product: matrix cores 47 %, vector units 62 % busy, 13 % waiting, 2.0 GHz.  Half as many
// products of 32 x 32, with the conversions between them, took as long.  16384 tokens through 8 of 64 experts of 2048 x 1024: gated 1113 us, 0.99 PFLOP/s, down 567 us, 0.97
// (a library's binary16 product 1.19); three inputs in turn, on another machine, 1131 and 604.
#include "qgemm_f8.h"

namespace ql {

// A wavefront holds MT x NT blocks of 16 x 16; WM x WN wavefronts.  WIDE: sums in binary16 products (f8.h)
template <int MT_, int NT_, int WM_, int WN_, int STAGES_, bool WIDE_>
struct TileF8 {
    static constexpr int MT = MT_, NT = NT_, WM = WM_, WN = WN_, STAGES = STAGES_;
    static constexpr bool WIDE = WIDE_;
    static constexpr int NW = WM * WN, NTHR = 64 * NW, BM = 16 * MT * WM, BN = 16 * NT * WN;
    static constexpr int NA = BM / 8 / NW, NB = BN / 8 / NW;             // DMA instructions of 8 rows for each wavefront and step
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, S_AT = A_BYTES + B_BYTES, STAGE = S_AT + BM * 4 + 256;
    static constexpr int ISSUED = NA + NB + 1;                           // and one for the rows' scales
    static constexpr int LDS_BYTES = STAGES * STAGE;
    static constexpr int BUFS = WIDE || NT < 4 ? 2 : 4, DIST = BUFS == 2 ? 1 : 2;            // weight fragments in registers, and how many groups ahead one is read
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && BM % 64 == 0 && NT % 2 == 0 && NT % BUFS == 0 && 16 * NT <= 128, "whole DMA instructions");
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
    // of GATED a tile is one block of 128 channels, in one pass over the steps or, 64 channels each, in two
    constexpr int PASSES = GATED ? F8_BLOCK / (T::BN / 2) : 1, COLS = GATED ? F8_BLOCK : T::BN;   // outputs of a tile
    static_assert(PASSES == 1 || PASSES == 2, "passes");
    extern __shared__ __align__(1024) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / T::WN, wn = wave % T::WN, p = lane & 15, g = lane >> 4;

    // ---- the tile: neighbours in the launch's order share an XCD's L2
    const int tiles = (EXPERTS ? within(a.tiles[0], tiles_m + 1) : tiles_m) * tiles_n, per_xcd = (tiles + XCDS - 1) / XCDS;
    const int in_xcd = blockIdx.x / XCDS, logical = (blockIdx.x % XCDS) * per_xcd + in_xcd;
    if (in_xcd >= per_xcd || logical >= tiles) return;
    int m0, n0, m_end = a.M;
    const uint8_t *w = a.w;
    const float *s_w = a.s_w;
    if constexpr (EXPERTS) {
        const int number = logical / tiles_n;
        const ExpertTile t(a.tiles, a.first, number, a.E, a.M);
        m0 = t.m0;
        n0 = (logical - number * tiles_n) * COLS;
        m_end = t.m_end;
        const long long matrix = (long long)t.e * (GATED ? 2 : 1);
        w += matrix * a.N * a.K;
        s_w += matrix * a.NB * a.KB;
    } else {
        const int group = group_m * tiles_n, first_m = logical / group * group_m, gm = min(tiles_m - first_m, group_m);
        m0 = (first_m + logical % group % gm) * T::BM;
        n0 = logical % group / gm * COLS;
    }

    // ---- DMA: lane l fills bytes [16 l, 16 l + 16) of 1024 = row l / 8, slot l % 8; chunk c of row r lies at slot c ^ ((r >> 1) & 7)
    unsigned offA[T::NA], offB[PASSES][T::NB], offS;
    bool dead[2];   // the chunk lies behind the end of a row in the last step (of rows with (row >> 1) & 4 clear, set)
    const unsigned bytesA = EXPERTS && a.order ? 0xffffffe0u : (unsigned)a.M * (unsigned)a.K;
    const unsigned bytesB = (unsigned)a.N * (unsigned)a.K * (GATED ? 2u : 1u);
    auto source_row = [&](int r) {
        int m = min(m0 + r, m_end - 1);
        if (EXPERTS && a.order) m = within(a.order[m], a.M) / a.k;
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
#pragma unroll
        for (int h = 0; h < PASSES; ++h) offB[h][i] = (unsigned)(min(n0 + 64 * h + c, a.N - 1) + half * a.N) * (unsigned)a.K + 16 * ((lane & 7) ^ ((r >> 1) & 7));
    }
    // rows of one DMA instruction begin at a multiple of 8: (r >> 1) & 3 is the lane's, bit 2 that of the instruction's number
#pragma unroll
    for (int h = 0; h < 2; ++h) dead[h] = 16 * ((lane & 7) ^ ((lane >> 4 & 3) + 4 * h)) >= last;
    // One operation a wavefront brings scales: the first BM / 64 wavefronts those of 64 rows, the others (all of them the same, so that every wavefront has as
    // many operations under way) those of the tile's two weight blocks: of neighbouring outputs, or of gate and up.
    constexpr int SW = T::BM / 64;
    const bool row_scales = wave < SW;
    const float *scales = row_scales ? a.s : s_w;
    if (row_scales) offS = (unsigned)source_row(64 * wave + lane) * (unsigned)a.KB * 4u;
    else offS = (unsigned)(GATED ? n0 / F8_BLOCK + (lane & 1) * a.NB : min(n0 / F8_BLOCK + (lane & 1), a.NB - 1)) * (unsigned)a.KB * 4u;
    const unsigned s_at = T::S_AT + (row_scales ? wave : SW) * 256;

    const int steps = PASSES * a.KB;
    auto issue = [&](int step, int stage) {
        unsigned char *st = smem + stage * T::STAGE;
        const bool second = PASSES == 2 && step >= a.KB;
        const int kt = second ? step - a.KB : step;
        const bool tail = kt == a.KB - 1 && last != F8_BLOCK;
        if (tail) {
#pragma unroll
            for (int i = 0; i < T::NA; ++i) {
                const int at = wave + i * T::NW;
                dma16_buf(a.q, bytesA, st + at * 1024, dead[at & 1] ? 0xfffffff0u : offA[i] + (unsigned)kt * 128u, 0);
            }
#pragma unroll
            for (int i = 0; i < T::NB; ++i) {
                const int at = wave + i * T::NW;
                const unsigned off = PASSES == 2 && second ? offB[PASSES - 1][i] : offB[0][i];
                dma16_buf(w, bytesB, st + T::A_BYTES + at * 1024, dead[at & 1] ? 0xfffffff0u : off + (unsigned)kt * 128u, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < T::NA; ++i) dma16_buf(a.q, bytesA, st + (wave + i * T::NW) * 1024, offA[i], kt * 128);
            if (second) {
#pragma unroll
                for (int i = 0; i < T::NB; ++i) dma16_buf(w, bytesB, st + T::A_BYTES + (wave + i * T::NW) * 1024, offB[PASSES - 1][i], kt * 128);
            } else {
#pragma unroll
                for (int i = 0; i < T::NB; ++i) dma16_buf(w, bytesB, st + T::A_BYTES + (wave + i * T::NW) * 1024, offB[0][i], kt * 128);
            }
        }
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(scales), 0, 0xffffffff, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(st + s_at), 4, offS, kt * 4, 0, 0);
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
    const int sw_at = T::S_AT + SW * 256 + (GATED ? 0 : (col0 - n0) / F8_BLOCK) * 4;

    // One step a pass, its weight fragments in groups of MT products.  A fragment is read DIST groups ahead.  Before the last group all of the step's
    // fragments are in registers: there the stages change hands (the next step has arrived, nobody reads this one any more), this stage is requested
    // again, and the next step's first fragments are read under the last products.  A group's sums are taken into the result one group later, when they are there.
    Wide x[T::WIDE ? MT : 1];
    v8i rx[MT], rf[T::BUFS];
    float rs[MT], rw, ru, scale[MT], scale_up[MT];
    static_assert(MT <= 4, "a fold behind each of a group's four rounds");
    v4f d[2][MT];
    auto read_scales = [&](const unsigned char *st) {
#pragma unroll
        for (int i = 0; i < MT; ++i) rs[i] = *reinterpret_cast<const float *>(st + T::S_AT + (wm * MT + i) * 64 + p * 4);
        rw = *reinterpret_cast<const float *>(st + sw_at);
        if (GATED) ru = *reinterpret_cast<const float *>(st + sw_at + 4);
    };
    auto read_x = [&](const unsigned char *st, int i) { rx[i] = read(st + (wm * MT + i) * 2048); };
    auto read_f = [&](const unsigned char *st, int j) { rf[j % T::BUFS] = read(st + T::A_BYTES + (wn * NT + j) * 2048); };
    auto fold = [&](int j, int i) {
        const float s = GATED && j >= NT / 2 ? scale_up[i] : scale[i];
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[j][i][r] = __builtin_fmaf(d[j & 1][i][r], s, acc[j][i][r]);
        asm volatile("" : "+v"(acc[j][i]));   // here: left to itself the compiler moves all of a step's behind its products, whose sums then have no room
    };
    float h[PASSES][GATED ? MT : 1][8];
    auto gated_product = [&](int pass, int i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[pass][GATED ? i : 0][e] = silu_dev(acc[e / 4][i][e % 4]) * acc[NT / 2 + e / 4][i][e % 4];
    };
#pragma unroll
    for (int s = 0; s < T::STAGES; ++s)
        if (s < steps) issue(s, s);
    if (steps >= T::STAGES) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(T::ISSUED * (T::STAGES - 1)) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < MT; ++i) read_x(smem, i);
#pragma unroll
    for (int j = 0; j < T::DIST; ++j) read_f(smem, j);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        d[1][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        scale[i] = scale_up[i] = 0.0f;
    }
    int stage = 0;
    for (int kt = 0; kt < steps; ++kt) {
        const unsigned char *st = smem + stage * T::STAGE;
        const int next = stage + 1 == T::STAGES ? 0 : stage + 1;
        const unsigned char *st_next = smem + next * T::STAGE;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if (j == NT - 1) {
                // (as many steps as there are stages are under way, fewer at the end; the oldest of them is the next)
                if (T::STAGES > 2 && kt + T::STAGES - 1 < steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(T::ISSUED * (T::STAGES - 2)) : "memory");
                else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                if (kt + T::STAGES < steps) issue(kt + T::STAGES, stage);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (T::WIDE) {
                if (j == 0) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) x[i] = Wide(rx[i]);
                }
            }
            const operand f(rf[j % T::BUFS]);
            if (j + T::DIST < NT) read_f(st, j + T::DIST);
            else if (j == NT - 1) {
#pragma unroll
                for (int k = 0; k < T::DIST; ++k) read_f(st_next, k);   // into the buffers of groups that are through
            }
            if (j == 0) read_scales(st);
            if constexpr (T::WIDE) {
                // a sum's four products in turn with those of the group's others, so that none waits for the one in front
#pragma unroll
                for (int q = 0; q < 4; ++q) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        if (q == 0) d[j & 1][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                        d[j & 1][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.h[q], x[i].h[q], d[j & 1][i], 0, 0, 0);
                    }
                    if (q < MT) fold(j == 0 ? NT - 1 : j - 1, q);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (j == NT - 1) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) read_x(st_next, i);
                }
            } else {
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    d[j & 1][i] = step_product(f, rx[i]);
                    fold(j == 0 ? NT - 1 : j - 1, i);
                    if (j == NT - 1) read_x(st_next, i);
                    __builtin_amdgcn_sched_barrier(0);   // in this order: a sum is four products old when it is folded
                }
            }
            if (j == 0) {
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    scale[i] = rs[i] * rw;
                    if (GATED) scale_up[i] = rs[i] * ru;
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        stage = next;
        if (PASSES == 2 && kt == a.KB - 1) {
            // the first 64 channels are there: the last group is taken in, and what it leaves for the next step has a scale of 0
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                fold(NT - 1, i);
                scale_up[i] = 0.0f;
                gated_product(0, i);
#pragma unroll
                for (int k = 0; k < NT; ++k) acc[k][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) fold(NT - 1, i);

    // ---- epilogue
    typedef _Float16 h8a __attribute__((ext_vector_type(8), may_alias));
    if constexpr (GATED) {
        // h = silu(g) * u of 8 channels (twice 8 in two passes) and MT rows a lane; the block's maximum over the lanes of a row and the WN wavefronts
        float *most = reinterpret_cast<float *>(smem);   // [BM][WN]
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();                    // the last step has been read everywhere
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            gated_product(PASSES - 1, i);
            float m = 0.0f;
#pragma unroll
            for (int k = 0; k < PASSES; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) m = fmaxf(m, col0 + 64 * k + 8 * g < a.N ? fabsf(h[k][i][e]) : 0.0f);
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
#pragma unroll
            for (int k = 0; k < PASSES; ++k) {
                const int c = col0 + 64 * k + 8 * g;
                if (c >= a.N) continue;
                uint2 out;
                out.x = f8_pack4(s.code(h[k][i][0]), s.code(h[k][i][1]), s.code(h[k][i][2]), s.code(h[k][i][3]));
                out.y = f8_pack4(s.code(h[k][i][4]), s.code(h[k][i][5]), s.code(h[k][i][6]), s.code(h[k][i][7]));
                *reinterpret_cast<uint2 *>(a.hq + (long long)m * a.N + c) = out;
            }
            if (wn == 0 && g == 0) a.hs[(long long)m * a.NB + n0 / F8_BLOCK] = F8Scale::scale(amax);
        }
    } else {
        constexpr bool LAYER = OUT == F8Out::LAYER;
        const _Float16 *bias = static_cast<const _Float16 *>(LAYER ? a.bias : nullptr), *res = static_cast<const _Float16 *>(LAYER ? a.residual : nullptr),
                       *gate = static_cast<const _Float16 *>(LAYER ? a.gate : nullptr);
        _Float16 *y = static_cast<_Float16 *>(a.y);
        // outputs that the caches will not hold until they are read are streamed (16384 x 1152 x 4608 with its quantizer, inputs from memory: 152 -> 140 us)
        const bool streamed = LAYER && (long long)a.M * a.N > (32ll << 20);
        // u -> fp16(act(u + bias)), of 8 neighbouring outputs
        auto value = [&](int i, int b, const float (&add)[8]) {
            h8 out;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float u = acc[2 * b + e / 4][i][e % 4] + add[e];
                if (LAYER && a.act == 1) u = gelu_tanh_dev(u);
                asm volatile("" : "+v"(u));   // the fp32 value is rounded to fp16 here and nowhere earlier
                out[e] = (_Float16)u;
            }
            return out;
        };
        auto bias8 = [&](int n, float (&add)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) add[e] = bias ? (float)bias[min(n + e, a.N - 1)] : -0.0f;   // x + -0.0 is x, signed zeros included
        };
        if (a.N % 8 == 0 && (uintptr_t)res % 16 == 0 && (uintptr_t)gate % 16 == 0) {
            float add[NT / 2][8];
#pragma unroll
            for (int b = 0; b < NT / 2; ++b) bias8(col0 + 32 * b + 8 * g, add[b]);
            if constexpr (OUT == F8Out::ROWS) {
                // A row's 64 outputs of this wavefront, where they reach 2^15: with the power of two that takes them below it, which the sum over the choices gives back.
                // (Weights follow there, so that an output beyond binary16 need be none of y; infinite ones stay so.)
                static_assert(16 * NT == F8_UP, "outputs that share a power");
                float most[MT];
                int up[MT];
                bool far = false;
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    most[i] = 0.0f;
                    up[i] = 0;
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) most[i] = fmaxf(most[i], fabsf(acc[j][i][e]));
                    far |= most[i] >= 0x1p15f;
                }
                if (__any(far)) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        most[i] = fmaxf(most[i], __shfl_xor(most[i], 16));
                        most[i] = fmaxf(most[i], __shfl_xor(most[i], 32));
                        up[i] = most[i] >= 0x1p15f && most[i] < __builtin_inff() ? __builtin_amdgcn_frexp_expf(most[i]) - 15 : 0;
                        const float down = __builtin_bit_cast(float, (127 - up[i]) << 23);
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[j][i][e] *= down;
                    }
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const int m = m0 + (wm * MT + i) * 16 + p;
                    if (g == 0 && m < m_end && col0 < a.N) a.up[(long long)m * ((a.N + F8_UP - 1) / F8_UP) + col0 / F8_UP] = (uint8_t)up[i];
                }
            }
            auto store_rows = [&](auto stream) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int m = m0 + (wm * MT + i) * 16 + p;
                h8 r[NT / 2], gt[NT / 2];
                if (res || gate) {
#pragma unroll
                    for (int b = 0; b < NT / 2; ++b) {
                        const int n = min(col0 + 32 * b + 8 * g, a.N - 8), from = min(m, m_end - 1);
                        if (res) r[b] = *reinterpret_cast<const h8a *>(res + (long long)from * a.N + n);
                        if (gate) gt[b] = *reinterpret_cast<const h8a *>(gate + (long long)(from / a.gate_rows) * a.N + n);
                    }
                }
#pragma unroll
                for (int b = 0; b < NT / 2; ++b) {   // (the halves of a line one behind the other)
                    const int n = col0 + 32 * b + 8 * g;
                    h8 out = value(i, b, add[b]);
                    if (res || gate) out = __builtin_bit_cast(h8, glue_piece(gate != nullptr, res != nullptr, __builtin_bit_cast(v4i, out), gt[b], r[b]));
                    if (m >= m_end || n >= a.N) continue;
                    h8a *to = reinterpret_cast<h8a *>(y + (long long)m * a.N + n);
                    if constexpr (decltype(stream)::value) __builtin_nontemporal_store(out, to);
                    else *to = out;
                }
            }
            };
            if constexpr (!LAYER) store_rows(std::false_type{});
            else if (streamed) store_rows(std::true_type{});   // (two copies: of one with both stores the compiler makes plain ones)
            else store_rows(std::false_type{});
        } else {
            // rows that do not begin at a multiple of 16 bytes: through LDS, so that 64 neighbouring outputs leave together (one by one from where they
            // are summed, 128 stores of 64 rows each a wavefront, the epilogue took longer than the sums)
            constexpr int PITCH = T::BN * 2 + 8;
            static_assert(T::BM * PITCH <= T::LDS_BYTES, "the tile in binary16");
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();                // the last step has been read everywhere
            asm volatile("" ::: "memory");
#pragma unroll
            for (int b = 0; b < NT / 2; ++b) {
                float add[8];
                bias8(col0 + 32 * b + 8 * g, add);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const uint4 out = __builtin_bit_cast(uint4, value(i, b, add));
                    uint2 *to = reinterpret_cast<uint2 *>(smem + ((wm * MT + i) * 16 + p) * PITCH + (wn * 16 * NT + 32 * b + 8 * g) * 2);
                    to[0] = make_uint2(out.x, out.y);
                    to[1] = make_uint2(out.z, out.w);
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            const int rows = min(T::BM, m_end - m0), columns = min(T::BN, a.N - n0);
            // four rows of a wavefront together, so that gate and residual are not one trip to memory after the other (7897 x 1664 x 3340 with a residual 140 -> 105 us)
            constexpr int ROWS = 4, PARTS = T::BN / 64;
            for (int first = wave; first < rows; first += ROWS * T::NW) {
                _Float16 r[ROWS][PARTS], gt[ROWS][PARTS];
                if (res || gate) {
#pragma unroll
                    for (int k = 0; k < ROWS; ++k) {
                        const int row = m0 + min(first + k * T::NW, rows - 1);
                        const long long at = (long long)row * a.N + n0, gate_at = gate ? (long long)(row / a.gate_rows) * a.N + n0 : 0;
#pragma unroll
                        for (int c = 0; c < PARTS; ++c) {
                            const int col = min(64 * c + lane, columns - 1);
                            if (res) r[k][c] = res[at + col];
                            if (gate) gt[k][c] = gate[gate_at + col];
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    const int row = first + k * T::NW;
                    if (row >= rows) break;
#pragma unroll
                    for (int c = 0; c < PARTS; ++c) {
                        if (64 * c + lane >= columns) continue;
                        _Float16 h = *reinterpret_cast<const half_alias *>(smem + row * PITCH + (64 * c + lane) * 2);
                        if (res || gate) {
                            float v = __builtin_fmaf(gate ? (float)gt[k][c] : 1.0f, (float)h, res ? (float)r[k][c] : 0.0f);
                            asm volatile("" : "+v"(v));
                            h = (_Float16)v;
                        }
                        y[(long long)(m0 + row) * a.N + n0 + 64 * c + lane] = h;
                    }
                }
            }
        }
    }
}

template <class T, F8Out OUT>
static hipError_t run_tile(const F8Gemm &a, hipStream_t s)
{
    const hipError_t opt_in = allow_lds<&qgemm_f8_tile<T, OUT>>();
    if (opt_in != hipSuccess) return opt_in;
    const int cols = OUT == F8Out::GATED ? F8_BLOCK : T::BN;
    const int tiles_m = OUT == F8Out::LAYER ? (a.M + T::BM - 1) / T::BM : a.tiles_most, tiles_n = (a.N + cols - 1) / cols;
    const unsigned grid = (unsigned)((tiles_m * tiles_n + XCDS - 1) / XCDS * XCDS);
    hipLaunchKernelGGL((qgemm_f8_tile<T, OUT>), dim3(grid), dim3(T::NTHR), T::LDS_BYTES, s, a, tiles_m, tiles_n, pick_group_m(T::BM));
    return hipGetLastError();
}

using Core256 = TileF8<4, 8, 4, 2, 2, false>;      // 256 x 256, one on a CU
using Core128 = TileF8<4, 4, 2, 2, 2, false>;      // 128 x 128, two
using Core64 = TileF8<2, 2, 2, 2, 2, false>;       // 64 x 64, four
using Wide128 = TileF8<4, 4, 2, 2, 2, true>;
using Wide64 = TileF8<2, 2, 2, 2, 2, true>;
using Rows64 = TileF8<2, 4, 2, 2, 2, true>;        // 64 x 128, three
static_assert(Rows64::BM == F8_TILE_ROWS && Wide128::BM == 2 * F8_TILE_ROWS, "what the rows of experts are cut into");

// What a layer takes on tiles of `side` of which `fit` are on a CU at a time: rounds of tiles, in each KB steps at step[l - 1] us where a CU has l of them, and `ends` us in
// front of the first step and behind the last.  The steps are those of 4096 x 4096 and 8192 x 8192 weights; us, measured and so, with the matrix cores' own
// sums: 1021 x 2224 x 1001 on 64 11.3 and 11.4, on 128 20.2 and 20.1, on 256 41 and 42; 2048 x 4096 x 4096 64, 42, 59 and 67, 42, 66; 16384 x 1152 x 4608 162, 124, 124 and 166, 127, 136.
static float tiles_us(const F8Gemm &a, int side, int fit, const float *step, float ends)
{
    const int64_t tiles = ((a.M + side - 1ll) / side) * ((a.N + side - 1ll) / side), slots = 256ll * fit;
    const int64_t left = tiles % slots;
    float us = 2.0f + (float)(tiles / slots) * (step[fit - 1] * a.KB + ends);
    if (left) us += step[(left + 255) / 256 - 1] * a.KB + ends;
    return us;
}
constexpr float CORE64[] = {0.52f, 0.64f, 0.82f, 1.01f}, CORE128[] = {0.81f, 1.14f}, CORE256[] = {1.85f}, WIDE64[] = {0.60f, 0.80f, 1.04f, 1.27f}, WIDE128[] = {1.17f, 1.85f};

// The tile of a layer and what it takes.  Sums in binary16 products (f8.h) up to F8_MANY rows and behind gated products
struct LayerTile {
    int side;
    float us;
};
static LayerTile layer_tile(const F8Gemm &a)
{
    const bool core = a.codes && a.M > F8_MANY;
    const float by64 = tiles_us(a, 64, 4, core ? CORE64 : WIDE64, 0.2f), by128 = tiles_us(a, 128, 2, core ? CORE128 : WIDE128, 3.5f),
                by256 = core ? tiles_us(a, 256, 1, CORE256, 10.0f) : 1e30f;
    if (by64 <= by128 && by64 <= by256) return {64, by64};
    return by128 <= by256 ? LayerTile{128, by128} : LayerTile{256, by256};
}

float qgemm_f8_tiles_us(const F8Gemm &a) { return layer_tile(a).us; }

hipError_t launch_qgemm_f8_tiles(const F8Gemm &a, hipStream_t s)
{
    if (a.first && a.tile == 64) return a.gated ? run_tile<Rows64, F8Out::GATED>(a, s) : run_tile<Rows64, F8Out::ROWS>(a, s);
    if (a.first) return a.gated ? run_tile<Wide128, F8Out::GATED>(a, s) : run_tile<Wide128, F8Out::ROWS>(a, s);
    const int side = layer_tile(a).side;
    if (!a.codes || a.M <= F8_MANY) return side == 64 ? run_tile<Wide64, F8Out::LAYER>(a, s) : run_tile<Wide128, F8Out::LAYER>(a, s);
    return side == 64 ? run_tile<Core64, F8Out::LAYER>(a, s) : side == 128 ? run_tile<Core128, F8Out::LAYER>(a, s) : run_tile<Core256, F8Out::LAYER>(a, s);
}

}  // namespace ql
