// e4m3 x e4m3 -> fp32 products with a scale for every row and 128 channels of the activations and every 128 x 128 block of the weights (gfx950),
// of a layer and of the experts' layers.
//
// A K step is one block of 128 channels: the matrix cores give its 16 x 16 sums from zero (f8.h), one fma a sum takes them into the
// result with the product of the two scales.  The weights are the instruction's first operand: a lane's four sums are then four outputs of one row, and as
// 16 outputs lie in one weight block, all its sums of a step have one scale: s[row] * s_w.
#include "daq_device.h"
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

// (row_of: the output's row of a tile's row, -1: none)
// The wavefronts' sums (those of wavefront k from sums + k * pitch on), added up in their order, and what becomes of them
template <int MB, int NB, int WAVES, bool EXPERTS, bool GATED, class RowFn>
__device__ __forceinline__ void finish_few(const F8Gemm &a, const v4f *sums, int pitch, int n0, RowFn row_of)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, p = lane & 15, g = lane >> 4;
    auto total = [&](int t) {
        v4f v = sums[t * 64 + lane];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) v += sums[k * pitch + t * 64 + lane];
        return v;
    };
    for (int t = wave; t < MB * NB; t += WAVES) {
        const int j = t / MB, i = t % MB, m = row_of(16 * i + p), n = n0 + 16 * j + 4 * g;
        const v4f d = total(t);
        float u[4] = {d[0], d[1], d[2], d[3]};
        if (m < 0 || n >= a.N) continue;
        if constexpr (GATED) {
            const v4f up = total(t + MB * NB);
#pragma unroll
            for (int r = 0; r < 4; ++r) u[r] = silu_dev(u[r]) * up[r];
            store4<true>(a.y, m, a.N, n, u);
        } else if constexpr (EXPERTS) {
            store4<true>(a.y, m, a.N, n, u);
        } else {
            finish4(a, m, n, u);
            store4<false>(a.y, m, a.N, n, u);
        }
    }
}

// Few rows: 16 MB rows and 16 NB outputs a workgroup, whose wavefronts take every WAVES-th step and add up through LDS.  Every byte of the weights is read by one
// wavefront alone: bound by memory.  A wavefront brings its own steps to its own STAGES places in LDS by DMA (no barrier): loads straight into the operands' order touch
// 16 lines of memory each and pass 16 bytes a clock through a CU, by DMA, 8 rows of 128 bytes at a time, it is 45 (64 x 8192 x 4096 27 -> 13 us, 16 x 14336 x 4096
// 20 -> 12, the rate of a copy; with inputs from memory the first takes 15 to 17).
// EXPERTS: the rows of a tile of ExpertRows, whose number is blockIdx.y (as one number workgroups would pass 2^32 threads); GATED: NB blocks of the gate and the same
// NB of the up matrix, y = silu(g) * u.
template <int MB, int NB, int WAVES, int STAGES, bool EXPERTS, bool GATED>
__global__ __launch_bounds__(64 * WAVES) void qgemm_f8_few(F8Gemm a)
{
    constexpr int COLS = NB * (GATED ? 2 : 1), TOTAL = MB * COLS, X_BYTES = MB * 2048, S_AT = X_BYTES + COLS * 2048, STEP = S_AT + 512;
    constexpr int ISSUED = 2 * MB + 2 * COLS + 2;
    static_assert(WAVES * STAGES * STEP >= WAVES * TOTAL * 1024 && ISSUED * (STAGES - 1) < 64 && MB <= 4, "the sums fit where the steps were");
    extern __shared__ __align__(1024) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p = lane & 15, g = lane >> 4;
    const int across = (a.N + 16 * NB - 1) / (16 * NB), tile = EXPERTS ? blockIdx.y : blockIdx.x / across;
    int m0 = tile * 16 * MB, m_end = a.M;
    const uint8_t *w = a.w;
    const float *s_w = a.s_w;
    if constexpr (EXPERTS) {
        if (tile >= a.tiles[0]) return;   // (the grid has tiles_most of them)
        const ExpertTile t(a.tiles, a.first, tile, a.E, a.M);
        m0 = t.m0;
        m_end = t.m_end;
        const long long matrix = (long long)t.e * (GATED ? 2 : 1);
        w += matrix * a.N * a.K;
        s_w += matrix * a.NB * a.KB;
    }
    const int n0 = ((int)blockIdx.x - (EXPERTS ? 0 : tile * across)) * 16 * NB;
    const unsigned bytes_w = (unsigned)a.N * (unsigned)a.K * (GATED ? 2u : 1u);
    auto source_row = [&](int r) {
        int m = min(m0 + r, m_end - 1);
        if (EXPERTS && a.order) m = within(a.order[m], a.M) / a.k;
        return m;
    };
    // lane l fills bytes [16 l, 16 l + 16) of 8 rows; chunk c of row r lies at slot c ^ ((r >> 1) & 7)
    unsigned at_x[2 * MB], at_w[2 * COLS];
#pragma unroll
    for (int i = 0; i < 2 * MB; ++i) {
        const int r = 8 * i + (lane >> 3);
        at_x[i] = (unsigned)source_row(r) * (unsigned)a.K + 16 * ((lane & 7) ^ ((r >> 1) & 7));
    }
#pragma unroll
    for (int i = 0; i < 2 * COLS; ++i) {
        const int r = 8 * i + (lane >> 3), j = r / 16;
        at_w[i] = (unsigned)(min(n0 + 16 * (j % NB) + r % 16, a.N - 1) + (j < NB ? 0 : a.N)) * (unsigned)a.K + 16 * ((lane & 7) ^ ((r >> 1) & 7));
    }
    const unsigned at_s = (unsigned)source_row(lane % (16 * MB)) * (unsigned)a.KB * 4u;
    const int sw_block = lane % COLS;
    const unsigned at_sw = (unsigned)((sw_block < NB ? 0 : a.NB) + min(n0 + 16 * (sw_block % NB), a.N - 1) / F8_BLOCK) * (unsigned)a.KB * 4u;
    const int last = a.K - (a.KB - 1) * F8_BLOCK;
    bool dead[2];   // a chunk behind the end of a row in the last step: rows with (row >> 1) & 4 clear, set
#pragma unroll
    for (int h = 0; h < 2; ++h) dead[h] = 16 * ((lane & 7) ^ ((lane >> 4 & 3) + 4 * h)) >= last;
    unsigned char *mine = smem + wave * STAGES * STEP;
    auto issue = [&](int n, int stage) {
        const int kb = min(wave + n * WAVES, a.KB - 1);
        unsigned char *st = mine + stage * STEP;
        const bool tail = kb == a.KB - 1 && last != F8_BLOCK;
        const unsigned step = (unsigned)kb * F8_BLOCK;
#pragma unroll
        for (int i = 0; i < 2 * COLS; ++i) dma16_buf(w, bytes_w, st + X_BYTES + i * 1024, tail && dead[i & 1] ? 0xfffffff0u : at_w[i] + step, 0);
#pragma unroll
        for (int i = 0; i < 2 * MB; ++i) dma16_buf(a.q, 0xffffffe0u, st + i * 1024, tail && dead[i & 1] ? 0xfffffff0u : at_x[i] + step, 0);
        dma4_buf(a.s, 0xffffffffu, st + S_AT, at_s + kb * 4);
        dma4_buf(s_w, 0xffffffffu, st + S_AT + 256, at_sw + kb * 4);
    };
    const int lo = p * 128 + (g ^ ((p >> 1) & 7)) * 16, hi = p * 128 + ((4 + g) ^ ((p >> 1) & 7)) * 16;
    auto read = [&](const unsigned char *rows) {
        const v4i x = *reinterpret_cast<const v4i *>(rows + lo), y = *reinterpret_cast<const v4i *>(rows + hi);
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    v4f acc[TOTAL];
#pragma unroll
    for (int t = 0; t < TOTAL; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = (a.KB + WAVES - 1) / WAVES;   // (those behind the last one are the last one again, with a scale of 0)
#pragma unroll
    for (int n = 0; n < STAGES; ++n)
        if (n < steps) issue(n, n);
    for (int n = 0, stage = 0; n < steps; ++n) {
        const int left = min(steps - n, STAGES) - 1;   // steps under way behind this one
        if (left == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        else if (left == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(STAGES > 1 ? ISSUED : 0) : "memory");
        else if (left == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(STAGES > 2 ? 2 * ISSUED : 0) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(STAGES > 3 ? 3 * ISSUED : 0) : "memory");
        const unsigned char *st = mine + stage * STEP;
        v8i x[MB], f[COLS];
        float sa[MB], sw[COLS];
#pragma unroll
        for (int j = 0; j < COLS; ++j) {
            f[j] = read(st + X_BYTES + j * 2048);
            sw[j] = *reinterpret_cast<const float *>(st + S_AT + 256 + 4 * j);
        }
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            x[i] = read(st + i * 2048);
            sa[i] = *reinterpret_cast<const float *>(st + S_AT + 64 * i + 4 * p);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the place is free again
        if (n + STAGES < steps) issue(n + STAGES, stage);
        const bool there = wave + n * WAVES < a.KB;
        Wide xw[MB];
#pragma unroll
        for (int i = 0; i < MB; ++i) xw[i] = Wide(x[i]);
#pragma unroll
        for (int j = 0; j < COLS; ++j) {
            const Wide fw(f[j]);
            const float sj = there ? sw[j] : 0.0f;
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const v4f d = step_product(fw, xw[i]);
                const float scale = sa[i] * sj;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j * MB + i][r] = __builtin_fmaf(d[r], scale, acc[j * MB + i][r]);
            }
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    // every wavefront writes where its own steps were, which it has read
    v4f *sums = reinterpret_cast<v4f *>(smem);
    constexpr int PITCH = STAGES * STEP / 16;   // v4f from one wavefront's place to the next one's
    asm volatile("" ::: "memory");
#pragma unroll
    for (int t = 0; t < TOTAL; ++t) sums[wave * PITCH + t * 64 + lane] = acc[t];
    __syncthreads();
    finish_few<MB, NB, WAVES, EXPERTS, GATED>(a, sums, PITCH, n0, [&](int r) { return m0 + r < m_end ? m0 + r : -1; });
}

// Up to 16 rows that every workgroup quantizes itself: one launch in the place of two (a small launch costs the GPU 2 to 3 us, the host 3.6).  All of a
// wavefront's steps of weights, up to STEPS, are requested at once; while they come, the workgroup quantizes its rows into LDS as daq_f8.hip does.  Bound by the latencies of one
// such chain: 1 x 4096 x 4096 7.0 us, with inputs from memory 5.1 to 7.2 in the trace (16.8 MB: 3.3 at the rate of a copy); with the rows requested behind the weights, which they then wait for, 7.2.
//   LAYER  a layer's rows, binary16 (GLU: silu(g) * u of rows [g | u])
//   UP     up to 16 rows of (token, choice) without a plan: every workgroup finds its expert's among the ids; x of the token, h at row (token, choice)
//   DOWN   the same rows of h, fp32
enum class Self { LAYER, LAYER_GLU, UP, DOWN };

// n / d of n up to 1023 and d up to 32, with by = divisor(d)
__device__ __forceinline__ int divisor(int d) { return 65536 / d + 1; }
__device__ __forceinline__ int divided(int n, int by) { return n * by >> 16; }

// Stores to LDS that do not wait for the DMA under way to other parts of it (the compiler lets its own wait).  Whoever reads them waits for lgkmcnt in front of the barrier.
__device__ __forceinline__ unsigned lds_at(void *to) { return (unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)to; }
__device__ __forceinline__ void store_lds(void *to, uint2 v)
{
    typedef unsigned v2u __attribute__((ext_vector_type(2)));
    asm volatile("ds_write_b64 %0, %1" ::"v"(lds_at(to)), "v"(v2u{v.x, v.y}) : "memory");
}
__device__ __forceinline__ void store_lds(void *to, float v) { asm volatile("ds_write_b32 %0, %1" ::"v"(lds_at(to)), "v"(v) : "memory"); }

template <int STEPS, Self SELF>
__global__ __launch_bounds__(512) void qgemm_f8_self(F8Gemm a, int most)   // most: rows of a tile
{
    constexpr int WAVES = 8, COLS = SELF == Self::UP ? 2 : 1, PLACE = COLS * 2048;
    constexpr bool EXPERTS = SELF == Self::UP || SELF == Self::DOWN, GATED = SELF == Self::UP;
    extern __shared__ __align__(1024) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p = lane & 15, g = lane >> 4;
    const int tile = blockIdx.y, n0 = (int)blockIdx.x * 16;
    const uint8_t *w = a.w;
    const float *s_w = a.s_w;
    int row, rows_here;   // the row of this lane's place p in the tile (-1: none); how many there are
    if constexpr (EXPERTS) {
        // A tile is an expert's rows, the experts in the order of their first rows
        const int pair = lane < a.M ? a.ids[lane] : -1, id = pair >= 0 && pair < a.E ? pair : -1;
        unsigned long long rows = 0;
        int e = 0;
        for (int r = 0, before = tile; r < a.M; ++r) {
            e = __builtin_amdgcn_readlane(id, r);
            rows = __ballot(id == e);
            if (e >= 0 && __builtin_ctzll(rows) == r && before-- == 0) break;
            rows = 0;
        }
        if (!rows) return;
        row = -1;
        rows_here = __popcll(rows);
        for (int i = 0; i < rows_here; ++i, rows &= rows - 1) row = p == i ? __builtin_ctzll(rows) : row;
        const long long matrix = (long long)e * COLS;
        w += matrix * a.N * a.K;
        s_w += matrix * a.NB * a.KB;
    } else {
        row = p < a.M ? p : -1;
        rows_here = a.M;
    }
    const unsigned bytes_w = (unsigned)a.N * (unsigned)a.K * COLS;
    unsigned at_w[2 * COLS];
#pragma unroll
    for (int i = 0; i < 2 * COLS; ++i) {
        const int r = 8 * (i & 1) + (lane >> 3);
        at_w[i] = (unsigned)(min(n0 + r, a.N - 1) + i / 2 * a.N) * (unsigned)a.K + 16 * ((lane & 7) ^ ((r >> 1) & 7));
    }
    // ---- the first of the rows' values are requested in front of the weights: they come first, and are quantized while the weights come
    typedef _Float16 h8 __attribute__((ext_vector_type(8)));
    const int blocks = rows_here * a.KB, by_kb = divisor(a.KB), source = SELF == Self::UP ? divided(row, divisor(a.k)) : row;
    float4 one, two;   // 8 values: of binary16 one, and two the other half of [g | u]
    auto request = [&](int b) {   // (the rows' numbers are in a wavefront's first 16 lanes, whose b is its least: they are there as long as any lane is)
        const int r = divided(b, by_kb), k = (b - r * a.KB) * F8_BLOCK + (threadIdx.x & 15) * 8, from_row = __shfl(source, r);
        one = two = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (b < blocks && k < a.K) {
            if constexpr (SELF == Self::DOWN) {
                const float4 *from = reinterpret_cast<const float4 *>(static_cast<const float *>(a.x) + (long long)from_row * a.K + k);
                one = from[0];
                two = from[1];
            } else {
                const _Float16 *from = static_cast<const _Float16 *>(a.x) + (long long)from_row * a.K * (SELF == Self::LAYER_GLU ? 2 : 1) + k;
                one = *reinterpret_cast<const float4 *>(from);
                if constexpr (SELF == Self::LAYER_GLU) two = *reinterpret_cast<const float4 *>(from + a.K);
            }
        }
    };
    request((int)(threadIdx.x >> 4));
    float sw[STEPS][COLS];
#pragma unroll
    for (int n = 0; n < STEPS; ++n)
#pragma unroll
        for (int j = 0; j < COLS; ++j) sw[n][j] = s_w[((j ? a.NB : 0) + min(n0, a.N - 1) / F8_BLOCK) * a.KB + min(wave + n * WAVES, a.KB - 1)];
    const int last = a.K - (a.KB - 1) * F8_BLOCK;
    unsigned char *mine = smem + wave * STEPS * PLACE;
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
        const int kb = wave + n * WAVES, left = kb < a.KB - 1 ? F8_BLOCK : kb == a.KB - 1 ? last : 0;   // channels of this step; what there is not is read as nothing
#pragma unroll
        for (int i = 0; i < 2 * COLS; ++i) {
            const bool dead = 16 * ((lane & 7) ^ ((lane >> 4 & 3) + 4 * (i & 1))) >= left;
            dma16_buf(w, bytes_w, mine + n * PLACE + i * 1024, dead ? 0xfffffff0u : at_w[i] + (unsigned)kb * F8_BLOCK, 0);
        }
    }
    // ---- the rows: block kb of row r at kb * most + r, 128 codes whose 16-byte chunk c lies at c ^ ((r >> 1) & 7), and a scale.  (What a lane without a row reads is
    // another row's, or nothing's: its results go nowhere.)
    unsigned char *codes = smem + WAVES * STEPS * PLACE;
    float *scales = reinterpret_cast<float *>(codes + (size_t)a.KB * most * F8_BLOCK + 2048);
    for (int b = threadIdx.x >> 4; b < blocks; b += 32) {
        const int r = divided(b, by_kb), kb = b - r * a.KB, sub = threadIdx.x & 15;
        float v[8] = {one.x, one.y, one.z, one.w, two.x, two.y, two.z, two.w};
        if constexpr (SELF != Self::DOWN) {
            const h8 f = __builtin_bit_cast(h8, one), u = __builtin_bit_cast(h8, two);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = SELF == Self::LAYER_GLU ? silu_dev((float)f[i]) * (float)u[i] : (float)f[i];
        }
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[i]));
        amax = max16(amax);
        const F8Scale s(amax);
        uint2 out;
        out.x = f8_pack4(s.code(v[0]), s.code(v[1]), s.code(v[2]), s.code(v[3]));
        out.y = f8_pack4(s.code(v[4]), s.code(v[5]), s.code(v[6]), s.code(v[7]));
        store_lds(codes + ((size_t)kb * most + r) * F8_BLOCK + ((sub / 2) ^ ((r >> 1) & 7)) * 16 + (sub & 1) * 8, out);
        if (sub == 0) store_lds(scales + kb * most + r, F8Scale::scale(amax));
        if (b + 32 < blocks) request(b + 32);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    // ---- the products
    const int lo = p * 128 + (g ^ ((p >> 1) & 7)) * 16, hi = p * 128 + ((4 + g) ^ ((p >> 1) & 7)) * 16;
    auto read = [&](const unsigned char *from) {
        const v4i f = *reinterpret_cast<const v4i *>(from + lo), f2 = *reinterpret_cast<const v4i *>(from + hi);
        return Wide(__builtin_shufflevector(f, f2, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    v4f acc[COLS];
#pragma unroll
    for (int j = 0; j < COLS; ++j) acc[j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
        const int kb = wave + n * WAVES;
        if (kb >= a.KB) break;
        const Wide xw = read(codes + (size_t)kb * most * F8_BLOCK);
        const float sx = scales[kb * most + p];
#pragma unroll
        for (int j = 0; j < COLS; ++j) {
            const v4f d = step_product(read(mine + n * PLACE + j * 2048), xw);
            const float scale = sx * sw[n][j];
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[j][r] = __builtin_fmaf(d[r], scale, acc[j][r]);
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    v4f *sums = reinterpret_cast<v4f *>(smem);
    constexpr int PITCH = STEPS * PLACE / 16;
    static_assert(PITCH >= COLS * 64, "the sums fit where the steps were");
#pragma unroll
    for (int j = 0; j < COLS; ++j) sums[wave * PITCH + j * 64 + lane] = acc[j];
    __syncthreads();
    finish_few<1, 1, WAVES, EXPERTS, GATED>(a, sums, PITCH, n0, [&](int) { return row; });   // (a lane's place in the tile is p here as there)
}

// Rows that are quantized by every workgroup that reads them: up to four steps of eight wavefronts, and workgroups
constexpr int64_t SELF_K = 4096, SELF_N = 8192, SELF_VALUES = 32768;

// Tiles of 16 rows read an expert's weights once for every 16, tiles of 64 and 128 (qgemm_f8_tile.hip) quantize the gated product themselves and have fewer workgroups with
// longer chains.  us on 16, 64 and 128 rows, T tokens: k = 8 of 64 experts, 2048 and 1024 inputs: T = 64 85, 87, 119; 256 151, 114, 165; 2048 703, 316, 322; 8192 -, 1026, 958;
// 4 of 60, 1152 and 720: T = 128 47, 51, 67, 300 65, 53, 71; 2 of 8, 4096 and 2048: T = 128 64, 89, 114, 512 165, 126, 130, 4096 -, 548, 503
int f8_expert_tile(int64_t P, int64_t E) { return P < f8_expert_few(E) ? 16 : P >= 384 * E ? 128 : 64; }

template <int MB, int NB, int WAVES, int STAGES, bool EXPERTS, bool GATED>
static hipError_t run_few(const F8Gemm &a, hipStream_t s)
{
    constexpr int bytes = WAVES * STAGES * ((MB + NB * (GATED ? 2 : 1)) * 2048 + 512);
    static_assert(bytes <= 160 * 1024, "LDS");
    const hipError_t opt_in = allow_lds<&qgemm_f8_few<MB, NB, WAVES, STAGES, EXPERTS, GATED>>();
    if (opt_in != hipSuccess) return opt_in;
    const unsigned across = (unsigned)((a.N + 16 * NB - 1) / (16 * NB)), down = EXPERTS ? (unsigned)a.tiles_most : (unsigned)((a.M + 16 * MB - 1) / (16 * MB));
    hipLaunchKernelGGL((qgemm_f8_few<MB, NB, WAVES, STAGES, EXPERTS, GATED>), EXPERTS ? dim3(across, down) : dim3(across * down), dim3(64 * WAVES), bytes, s, a);
    return hipGetLastError();
}

template <int STEPS, Self SELF>
static hipError_t run_self_steps(const F8Gemm &a, hipStream_t s)
{
    constexpr bool EXPERTS = SELF == Self::UP || SELF == Self::DOWN;
    const int most = a.M < 16 ? a.M : 16, bytes = (int)f8_self_bytes(most, a.KB, SELF == Self::UP);
    const hipError_t opt_in = allow_lds<&qgemm_f8_self<STEPS, SELF>>();
    if (opt_in != hipSuccess) return opt_in;
    if (bytes > F8_LDS || STEPS != f8_self_steps(a.KB)) return hipErrorInvalidValue;
    const unsigned tiles = EXPERTS ? (unsigned)a.M : 1u;   // a tile has a row at least
    hipLaunchKernelGGL((qgemm_f8_self<STEPS, SELF>), dim3((unsigned)((a.N + 15) / 16), tiles), dim3(512), bytes, s, a, most);
    return hipGetLastError();
}

template <Self SELF>
static hipError_t run_self(const F8Gemm &a, hipStream_t s)
{
    const int steps = f8_self_steps(a.KB);
    return steps == 1 ? run_self_steps<1, SELF>(a, s) : steps == 2 ? run_self_steps<2, SELF>(a, s) : run_self_steps<4, SELF>(a, s);
}

// What few rows take on workgroups of 16 mb rows and 16 nb outputs: what such a workgroup brings to LDS at 55 bytes a nanosecond, and 2.5 us for the launch, the first bytes'
// way and the sum over the wavefronts.  us with inputs in the caches, measured and so: 64 x 8192 x 4096 on 32 x 32 12.5 and 12.0, on 64 x 32 17.7 and 16.8; 128 x 4096 x 4096 on 64 x 32 11.3 and
// 9.6, on 32 x 32 13.4 and 12.0, on 32 x 16 20.9 and 16.8; 128 x 12288 x 512 on 32 x 16 11.5 and 13.2, on 64 x 32 22.6 and 23.9.
static float few_us(const F8Gemm &a, int mb, int nb)
{
    const int64_t groups = ((a.M + 16ll * mb - 1) / (16 * mb)) * ((a.N + 16ll * nb - 1) / (16 * nb));
    return (float)((groups + 255) / 256) * ((float)((mb + nb) * 16) * (float)(a.KB * F8_BLOCK) / 55e3f + 2.5f);
}

bool qgemm_f8_takes_rows(int64_t M, int64_t K, int64_t N, bool glu)
{
    return M <= 16 && K <= SELF_K && N <= SELF_N && M * K <= (glu ? SELF_VALUES / 2 : SELF_VALUES);
}

hipError_t launch_qgemm_f8(const F8Gemm &a, hipStream_t s)
{
    if (a.ids) return a.gated ? run_self<Self::UP>(a, s) : run_self<Self::DOWN>(a, s);
    if (a.x) return a.glu ? run_self<Self::LAYER_GLU>(a, s) : run_self<Self::LAYER>(a, s);
    if (a.first) {
        if (a.tile >= F8_TILE_ROWS) return launch_qgemm_f8_tiles(a, s);
        return a.gated ? run_few<1, 1, 4, 2, true, true>(a, s) : run_few<1, 2, 4, 2, true, false>(a, s);
    }
    const float tiles = qgemm_f8_tiles_us(a), by16 = few_us(a, 1, 1), by32 = few_us(a, 2, 1), by32w = few_us(a, 2, 2), by64w = few_us(a, 4, 2);
    const float least = fminf(fminf(fminf(by32, by32w), by64w), a.M <= 16 ? by16 : 1e30f);
    if (tiles < least) return launch_qgemm_f8_tiles(a, s);
    if (a.M <= 16 && by16 <= least) return run_few<1, 1, 8, 2, false, false>(a, s);
    if (by32 <= least) return run_few<2, 1, 8, 3, false, false>(a, s);
    return by32w <= least ? run_few<2, 2, 8, 2, false, false>(a, s) : run_few<4, 2, 4, 3, false, false>(a, s);
}

}  // namespace ql
