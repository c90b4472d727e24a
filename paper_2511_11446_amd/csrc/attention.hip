// Attention over binary16 rows for gfx950: one pass over the keys with the running maximum and sum of the softmax.
//
// A workgroup of NW wavefronts has 32 NW packed rows (attention.h) of one sequence and key head; keys and values go by tiles of 64 from global memory into
// LDS (global_load_lds, no registers), two tiles deep, and every wavefront reads them from there: attention_tile.h says how.
#include "attention_tile.h"

namespace ql {

struct AttnPlan {
    int tiles, per_seq, splits;   // row tiles of the launch (a bound with cu_q), per sequence without, parts of the keys
};

// Weights may grow by 2^8 before the sums are brought to a new maximum: they stay far inside binary16, and most tiles skip the scaling.
constexpr float GROWTH = 8.0f;

template <int KS, int NW>   // KS: 16-channel steps of the scores
__global__ __launch_bounds__(64 * NW, KS <= 8 ? 2 : 1) void attend_tiles(AttnArgs a, AttnPlan plan)
{
    constexpr int CHP = 2 * KS, DT = (KS + 1) / 2;
    constexpr int TILE = ATT_KEYS * CHP * 16;          // bytes of a tile of keys or values
    constexpr int NI = (CHP + NW - 1) / NW;            // DMA instructions of a wavefront for one tile
    extern __shared__ __align__(1024) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5;

    // workgroups of one key head follow each other on one XCD: they read the same keys and values
    const int total = gridDim.x, per_xcd = (total + 7) / 8;
    int id = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per_xcd || id >= plan.tiles * a.Hkv * plan.splits) return;
    const int split = id % plan.splits;
    id /= plan.splits;
    const int rows_per = 32 * NW;
    int tile, hk, b;
    if (a.cu_q) {
        tile = id % plan.tiles;
        hk = id / plan.tiles;
        b = find_sequence(a.B, tile, [&](int s) { return (seq_rows(a.cu_q, s, a.Tq, a.B).n * a.G + rows_per - 1) / rows_per; });
        if (b < 0) return;
    } else {
        tile = id % plan.per_seq;
        hk = id / plan.per_seq % a.Hkv;
        b = id / plan.per_seq / a.Hkv;
    }
    const SeqRows sq = seq_rows(a.cu_q, b, a.Tq, a.B), sk = seq_rows(a.cu_k, b, a.Tk, a.B);
    const int rows = sq.n * a.G;
    const int wrow = tile * rows_per + wave * 32 + (lane & 31);   // packed row of this lane
    const int row = min(wrow, rows - 1);
    const int token = row / a.G, head = hk * a.G + row % a.G;
    const int pos = token + sk.n - sq.n;
    const int prefix = a.prefix ? a.prefix[b] : 0;
    const int end = visible_end(a.mask, prefix, pos, sk.n);
    const int last_token = (min(tile * rows_per + rows_per, rows) - 1) / a.G;
    const int end_all = visible_end(a.mask, prefix, last_token + sk.n - sq.n, sk.n);   // what the workgroup reads
    int end_min = end, end_max = end;
#pragma unroll
    for (int m = 16; m; m >>= 1) {
        end_min = min(end_min, __shfl_xor(end_min, m, 64));
        end_max = max(end_max, __shfl_xor(end_max, m, 64));
    }
    end_min = __builtin_amdgcn_readfirstlane(end_min);
    end_max = __builtin_amdgcn_readfirstlane(end_max);

    const int key_tiles = (end_all + ATT_KEYS - 1) / ATT_KEYS;
    const int share = (key_tiles + plan.splits - 1) / plan.splits;
    const int t0 = min(split * share, key_tiles), t1 = min(t0 + share, key_tiles);

    // queries stay in registers: channels 16 ks + 8 half .. + 7 of the lane's row, zeros behind D
    const int CH = a.D / 8;
    const bool negative = a.scale < 0.0f;              // scores are |scale| * (-q).k
    f16x8 qf[KS];
    {
        const _Float16 *q = static_cast<const _Float16 *>(a.q) + (sq.first + token) * a.q_row + head * a.q_head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int c = 2 * ks + half;
            uint4 w = make_uint4(0, 0, 0, 0);
            if (c < CH) w = *reinterpret_cast<const uint4 *>(q + 8 * c);
            if (negative) {
                w.x ^= 0x80008000u;
                w.y ^= 0x80008000u;
                w.z ^= 0x80008000u;
                w.w ^= 0x80008000u;
            }
            qf[ks] = __builtin_bit_cast(f16x8, w);
        }
    }
    const bool shaped = a.cap > 0.0f || a.slopes || a.scale == 0.0f;
    const float scale2 = fabsf(a.scale) * LOG2E;       // scores in powers of two
    const float c2 = shaped ? 1.0f : scale2;
    const float slope2 = a.slopes ? a.slopes[head] * LOG2E : 0.0f;
    const float cap2 = a.cap * LOG2E, cap_in = a.cap > 0.0f ? 2.0f * scale2 / a.cap : 0.0f;

    // DMA: instruction i of this wavefront fills pieces [64 (i NW + wave), + 64) of the tile; a row behind the last key reads the last
    // one, a piece behind D the row's last one: what is read there meets weights or queries that are zero
    const unsigned char *kb = static_cast<const unsigned char *>(a.k) + 2 * (sk.first * a.k_row + hk * a.k_head);
    const unsigned char *vb = static_cast<const unsigned char *>(a.v) + 2 * (sk.first * a.v_row + hk * a.v_head);
    int drow[NI];
    unsigned kch[NI], vch[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int ci = 64 * (i * NW + wave) + lane, r = ci / CHP, c = ci % CHP;
        drow[i] = r;
        kch[i] = 16 * min(c ^ key_swizzle<CHP>(r), CH - 1);
        vch[i] = 16 * min(c ^ value_swizzle<CHP>(r), CH - 1);
    }
    const unsigned krow = 2 * (unsigned)a.k_row, vrow = 2 * (unsigned)a.v_row;
    auto issue = [&](int t, int stage) {
        const int left = sk.n - t * ATT_KEYS - 1;
        const unsigned char *kt = kb + (size_t)t * ATT_KEYS * 2 * a.k_row, *vt = vb + (size_t)t * ATT_KEYS * 2 * a.v_row;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            if (CHP % NW != 0 && i * NW + wave >= CHP) break;
            const unsigned r = min(drow[i], left);
            __builtin_amdgcn_global_load_lds((attn_global *)(kt + (r * krow + kch[i])), (attn_lds *)(smem + stage * 2 * TILE + (i * NW + wave) * 1024), 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            if (CHP % NW != 0 && i * NW + wave >= CHP) break;
            const unsigned r = min(drow[i], left);
            __builtin_amdgcn_global_load_lds((attn_global *)(vt + (r * vrow + vch[i])), (attn_lds *)(smem + stage * 2 * TILE + TILE + (i * NW + wave) * 1024), 16, 0, 0);
        }
    };

    f32x16 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f32x16{};
    float m = -__builtin_inff(), l = 0.0f;             // of this lane's row; l over this lane's keys only

    // addresses inside a tile
    const int krow_at = lane & 31;
    int vtok = 4 * half + (lane >> 2 & 3), vcol = 2 * (lane >> 4 & 1) + (lane >> 1 & 1), vbyte = 8 * (lane & 1);

    if (t0 < t1) issue(t0, 0);
    for (int t = t0; t < t1; ++t) {
        const int stage = (t - t0) & 1;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (t + 1 < t1) issue(t + 1, stage ^ 1);
        const int j0 = t * ATT_KEYS;
        if (j0 >= end_max) continue;                   // nothing there for this wavefront's rows
        const unsigned char *kt = smem + stage * 2 * TILE, *vt = kt + TILE;
        f32x16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            s[u] = f32x16{};
            const int r = 32 * u + krow_at;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const f16x8 kf = *reinterpret_cast<const f16x8 *>(kt + r * (CHP * 16) + 16 * ((2 * ks + half) ^ key_swizzle<CHP>(r)));
                s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[ks], s[u], 0, 0, 0);
            }
        }
        // register r of s[u] is key j0 + 32 u + 8 (r / 4) + 4 half + r % 4
        if (shaped) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float y = a.cap > 0.0f ? capped(s[u][r] * cap_in, cap2) : s[u][r] * scale2;
                    const int j = j0 + 32 * u + 8 * (r / 4) + 4 * half + r % 4;
                    y = __builtin_fmaf(-slope2, fabsf((float)(pos - j)), y);
                    s[u][r] = y;
                }
        }
        if (j0 + ATT_KEYS > end_min) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int j = j0 + 32 * u + 8 * (r / 4) + 4 * half + r % 4;
                    s[u][r] = j < end ? s[u][r] : -__builtin_inff();
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[u][r]);
        const Halves tops = both_halves(top);
        top = fmaxf(tops.a, tops.b);
        // m: what the weights are relative to, in the scores' own units
        if (__any((top - m) * c2 > GROWTH || (m == -__builtin_inff() && top > m))) {
            const float m2 = fmaxf(m, top);
            const float keep = m == -__builtin_inff() ? 0.0f : exp2_fast((m - m2) * c2);
            l *= keep;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[d][r] *= keep;
            m = m2;
        }
        const float mc = m == -__builtin_inff() ? 0.0f : -m * c2;
        f16x8 p[4];
        float sum = 0.0f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float w = exp2_fast(__builtin_fmaf(s[u][r], c2, mc));
                sum += w;
                p[2 * u + r / 8][r % 8] = (_Float16)w;
            }
        l += sum;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                s16x4 lo, hi;
                const int r0 = 16 * st + vtok, r1 = r0 + 8, c = 4 * d + vcol;
                lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((attn_lds_s4 *)(vt + r0 * (CHP * 16) + 16 * (c ^ value_swizzle<CHP>(r0)) + vbyte));
                hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((attn_lds_s4 *)(vt + r1 * (CHP * 16) + 16 * (c ^ value_swizzle<CHP>(r1)) + vbyte));
                typedef short s16x8 __attribute__((ext_vector_type(8)));
                const s16x8 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, vf), p[st], acc[d], 0, 0, 0);
            }
    }
    const Halves ls = both_halves(l);
    l = ls.a + ls.b;
    if (plan.splits > 1) {
        // [rows_per][D] sums, then maxima (in powers of two) and weights of this part
        float *part = a.partial + ((size_t)((b * 0 + (a.cu_q ? (id % plan.tiles) : (b * plan.per_seq + tile))) * a.Hkv + hk) * plan.splits + split) * (size_t)(rows_per * (a.D + 2));
        const int lr = wave * 32 + (lane & 31);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int ch = 32 * d + 8 * g + 4 * half;
                if (ch < a.D) *reinterpret_cast<float4 *>(part + (size_t)lr * a.D + ch) = make_float4(acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]);
            }
        if (half == 0) {
            part[(size_t)rows_per * a.D + lr] = m == -__builtin_inff() ? m : m * c2;
            part[(size_t)rows_per * (a.D + 1) + lr] = l;
        }
        return;
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    unsigned amax = 0;
    _Float16 *o = static_cast<_Float16 *>(a.o) + (sq.first + token) * a.o_row + head * a.o_head;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            // channels 8 g + 4 half of this lane and of lane ^ 32 together are 8 neighbours for each of the two
            unsigned w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f16x2 h = {(_Float16)(acc[d][4 * g + 2 * e] * inv), (_Float16)(acc[d][4 * g + 2 * e + 1] * inv)};
                w[e] = __builtin_bit_cast(unsigned, h);
            }
            const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
            const int ch = 32 * d + 8 * g + 8 * half;
            const uint4 out = make_uint4(x[0], y[0], x[1], y[1]);
            if (ch < a.D && wrow < rows) {
                *reinterpret_cast<uint4 *>(o + ch) = out;
                if (a.row_absmax) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned v = e == 0 ? out.x : e == 1 ? out.y : e == 2 ? out.z : out.w;
                        amax = max(amax, max(v & 0x7fffu, v >> 16 & 0x7fffu));
                    }
                }
            }
        }
    if (a.row_absmax && wrow < rows) atomicMax(a.row_absmax + sq.first + token, amax);
}

namespace {
template <int KS, int NW>
hipError_t launch_tiles(const AttnArgs &a, hipStream_t stream)
{
    constexpr int LDS = 4 * ATT_KEYS * 2 * KS * 16 + 1024;   // two stages of keys and values; a value read of channels behind D may pass the last row
    constexpr int ROWS = 32 * NW;
    AttnPlan p{};
    const int per = a.Tq / a.B;
    p.per_seq = (int)(((long long)per * a.G + ROWS - 1) / ROWS);
    p.tiles = a.cu_q ? (int)((long long)a.Tq * a.G / ROWS + a.B) : p.per_seq * a.B;
    p.splits = 1;
    const long long wgs = (long long)p.tiles * a.Hkv * p.splits;
    auto *kernel = attend_tiles<KS, NW>;
    static bool sized = false;
    if (LDS > 64 * 1024 && !sized) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e != hipSuccess) return e;
        sized = true;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)((wgs + 7) / 8 * 8)), dim3(64 * NW), LDS, stream, a, p);
    return hipGetLastError();
}

template <int NW>
hipError_t launch_by_head(const AttnArgs &a, hipStream_t stream)
{
    const int ks = (a.D + 15) / 16;
    if (ks <= 1) return launch_tiles<1, NW>(a, stream);
    if (ks <= 2) return launch_tiles<2, NW>(a, stream);
    if (ks <= 3) return launch_tiles<3, NW>(a, stream);
    if (ks <= 4) return launch_tiles<4, NW>(a, stream);
    if (ks <= 5) return launch_tiles<5, NW>(a, stream);
    if (ks <= 6) return launch_tiles<6, NW>(a, stream);
    if (ks <= 8) return launch_tiles<8, NW>(a, stream);
    if (ks <= 12) return launch_tiles<12, NW>(a, stream);
    return launch_tiles<16, NW>(a, stream);
}
}  // namespace

hipError_t launch_attention_f16(const AttnArgs &a, hipStream_t stream)
{
    return launch_by_head<4>(a, stream);
}

}  // namespace ql
