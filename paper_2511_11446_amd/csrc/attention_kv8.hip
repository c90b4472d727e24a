// Attention of few rows over the paged 8-bit cache for gfx950: single tokens, and short runs of them.
//
// The work is the cache's bytes: a unit is one group of 64 tokens of one key head for up to 16 packed rows (attention.h).  The launch is a fixed number
// of workgroups that share all units of all sequences evenly, whatever the lengths: every workgroup has the next U / W units (some one more) of the list that goes
// sequence by sequence, key head by key head.  Where an item (the units of one set of rows) is cut between workgroups, each leaves sums, maximum and
// weight in the workspace and join_parts puts them together.
//
// Codes go from global memory straight into the registers where the matrix instruction (16x16x32) wants them: a lane has 16 neighbouring bytes of a
// key for two steps of the scores, and 16 neighbouring bytes of the value codes of one channel - four tokens of each of the group's four tiles - which
// are the left operand of O^T = V^T P^T in the order in which S^T = K Q^T leaves the weights.  So nothing goes through LDS but the join of
// the workgroup's four wavefronts, which take the units in turn.
//
// Codes become binary16 exactly; key scales multiply the scores.  Value scales multiply the weights, relative to the largest one that the row has met so far (which its
// sums are relative to in turn): a weight times a bare scale could fall below binary16's range.
//
// 64 sequences of 1 to 8192 tokens, 32 heads of 128 on 8: 78 us and 6 of join_parts for 355 MB, 4.5 TB/s; two of 131071 tokens, 102 + 8 us for 537 MB, 5.2 TB/s, what
// a copy of that size reaches on this card (5.1 read and written): bound by memory.  Heads of 256, 16 on 2, 64 sequences of 4096 tokens: 65 us a call, 4.1 TB/s.  One token on 4096, 11 + 5 us: a chain of latencies (queries, page,
// keys, scores, values, the wavefronts' join, the second launch).
#include "attention_tile.h"

namespace ql {

struct CachedPlan {
    int workers;          // workgroups of the launch
};

constexpr int UNITS_PER_WORKER = 4;   // at least, where there are as many: one for every wavefront
// What beginning an item costs a workgroup (its sequence, pages, queries, the join of its wavefronts), in units: so many go in front of the item's own in
// the list that is shared out.  Without, workgroups with many short sequences end last: 64 sequences of 1 to 8192 tokens took 129 us, with it 79.
constexpr unsigned ITEM_UNITS = 5;

// what one sequence has of units and items
struct SeqUnits {
    int n_q, first, n_k, row_tiles, groups;
    __device__ __forceinline__ SeqUnits of_lane(int l) const
    {
        auto from = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
        return {from(n_q), from(first), from(n_k), from(row_tiles), from(groups)};
    }
};
__device__ __forceinline__ SeqUnits seq_units(const AttnArgs &a, int b)
{
    const SeqRows q = seq_rows(a.cu_q, b, a.Tq, a.B);
    SeqUnits s;
    s.n_q = q.n;
    s.first = q.first;
    s.n_k = min(max(a.len_k[b], 0), a.max_pages * a.page);
    s.row_tiles = (int)(((long long)q.n * a.G + 15) / 16);
    s.groups = max((s.n_k + KV_GROUP - 1) / KV_GROUP, 1);   // rows without keys are written too
    return s;
}
// Units and items are counted in 32 bits (the host refuses what could pass them): 64-bit divisions cost more than a unit.
__device__ __forceinline__ unsigned lanes_upto(unsigned v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const unsigned o = (unsigned)__shfl_up((int)v, d, 64);
        if (lane >= d) v += o;
    }
    return v;
}
__device__ __forceinline__ unsigned last_lane(unsigned v) { return (unsigned)__builtin_amdgcn_readlane((int)v, 63); }
__device__ __forceinline__ unsigned units_of(const AttnArgs &a, const SeqUnits &s)
{
    return (unsigned)s.row_tiles * ((unsigned)s.groups + ITEM_UNITS) * (unsigned)a.Hkv;
}
// Of `units` units every one of `workers` workgroups has `each`, the first `more` of them one more
struct Shares {
    unsigned workers, each, more;
    __device__ __forceinline__ unsigned first(unsigned w) const { return w * each + min(w, more); }
    __device__ __forceinline__ unsigned owner(unsigned u) const { return min(u < more * (each + 1) ? u / (each + 1) : more + (u - more * (each + 1)) / each, workers - 1); }
};
__device__ __forceinline__ Shares shares_of(unsigned units, unsigned most)
{
    Shares s;
    s.workers = min((units + UNITS_PER_WORKER - 1) / UNITS_PER_WORKER, most);
    s.each = s.workers ? units / s.workers : 0;
    s.more = units - s.each * s.workers;
    return s;
}

__device__ __forceinline__ float lanes16_max(float x)   // over the four lanes that have the same row
{
    unsigned w = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const unsigned a = r[0], b = r[1];
    x = fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
    w = __builtin_bit_cast(unsigned, x);
    const auto s = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    const unsigned c = s[0], d = s[1];
    return fmaxf(__builtin_bit_cast(float, c), __builtin_bit_cast(float, d));
}
__device__ __forceinline__ float lanes16_sum(float x)
{
    unsigned w = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const unsigned a = r[0], b = r[1];
    x = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
    w = __builtin_bit_cast(unsigned, x);
    const auto s = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    const unsigned c = s[0], d = s[1];
    return __builtin_bit_cast(float, c) + __builtin_bit_cast(float, d);
}

// The largest weight: what is below 2^-14 of binary16 is rounded in steps of 2^-24, so far weights are off by at most 2^-40 of the largest one
constexpr float CACHED_HEAD = 32768.0f;

// wavefronts per SIMD: as many as a unit's bytes leave registers for
constexpr int cached_waves(int NK) { return NK <= 1 ? 4 : NK <= 2 ? 3 : NK <= 4 ? 2 : 1; }

// NK: 32-channel steps of the scores; WIDE: D is a multiple of 64, keys in 16-byte pieces (else 8)
template <int NK, bool WIDE>
__global__ __launch_bounds__(256, cached_waves(NK)) void attend_cached(AttnArgs a, CachedPlan plan)
{
    constexpr int DT = 2 * NK, KP = (NK + 1) / 2;
    extern __shared__ __align__(16) float join[];     // [4][16][D] sums, [4][16] maxima, [4][16] weights, [4][128] scales
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int quarter = lane >> 4, r16 = lane & 15;
    const int D = a.D;
    float *join_m = join + 64 * D, *join_l = join_m + 64;
    float *scales = join_l + 64 + 128 * wave;         // of the keys and the values of a unit

    // units of the first 64 sequences (as a rule all), one per lane, and their sums from the front
    SeqUnits seq0{};
    if (lane < a.B) seq0 = seq_units(a, lane);
    const unsigned mine0 = units_of(a, seq0), upto0 = lanes_upto(mine0);
    unsigned units = last_lane(upto0);
    for (int base = 64; base < a.B; base += 64) units += last_lane(lanes_upto(base + lane < a.B ? units_of(a, seq_units(a, base + lane)) : 0));
    const Shares shares = shares_of(units, plan.workers);
    if (blockIdx.x >= shares.workers) return;
    unsigned u = shares.first(blockIdx.x);
    const unsigned u_end = shares.first(blockIdx.x + 1);
    const bool shaped = a.cap > 0.0f || a.slopes;
    const float cap2 = a.cap * LOG2E, scale2 = a.scale * LOG2E;
    const float cap_in = a.cap > 0.0f ? 2.0f * LOG2E / cap2 : 0.0f;
    const unsigned page_groups = (unsigned)a.page / KV_GROUP, blocks = KV_GROUP / a.scale_tokens;   // of a group

    while (u < u_end) {
        // the sequence and item of unit u
        int b = -1;
        unsigned at = u;
        SeqUnits s{};
        for (int base = 0; base < a.B; base += 64) {
            SeqUnits seq = seq0;
            unsigned mine = mine0, upto = upto0;
            if (base > 0) {
                seq = SeqUnits{};
                if (base + lane < a.B) seq = seq_units(a, base + lane);
                mine = units_of(a, seq);
                upto = lanes_upto(mine);
            }
            const unsigned long long behind = __ballot(upto > at);
            if (behind) {
                s = seq.of_lane(__ffsll(behind) - 1);
                at -= (unsigned)__builtin_amdgcn_readlane((int)(upto - mine), __ffsll(behind) - 1);
                b = base + __ffsll(behind) - 1;
                break;
            }
            at -= last_lane(upto);
        }
        if (b < 0) return;
        const unsigned length = (unsigned)s.groups + ITEM_UNITS, item = at / length;
        const unsigned v0 = at - item * length, v1 = min(length, v0 + (u_end - u));
        u += v1 - v0;
        const int g0 = (int)max(v0, ITEM_UNITS) - (int)ITEM_UNITS, g1 = (int)max(v1, ITEM_UNITS) - (int)ITEM_UNITS;
        if (g0 == g1) continue;
        const int hk = (int)(item / (unsigned)s.row_tiles), r0 = (int)(item - hk * s.row_tiles) * 16;
        const int rows = s.n_q * a.G;
        const int row = min(r0 + r16, rows - 1), token = row / a.G, head = hk * a.G + row - token * a.G;
        const int pos = token + s.n_k - s.n_q;
        const int prefix = a.prefix ? a.prefix[b] : 0;
        const int end = visible_end(a.mask, prefix, pos, s.n_k);
        const int end_first = visible_end(a.mask, prefix, r0 / a.G + s.n_k - s.n_q, s.n_k);   // the fewest keys of the item's rows
        const int end_last = visible_end(a.mask, prefix, (min(r0 + 15, rows - 1)) / a.G + s.n_k - s.n_q, s.n_k);
        const float slope2 = a.slopes ? a.slopes[head] * LOG2E : 0.0f;

        // this wavefront's groups are g0 + wave + 4 i; pages of 64 of them, one per lane
        int pages = -1, pages_at = -64;
        auto page_of = [&](int i) {
            if (i - pages_at >= 64) {
                pages_at = i;
                const int g = g0 + wave + 4 * (i + lane);
                pages = g < g1 ? a.page_table[(size_t)b * a.max_pages + (unsigned)g / page_groups] : -1;
            }
            return __builtin_amdgcn_readlane(pages, i - pages_at);
        };
        // the first group from i on that has a page and a key to see, or the first behind the last
        const int mine = (min(g1, (end_last + KV_GROUP - 1) / KV_GROUP) - g0 - wave + 3) / 4;
        auto next = [&](int i) {
            while (i < mine) {
                const int p = page_of(i);
                if (p >= 0 && p < a.num_pages) break;
                ++i;
            }
            return i;
        };
        uint4 kw[4][KP], vw[DT];
        float kscale, vscale;                          // of token `lane`
        // group i of this wavefront among those of the cache
        auto group_of = [&](int i) { return ((size_t)page_of(i) * a.Hkv + hk) * page_groups + (unsigned)(g0 + wave + 4 * i) % page_groups; };
        auto request_keys = [&](size_t group) __attribute__((always_inline)) {
            const unsigned char *kp = reinterpret_cast<const unsigned char *>(a.kc) + group * (KV_GROUP * (size_t)D);
            const size_t block = group * blocks + (unsigned)lane / (unsigned)a.scale_tokens;
            kscale = a.ks[block];
            vscale = a.vs[block];
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
                for (int k = 0; k < NK; k += WIDE ? 2 : 1) {
                    if (WIDE) {
                        kw[i4][k / 2] = *reinterpret_cast<const uint4 *>(kp + (unsigned)((16 * i4 + r16) * D + 32 * k + 16 * quarter));
                    } else {
                        const int c = min(32 * k + 8 * quarter, D - 8);   // behind D: any codes, the queries there are zero
                        const uint2 w = *reinterpret_cast<const uint2 *>(kp + (unsigned)((16 * i4 + r16) * D + c));
                        if (k % 2 == 0) {
                            kw[i4][k / 2].x = w.x;
                            kw[i4][k / 2].y = w.y;
                        } else {
                            kw[i4][k / 2].z = w.x;
                            kw[i4][k / 2].w = w.y;
                        }
                    }
                }
        };
        auto request_values = [&](size_t group) __attribute__((always_inline)) {
            const unsigned char *vp = reinterpret_cast<const unsigned char *>(a.vc) + group * (KV_GROUP * (size_t)D);
#pragma unroll
            for (int d = 0; d < DT; ++d) vw[d] = *reinterpret_cast<const uint4 *>(vp + (unsigned)(min(16 * d + r16, D - 1) * KV_GROUP + 16 * quarter));
        };

        int i = next(0);
        if (i < mine) {
            const size_t group = group_of(i);
            request_keys(group);
            request_values(group);
        }
        f16x8 qf[NK];
        {
            const _Float16 *q = static_cast<const _Float16 *>(a.q) + (s.first + token) * a.q_row + head * a.q_head;
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                // step k, lane quarter: channels 64 (k / 2) + 16 quarter + 8 (k % 2) in wide pieces, 32 k + 8 quarter otherwise
                const int c = WIDE ? 64 * (k / 2) + 16 * quarter + 8 * (k % 2) : 32 * k + 8 * quarter;
                qf[k] = f16x8{};
                if (c < D) qf[k] = *reinterpret_cast<const f16x8 *>(q + c);
            }
        }
        f32x4 acc[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = f32x4{};
        float m = -__builtin_inff(), l = 0.0f, unit_v = 0.0f;   // of this lane's row; unit_v: the value scale that its sums are in
        while (i < mine) {
            const int j0 = (g0 + wave + 4 * i) * KV_GROUP;
            f32x4 sc[4];
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                sc[i4] = f32x4{};
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    const uint4 w = kw[i4][k / 2];
                    sc[i4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k % 2 == 0 ? codes_f16x8(w.x, w.y) : codes_f16x8(w.z, w.w), qf[k], sc[i4], 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);     // (else the compiler turns all codes into binary16 first, and has no registers for that)
            }
            // scales of this lane's tokens 16 i + 4 quarter + e, through LDS; of tokens behind the end they may hold anything, and are masked below
            scales[lane] = kscale * scale2;
            scales[64 + lane] = vscale;
            // the next unit's keys come in while this one's weights are taken, its values behind this one's
            const int n = next(i + 1);
            size_t group = 0;
            if (n < mine) {
                group = group_of(n);
                request_keys(group);
            }
            f32x4 sk[4], sv[4];
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) sk[i4] = *reinterpret_cast<const f32x4 *>(scales + 16 * i4 + 4 * quarter);
            float top = -__builtin_inff();
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + 16 * i4 + 4 * quarter + e;
                    float y = sc[i4][e] * sk[i4][e];
                    if (shaped) {
                        if (a.cap > 0.0f) y = capped(y * cap_in, cap2);
                        y = __builtin_fmaf(-slope2, fabsf((float)(pos - j)), y);
                    }
                    y = j < end ? y : -__builtin_inff();
                    sc[i4][e] = y;
                    top = fmaxf(top, y);
                }
            top = lanes16_max(top);
            const float m2 = fmaxf(m, top);
            float keep = m == -__builtin_inff() ? 0.0f : exp2_fast(m - m2);
            m = m2;
            l *= keep;
            // the largest value scale that the row has met so far.  One that its mask hides does not count: the weights are rounded relative to it
            float big = 0.0f;
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) sv[i4] = *reinterpret_cast<const f32x4 *>(scales + 64 + 16 * i4 + 4 * quarter);
            if (j0 + KV_GROUP > end_first) {
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sv[i4][e] = j0 + 16 * i4 + 4 * quarter + e < end ? sv[i4][e] : 0.0f;
            }
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
                for (int e = 0; e < 4; ++e) big = fmaxf(big, sv[i4][e]);
            big = lanes16_max(big);
            if (big > unit_v) {
                keep *= unit_v / big;
                unit_v = big;
            }
            const float per = unit_v > LEAST_UNIT ? CACHED_HEAD / unit_v : 0.0f;
            const float mc = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] *= keep;
            f16x8 p[2];
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float w = exp2_fast(sc[i4][e] - mc);
                    l += w;
                    p[i4 / 2][4 * (i4 % 2) + e] = (_Float16)(w * (sv[i4][e] * per));
                }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16x8(vw[d].x, vw[d].y), p[0], acc[d], 0, 0, 0);
                acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16x8(vw[d].z, vw[d].w), p[1], acc[d], 0, 0, 0);
                if (d % 2) __builtin_amdgcn_sched_barrier(0);
            }
            if (n < mine) request_values(group);
            i = n;
        }
        // the four wavefronts' parts: channels 16 d + 4 quarter .. + 3 of row r16
        l = lanes16_sum(l);
        __syncthreads();                               // what an earlier item left here has been read
#pragma unroll
        for (int d = 0; d < DT; ++d)
            if (16 * d + 4 * quarter < D) *reinterpret_cast<f32x4 *>(join + (wave * 16 + r16) * D + 16 * d + 4 * quarter) = acc[d] * (unit_v / CACHED_HEAD);
        if (quarter == 0) {
            join_m[wave * 16 + r16] = m;
            join_l[wave * 16 + r16] = l;
        }
        __syncthreads();
        const bool whole = g0 == 0 && g1 == s.groups;
        float *part = a.partial + (2 * (size_t)blockIdx.x + (g0 == 0 ? 1 : 0)) * (size_t)(16 * (D + 2));
        for (int e = threadIdx.x; e < 16 * (D / 8); e += 256) {
            const int r = e / (D / 8), c = e % (D / 8) * 8;
            if (r0 + r >= rows) continue;
            const float m_all = fmaxf(fmaxf(join_m[r], join_m[16 + r]), fmaxf(join_m[32 + r], join_m[48 + r]));
            float sum[8] = {}, weight = 0.0f;
            if (m_all > -__builtin_inff()) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float k = exp2_fast(join_m[16 * w + r] - m_all);
                    weight += k * join_l[16 * w + r];
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(join + (w * 16 + r) * D + c), y = *reinterpret_cast<const f32x4 *>(join + (w * 16 + r) * D + c + 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        sum[i] += k * x[i];
                        sum[4 + i] += k * y[i];
                    }
                }
            }
            if (whole) {
                const float inv = weight > 0.0f ? 1.0f / weight : 0.0f;
                f16x8 o;
                unsigned amax = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    o[i] = (_Float16)(sum[i] * inv);
                    amax = max(amax, absmax_bits(o[i]));
                }
                const int t = s.first + (r0 + r) / a.G, h = hk * a.G + (r0 + r) % a.G;
                *reinterpret_cast<f16x8 *>(static_cast<_Float16 *>(a.o) + t * a.o_row + h * a.o_head + c) = o;
                if (a.row_absmax) atomicMax(a.row_absmax + t, amax);
            } else {
                *reinterpret_cast<f32x4 *>(part + r * D + c) = f32x4{sum[0], sum[1], sum[2], sum[3]};
                *reinterpret_cast<f32x4 *>(part + r * D + c + 4) = f32x4{sum[4], sum[5], sum[6], sum[7]};
                if (c == 0) {
                    part[16 * D + r] = m_all;
                    part[16 * D + 16 + r] = weight;
                }
            }
        }
    }
}

// Adds up the parts of the items that several workgroups shared: one wavefront per packed row (blockIdx.y: four of an item's 16), blockIdx.x a bound of the
// items.  The parts' maxima and weights go one per lane; the sums are read eight parts at a time.
__global__ __launch_bounds__(256) void join_parts(AttnArgs a, CachedPlan plan)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int D = a.D;
    int b = -1;
    unsigned item = blockIdx.x, u0 = 0, units = 0;
    SeqUnits s{};
    for (int base = 0; base < a.B; base += 64) {
        SeqUnits mine{};
        if (base + lane < a.B) mine = seq_units(a, base + lane);
        const unsigned items = (unsigned)mine.row_tiles * (unsigned)a.Hkv, its_units = units_of(a, mine);
        const unsigned upto = lanes_upto(items), units_upto = lanes_upto(its_units);
        const unsigned long long behind = __ballot(upto > item);
        if (b < 0 && behind) {
            const int l = __ffsll(behind) - 1;
            item -= (unsigned)__builtin_amdgcn_readlane((int)(upto - items), l);
            u0 = units + (unsigned)__builtin_amdgcn_readlane((int)(units_upto - its_units), l);
            s = mine.of_lane(l);
            b = base + l;
        } else if (b < 0) {
            item -= last_lane(upto);
        }
        units += last_lane(units_upto);
    }
    if (b < 0) return;
    const int hk = (int)(item / (unsigned)s.row_tiles), r = 4 * blockIdx.y + wave, row = (int)(item - hk * s.row_tiles) * 16 + r;
    if (row >= s.n_q * a.G) return;
    const Shares shares = shares_of(units, plan.workers);
    u0 += item * ((unsigned)s.groups + ITEM_UNITS) + ITEM_UNITS;
    // the workgroups of the item's first and last group
    const int wa = (int)shares.owner(u0), wb = (int)shares.owner(u0 + s.groups - 1), n = wb - wa + 1;
    if (n == 1) return;
    const size_t stride = 16 * (size_t)(D + 2);
    // workgroup wa's last items's part is its second, the others begin with this item
    auto part = [&](int i) { return a.partial + (2 * (size_t)(wa + i) + (i == 0 ? 1 : 0)) * stride; };
    float m = -__builtin_inff();
    for (int i = lane; i < n; i += 64) m = fmaxf(m, part(i)[16 * D + r]);
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
    const int token = s.first + row / a.G, head = hk * a.G + row % a.G;
    _Float16 *o = static_cast<_Float16 *>(a.o) + token * a.o_row + head * a.o_head;
    f32x4 sum = {};                                    // channels 4 lane .. + 3
    float weight = 0.0f;
    if (m > -__builtin_inff())
        for (int first = 0; first < n; first += 64) {
            float k = 0.0f;
            if (first + lane < n) {
                const float *x = part(first + lane);
                k = exp2_fast(x[16 * D + r] - m);
                weight += k * x[16 * D + 16 + r];
            }
            const int here = min(64, n - first);
            for (int at = 0; at < here; at += 8) {
                f32x4 x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const f32x4 *>(part(first + min(at + i, here - 1)) + r * D + min(4 * lane, D - 4));
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[i] * (at + i < here ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, k), at + i)) : 0.0f);
            }
        }
#pragma unroll
    for (int d = 32; d; d >>= 1) weight += __shfl_xor(weight, d, 64);
    const float inv = weight > 0.0f ? 1.0f / weight : 0.0f;
    unsigned amax = 0;
    if (4 * lane < D) {
        f16x4 h;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const _Float16 x = (_Float16)(sum[e] * inv);
            h[e] = x;
            amax = max(amax, absmax_bits(x));
        }
        *reinterpret_cast<f16x4 *>(o + 4 * lane) = h;
    }
    if (a.row_absmax) {
#pragma unroll
        for (int d = 32; d; d >>= 1) amax = max(amax, (unsigned)__shfl_xor((int)amax, d, 64));
        if (lane == 0) atomicMax(a.row_absmax + token, amax);
    }
}

namespace {
template <int NK, bool WIDE>
hipError_t launch_cached(const AttnArgs &a, const CachedPlan &p, hipStream_t stream)
{
    const int lds = 4 * (64 * a.D + 128 + 512);
    auto *kernel = attend_cached<NK, WIDE>;
    static const hipError_t opt_in = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 4 * (64 * 32 * NK + 128 + 512));
    if (opt_in != hipSuccess) return opt_in;
    hipLaunchKernelGGL(kernel, dim3(p.workers), dim3(256), lds, stream, a, p);
    return hipGetLastError();
}
hipError_t launch_by_head(const AttnArgs &a, const CachedPlan &p, hipStream_t stream)
{
    if (a.D % 64 == 0) {
        if (a.D == 64) return launch_cached<2, true>(a, p, stream);
        if (a.D == 128) return launch_cached<4, true>(a, p, stream);
        if (a.D == 192) return launch_cached<6, true>(a, p, stream);
        return launch_cached<8, true>(a, p, stream);
    }
    if (a.D <= 32) return launch_cached<1, false>(a, p, stream);
    if (a.D <= 64) return launch_cached<2, false>(a, p, stream);
    if (a.D <= 96) return launch_cached<3, false>(a, p, stream);
    if (a.D <= 128) return launch_cached<4, false>(a, p, stream);
    if (a.D <= 192) return launch_cached<6, false>(a, p, stream);
    return launch_cached<8, false>(a, p, stream);
}
}  // namespace

// as many workgroups as the chip holds at once: one more round of them would be a short one
constexpr int CUS = 256;
int cached_workers(int D) { return CUS * cached_waves((D + 31) / 32); }

size_t few_partial_bytes(int D) { return (size_t)cached_workers(D) * 2 * 16 * (D + 2) * 4; }

size_t cached_partial_bytes(long long Tq, int B, int Hq, int Hkv, int D)
{
    const size_t few = few_partial_bytes(D), many = chunks_partial_bytes(Tq, B, Hq, Hkv, D);
    return few > many ? few : many;
}

size_t cached_most_bytes(long long Tq, int B, int Hq, int Hkv, int D)
{
    const size_t few = few_partial_bytes(D), many = chunks_most_bytes(Tq, B, Hq, Hkv, D);
    return few > many ? few : many;
}

// Packed rows of a sequence and key head, on average, up to which they go by 16 rather than by 256 (attention_chunks.hip).  us by 16 / by 256, 32 sequences of 4096 tokens,
// 8 key heads of 128: 32 rows 91 / 189, 64 rows 163 / 192, 128 rows 314 / 201; heads of 64, 1024 tokens: 16 rows 22 / 22, 32 rows 34 / 29, 64 rows 49 / 30.
// The average is right for sequences of about as many rows.  Where one has many and others a single token, all go one way (32 heads of 128 on 8, 4096 tokens each): 63 x 1 row 117 us and
// 1024 rows 162, together by 256 597; 512 rows 108, together with them by 16 233.  By 256 the keys are cut only where the row tiles are few: a row on 131071 tokens, 61 us alone, took 6200
// beside 2048 rows on 4096 (195 alone).  Such a batch is better called in two.
int few_rows(int D) { return D > 64 ? 64 : 16; }

hipError_t launch_attention_kv8(const AttnArgs &a, hipStream_t stream)
{
    if ((long long)a.Tq * a.G > (long long)few_rows(a.D) * a.B) return launch_attention_chunks(a, stream);
    const CachedPlan p{cached_workers(a.D)};
    const hipError_t e = launch_by_head(a, p, stream);
    if (e != hipSuccess) return e;
    const long long items = ((long long)a.Tq * a.G / 16 + a.B) * a.Hkv;
    const long long of_seq = (long long)(a.cu_q ? a.Tq : a.Tq / a.B) * a.G;   // packed rows of a sequence, at most
    hipLaunchKernelGGL(join_parts, dim3((unsigned)items, of_seq < 16 ? (unsigned)(of_seq + 3) / 4 : 4), dim3(256), 0, stream, a, p);
    return hipGetLastError();
}

}  // namespace ql
