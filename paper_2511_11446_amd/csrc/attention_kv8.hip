// Attention of few rows over the paged 8-bit cache for gfx950: single tokens, and short runs of them.
//
// The work is the cache's bytes: a unit is one group of 64 tokens of one key head for up to 16 packed rows (attention.h).  The launch is a fixed number
// of workgroups that share all units of all sequences evenly, whatever the lengths: workgroup w has the units [w U / W, (w + 1) U / W) of the list that goes
// sequence by sequence, key head by key head.  Where an item (the units of one set of rows) is cut between workgroups, each leaves sums, maximum and
// weight in the workspace and join_parts puts them together.
//
// Codes go from global memory straight into the registers where the matrix instruction (16x16x32) wants them: a lane has 16 neighbouring bytes of a
// key for two steps of the scores, and 16 neighbouring bytes of the value codes of one channel - four tokens of each of the group's four tiles - which
// are the left operand of O^T = V^T P^T in the order in which S^T = K Q^T leaves the weights.  So nothing goes through LDS but the join of
// the workgroup's four wavefronts, which take the units in turn.
//
// Codes become binary16 exactly; key scales multiply the scores.  Value scales multiply the weights, relative to the largest one met so far (which the sums are
// relative to in turn): a weight times a bare scale could fall below binary16's range.
#include "attention_tile.h"

namespace ql {

struct CachedPlan {
    int workers;          // workgroups of the launch
};

constexpr int UNITS_PER_WORKER = 4;   // at least, where there are as many: one for every wavefront

// what one sequence has of units and items
struct SeqUnits {
    int n_q, first, n_k, row_tiles, groups;
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
__device__ __forceinline__ long long lanes_upto(long long v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const long long o = __shfl_up(v, d, 64);
        if (lane >= d) v += o;
    }
    return v;
}
__device__ __forceinline__ long long units_of(const AttnArgs &a, int b)
{
    const SeqUnits s = seq_units(a, b);
    return (long long)s.row_tiles * s.groups * a.Hkv;
}
__device__ __forceinline__ long long all_units(const AttnArgs &a)
{
    const int lane = threadIdx.x & 63;
    long long total = 0;
    for (int base = 0; base < a.B; base += 64) total += __shfl(lanes_upto(base + lane < a.B ? units_of(a, base + lane) : 0), 63, 64);
    return total;
}
__device__ __forceinline__ long long workers_of(long long units, int most)
{
    const long long w = (units + UNITS_PER_WORKER - 1) / UNITS_PER_WORKER;
    return w < most ? w : most;
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

// wavefronts per SIMD: as many as the loads of a whole unit leave registers for
constexpr int cached_waves(int NK, bool TOKEN) { return NK <= 2 ? (TOKEN ? 3 : 4) : NK <= 4 ? (TOKEN ? 2 : 3) : NK <= 6 ? 2 : 1; }

// NK: 32-channel steps of the scores; WIDE: D is a multiple of 64, keys in 16-byte pieces (else 8); TOKEN: a scale for every token
template <int NK, bool WIDE, bool TOKEN>
__global__ __launch_bounds__(256, cached_waves(NK, TOKEN)) void attend_cached(AttnArgs a, CachedPlan plan)
{
    constexpr int DT = 2 * NK;
    extern __shared__ __align__(16) float join[];     // [4][16][D] sums, [4][16] maxima, [4][16] weights
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int quarter = lane >> 4, r16 = lane & 15;
    const int D = a.D;
    float *join_m = join + 64 * D, *join_l = join_m + 64;

    const long long units = all_units(a);
    const long long workers = workers_of(units, plan.workers);
    if (blockIdx.x >= workers) return;
    long long u = blockIdx.x * units / workers;
    const long long u_end = (blockIdx.x + 1) * units / workers;
    const bool shaped = a.cap > 0.0f || a.slopes;
    const float cap2 = a.cap * LOG2E;

    while (u < u_end) {
        // the sequence and item of unit u
        int b = -1;
        long long at = u;
        for (int base = 0; base < a.B; base += 64) {
            const long long mine = base + lane < a.B ? units_of(a, base + lane) : 0, upto = lanes_upto(mine);
            const unsigned long long behind = __ballot(upto > at);
            if (behind) {
                const int l = __ffsll(behind) - 1;
                at -= __shfl(upto - mine, l, 64);
                b = __builtin_amdgcn_readfirstlane(base + l);
                break;
            }
            at -= __shfl(upto, 63, 64);
        }
        if (b < 0) return;
        const SeqUnits s = seq_units(a, b);
        const int item = __builtin_amdgcn_readfirstlane((int)(at / s.groups));
        const int g0 = __builtin_amdgcn_readfirstlane((int)(at % s.groups));
        const int g1 = (int)(s.groups - g0 < u_end - u ? s.groups : g0 + (u_end - u));
        const int hk = item / s.row_tiles, r0 = item % s.row_tiles * 16;
        const int rows = s.n_q * a.G;
        const int row = min(r0 + r16, rows - 1), token = row / a.G, head = hk * a.G + row % a.G;
        const int pos = token + s.n_k - s.n_q;
        const int prefix = a.prefix ? a.prefix[b] : 0;
        const int end = visible_end(a.mask, prefix, pos, s.n_k);
        const int end_last = visible_end(a.mask, prefix, (min(r0 + 15, rows - 1)) / a.G + s.n_k - s.n_q, s.n_k);

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
        const float scale2 = a.scale * LOG2E, cap_in = a.cap > 0.0f ? 2.0f * scale2 / a.cap : scale2;
        const float slope2 = a.slopes ? a.slopes[head] * LOG2E : 0.0f;

        f32x4 acc[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = f32x4{};
        float m = -__builtin_inff(), l = 0.0f, unit_v = 0.0f;   // unit_v: the value scale that the sums are in
        int pages = -1;
        for (int i = 0, g = g0 + wave; g < g1; ++i, g += 4) {
            if (i % 64 == 0) {
                // page of this wavefront's next 64 groups, one per lane
                const int mine = g + 4 * lane;
                pages = mine < g1 ? a.page_table[(size_t)b * a.max_pages + mine * KV_GROUP / a.page] : -1;
            }
            const int page = __builtin_amdgcn_readlane(pages, i % 64);
            const int j0 = g * KV_GROUP;
            if (j0 >= end_last || page < 0 || page >= a.num_pages) continue;
            const size_t ph = (size_t)page * a.Hkv + hk;
            const int in_page = j0 % a.page;
            const unsigned char *kp = reinterpret_cast<const unsigned char *>(a.kc) + (ph * a.page + in_page) * D;
            const unsigned char *vp = reinterpret_cast<const unsigned char *>(a.vc) + (ph * a.page + in_page) * D;
            uint4 kw[4][WIDE ? NK / 2 : (NK + 1) / 2];
            uint4 vw[DT];
            if (WIDE) {
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
                    for (int k = 0; k < NK / 2; ++k) kw[i4][k] = *reinterpret_cast<const uint4 *>(kp + (unsigned)((16 * i4 + r16) * D + 64 * k + 16 * quarter));
            } else {
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
                    for (int k = 0; k < NK; ++k) {
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
#pragma unroll
            for (int d = 0; d < DT; ++d) vw[d] = *reinterpret_cast<const uint4 *>(vp + (unsigned)(min(16 * d + r16, D - 1) * KV_GROUP + 16 * quarter));
            // scales of this lane's tokens 16 i + 4 quarter + e
            const float *ks = a.ks + ph * (a.page / a.scale_tokens) + in_page / a.scale_tokens, *vs = a.vs + ph * (a.page / a.scale_tokens) + in_page / a.scale_tokens;
            f32x4 sk[4], sv[4];
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                if (TOKEN) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sk[i4][e] = ks[16 * i4 + 4 * quarter + e];
                        sv[i4][e] = vs[16 * i4 + 4 * quarter + e];
                    }
                } else {
                    const float x = ks[16 * i4 / a.scale_tokens], y = vs[16 * i4 / a.scale_tokens];
                    sk[i4] = f32x4{x, x, x, x};
                    sv[i4] = f32x4{y, y, y, y};
                }
                // of tokens behind the end a scale may hold anything
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = TOKEN ? j0 + 16 * i4 + 4 * quarter + e : j0 + 16 * i4;
                    if (j >= s.n_k) sv[i4][e] = 0.0f;
                }
            }
            f32x4 sc[4];
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                sc[i4] = f32x4{};
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    const uint4 w = kw[i4][k / 2];
                    sc[i4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k % 2 == 0 ? codes_f16x8(w.x, w.y) : codes_f16x8(w.z, w.w), qf[k], sc[i4], 0, 0, 0);
                }
            }
            float top = -__builtin_inff();
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + 16 * i4 + 4 * quarter + e;
                    float y = sc[i4][e] * (sk[i4][e] * cap_in);
                    if (shaped) {
                        if (a.cap > 0.0f) y = capped(y, cap2);
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
            // the largest value scale so far
            float big = 0.0f;
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
                for (int e = 0; e < (TOKEN ? 4 : 1); ++e) big = fmaxf(big, sv[i4][e]);
            if (TOKEN) big = lanes16_max(big);
            if (big > unit_v) {
                keep *= unit_v / big;
                unit_v = big;
            }
            const float per = unit_v > 0.0f ? 1.0f / unit_v : 0.0f;
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
            }
        }
        // the four wavefronts' parts: channels 16 d + 4 quarter .. + 3 of row r16
        l = lanes16_sum(l);
        __syncthreads();                               // what an earlier item left here has been read
#pragma unroll
        for (int d = 0; d < DT; ++d)
            if (16 * d + 4 * quarter < D) *reinterpret_cast<f32x4 *>(join + (wave * 16 + r16) * D + 16 * d + 4 * quarter) = acc[d] * unit_v;
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
        u += g1 - g0;
    }
}

// one workgroup per item (a bound of them): adds up the parts of those that several workgroups shared
__global__ __launch_bounds__(256) void join_parts(AttnArgs a, CachedPlan plan)
{
    const int lane = threadIdx.x & 63;
    const int D = a.D;
    const long long units = all_units(a);
    const long long workers = workers_of(units, plan.workers);
    int b = -1;
    long long item = blockIdx.x, u0 = 0;
    for (int base = 0; base < a.B; base += 64) {
        SeqUnits s{};
        if (base + lane < a.B) s = seq_units(a, base + lane);
        const long long items = (long long)s.row_tiles * a.Hkv, mine = items * s.groups;
        const long long upto = lanes_upto(items), units_upto = lanes_upto(mine);
        const unsigned long long behind = __ballot(upto > item);
        if (behind) {
            const int l = __ffsll(behind) - 1;
            item -= __shfl(upto - items, l, 64);
            u0 += __shfl(units_upto - mine, l, 64);
            b = __builtin_amdgcn_readfirstlane(base + l);
            break;
        }
        item -= __shfl(upto, 63, 64);
        u0 += __shfl(units_upto, 63, 64);
    }
    if (b < 0) return;
    const SeqUnits s = seq_units(a, b);
    u0 += item * s.groups;
    const long long u1 = u0 + s.groups;
    // workgroup w has units [w U / W, (w + 1) U / W): the ones of the first and the last unit
    auto owner = [&](long long u) {
        long long w = u * workers / units;
        while (w > 0 && w * units / workers > u) --w;
        while ((w + 1) * units / workers <= u) ++w;
        return w;
    };
    const long long wa = owner(u0), wb = owner(u1 - 1);
    if (wa == wb) return;
    const int hk = (int)(item / s.row_tiles), r0 = (int)(item % s.row_tiles) * 16, rows = s.n_q * a.G;
    const size_t stride = 16 * (size_t)(D + 2);
    auto part = [&](long long w) { return a.partial + (2 * (size_t)w + (w == wa ? 1 : 0)) * stride; };
    for (int e = threadIdx.x; e < 16 * (D / 8); e += 256) {
        const int r = e / (D / 8), c = e % (D / 8) * 8;
        if (r0 + r >= rows) continue;
        float m = -__builtin_inff();
        for (long long w = wa; w <= wb; ++w) m = fmaxf(m, part(w)[16 * D + r]);
        float sum[8] = {}, weight = 0.0f;
        if (m > -__builtin_inff())
            for (long long w = wa; w <= wb; ++w) {
                const float *x = part(w);
                const float k = exp2_fast(x[16 * D + r] - m);
                weight += k * x[16 * D + 16 + r];
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += k * x[r * D + c + i];
            }
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
    }
}

namespace {
template <int NK, bool WIDE, bool TOKEN>
hipError_t launch_cached(const AttnArgs &a, const CachedPlan &p, hipStream_t stream)
{
    const int lds = 4 * (64 * a.D + 128);
    auto *kernel = attend_cached<NK, WIDE, TOKEN>;
    static const hipError_t opt_in = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 4 * (64 * 32 * NK + 128));
    if (opt_in != hipSuccess) return opt_in;
    hipLaunchKernelGGL(kernel, dim3(p.workers), dim3(256), lds, stream, a, p);
    return hipGetLastError();
}
template <bool TOKEN>
hipError_t launch_by_head(const AttnArgs &a, const CachedPlan &p, hipStream_t stream)
{
    if (a.D % 64 == 0) {
        if (a.D == 64) return launch_cached<2, true, TOKEN>(a, p, stream);
        if (a.D == 128) return launch_cached<4, true, TOKEN>(a, p, stream);
        if (a.D == 192) return launch_cached<6, true, TOKEN>(a, p, stream);
        return launch_cached<8, true, TOKEN>(a, p, stream);
    }
    if (a.D <= 32) return launch_cached<1, false, TOKEN>(a, p, stream);
    if (a.D <= 64) return launch_cached<2, false, TOKEN>(a, p, stream);
    if (a.D <= 96) return launch_cached<3, false, TOKEN>(a, p, stream);
    if (a.D <= 128) return launch_cached<4, false, TOKEN>(a, p, stream);
    if (a.D <= 192) return launch_cached<6, false, TOKEN>(a, p, stream);
    return launch_cached<8, false, TOKEN>(a, p, stream);
}
}  // namespace

int cached_workers(int D) { return D <= 128 ? 1024 : 512; }

size_t cached_partial_bytes(long long Tq, int B, int Hq, int Hkv, int D)
{
    const size_t few = (size_t)cached_workers(D) * 2 * 16 * (D + 2) * 4, many = chunks_partial_bytes(Tq, B, Hq, Hkv, D);
    return few > many ? few : many;
}

// packed rows of a sequence and key head, on average, up to which they go by 16
constexpr int FEW_ROWS = 16;

hipError_t launch_attention_kv8(const AttnArgs &a, hipStream_t stream)
{
    if ((long long)a.Tq * a.G > (long long)FEW_ROWS * a.B) return launch_attention_chunks(a, stream);
    const CachedPlan p{cached_workers(a.D)};
    const hipError_t e = a.scale_tokens == 1 ? launch_by_head<true>(a, p, stream) : launch_by_head<false>(a, p, stream);
    if (e != hipSuccess) return e;
    const long long items = ((long long)a.Tq * a.G / 16 + a.B) * a.Hkv;
    hipLaunchKernelGGL(join_parts, dim3((unsigned)items), dim3(256), 0, stream, a, p);
    return hipGetLastError();
}

}  // namespace ql
