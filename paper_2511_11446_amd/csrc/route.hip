// Routing of tokens to experts, the order in which the experts' layers take their rows, and the sum of what the experts give back (gfx950).
#include "daq_f8.h"

#include <type_traits>

namespace ql {

// ---- scores and choice: a wavefront per token -------------------------------------------------------------------------------------------
// In 64 bits throughout: two experts that 32 bits cannot tell apart would make the choice a matter of rounding.
struct Best {
    double c;
    int e;
};
__device__ __forceinline__ Best better(Best a, Best b) { return b.c > a.c || (b.c == a.c && b.e < a.e) ? b : a; }
__device__ __forceinline__ Best best_of_wave(Best b)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) b = better(b, Best{__shfl_xor(b.c, d), __shfl_xor(b.e, d)});
    return b;
}

// One token by the definition.  Experts lane + 64 i in a lane's registers; by: [E] in LDS where there are groups
template <int PER, bool WIDE>
__device__ __forceinline__ void route_exact(const RouteArgs &a, long long t, double *by)
{
    const int lane = threadIdx.x & 63;
    const double none = -__builtin_inf();
    double s[PER], c[PER], key[PER];
    double top = none;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane + 64 * i;
        double x = none;
        if (e < a.E) {
            float f = WIDE ? static_cast<const float *>(a.logits)[t * a.E + e] : (float)static_cast<const _Float16 *>(a.logits)[t * a.E + e];
            const float most = WIDE ? 3.402823466e38f : 65504.0f;
            f = f > most ? most : f;
            x = f > -__builtin_inff() ? (double)f : none;   // NaN is not greater
        }
        key[i] = x;
        top = fmax(top, x);
    }
    if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] = key[i] == none ? 0.0 : 1.0 / (1.0 + exp(-key[i]));
    } else {
#pragma unroll
        for (int d = 32; d; d >>= 1) top = fmax(top, __shfl_xor(top, d));
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s[i] = key[i] == none ? 0.0 : exp(key[i] - top);
            sum += s[i];
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] = sum > 0.0 ? s[i] / sum : 0.0;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        c[i] = key[i] == none ? none : s[i];
        if (a.bias && key[i] != none) {
            c[i] = s[i] + (double)a.bias[lane + 64 * i];
            if (!(c[i] > none)) c[i] = none;   // NaN
            key[i] = c[i];
        }
    }
    if (a.groups > 1 && a.top_groups < a.groups) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (lane + 64 * i < a.E) by[lane + 64 * i] = c[i];
        __threadfence_block();
        __builtin_amdgcn_wave_barrier();
        const int size = a.E / a.groups;
        double worth[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int group = lane + 64 * h;
            worth[h] = none;
            if (group < a.groups) {
                double one = none, two = none;
                for (int j = 0; j < size; ++j) {
                    const double v = by[group * size + j];
                    two = fmax(two, fmin(one, v));
                    one = fmax(one, v);
                }
                worth[h] = a.group_top == 2 && two != none ? one + two : one;
            }
        }
        unsigned long long keep[2] = {0, 0};
        for (int j = 0; j < a.top_groups; ++j) {
            const Best b = best_of_wave(better(Best{worth[0], lane}, Best{worth[1], lane + 64}));
            if (b.c == none) break;
            keep[b.e >> 6] |= 1ull << (b.e & 63);
            if ((b.e & 63) == lane) worth[b.e >> 6] = none;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int group = (lane + 64 * i) / size;
            if (!(keep[(group >> 6) & 1] >> (group & 63) & 1)) key[i] = none;
        }
    }
    // the j-th choice stays with lane j
    double mine = 0.0, sum = 0.0;
    int id = -1;
    for (int j = 0; j < a.k; ++j) {
        Best b{none, 0x7fffffff};
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (key[i] > b.c) b = Best{key[i], lane + 64 * i};
        b = best_of_wave(b);
        if (b.c == none) break;
        double chosen = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (b.e == lane + 64 * i) {
                chosen = s[i];
                key[i] = none;
            }
        chosen = __shfl(chosen, b.e & 63);
        sum += chosen;
        if (lane == j) {
            mine = chosen;
            id = b.e;
        }
    }
    if (lane < a.k) {
        if (a.renorm && sum > 0.0) mine /= sum;
        a.ids[t * a.k + lane] = id;
        a.weights[t * a.k + lane] = (float)(mine * (double)a.scale);
    }
}

// ---- the same where 32 bits can tell the choices apart ---------------------------------------------------------------------------------
// A lane's PER neighbouring experts as keys: whole numbers in the order of the floats (0: cannot be chosen) whose lowest bits say which expert it is, the lower
// number the larger.  The lane sorts its own; a choice is then the largest of 64 heads (six instructions by DPP and a read), whose lane brings up its next.
//   binary16 logits without a bias: the float's lowest 13 bits are free, 9 of them hold the number: every key is another one, the order is exact.
//   fp32 logits without a bias: 3 bits hold the place in the lane.  Two keys that are alike above them: the token is done again in 64 bits.
//   with a bias: s + bias in 32 bits, off by at most ROUTE_NEAR / 2 (exponent, reciprocal and sum 2^-20 of at most 1, the addition 2^-24 of at most 4, the bits
//   for the place 2^-19): two that follow each other and are nearer, or two groups at the border of those that are kept and nearer than GROUP_NEAR: in 64 bits, too.
// The weights are taken in 64 bits, of the chosen alone, those of a workgroup's tokens in one wavefront (k = 8: half of its lanes in the place of 8 of 64 in four of them).
// Where whole lanes hold a group, its two largest are found in registers, else through LDS.
// Bound by vector instructions, 476 a token: T = 16384, E = 256, k = 8, sigmoid, bias, 4 of 8 groups takes 25 us (its logits and choices at the rate of a copy: 3.5), 55 us in 64 bits
// throughout, 35 with each wavefront's weights by itself and groups through LDS.  GROUP_NEAR does not follow the scores' size: of softmax scores, a few hundredths among hundreds of experts,
// two groups are nearer than that more often (as above without a bias 27.5 us, the best 32 of 64 groups 109).
constexpr float ROUTE_NEAR = 0x1p-17f, GROUP_NEAR = 0x1p-12f;

__device__ __forceinline__ unsigned key_of(float f)
{
    const unsigned u = __builtin_bit_cast(unsigned, f + 0.0f);   // -0 is 0
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
constexpr unsigned DEAD = 0x007fffffu;   // key_of(-inf)
__device__ __forceinline__ float float_of(unsigned k) { return __builtin_bit_cast(float, k >> 31 ? k ^ 0x80000000u : ~k); }

// the largest over the wavefront
__device__ __forceinline__ unsigned top_of_wave(unsigned m)
{
#define QL_TOP(ctrl, rows) m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, ctrl, rows, 0xF, false));
    QL_TOP(0x111, 0xF)   // row_shr: 1, 2, 4, 8: lane 15 of a row has the row's
    QL_TOP(0x112, 0xF)
    QL_TOP(0x114, 0xF)
    QL_TOP(0x118, 0xF)
    QL_TOP(0x142, 0xA)   // row_bcast: 15 into rows 1 and 3, 31 into rows 2 and 3
    QL_TOP(0x143, 0xC)
#undef QL_TOP
    return (unsigned)__builtin_amdgcn_readlane((int)m, 63);
}

__device__ __forceinline__ float read_lane(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

// 1 / d of a finite d of ordinary size, to 2^-51 or so: two steps of Newton's iteration from the instruction's 2^-14
__device__ __forceinline__ double inverse(double d)
{
    double r = __builtin_amdgcn_rcp(d);
    r = __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
    r = __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
    return __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
}

template <bool WIDE>
__device__ __forceinline__ float tame(float f)
{
    const float most = WIDE ? 3.402823466e38f : 65504.0f;
    return f > most ? most : f > -__builtin_inff() ? f : -__builtin_inff();   // NaN is not greater
}
template <bool WIDE>
__device__ __forceinline__ float logit_at(const RouteArgs &a, long long at)
{
    return tame<WIDE>(WIDE ? static_cast<const float *>(a.logits)[at] : (float)static_cast<const _Float16 *>(a.logits)[at]);
}

constexpr int ROUTE_TOKENS = 4;   // wavefronts of a workgroup, each with a token
constexpr long long ROUTE_ACROSS = 1 << 23;   // workgroups of a row of the grid, which has less than 2^32 threads

// The choices of token t: true and, in lane j, the j-th one's number (-1: none), or false where 32 bits cannot tell.  top: the largest logit (of the softmax).
// whole: PER divides E and the logits and the bias begin at 16 bytes.  own: 2^own lanes hold a group (-1: they do not)
template <int PER, bool WIDE, bool BIAS, bool GROUPS>
__device__ __forceinline__ bool route_choices(const RouteArgs &a, bool whole, int own, long long t, double *by_expert, int &id, float &top)
{
    const int lane = threadIdx.x & 63;
    const float inf = __builtin_inff();
    constexpr bool EXACT = !WIDE && !BIAS;
    // ---- logits (-inf: dead)
    float x[PER], c[PER];
    top = -inf;
    const int e0 = lane * PER;
    if (whole) {
        typedef typename std::conditional<WIDE, float, _Float16>::type type;
        typedef type types __attribute__((ext_vector_type(PER)));
        types v;
        if (e0 < a.E) v = *reinterpret_cast<const types *>(static_cast<const type *>(a.logits) + t * a.E + e0);
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = e0 < a.E ? tame<WIDE>((float)v[i]) : -inf;
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            x[i] = -inf;
            if (e0 + i < a.E) x[i] = logit_at<WIDE>(a, t * a.E + e0 + i);
        }
    }
    if (!a.sigmoid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) top = fmaxf(top, x[i]);
    }
    if (!a.sigmoid) top = float_of(top_of_wave(key_of(top)));
    bool near = false;
    if constexpr (BIAS || GROUPS) {
        constexpr float LOG2E = 1.44269504f;
        if (a.sigmoid) {
#pragma unroll
            for (int i = 0; i < PER; ++i) c[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-x[i] * LOG2E));   // (dead: 0)
        } else {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                c[i] = x[i] > -inf ? __builtin_amdgcn_exp2f((x[i] - top) * LOG2E) : 0.0f;
                sum += c[i];
            }
#pragma unroll
            for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
            const float r = sum > 0.0f ? __builtin_amdgcn_rcpf(sum) : 0.0f;
#pragma unroll
            for (int i = 0; i < PER; ++i) c[i] *= r;
        }
        if constexpr (BIAS) {
            float bias[PER];
            if (whole) {
                typedef float floats __attribute__((ext_vector_type(PER)));
                floats v;
                if (e0 < a.E) v = *reinterpret_cast<const floats *>(a.bias + e0);
#pragma unroll
                for (int i = 0; i < PER; ++i) bias[i] = v[i];
            } else {
#pragma unroll
                for (int i = 0; i < PER; ++i) bias[i] = a.bias[min(e0 + i, a.E - 1)];
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (x[i] > -inf) c[i] += bias[i];
                near |= fabsf(c[i]) > 4.0f && c[i] > -inf;   // of another size than the scores: more is lost than the bound says
            }
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) c[i] = x[i] > -inf && c[i] > -inf ? c[i] : -inf;   // (NaN is not greater)
        if (BIAS) near = __any(near);
    }
    // ---- keys
    unsigned key[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float f = BIAS ? c[i] : x[i];
        const unsigned k = key_of(f);
        key[i] = f == -inf ? 0u : EXACT ? (k & ~511u) | (511 - (e0 + i)) : (k & ~7u) | (7 - i);
    }
    if (GROUPS && !near && own >= 0) {
        // 2^own lanes hold a group's experts and no others': its two largest in registers, as keys
        unsigned one = key_of(c[0]), two = 0;
#pragma unroll
        for (int i = 1; i < PER; ++i) {
            const unsigned v = key_of(c[i]);
            two = max(two, min(one, v));
            one = max(one, v);
        }
        auto join = [&](unsigned o1, unsigned o2) {
            two = max(max(two, o2), min(one, o1));
            one = max(one, o1);
        };
#define QL_JOIN(ctrl) join((unsigned)__builtin_amdgcn_mov_dpp((int)one, ctrl, 0xF, 0xF, true), (unsigned)__builtin_amdgcn_mov_dpp((int)two, ctrl, 0xF, 0xF, true))
        if (own > 0) QL_JOIN(0xB1);    // the neighbour's, the neighbouring pair's, the other half's of 8 lanes, of 16
        if (own > 1) QL_JOIN(0x4E);
        if (own > 2) QL_JOIN(0x141);
        if (own > 3) QL_JOIN(0x140);
#undef QL_JOIN
        if (own > 4) join(__shfl_xor(one, 16), __shfl_xor(two, 16));
        if (own > 5) join(__shfl_xor(one, 32), __shfl_xor(two, 32));
        const float most = float_of(one), worth = a.group_top == 2 && two > DEAD ? most + float_of(two) : most;
        const int group = lane >> own;
        unsigned group_key = one > DEAD && group < a.groups ? (key_of(worth) & ~127u) | (127 - group) : 0u;
        bool kept = false;
        unsigned before = 0;
        for (int j = 0; j < a.top_groups; ++j) {
            before = top_of_wave(group_key);
            const bool best = group_key == before;
            kept |= best;
            group_key = best ? 0u : group_key;
        }
        const unsigned beyond = top_of_wave(group_key);
        near = beyond && float_of(before) - float_of(beyond) < GROUP_NEAR;
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = kept ? key[i] : 0u;
    } else if (GROUPS && !near) {
        float *by = reinterpret_cast<float *>(by_expert);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (e0 + i < a.E) by[e0 + i] = c[i];
        __threadfence_block();
        __builtin_amdgcn_wave_barrier();
        const int size = a.E / a.groups;
        // 2^l lanes a group, each with every 2^l-th of its experts; groups beyond 64 in a second round
        int l = 0;
        while (a.groups << (l + 1) <= 64) ++l;
        const int rounds = a.groups > 64 ? 2 : 1;
        float worth[2] = {-inf, -inf};
        for (int h = 0; h < rounds; ++h) {
            const int group = (lane >> l) + 64 * h;
            float one = -inf, two = -inf;
            if (group < a.groups) {
                for (int j = lane & ((1 << l) - 1); j < size; j += 1 << l) {
                    const float v = by[group * size + j];
                    two = fmaxf(two, fminf(one, v));
                    one = fmaxf(one, v);
                }
            }
            for (int d = 1; d >> l == 0; d *= 2) {
                const float o1 = __shfl_xor(one, d), o2 = __shfl_xor(two, d);
                two = fmaxf(fmaxf(two, o2), fminf(one, o1));
                one = fmaxf(one, o1);
            }
            worth[h] = a.group_top == 2 && two > -inf ? one + two : one;
        }
        // The worthiest groups, as keys with the number in 7 bits (2^-14 of a worth of up to 8): where the last that is kept and the first that is not are
        // nearer than GROUP_NEAR, in 64 bits.  Every lane of a group has its key, and the group's bit in `keep` is its number.
        unsigned group_key[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int group = (lane >> l) + 64 * h;
            group_key[h] = h < rounds && group < a.groups && worth[h] > -inf ? (key_of(worth[h]) & ~127u) | (127 - group) : 0u;
        }
        unsigned long long keep[2] = {0, 0};
        unsigned before = 0, best = 0;
        for (int j = 0; j <= a.top_groups; ++j) {
            before = best;
            best = top_of_wave(max(group_key[0], group_key[1]));
            const int group = 127 - (int)(best & 127);
            const unsigned long long bit = best && j < a.top_groups ? 1ull << (group & 63) : 0;
            if (group < 64) keep[0] |= bit;
            else keep[1] |= bit;
#pragma unroll
            for (int h = 0; h < 2; ++h) group_key[h] = group_key[h] == best ? 0u : group_key[h];
        }
        near = best && float_of(before) - float_of(best) < GROUP_NEAR;
        const float per_group = __builtin_amdgcn_rcpf((float)size);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int group = (int)(((float)(e0 + i) + 0.5f) * per_group);   // ((e + 1/2) / size is 1/1024 from any whole number at least)
            key[i] = (group < 64 ? keep[0] : keep[1]) >> (group & 63) & 1 ? key[i] : 0u;
        }
    }
    // ---- a lane's own in order
#pragma unroll
    for (int i = 1; i < PER; ++i)
#pragma unroll
        for (int j = i; j > 0; --j) {
            const unsigned hi = max(key[j - 1], key[j]), lo = min(key[j - 1], key[j]);
            key[j - 1] = hi, key[j] = lo;
        }
    // ---- choices: the j-th one's key and the lane that it came from stay with lane j.  (Without branches: a choice that there is not is key 0.)
    unsigned picked = 0;
    int from = 0;
    unsigned long long alike = 0;
    auto look = [&](int &at) {
        const unsigned best = top_of_wave(key[0]);
        const unsigned long long owners = __ballot(key[0] == best);
        if (!EXACT) {
            alike |= best ? owners & (owners - 1) : 0;
            at = __builtin_ctzll(owners);
        }
        const bool mine = key[0] == best;
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = mine ? (i + 1 < PER ? key[i + 1 < PER ? i + 1 : i] : 0u) : key[i];
        return best;
    };
    for (int j = 0; j < a.k; ++j) {
        int at = 0;
        const unsigned best = look(at);
        picked = lane == j ? best : picked;
        if (!EXACT) from = lane == j ? at : from;
    }
    const unsigned k = picked;
    if (EXACT) id = 511 - (int)(k & 511);
    else {
        // where keys are not exact, the next one after each has to be far enough away, also that after the last
        int at;
        const unsigned beyond = look(at);
        unsigned next = __shfl_down(k, 1);
        next = lane == a.k - 1 ? beyond : next;
        near |= __any(lane < a.k && next && ((k ^ next) < 8u || (BIAS && float_of(k) - float_of(next) < ROUTE_NEAR)));
        near |= alike != 0;
        id = from * PER + 7 - (int)(k & 7);
    }
    if (!k || lane >= a.k) id = -1;
    return !near;
}

template <int PER, bool WIDE, bool BIAS, bool GROUPS>
__global__ __launch_bounds__(64 * ROUTE_TOKENS) void route(RouteArgs a, bool whole, int own, int places)   // 2^places: k, rounded up
{
    extern __shared__ double by_expert[];   // [ROUTE_TOKENS][E] where there are groups
    __shared__ int chosen[ROUTE_TOKENS][64];
    __shared__ double totals[ROUTE_TOKENS];
    __shared__ float tops[ROUTE_TOKENS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long t0 = ((long long)blockIdx.y * ROUTE_ACROSS + blockIdx.x) * ROUTE_TOKENS, t = t0 + wave;
    constexpr int ELSEWHERE = -2;   // no token, or one whose choices are made in 64 bits
    int id = ELSEWHERE;
    float top = 0.0f;
    bool exact = false;
    if (t < a.T) {
        exact = !route_choices<PER, WIDE, BIAS, GROUPS>(a, whole, own, t, by_expert + (GROUPS ? wave * a.E : 0), id, top);
        if (exact) id = ELSEWHERE;
        else if (!a.renorm && !a.sigmoid) {
            double total = 0.0;
            for (int e = lane; e < a.E; e += 64) {
                const float f = logit_at<WIDE>(a, t * a.E + e);
                if (f > -__builtin_inff()) total += exp((double)f - (double)top);
            }
#pragma unroll
            for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
            if (lane == 0) totals[wave] = total;
        }
    }
    chosen[wave][lane] = id;
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    // ---- weights: the workgroup's choices, 2^places lanes a token
    const int width = 1 << places, token = (int)threadIdx.x >> places, j = (int)threadIdx.x & (width - 1);
    if (token < ROUTE_TOKENS) {
        id = chosen[token][j];
        const long long to = t0 + token;
        double total = 1.0, w = 0.0;
        if (id >= 0) {
            const double l = (double)logit_at<WIDE>(a, to * a.E + id);
            const double e = exp(a.sigmoid ? -l : l - (double)tops[token]);
            w = !a.sigmoid ? e : e < __builtin_inf() ? inverse(1.0 + e) : 0.0;
        }
        if (a.renorm) {
            total = w;
            for (int d = 1; d < width; d *= 2) total += __shfl_xor(total, d);   // (lanes behind the last choice have 0)
        } else if (!a.sigmoid) total = totals[token];
        if (id != ELSEWHERE && j < a.k) {
            if (total != 1.0) w = total > 0.0 ? w / total : 0.0;
            a.ids[to * a.k + j] = id;
            a.weights[to * a.k + j] = (float)(w * (double)a.scale);
        }
    }
    if (exact) route_exact<PER, WIDE>(a, t, by_expert + wave * a.E);
}

template <int PER>
static void run_route(const RouteArgs &a, hipStream_t s)
{
    const long long groups_of_tokens = (a.T + ROUTE_TOKENS - 1ll) / ROUTE_TOKENS;
    const dim3 grid((unsigned)(groups_of_tokens < ROUTE_ACROSS ? groups_of_tokens : ROUTE_ACROSS), (unsigned)((groups_of_tokens + ROUTE_ACROSS - 1) / ROUTE_ACROSS));
    const size_t lds = a.groups > 1 ? (size_t)ROUTE_TOKENS * a.E * sizeof(double) : 0;
    int own = -1, places = 0;
    for (int l = 0; l <= 6; ++l)
        if ((a.E / a.groups) == PER << l) own = l;
    while (1 << places < a.k) ++places;
    const bool groups = a.groups > 1 && a.top_groups < a.groups, whole = a.E % PER == 0 && (uintptr_t)a.logits % 16 == 0 && (uintptr_t)a.bias % 16 == 0;
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * ROUTE_TOKENS), lds, s, a, whole, own, places); };
    if (a.wide) {
        if (a.bias) groups ? run(route<PER, true, true, true>) : run(route<PER, true, true, false>);
        else groups ? run(route<PER, true, false, true>) : run(route<PER, true, false, false>);
    } else {
        if (a.bias) groups ? run(route<PER, false, true, true>) : run(route<PER, false, true, false>);
        else groups ? run(route<PER, false, false, true>) : run(route<PER, false, false, false>);
    }
}

hipError_t launch_route(const RouteArgs &a, hipStream_t s)
{
    if (a.E <= 64) run_route<1>(a, s);
    else if (a.E <= 128) run_route<2>(a, s);
    else if (a.E <= 256) run_route<4>(a, s);
    else run_route<8>(a, s);
    return hipGetLastError();
}

// ---- rows in the order of their experts -------------------------------------------------------------------------------------------------
// A stable counting sort of (token, choice) by expert, in chunks of EXPERT_CHUNK.  A wavefront ranks 64 of them at a time: lanes of the same expert
// find each other by one ballot for each bit of its number.  No atomics: the order is that of the tokens, every time.
constexpr int ROWS_THREADS = 1024, ROWS_WAVES = ROWS_THREADS / 64, ROWS_STEPS = EXPERT_CHUNK / ROWS_THREADS;

// lanes whose `e` is this lane's (lanes without an expert: e = -1)
__device__ __forceinline__ unsigned long long same_lanes(int e, int bits)
{
    unsigned long long same = __ballot(e >= 0);
    for (int b = 0; b < bits; ++b) {
        const unsigned long long set = __ballot(e >> b & 1);
        same &= (e >> b & 1) ? set : ~set;
    }
    return same;
}

__device__ __forceinline__ int expert_of(const int *ids, long long p, int P, int E)
{
    const int e = p < P ? ids[p] : -1;
    return e >= 0 && e < E ? e : -1;
}

// counts[wave][E] of this workgroup's chunk, which has to be zero
__device__ __forceinline__ void count_chunk(const int *ids, const ExpertRows &r, int bits, int *counts)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = 0; i < ROWS_STEPS; ++i) {
        const long long p = (long long)blockIdx.x * EXPERT_CHUNK + wave * (64 * ROWS_STEPS) + 64 * i + lane;
        const int e = expert_of(ids, p, r.P, r.E);
        const unsigned long long same = same_lanes(e, bits);
        if (e >= 0 && (same & ((1ull << lane) - 1)) == 0) counts[wave * r.E + e] += __popcll(same);
        __threadfence_block();
    }
}

__global__ __launch_bounds__(ROWS_THREADS) void expert_count(const int *ids, ExpertRows r, int bits)
{
    extern __shared__ int counts[];   // [waves][E]
    for (int i = threadIdx.x; i < ROWS_WAVES * r.E; i += ROWS_THREADS) counts[i] = 0;
    __syncthreads();
    count_chunk(ids, r, bits, counts);
    __syncthreads();
    for (int e = threadIdx.x; e < r.E; e += ROWS_THREADS) {
        int sum = 0;
        for (int w = 0; w < ROWS_WAVES; ++w) sum += counts[w * r.E + e];
        r.counts[blockIdx.x * r.E + e] = sum;
    }
}

// sums over the threads in front of this one, of two numbers at once
__device__ __forceinline__ int2 before_me(int2 v, int2 *of_wave)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int2 s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(s.x, d), y = __shfl_up(s.y, d);
        if (lane >= d) s = make_int2(s.x + x, s.y + y);
    }
    if (lane == 63) of_wave[wave] = s;
    __syncthreads();
    int2 front = make_int2(s.x - v.x, s.y - v.y);
    for (int w = 0; w < wave; ++w) front = make_int2(front.x + of_wave[w].x, front.y + of_wave[w].y);
    __syncthreads();
    return front;
}

// The workgroups behind the chunks quantize the tokens meanwhile (64 tokens of 2048 channels, 8 of 128 experts: 7.7 us, apart 6.9 and
// 4.8; 16384 tokens, 8 of 64: 29.5, apart 10.3 and 21.6)
__global__ __launch_bounds__(ROWS_THREADS) void expert_place(const int *ids, ExpertRows r, int bits, int chunks, int most, F8DaqArgs x)
{
    extern __shared__ int counts[];   // [waves][E]
    if ((int)blockIdx.x >= chunks) {
        constexpr int AT_ONCE = ROWS_THREADS / 16;
        daq_f8_blocks<false, false>(x, (long long)(blockIdx.x - chunks) * AT_ONCE + (threadIdx.x >> 4), (long long)(gridDim.x - chunks) * AT_ONCE);
        return;
    }
    __shared__ int2 of_wave[ROWS_WAVES];
    for (int i = threadIdx.x; i < ROWS_WAVES * r.E; i += ROWS_THREADS) counts[i] = 0;
    __syncthreads();
    count_chunk(ids, r, bits, counts);
    __syncthreads();
    // thread e: the rows of expert e, those in the chunks in front of this one, and where they begin
    const int e = threadIdx.x;
    int all = 0, front = 0;
    if (e < r.E) {
        if (chunks == 1) {
            for (int w = 0; w < ROWS_WAVES; ++w) all += counts[w * r.E + e];
        } else {
            for (int first = 0; first < chunks; first += 16) {   // sixteen under way together: one after the other they were 18 us of 131072 rows' 23
                int n[16];
#pragma unroll
                for (int c = 0; c < 16; ++c) n[c] = r.counts[min(first + c, chunks - 1) * r.E + e];
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    n[c] = within(n[c], EXPERT_CHUNK + 1);
                    all += first + c < chunks ? n[c] : 0;
                    front += first + c < (int)blockIdx.x ? n[c] : 0;
                }
            }
        }
    }
    const int tiles = (all + r.tile - 1) / r.tile;
    const int2 at = before_me(make_int2(all, tiles), of_wave);
    if (e < r.E) {
        int base = at.x + front;
        for (int w = 0; w < ROWS_WAVES; ++w) {
            const int n = counts[w * r.E + e];
            counts[w * r.E + e] = base;
            base += n;
        }
        if (blockIdx.x == 0) {
            r.first[e] = at.x;
            for (int i = 0; i < tiles && (unsigned)(at.y + i) < (unsigned)most; ++i) {
                r.tiles[1 + 2 * (at.y + i)] = e;
                r.tiles[2 + 2 * (at.y + i)] = at.x + i * r.tile;
            }
            if (e == r.E - 1) {
                r.first[r.E] = at.x + all;
                r.tiles[0] = at.y + tiles;
            }
        }
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = 0; i < ROWS_STEPS; ++i) {
        const long long p = (long long)blockIdx.x * EXPERT_CHUNK + wave * (64 * ROWS_STEPS) + 64 * i + lane;
        const int mine = expert_of(ids, p, r.P, r.E);
        const unsigned long long same = same_lanes(mine, bits);
        int row = -1;
        if (mine >= 0) row = within(counts[wave * r.E + mine] + __popcll(same & ((1ull << lane) - 1)), r.P);
        __threadfence_block();
        if (mine >= 0 && (same & ((1ull << lane) - 1)) == 0) counts[wave * r.E + mine] += __popcll(same);
        __threadfence_block();
        if (p < r.P) r.place[p] = row;
        if (row >= 0) r.order[row] = (int)p;
    }
}

hipError_t launch_expert_rows(const int *ids, const ExpertRows &r, const F8DaqArgs &x, hipStream_t s)
{
    int bits = 0;
    while (1 << bits < r.E) ++bits;
    const unsigned chunks = (unsigned)expert_chunks(r.P);
    const size_t lds = (size_t)ROWS_WAVES * r.E * sizeof(int);
    if (chunks > 1) {
        hipLaunchKernelGGL(expert_count, dim3(chunks), dim3(ROWS_THREADS), lds, s, ids, r, bits);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const long long blocks = ((long long)x.M * x.KB * 16 + ROWS_THREADS - 1) / ROWS_THREADS;
    hipLaunchKernelGGL(expert_place, dim3(chunks + (unsigned)(blocks < 1024 ? blocks : 1024)), dim3(ROWS_THREADS), lds, s, ids, r, bits, (int)chunks,
                       (int)expert_tiles_most(r.P, r.E, r.tile), x);
    return hipGetLastError();
}

// ---- the sum over a token's experts ----------------------------------------------------------------------------------------------------
// One pass: each output row is read once, the token's rows are added up in fp32 in the order of its choices.  8 outputs a thread (16-byte pieces).
template <bool WIDE>
__global__ __launch_bounds__(256) void expert_sum(ExpertSumArgs a)
{
    typedef _Float16 h8 __attribute__((ext_vector_type(8)));
    constexpr int TOGETHER = 8;   // choices whose rows are under way together
    const long long pieces = a.N / 8, all = pieces * a.T;
    const int rows = a.T * a.k;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
        const long long t = i / pieces, n = (i - t * pieces) * 8;
        float y[8];
        h8 res = {0, 0, 0, 0, 0, 0, 0, 0};
        if (a.residual) res = *reinterpret_cast<const h8 *>(static_cast<const _Float16 *>(a.residual) + t * a.N + n);
#pragma unroll
        for (int c = 0; c < 8; ++c) y[c] = (float)res[c];
        for (int first = 0; first < a.k; first += TOGETHER) {
            int row[TOGETHER];
            float w[TOGETHER];
#pragma unroll
            for (int j = 0; j < TOGETHER; ++j) {
                const long long at = t * a.k + min(first + j, a.k - 1);
                const int place = a.place[at];
                w[j] = a.weights[at];
                row[j] = first + j >= a.k ? -1 : !a.ids ? place : place >= 0 && place < a.E ? (int)at : -1;
            }
            if constexpr (WIDE) {
                float4 o[TOGETHER][2];
#pragma unroll
                for (int j = 0; j < TOGETHER; ++j) {
                    const float4 *from = reinterpret_cast<const float4 *>(static_cast<const float *>(a.o) + (long long)within(row[j], rows) * a.N + n);
                    o[j][0] = from[0], o[j][1] = from[1];
                }
#pragma unroll
                for (int j = 0; j < TOGETHER; ++j) {
                    const float v[8] = {o[j][0].x, o[j][0].y, o[j][0].z, o[j][0].w, o[j][1].x, o[j][1].y, o[j][1].z, o[j][1].w};
#pragma unroll
                    for (int c = 0; c < 8; ++c) y[c] = row[j] >= 0 ? __builtin_fmaf(w[j], v[c], y[c]) : y[c];
                }
            } else {
                h8 o[TOGETHER];
                int up[TOGETHER];
#pragma unroll
                for (int j = 0; j < TOGETHER; ++j) {
                    const long long from = within(row[j], rows);
                    o[j] = *reinterpret_cast<const h8 *>(static_cast<const _Float16 *>(a.o) + from * a.N + n);
                    up[j] = a.up[from * ((a.N + F8_UP - 1) / F8_UP) + n / F8_UP];
                }
#pragma unroll
                for (int j = 0; j < TOGETHER; ++j) w[j] = __builtin_ldexpf(w[j], up[j]);
#pragma unroll
                for (int j = 0; j < TOGETHER; ++j)
#pragma unroll
                    for (int c = 0; c < 8; ++c) y[c] = row[j] >= 0 ? __builtin_fmaf(w[j], (float)o[j][c], y[c]) : y[c];
            }
        }
        h8 out;
#pragma unroll
        for (int c = 0; c < 8; ++c) out[c] = (_Float16)y[c];
        *reinterpret_cast<h8 *>(static_cast<_Float16 *>(a.y) + t * a.N + n) = out;
    }
}

hipError_t launch_expert_sum(const ExpertSumArgs &a, hipStream_t s)
{
    const long long blocks = ((long long)a.T * (a.N / 8) + 255) / 256;
    const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192));
    if (a.wide) hipLaunchKernelGGL((expert_sum<true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((expert_sum<false>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace ql
