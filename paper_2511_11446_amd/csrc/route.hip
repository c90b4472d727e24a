// Routing of tokens to experts, the order in which the experts' layers take their rows, and the sum of what the experts give back (gfx950).
#include "daq_device.h"
#include "f8.h"

namespace ql {

// ---- scores and choice: a wavefront per token, experts lane + 64 i in a lane's registers -----------------------------------------------
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

template <int PER, bool WIDE>
__global__ __launch_bounds__(256) void route(RouteArgs a)
{
    extern __shared__ double by_expert[];   // [4][E] where there are groups
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long t = (long long)blockIdx.x * 4 + wave;
    if (t >= a.T) return;
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
        double *by = by_expert + wave * a.E;
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

template <int PER>
static void run_route(const RouteArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.T + 3ll) / 4));
    const size_t lds = a.groups > 1 ? (size_t)4 * a.E * sizeof(double) : 0;
    if (a.wide) hipLaunchKernelGGL((route<PER, true>), grid, dim3(256), lds, s, a);
    else hipLaunchKernelGGL((route<PER, false>), grid, dim3(256), lds, s, a);
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

__global__ __launch_bounds__(ROWS_THREADS) void expert_place(const int *ids, ExpertRows r, int bits)
{
    extern __shared__ int counts[];   // [waves][E]
    __shared__ int2 of_wave[ROWS_WAVES];
    for (int i = threadIdx.x; i < ROWS_WAVES * r.E; i += ROWS_THREADS) counts[i] = 0;
    __syncthreads();
    count_chunk(ids, r, bits, counts);
    __syncthreads();
    // thread e: the rows of expert e, those in the chunks in front of this one, and where they begin
    const int e = threadIdx.x;
    int all = 0, front = 0;
    if (e < r.E) {
        if (gridDim.x == 1) {
            for (int w = 0; w < ROWS_WAVES; ++w) all += counts[w * r.E + e];
        } else {
            for (int c = 0; c < (int)gridDim.x; ++c) {
                const int n = r.counts[c * r.E + e];
                all += n;
                front += c < (int)blockIdx.x ? n : 0;
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
            for (int i = 0; i < tiles; ++i) {
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
        if (mine >= 0) row = counts[wave * r.E + mine] + __popcll(same & ((1ull << lane) - 1));
        __threadfence_block();
        if (mine >= 0 && (same & ((1ull << lane) - 1)) == 0) counts[wave * r.E + mine] += __popcll(same);
        __threadfence_block();
        if (p < r.P) r.place[p] = row;
        if (row >= 0) r.order[row] = (int)p;
    }
}

hipError_t launch_expert_rows(const int *ids, const ExpertRows &r, hipStream_t s)
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
    hipLaunchKernelGGL(expert_place, dim3(chunks), dim3(ROWS_THREADS), lds, s, ids, r, bits);
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
                    const float4 *from = reinterpret_cast<const float4 *>(static_cast<const float *>(a.o) + (long long)max(row[j], 0) * a.N + n);
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
#pragma unroll
                for (int j = 0; j < TOGETHER; ++j) o[j] = *reinterpret_cast<const h8 *>(static_cast<const _Float16 *>(a.o) + (long long)max(row[j], 0) * a.N + n);
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
