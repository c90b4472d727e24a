// New keys and values into the paged 8-bit cache, with the position rotation on the way, for gfx950.
//
//   h = fp16(rot(k)), fp16(v);  per block of S tokens and key head: amax = max |h| over the new tokens
//   alpha = max(alpha_old, amax / 127)   alpha_old: the block's scale where it holds earlier tokens of the sequence, else 0
//   new codes  clamp(rne(h / alpha), -127, 127);   earlier codes of the block, where alpha grew, clamp(rne(code * alpha_old / alpha))
// A block of zeros has scale 0 and codes 0 (not 1 as a row of daq.hip: a later token may raise it).
//
// One workgroup per sequence, touched group of 64 tokens and key head: it alone writes that group's codes and scales, so nothing is
// atomic in global memory and results do not depend on order.  Keys and values are read once and held in registers between the
// maximum and the codes.  A thread has an 8-channel piece of four neighbouring tokens, whose value codes are one word of the cache.
#include "attention.h"
#include "daq_device.h"

namespace ql {

typedef _Float16 h8v __attribute__((ext_vector_type(8)));

// piece p (8 channels) of the turned row at x; `angle` is the row's cos / sin table row
__device__ __forceinline__ uint4 turned_piece(const _Float16 *x, int p, const float *angle, int rot_dim, bool pairs)
{
    const uint4 own = *reinterpret_cast<const uint4 *>(x + 8 * p);
    if (8 * p >= rot_dim) return own;
    const h8v a = __builtin_bit_cast(h8v, own);
    h8v out;
    if (pairs) {
        const float4 t0 = *reinterpret_cast<const float4 *>(angle + 8 * p), t1 = *reinterpret_cast<const float4 *>(angle + 8 * p + 4);
        const float c[4] = {t0.x, t0.z, t1.x, t1.z}, s[4] = {t0.y, t0.w, t1.y, t1.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float u = (float)a[2 * i] * c[i] - (float)a[2 * i + 1] * s[i], v = (float)a[2 * i + 1] * c[i] + (float)a[2 * i] * s[i];
            asm volatile("" : "+v"(u), "+v"(v));   // keep the fp32 rounding before the fp16 one
            out[2 * i] = (_Float16)u;
            out[2 * i + 1] = (_Float16)v;
        }
    } else {
        const int half = rot_dim / 16;             // in pieces
        const bool low = p < half;
        const int first = low ? p : p - half;
        const h8v b = *reinterpret_cast<const h8v *>(x + 8 * (low ? p + half : p - half));
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float4 t = *reinterpret_cast<const float4 *>(angle + 2 * (8 * first + i));   // cos, sin of two channels
            const float s0 = low ? -t.y : t.y, s1 = low ? -t.w : t.w;
            float u = (float)a[i] * t.x + (float)b[i] * s0, v = (float)a[i + 1] * t.z + (float)b[i + 1] * s1;
            asm volatile("" : "+v"(u), "+v"(v));
            out[i] = (_Float16)u;
            out[i + 1] = (_Float16)v;
        }
    }
    return __builtin_bit_cast(uint4, out);
}

__device__ __forceinline__ unsigned piece_absmax(uint4 v)
{
    const unsigned m = absmax_word(absmax_word(absmax_word(absmax_word(0, v.x), v.y), v.z), v.w);
    return max(m & 0xffffu, m >> 16);
}

// binary16 values of a piece's codes
__device__ __forceinline__ uint4 code_values(uint2 c, float alpha)
{
    h8v o;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float u = (float)(int8_t)((i < 4 ? c.x : c.y) >> (8 * (i % 4))) * alpha;
        asm volatile("" : "+v"(u));
        o[i] = (_Float16)u;
    }
    return __builtin_bit_cast(uint4, o);
}

// byte i of a word of earlier codes under the grown scale
__device__ __forceinline__ unsigned code_again(unsigned word, int i, float old_alpha, float alpha)
{
    const float v = (float)(int8_t)(word >> (8 * i)) * old_alpha;
    return (unsigned)(daq_code(v, alpha) & 0xff);
}

// tokens of sequence b that are new: rows of k, v, q and places in the cache
struct NewTokens {
    int row, first, n, groups;   // row of the token at place `first`; groups of 64 that they touch
};
__device__ __forceinline__ NewTokens new_tokens(const KvAppendArgs &a, int b)
{
    const SeqRows r = seq_rows(a.cu, b, a.T, a.B);
    const int len = max(a.len_k[b], 0);
    const int cut = max(r.n - len, 0);            // rows that would lie in front of the sequence
    NewTokens t;
    t.row = r.first + cut;
    t.n = r.n - cut;
    t.first = len - t.n;
    t.groups = t.n ? (len - 1) / KV_GROUP - t.first / KV_GROUP + 1 : 0;
    return t;
}

constexpr int VT_PITCH = KV_GROUP + 4;

template <int NI>   // pieces of four tokens per thread
__global__ __launch_bounds__(256) void kv_append(KvAppendArgs a)
{
    __shared__ unsigned amax_k[KV_GROUP], amax_v[KV_GROUP];
    __shared__ float alpha_k[KV_GROUP], alpha_v[KV_GROUP];
    __shared__ float was_k, was_v;
    extern __shared__ __align__(16) unsigned char vt[];   // [D][VT_PITCH] value codes of the group

    const int tid = threadIdx.x, lane = tid & 63;
    const int hk = blockIdx.x % a.Hkv;
    int item = blockIdx.x / a.Hkv;
    // the sequence and group of this workgroup: 64 sequences at a time, one per lane
    int b = -1;
    NewTokens nt{};
    for (int base = 0; base < a.B; base += 64) {
        NewTokens mine{};
        if (base + lane < a.B) mine = new_tokens(a, base + lane);
        int upto = mine.groups;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d, 64);
            if (lane >= d) upto += o;
        }
        const unsigned long long behind = __ballot(upto > item);
        if (behind) {
            const int l = __ffsll((unsigned long long)behind) - 1;
            b = base + l;
            nt.row = __shfl(mine.row, l, 64);
            nt.first = __shfl(mine.first, l, 64);
            nt.n = __shfl(mine.n, l, 64);
            item -= __shfl(upto - mine.groups, l, 64);
            break;
        }
        item -= __shfl(upto, 63, 64);
    }
    if (b < 0) return;
    const int group = nt.first / KV_GROUP + item;
    // places in the group: new tokens are [tlo, thi); earlier ones of the sequence lie in front
    const int base = group * KV_GROUP;
    const int tlo = max(nt.first - base, 0), thi = min(nt.first + nt.n - base, KV_GROUP);
    const int row0 = nt.row + base - nt.first;            // row of place 0
    const int page_at = base / a.page, in_page = base % a.page;
    int page = page_at < a.max_pages ? a.page_table[(size_t)b * a.max_pages + page_at] : -1;
    const bool held = page >= 0 && page < a.num_pages;
    if (!held) page = 0;
    const size_t ph = (size_t)page * a.Hkv + hk;
    int8_t *kc = a.kc + (ph * a.page + in_page) * a.D;
    unsigned char *vc = reinterpret_cast<unsigned char *>(a.vc) + (ph * (a.page / KV_GROUP) + in_page / KV_GROUP) * (size_t)(a.D * KV_GROUP);
    const int S = a.scale_tokens;
    float *ks = a.ks + ph * (a.page / S) + in_page / S, *vs = a.vs + ph * (a.page / S) + in_page / S;

    if (tid < KV_GROUP) {
        amax_k[tid] = 0;
        amax_v[tid] = 0;
    }
    __syncthreads();
    const int P8 = a.D / 8;
    const _Float16 *k = static_cast<const _Float16 *>(a.k) + hk * a.k_head, *v = static_cast<const _Float16 *>(a.v) + hk * a.v_head;
    auto angle_of = [&](int t) {
        const int p = min(max(a.pos ? a.pos[row0 + t] : base + t, 0), a.rot_rows - 1);
        return a.rot + (size_t)p * a.rot_dim;
    };
    uint4 kp[NI][4], vp[NI][4];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int id = tid + 256 * n, piece = id % P8, quad = id / P8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * quad + i;
            kp[n][i] = vp[n][i] = make_uint4(0, 0, 0, 0);
            if (t < tlo || t >= thi) continue;
            const _Float16 *kr = k + (row0 + t) * a.k_row;
            kp[n][i] = a.rot ? turned_piece(kr, piece, angle_of(t), a.rot_dim, a.rot_pairs) : *reinterpret_cast<const uint4 *>(kr + 8 * piece);
            vp[n][i] = *reinterpret_cast<const uint4 *>(v + (row0 + t) * a.v_row + 8 * piece);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * quad + i;
            if (t < tlo || t >= thi) continue;
            atomicMax(&amax_k[t / S], piece_absmax(kp[n][i]));
            atomicMax(&amax_v[t / S], piece_absmax(vp[n][i]));
        }
    }
    __syncthreads();
    // scales: thread i has block i of the keys, thread 64 + i block i of the values
    const int shared_block = tlo / S;                       // the one block that may hold earlier tokens
    const bool earlier = held && tlo % S != 0;
    if (tid < 128 && tid % 64 < KV_GROUP / S) {
        const int blk = tid % 64;
        float *scale = tid < 64 ? ks : vs;
        const float old = earlier && blk == shared_block ? scale[blk] : 0.0f;
        const float alpha = fmaxf(old, half_bits_to_float(tid < 64 ? amax_k[blk] : amax_v[blk]) / 127.0f);
        (tid < 64 ? alpha_k : alpha_v)[blk] = alpha;
        if (blk == shared_block) (tid < 64 ? was_k : was_v) = old;
        if (held && blk * S < thi && (blk + 1) * S > tlo) scale[blk] = alpha;
    }
    __syncthreads();
    const bool again_k = earlier && alpha_k[shared_block] > was_k, again_v = earlier && alpha_v[shared_block] > was_v;
    // many new value codes, or earlier ones that change, go through LDS: whole 16-byte pieces of the group
    const bool whole = held && (again_v || thi - tlo >= 16);
    if (whole && (tlo > 0 || thi < KV_GROUP)) {
        for (int c = tid; c < a.D * 4; c += 256) {
            const uint4 w = *reinterpret_cast<const uint4 *>(vc + c * 16);
            unsigned *to = reinterpret_cast<unsigned *>(vt + (c / 4) * VT_PITCH + (c % 4) * 16);
            to[0] = w.x;
            to[1] = w.y;
            to[2] = w.z;
            to[3] = w.w;
        }
        __syncthreads();
    }
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int id = tid + 256 * n, piece = id % P8, quad = id / P8;
        if (quad >= 16) continue;
        uint2 vcode[4];
        unsigned fresh = 0;                                 // bytes of the word that are new
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * quad + i;
            vcode[i] = make_uint2(0, 0);
            if (t >= tlo && t < thi) {
                fresh |= 0xffu << (8 * i);
                const float ak = alpha_k[t / S] > 0.0f ? alpha_k[t / S] : 1.0f, av = alpha_v[t / S] > 0.0f ? alpha_v[t / S] : 1.0f;
                const uint2 kcode = daq_piece(kp[n][i], ak, 1.0f / ak);
                vcode[i] = daq_piece(vp[n][i], av, 1.0f / av);
                if (held) *reinterpret_cast<uint2 *>(kc + (size_t)t * a.D + 8 * piece) = kcode;
                const size_t out = ((size_t)(row0 + t) * a.Hkv + hk) * a.D + 8 * piece;
                if (a.k_out) *reinterpret_cast<uint4 *>(static_cast<_Float16 *>(a.k_out) + out) = code_values(kcode, ak);
                if (a.v_out) *reinterpret_cast<uint4 *>(static_cast<_Float16 *>(a.v_out) + out) = code_values(vcode[i], av);
            } else if (again_k && t < tlo && t / S == shared_block) {
                uint2 *at = reinterpret_cast<uint2 *>(kc + (size_t)t * a.D + 8 * piece);
                const uint2 w = *at;
                uint2 o = make_uint2(0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o.x |= code_again(w.x, e, was_k, alpha_k[shared_block]) << (8 * e);
                    o.y |= code_again(w.y, e, was_k, alpha_k[shared_block]) << (8 * e);
                }
                *at = o;
            }
        }
        if (!held) continue;
        const int at = 16 * (quad % 4) + 4 * (quad / 4);    // of the quad's word among the 64 bytes of a channel
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int sh = 8 * (e % 4);
            unsigned word = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) word |= ((e < 4 ? vcode[i].x : vcode[i].y) >> sh & 0xffu) << (8 * i);
            const int d = 8 * piece + e;
            if (whole) {
                unsigned *to = reinterpret_cast<unsigned *>(vt + d * VT_PITCH + at);
                if (fresh != 0xffffffffu) {
                    unsigned was = *to;
                    if (again_v) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int t = 4 * quad + i;
                            if (t < tlo && t / S == shared_block) was = (was & ~(0xffu << (8 * i))) | code_again(was, i, was_v, alpha_v[shared_block]) << (8 * i);
                        }
                    }
                    word = (word & fresh) | (was & ~fresh);
                }
                *to = word;
            } else if (fresh == 0xffffffffu) {
                *reinterpret_cast<unsigned *>(vc + d * KV_GROUP + at) = word;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (fresh >> (8 * i) & 1) vc[d * KV_GROUP + at + i] = (unsigned char)(word >> (8 * i));
            }
        }
    }
    if (whole) {
        __syncthreads();
        for (int c = tid; c < a.D * 4; c += 256) {
            const unsigned *from = reinterpret_cast<const unsigned *>(vt + (c / 4) * VT_PITCH + (c % 4) * 16);
            *reinterpret_cast<uint4 *>(vc + c * 16) = make_uint4(from[0], from[1], from[2], from[3]);
        }
    }
    // the query heads that read this key head
    if (!a.q_out) return;
    const int pieces = (thi - tlo) * a.G * P8;
    for (int c = tid; c < pieces; c += 256) {
        const int piece = c % P8, h = hk * a.G + c / P8 % a.G, t = tlo + c / (P8 * a.G);
        const _Float16 *qr = static_cast<const _Float16 *>(a.q) + (row0 + t) * a.q_row + h * a.q_head;
        const uint4 o = a.rot ? turned_piece(qr, piece, angle_of(t), a.rot_dim, a.rot_pairs) : *reinterpret_cast<const uint4 *>(qr + 8 * piece);
        *reinterpret_cast<uint4 *>(static_cast<_Float16 *>(a.q_out) + ((size_t)(row0 + t) * a.Hq + h) * a.D + 8 * piece) = o;
    }
}

hipError_t launch_kv_append(const KvAppendArgs &a, hipStream_t stream)
{
    // n >= 1 tokens touch at most (n + 62) / 64 + 1 groups
    const long long per_seq = a.T / a.B;
    const long long groups = a.cu ? (long long)a.T / KV_GROUP + 2LL * a.B : (per_seq + KV_GROUP - 2) / KV_GROUP * a.B + a.B;
    const dim3 grid((unsigned)(groups * a.Hkv));
    if (a.D <= 128) hipLaunchKernelGGL(kv_append<1>, grid, dim3(256), a.D * VT_PITCH, stream, a);
    else hipLaunchKernelGGL(kv_append<2>, grid, dim3(256), a.D * VT_PITCH, stream, a);
    return hipGetLastError();
}

}  // namespace ql
