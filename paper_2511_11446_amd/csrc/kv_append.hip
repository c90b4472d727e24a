// New keys and values into the paged 8-bit cache, with the position rotation on the way, for gfx950.
//
//   h = fp16(rot(k)), fp16(v);  per block of S tokens and key head: amax = max |h| over the new tokens
//   alpha = max(alpha_old, amax / 127)   alpha_old: the block's scale where it holds earlier tokens of the sequence, else 0
//   new codes  clamp(rne(h / alpha), -127, 127);   earlier codes of the block, where alpha grew, clamp(rne(code * alpha_old / alpha))
// A block of zeros has scale 0 and codes 0 (not 1 as a row of daq.hip: a later token may raise it).
//
// One workgroup per sequence, touched group of 64 tokens and key head: it alone writes that group's codes and scales, so nothing is
// atomic in global memory and results do not depend on order.  Keys and values are read once and held in registers between the
// maximum and the codes.  Of the values a thread has an 8-channel piece of four neighbouring tokens, whose codes are one word of the cache;
// of the keys what a few cosines turn, which it then uses for the queries of all heads that read the key head.
//
// 16 prompts of 1 to 1024 tokens, 32 heads of 128 on 8, queries turned: 59 us for 219 MB, 3.7 TB/s, 1.37 times a copy's time: a thread has nothing of its next unit of
// keys and queries under way while it turns and stores one.  One token
// for each of 64 sequences: 8.6 us, a chain of latencies (find the sequence, its length, its page, the earlier scale, the block's maximum, the codes).
#include "attention.h"
#include "daq_device.h"

namespace ql {

typedef _Float16 h8v __attribute__((ext_vector_type(8)));

// A row is turned by units: two 8-channel pieces that 8 neighbouring (cos, sin) of the table turn - pieces e and e + rot_dim / 16, or the neighbours
// 2 e and 2 e + 1 - and single pieces behind the turned channels, as they are.
struct Turn {
    float4 t[4];   // cos, sin, cos, sin
};
struct Pieces {
    uint4 a, b;
};
__device__ __forceinline__ Turn load_turn(const float *angle, int e)
{
    Turn r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.t[i] = *reinterpret_cast<const float4 *>(angle + 16 * e + 4 * i);
    return r;
}
__device__ __forceinline__ Pieces turned(const Pieces &x, const Turn &r, bool pairs)
{
    const h8v a = __builtin_bit_cast(h8v, x.a), b = __builtin_bit_cast(h8v, x.b);
    h8v p, q;
    if (pairs) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = i % 2 ? r.t[i / 2].z : r.t[i / 2].x, s = i % 2 ? r.t[i / 2].w : r.t[i / 2].y;
            const int at = 2 * (i % 4);
            const float u0 = i < 4 ? (float)a[at] : (float)b[at], v0 = i < 4 ? (float)a[at + 1] : (float)b[at + 1];
            float u = u0 * c - v0 * s, v = v0 * c + u0 * s;
            asm volatile("" : "+v"(u), "+v"(v));   // keep the fp32 rounding before the fp16 one
            if (i < 4) {
                p[at] = (_Float16)u;
                p[at + 1] = (_Float16)v;
            } else {
                q[at] = (_Float16)u;
                q[at + 1] = (_Float16)v;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = i % 2 ? r.t[i / 2].z : r.t[i / 2].x, s = i % 2 ? r.t[i / 2].w : r.t[i / 2].y;
            float u = (float)a[i] * c - (float)b[i] * s, v = (float)b[i] * c + (float)a[i] * s;
            asm volatile("" : "+v"(u), "+v"(v));
            p[i] = (_Float16)u;
            q[i] = (_Float16)v;
        }
    }
    return {__builtin_bit_cast(uint4, p), __builtin_bit_cast(uint4, q)};
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

// an LDS maximum per block: lanes of one block first among themselves where that is the whole wavefront
__device__ __forceinline__ void block_max(unsigned *of_block, int t, int S, unsigned m, bool live)
{
    if (S == KV_GROUP) {
        m = wave_max_u32(live ? m : 0u);
        if ((threadIdx.x & 63) == 0) atomicMax(of_block, m);
    } else if (live) {
        atomicMax(of_block + t / S, m);
    }
}

template <int NI>   // 128-channel parts of a head: a thread has NI pieces of four tokens (values) and up to 4 NI units of a token (keys)
__global__ __launch_bounds__(256) void kv_append(KvAppendArgs a)
{
    __shared__ unsigned amax_k[KV_GROUP], amax_v[KV_GROUP];
    __shared__ float alpha_k[KV_GROUP], alpha_v[KV_GROUP];
    __shared__ float was_k, was_v;
    extern __shared__ __align__(16) unsigned char vt[];   // [D][VT_PITCH] value codes of the group

    const int tid = threadIdx.x;
    const int hk = blockIdx.x % a.Hkv;
    int item = blockIdx.x / a.Hkv;
    const int b = find_sequence(a.B, item, [&](int s) { return new_tokens(a, s).groups; });
    if (b < 0) return;
    const NewTokens nt = new_tokens(a, b);
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
    // scales: thread i has block i of the keys, thread 64 + i block i of the values
    const int blk = tid % 64, shared_block = tlo / S;     // the one block that may hold earlier tokens
    const bool earlier = held && tlo % S != 0;
    float *scale = tid < 64 ? ks : vs;
    const float old = earlier && tid < 128 && blk == shared_block ? scale[blk] : 0.0f;
    const int P8 = a.D / 8, R16 = a.rot ? a.rot_dim / 16 : 0, units = P8 - R16;   // of a row: R16 turned ones, then single pieces
    const int count = (thi - tlo) * units;                // units of the new tokens, token by token
    const _Float16 *k = static_cast<const _Float16 *>(a.k) + hk * a.k_head, *v = static_cast<const _Float16 *>(a.v) + hk * a.v_head;
    auto angle_of = [&](int t) {
        const int p = min(max(a.pos ? a.pos[row0 + t] : base + t, 0), a.rot_rows - 1);
        return a.rot + (size_t)p * a.rot_dim;
    };
    auto first_piece = [&](int e) { return e >= R16 ? e + R16 : a.rot_pairs ? 2 * e : e; };
    const int second = a.rot_pairs ? 1 : R16;             // from a turned unit's first piece to its second
    auto load = [&](const _Float16 *x, int e) {
        const int p = first_piece(e);
        Pieces r;
        r.a = *reinterpret_cast<const uint4 *>(x + 8 * p);
        r.b = make_uint4(0, 0, 0, 0);
        if (e < R16) r.b = *reinterpret_cast<const uint4 *>(x + 8 * (p + second));
        return r;
    };
    // values: four tokens of a piece, whose codes are one word of the cache
    uint4 vp[NI][4];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int id = tid + 256 * n, quad = id / P8, piece = id - quad * P8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * quad + i;
            vp[n][i] = make_uint4(0, 0, 0, 0);
            if (t >= tlo && t < thi) vp[n][i] = *reinterpret_cast<const uint4 *>(v + (row0 + t) * a.v_row + 8 * piece);
        }
    }
    // queries of the heads that read this key head: with the cosines of the keys below, or, where there are few, a thread each
    const bool few = count * a.G <= 256;
    const _Float16 *q0 = static_cast<const _Float16 *>(a.q) + hk * a.G * a.q_head;
    _Float16 *q_out = static_cast<_Float16 *>(a.q_out) + hk * a.G * a.D;
    if (a.q_out && few && tid < count * a.G) {
        const int h = tid / count, id = tid - h * count, in = id / units, e = id - in * units, t = tlo + in;
        Pieces x = load(q0 + (row0 + t) * a.q_row + h * a.q_head, e);
        if (e < R16) x = turned(x, load_turn(angle_of(t), e), a.rot_pairs);
        _Float16 *out = q_out + ((size_t)(row0 + t) * a.Hq + h) * a.D + 8 * first_piece(e);
        *reinterpret_cast<uint4 *>(out) = x.a;
        if (e < R16) *reinterpret_cast<uint4 *>(out + 8 * second) = x.b;
    }
    // keys, turned
    Pieces kp[4 * NI];
#pragma unroll
    for (int n = 0; n < 4 * NI; ++n) {
        const int id = tid + 256 * n, in = id / units, e = id - in * units, t = tlo + in;
        kp[n].a = kp[n].b = make_uint4(0, 0, 0, 0);
        const bool live = id < count;
        if (live) {
            kp[n] = load(k + (row0 + t) * a.k_row, e);
            Turn r{};
            if (e < R16) {
                r = load_turn(angle_of(t), e);
                kp[n] = turned(kp[n], r, a.rot_pairs);
            }
            if (a.q_out && !few) {
                const _Float16 *q = q0 + (row0 + t) * a.q_row;
                _Float16 *out = q_out + (size_t)(row0 + t) * a.Hq * a.D + 8 * first_piece(e);
                for (int h0 = 0; h0 < a.G; h0 += 4) {
                    Pieces x[4];
#pragma unroll
                    for (int h = 0; h < 4; ++h) x[h] = load(q + min(h0 + h, a.G - 1) * a.q_head, e);
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        if (h0 + h >= a.G) break;
                        const Pieces y = e < R16 ? turned(x[h], r, a.rot_pairs) : x[h];
                        *reinterpret_cast<uint4 *>(out + (h0 + h) * a.D) = y.a;
                        if (e < R16) *reinterpret_cast<uint4 *>(out + (h0 + h) * a.D + 8 * second) = y.b;
                    }
                }
            }
        }
        if (256 * n < count) block_max(amax_k, t, S, max(piece_absmax(kp[n].a), piece_absmax(kp[n].b)), live);
    }
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int quad = (tid + 256 * n) / P8;
        if (S == KV_GROUP) {
            unsigned m = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) m = max(m, piece_absmax(vp[n][i]));
            block_max(amax_v, 0, S, m, true);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) block_max(amax_v, 4 * quad + i, S, piece_absmax(vp[n][i]), 4 * quad + i >= tlo && 4 * quad + i < thi);
        }
    }
    __syncthreads();
    if (tid < 128 && blk < KV_GROUP / S) {
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
    // key codes
#pragma unroll
    for (int n = 0; n < 4 * NI; ++n) {
        const int id = tid + 256 * n, in = id / units, e = id - in * units, t = tlo + in;
        if (id >= count) break;
        const float alpha = alpha_k[t / S] > 0.0f ? alpha_k[t / S] : 1.0f, rcp = 1.0f / alpha;
        const int p = first_piece(e);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i && e >= R16) break;
            const int c = 8 * (p + i * second);
            const uint2 code = daq_piece(i ? kp[n].b : kp[n].a, alpha, rcp);
            if (held) *reinterpret_cast<uint2 *>(kc + (size_t)t * a.D + c) = code;
            if (a.k_out) *reinterpret_cast<uint4 *>(static_cast<_Float16 *>(a.k_out) + ((size_t)(row0 + t) * a.Hkv + hk) * a.D + c) = code_values(code, alpha);
        }
    }
    if (again_k) {
        const int t0 = shared_block * S;                  // earlier tokens [t0, tlo) of the block
        for (int id = tid; id < (tlo - t0) * P8; id += 256) {
            uint2 *at = reinterpret_cast<uint2 *>(kc + (size_t)t0 * a.D) + id;
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
    // value codes
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int id = tid + 256 * n, quad = id / P8, piece = id - quad * P8;
        if (quad >= 16) continue;
        uint2 vcode[4];
        unsigned fresh = 0;                                 // bytes of the word that are new
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * quad + i;
            vcode[i] = make_uint2(0, 0);
            if (t < tlo || t >= thi) continue;
            fresh |= 0xffu << (8 * i);
            const float alpha = alpha_v[t / S] > 0.0f ? alpha_v[t / S] : 1.0f;
            vcode[i] = daq_piece(vp[n][i], alpha, 1.0f / alpha);
            if (a.v_out) *reinterpret_cast<uint4 *>(static_cast<_Float16 *>(a.v_out) + ((size_t)(row0 + t) * a.Hkv + hk) * a.D + 8 * piece) = code_values(vcode[i], alpha);
        }
        if (!held || (!whole && fresh == 0)) continue;
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
