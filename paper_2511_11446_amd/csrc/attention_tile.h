// The tile of attention: a wavefront's 32 packed rows against 64 keys at a time, keys and values from binary16 rows or from the 8-bit cache
// (attention.hip, attention_chunks.hip).  Not part of the public ABI.
//
// Scores come as S^T = K Q^T (mfma 32x32x16): a lane has ONE row (lane & 31) and 16 of 32 keys, so the running maximum and sum of a row
// are the lane's own up to one exchange with lane ^ 32, masks and biases know the row without an index, and the weights are in the
// place where O^T = V^T P^T wants its right operand: keys 16 s + 8 (j / 4) + 4 (lane / 32) + j % 4 of a lane are slots j of step s on
// both sides, whatever their order.
//
// A tile is worked on in one go - scores, weights, values - while the next one comes into the other stage of LDS; what a wavefront waits for, the others
// of its SIMD fill.  What did not shorten it (us at 16 images of 1024 tokens with heads of 72, and at 8192 tokens with a prefix and heads of 128): a loop that
// multiplies the scores of the next tile and the values of the last one between the exponentials of this one, 150 and 343 against 137 and 340; 64 rows a
// wavefront, which halves the LDS reads, 130 and 382 against 134 and 337; rows of 9 pieces without bank conflicts for heads of 72, 135 against
// 135.  The chip runs these two at 1.95 and 1.77 GHz, kernels that wait for memory at 2.45 and more.
#pragma once
#include "attention.h"

namespace ql {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void attn_lds;
typedef const __attribute__((address_space(1))) void attn_global;
typedef __attribute__((address_space(3))) s16x4 attn_lds_s4;

constexpr int ATT_KEYS = 64;   // keys of a tile
static_assert(ATT_KEYS == KV_GROUP, "a tile of the cache is one group");
constexpr float LOG2E = 1.4426950408889634f;

// a lane's value and that of lane ^ 32, which has the same row (the two results are taken out as whole words first: a bit cast of a vector
// element reads element 0)
struct Halves {
    float a, b;
};
__device__ __forceinline__ Halves both_halves(float x)
{
    const unsigned w = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const unsigned a = r[0], b = r[1];
    return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// cap * tanh(x / cap) from t = 2 log2(e) x / cap: cap - 2 cap / (1 + e^(2 x / cap)), absolute error about 1e-7 of the cap
__device__ __forceinline__ float capped(float t, float cap) { return __builtin_fmaf(-2.0f * cap, __builtin_amdgcn_rcpf(1.0f + exp2_fast(t)), cap); }

// four codes -> four binary16: the byte with its sign bit turned is code + 128; 0x6400 | byte is 1024 + byte in binary16
__device__ __forceinline__ void codes_f16(unsigned w, f16x2 &lo, f16x2 &hi)
{
    const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    const unsigned u = w ^ 0x80808080u;
    lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - bias;
    hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - bias;
}
__device__ __forceinline__ f16x8 codes_f16x8(unsigned w0, unsigned w1)
{
    f16x2 a, b, c, d;
    codes_f16(w0, a, b);
    codes_f16(w1, c, d);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ unsigned absmax_bits(_Float16 x) { return (unsigned)__builtin_bit_cast(unsigned short, x) & 0x7fffu; }

// CHP: 16-byte pieces of a tile row, an even number.  Rows are kept without padding (a wavefront's DMA fills 1024 neighbouring bytes); the piece c of row r sits
// at slot c ^ f(r).  LDS serves 256 bytes at a time: the 16 lanes of a key read (16 rows, one piece each) lie in different sixteenths of them, the 32
// of a transposing value read (4 rows, 4 neighbouring pieces each) where a row is a multiple of 4 pieces.  (With 8 places for the 16 rows of
// heads of 128, a third of the LDS cycles were conflicts; the time at 8192 tokens did not change, 351 against 355 us.)
template <int CHP> __device__ __forceinline__ constexpr int key_swizzle(int r)
{
    return CHP % 16 == 0 ? (r & 15) : CHP % 16 == 8 ? (r >> 1 & 7) : CHP % 4 == 0 ? (r >> 2 & 3) : CHP > 2 ? (r >> 3 & 1) : 0;
}
template <int CHP> __device__ __forceinline__ constexpr int value_swizzle(int r)
{
    return CHP % 16 == 0 ? (r & 3) << 2 : CHP % 16 == 8 ? (r >> 1 & 1) << 2 : 0;
}

struct TilePlan {
    int tiles;     // row tiles of the launch: a bound with cu_q
    int per_seq;   // row tiles of a sequence without cu_q
    int splits;    // parts that the keys are cut into
    int mix;       // workgroups go through all heads tile by tile, the last rows first (else head by head on one XCD)
};

// The largest weight is 2^HEADROOM when the sums are brought to a new maximum, and 2^(HEADROOM + GROWTH) before the next time: inside binary16, and most
// tiles skip the scaling.  Binary16 rounds what is below 2^-14 in steps of 2^-24, so far weights are off by at most 2^-25-HEADROOM of the largest one: without the
// headroom 131071 keys that lie 17 nats below a single one were all 0, an error of 7 x 2^-11 of their values.
constexpr float HEADROOM = 7.0f, HEAD = 128.0f, GROWTH = 7.0f;   // HEAD = 2^HEADROOM
// Maxima (in powers of two) beyond which the weights' exponents are taken in two steps, rounded scores less the maximum: one fma has the exact product, whose
// distance from the rounded maximum grows to half a step of it - 16 at 2^28, where a weight would pass binary16 or all of them be 0 - and its addend,
// shift - maximum, is rounded to half a step too, 2^-15 here.
constexpr float EXACT_SCORES = 1024.0f;
constexpr float LEAST_SCALE = 1e-30f;   // stands for a scale of 0, so that -inf times it stays -inf
constexpr float LEAST_RATIO = -41.0f;   // log2 of the smallest value scale that counts beside the largest: below, a weight of 2^15 is 0 in binary16
// Value scales up to here: 127 of them are 0 in binary16, and so is the result.  Their reciprocal, and its product with a hidden token's scale, could pass fp32.
constexpr float LEAST_UNIT = 0x1p-60f;

// CHP: pieces of a tile row; NW: wavefronts; CACHE: keys and values from the 8-bit cache; SHAPED: scores may be capped or biased
template <int CHP_, int NW, bool CACHE>
struct AttnTile {
    static_assert(CHP_ % 2 == 0, "whole steps of 16 channels");
    static constexpr int CHP = CHP_, KS = CHP / 2, DT = (CHP + 3) / 4, ROWS = 32 * NW, NT = 64 * NW;
    static constexpr int K_BYTES = ATT_KEYS * CHP * 16;
    // values: rows like the keys' (a read of channels behind D may pass the last row: 1024 bytes behind the last stage), or transposed codes
    static constexpr int V_BYTES = CACHE ? DT * 32 * 128 : K_BYTES;
    static constexpr int V_AT = 2 * K_BYTES, SCALES_AT = V_AT + 2 * V_BYTES;
    static constexpr int LDS_BYTES = SCALES_AT + (CACHE ? 4 * ATT_KEYS * 4 : 1024);   // scales of both stages, or the slack
    // CACHE: register-staged pieces of a thread: 8 key codes each; 32 value codes of a channel each
    static constexpr int NKP = CACHE ? (ATT_KEYS * CHP + NT - 1) / NT : 1, NVP = CACHE ? (64 * DT + NT - 1) / NT : 1;
};

template <int CHP, int NW, bool CACHE, bool SHAPED>
__device__ __forceinline__ void attend_tile(const AttnArgs &a, const TilePlan &plan)
{
    using T = AttnTile<CHP, NW, CACHE>;
    constexpr int KS = T::KS, DT = T::DT;
    constexpr int NI = (CHP + NW - 1) / NW;            // DMA instructions of a wavefront for one tile
    extern __shared__ __align__(1024) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5;

    const int wgs = plan.tiles * a.Hkv * plan.splits;
    int id = blockIdx.x;
    if (!plan.mix) {
        const int per_xcd = (gridDim.x + 7) / 8;
        id = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    }
    if (id >= wgs) return;
    const int split = id % plan.splits;
    id /= plan.splits;
    int tile, hk, b, flat;                             // flat: number of the row tile in the launch
    if (a.cu_q) {
        flat = plan.mix ? plan.tiles - 1 - id / a.Hkv : id % plan.tiles;
        hk = plan.mix ? id % a.Hkv : id / plan.tiles;
        tile = flat;
        b = find_sequence(a.B, tile, [&](int s) { return (seq_rows(a.cu_q, s, a.Tq, a.B).n * a.G + T::ROWS - 1) / T::ROWS; });
        if (b < 0) return;
    } else {
        const int heads = a.Hkv * a.B, bh = plan.mix ? id % heads : id / plan.per_seq;
        tile = plan.mix ? plan.per_seq - 1 - id / heads : id % plan.per_seq;
        hk = bh % a.Hkv;
        b = bh / a.Hkv;
        flat = b * plan.per_seq + tile;
    }
    const SeqRows sq = seq_rows(a.cu_q, b, a.Tq, a.B);
    const SeqRows sk = CACHE ? SeqRows{0, min(max(a.len_k[b], 0), a.max_pages * a.page)} : seq_rows(a.cu_k, b, a.Tk, a.B);
    const int rows = sq.n * a.G;
    const int wrow = tile * T::ROWS + wave * 32 + (lane & 31);   // packed row of this lane
    const int row = min(wrow, rows - 1);
    const int token = row / a.G, head = hk * a.G + row % a.G;
    const int pos = token + sk.n - sq.n;
    const int prefix = a.prefix ? a.prefix[b] : 0;
    const int end = visible_end(a.mask, prefix, pos, sk.n);
    const int last_token = (min(tile * T::ROWS + T::ROWS, rows) - 1) / a.G;
    const int end_all = visible_end(a.mask, prefix, last_token + sk.n - sq.n, sk.n);   // what the workgroup reads
    const int wrow0 = min(tile * T::ROWS + wave * 32, rows - 1), wrow1 = min(tile * T::ROWS + wave * 32 + 31, rows - 1);
    // of this wavefront's rows: the fewest and the most keys (visible_end grows with the row)
    const int end_min = __builtin_amdgcn_readfirstlane(visible_end(a.mask, prefix, wrow0 / a.G + sk.n - sq.n, sk.n));
    const int end_max = tile * T::ROWS + wave * 32 < rows ? __builtin_amdgcn_readfirstlane(visible_end(a.mask, prefix, wrow1 / a.G + sk.n - sq.n, sk.n)) : 0;

    const int key_tiles = (end_all + ATT_KEYS - 1) / ATT_KEYS;
    const int share = (key_tiles + plan.splits - 1) / plan.splits;
    const int t0 = min(split * share, key_tiles), t1 = min(t0 + share, key_tiles);
    const int tw = min((end_max + ATT_KEYS - 1) / ATT_KEYS, t1);   // this wavefront's tiles end here

    // queries stay in registers: channels 16 ks + 8 half .. + 7 of the lane's row, zeros behind D
    const int CH = a.D / 8;
    const unsigned negative = a.scale < 0.0f ? 0x80008000u : 0u;   // scores are |scale| * (-q).k
    f16x8 qf[KS];
    {
        const _Float16 *q = static_cast<const _Float16 *>(a.q) + (sq.first + token) * a.q_row + head * a.q_head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int c = 2 * ks + half;
            uint4 w = make_uint4(0, 0, 0, 0);
            if (c < CH) w = *reinterpret_cast<const uint4 *>(q + 8 * c);
            w.x ^= negative;
            w.y ^= negative;
            w.z ^= negative;
            w.w ^= negative;
            qf[ks] = __builtin_bit_cast(f16x8, w);
        }
    }
    const float scale2 = fmaxf(fabsf(a.scale) * LOG2E, LEAST_SCALE);   // scores in powers of two
    const float slope2 = a.slopes ? a.slopes[head] * LOG2E : 0.0f;
    const float cap2 = a.cap * LOG2E, cap_in = a.cap > 0.0f ? 2.0f * LOG2E / cap2 : 0.0f;

    const unsigned lds0 = (unsigned)(uintptr_t)(attn_lds *)smem;
    // ---- tiles into LDS ------------------------------------------------------------------------------------------------------------
    // rows: instruction i of this wavefront fills pieces [64 (i NW + wave), + 64) of the tile; a row behind the last key reads the last
    // one, a piece behind D the row's last one: what is read there meets weights or queries that are zero
    const unsigned char *kb = static_cast<const unsigned char *>(a.k) + 2 * (sk.first * a.k_row + hk * a.k_head);
    const unsigned char *vb = static_cast<const unsigned char *>(a.v) + 2 * (sk.first * a.v_row + hk * a.v_head);
    unsigned koff[NI], voff[NI];                       // of this lane's piece from the tile's first row
    auto piece_at = [&](int i, bool value, int last_row, unsigned row_bytes) {
        const int ci = 64 * (i * NW + wave) + lane, r = ci / CHP, c = ci % CHP;
        return min(r, last_row) * row_bytes + 16 * min(c ^ (value ? value_swizzle<CHP>(r) : key_swizzle<CHP>(r)), CH - 1);
    };
    const unsigned krow = 2 * (unsigned)a.k_row, vrow = 2 * (unsigned)a.v_row;
    if constexpr (!CACHE) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            koff[i] = piece_at(i, false, ATT_KEYS, krow);
            voff[i] = piece_at(i, true, ATT_KEYS, vrow);
        }
    }
    auto dma = [&](bool value, int t, int stage) {
        const int left = sk.n - t * ATT_KEYS - 1;      // rows behind the tile's first one
        const unsigned char *from = value ? vb + (size_t)t * ATT_KEYS * 2 * a.v_row : kb + (size_t)t * ATT_KEYS * 2 * a.k_row;
        const unsigned to = value ? T::V_AT + stage * T::V_BYTES : stage * T::K_BYTES;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            if (CHP % NW != 0 && i * NW + wave >= CHP) break;   // (a tile is CHP times 64 pieces)
            unsigned at = value ? voff[i] : koff[i];
            if (left < ATT_KEYS - 1) at = piece_at(i, value, left, value ? vrow : krow);
            __builtin_amdgcn_global_load_lds((attn_global *)(from + at), (attn_lds *)(smem + to + (i * NW + wave) * 1024), 16, 0, 0);
        }
    };
    // cache: codes through registers; a page that is none reads page 0 and counts as masked
    uint2 kreg[T::NKP];
    uint4 vreg[T::NVP][2];
    float kscale_reg = 0.0f, vscale_reg = 0.0f;
    float *lds_ks = reinterpret_cast<float *>(smem + T::SCALES_AT), *lds_vs = lds_ks + 2 * ATT_KEYS;   // [stage][token]
    struct Where {
        size_t at;      // token of the cache where the tile begins, counted within its key head: (page * Hkv + hk) * page_tokens + in_page
        bool held;
    };
    int pages = 0;                                     // of 64 tiles from tile pages_at on, one per lane
    int pages_at = -ATT_KEYS;
    unsigned held_tiles = 0;                           // bit: whether the keys' stage has a page
    auto where = [&](int t) {
        if (t - pages_at >= 64) {
            pages_at = t;
            const int mine = pages_at + lane;
            pages = mine < t1 ? a.page_table[(size_t)b * a.max_pages + (unsigned)(mine * ATT_KEYS) / (unsigned)a.page] : -1;
        }
        int page = __builtin_amdgcn_readlane(pages, t - pages_at);
        const bool held = page >= 0 && page < a.num_pages;
        if (!held) page = 0;
        return Where{((size_t)page * a.Hkv + hk) * a.page + (unsigned)(t * ATT_KEYS) % (unsigned)a.page, held};
    };
    auto request = [&](int t) {
        const Where w = where(t);
        const unsigned bit = 1u << ((t - t0) & 1);
        held_tiles = w.held ? held_tiles | bit : held_tiles & ~bit;
        const unsigned char *kfrom = reinterpret_cast<const unsigned char *>(a.kc) + w.at * a.D, *vfrom = reinterpret_cast<const unsigned char *>(a.vc) + w.at * a.D;
#pragma unroll
        for (int i = 0; i < T::NKP; ++i) kreg[i] = *reinterpret_cast<const uint2 *>(kfrom + 8u * min((int)threadIdx.x + i * T::NT, ATT_KEYS * CH - 1));
#pragma unroll
        for (int i = 0; i < T::NVP; ++i) {
            const unsigned e = min((int)threadIdx.x + i * T::NT, 2 * a.D - 1);
            vreg[i][0] = *reinterpret_cast<const uint4 *>(vfrom + (e / 2 * 64 + e % 2 * 16));
            vreg[i][1] = *reinterpret_cast<const uint4 *>(vfrom + (e / 2 * 64 + e % 2 * 16 + 32));
        }
        if (threadIdx.x < ATT_KEYS) {
            // pages and groups begin at whole blocks; of blocks behind the end a scale may hold anything
            const unsigned in_tile = threadIdx.x / (unsigned)a.scale_tokens;
            const size_t block = w.at / ATT_KEYS * (unsigned)(ATT_KEYS / a.scale_tokens) + in_tile;
            const bool there = w.held && t * ATT_KEYS + (int)in_tile * a.scale_tokens < sk.n;
            kscale_reg = there ? a.ks[block] : 0.0f;
            vscale_reg = there ? a.vs[block] : 0.0f;
        }
    };
    unsigned kput[T::NKP];                             // where this thread's key pieces go
    if constexpr (CACHE) {
#pragma unroll
        for (int i = 0; i < T::NKP; ++i) {
            const int e = min((int)threadIdx.x + i * T::NT, ATT_KEYS * CH - 1), r = e / CH, cc = e % CH;
            kput[i] = r * (CHP * 16) + 16 * (cc ^ key_swizzle<CHP>(r));
        }
    }
    auto put_keys = [&](int stage) {
        // threads behind the last piece have the last piece too: they write the same bytes
#pragma unroll
        for (int i = 0; i < T::NKP; ++i) *reinterpret_cast<f16x8 *>(smem + stage * T::K_BYTES + kput[i]) = codes_f16x8(kreg[i].x, kreg[i].y);
        if (threadIdx.x < ATT_KEYS) {
            lds_ks[stage * ATT_KEYS + threadIdx.x] = kscale_reg;
            lds_vs[stage * ATT_KEYS + threadIdx.x] = vscale_reg;
        }
    };
    auto put_values = [&](int stage) {
        // channel d: 16-byte piece 2 s + half of its row has the slots of step s
#pragma unroll
        for (int i = 0; i < T::NVP; ++i) {
            const int e = threadIdx.x + i * T::NT;
            if (e >= 2 * a.D) break;
            const int d = e / 2, h = e % 2;
            unsigned char *to = smem + T::V_AT + stage * T::V_BYTES + d * 128;
            const unsigned x[4] = {vreg[i][0].x, vreg[i][0].y, vreg[i][0].z, vreg[i][0].w}, y[4] = {vreg[i][1].x, vreg[i][1].y, vreg[i][1].z, vreg[i][1].w};
#pragma unroll
            for (int s = 0; s < 4; ++s) *reinterpret_cast<f16x8 *>(to + 16 * ((2 * s + h) ^ (d >> 1 & 7))) = codes_f16x8(x[s], y[s]);
        }
    };

    f32x16 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f32x16{};
    float m = -__builtin_inff(), l = 0.0f;             // of this lane's row, m in powers of two; l over this lane's keys only
    bool far = false;                                  // of the wavefront's rows: some maximum lies beyond EXACT_SCORES
    float unit_v = 0.0f;                               // CACHE: the value scale that the row's sums are in

    // left operands: step ks of keys 32 u .. 32 u + 31, step st of value channels 32 d .. 32 d + 31.  A swizzle turns the low bits of a piece's
    // number, so pieces that differ above them lie a constant apart: few addresses are kept, the rest is in the instructions.
    constexpr int KA = CHP % 16 == 0 ? 8 : CHP % 8 == 0 ? 4 : CHP % 4 == 0 ? 2 : 1;
    constexpr int VA = CACHE ? 4 : CHP % 16 == 0 ? 4 : CHP % 16 == 8 ? 2 : 1;
    unsigned kaddr[KA], vaddr[VA];
#pragma unroll
    for (int i = 0; i < KA; ++i) kaddr[i] = lds0 + (lane & 31) * (CHP * 16) + 16 * ((2 * i + half) ^ key_swizzle<CHP>(lane & 31));
#pragma unroll
    for (int i = 0; i < VA; ++i) {
        // CACHE: transposed, channel lane & 31, step i.  Rows: the transposing read takes 4 keys of 16 channels for 16 lanes, lane i of them with the
        // address of key i / 4, channels 4 (i % 4)
        const int r = 4 * half + (lane >> 2 & 3), ch = 4 * i + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
        vaddr[i] = lds0 + T::V_AT + (CACHE ? (lane & 31) * 128 + 16 * ((2 * i + half) ^ (lane >> 1 & 7)) : r * (CHP * 16) + 16 * (ch ^ value_swizzle<CHP>(r)) + 8 * (lane & 1));
    }
    auto key_part = [&](int stage, int u, int ks) {
        typedef __attribute__((address_space(3))) f16x8 lds_h8;
        return *(lds_h8 *)(uintptr_t)(kaddr[ks % KA] + (unsigned)(stage * T::K_BYTES + u * 32 * CHP * 16 + (ks / KA) * KA * 32));
    };
    auto value_part = [&](int stage, int d, int st) -> f16x8 {
        if constexpr (CACHE) {
            typedef __attribute__((address_space(3))) f16x8 lds_h8;
            return *(lds_h8 *)(uintptr_t)(vaddr[st] + (unsigned)(stage * T::V_BYTES + d * 4096));
        } else {
            const unsigned at = vaddr[d % VA] + (unsigned)(stage * T::V_BYTES + st * 16 * CHP * 16 + (d / VA) * VA * 64);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((attn_lds_s4 *)(uintptr_t)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((attn_lds_s4 *)(uintptr_t)(at + 8 * CHP * 16));
            const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(f16x8, both);
        }
    };
    // what turns scores into powers of two: returns the factor that is left
    const bool one_scale = CACHE && a.scale_tokens == ATT_KEYS;
    auto shape = [&](f32x16 (&s)[2], int t, int stage) -> float {
        const int j0 = t * ATT_KEYS;
        float c = scale2;
        bool held = true;
        if constexpr (CACHE) {
            if (one_scale) {
                const float k = lds_ks[stage * ATT_KEYS];
                c = fmaxf(scale2 * k, LEAST_SCALE);
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4 k = *reinterpret_cast<const f32x4 *>(lds_ks + stage * ATT_KEYS + 32 * u + 8 * g + 4 * half);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[u][4 * g + e] *= k[e];
                    }
            }
            held = held_tiles >> stage & 1;
        }
        if (SHAPED && a.cap > 0.0f) {
            const float k = c * cap_in;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = capped(s[u][r] * k, cap2);
            c = 1.0f;
        }
        if (SHAPED && a.slopes) {
            // distances are whole numbers: exact up to 2^24
            const float far = (float)(pos - j0 - 4 * half);
            if (c != 1.0f)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[u][r] *= c;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = __builtin_fmaf(fabsf(far - (float)(32 * u + 8 * (r / 4) + r % 4)), -slope2, s[u][r]);
            c = 1.0f;
        }
        if (j0 + ATT_KEYS > end_min || !held) {
            const int lim = held ? end - j0 - 4 * half : -ATT_KEYS;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = 32 * u + 8 * (r / 4) + r % 4 < lim ? s[u][r] : -__builtin_inff();
        }
        return c;
    };
    auto largest = [&](const f32x16 (&s)[2]) {
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[u][r]);
        return top;
    };

    if constexpr (CACHE) {
        // pieces behind D meet zero queries: they have to be finite
        if (CH < CHP)
            for (int e = threadIdx.x; e < 2 * ATT_KEYS * (CHP - CH); e += T::NT) {
                const int r = e / (CHP - CH) % ATT_KEYS, c = CH + e % (CHP - CH), stage = e / (CHP - CH) / ATT_KEYS;
                *reinterpret_cast<f16x8 *>(smem + stage * T::K_BYTES + r * (CHP * 16) + 16 * (c ^ key_swizzle<CHP>(r))) = f16x8{};
            }
    }
    auto work = [&](int t, int stage) __attribute__((always_inline)) {
        // scores: register r of s[u] is key 32 u + 8 (r / 4) + 4 half + r % 4 of the tile
        f32x16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key_part(stage, u, ks), qf[ks], ks ? s[u] : f32x16{}, 0, 0, 0);
        float c = shape(s, t, stage);
        // the running maximum, and the value scale that the sums are in
        const Halves tops = both_halves(largest(s));
        const float top = fmaxf(tops.a, tops.b) * c;
        float shift = HEADROOM, grow = 1.0f, per = 0.0f;
        if constexpr (CACHE) {
            // the tile's largest value scale of those that the row sees, by the running maximum over the tokens: the weights are rounded relative to it
            const int seen = min(end - t * ATT_KEYS, ATT_KEYS);
            float big = lds_vs[stage * ATT_KEYS + (one_scale ? 0 : lane)];
            if (!one_scale) {
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const float before = __shfl_up(big, d, 64);
                    big = lane >= d ? fmaxf(big, before) : big;
                }
                big = __shfl(big, max(seen, 1) - 1, 64);
            }
            big = seen > 0 ? big : 0.0f;
            if (big > unit_v) {
                grow = unit_v / big;
                unit_v = big;
            }
            per = unit_v > LEAST_UNIT ? 1.0f / unit_v : 0.0f;
            // the headroom is in the exponent, or, where the weights are multiplied by their scales, in that factor
            if (one_scale) {
                shift += fmaxf(__builtin_amdgcn_logf(big * per), LEAST_RATIO);   // (a row that sees nothing of the tile: any)
            } else {
                shift = 0.0f;
                per *= HEAD;
            }
        }
        if (__any(top - m > GROWTH || (m == -__builtin_inff() && top > m)) || (CACHE && __any(grow != 1.0f))) {
            const float m2 = fmaxf(m, top);
            const float keep = m == -__builtin_inff() ? 0.0f : exp2_fast(m - m2);
            l *= keep;
            m = m2;
            far = __any(fabsf(m) > EXACT_SCORES && m > -__builtin_inff());
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[d][r] *= keep * grow;
        }
        const float m0 = m == -__builtin_inff() ? 0.0f : m;
        float mc = shift - m0;
        if (far) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = s[u][r] * c - m0;
            c = 1.0f;
            mc = shift;
        }
        f16x8 p[4];                                    // weights, as steps of 16 keys
        float sum = 0.0f;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const int u = x / 8, r = 2 * (x % 8), g = x / 4, e = 2 * (x % 4);   // scores s[u][r], s[u][r + 1]; slots e, e + 1 of step g
            float w0 = exp2_fast(__builtin_fmaf(s[u][r], c, mc)), w1 = exp2_fast(__builtin_fmaf(s[u][r + 1], c, mc));
            if constexpr (CACHE) {
                sum += w0 + w1;
                if (!one_scale) {
                    const float2 v = *reinterpret_cast<const float2 *>(lds_vs + stage * ATT_KEYS + 16 * g + (e < 4 ? e : e + 4) + 4 * half);
                    w0 *= v.x * per;
                    w1 *= v.y * per;
                }
            }
            const f16x2 h = {(_Float16)w0, (_Float16)w1};
            // the sum takes the weights as they are multiplied, unless they carry a value scale
            if constexpr (!CACHE) sum = __builtin_amdgcn_fdot2(h, f16x2{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
            p[g][e] = h[0];
            p[g][e + 1] = h[1];
        }
        if (CACHE && one_scale) sum *= exp2_fast(-shift);
        l += sum;
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value_part(stage, d, st), p[st], acc[d], 0, 0, 0);
    };
    if (t0 < t1) {
        if constexpr (CACHE) {
            request(t0);
            put_keys(0);
            put_values(0);
        } else {
            dma(false, t0, 0);
            dma(true, t0, 0);
        }
        auto turn = [&](int t, int stage) __attribute__((always_inline)) {
            // tile t is there, and what tile t - 1 had is read by all
            if constexpr (!CACHE) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (t + 1 < t1) {
                if constexpr (CACHE) {
                    request(t + 1);
                } else {
                    dma(false, t + 1, stage ^ 1);
                    dma(true, t + 1, stage ^ 1);
                }
            }
            if (t < tw) work(t, stage);
            if constexpr (CACHE) {
                if (t + 1 < t1) {
                    put_keys(stage ^ 1);
                    put_values(stage ^ 1);
                }
            }
        };
        for (int t = t0; t < t1; t += 2) {
            turn(t, 0);
            if (t + 1 < t1) turn(t + 1, 1);
        }
    }
    const Halves ls = both_halves(l);
    l = ls.a + ls.b;
    if (plan.splits > 1) {
        // [ROWS][D] sums, then maxima (in powers of two) and weights of this part (rows: sums and weights 2^HEADROOM times as large, in all parts)
        float *part = a.partial + (((size_t)flat * a.Hkv + hk) * plan.splits + split) * (size_t)(T::ROWS * (a.D + 2));
        const int lr = wave * 32 + (lane & 31);
        const float back = CACHE ? unit_v / HEAD : 1.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int ch = 32 * d + 8 * g + 4 * half;
                if (ch < a.D) *reinterpret_cast<f32x4 *>(part + (size_t)lr * a.D + ch) = f32x4{acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]} * back;
            }
        if (half == 0) {
            part[(size_t)T::ROWS * a.D + lr] = m;
            part[(size_t)T::ROWS * (a.D + 1) + lr] = l;
        }
        return;
    }
    const float inv = l > 0.0f ? (CACHE ? unit_v / HEAD : 1.0f) / l : 0.0f;   // (rows: the sum has the headroom too)
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

// Adds up the parts of the row tiles: a thread has four channels of a packed row and takes four parts at a time, maxima, weights and sums requested
// together.  blockIdx.x: row tile and key head; blockIdx.y: the tile's next JOIN_THREADS / (D / 4) rows.
constexpr int JOIN_THREADS = 256;
__device__ __forceinline__ void join_splits(const AttnArgs &a, const TilePlan &plan, int rows_per)
{
    const int hk = blockIdx.x % a.Hkv, flat = blockIdx.x / a.Hkv;
    int tile = flat, b;
    if (a.cu_q) {
        b = find_sequence(a.B, tile, [&](int s) { return (seq_rows(a.cu_q, s, a.Tq, a.B).n * a.G + rows_per - 1) / rows_per; });
        if (b < 0) return;
    } else {
        b = flat / plan.per_seq;
        tile = flat % plan.per_seq;
    }
    const SeqRows sq = seq_rows(a.cu_q, b, a.Tq, a.B);
    const int fours = a.D / 4, at_once = JOIN_THREADS / fours, in = threadIdx.x / fours, ch = 4 * (threadIdx.x - in * fours);
    const int lr = at_once * blockIdx.y + in, row = tile * rows_per + lr;
    if (in >= at_once || lr >= rows_per || row >= sq.n * a.G) return;
    const size_t stride = (size_t)rows_per * (a.D + 2);
    const float *part = a.partial + ((size_t)flat * a.Hkv + hk) * plan.splits * stride;
    float m = -__builtin_inff(), weight = 0.0f;
    f32x4 sum = {};
    for (int first = 0; first < plan.splits; first += 4) {
        float pm[4], pl[4];
        f32x4 px[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float *x = part + min(first + i, plan.splits - 1) * stride;
            pm[i] = x[(size_t)rows_per * a.D + lr];
            pl[i] = x[(size_t)rows_per * (a.D + 1) + lr];
            px[i] = *reinterpret_cast<const f32x4 *>(x + (size_t)lr * a.D + ch);
        }
        float m2 = m;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (first + i < plan.splits) m2 = fmaxf(m2, pm[i]);
        if (m2 == -__builtin_inff()) continue;
        const float keep = exp2_fast(m - m2);
        weight *= keep;
        sum *= keep;
        m = m2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float k = first + i < plan.splits ? exp2_fast(pm[i] - m) : 0.0f;
            weight += k * pl[i];
            sum += px[i] * k;
        }
    }
    const int token = row / a.G, head = hk * a.G + row % a.G;
    const float inv = weight > 0.0f ? 1.0f / weight : 0.0f;
    f16x4 o;
    unsigned amax = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const _Float16 h = (_Float16)(sum[e] * inv);
        o[e] = h;
        amax = max(amax, absmax_bits(h));
    }
    *reinterpret_cast<f16x4 *>(static_cast<_Float16 *>(a.o) + (sq.first + token) * a.o_row + head * a.o_head + ch) = o;
    if (a.row_absmax) atomicMax(a.row_absmax + sq.first + token, amax);
}
inline unsigned join_blocks(int rows_per, int D) { return (unsigned)((rows_per + JOIN_THREADS / (D / 4) - 1) / (JOIN_THREADS / (D / 4))); }

// row tiles of `rows` packed rows, and the parts that the keys are cut into so that few of them still fill the chip: enough
// workgroups for two on every CU, no part below 4 key tiles
constexpr int TILE_SPLITS = 16;
inline TilePlan tile_plan(long long Tq, int B, int G, int Hkv, int rows, bool cu_q, int mask, long long keys, int least_wgs, int wanted_wgs)
{
    TilePlan p{};
    p.per_seq = (int)((Tq / B * G + rows - 1) / rows);
    p.tiles = cu_q ? (int)(Tq * G / rows + B) : p.per_seq * B;
    const long long bound = (Tq * G / rows + B) * Hkv;   // of the workgroups, with or without cu_q
    long long splits = bound >= least_wgs ? 1 : wanted_wgs / bound;
    const long long most = keys / (4 * ATT_KEYS);
    splits = splits > TILE_SPLITS ? TILE_SPLITS : splits;
    splits = splits > most ? most : splits;
    p.splits = splits < 1 ? 1 : (int)splits;
    p.mix = mask != 0;
    return p;
}
// parts of the cut calls among those of at most Tq rows, B sequences and so many keys: what their workspace has to hold
inline long long most_parts(long long Tq, int B, int G, int Hkv, int rows, long long keys, int wanted_wgs)
{
    long long splits = keys / (4 * ATT_KEYS);
    splits = splits > TILE_SPLITS ? TILE_SPLITS : splits;
    const long long parts = (Tq * G / rows + B) * Hkv * splits;
    return splits < 2 ? 0 : parts > wanted_wgs ? wanted_wgs : parts;
}

}  // namespace ql
