// Attention between the qkv layer and the output projection, and the paged 8-bit cache of keys and values (internal).
// Not part of the public ABI.
//
//   x = scale * q.k,  c = cap * tanh(x / cap) (x without a cap),  s = c - slope_h * |p - j|
//   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m) over the visible keys j of the row's sequence, 0 where there are none
// Row i of a sequence with n_q rows and n_k keys stands at position p = i + n_k - n_q.  Query head h reads key head h / (Hq / Hkv);
// the G = Hq / Hkv heads that share one are handled as G rows per token ("packed rows": row r = token r / G, head r % G), so that keys
// and values are read once for all of them.
#pragma once
#include "ql_internal.h"

namespace ql {

// tokens whose value codes the cache keeps together, [D][64] bytes
constexpr int KV_GROUP = 64;
// where token t (0..63) of a group keeps its value codes: a lane of the 16-wide matrix instruction that has tokens 4 g .. 4 g + 3 of
// each of the group's four 16-token tiles finds them in 16 neighbouring bytes
__host__ __device__ constexpr int kv_slot(int t) { return 16 * (t % 16 / 4) + 4 * (t / 16) + t % 4; }

struct AttnArgs {
    const void *q;            // binary16, element (t, h, d) at t * q_row + h * q_head + d
    void *o;
    long long q_row, q_head, o_row, o_head;
    int Tq, B, Hq, Hkv, D, G; // G = Hq / Hkv
    const int *cu_q;          // [B+1] first row of every sequence, or null: Tq / B rows each
    int mask;                 // QL_MASK_*
    float scale, cap;
    const float *slopes;      // [Hq] or null
    const int *prefix;        // [B], QL_MASK_PREFIX only
    unsigned *row_absmax;     // [Tq] or null (cleared by the caller of the launch)
    // attention_f16
    const void *k, *v;        // binary16, element (t, h, d) at t * k_row + h * k_head + d
    long long k_row, k_head, v_row, v_head;
    int Tk;
    const int *cu_k;          // [B+1] or null: Tk / B keys each
    // attention_kv8
    const int8_t *kc, *vc;    // [pages, Hkv, page, D] and [pages, Hkv, page / 64, D, 64]
    const float *ks, *vs;     // [pages, Hkv, page / scale_tokens]
    const int *page_table;    // [B, max_pages]
    const int *len_k;         // [B]
    int num_pages, page, scale_tokens, max_pages;
    // workspace
    float *partial;
};

hipError_t launch_attention_f16(const AttnArgs &a, hipStream_t stream);
hipError_t launch_attention_kv8(const AttnArgs &a, hipStream_t stream);
hipError_t launch_attention_chunks(const AttnArgs &a, hipStream_t stream);
// workspace of the launches (fewer rows may need more: their keys are cut), and the most that a call of no more rows, keys and sequences needs
size_t tiles_partial_bytes(long long Tq, long long Tk, int B, int Hq, int Hkv, int D);
size_t tiles_most_bytes(long long Tq, long long Tk, int B, int Hq, int Hkv, int D);
size_t chunks_partial_bytes(long long Tq, int B, int Hq, int Hkv, int D);
size_t chunks_most_bytes(long long Tq, int B, int Hq, int Hkv, int D);
size_t cached_partial_bytes(long long Tq, int B, int Hq, int Hkv, int D);   // either
size_t cached_most_bytes(long long Tq, int B, int Hq, int Hkv, int D);

struct KvAppendArgs {
    int8_t *kc, *vc;
    float *ks, *vs;
    const int *page_table, *len_k;
    int num_pages, page, scale_tokens, max_pages;
    int T, B, Hq, Hkv, D, G;  // Hq = 0: no queries
    const int *cu;            // [B+1] or null: T / B new tokens each
    const void *q, *k, *v;    // binary16, strided as in AttnArgs
    long long q_row, q_head, k_row, k_head, v_row, v_head;
    const float *rot;         // [rot_rows, rot_dim / 2, 2] cos, sin or null
    int rot_rows, rot_dim, rot_pairs; // pairs: channels 2 i and 2 i + 1 turn together, else i and i + rot_dim / 2
    const int *pos;           // [T] row of rot for every new token, or null: its place in the sequence
    void *q_out, *k_out, *v_out; // binary16 [T, H, D] or null
};

hipError_t launch_kv_append(const KvAppendArgs &a, hipStream_t stream);

#ifdef __HIPCC__
// rows [first, first + n) of sequence b of T packed rows; what a cu array says beyond the tensor is cut off
struct SeqRows {
    int first, n;
};
__device__ __forceinline__ SeqRows seq_rows(const int *cu, int b, int T, int B)
{
    if (!cu) {
        const int n = T / B;
        return {b * n, n};
    }
    const int lo = min(max(cu[b], 0), T), hi = min(max(cu[b + 1], lo), T);
    return {lo, hi - lo};
}

// Item `item` of a list that has count(b) items of every sequence b one behind the other: its sequence (-1: behind the last) and its number
// there.  64 sequences at a time, one per lane; the result is the same in all lanes.
template <class CountFn>
__device__ __forceinline__ int find_sequence(int B, int &item, CountFn count)
{
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < B; base += 64) {
        const int mine = base + lane < B ? count(base + lane) : 0;
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d, 64);
            if (lane >= d) upto += o;
        }
        const unsigned long long behind = __ballot(upto > item);
        if (behind) {
            const int l = __ffsll((unsigned long long)behind) - 1;
            item = __builtin_amdgcn_readfirstlane(item - __shfl(upto - mine, l, 64));
            return __builtin_amdgcn_readfirstlane(base + l);
        }
        item = __builtin_amdgcn_readfirstlane(item - __shfl(upto, 63, 64));
    }
    return -1;
}

// keys that row position p sees: [0, n_k) cut by the mask; those below the prefix always
__device__ __forceinline__ int visible_end(int mask, int prefix, int p, int n_k)
{
    if (mask == 0) return n_k;
    const int own = max(p + 1, mask == 2 ? prefix : 0);
    return min(max(own, 0), n_k);
}
#endif

}  // namespace ql
