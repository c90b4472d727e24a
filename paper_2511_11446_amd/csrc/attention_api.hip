// Host side of the attention and 8-bit cache calls of include/diffpro_qlinear.h: argument checks (before the first HIP call), workspace, launches.
#include "../../include/diffpro_qlinear.h"
#include "attention.h"

#include <cmath>

namespace {

constexpr int64_t INT_MAX64 = 2147483647;

constexpr int64_t ROWS_MAX = 1 << 30, SEQUENCES_MAX = 1 << 20;
constexpr int64_t STRIDE_MAX = 1 << 24;   // elements between rows: 64 of them are addressed with 32 bits

inline bool off(const void *p, size_t a) { return p && (uintptr_t)p % a != 0; }

// a strided [T, H, D] tensor of binary16: strides in elements
int check_rows(const void *p, int64_t row, int64_t head)
{
    if (!p) return QL_ERR_NULL;
    if (row < 0 || head < 0 || row % 8 != 0 || head % 8 != 0 || row > STRIDE_MAX || head > INT_MAX64) return QL_ERR_SHAPE;
    return off(p, 16) ? QL_ERR_ALIGN : QL_OK;
}

int check_heads(int64_t T, int64_t B, int64_t H, int64_t D, bool equal)
{
    if (T < 1 || B < 1 || H < 1 || D < 8 || D > 256 || D % 8 != 0) return QL_ERR_SHAPE;
    // threads of a launch stay below 2^32: 256 for every 128 packed rows, and for every sequence and key head
    if (T > ROWS_MAX / H || B > SEQUENCES_MAX / H || (equal && T % B != 0)) return QL_ERR_SHAPE;
    return QL_OK;
}

int check_attention(const ql_attention *a)
{
    if (!a || !a->q || !a->o) return QL_ERR_NULL;
    if (a->mask < QL_MASK_NONE || a->mask > QL_MASK_PREFIX || a->reserved != 0) return QL_ERR_UNSUPPORTED;
    if (a->mask == QL_MASK_PREFIX && !a->prefix) return QL_ERR_NULL;
    if (!std::isfinite(a->scale)) return QL_ERR_UNSUPPORTED;
    // the capped score is off by about 2^-22 of the cap (attention_tile.h): beyond 2^10 that would be more than the rounding of the weights
    if (a->cap != 0.0f && !(a->cap >= 0x1p-10f && a->cap <= 0x1p10f)) return QL_ERR_UNSUPPORTED;
    int rc = check_heads(a->T_q, a->B, a->Hq, a->D, !a->cu_q);
    if (rc) return rc;
    if (a->Hkv < 1 || a->Hq % a->Hkv != 0) return QL_ERR_SHAPE;
    if ((rc = check_rows(a->q, a->q_row, a->q_head)) || (rc = check_rows(a->o, a->o_row, a->o_head))) return rc;
    // the outputs of different rows and heads lie apart: heads within rows, or rows within heads
    const bool heads_in = a->o_row >= (a->Hq - 1) * a->o_head + a->D || a->T_q == 1, rows_in = a->o_head >= (a->T_q - 1) * a->o_row + a->D || a->Hq == 1;
    const bool apart = (a->o_head >= a->D || a->Hq == 1) && (a->o_row >= a->D || a->T_q == 1);
    if (!apart || !(heads_in || rows_in)) return QL_ERR_SHAPE;
    if (off(a->prefix, 4) || off(a->slopes, 4) || off(a->cu_q, 4) || off(a->row_absmax, 4)) return QL_ERR_ALIGN;
    return QL_OK;
}

int check_cache(const ql_kv_cache *c)
{
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->page_table || !c->len_k) return QL_ERR_NULL;
    if (c->scale_tokens != 1 && c->scale_tokens != 16 && c->scale_tokens != 32 && c->scale_tokens != 64) return QL_ERR_UNSUPPORTED;
    if (c->page < 64 || c->page % 64 != 0 || c->num_pages < 1 || c->num_pages > INT_MAX64 || c->B < 1 || c->Hkv < 1 || c->max_pages < 1) return QL_ERR_SHAPE;
    if (c->D < 8 || c->D > 256 || c->D % 8 != 0 || c->max_pages > INT_MAX64 / c->page) return QL_ERR_SHAPE;
    if (off(c->k, 16) || off(c->v, 16) || off(c->k_scale, 4) || off(c->v_scale, 4) || off(c->page_table, 4) || off(c->len_k, 4)) return QL_ERR_ALIGN;
    return QL_OK;
}

int check_workspace(const void *ws, size_t have, size_t need)
{
    if (need == 0) return QL_OK;
    if (!ws || have < need) return QL_ERR_WORKSPACE;
    return off(ws, 256) ? QL_ERR_ALIGN : QL_OK;
}

ql::AttnArgs attention_args(const ql_attention *a)
{
    ql::AttnArgs g{};
    g.q = a->q;
    g.o = a->o;
    g.q_row = a->q_row;
    g.q_head = a->q_head;
    g.o_row = a->o_row;
    g.o_head = a->o_head;
    g.Tq = (int)a->T_q;
    g.B = a->B;
    g.Hq = a->Hq;
    g.Hkv = a->Hkv;
    g.D = a->D;
    g.G = a->Hq / a->Hkv;
    g.cu_q = static_cast<const int *>(a->cu_q);
    g.mask = a->mask;
    g.scale = a->scale;
    g.cap = a->cap;
    g.slopes = static_cast<const float *>(a->slopes);
    g.prefix = a->mask == QL_MASK_PREFIX ? static_cast<const int *>(a->prefix) : nullptr;
    g.row_absmax = static_cast<unsigned *>(a->row_absmax);
    return g;
}

int clear_absmax(const ql_attention *a, hipStream_t s)
{
    return a->row_absmax ? ql::status_of(ql::launch_fill_u32(static_cast<unsigned *>(a->row_absmax), (int)a->T_q, 0u, s)) : QL_OK;
}

}  // namespace

extern "C" {

size_t attention_f16_workspace_bytes(int64_t T_q, int64_t T_k, int32_t B, int32_t Hq, int32_t Hkv, int32_t D)
{
    if (check_heads(T_q, B, Hq, D, false) || Hkv < 1 || Hq % Hkv != 0 || check_heads(T_k, B, Hkv, D, false)) return 0;
    return ql::tiles_most_bytes(T_q, T_k, B, Hq, Hkv, D);
}

int attention_f16(const ql_attention *attn, const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row, int64_t v_head,
                  int64_t T_k, const void *cu_k, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_attention(attn);
    if (rc) return rc;
    if ((rc = check_heads(T_k, attn->B, attn->Hkv, attn->D, !cu_k))) return rc;
    if ((rc = check_rows(k, k_row, k_head)) || (rc = check_rows(v, v_row, v_head))) return rc;
    if (off(cu_k, 4)) return QL_ERR_ALIGN;
    if ((rc = check_workspace(workspace, workspace_bytes, ql::tiles_partial_bytes(attn->T_q, T_k, attn->B, attn->Hq, attn->Hkv, attn->D)))) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if ((rc = clear_absmax(attn, s))) return rc;
    ql::AttnArgs g = attention_args(attn);
    g.k = k;
    g.v = v;
    g.k_row = k_row;
    g.k_head = k_head;
    g.v_row = v_row;
    g.v_head = v_head;
    g.Tk = (int)T_k;
    g.cu_k = static_cast<const int *>(cu_k);
    g.partial = static_cast<float *>(workspace);
    return ql::status_of(ql::launch_attention_f16(g, s));
}

int daq_kv_append(const ql_kv_cache *cache, const ql_kv_new *n, void *stream)
{
    int rc = check_cache(cache);
    if (rc) return rc;
    if (!n || !n->k || !n->v || (n->q_out && !n->q)) return QL_ERR_NULL;
    if (n->reserved != 0 || (n->rot_pairs != 0 && n->rot_pairs != 1)) return QL_ERR_UNSUPPORTED;
    if ((rc = check_heads(n->T, cache->B, cache->Hkv, cache->D, !n->cu))) return rc;
    if ((rc = check_rows(n->k, n->k_row, n->k_head)) || (rc = check_rows(n->v, n->v_row, n->v_head))) return rc;
    if (n->q_out) {
        if (n->Hq < 1 || n->Hq % cache->Hkv != 0 || n->T > ROWS_MAX / n->Hq) return QL_ERR_SHAPE;
        if ((rc = check_rows(n->q, n->q_row, n->q_head))) return rc;
    }
    if (n->rot && (n->rot_dim < 16 || n->rot_dim % 16 != 0 || n->rot_dim > cache->D || n->rot_rows < 1 || n->rot_rows > INT_MAX64)) return QL_ERR_SHAPE;
    if (off(n->rot, 16) || off(n->q_out, 16) || off(n->k_out, 16) || off(n->v_out, 16) || off(n->cu, 4) || off(n->pos, 4)) return QL_ERR_ALIGN;
    // workgroups of the launch: groups of 64 tokens that new ones may touch, for every key head
    if ((n->T / 64 + 2LL * cache->B) > INT_MAX64 / 256 / cache->Hkv) return QL_ERR_SHAPE;
    ql::KvAppendArgs g{};
    g.kc = static_cast<int8_t *>(cache->k);
    g.vc = static_cast<int8_t *>(cache->v);
    g.ks = static_cast<float *>(cache->k_scale);
    g.vs = static_cast<float *>(cache->v_scale);
    g.page_table = static_cast<const int *>(cache->page_table);
    g.len_k = static_cast<const int *>(cache->len_k);
    g.num_pages = (int)cache->num_pages;
    g.page = cache->page;
    g.scale_tokens = cache->scale_tokens;
    g.max_pages = cache->max_pages;
    g.T = (int)n->T;
    g.B = cache->B;
    g.Hkv = cache->Hkv;
    g.D = cache->D;
    g.Hq = n->q_out ? n->Hq : 0;
    g.G = g.Hq / g.Hkv;
    g.cu = static_cast<const int *>(n->cu);
    g.q = n->q;
    g.k = n->k;
    g.v = n->v;
    g.q_row = n->q_row;
    g.q_head = n->q_head;
    g.k_row = n->k_row;
    g.k_head = n->k_head;
    g.v_row = n->v_row;
    g.v_head = n->v_head;
    g.rot = static_cast<const float *>(n->rot);
    g.rot_rows = (int)n->rot_rows;
    g.rot_dim = n->rot_dim;
    g.rot_pairs = n->rot_pairs;
    g.pos = static_cast<const int *>(n->pos);
    g.q_out = n->q_out;
    g.k_out = n->k_out;
    g.v_out = n->v_out;
    return ql::status_of(ql::launch_kv_append(g, static_cast<hipStream_t>(stream)));
}

size_t attention_kv8_workspace_bytes(int64_t T_q, int32_t B, int32_t Hq, int32_t Hkv, int32_t D)
{
    if (check_heads(T_q, B, Hq, D, false) || Hkv < 1 || Hq % Hkv != 0) return 0;
    return ql::cached_most_bytes(T_q, B, Hq, Hkv, D);
}

int attention_kv8(const ql_attention *attn, const ql_kv_cache *cache, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_attention(attn);
    if (rc) return rc;
    if ((rc = check_cache(cache))) return rc;
    if (attn->B != cache->B || attn->Hkv != cache->Hkv || attn->D != cache->D) return QL_ERR_SHAPE;
    // the kernels count groups of 64 tokens of 16 rows of a key head in 32 bits
    const int64_t row_tiles = (attn->T_q * (attn->Hq / attn->Hkv) / 16 + attn->B) * attn->Hkv, groups = (int64_t)cache->max_pages * (cache->page / 64);
    if (row_tiles > INT_MAX64 / groups) return QL_ERR_SHAPE;
    if ((rc = check_workspace(workspace, workspace_bytes, ql::cached_partial_bytes(attn->T_q, attn->B, attn->Hq, attn->Hkv, attn->D)))) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if ((rc = clear_absmax(attn, s))) return rc;
    ql::AttnArgs g = attention_args(attn);
    g.kc = static_cast<const int8_t *>(cache->k);
    g.vc = static_cast<const int8_t *>(cache->v);
    g.ks = static_cast<const float *>(cache->k_scale);
    g.vs = static_cast<const float *>(cache->v_scale);
    g.page_table = static_cast<const int *>(cache->page_table);
    g.len_k = static_cast<const int *>(cache->len_k);
    g.num_pages = (int)cache->num_pages;
    g.page = cache->page;
    g.scale_tokens = cache->scale_tokens;
    g.max_pages = cache->max_pages;
    g.partial = static_cast<float *>(workspace);
    return ql::status_of(ql::launch_attention_kv8(g, s));
}

}  // extern "C"
