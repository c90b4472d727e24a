// Host side of the 8-bit floating point, routing and experts' calls of include/diffpro_qlinear.h: argument checks (before the first HIP call), workspace, launches.
#include "../../include/diffpro_qlinear.h"
#include "f8.h"

#include <algorithm>
#include <cmath>

namespace {

constexpr int64_t ELEMS_MAX = 2147483647;   // int32 indexing inside the kernels
constexpr int64_t EXPERTS_MAX = 512, CHOICES_MAX = 64, GROUPS_MAX = 128, EXPERT_ROWS_MAX = 1 << 24;

inline bool off(const void *p, size_t a) { return p && (uintptr_t)p % a != 0; }
inline size_t align_up(size_t v) { return (v + 255) / 256 * 256; }
inline bool over(int64_t a, int64_t b) { return a > ELEMS_MAX / b; }

int check_layer(int64_t M, int64_t K, int64_t N, int32_t glu)
{
    if (M < 1 || K < 1 || N < 1 || K % 16 != 0) return QL_ERR_SHAPE;
    if (over(M, K) || over(M, N) || over(N, K) || (glu && over(M, 2 * K))) return QL_ERR_SHAPE;
    return QL_OK;
}

int check_glu(int32_t glu) { return glu == 0 || glu == 1 ? QL_OK : QL_ERR_UNSUPPORTED; }

int check_fusion(const ql_fusion *f, int64_t M)
{
    if (!f) return QL_OK;
    if ((f->act != QL_ACT_NONE && f->act != QL_ACT_GELU_TANH) || f->reserved != 0 || f->row_absmax) return QL_ERR_UNSUPPORTED;
    if (f->gate && (f->gate_rows < 1 || M % f->gate_rows != 0)) return QL_ERR_SHAPE;
    return off(f->residual, 2) || off(f->gate, 2) ? QL_ERR_ALIGN : QL_OK;
}

int check_workspace(const void *ws, size_t have, size_t need)
{
    if (!ws || have < need) return QL_ERR_WORKSPACE;
    return off(ws, 256) ? QL_ERR_ALIGN : QL_OK;
}

ql::F8DaqArgs daq_args(const void *x, int64_t M, int64_t K, int32_t glu, void *q, void *scales)
{
    ql::F8DaqArgs d{};
    d.x = x;
    d.q = q;
    d.scales = static_cast<float *>(scales);
    d.M = (int)M;
    d.K = (int)K;
    d.KB = ql::f8_blocks(K);
    d.glu = glu != 0;
    return d;
}

ql::F8Gemm gemm_args(const void *q, const void *scales, int64_t M, int64_t K, const void *w, const void *w_scale, int64_t N, void *y)
{
    ql::F8Gemm g{};
    g.q = static_cast<const uint8_t *>(q);
    g.s = static_cast<const float *>(scales);
    g.w = static_cast<const uint8_t *>(w);
    g.s_w = static_cast<const float *>(w_scale);
    g.M = (int)M;
    g.N = (int)N;
    g.K = (int)K;
    g.KB = ql::f8_blocks(K);
    g.NB = ql::f8_blocks(N);
    g.gate_rows = 1;
    g.y = y;
    return g;
}

int run_layer(ql::F8Gemm g, const void *bias, const ql_fusion *f, bool glu, hipStream_t s)
{
    g.codes = !glu;
    g.bias = bias;
    if (f) {
        g.act = f->act;
        g.residual = f->residual;
        g.gate = f->gate;
        g.gate_rows = f->gate ? (int)f->gate_rows : 1;
    }
    return ql::status_of(ql::launch_qgemm_f8(g, s));
}

// codes and scales of a layer's input
struct LayerRoom {
    size_t scales, total;
    LayerRoom(int64_t M, int64_t K) : scales(align_up((size_t)(M * K))), total(scales + align_up((size_t)M * ql::f8_blocks(K) * 4)) {}
};

// what the experts' layers keep between their launches: sizes grow with T and k
struct ExpertRoom {
    size_t first, order, place, tiles, counts, q, s, h, hq, hs, o, up, total;
    int64_t P, tiles_most;
    int tile;
    bool wide;   // h and o are fp32
    ExpertRoom(int64_t T, int64_t k, int64_t E, int64_t K, int64_t I, int64_t N)
    {
        P = T * k;
        tile = ql::f8_expert_tile(P, E);
        tiles_most = ql::expert_tiles_most(P, E, tile);
        // The rows' outputs: from tiles in binary16, which the sum over the choices reads again (in fp32 256 tokens through 8 of 64 experts of 2048 x 1024 took 117 us in the
        // place of 113, 4096 through 2 of 8 201 in the place of 175).  The rounding is the one of every layer's output here; y is 3.0e-4 of its size off with it, 2.1e-4 without.
        // Their range is fp32's all the same: 64 neighbours that reach 2^15 are kept with a power of two that they share (2048 tokens through 8 of 64 316 -> 319 us).
        wide = tile < ql::F8_TILE_ROWS;
        const int64_t few = std::min(P, ql::f8_expert_few(E) - 1);   // (a call with fewer rows than this one's may be of few)
        size_t at = 0;
        auto take = [&](size_t bytes) {
            const size_t here = at;
            at += align_up(bytes);
            return here;
        };
        first = take((size_t)(E + 1) * 4);
        order = take((size_t)P * 4);
        place = take((size_t)P * 4);
        tiles = take((size_t)(1 + 2 * ql::expert_tiles_most(P, E, 16)) * 4);
        counts = take((size_t)ql::expert_chunks(P) * E * 4);
        q = take((size_t)(T * K));
        s = take((size_t)T * ql::f8_blocks(K) * 4);
        h = take((size_t)(few * I) * 4);
        hq = take((size_t)(P * I));
        hs = take((size_t)P * ql::f8_blocks(I) * 4);
        o = take((size_t)std::max(P * N * 2, few * N * 4));
        up = take((size_t)P * ((N + ql::F8_UP - 1) / ql::F8_UP));
        total = at;
    }
};

int check_experts(int64_t T, int64_t k, int64_t E, int64_t K, int64_t I, int64_t N)
{
    if (T < 1 || k < 1 || E < 1 || K < 1 || I < 1 || N < 1 || k > CHOICES_MAX || E > EXPERTS_MAX) return QL_ERR_SHAPE;
    if (K % 16 != 0 || I % 16 != 0 || N % 8 != 0 || T > EXPERT_ROWS_MAX / k) return QL_ERR_SHAPE;
    if (over(T, K) || over(T * k, I) || over(T * k, N) || over(I, K) || over(N, I)) return QL_ERR_SHAPE;
    return QL_OK;
}

}  // namespace

extern "C" {

int daq_quantize_f8(const void *x, int64_t M, int64_t K, int32_t glu, void *q, void *scales, void *stream)
{
    if (!x || !q || !scales) return QL_ERR_NULL;
    int rc = check_glu(glu);
    if (rc || (rc = check_layer(M, K, 1, glu))) return rc;
    if (off(x, 16) || off(q, 16) || off(scales, 4)) return QL_ERR_ALIGN;
    return ql::status_of(ql::launch_daq_f8(daq_args(x, M, K, glu, q, scales), static_cast<hipStream_t>(stream)));
}

int qgemm_f8(const void *q, const void *scales, int64_t M, int64_t K, const void *w, const void *w_scale, const void *bias, int64_t N,
             const ql_fusion *fusion, void *y, void *stream)
{
    if (!q || !scales || !w || !w_scale || !y) return QL_ERR_NULL;
    int rc = check_layer(M, K, N, 0);
    if (rc || (rc = check_fusion(fusion, M))) return rc;
    if (off(q, 16) || off(w, 16) || off(y, 16) || off(scales, 4) || off(w_scale, 4) || off(bias, 2)) return QL_ERR_ALIGN;
    return run_layer(gemm_args(q, scales, M, K, w, w_scale, N, y), bias, fusion, false, static_cast<hipStream_t>(stream));
}

size_t qlinear_f8_workspace_bytes(int64_t M, int64_t K, int64_t N)
{
    return check_layer(M, K, N, 0) ? 0 : LayerRoom(M, K).total;
}

int qlinear_f8(const void *x, int64_t M, int64_t K, int32_t glu, const void *w, const void *w_scale, const void *bias, int64_t N,
               const ql_fusion *fusion, void *y, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!x || !w || !w_scale || !y) return QL_ERR_NULL;
    int rc = check_glu(glu);
    if (rc || (rc = check_layer(M, K, N, glu)) || (rc = check_fusion(fusion, M))) return rc;
    if (off(x, 16) || off(w, 16) || off(y, 16) || off(w_scale, 4) || off(bias, 2)) return QL_ERR_ALIGN;
    const LayerRoom room(M, K);
    if ((rc = check_workspace(workspace, workspace_bytes, room.total))) return rc;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (ql::qgemm_f8_takes_rows(M, K, N, glu != 0)) {
        ql::F8Gemm g = gemm_args(nullptr, nullptr, M, K, w, w_scale, N, y);
        g.x = x;
        g.glu = glu != 0;
        return run_layer(g, bias, fusion, g.glu, s);
    }
    if ((rc = ql::status_of(ql::launch_daq_f8(daq_args(x, M, K, glu, ws, ws + room.scales), s)))) return rc;
    return run_layer(gemm_args(ws, ws + room.scales, M, K, w, w_scale, N, y), bias, fusion, glu != 0, s);
}

int route_experts(const ql_routing *r, void *stream)
{
    if (!r || !r->logits || !r->ids || !r->weights) return QL_ERR_NULL;
    if ((r->score != QL_SCORE_SOFTMAX && r->score != QL_SCORE_SIGMOID) || (r->logits_fp32 != 0 && r->logits_fp32 != 1) || (r->renorm != 0 && r->renorm != 1) ||
        (r->group_top != 1 && r->group_top != 2) || r->reserved != 0 || !std::isfinite(r->scale))
        return QL_ERR_UNSUPPORTED;
    if (r->T < 1 || r->E < 1 || r->E > EXPERTS_MAX || r->k < 1 || r->k > r->E || r->k > CHOICES_MAX || over(r->T, r->E)) return QL_ERR_SHAPE;
    if (r->groups < 1 || r->groups > GROUPS_MAX || r->E % r->groups != 0 || r->top_groups < 1 || r->top_groups > r->groups) return QL_ERR_SHAPE;
    if (off(r->logits, r->logits_fp32 ? 4 : 2) || off(r->bias, 4) || off(r->ids, 4) || off(r->weights, 4)) return QL_ERR_ALIGN;
    ql::RouteArgs a{};
    a.logits = r->logits;
    a.bias = static_cast<const float *>(r->bias);
    a.ids = static_cast<int *>(r->ids);
    a.weights = static_cast<float *>(r->weights);
    a.T = (int)r->T;
    a.E = r->E;
    a.k = r->k;
    a.groups = r->groups;
    a.top_groups = r->top_groups;
    a.group_top = r->group_top;
    a.wide = r->logits_fp32 != 0;
    a.sigmoid = r->score == QL_SCORE_SIGMOID;
    a.renorm = r->renorm != 0;
    a.scale = r->scale;
    return ql::status_of(ql::launch_route(a, static_cast<hipStream_t>(stream)));
}

size_t experts_f8_workspace_bytes(int64_t T, int32_t k, int32_t E, int64_t K, int64_t I, int64_t N)
{
    return check_experts(T, k, E, K, I, N) ? 0 : ExpertRoom(T, k, E, K, I, N).total;
}

int experts_f8(const ql_experts_f8 *x, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!x || !x->x || !x->ids || !x->weights || !x->w_up || !x->up_scale || !x->w_down || !x->down_scale || !x->y) return QL_ERR_NULL;
    int rc = check_experts(x->T, x->k, x->E, x->K, x->I, x->N);
    if (rc) return rc;
    if (off(x->x, 16) || off(x->w_up, 16) || off(x->w_down, 16) || off(x->residual, 16) || off(x->y, 16) || off(x->ids, 4) || off(x->weights, 4) ||
        off(x->up_scale, 4) || off(x->down_scale, 4))
        return QL_ERR_ALIGN;
    const ExpertRoom room(x->T, x->k, x->E, x->K, x->I, x->N);
    if ((rc = check_workspace(workspace, workspace_bytes, room.total))) return rc;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto ints = [&](size_t at) { return reinterpret_cast<int *>(ws + at); };

    const int *ids = static_cast<const int *>(x->ids);
    const bool few = ql::experts_f8_takes_ids(room.P, x->K, x->I, x->N);
    ql::F8Gemm up = gemm_args(ws + room.q, ws + room.s, room.P, x->K, x->w_up, x->up_scale, x->I, ws + room.h);
    ql::F8Gemm down = gemm_args(ws + room.hq, ws + room.hs, room.P, x->I, x->w_down, x->down_scale, x->N, ws + room.o);
    up.k = down.k = x->k;
    up.E = down.E = x->E;
    up.gated = true;
    down.up = ws + room.up;
    if (few) {
        up.ids = down.ids = ids;
        up.x = x->x;
        down.x = ws + room.h;
        if ((rc = ql::status_of(ql::launch_qgemm_f8(up, s)))) return rc;
        if ((rc = ql::status_of(ql::launch_qgemm_f8(down, s)))) return rc;
    } else {
        ql::ExpertRows rows{};
        rows.first = ints(room.first);
        rows.order = ints(room.order);
        rows.place = ints(room.place);
        rows.tiles = ints(room.tiles);
        rows.counts = ints(room.counts);
        rows.P = (int)room.P;
        rows.E = x->E;
        rows.tile = room.tile;
        if ((rc = ql::status_of(ql::launch_expert_rows(ids, rows, daq_args(x->x, x->T, x->K, 0, ws + room.q, ws + room.s), s)))) return rc;
        up.first = down.first = rows.first;
        up.tiles = down.tiles = rows.tiles;
        up.tiles_most = down.tiles_most = (int)room.tiles_most;
        up.tile = down.tile = room.tile;
        up.order = rows.order;
        up.hq = ws + room.hq;
        up.hs = reinterpret_cast<float *>(ws + room.hs);
        if ((rc = ql::status_of(ql::launch_qgemm_f8(up, s)))) return rc;
        if (room.wide) {
            ql::F8DaqArgs d = daq_args(ws + room.h, room.P, x->I, 0, ws + room.hq, ws + room.hs);
            d.wide = true;
            d.rows = rows.first + x->E;
            if ((rc = ql::status_of(ql::launch_daq_f8(d, s)))) return rc;
        }
        if ((rc = ql::status_of(ql::launch_qgemm_f8(down, s)))) return rc;
    }

    ql::ExpertSumArgs sum{};
    sum.o = ws + room.o;
    sum.up = ws + room.up;
    sum.place = few ? ids : ints(room.place);
    sum.ids = few;
    sum.E = x->E;
    sum.weights = static_cast<const float *>(x->weights);
    sum.residual = x->residual;
    sum.y = x->y;
    sum.T = (int)x->T;
    sum.k = x->k;
    sum.N = (int)x->N;
    sum.wide = room.wide;
    return ql::status_of(ql::launch_expert_sum(sum, s));
}

}  // extern "C"
