// Attention, the plain way: one wavefront per row and head, one key after the other.
#include "attention.h"

namespace ql {

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m, 64);
    return v;
}

template <bool KV8>
__global__ __launch_bounds__(256) void attend_rows(AttnArgs a)
{
    const int lane = threadIdx.x & 63;
    const long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = (int)(id / a.Hq), h = (int)(id % a.Hq);
    if (t >= a.Tq) return;
    int b = 0;
    SeqRows sq = seq_rows(a.cu_q, 0, a.Tq, a.B);
    while (t >= sq.first + sq.n) {
        if (++b == a.B) return;   // behind the last sequence
        sq = seq_rows(a.cu_q, b, a.Tq, a.B);
    }
    if (t < sq.first) return;     // in front of the first
    const SeqRows sk = KV8 ? SeqRows{0, min(max(a.len_k[b], 0), a.max_pages * a.page)} : seq_rows(a.cu_k, b, a.Tk, a.B);
    const int p = t - sq.first + sk.n - sq.n;
    const int end = visible_end(a.mask, a.prefix ? a.prefix[b] : 0, p, sk.n);
    const int hk = h / a.G;
    const _Float16 *q = static_cast<const _Float16 *>(a.q) + t * a.q_row + h * a.q_head;
    float qv[4], acc[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) qv[i] = lane + 64 * i < a.D ? (float)q[lane + 64 * i] : 0.0f;
    float m = -__builtin_inff(), l = 0.0f;
    const float slope = a.slopes ? a.slopes[h] : 0.0f;
    for (int j = 0; j < end; ++j) {
        float kd[4], vd[4];
        if (KV8) {
            const int page = a.page_table[(long long)b * a.max_pages + j / a.page], at = j % a.page;
            if (page < 0 || page >= a.num_pages) continue;
            const size_t ph = (size_t)page * a.Hkv + hk;
            const float sk_ = a.ks[ph * (a.page / a.scale_tokens) + at / a.scale_tokens], sv = a.vs[ph * (a.page / a.scale_tokens) + at / a.scale_tokens];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = lane + 64 * i;
                kd[i] = d < a.D ? sk_ * (float)a.kc[(ph * a.page + at) * a.D + d] : 0.0f;
                vd[i] = d < a.D ? sv * (float)a.vc[((ph * (a.page / KV_GROUP) + at / KV_GROUP) * a.D + d) * KV_GROUP + kv_slot(at % KV_GROUP)] : 0.0f;
            }
        } else {
            const _Float16 *k = static_cast<const _Float16 *>(a.k) + (sk.first + j) * a.k_row + hk * a.k_head;
            const _Float16 *v = static_cast<const _Float16 *>(a.v) + (sk.first + j) * a.v_row + hk * a.v_head;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = lane + 64 * i;
                kd[i] = d < a.D ? (float)k[d] : 0.0f;
                vd[i] = d < a.D ? (float)v[d] : 0.0f;
            }
        }
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) s = __builtin_fmaf(qv[i], kd[i], s);
        s = wave_sum(s) * a.scale;
        if (a.cap > 0.0f) s = a.cap * tanhf(s / a.cap);
        s -= slope * fabsf((float)(p - j));
        const float m2 = fmaxf(m, s);
        const float keep = __expf(m - m2), w = __expf(s - m2);
        l = l * keep + w;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = acc[i] * keep + w * vd[i];
        m = m2;
    }
    _Float16 *o = static_cast<_Float16 *>(a.o) + t * a.o_row + h * a.o_head;
    unsigned amax = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (lane + 64 * i < a.D) {
            const _Float16 v = (_Float16)(l > 0.0f ? acc[i] / l : 0.0f);
            o[lane + 64 * i] = v;
            amax = max(amax, (unsigned)__builtin_bit_cast(unsigned short, v) & 0x7fffu);
        }
    }
    if (a.row_absmax) atomicMax(a.row_absmax + t, amax);
}

hipError_t launch_attention_f16(const AttnArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL(attend_rows<false>, dim3((unsigned)(((long long)a.Tq * a.Hq + 3) / 4)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_attention_kv8(const AttnArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL(attend_rows<true>, dim3((unsigned)(((long long)a.Tq * a.Hq + 3) / 4)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ql
