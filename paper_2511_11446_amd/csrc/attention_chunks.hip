// Attention of many rows over the paged 8-bit cache for gfx950: prompts that enter it by chunks.
//
// The tile of attention_tile.h, its keys and values made from the codes: a workgroup reads a group of 64 tokens once, through registers, turns the codes into
// binary16 (exactly) and leaves them in LDS for its 256 rows.  Where one scale covers the group it goes into the factor of the
// scores and into the exponent of the weights; smaller blocks multiply both.  Which of them it is is asked at run time, among the weights too.
//
// 8 sequences of 512 new tokens, the longest on 4096 kept ones, 16 heads of 128 on 2, scores capped: 143 us and 17 of join_chunks, 0.26 PFLOP/s.  The wavefronts
// wait for 44 % of their cycles, the vector units work 50 % of the busy ones, the matrix cores 18 %: 602 vector instructions for a wavefront's tile, 32 of them of the matrix
// cores, and 32 to 34 registers of heads of 128 are spilled (49 to 52 of heads of 256): both scale forms are in one kernel, with a branch for every two weights.  Without the cap,
// 512 rows on 4096 tokens for 8 sequences, 16 heads on 2, blocks of 64 / 16 / 1 tokens: heads of 128 228 / 286 / 288 us, heads of 256 638 / 852 / 851.
#include "attention_tile.h"

namespace ql {

// wavefronts of a workgroup: long heads need all registers of a SIMD for one.  Four of them for the others (two workgroups on a CU, the codes turned into
// binary16 twice as often) took 145 + 18 us against 141 + 17 at the sizes above, the keys cut into three parts; into two 153 + 15, into four 145 + 26.
constexpr int chunk_waves(int CHP) { return CHP <= 16 ? 8 : 4; }

template <int CHP, bool SHAPED>
__global__ __launch_bounds__(64 * chunk_waves(CHP), CHP <= 16 ? 2 : 1) void attend_chunks(AttnArgs a, TilePlan plan)
{
    attend_tile<CHP, chunk_waves(CHP), true, SHAPED>(a, plan);
}

__global__ __launch_bounds__(JOIN_THREADS) void join_chunks(AttnArgs a, TilePlan plan, int rows_per) { join_splits(a, plan, rows_per); }

namespace {
// Workgroups that few row tiles are cut into along the keys, us of the kernel + the join at the sizes above (256 without a cut):
// 256 227 + 0, 384 150 + 23, 512 148 + 15, 768 140 + 17, 1024 140 + 24, 1536 149 + 30.
constexpr int CUS = 256, WANTED = 768;
constexpr int chunk_rows(int D) { return 32 * chunk_waves(D / 8); }

template <int CHP>
hipError_t launch_chunks(const AttnArgs &a, hipStream_t stream)
{
    using T = AttnTile<CHP, chunk_waves(CHP), true>;
    const TilePlan p = tile_plan(a.Tq, a.B, a.G, a.Hkv, T::ROWS, a.cu_q, a.mask, (long long)a.max_pages * a.page, CUS, WANTED);
    static const hipError_t opt_in[2] = {
        hipFuncSetAttribute(reinterpret_cast<const void *>(&attend_chunks<CHP, false>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES),
        hipFuncSetAttribute(reinterpret_cast<const void *>(&attend_chunks<CHP, true>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES)};
    const bool shaped = a.cap > 0.0f || a.slopes;
    if (opt_in[shaped] != hipSuccess) return opt_in[shaped];
    const long long wgs = (long long)p.tiles * a.Hkv * p.splits;
    const dim3 grid((unsigned)((wgs + 7) / 8 * 8));
    if (shaped) hipLaunchKernelGGL((attend_chunks<CHP, true>), grid, dim3(T::NT), T::LDS_BYTES, stream, a, p);
    else hipLaunchKernelGGL((attend_chunks<CHP, false>), grid, dim3(T::NT), T::LDS_BYTES, stream, a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL(join_chunks, dim3((unsigned)(p.tiles * a.Hkv), join_blocks(T::ROWS, a.D)), dim3(JOIN_THREADS), 0, stream, a, p, T::ROWS);
    return hipGetLastError();
}
}  // namespace

size_t chunks_partial_bytes(long long Tq, int B, int Hq, int Hkv, int D)
{
    const TilePlan p = tile_plan(Tq, B, Hq / Hkv, Hkv, chunk_rows(D), true, 0, 1LL << 31, CUS, WANTED);
    return p.splits == 1 ? 0 : (size_t)p.tiles * Hkv * p.splits * chunk_rows(D) * (D + 2) * 4;
}

size_t chunks_most_bytes(long long Tq, int B, int Hq, int Hkv, int D)
{
    return (size_t)most_parts(Tq, B, Hq / Hkv, Hkv, chunk_rows(D), 1LL << 31, WANTED) * chunk_rows(D) * (D + 2) * 4;
}

hipError_t launch_attention_chunks(const AttnArgs &a, hipStream_t stream)
{
    const int ch = a.D / 8;
    if (ch <= 4) return launch_chunks<4>(a, stream);
    if (ch <= 8) return launch_chunks<8>(a, stream);
    if (ch <= 10) return launch_chunks<10>(a, stream);
    if (ch <= 12) return launch_chunks<12>(a, stream);
    if (ch <= 16) return launch_chunks<16>(a, stream);
    if (ch <= 24) return launch_chunks<24>(a, stream);
    return launch_chunks<32>(a, stream);
}

}  // namespace ql
