// Attention over binary16 rows for gfx950: one pass over the keys with the running maximum and sum of the softmax.
//
// A workgroup of 4 wavefronts has 128 packed rows (attention.h) of one sequence and key head; keys and values go by tiles of 64 from global memory into
// LDS (global_load_lds, no registers), two tiles deep, and every wavefront reads them from there: attention_tile.h says how.  With fewer rows than
// that the other wavefronts still load, and tiles of 32 or 64 rows that bring more workgroups were no better (us with 32 or 64 / 128 rows): one image of 256
// tokens, 6 heads of 64, 8.3 or 7.7 / 7.6; one of 1024 19.4 or 16.5 / 14.8; one row on 4096 keys, 8 heads of 64, 14.4 or 13.5 / 13.1; 30 tokens 5.5 or
// 5.0 / 4.8; only two sequences of 77 tokens with heads of 16 gained, 4.8 or 4.7 / 4.9.  Many rows lose by them, as each row then reads the keys with
// fewer others: 16 images of 1024 tokens, 16 heads of 72, 283 or 191 / 140.
//
// 16 images of 1024 tokens, 16 heads of 72: 120 to 130 us a call, by the machine; at 130 0.59 PFLOP/s of the products that D = 72 needs, and 0.73 of those that the matrix
// instructions do (80 channels for the scores, 96 for the values).  8192 tokens, 16 heads of 128 on 2, a prefix of 1000: 315 us a call, 0.89 PFLOP/s (the profiler's trace
// has 340 to 386 us).  Of the busy cycles the matrix cores work 42 and 52 %, the vector units 58 and 44 %, LDS conflicts 11 and 0 %; the wavefronts wait for 31 and 32 % of
// theirs, three a SIMD with heads of 72 (2048 workgroups are 2.67 rounds of them), two with heads of 128.  With a cap and a distance bias (24 packed sequences of up to 1000 tokens,
// heads of 64; 83 us) the vector units work 83 %, the matrix cores 19 %: 452 vector instructions for a wavefront's tile.  Heads of 192 and 256, causal, 8192 tokens, 16 on 2: 603 and 743 us, 0.68 and
// 0.74 PFLOP/s (64: 184 us, 0.75; 128: 315, 0.87).  Small calls are a chain of latencies: launch, first tile, a few more, writing.
#include "attention_tile.h"

namespace ql {

constexpr int TILE_WAVES = 4, TILE_ROWS = 32 * TILE_WAVES;

template <int CHP, bool SHAPED>
__global__ __launch_bounds__(64 * TILE_WAVES, CHP <= 16 ? 2 : 1) void attend_tiles(AttnArgs a, TilePlan plan)
{
    attend_tile<CHP, TILE_WAVES, false, SHAPED>(a, plan);
}

__global__ __launch_bounds__(JOIN_THREADS) void join_tiles(AttnArgs a, TilePlan plan, int rows_per) { join_splits(a, plan, rows_per); }

namespace {
constexpr int CUS = 256;

template <int CHP>
hipError_t launch_tiles(const AttnArgs &a, hipStream_t stream)
{
    using T = AttnTile<CHP, TILE_WAVES, false>;
    const TilePlan p = tile_plan(a.Tq, a.B, a.G, a.Hkv, TILE_ROWS, a.cu_q, a.mask, a.Tk / a.B, CUS, 2 * CUS);
    static const hipError_t opt_in[2] = {
        hipFuncSetAttribute(reinterpret_cast<const void *>(&attend_tiles<CHP, false>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES),
        hipFuncSetAttribute(reinterpret_cast<const void *>(&attend_tiles<CHP, true>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES)};
    const bool shaped = a.cap > 0.0f || a.slopes;
    if (opt_in[shaped] != hipSuccess) return opt_in[shaped];
    const long long wgs = (long long)p.tiles * a.Hkv * p.splits;
    const dim3 grid((unsigned)((wgs + 7) / 8 * 8));
    if (shaped) hipLaunchKernelGGL((attend_tiles<CHP, true>), grid, dim3(T::NT), T::LDS_BYTES, stream, a, p);
    else hipLaunchKernelGGL((attend_tiles<CHP, false>), grid, dim3(T::NT), T::LDS_BYTES, stream, a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL(join_tiles, dim3((unsigned)(p.tiles * a.Hkv), join_blocks(TILE_ROWS, a.D)), dim3(JOIN_THREADS), 0, stream, a, p, TILE_ROWS);
    return hipGetLastError();
}

}  // namespace

size_t tiles_partial_bytes(long long Tq, long long Tk, int B, int Hq, int Hkv, int D)
{
    const TilePlan p = tile_plan(Tq, B, Hq / Hkv, Hkv, TILE_ROWS, true, 0, Tk / B, CUS, 2 * CUS);
    return p.splits == 1 ? 0 : (size_t)p.tiles * Hkv * p.splits * TILE_ROWS * (D + 2) * 4;
}

size_t tiles_most_bytes(long long Tq, long long Tk, int B, int Hq, int Hkv, int D)
{
    return (size_t)most_parts(Tq, B, Hq / Hkv, Hkv, TILE_ROWS, Tk, 2 * CUS) * TILE_ROWS * (D + 2) * 4;
}

hipError_t launch_attention_f16(const AttnArgs &a, hipStream_t stream)
{
    const int ch = a.D / 8;
    if (ch <= 2) return launch_tiles<2>(a, stream);
    if (ch <= 4) return launch_tiles<4>(a, stream);
    if (ch <= 6) return launch_tiles<6>(a, stream);
    if (ch <= 8) return launch_tiles<8>(a, stream);
    if (ch <= 10) return launch_tiles<10>(a, stream);
    if (ch <= 12) return launch_tiles<12>(a, stream);
    if (ch <= 16) return launch_tiles<16>(a, stream);
    if (ch <= 24) return launch_tiles<24>(a, stream);
    return launch_tiles<32>(a, stream);
}

}  // namespace ql
