// The product on the 8-bit integer matrix cores for many digit rows (see pb_imma.h for the arithmetic).
#include <type_traits>

#include "pb_imma.h"

namespace pb {

// Many digit rows: the eight waves of a workgroup share the expanded weight codes through LDS.
//   NT waves lie along the digit rows, TM tiles of sixteen each; 8 / NT groups of waves share out the columns.  A tile is one digit
//   of sixteen vectors: a wave of four tiles has all digits of sixteen vectors of 32 bits, and of two waves of two tiles one has the
//   lower two and the other the upper two.  Sixteen vectors that need only three digits cost three tiles: the fourth is neither read
//   nor multiplied, and the waves are numbered so that every SIMD has as many waves of lower as of upper digits.
//   NT column slots (a row tile and a group of bitlayers each); a step of a group of waves covers a chunk of 512 columns,
//   and every wave expands one unit (slot, chunk) per step: it loads the words two steps ahead, turns them into codes
//   one step ahead, and multiplies its own digit rows, which come straight from memory (each byte is used by one
//   wave only), with the codes of all units of the step.
// Bound: the matrix instructions at the large end (one in 16 cycles per SIMD); for few vectors the digit rows, which every
// workgroup reads at 64 bytes per cycle, LDS, the expansion and the matrix instructions, about as long each.  Operands of the codes
// are read from LDS three (six, seven) products ahead and the scheduler is kept from moving work across a (t, h): without that barrier
// the products waited for their operands (64 vectors: 39 -> 32 us).
// us per call in a graph, digits included, 8192 x 8192, 8 bitlayers, values within three digits, against four digits with a vector's digits
// next to each other in memory: 16 vectors 24.4 -> 22.3, 64 31.2 -> 28.1, 256 74.9 -> 64.6, 1024 260 -> 214 (pairs layout 261 -> 214);
// 16384 x 16384, 64 vectors 117 -> 103, 256 255 -> 214.  Vectors of 8 bits, whose rows now are four pieces of 256 bytes and were sixteen
// of 64: 64 vectors 41.5 -> 23.4, 256 47.2 -> 34.6, 1024 94.6 -> 85.1; of 16 bits 30.8 -> 28.0, 63.7 -> 60.5, 151 -> 149.
// Values beyond three digits, one in every sixteen vectors, against four digits of every value as it was: 64 vectors 31.3 -> 30.2, 256 73.9 -> 71.5,
// 1024 260 -> 248; 3795 x 5918, 16 bitlayers, 301 vectors 133.8 -> 133.6.
// A kernel for each number of digits: one kernel for all of them had the loop over the steps three times and every kind of output, which
// filled the registers (scratch memory also in the shape of eight waves and two tiles), and turned a digit of 8- and 16-bit vectors by zero.
// One kernel -> three: 64 vectors 28.0 -> 27.3, with values beyond three digits 30.8 -> 30.2, 4096 x 4096 16.5 -> 15.8; 1024 vectors of 8 bits 86.4 ->
// 84.0, 256 34.7 -> 34.0; LSTM step 6000 x 3000, 5 bitlayers, 64 vectors 18.3 -> 17.3.
// The shape with four tiles per wave still needs more than the 256 registers of a wave (up to 196 bytes of scratch): the loop of three digits
// has none of them, those of four, two and one reload up to twelve registers in a step of 264 matrix instructions.  A kernel with scratch takes
// 0.3 us longer to launch.
// Calls with several groups of bitlayers (more than eight bitlayers, scales that do not halve, the parity hooks) give them
// slots of their own, so that the sums of a row tile's groups meet in a lane.
template <int ND, int Q, bool IL, int NT, int TM, int EPI>
__global__ __launch_bounds__(512) void k_i8_tile(const I8Args a, const int rows_per_wg)
{
#include "pb_i8_tile.inc"
}

// The same product with act(g) u of a gated block behind it, in the shape that has registers left for it (the others leave the pre-activations in
// memory for k_gated).  21844 x 4096, 5 of 8 bitlayers, 24 vectors: 30.2 us; k_i8_tile 28.5 and k_gated 4.9.
template <int ND, int Q>
__global__ __launch_bounds__(512) void k_gated_tile(const I8Args a, const int rows_per_wg)
{
    constexpr bool IL = false;
    constexpr int NT = 4, TM = 2, EPI = kGated;
#include "pb_i8_tile.inc"
}

// ---------------------------------------------------------------------------------------------------------------

template <int ND, int Q, bool IL, int NT, int TM, int EPI>
static const void *tile_kernel()
{
    // (the sums themselves are asked for in groups of one or two: four slots)
    if constexpr ((EPI == kSums && Q > 1) || (EPI == kCell && IL)) return nullptr;
    else return reinterpret_cast<const void *>(k_i8_tile<ND, Q, IL, NT, TM, EPI>);
}
#define PB_TILE_E(ND, NT, TM, E) {{tile_kernel<ND, 1, false, NT, TM, E>(), tile_kernel<ND, 1, true, NT, TM, E>()}, \
                                  {tile_kernel<ND, 2, false, NT, TM, E>(), tile_kernel<ND, 2, true, NT, TM, E>()}}
#define PB_TILE_ND(ND, NT, TM) {PB_TILE_E(ND, NT, TM, kStore), PB_TILE_E(ND, NT, TM, kCell), PB_TILE_E(ND, NT, TM, kSums)}
#define PB_TILE(NT, TM) {PB_TILE_ND(1, NT, TM), PB_TILE_ND(2, NT, TM), PB_TILE_ND(4, NT, TM)}
static const void *const kTileFn[kTileShapes][3][3][2][2] = {PB_TILE(4, 2), PB_TILE(8, 2), PB_TILE(8, 4)};
static const void *const kGatedTileFn[3][2] = {{reinterpret_cast<const void *>(k_gated_tile<1, 1>), reinterpret_cast<const void *>(k_gated_tile<1, 2>)},
                                               {reinterpret_cast<const void *>(k_gated_tile<2, 1>), reinterpret_cast<const void *>(k_gated_tile<2, 2>)},
                                               {reinterpret_cast<const void *>(k_gated_tile<4, 1>), reinterpret_cast<const void *>(k_gated_tile<4, 2>)}};
constexpr int kTileLds = 128 * 1024;

int launch_imma_tile(int shape, const I8Args &a, int nd, bool il, hipStream_t st)
{
    const int epi = a.A ? kSums : (a.c_prev ? kCell : kStore), q = (epi != kSums && a.m > 4) ? 1 : 0, ndi = nd == 4 ? 2 : nd - 1;
    const bool gated = gated_tile(shape) && a.gate >= 0;
    const void *fn = gated ? kGatedTileFn[ndi][q] : kTileFn[shape][ndi][epi][q][il];
    static uint64_t declared[2][kTileShapes][3][3][2][2];
    if (!fn) return (int)hipErrorInvalidValue;
    const int d = declare_lds(fn, kTileLds, &declared[gated][shape][ndi][epi][q][il]);
    if (d) return d;
    const TileShape &t = kTile[shape];
    int rows_per_wg = tile_rows(t, a.m, epi == kSums);
    const int vpt = 16 / nd, tiles = (a.act.batch + vpt - 1) / vpt;
    const int groups = (tiles + t.nt * t.tm - 1) / (t.nt * t.tm), wgs = (a.rt_count + rows_per_wg - 1) / rows_per_wg;
    void *args[] = {const_cast<I8Args *>(&a), &rows_per_wg};
    const hipError_t e = hipLaunchKernel(fn, dim3((unsigned)wgs, (unsigned)groups), dim3(512), args, kTileLds, st);
    return (int)(e != hipSuccess ? e : hipGetLastError());
}

}  // namespace pb
