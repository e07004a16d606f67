// The product of Algorithm 2 for batches, and for the layout that stores bitlayer pairs, on the 8-bit integer matrix cores
// (see pb_imma.h for the arithmetic): the activations as byte digits, the kernel for few digit rows, and the choice
// between it and the kernel for many.
#include <stdlib.h>

#include "pb_imma.h"

namespace pb {

template <int ND>
__global__ __launch_bounds__(128) void k_digits(ActSource s, int cq, uint8_t *__restrict__ digits, uint8_t *__restrict__ wide,
                                                int32_t *__restrict__ xq_out, const uint32_t turn)
{
    __shared__ int s_wide[2];
    digits_unit<ND>(s, cq, digits, wide, xq_out, turn, blockIdx.x, blockIdx.y, threadIdx.x >> 6, s_wide);
}

// ---------------------------------------------------------------------------------------------------------------

// Waves of a workgroup at most: sixteen have 128 registers each, which four tiles of digit rows exceed
__host__ __device__ constexpr int stream_waves(int tm) { return tm >= 4 ? 8 : 16; }

// LDS of a workgroup beside the staged digits: sums, sums of the codes, sums over the groups, scales
__host__ __device__ constexpr int stream_lds(int nd, int tm, int epi)
{
    return 2 * tm * 4 * 256 + (nd > 1 ? 3 * 256 : 0) + (epi == kSums ? 0 : tm * (4 / nd) * 512) + PB_MAX_BITS * 4;
}

// Bytes of one staged operand of `rows` digit rows (64 each, and 16 more so that the eight operands that a group of eight
// lanes writes to start in different banks); a tile of a chunk has eight of them
__host__ __device__ inline int stage_operand(int rows) { return rows * 64 + 16; }

// Few digit rows (one or two tiles of sixteen), or small matrices: a wave owns a slice of the columns and turns the words of row
// tile after row tile into codes in its registers; the slices of a row meet in LDS once per row tile.
//   FUSED: the activations are converted in this launch.  Every wave leaves the digits of its slice in LDS, in the order in
//   which the matrix instructions read them, and keeps reading them from there.  Else they come from memory (k_digits).
// Bound: latencies at the small end (launch, activations, weights, barrier), the weight stream at the large end.  The words of
// the next unit are requested before this one is multiplied: 8 KB in flight per wave, sixteen waves.  Turning the words of a unit
// into codes takes 160 operations of the vector ALU, its products 16 (one tile) matrix instructions.
// In a graph, us per call, against the FP4 form that this replaces (two bitlayers and two planes per operand):
// 1024 x 1024, 8 bitlayers, 16 vectors 7.3 -> 4.3; 4096 x 4096, 4 vectors 8.1 -> 6.1; 8192 x 8192, 4 vectors 17.5 -> 14.7; 135 x 69, 7
// bitlayers, 113 vectors 14.7 -> 4.6.  The conversion and the codes of a few vectors are more instructions per wave than their FP4
// operands were, which shows where there is little else: 2 to 4 vectors, one or two bitlayers on wide rows (2002 x 5817, one
// bitlayer, 2 vectors 5.0 -> 5.4), more than eight bitlayers (67 x 6211, 16 bitlayers, 3 vectors of 8 bits 9.5 -> 11.8), and one vector on
// the pairs layout (565 x 14030, two bitlayers 5.6 -> 7.9; 4096 x 4096, 8 bitlayers 5.7 -> 5.1).  2148 drawn calls of several vectors
// are 1.7 times as fast on average, 51 of them slower by more than 1.5 %.

template <int ND, int Q, bool IL, int TM, bool FUSED, int EPI, int POLICY, bool PLAIN>
// (the waves per SIMD: one tile, digits from memory, has four at most where a row has sixteen slices, and the registers that this leaves
// let the compiler request the digits earlier: 67 x 4604, 7 vectors of 16 bits 6.4 -> 5.8 us, 913 x 8013, 15 vectors 7.1 -> 6.7, over 194 drawn
// calls 1.7 % on average)
__global__ __launch_bounds__(stream_waves(TM) * 64)
__attribute__((amdgpu_waves_per_eu(stream_waves(TM) / 4, !FUSED && TM == 1 ? 4 : 8))) void k_i8(const I8Args a)
{
#include "pb_i8_stream.inc"
}

// The same product with act(g) u of a gated block behind it.  (One text for both kernels: a function that both call came out with other registers,
// and with scratch memory in one shape of k_i8.)
template <int ND, int Q, int TM, bool FUSED>
__global__ __launch_bounds__(stream_waves(TM) * 64)
__attribute__((amdgpu_waves_per_eu(stream_waves(TM) / 4, !FUSED && TM == 1 ? 4 : 8))) void k_gated_stream(const I8Args a)
{
    constexpr bool IL = false, PLAIN = false;
    constexpr int EPI = kGated, POLICY = 0;
#include "pb_i8_stream.inc"
}

// ---------------------------------------------------------------------------------------------------------------

// Digits per value that `act_bits` needs
static int digits_of(int act_bits) { return act_bits <= 8 ? 1 : (act_bits <= 16 ? 2 : 4); }

static ActSource act_source(const float *X0, int cols0, const float *X1, int cols1, int batch, int frac_bits, int act_bits)
{
    ActSource s;
    s.X0 = X0; s.X1 = X1; s.cols0 = cols0; s.cols1 = X1 ? cols1 : 0;
    s.batch = batch;
    s.fscale = ldexpf(1.0f, frac_bits);
    s.imax = (act_bits == 32) ? INT32_MAX : (int32_t)((1u << (act_bits - 1)) - 1u);
    s.imin = -s.imax - 1;
    return s;
}

int launch_digits(const float *X0, int cols0, const float *X1, int cols1, int batch, const Layout &L, int frac_bits,
                  int act_bits, void *digits, void *wide, int32_t *xq_out, bool plain, hipStream_t st)
{
    const ActSource s = act_source(X0, cols0, X1, cols1, batch, frac_bits, act_bits);
    const dim3 grid((unsigned)L.cq, (unsigned)((batch + 3) / 4));
    const uint32_t turn = plain ? 0x80808080u : 0u;
    uint8_t *d = static_cast<uint8_t *>(digits), *w = static_cast<uint8_t *>(wide);
    switch (digits_of(act_bits)) {
        case 1: hipLaunchKernelGGL(k_digits<1>, grid, dim3(128), 0, st, s, L.cq, d, w, xq_out, turn); break;
        case 2: hipLaunchKernelGGL(k_digits<2>, grid, dim3(128), 0, st, s, L.cq, d, w, xq_out, turn); break;
        default: hipLaunchKernelGGL(k_digits<4>, grid, dim3(128), 0, st, s, L.cq, d, w, xq_out, turn); break;
    }
    return (int)hipGetLastError();
}

// [what follows][digits 1, 2, 4][four or eight slots][bits, pairs][way]: digits from memory, one tile or four; converted in the
// launch, one tile or two, one tile with non-temporal loads of the weights; one tile, digits from memory, the third as it stands
// (the sums themselves are asked for in groups of one or two: four slots)
enum { kMemory1 = 0, kMemory4 = 1, kFused1 = 2, kFused2 = 3, kFusedNt = 4, kPlain1 = 5, kStreams = 6 };
static bool is_fused(int way) { return way >= kFused1 && way <= kFusedNt; }
static int way_tiles(int way) { return way == kMemory4 ? 4 : (way == kFused2 ? 2 : 1); }
template <int ND, int Q, bool IL, int TM, bool FUSED, int EPI, int POLICY = 0, bool PLAIN = false>
static const void *stream_kernel()
{
    if constexpr ((EPI == kSums && Q > 1) || (EPI == kCell && IL) || ((POLICY || PLAIN) && EPI != kStore) || (PLAIN && ND != 4)) return nullptr;
    else return reinterpret_cast<const void *>(k_i8<ND, Q, IL, TM, FUSED, EPI, POLICY, PLAIN>);
}
#define PB_I8_IL(ND, Q, IL, E)                                                                                     \
    {stream_kernel<ND, Q, IL, 1, false, E>(), stream_kernel<ND, Q, IL, 4, false, E>(),                              \
     stream_kernel<ND, Q, IL, 1, true, E>(), stream_kernel<ND, Q, IL, 2, true, E>(), stream_kernel<ND, Q, IL, 1, true, E, 2>(), \
     stream_kernel<ND, Q, IL, 1, false, E, 0, true>()}
#define PB_I8_ND(ND, E) {{PB_I8_IL(ND, 1, false, E), PB_I8_IL(ND, 1, true, E)}, {PB_I8_IL(ND, 2, false, E), PB_I8_IL(ND, 2, true, E)}}
#define PB_I8(E) {PB_I8_ND(1, E), PB_I8_ND(2, E), PB_I8_ND(4, E)}
static const void *const kI8[3][3][2][2][kStreams] = {PB_I8(kStore), PB_I8(kCell), PB_I8(kSums)};
// (the gated block: [digits][four or eight slots][way])
#define PB_GATED_Q(ND, Q)                                                                                                          \
    {reinterpret_cast<const void *>(k_gated_stream<ND, Q, 1, false>), reinterpret_cast<const void *>(k_gated_stream<ND, Q, 4, false>), \
     reinterpret_cast<const void *>(k_gated_stream<ND, Q, 1, true>), reinterpret_cast<const void *>(k_gated_stream<ND, Q, 2, true>)}
#define PB_GATED(ND) {PB_GATED_Q(ND, 1), PB_GATED_Q(ND, 2)}
static const void *const kGatedFn[3][2][4] = {PB_GATED(1), PB_GATED(2), PB_GATED(4)};

// Staged digits of a workgroup at most (a compute unit has 160 KB of LDS)
constexpr int kMaxStage = 140 * 1024;

// Compute units (at least one, or an error); their number does not change while the process lives
static hipError_t compute_units(int *cus)
{
    static int cache;
    *cus = __atomic_load_n(&cache, __ATOMIC_RELAXED);
    if (*cus > 0) return hipSuccess;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess) e = hipDeviceGetAttribute(cus, hipDeviceAttributeMultiprocessorCount, dev);
    if (e != hipSuccess) return e;
    if (*cus < 1) return hipErrorInvalidDevice;
    __atomic_store_n(&cache, *cus, __ATOMIC_RELAXED);
    return hipSuccess;
}
// Workgroups of a kernel that a compute unit runs at once (0: the query failed; the answer does not change either).  The query is too high
// twice (256 n workgroups of a kernel that only computes take twice as long from the n on where one more has to wait):
//   It divides the waves of the unit by those of the workgroup.  A workgroup of five to eight waves takes two on every SIMD, one of nine to
//   twelve three: with three places a SIMD one workgroup of five waves runs, not two; with four places two, not three.
//   LDS is given out by 1280 bytes: eleven workgroups of 13120 bytes run, not twelve.
// A grid made for more leaves a rest that runs by itself: 12135 x 2547, 8 bitlayers, 13 vectors (five waves) for two per unit 15.7 us, for one
// 12.5; 10440 x 2457, 6 bitlayers, 55 vectors of 8 bits 16.4, 12.7; 9551 x 2050, 2 bitlayers, 13 vectors of 16 bits for three 9.9, for two 8.8;
// 1731 x 276, 6 bitlayers, 887 vectors of 16 bits (13120 bytes) 19.0, 15.8.
constexpr size_t kLds = 160 * 1024, kLdsPiece = 1280;
static int per_unit(const void *fn, int threads, size_t lds, size_t stage, int *slot)
{
    int v = __atomic_load_n(slot, __ATOMIC_RELAXED);
    if (v > 0) return v;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&v, fn, threads, stage) != hipSuccess) return 0;
    auto at_most = [&](int n) { v = n < 1 ? 1 : (n < v ? n : v); };
    if (v > 1 && threads > 256) {
        int places = 0;     // waves of a SIMD: workgroups of four waves
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&places, fn, 256, stage) != hipSuccess) return 0;
        at_most(places / ((threads + 255) / 256));
    }
    if (v > 1) at_most((int)(kLds / ((lds + stage + kLdsPiece - 1) / kLdsPiece * kLdsPiece)));
    if (v > 0) __atomic_store_n(slot, v, __ATOMIC_RELAXED);
    return v;
}

// The call as the choice of the kernel sees it
struct I8Call {
    int rt, cq, tiles, batch, nd, m, groups;
    double weights;   // MB of packed words
};
static int stage_rows(const I8Call &c, int tm)
{
    const int rows = c.nd * ((c.batch + 1) & ~1);   // (vectors are converted two at a time)
    return tm > 1 || rows > 16 ? 16 : rows;
}
static size_t stage_bytes(const I8Call &c, int tm) { return (size_t)c.cq * (size_t)(tm * 8 * stage_operand(stage_rows(c, tm))); }
static int slice(int cq, int tm) { return (cq + stream_waves(tm) - 1) / stream_waves(tm); }   // chunks per wave

// Workgroups of S waves per compute unit of the kernels that convert the activations: each repeats the conversion, so no more than
// eight waves need.  (5003 x 3001, 5 vectors of 16 bits, six waves: one per compute unit 7.5 us, two 8.6; 4096 x 1024, 16
// vectors, two waves: one 7.5, two 6.8, four 5.8 us.)
static int fused_per_cu(int S) { return S >= 4 ? 1 : 8 / S; }

// Weights that are read once (one tile of digit rows): non-temporal loads, which find them in the last-level cache but leave nothing
// there.  Graph of calls, 8 bitlayers, 8192 columns, two vectors, plain / non-temporal loads in us where something else has put the
// weights there (packing) / where only the calls themselves read them, after 1 GB of other data:
//   33 MB 7.9 / 8.0, 8.0 / 10.0    40 MB 11.0 / 11.3, 11.3 / 12.8    48 MB 12.6 / 11.8, 12.8 / 13.1    56 MB 13.4 / 12.9, 13.5 / 14.6
//   64 MB 14.4 / 13.1, 14.6 / 14.4    76 MB 16.6 / 16.3, 16.6 / 17.2    90 MB 18.2 / 18.6, 18.2 / 19.7
// (3072 columns, 5 vectors of 16 bits: 34 MB 9.4 / 9.5, 9.4 / 10.4; 48 MB 12.4 / 11.5, 12.5 / 12.1; 64 MB 15.0 / 14.8, 15.2 / 15.4)
static bool streaming(const I8Call &c) { return c.tiles == 1 && c.weights > 44.0 && c.weights <= 72.0; }

// Which kernel: the one with the least estimated time.  The estimates are in us, fitted to the times of 280 layers on an MI355X (64
// to 16384 rows, 64 to 32768 columns, 2 to 1024 vectors, 1 to 16 bitlayers, 8, 16 and 32 activation bits, both layouts).  Over 2148 other
// calls with every kernel timed, the choice costs 2.6 % on average over the best one, 19 % at the 95th percentile, 1.85 times in
// the worst case: it is weakest with 8- and 16-bit activations of many vectors on a small matrix, whose conversion one after the other
// the estimate takes for shorter than it is (284 x 1200, 21 vectors of 8 bits, cell update 12.2 us, from memory 6.9).  A term for that
// chain, fitted to 900 of the calls, moved 62 of the other 1500 to a kernel over 3 % slower and 48 to one as much faster: left out.
// With digits by groups of sixteen vectors and three of four, 420 more calls: 3.3 % on average over the best, 19 %, 1.55 times; fitted again to
// half of them the estimates were no better on the other half (3.1 %, 3.0 % before) and stay.
// The bitlayers count by themselves: with one cost for all,
// one and two bitlayers of a few vectors went to the wrong kernel (3841 x 7174, one bitlayer, 14 vectors: 13.4 us, here 10.9).
//   few digit rows: rounds of workgroups over the chip (16 / S at once, which they were fitted with; per_unit has what runs), units
//                   (row tile, group, tile of digit rows, chunk), conversion
//   many:           rounds of workgroups times (start and end + steps), the digits of all vectors through memory
static int pick_way(const I8Call &c, bool prepared, int cus)
{
#ifdef PB_TUNING
    if (const char *e = getenv("PB_TUNE_WAY")) {
        const int w = atoi(e);
        if (w >= 0 && (!is_fused(w) || (!prepared && stage_bytes(c, way_tiles(w)) <= kMaxStage))) return w;
    }
#endif
    int best = kMemory1;
    double least = 1e30;
    auto offer = [&](int way, double t) {
        if (t < least) { least = t; best = way; }
    };
    const double bits = (c.m < 8 ? c.m : 8) / 8.0;
    const double quad = c.m > 4 ? 4.0 : 2.0;       // (the codes of a unit cost about as much as that many matrix tiles)
    for (int way = 0; way < kFusedNt; ++way) {
        const int tm = way_tiles(way), groups = (c.tiles + tm - 1) / tm;
        const size_t lds = is_fused(way) ? stage_bytes(c, tm) : 0;
        if (is_fused(way) && (prepared || lds > kMaxStage)) continue;
        const int cpw = slice(c.cq, tm), S = (c.cq + cpw - 1) / cpw;
        int per_cu = is_fused(way) ? fused_per_cu(S) : 16 / S;
        if (is_fused(way) && (size_t)per_cu * (lds + 4096) > 155 * 1024) per_cu = (int)(155 * 1024 / (lds + 4096));
        const int cap = cus * (per_cu < 1 ? 1 : per_cu);
        int wgs = cap / groups < 1 ? 1 : cap / groups;
        if (wgs > c.rt) wgs = c.rt;
        const int rounds = (c.rt + wgs - 1) / wgs;
        const int waves = (((c.rt + rounds - 1) / rounds) * groups + cap - 1) / cap;   // (workgroups after another on a place)
        const double sets = (double)waves * rounds * c.groups;
        const double units = (double)c.rt * groups * c.cq * c.groups * (1.0 + tm / quad) / 1000.0;
        const int pairs = (c.batch + 1) / 2 < 8 * tm / c.nd ? (c.batch + 1) / 2 : 8 * tm / c.nd;     // of vectors of a workgroup
        const double conversions = (double)((((c.rt + rounds - 1) / rounds) * groups + cus - 1) / cus) * c.cq * pairs / 10.0;
        const double digits = c.tiles * c.cq / 100.0;
        const double steps = sets * cpw;
        switch (way) {
        case kMemory1: offer(way, (prepared ? 2.9 : 4.9) + 1.34 * steps + 1.51 * digits + (0.10 + 0.27 * bits) * units + 0.051 * c.weights); break;
        case kMemory4: offer(way, (prepared ? 3.6 : 5.6) + (1.55 + 0.48 * bits) * steps + 1.33 * digits + (0.24 + 0.34 * bits) * units + 0.019 * c.weights); break;
        case kFused1: offer(way, 3.4 + (0.60 + 0.37 * bits) * steps + 0.69 * conversions + (0.20 + 0.15 * bits) * units); break;
        default: offer(way, 3.4 + 0.69 * bits * steps + 0.87 * sets + 0.79 * conversions + 0.137 * units); break;
        }
    }
    static const double cost[kTileShapes][5] = {   // start, step, start and end of a workgroup, weights (MB), digits
        {3.4, 1.67, 5.79, 0.074, 0.0094}, {3.6, 2.68, 7.80, 0.060, 0.0075}, {2.9, 4.31, 17.0, 0.100, 0.0143}};
    for (int i = 0; i < kTileShapes; ++i) {
        const TileShape &t = kTile[i];
        if (c.groups > t.nt) continue;      // (a row tile's groups would take several passes)
        const int rows = t.nt / c.groups;
        const int wgs = ((c.rt + rows - 1) / rows) * ((c.tiles + t.nt * t.tm - 1) / (t.nt * t.tm));
        const int rounds = (wgs + cus - 1) / cus;
        const int per_step = 8 / t.nt;      // chunks
        const int steps = (c.cq + per_step - 1) / per_step;
        offer(kStreams + i, cost[i][0] + rounds * (cost[i][2] + steps * cost[i][1]) + cost[i][3] * c.weights + cost[i][4] * c.tiles * c.cq);
    }
    return best == kFused1 && streaming(c) ? kFusedNt : best;
}

int launch_imma(const uint32_t *packed, const float *scales, const Layout &L, int bits_used, int frac_bits, int act_bits,
                const float *X0, int cols0, const float *X1, int cols1, void *digits, void *wide, bool prepared, int batch,
                float *Y, long long *A, bool pairs_out, const Epilogue &ep, hipStream_t st)
{
    const int nd = digits_of(act_bits);
    I8Args a;
    a.packed = packed;
    a.packed_bytes = (uint32_t)packed_bytes(L);   // (the host API refuses matrices of 4 GiB and more)
    a.layer_step = (uint32_t)(tile16_layer_stride(L) * 4);
    a.round_step = (uint32_t)(tile16_rowtile_stride(L) * 4);
    a.rt_count = L.rt_count; a.cq = L.cq; a.m = bits_used;
    a.digits = static_cast<const uint8_t *>(digits);
    a.digits_bytes = (uint32_t)batch * (uint32_t)L.cq * (uint32_t)(nd * 512);
    a.wide = static_cast<const uint8_t *>(wide);
    a.act = act_source(X0, cols0, X1, cols1, batch, frac_bits, act_bits);
    a.scales = scales; a.Y = Y; a.A = A; a.pairs_out = (A && pairs_out) ? 1 : 0;
    a.bias = ep.bias; a.relu = ep.relu; a.c_prev = ep.c_prev; a.h_out = ep.h_out; a.c_out = ep.c_out; a.gate = ep.gate;
    a.gate_h = L.gate_h; a.R = L.rows;
    a.out_scale = ldexp(1.0, -frac_bits);
    // (the epilogue addresses the bias and the cell state with 32-bit byte offsets)
    if (ep.bias && L.rows >= (1 << 29)) return (int)hipErrorInvalidValue;
    if (ep.c_prev && (size_t)batch * (size_t)L.gate_h >= ((size_t)1 << 29)) return (int)hipErrorInvalidValue;

    const int vpt = 16 / nd;
    const bool il = is_pairs(L.layout);
    I8Call c;
    c.rt = L.rt_count; c.cq = L.cq; c.tiles = (batch + vpt - 1) / vpt; c.batch = batch; c.nd = nd; c.m = bits_used;
    c.groups = A ? (pairs_out ? (bits_used + 1) / 2 : bits_used) : i8_groups(bits_used);
    c.weights = (double)L.layer_words * 4e-6 * bits_used;
    int cus;
    const hipError_t no_device = compute_units(&cus);
    if (no_device != hipSuccess) return (int)no_device;
    // The adapters' first products go along with the digits, a launch less.  us, together / one after the other: 4096 columns, 48 vectors 25.4 / 27.4,
    // 512 vectors 55.0 / 57.4, 2048 vectors 238 / 241; 768 columns, 2017 vectors 46.2 / 50.2.
    auto make_digits = [&](bool plain) {
        if (ep.down && nd == 4) return launch_adapter_down_digits(ep.down, a.act, L.cq, digits, wide, plain, st);
        return launch_digits(X0, cols0, X1, cols1, batch, L, frac_bits, act_bits, digits, wide, nullptr, plain, st);
    };
    // Large batches of the operators: the kernel of pb_batch.hip where its workgroups, one per compute unit, fill 65 % of their rounds over the chip.
    // us with it / with the kernels below, 8 bitlayers, digits included: 8192 x 2048, 300 vectors (192 workgroups) 31.0 / 34.7; 24600 x 4096, 65
    // (193) 46.1 / 52.7; 16384 x 4096, 140 (256) 49.2 / 53.0; 2048 x 8192, 2048 (256) 111 / 138; 6000 x 600, 2000 (752) 60 / 95; but 2048 x 8192, 1000 (128)
    // 80 / 72, 4096 x 4096, 512 (128) 50 / 42, 12000 x 8192, 5 bitlayers, 100 (94) 71 / 51.
    const int large = ep.pre && nd == 4 && batch > kBatchFrom ? batch_workgroups(L.rt_count, batch) : 0;
    if (large * 20 >= (large + cus - 1) / cus * cus * 13 && large) {
        const int e = make_digits(true);
        return e ? e : launch_imma_batch(a, il, ep.pre, a.Y ? a.Y : ep.more, st);
    }
    int way = pick_way(c, prepared, cus);
    if (way == kFusedNt && (A || ep.fused())) way = kFused1;
    // Third digits as they stand: what pb_act_prep leaves; and with at most four bitlayers and more than four tiles, whose digits take longer to read
    // than flags and XOR (1291 x 9493, 4 bitlayers, 17 vectors 11.5 us, all four digits 12.4; 393 x 14185, 2 bitlayers, 29 vectors 9.5, 9.9;
    // but 16337 x 1799, 4 bitlayers, 3 vectors 6.9, 6.5, and 870 x 9440, 8 bitlayers, 21 vectors 13.5, 12.5).
    if (way == kMemory1 && nd == 4 && (prepared || (c.tiles > 4 && bits_used <= 4 && !A && !ep.fused()))) way = kPlain1;
    const int shape = way - kStreams;
    if (!prepared && !is_fused(way)) {
        const int e = make_digits(way != kMemory1);
        if (e) return e;
    }
    if (shape >= 0) {
        if (a.gate < 0 || gated_tile(shape)) return launch_imma_tile(shape, a, nd, il, st);
        // a gated block in another shape: the pre-activations through memory
        if (!a.Y) a.Y = ep.pre;
        const int e = launch_imma_tile(shape, a, nd, il, st);
        return e ? e : launch_gated(a.Y, L.rows / 2, ep.gate, batch, ep.h_out, st);
    }

    const int epi = A ? kSums : (ep.c_prev ? kCell : (ep.gate >= 0 ? kGated : kStore)), q = (!A && bits_used > 4) ? 1 : 0;
    const int ndi = nd == 4 ? 2 : nd - 1, tm = way_tiles(way);
    const void *fn = epi == kGated ? kGatedFn[ndi][q][way] : kI8[epi][ndi][q][il][way];
    if (!fn) return (int)hipErrorInvalidValue;
    a.chunks_per_wave = slice(L.cq, tm);
    a.stage_rows = stage_rows(c, tm);
    const int S = (L.cq + a.chunks_per_wave - 1) / a.chunks_per_wave;
    const size_t lds = is_fused(way) ? stage_bytes(c, tm) : 0;
    static int cache[4][3][2][2][kStreams][17][24];   // (the last index: LDS in steps of 6 KB)
    if (lds > 32 * 1024) {
        static uint64_t declared[4][3][2][2][kStreams];
        const int d = declare_lds(fn, kMaxStage, &declared[epi][ndi][q][il][way]);
        if (d) return d;
    }
    int most = per_unit(fn, S * 64, (size_t)stream_lds(nd, tm, epi), lds, &cache[epi][ndi][q][il][way][S][lds / 6144]);
    if (most < 1) return (int)hipErrorInvalidValue;
    if (is_fused(way) && most > fused_per_cu(S)) most = fused_per_cu(S);
    const int groups = (c.tiles + tm - 1) / tm;
    // Workgroups, and the row tiles of each: as many as run at once.  Of those with more than four waves fewer where the unit that does the most
    // then has fewer row tiles to do: 9619 x 11869, one bitlayer, 16 vectors (eight waves, pairs layout) two workgroups of two row tiles 33.6 us, one
    // of three 30.1; 5888 x 3649, 3 bitlayers, 11 vectors of 16 bits 9.0, 8.5.  With as many to do, two at once are faster than one:
    // 14587 x 2129, 3 bitlayers, 51 vectors of 8 bits (five waves) two of two 12.4, one of four 15.5.
    int wgs = 1;
    for (int n = most, least = INT32_MAX; n >= 1; --n) {
        int w = cus * n / groups;
        w = w < 1 ? 1 : (w < L.rt_count ? w : L.rt_count);
        const int rounds = (L.rt_count + w - 1) / w;
        w = (L.rt_count + rounds - 1) / rounds;
        const int cost = rounds * (6 + (w * groups + cus - 1) / cus * S);
        if (cost < least) { least = cost; wgs = w; a.rounds_per_wg = rounds; }
        if (S <= 4 || is_fused(way)) break;
    }
    void *args[] = {&a};
    const hipError_t e = hipLaunchKernel(fn, dim3((unsigned)wgs, (unsigned)groups), dim3((unsigned)S * 64), args, lds, st);
    return (int)(e != hipSuccess ? e : hipGetLastError());
}

}  // namespace pb
