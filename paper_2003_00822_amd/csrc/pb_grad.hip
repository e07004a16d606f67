// Gradient through a packed matrix: dX[n][c] = sum_r dY[n][r] w[r][c], w[r][c] = sum_(i < bits_used) scales[i] bit_i[r][c], on the
// 8-bit integer matrix cores (pb_imma.h has the codes of the weights).
//
// dY as digits.  A vector's gradients are scaled by the power of two that brings the largest one below 2^30, rounded to integers g and
// split into four balanced byte digits, g = sum_d 256^d s_d with s_d in [-128, 127]: the bytes of (g + 0x808080) ^ 0x808080, because
// 0x808080 = sum_(d < 3) 256^d 128.  The rounding (half a unit, at most 2^-30 of the vector's largest gradient) is the only one before the last
// step: |s code| <= 2^14, so a sum over 65536 rows is exact in int32, and the digits' sums are put together in fp64.
// Batches, which the matrix instructions bound, take three digits (half a unit: at most 2^-23 / 0.995 of the largest gradient; 0.995: a largest value
// that three balanced digits just do not hold is halved) where no vector of sixteen has a value above L times the root of its mean square,
//   L = sqrt(R) / 4 for a sum over R < 2304 rows, 12 up to 4096, 12 sqrt(R / 4096) for more:
// a result is then off by L 2^-22 / sqrt(12) = 6.9e-8 L of the results' root mean square at most, typically a quarter of it, which is no more than a product
// in fp32 is off by: 1.75e-8 sqrt(R), measured from 1500 to 21844 rows.
//
// Few vectors (and small matrices): k_grad makes the digits itself, from the rows of its part of the sum; each part has a scale of its own, and the parts
// are added in fp32 anyway.  Else k_grad_digits leaves them in memory, for all of the columns' workgroups.
//
// The sum runs over the rows of W, and a packed word holds 32 columns of one row: the codes have to be turned, 16 rows of a column
// into the 16 bytes of a lane.  They go through LDS anyway, because every wave needs them, and DS_READ_B64_TR_B8 turns them on the
// way out: its 16 lanes read eight rows of sixteen bytes, and lane i receives byte i of each.
//
// Bound: the packed words for few vectors, the matrix instructions for batches.  us (rocprofv3): 8192 x 8192, 8 bitlayers, 4 vectors: k_grad 17.0 (3.9 TB/s
// of words: 67.5 MB fetched) and k_grad_join 3.9; 6 bitlayers, 768 vectors: k_grad 136 (2.28 POP/s in three digits; a library product of 8-bit integers
// 8192^3 reaches 1.83), the matrix pipelines busy for 60 % of the compute units' cycles, waves waiting for 36 % of theirs, at 2.07 GHz, scalings 7.3, digits 8.2,
// join 14.4; 21844 x 4096, 8 bitlayers, 1024 vectors: k_grad 253 (2.17 POP/s; 66 % and 39 %), in the first calls on an idle card up to 309, k_gated_grad 39
// (136 MB fetched and 91 written, 5.8 TB/s), digits 31 (137 and 68 MB, 6.6 TB/s).
#include <type_traits>

#include "pb_grad.h"

namespace pb {

typedef int v2i __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__global__ __launch_bounds__(1024) void k_grad_scalings(const float *__restrict__ dY, int rows, Scaling *__restrict__ scalings)
{
    scale_vector<16>(dY, rows, blockIdx.x, scalings);
}

// Gradients of the pre-activations [g; u] of H = act(g) u, and the scalings of their vectors
__global__ __launch_bounds__(1024) void k_gated_grad(const float *__restrict__ pre, const float *__restrict__ dH, int units, int gate,
                                                     float *__restrict__ dpre, Scaling *__restrict__ scalings)
{
    const size_t n = blockIdx.x;
    const float *g = pre + n * 2 * units, *u = g + units, *dh = dH + n * units;
    float *dg = dpre + n * 2 * units, *du = dg + units;
    Size size;
    auto one = [&](float g, float u, float dh, float *dg, float *du) {
        float a, da;
        gate_with_slope(gate, g, &a, &da);
        const float x = dh * u * da, y = dh * a;
        *dg = x;
        *du = y;
        size.take(x);
        size.take(y);
    };
    if (units % 2 == 0) {       // (a vector of 2 units values begins at a multiple of 16 bytes, its second half at one of 8)
#pragma unroll 2
        for (int r = threadIdx.x * 2; r < units; r += 2048) {
            const float2 vg = *reinterpret_cast<const float2 *>(g + r), vu = *reinterpret_cast<const float2 *>(u + r);
            const float2 vh = *reinterpret_cast<const float2 *>(dh + r);
            float2 x, y;
            one(vg.x, vu.x, vh.x, &x.x, &y.x);
            one(vg.y, vu.y, vh.y, &x.y, &y.y);
            *reinterpret_cast<float2 *>(dg + r) = x;
            *reinterpret_cast<float2 *>(du + r) = y;
        }
    } else {
        for (int r = threadIdx.x; r < units; r += 1024) one(g[r], u[r], dh[r], dg + r, du + r);
    }
    size.over_workgroup<16>();
    if (threadIdx.x == 0) scalings[n] = scaling_of(size.most, size.squares, 2 * units);
}

// Whether one of the group's vectors needs four digits; the lane's vector is the group's vector lane % 16
__device__ __forceinline__ bool group_is_wide(const Scaling &mine, bool live) { return __builtin_amdgcn_ballot_w64(live && mine.wide) != 0; }

// The values of the sixteen packed rows of row tile 4 step + lane / 16, zero behind the last row.  (Four rows of the tile are next to each other in the
// matrix; on the gate layout the units 4 t .. 4 t + 3 of a gate, rows 4 (unit) + gate of tile t.)  No branch per lane: a load in one is waited for there.
__device__ __forceinline__ void rows_of_step(const float *y, int step, int lane, int rows, int gate_h, float (&v)[16])
{
    const int tile = step * 4 + (lane >> 4), height = gate_h ? gate_h : rows, first = gate_h ? tile * 4 : tile * kTileRows;
    auto load = [&](auto whole) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = gate_h ? first : first + 4 * k;
            const float *const at = y + (gate_h ? (size_t)k * gate_h : 0);
            float4_at4 x;
            if constexpr (decltype(whole)::value) {
                x = *reinterpret_cast<const float4_at4 *>(at + r);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = at[min(r + i, height - 1)];
                    if (r + i >= height) x[i] = 0.0f;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (gate_h) v[4 * i + k] = x[i];
                else v[4 * k + i] = x[i];
            }
        }
    };
    if ((step * 4 + 4) * (gate_h ? 4 : kTileRows) <= height) load(std::integral_constant<bool, true>());
    else load(std::integral_constant<bool, false>());
}
// Their digits, rint(v 2^e): the sixteen bytes of each
__device__ __forceinline__ void digits_of(const float (&v)[16], int e, int balance, u32x4 (&out)[4])
{
    int g[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) g[i] = e == kNotFinite ? 0 : (__float2int_rn(ldexpf(v[i], e)) + balance) ^ balance;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const uint32_t a = __builtin_amdgcn_perm(g[4 * r + 1], g[4 * r], 0x05010400u), b = __builtin_amdgcn_perm(g[4 * r + 3], g[4 * r + 2], 0x05010400u);
        const uint32_t c = __builtin_amdgcn_perm(g[4 * r + 1], g[4 * r], 0x07030602u), d = __builtin_amdgcn_perm(g[4 * r + 3], g[4 * r + 2], 0x07030602u);
        out[0][r] = __builtin_amdgcn_perm(b, a, 0x05040100u);
        out[1][r] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        out[2][r] = __builtin_amdgcn_perm(d, c, 0x05040100u);
        out[3][r] = __builtin_amdgcn_perm(d, c, 0x07060302u);
    }
}

// The digits in memory: [group of 16 vectors][step of 64 packed rows][digit][lane 16 kb + v][16 bytes], the bytes being the
// sixteen rows of row tile 4 step + kb of vector v: an operand of a digit of sixteen vectors is 1 KB in one piece.  A wave writes one step.
// SCALES: every workgroup works the scalings of its sixteen vectors out by itself, a wave each, and the first of them leaves them in memory (a launch
// less; the vectors are read once per workgroup of sixteen steps).
template <bool SCALES>
__global__ __launch_bounds__(SCALES ? 1024 : 256) void k_grad_digits(const float *__restrict__ dY, Scaling *__restrict__ scalings, int batch, int rows,
                                                                     int gate_h, int steps, int may_narrow, uint8_t *__restrict__ digits)
{
    const int lane = threadIdx.x & 63, step = blockIdx.x * (SCALES ? 16 : 4) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = blockIdx.y, n = group * kGroupVectors + (lane & 15);
    Scaling sc = {kNotFinite, kNotFinite, 0, 0};
    if constexpr (SCALES) {
        __shared__ Scaling s_scalings[kGroupVectors];
        const int mine = group * kGroupVectors + (threadIdx.x >> 6);
        if (mine < batch) {
            const float *const y = dY + (size_t)mine * rows;
            Size size;
            size.take(y, rows, lane, 64);
            size.over_wave();
            if (lane == 0) {
                const Scaling s = scaling_of(size.most, size.squares, rows);
                s_scalings[threadIdx.x >> 6] = s;
                if (blockIdx.x == 0) scalings[mine] = s;
            }
        }
        __syncthreads();
        if (n < batch) sc = s_scalings[lane & 15];
    } else {
        if (n < batch) sc = scalings[n];
    }
    if (step >= steps) return;
    const bool narrow = may_narrow && !group_is_wide(sc, n < batch);
    const int e = narrow ? sc.e3 : sc.e4;
    float v[16];
    rows_of_step(dY + (size_t)min(n, batch - 1) * rows, step, lane, rows, gate_h, v);
    u32x4 out[4];
    digits_of(v, e, narrow ? 0x8080 : 0x808080, out);
    u32x4 *dst = reinterpret_cast<u32x4 *>(digits + ((size_t)group * steps + step) * 4096) + lane;
#pragma unroll
    for (int d = 0; d < 4; ++d)
        if (d < 3 || !narrow) dst[64 * d] = out[d];
}

// The same rows of [dg; du] = [dH u act'(g); dH act(g)] on the gate layout, from the pre-activations [g; u] and dH of the vector: a tile has the gates and
// the values of its units.  They go to `dpre` too, if that is given.
__device__ __forceinline__ void gated_rows_of_step(const float *pre, const float *dh, float *dpre, int gate, int step, int lane, int gate_h, float (&v)[16])
{
    const int first = (step * 4 + (lane >> 4)) * 4;
    float4_at4 x[4], h[2], out[4];      // x: gates of units first .. + 3 and gate_h + first .. + 3, then their values
    auto load = [&](const float *at, auto whole) {
        float4_at4 r;
        if constexpr (decltype(whole)::value) {
            r = *reinterpret_cast<const float4_at4 *>(at + first);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float one = at[min(first + i, gate_h - 1)];
                r[i] = first + i < gate_h ? one : 0.0f;
            }
        }
        return r;
    };
    auto load_all = [&](auto whole) {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = load(pre + (size_t)k * gate_h, whole);
#pragma unroll
        for (int k = 0; k < 2; ++k) h[k] = load(dh + (size_t)k * gate_h, whole);
    };
    if ((step * 4 + 4) * 4 <= gate_h) load_all(std::integral_constant<bool, true>());
    else load_all(std::integral_constant<bool, false>());
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float act, slope;
            gate_with_slope(gate, x[k][i], &act, &slope);
            v[4 * i + k] = out[k][i] = h[k][i] * x[2 + k][i] * slope;
            v[4 * i + 2 + k] = out[2 + k][i] = h[k][i] * act;
        }
    if (!dpre) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float *const at = dpre + (size_t)k * gate_h + first;
        if (first + 4 <= gate_h) {
            *reinterpret_cast<float4_at4 *>(at) = out[k];
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (first + i < gate_h) at[i] = out[k][i];
        }
    }
}

struct GradArgs {
    const uint32_t *packed;
    uint32_t packed_bytes, layer_step, round_step;   // (as in I8Args)
    int rt_count, cq, m, batch, cols;
    int steps, steps_per_split;                      // steps of 64 packed rows
    const float *scales;
    const uint8_t *digits;
    const Scaling *scalings;
    int may_narrow;
    float *out;                                      // [split][batch][cols]
    const float *dY;                                 // (FUSED)
    int rows, gate_h, held;                          // held: vectors in LDS, 4, 8 or 16
    int blocks, rows_of, workgroups;                 // column blocks, groups of vectors
    GatedSource gated;                               // (GATED)

    // What workgroup `id` does.  Workgroups go round the eight XCDs, each with an L2 of its own: those of an XCD (id % 8) take a contiguous range of an
    // order in which eight column blocks (two to a line of weights) and then the vectors are next to each other, and read less of both.
    __device__ void place(int id, int *block, int *vectors, int *split) const
    {
        const int each = workgroups / 8, rest = workgroups % 8, xcd = id % 8;
        int at = xcd * each + min(xcd, rest) + id / 8;
        *split = at / (blocks * rows_of);
        at -= *split * (blocks * rows_of);
        const int wide = at / (8 * rows_of), width = min(8, blocks - wide * 8);
        at -= wide * 8 * rows_of;
        *vectors = at / width;
        *block = wide * 8 + at % width;
    }
};

// The shape of a workgroup of eight waves: WM of them lie along the vectors (sixteen each), the others along the columns, NT operands of sixteen
// columns each.  Its codes are in two buffers of 64 KB: `columns` of a chunk's 512 and as many row tiles as fit.
template <int WM>
struct GradShape {
    static constexpr int WN = 8 / WM, NT = WM == 1 ? 4 : 8;
    static constexpr int GROUPS = WN * NT;               // operands of a row tile: 32, 16, 8
    static constexpr int PARTS = 32 / GROUPS;            // workgroups that share a chunk
    static constexpr int TILES = 256 / GROUPS;           // row tiles in a buffer
    static constexpr int KS = TILES / 4;                 // steps of 64 rows in a buffer
    static constexpr int TILE = GROUPS * 256 + 128;      // (the row tiles of an operand start in different halves of the banks)
    static constexpr int LDS = 2 * TILES * TILE;
};

// While a wave multiplies the codes of one buffer, it turns its share of the words of the next one into codes: four words of each bitlayer per
// lane, loaded with 16 bytes each (the vector-memory pipeline takes 16 cycles for a wave's load whatever its width).
// FUSED: the workgroup scales the gradients of its rows by their own largest and keeps their digits in LDS, behind the codes.
constexpr int kFusedSteps = 28;           // of four vectors; of eight half of them, of sixteen a quarter
constexpr int kFusedLds = kFusedSteps * 1024;
// GATED: these gradients are those of the pre-activations of a gated block on the gate layout, worked out here; every wave has one step at most, and
// the workgroups of the first columns leave them in memory.  us, with k_gated_grad before it / inside: 5460 x 1000, 4 bitlayers, 40 vectors 18.1 / 16.3;
// 5460 x 1024, 8 bitlayers, one vector 14.3 / 12.2, 16 vectors 17.2 / 16.0.
constexpr int kGatedSteps = 8;
template <int Q, bool IL, int WM, bool FUSED, bool GATED = false>
__global__ __launch_bounds__(512) void k_grad(const GradArgs a)
{
    static_assert((!FUSED || WM == 1) && (!GATED || FUSED));
    using S = GradShape<WM>;
    constexpr int WN = S::WN, NT = S::NT, TILES = S::TILES, KS = S::KS, TILE = S::TILE, BUF = TILES * TILE;
    extern __shared__ __align__(16) unsigned char s_codes[];
    __shared__ float s_scales[PB_MAX_BITS];
    __shared__ uint32_t s_most[FUSED ? 8 : 1][16];
    __shared__ int s_exponents[16];

    const int lane = threadIdx.x & 63, kb = lane >> 4, j = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = WN == 1 ? 0 : wave / WM;
    int block, vectors, split;
    a.place(blockIdx.x, &block, &vectors, &split);
    const int q = block / S::PARTS, part_of_chunk = block % S::PARTS;
    const int group = vectors * WM + wm;
    const int step0 = split * a.steps_per_split, step1 = min(step0 + a.steps_per_split, a.steps);   // (not empty)
    const int loops = (step1 - step0 + KS - 1) / KS;
    const int m = a.m;

    // (FUSED) the values of the wave's first step, which stay in registers
    const float *const y = FUSED && !GATED ? a.dY + (size_t)min(group * kGroupVectors + j, a.batch - 1) * a.rows : nullptr;
    float held[16];
    if constexpr (GATED) {
        const size_t n = (size_t)min(group * kGroupVectors + j, a.batch - 1);
        const bool writes = block == 0 && step0 + wave < step1 && group * kGroupVectors + j < a.batch;
        gated_rows_of_step(a.gated.pre + n * a.rows, a.gated.dH + n * (a.rows / 2), writes ? a.gated.dpre + n * a.rows : nullptr, a.gated.gate,
                           min(step0 + wave, step1 - 1), lane, a.gate_h, held);
    } else if constexpr (FUSED) {
        rows_of_step(y, min(step0 + wave, step1 - 1), lane, a.rows, a.gate_h, held);
    }

    // the scales: whether they halve (as in k_i8_tile)
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(a.scales), 0, m * 4, 0x00020000);
    const float scv = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, lane * 4, 0, 0));
    const float scn = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, lane * 4 + 4, 0, 0));
    if (wave == 0 && lane < PB_MAX_BITS) s_scales[lane] = scv;
    const bool off = lane + 1 < m && !(scv == (lane == 0 ? -2.0f : 2.0f) * scn);
    const bool merged = __builtin_amdgcn_ballot_w64(off) == 0;
    const int gs0 = merged ? 4 * Q : 1, gs1 = merged ? 4 * Q - 2 : 1;

    // the wave's share of a buffer: TILES / 8 row tiles, of each of which PER lanes read one piece; a lane has four words of a row
    constexpr int PER = 512 / TILES;
    const int my_tile = wave * (TILES / 8) + lane / PER, my_piece = lane % PER;
    const uint32_t my_at = (uint32_t)(lane / PER) * a.round_step + (uint32_t)(part_of_chunk * PER + my_piece) * 16u;
    unsigned char *const my_codes = s_codes + my_tile * TILE + (my_piece >> 4) * 2048 + (my_piece & 15) * 16;
    // the digits of the wave's vectors in these steps (nothing beyond them, and nothing for a group without vectors)
    const __amdgpu_buffer_rsrc_t rd = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t *>(a.digits) + ((size_t)group * a.steps + step0) * 4096, 0,
        !FUSED && group * kGroupVectors < a.batch ? (step1 - step0) * 4096 : 0, 0x00020000);
    unsigned char *const s_digits = s_codes + S::LDS;      // [step][digit][kb][vector][16 bytes]
    // the digits of the workgroup's rows: a wave has every eighth step (those behind its first are read again)
    auto convert = [&] {
        float v[16];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) most = max(most, __float_as_uint(held[i]) & 0x7FFFFFFFu);
        if constexpr (!GATED) {
#pragma unroll 1
            for (int s = step0 + wave + 8; s < step1; s += 8) {
                rows_of_step(y, s, lane, a.rows, a.gate_h, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
            }
        }
        most = max(most, (uint32_t)__shfl_xor((int)most, 16));
        most = max(most, (uint32_t)__shfl_xor((int)most, 32));
        if (lane < 16) s_most[wave][lane] = most;
        __syncthreads();
#pragma unroll
        for (int x = 0; x < 8; ++x) most = max(most, s_most[x][j]);
        const int e = scaling_of(most, 0.0, 0).e4;
        if (threadIdx.x < 16) s_exponents[threadIdx.x] = e;
#pragma unroll 1
        for (int s = wave; s < step1 - step0; s += 8) {
            if (!GATED && s >= 8) rows_of_step(y, step0 + s, lane, a.rows, a.gate_h, held);
            u32x4 out[4];
            digits_of(held, e, 0x808080, out);
            if (j < a.held) {
#pragma unroll
                for (int d = 0; d < 4; ++d) *reinterpret_cast<u32x4 *>(s_digits + (((s * 4 + d) * 4 + kb) * a.held + j) * 16) = out[d];
            }
        }
    };
    // where the wave's operands begin in a buffer
    const unsigned char *const operands = s_codes + kb * TILE + wn * NT * 256 + j * 8;

    // everything of the sum over the rows with ND digits
    auto sum_up = [&](auto nd) {
        constexpr int ND = decltype(nd)::value;
        // digits at once: where the sums of four digits nearly fill the registers, the codes are read twice, for two digits each
        constexpr int DC = WM >= 4 && ND == 4 ? 2 : ND, TURNS = KS * (ND / DC);
        constexpr int BR = 3;                               // operands of codes on their way from LDS
        static_assert(TURNS % 2 == 0, "the digits of two turns share the registers");
        for (int f = 0, e; f < m; f = e) {
            e = min(m, f + (f == 0 ? gs0 : gs1));
            const int l0 = (f & ~1) == 0 ? 0 : (f & ~1) - 2;
            uint32_t mask[2 * Q];
#pragma unroll
            for (int p = 0; p < 2 * Q; ++p) {
                const int l = l0 + 2 * p;
                mask[p] = (l >= f && l < e ? 0xAAAAAAAAu : 0u) | (l + 1 >= f && l + 1 < e ? 0x55555555u : 0u);
            }
            const uint32_t flip = l0 == 0 ? 0xAAAAAAAAu : 0u;
            const Masks masks = make_masks();
            u32x4 w[4 * Q];
            // the words of buffer `loop`; those of row tiles beyond the end are zero
            const int end = min(a.rt_count, step1 * 4);
            auto inside = [&](int loop) { return (step0 + loop * KS) * 4 + my_tile < end; };
            auto issue = [&](int loop) {
                const uint32_t at = (uint32_t)((step0 + loop * KS) * 4 + wave * (TILES / 8)) * a.round_step + (uint32_t)q * 1024u;
                const int mine = inside(loop) ? (int)my_at : -16;      // (beyond every buffer)
#pragma unroll
                for (int s = 0; s < 4 * Q; ++s) {
                    const int l = l0 + s, lu = l0 + (s & ~1);
                    const bool has = loop < loops && (IL ? lu + 1 >= f && lu < e : l >= f && l < e);
                    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint32_t *>(a.packed), 0,
                                                                                        has ? (int)a.packed_bytes : 0, 0x00020000);
                    w[s] = __builtin_amdgcn_raw_buffer_load_b128(rw, mine, has ? (int)(at + (uint32_t)l * a.layer_step) : 0, 0);
                }
            };
            // The codes of a buffer from its words, word after word in the six steps of weight_codes(): 0, 1 pairs of words, 2, 3 nibbles, 4, 5 bytes and
            // their way to LDS, so that they can stand between the products of the other buffer.
            constexpr int STAGES = 24;
            uint64_t part[4];         // first h, l (then the nibbles' two halves), second h, l
            uint32_t keep[2 * Q];     // (IL)
            auto expand = [&](int stage, int loop, unsigned char *to) {
                const int t = stage / 6, o = stage & 1;
                if (stage % 6 < 2) {
                    if (stage == 0) {
#pragma unroll
                        for (int i = 0; i < 2 * Q; ++i) keep[i] = inside(loop) ? mask[i] : 0u;
                    }
                    if (o == 1 && Q == 1) return;      // (the upper or the lower four slots)
                    uint32_t p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[i] = w[4 * o + i][t];
                        if constexpr (IL) p[i] = (o == 0 && i < 2 ? p[i] ^ flip : p[i]) & keep[2 * o + i / 2];
                    }
                    if constexpr (IL) {
                        part[2 * o] = both(p[0], p[1]);
                        part[2 * o + 1] = both(p[2], p[3]);
                    } else {
                        part[2 * o] = both(pick(masks.m1, twice(p[0]), p[1]), pick(masks.m1, p[0], p[1] >> 1));
                        part[2 * o + 1] = both(pick(masks.m1, twice(p[2]), p[3]), pick(masks.m1, p[2], p[3] >> 1));
                    }
                } else if (stage % 6 < 4) {
                    if (o == 1 && Q == 1) return;
                    const uint64_t h = part[2 * o], l = part[2 * o + 1];
                    part[2 * o] = mix(masks.m2, up<2>(h), l);
                    part[2 * o + 1] = mix(masks.m2, h, down<2>(l));
                } else {
                    v4i out;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint64_t x = part[k], y = Q == 2 ? part[2 + k] : 0;
                        const uint64_t r = o ? mix(masks.m4, x, Q == 2 ? down<4>(y) : 0) : mix(masks.m4, up<4>(x), y);
                        out[2 * k] = (int)(uint32_t)r;
                        out[2 * k + 1] = (int)(r >> 32);
                    }
                    *reinterpret_cast<v4i *>(to + t * 512 + o * 256) = out;
                }
            };
            u32x4 ar[2][DC];
            auto load_digits = [&](u32x4 (&dst)[DC], int step, int from) {
#pragma unroll
                for (int d = 0; d < DC; ++d) {
                    if constexpr (FUSED)      // (lanes and steps beyond have others' digits: their vectors are not stored, their codes are zero)
                        dst[d] = *reinterpret_cast<const u32x4 *>(s_digits + ((min(step, step1 - step0 - 1) * 4 + from + d) * 4 + kb) * a.held * 16 + min(j, a.held - 1) * 16);
                    else
                        dst[d] = __builtin_amdgcn_raw_buffer_load_b128(rd, lane * 16, step * 4096 + (from + d) * 1024, 0);
                }
            };
            issue(0);
            if constexpr (FUSED) {
                if (f == 0) convert();
            } else {
                load_digits(ar[0], 0, 0);
            }
#pragma unroll
            for (int i = 0; i < STAGES; ++i) {
                expand(i, 0, my_codes);
                __builtin_amdgcn_sched_barrier(0);
            }
            issue(1);
            __syncthreads();
            if constexpr (FUSED) load_digits(ar[0], 0, 0);
            v4i acc[ND][NT];
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[d][nt] = v4i{0, 0, 0, 0};
            for (int loop = 0; loop < loops; ++loop) {
                const int here = loop & 1 ? BUF : 0;
                const unsigned char *src = operands + here;
                unsigned char *const to = my_codes + (BUF - here);
                // operand nt of step k of the buffer
                auto codes = [&](int k, int nt) {
                    const unsigned char *at = src + k * 4 * TILE + nt * 256;
                    const v2i x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((v2i __attribute__((address_space(3))) *)(at));
                    const v2i y = __builtin_amdgcn_ds_read_tr8_b64_v2i32((v2i __attribute__((address_space(3))) *)(at + 128));
                    return v4i{x[0], x[1], y[0], y[1]};
                };
                v4i br[BR];
#pragma unroll
                for (int i = 0; i < BR - 1; ++i) br[i] = codes(0, i);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int k = 0; k < TURNS; ++k) {
                    // (turn k: step k / (TURNS / KS) of the buffer, the digits from k % (TURNS / KS) * DC on)
                    load_digits(ar[(k + 1) & 1], loop * KS + (k + 1) / (TURNS / KS), (k + 1) % (TURNS / KS) * DC);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const int i = k * NT + nt, ahead = i + BR - 1;
                        if (ahead < TURNS * NT) br[ahead % BR] = codes(ahead / NT / (TURNS / KS), ahead % NT);
                        // (the next buffer's codes, in the first half of the loop: the words after them then have the second half to arrive)
                        constexpr int AT_ONCE = 48 / (TURNS * NT) > 1 ? 48 / (TURNS * NT) : 1;
#pragma unroll
                        for (int x = AT_ONCE * i; x < AT_ONCE * i + AT_ONCE && x < STAGES; ++x) {
                            expand(x, loop + 1, to);
                            if (x == 19) issue(loop + 2);       // (the last word has been taken)
                        }
#pragma unroll
                        for (int d = 0; d < DC; ++d) {
                            v4i &sum = acc[k % (TURNS / KS) * DC + d][nt];
                            sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, ar[k & 1][d]), br[i % BR], sum, 0, 0, 0);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __syncthreads();
            }
            // ---- a lane has column j of every sixteen and the vectors 4 kb + c ----
            int at = lane;
            asm volatile("" : "+v"(at));       // (the addresses of the results are worked out here and not kept during the loop)
            const int jj = at & 15, first = group * kGroupVectors + (at >> 4) * 4;
            const int slot = e - 1 - l0;
            const double s = (double)s_scales[e - 1], gscale = ldexp(slot == 0 ? -s : s, slot - 7);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int n = first + c;
                if (n < a.batch) {
                    const int ex = FUSED ? s_exponents[n % kGroupVectors] : (ND == 3 ? a.scalings[n].e3 : a.scalings[n].e4);
                    const double factor = ex == kNotFinite ? (double)NAN : ldexp(gscale, -ex);
                    float *out = a.out + ((size_t)split * a.batch + n) * a.cols;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const int g = wn * NT + nt, h = g & 1, word = part_of_chunk * (16 / S::PARTS) + (g >> 1);
                        const int col = q * 512 + word * 32 + 8 * (jj & 3) + 4 * h + (jj >> 2);
                        if (col < a.cols) {
                            double v = fma(256.0, (double)acc[1][nt][c], (double)acc[0][nt][c]);
                            v = fma(65536.0, (double)acc[2][nt][c], v);
                            if constexpr (ND == 4) v = fma(16777216.0, (double)acc[3][nt][c], v);
                            const float y = (float)(v * factor);
                            out[col] = f == 0 ? y : out[col] + y;      // (later groups of bitlayers add to the thread's own result)
                        }
                    }
                }
            }
            __syncthreads();
        }
    };
    // (the waves of a workgroup may differ: both ways pass the same barriers)
    if constexpr (WM >= 4) {
        const int n = group * kGroupVectors + j;
        Scaling mine = {0, 0, 0, 0};
        if (n < a.batch) mine = a.scalings[n];
        if (a.may_narrow && !group_is_wide(mine, n < a.batch)) {
            sum_up(std::integral_constant<int, 3>{});
            return;
        }
        sum_up(std::integral_constant<int, 4>{});
    } else {
        sum_up(std::integral_constant<int, 4>{});
    }
}

__global__ __launch_bounds__(256) void k_grad_join(const GradParts p) { join_parts(p, ((size_t)blockIdx.x * 256 + threadIdx.x) * 2); }

// ---------------------------------------------------------------------------------------------------------------

// How a call is shared out; the workspace holds [scalings][digits][parts of the split sum]
struct GradPlan {
    int wm, blocks, ks, steps, splits, steps_per_split, held;       // held: 0, or the digits are made by k_grad
    size_t digits_off, parts_off;
};
constexpr int kGradCus = 256;
// A workspace has to serve every smaller batch too, and the fastest number of parts goes up and down with the batch: the parts together get no more room
// than this, which grows with the batch.  64 MB, or three times dX (more parts than that paid in 3 of 1000 drawn calls, by 3 % of the estimated time).
static int least_parts(int steps) { return (steps + 1023) / 1024; }       // (int32 sums: 65536 rows)
static size_t parts_room(const Layout &L, int steps, int batch)
{
    const size_t one = (size_t)batch * L.cols * 4, most = (size_t)((steps + 1) / 2), least = (size_t)least_parts(steps);
    const size_t few = (least > 3 ? least : 3) * one, room = few > (64u << 20) ? few : 64u << 20;
    return most > 1 ? (most * one < room ? most * one : room) : 0;
}
static size_t digits_offset(int batch) { return ((size_t)batch * sizeof(Scaling) + 255) & ~(size_t)255; }
static size_t digits_bytes(int steps, int batch) { return (size_t)((batch + 15) / 16) * (size_t)steps * 4096; }
static GradPlan grad_plan(const Layout &L, int batch)
{
    GradPlan p;
    p.steps = (L.rt_count + 3) / 4;
    const size_t room = parts_room(L, p.steps, batch);
    double least_time = 1e30;
    // The shape: one wave along the vectors for up to 32, four for up to 64, eight for more, or one all the same where that is estimated to be faster
    // (the digits then need no launch).  us, digits in launches of their own / in k_grad: 670 x 2642, 71 vectors 20.0 / 13.8; 1024 x 1024, 128 vectors
    // 18.4 / 13.7; 2048 x 2048, 48 vectors 20.0 / 14.6; 801 x 1549, 282 vectors 21.0 / 16.1; 8192 x 8192, 4 vectors 27.3 / 20.3; 4096 x 4096, 16 vectors
    // 22.0 / 17.1.  (Two waves along 17 to 32 vectors were slower than two workgroups with one: 8192 x 8192, 32 vectors 32.8, 30.7.)
    for (int wm = batch <= 32 ? 1 : (batch <= 64 ? 4 : 8); wm; wm = wm > 1 ? 1 : 0) {
        const int blocks = L.cq * (wm == 8 ? 4 : (wm == 4 ? 2 : 1)), ks = wm == 8 ? 8 : (wm == 4 ? 4 : 2);
        const int rows_of = (batch + 16 * wm - 1) / (16 * wm), held = wm > 1 ? 0 : (batch <= 4 ? 4 : (batch <= 8 ? 8 : 16));
        // Parts of the sum: rounds of workgroups over the chip (one per compute unit), each of so many us for its start and end and for a step; more
        // than one part costs the way of the parts through memory and a launch, digits that do not fit a workgroup a launch or two.
        const double step = wm == 8 ? 0.67 : (wm == 4 ? 0.75 : 1.5);
        for (int splits = least_parts(p.steps), n = 0; n < 64; ++splits, ++n) {
            const int each = ((p.steps + splits - 1) / splits + ks - 1) / ks * ks, parts = (p.steps + each - 1) / each;   // (whole buffers)
            if (parts < splits && n) continue;
            if (parts > 1 && (size_t)parts * batch * L.cols * 4 > room) break;
            const bool fits = held && each * held <= kFusedSteps * 4;
            const double rounds = (double)(((long long)blocks * rows_of * parts + kGradCus - 1) / kGradCus);
            const double time = (fits ? 0.0 : 4.0 + (batch > 16 ? 2.0 : 0.0)) + rounds * (3.0 + (fits ? 2.0 : 0.0) + step * each) +
                                (parts > 1 ? 3.0 + (parts + 2) * 4e-6 * batch * L.cols / 4.0 : 0.0);
            if (time < least_time) {
                least_time = time;
                p.wm = wm; p.blocks = blocks; p.ks = ks; p.splits = parts; p.steps_per_split = each; p.held = fits ? held : 0;
            }
        }
    }
    p.digits_off = digits_offset(batch);
    p.parts_off = p.digits_off + (p.held ? 0 : digits_bytes(p.steps, batch));
    return p;
}
// (the digits count also where k_grad makes them: a smaller batch may have them in memory)
size_t grad_workspace_bytes(const Layout &L, int batch)
{
    const int steps = (L.rt_count + 3) / 4;
    return digits_offset(batch) + digits_bytes(steps, batch) + ((parts_room(L, steps, batch) + 255) & ~(size_t)255);
}

#define PB_GRAD(WM, FUSED) {{reinterpret_cast<const void *>(k_grad<1, false, WM, FUSED>), reinterpret_cast<const void *>(k_grad<1, true, WM, FUSED>)}, \
                            {reinterpret_cast<const void *>(k_grad<2, false, WM, FUSED>), reinterpret_cast<const void *>(k_grad<2, true, WM, FUSED>)}}
static const void *const kGradFn[5][2][2] = {PB_GRAD(1, false), PB_GRAD(4, false), PB_GRAD(8, false), PB_GRAD(1, true),
                                             {{reinterpret_cast<const void *>(k_grad<1, false, 1, true, true>), nullptr},
                                              {reinterpret_cast<const void *>(k_grad<2, false, 1, true, true>), nullptr}}};
constexpr int kGradLds[5] = {GradShape<1>::LDS, GradShape<4>::LDS, GradShape<8>::LDS, GradShape<1>::LDS + kFusedLds, GradShape<1>::LDS + kFusedLds};

int launch_grad(const uint32_t *packed, const float *scales, const Layout &L, int bits_used, const float *dY, const GatedSource *gated,
                int batch, float *dX, void *workspace, hipStream_t st, AdapterDown *down)
{
    const GradPlan p = grad_plan(L, batch);
    char *const ws = static_cast<char *>(workspace);
    Scaling *const scalings = reinterpret_cast<Scaling *>(ws);
    uint8_t *const digits = reinterpret_cast<uint8_t *>(ws + p.digits_off);
    // Whether the workgroups of the digits work the scalings out themselves: up to 128 KB of vectors each.  us with it / with a launch of its own:
    // 2000 x 2000, 1000 vectors 35.6 / 38.2; 4096 columns, 1000 rows, 1000 vectors 27.2 / 29.7; 2048 x 2048, 256 vectors 24.4 / 24.2; but 1800 columns, 4100
    // rows, 104 vectors (262 KB) 24.4 / 23.2; 4096 x 4096, 64 vectors (262 KB) 29.2 / 28.4.
    const bool own = !gated && !p.held && (long long)(batch < 16 ? batch : 16) * L.rows <= 32768;
    const bool gated_inside = gated && p.held && L.gate_h && p.steps_per_split <= kGatedSteps;
    int err = 0;
    if (gated && !gated_inside) {
        hipLaunchKernelGGL(k_gated_grad, dim3((unsigned)batch), dim3(1024), 0, st, gated->pre, gated->dH, L.rows / 2, gated->gate, gated->dpre,
                           scalings);
        dY = gated->dpre;
    } else if (!gated && !own && !p.held) {
        if (down) {
            err = launch_adapter_down_scalings(down, dY, batch, scalings, st);
            if (err) return err;
        } else {
            hipLaunchKernelGGL(k_grad_scalings, dim3((unsigned)batch), dim3(1024), 0, st, dY, L.rows, scalings);
        }
    }
    err = (int)hipGetLastError();
    if (err) return err;
    const int waves = own ? 16 : 4, may_narrow = p.wm >= 4;
    if (!p.held)
        hipLaunchKernelGGL(own ? k_grad_digits<true> : k_grad_digits<false>,
                           dim3((unsigned)((p.steps + waves - 1) / waves), (unsigned)((batch + 15) / 16)), dim3((unsigned)waves * 64), 0, st, dY,
                           scalings, batch, L.rows, L.gate_h, p.steps, may_narrow, digits);
    err = (int)hipGetLastError();
    if (err) return err;
    GradArgs a;
    a.packed = packed;
    a.packed_bytes = (uint32_t)packed_bytes(L);
    a.layer_step = (uint32_t)(tile16_layer_stride(L) * 4);
    a.round_step = (uint32_t)(tile16_rowtile_stride(L) * 4);
    a.rt_count = L.rt_count; a.cq = L.cq; a.m = bits_used; a.batch = batch; a.cols = L.cols;
    a.steps = p.steps; a.steps_per_split = p.steps_per_split;
    a.scales = scales; a.digits = digits; a.scalings = scalings; a.may_narrow = may_narrow;
    a.dY = dY; a.rows = L.rows; a.gate_h = L.gate_h; a.held = p.held;
    a.blocks = p.blocks; a.rows_of = (batch + 16 * p.wm - 1) / (16 * p.wm);
    a.workgroups = a.blocks * a.rows_of * p.splits;
    float *const parts = reinterpret_cast<float *>(ws + p.parts_off);
    a.out = p.splits > 1 ? parts : dX;
    if (gated) a.gated = *gated;
    const int shape = gated_inside ? 4 : p.held ? 3 : (p.wm == 8 ? 2 : p.wm / 4), wide = bits_used > 4, il = is_pairs(L.layout);
    const void *fn = kGradFn[shape][wide][il];
    static uint64_t declared[5][2][2];
    err = declare_lds(fn, (size_t)kGradLds[shape], &declared[shape][wide][il]);
    if (err) return err;
    void *args[] = {&a};
    hipError_t e = hipLaunchKernel(fn, dim3((unsigned)a.workgroups), dim3(512), args, (size_t)kGradLds[shape], st);
    if (e == hipSuccess) e = hipGetLastError();
    if (e != hipSuccess) return (int)e;
    if (p.splits > 1) {
        const size_t total = (size_t)batch * L.cols;
        const GradParts joined = {parts, dX, total, p.splits};
        if (down && !down->done) return launch_adapter_down_join(down, joined, batch, st);
        hipLaunchKernelGGL(k_grad_join, dim3((unsigned)((total + 511) / 512)), dim3(256), 0, st, joined);
        e = hipGetLastError();
    }
    return (int)e;
}

}  // namespace pb
