// Gradient through a packed matrix: dX[n][c] = sum_r dY[n][r] w[r][c], w[r][c] = sum_(i < bits_used) scales[i] bit_i[r][c], on the
// 8-bit integer matrix cores (pb_imma.h has the codes of the weights).
//
// dY as digits.  A vector's gradients are scaled by the power of two that brings the largest one below 2^30, rounded to integers g and
// split into four balanced byte digits, g = sum_d 256^d s_d with s_d in [-128, 127]: the bytes of (g + 0x808080) ^ 0x808080, because
// 0x808080 = sum_(d < 3) 256^d 128.  The rounding (half a unit, 2^-31 of the vector's largest gradient) is the only one before the last
// step: |s code| <= 2^14, so a sum over 65536 rows is exact in int32, and the digits' sums are put together in fp64.
//
// The sum runs over the rows of W, and a packed word holds 32 columns of one row: the codes have to be turned, 16 rows of a column
// into the 16 bytes of a lane.  They go through LDS anyway, because every wave needs them, and DS_READ_B64_TR_B8 turns them on the
// way out: its 16 lanes read eight rows of sixteen bytes, and lane i receives byte i of each.
#include <type_traits>

#include "pb_imma.h"

namespace pb {

typedef int v2i __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kNotFinite = INT32_MIN;      // in the place of an exponent: the vector's results are NaN

// The exponent e of every vector: its gradients enter as rint(dy 2^e)
__device__ __forceinline__ int exponent_of(uint32_t largest)     // (bits of the largest magnitude)
{
    if (largest >= 0x7F800000u) return kNotFinite;
    if (largest == 0) return 0;
    int e;
    frexpf(__uint_as_float(largest), &e);
    return 30 - e;
}

// The largest of a value per thread, in thread 0
template <int WAVES>
__device__ __forceinline__ uint32_t largest_of_workgroup(uint32_t v)
{
    __shared__ uint32_t s_max[WAVES];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v = max(v, s_max[w]);
    }
    return v;
}

__global__ __launch_bounds__(1024) void k_grad_exponents(const float *__restrict__ dY, int rows, int *__restrict__ exps)
{
    const float *y = dY + (size_t)blockIdx.x * rows;
    uint32_t most = 0;
    for (int r = threadIdx.x; r < rows; r += 1024) most = max(most, __float_as_uint(y[r]) & 0x7FFFFFFFu);
    most = largest_of_workgroup<16>(most);
    if (threadIdx.x == 0) exps[blockIdx.x] = exponent_of(most);
}

// Gradients of the pre-activations [g; u] of H = act(g) u, and the exponents of their vectors
__global__ __launch_bounds__(1024) void k_gated_grad(const float *__restrict__ pre, const float *__restrict__ dH, int units, int gate,
                                                     float *__restrict__ dpre, int *__restrict__ exps)
{
    const size_t n = blockIdx.x;
    const float *g = pre + n * 2 * units, *u = g + units, *dh = dH + n * units;
    float *dg = dpre + n * 2 * units, *du = dg + units;
    uint32_t most = 0;
    for (int r = threadIdx.x; r < units; r += 1024) {
        float a, da;
        gate_with_slope(gate, g[r], &a, &da);
        const float x = dh[r] * u[r] * da, y = dh[r] * a;
        dg[r] = x;
        du[r] = y;
        most = max(most, max(__float_as_uint(x) & 0x7FFFFFFFu, __float_as_uint(y) & 0x7FFFFFFFu));
    }
    most = largest_of_workgroup<16>(most);
    if (threadIdx.x == 0) exps[n] = exponent_of(most);
}

// The digits in memory: [group of 16 vectors][step of 64 packed rows][digit][lane 16 kb + v][16 bytes], the bytes being the
// sixteen rows of row tile 4 step + kb of vector v: an operand of a digit of sixteen vectors is 1 KB in one piece.  A wave writes one step.
__global__ __launch_bounds__(256) void k_grad_digits(const float *__restrict__ dY, const int *__restrict__ exps, int batch, int rows,
                                                     int gate_h, int steps, uint8_t *__restrict__ digits)
{
    const int lane = threadIdx.x & 63, step = blockIdx.x * 4 + (threadIdx.x >> 6), group = blockIdx.y;
    if (step >= steps) return;
    const int n = group * kGroupVectors + (lane & 15), tile = step * 4 + (lane >> 4);
    const int e = n < batch ? exps[n] : kNotFinite;
    int g[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int r = gate_h ? gates_matrix_row(tile * kTileRows + i, gate_h) : tile * kTileRows + i;
        const bool live = e != kNotFinite && r >= 0 && r < rows;
        const float y = live ? dY[(size_t)n * rows + r] : 0.0f;
        g[i] = live ? (__float2int_rn(ldexpf(y, e)) + 0x808080) ^ 0x808080 : 0;
    }
    u32x4 out[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const uint32_t a = __builtin_amdgcn_perm(g[4 * r + 1], g[4 * r], 0x05010400u), b = __builtin_amdgcn_perm(g[4 * r + 3], g[4 * r + 2], 0x05010400u);
        const uint32_t c = __builtin_amdgcn_perm(g[4 * r + 1], g[4 * r], 0x07030602u), d = __builtin_amdgcn_perm(g[4 * r + 3], g[4 * r + 2], 0x07030602u);
        out[0][r] = __builtin_amdgcn_perm(b, a, 0x05040100u);
        out[1][r] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        out[2][r] = __builtin_amdgcn_perm(d, c, 0x05040100u);
        out[3][r] = __builtin_amdgcn_perm(d, c, 0x07060302u);
    }
    u32x4 *dst = reinterpret_cast<u32x4 *>(digits + ((size_t)group * steps + step) * 4096) + lane;
#pragma unroll
    for (int d = 0; d < 4; ++d) dst[64 * d] = out[d];
}

struct GradArgs {
    const uint32_t *packed;
    uint32_t packed_bytes, layer_step, round_step;   // (as in I8Args)
    int rt_count, cq, m, batch, cols;
    int steps, steps_per_split;                      // steps of 64 packed rows
    const float *scales;
    const uint8_t *digits;
    const int *exps;
    float *out;                                      // [split][batch][cols]
};

// A workgroup of eight waves: WM of them along the vectors (sixteen each), the others along the columns: 512, or with WM = 4 half of
// the words of each lane's four, 256.  32 KB of codes at a time, two buffers: every wave turns two words of each bitlayer of a row tile
// into codes while it multiplies those of the other buffer.
template <int Q, bool IL, int WM>
__global__ __launch_bounds__(512) void k_grad(const GradArgs a)
{
    constexpr int WN = 8 / WM, NT = WM == 1 ? 4 : 8;
    constexpr int GROUPS = WN * NT;                      // of sixteen columns: 32 or 16
    constexpr int TILES = 128 / GROUPS;                  // row tiles in a buffer: 4 or 8
    constexpr int KS = TILES / 4;                        // steps of 64 rows in a buffer
    constexpr int BR = 3;                                // operands of codes on their way from LDS
    constexpr int TILE = GROUPS * 256 + 128;             // (the row tiles of an operand start in different halves of the banks)
    __shared__ __align__(16) unsigned char s_codes[2][TILES * TILE];
    __shared__ float s_scales[PB_MAX_BITS];

    const int lane = threadIdx.x & 63, kb = lane >> 4, j = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const int q = GROUPS == 32 ? blockIdx.x : blockIdx.x >> 1;
    const int group = blockIdx.y * WM + wm;
    const int step0 = blockIdx.z * a.steps_per_split, step1 = min(step0 + a.steps_per_split, a.steps);   // (not empty)
    const int loops = (step1 - step0 + KS - 1) / KS;
    const int m = a.m;
    const Masks masks = make_masks();

    // the scales: whether they halve (as in k_i8_tile)
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(a.scales), 0, m * 4, 0x00020000);
    const float scv = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, lane * 4, 0, 0));
    const float scn = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, lane * 4 + 4, 0, 0));
    if (wave == 0 && lane < PB_MAX_BITS) s_scales[lane] = scv;
    const bool off = lane + 1 < m && !(scv == (lane == 0 ? -2.0f : 2.0f) * scn);
    const bool merged = __builtin_amdgcn_ballot_w64(off) == 0;
    const int gs0 = merged ? 4 * Q : 1, gs1 = merged ? 4 * Q - 2 : 1;

    // the wave's part of the codes: row tile and two of four words
    const int my_tile = GROUPS == 32 ? wave >> 1 : wave, my_half = GROUPS == 32 ? wave & 1 : blockIdx.x & 1;
    unsigned char *const my_codes =
        &s_codes[0][0] + my_tile * TILE + (GROUPS == 32 ? (kb * 4 + my_half * 2) * 512 : kb * 2 * 512) + j * 16;
    const u32x4 *const dig = reinterpret_cast<const u32x4 *>(a.digits + (size_t)group * a.steps * 4096) + lane;
    const bool have = group * kGroupVectors < a.batch;
    // where the wave's operands begin in a buffer
    const unsigned char *const operands = &s_codes[0][0] + kb * TILE + wn * NT * 256 + j * 8;

    bool first = true;
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
        u32x2 w[4 * Q];
        // the words of buffer `loop` (beyond the last row tile they are zero)
        auto tile_of = [&](int loop) { return (step0 + loop * KS) * 4 + my_tile; };
        auto inside = [&](int loop) { return loop < loops && tile_of(loop) < min(a.rt_count, step1 * 4); };
        auto issue = [&](int loop) {
            const bool ok = inside(loop);
            const uint32_t at = (uint32_t)tile_of(loop) * a.round_step + (uint32_t)q * 1024u;
#pragma unroll
            for (int s = 0; s < 4 * Q; ++s) {
                const int l = l0 + s, lu = l0 + (s & ~1);
                const bool has = ok && (IL ? lu + 1 >= f && lu < e : l >= f && l < e);
                const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint32_t *>(a.packed), 0,
                                                                                    has ? (int)a.packed_bytes : 0, 0x00020000);
                w[s] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rw, lane * 16 + my_half * 8,
                                                                                     (int)(at + (uint32_t)l * a.layer_step), 0));
            }
        };
        auto expand = [&](int loop) {
            const bool in = inside(loop);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                uint32_t p[4 * Q];
#pragma unroll
                for (int s = 0; s < 4 * Q; ++s) {
                    p[s] = w[s][t];
                    if constexpr (IL) p[s] = (s < 2 ? p[s] ^ flip : p[s]) & (in ? mask[s / 2] : 0u);
                }
                v4i lo, hi;
                weight_codes<Q, IL, true>(masks, p, lo, hi);
                unsigned char *dst = my_codes + (loop & 1) * (TILES * TILE) + t * 512;
                *reinterpret_cast<v4i *>(dst) = lo;
                *reinterpret_cast<v4i *>(dst + 256) = hi;
            }
        };
        v4i acc[4][NT];
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[d][nt] = v4i{0, 0, 0, 0};
        u32x4 ar[2][4];
        auto load_digits = [&](u32x4 (&dst)[4], int step) {
            const u32x4 *src = dig + (size_t)min(step, a.steps - 1) * 256;
#pragma unroll
            for (int d = 0; d < 4; ++d) dst[d] = have ? src[64 * d] : u32x4{0, 0, 0, 0};
        };
        issue(0);
        load_digits(ar[0], step0);
        expand(0);
        issue(1);
        __syncthreads();
        for (int loop = 0; loop < loops; ++loop) {
            expand(loop + 1);
            issue(loop + 2);
            const unsigned char *src = operands + (loop & 1) * (TILES * TILE);
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
            for (int k = 0; k < KS; ++k) {
                const int step = step0 + loop * KS + k;
                // (a wave's steps alternate between two sets of registers only where a buffer has two)
                u32x4 (&now)[4] = ar[KS == 2 ? k : 0], (&next)[4] = ar[KS == 2 ? k ^ 1 : 1];
                load_digits(next, step + 1);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int i = k * NT + nt, ahead = i + BR - 1;
                    if (ahead < KS * NT) br[ahead % BR] = codes(ahead / NT, ahead % NT);
#pragma unroll
                    for (int d = 0; d < 4; ++d)
                        acc[d][nt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, now[d]), br[i % BR], acc[d][nt], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (KS == 1) {
#pragma unroll
                    for (int d = 0; d < 4; ++d) now[d] = next[d];
                }
            }
            __syncthreads();
        }
        // ---- a lane has column j of every sixteen and the vectors 4 kb + c ----
        int jj = j;
        asm volatile("" : "+v"(jj));       // (the addresses of the results are worked out here and not kept during the loop)
        const int slot = e - 1 - l0;
        const double s = (double)s_scales[e - 1], gscale = ldexp(slot == 0 ? -s : s, slot - 7);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int n = group * kGroupVectors + kb * 4 + c;
            if (n < a.batch) {
                const int ex = a.exps[n];
                const double factor = ex == kNotFinite ? (double)NAN : ldexp(gscale, -ex);
                float *out = a.out + ((size_t)blockIdx.z * a.batch + n) * a.cols;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int g = wn * NT + nt, h = g & 1, word = GROUPS == 32 ? g >> 1 : (g >> 2) * 4 + my_half * 2 + ((g >> 1) & 1);
                    const int col = q * 512 + word * 32 + 8 * (jj & 3) + 4 * h + (jj >> 2);
                    if (col < a.cols) {
                        const double v = fma(16777216.0, (double)acc[3][nt][c],
                                             fma(65536.0, (double)acc[2][nt][c], fma(256.0, (double)acc[1][nt][c], (double)acc[0][nt][c])));
                        const float y = (float)(v * factor);
                        out[col] = first ? y : out[col] + y;      // (later groups of bitlayers add to the thread's own result)
                    }
                }
            }
        }
        first = false;
        __syncthreads();
    }
}

// The parts of a split sum, in the order of the rows
__global__ __launch_bounds__(256) void k_grad_join(const float *__restrict__ parts, int splits, size_t total, float *__restrict__ dX)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    float v = parts[i];
    for (int s = 1; s < splits; ++s) v += parts[(size_t)s * total + i];
    dX[i] = v;
}

// ---------------------------------------------------------------------------------------------------------------

// How a call is shared out; the workspace holds [exponents][digits][parts of the split sum]
struct GradPlan {
    int wm, blocks, steps, splits, steps_per_split;
    size_t digits_off, parts_off, bytes;
};
constexpr int kGradCus = 256;
static GradPlan grad_plan(const Layout &L, int batch)
{
    GradPlan p;
    p.wm = batch <= 16 ? 1 : (batch <= 32 ? 2 : 4);
    p.blocks = L.cq * (p.wm == 4 ? 2 : 1);
    p.steps = (L.rt_count + 3) / 4;
    const int rows_of = (batch + 16 * p.wm - 1) / (16 * p.wm);
    int splits = kGradCus / (p.blocks * rows_of);
    if (splits > p.steps / 4) splits = p.steps / 4;
    if (splits < 1) splits = 1;
    const int least = (p.steps + 1023) / 1024;        // (int32 sums: 65536 rows)
    if (splits < least) splits = least;
    p.steps_per_split = ((p.steps + splits - 1) / splits + 1) & ~1;      // (whole buffers)
    p.splits = (p.steps + p.steps_per_split - 1) / p.steps_per_split;
    auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
    p.digits_off = up((size_t)batch * 4);
    p.parts_off = p.digits_off + (size_t)((batch + 15) / 16) * (size_t)p.steps * 4096;
    p.bytes = p.parts_off + (p.splits > 1 ? up((size_t)p.splits * batch * L.cols * 4) : 0);
    return p;
}
size_t grad_workspace_bytes(const Layout &L, int batch) { return grad_plan(L, batch).bytes; }

template <int WM>
static const void *grad_kernel(bool wide, bool il)
{
    if (wide) return il ? reinterpret_cast<const void *>(k_grad<2, true, WM>) : reinterpret_cast<const void *>(k_grad<2, false, WM>);
    return il ? reinterpret_cast<const void *>(k_grad<1, true, WM>) : reinterpret_cast<const void *>(k_grad<1, false, WM>);
}

int launch_grad(const uint32_t *packed, const float *scales, const Layout &L, int bits_used, const float *dY, const GatedSource *gated,
                int batch, float *dX, void *workspace, hipStream_t st)
{
    const GradPlan p = grad_plan(L, batch);
    char *const ws = static_cast<char *>(workspace);
    int *const exps = reinterpret_cast<int *>(ws);
    uint8_t *const digits = reinterpret_cast<uint8_t *>(ws + p.digits_off);
    if (gated) {
        hipLaunchKernelGGL(k_gated_grad, dim3((unsigned)batch), dim3(1024), 0, st, gated->pre, gated->dH, L.rows / 2, gated->gate, gated->dpre,
                           exps);
        dY = gated->dpre;
    } else {
        hipLaunchKernelGGL(k_grad_exponents, dim3((unsigned)batch), dim3(1024), 0, st, dY, L.rows, exps);
    }
    int err = (int)hipGetLastError();
    if (err) return err;
    hipLaunchKernelGGL(k_grad_digits, dim3((unsigned)((p.steps + 3) / 4), (unsigned)((batch + 15) / 16)), dim3(256), 0, st, dY, exps, batch,
                       L.rows, L.gate_h, p.steps, digits);
    err = (int)hipGetLastError();
    if (err) return err;
    GradArgs a;
    a.packed = packed;
    a.packed_bytes = (uint32_t)packed_bytes(L);
    a.layer_step = (uint32_t)(tile16_layer_stride(L) * 4);
    a.round_step = (uint32_t)(tile16_rowtile_stride(L) * 4);
    a.rt_count = L.rt_count; a.cq = L.cq; a.m = bits_used; a.batch = batch; a.cols = L.cols;
    a.steps = p.steps; a.steps_per_split = p.steps_per_split;
    a.scales = scales; a.digits = digits; a.exps = exps;
    float *const parts = reinterpret_cast<float *>(ws + p.parts_off);
    a.out = p.splits > 1 ? parts : dX;
    const bool wide = bits_used > 4, il = is_pairs(L.layout);
    const void *fn = p.wm == 1 ? grad_kernel<1>(wide, il) : (p.wm == 2 ? grad_kernel<2>(wide, il) : grad_kernel<4>(wide, il));
    void *args[] = {&a};
    const dim3 grid((unsigned)p.blocks, (unsigned)((batch + 16 * p.wm - 1) / (16 * p.wm)), (unsigned)p.splits);
    hipError_t e = hipLaunchKernel(fn, grid, dim3(512), args, 0, st);
    if (e == hipSuccess) e = hipGetLastError();
    if (e != hipSuccess) return (int)e;
    if (p.splits > 1) {
        const size_t total = (size_t)batch * L.cols;
        hipLaunchKernelGGL(k_grad_join, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, st, parts, p.splits, total, dX);
        e = hipGetLastError();
    }
    return (int)e;
}

}  // namespace pb
