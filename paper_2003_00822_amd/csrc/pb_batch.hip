// The product of Algorithm 2 for large batches, as the gated block and the adapters use it (pb_imma.h has the arithmetic; the digits are those of
// k_digits): workgroups of 128 vectors and 128 weight rows, and act(g) u of a gated block behind the product.
//
// The eight waves of a workgroup lie along the vectors, sixteen each, and all multiply the codes of the same eight row tiles, which are in
// LDS: two buffers of 64 KB (a chunk of 512 columns each).  While a wave multiplies one buffer it turns the words of its row tile for the other
// one into codes, step by step between the products.  Per chunk and wave: 8 KB of words and 24 KB of digits (three of four, see pb_imma.h) from
// memory, 64 KB of codes from LDS, 192 matrix instructions.
// Bound: the matrix instructions and what does not run beside them.  us (rocprofv3): 8192 x 4096, 8 bitlayers, 2048 vectors 190 (2.17 POP/s in three digits),
// the matrix pipelines busy for 57 % of the compute units' cycles, waves waiting for 35 % of theirs, at 2.0 GHz; a gated block of 21844 x 4096,
// 1024 vectors 288 (1.91 POP/s; its 1368 workgroups are 5.3 rounds over the chip), 53 % and 35 %.  The first calls on an idle card take up to a fifth longer.
#include <type_traits>

#include "pb_imma.h"

namespace pb {

constexpr int kBatchTiles = 8, kBatchVectors = 128, kBatchBuffer = kBatchTiles * 8192;
constexpr int kBatchRow = 4 * 33;                  // (kGated) floats per vector in LDS: four gates of 32 units

// Workgroups and what they do: those of an XCD (id % 8) take a contiguous range of an order in which eight blocks of rows and then the
// vectors are next to each other, and read less of both through their L2.
struct BatchGrid {
    int blocks, rows_of, workgroups;
    __device__ void place(int id, int *block, int *vectors) const
    {
        const int each = workgroups / 8, rest = workgroups % 8, xcd = id % 8;
        int at = xcd * each + min(xcd, rest) + id / 8;
        const int wide = at / (8 * rows_of), width = min(8, blocks - wide * 8);
        at -= wide * 8 * rows_of;
        *vectors = at / width;
        *block = wide * 8 + at % width;
    }
};

template <int Q, bool IL, int EPI>
__global__ __launch_bounds__(512) void k_batch(const I8Args a, const BatchGrid grid, float *const low, float *const high)
{
    extern __shared__ __align__(16) unsigned char s_codes[];
    __shared__ int s_ones[kBatchTiles][kTileRows];
    __shared__ float s_scales[PB_MAX_BITS];

    const int lane = threadIdx.x & 63, kb = lane >> 4, j = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int block, vectors;
    grid.place(blockIdx.x, &block, &vectors);
    const int group = vectors * 8 + wave, first_tile = block * kBatchTiles, my_tile = first_tile + wave;
    const int m = a.m;

    // the scales: whether they halve (as in k_i8_tile)
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(a.scales), 0, m * 4, 0x00020000);
    const float scv = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, lane * 4, 0, 0));
    const float scn = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, lane * 4 + 4, 0, 0));
    if (wave == 0 && lane < PB_MAX_BITS) s_scales[lane] = scv;
    const bool off = lane + 1 < m && !(scv == (lane == 0 ? -2.0f : 2.0f) * scn);
    const bool merged = __builtin_amdgcn_ballot_w64(off) == 0;
    const int gs0 = merged ? 4 * Q : 1, gs1 = merged ? 4 * Q - 2 : 1;

    // the digits of the wave's vectors (a group without vectors reads none)
    const __amdgpu_buffer_rsrc_t rd =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.digits), 0, (int)a.digits_bytes, 0x00020000);
    const int count = group_vectors(a.act.batch, group);
    const uint32_t doff = j < count ? digits_at(group, count, a.cq, 4, 0, kb, j) : (uint32_t)kNowhere;
    const uint32_t per_digit = (uint32_t)min(count - (j & ~3), 4) * 64u, dstep = digits_step(count, 4);

    unsigned char *const my_codes = s_codes + wave * 8192 + lane * 16;
    const unsigned char *const operands = s_codes + lane * 16;

    // everything of the product with ND of four digits
    auto sum_up = [&](auto nd) {
        constexpr int ND = decltype(nd)::value;
        // (four digits: the codes are read twice, for two digits each, as in k_grad)
        constexpr int DC = ND == 4 ? 2 : 3, TURNS = 8 * (ND == 4 ? 2 : 1), NT = kBatchTiles, BR = 3, STAGES = 24;
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
            auto inside = [&](int q) { return q < a.cq && my_tile < a.rt_count; };
            // the words of chunk q; absent ones are zero
            auto issue = [&](int q) {
                const uint32_t at = (uint32_t)my_tile * a.round_step + (uint32_t)q * 1024u;
#pragma unroll
                for (int s = 0; s < 4 * Q; ++s) {
                    const int l = l0 + s, lu = l0 + (s & ~1);
                    const bool has = inside(q) && (IL ? lu + 1 >= f && lu < e : l >= f && l < e);
                    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint32_t *>(a.packed), 0,
                                                                                        has ? (int)a.packed_bytes : 0, 0x00020000);
                    w[s] = __builtin_amdgcn_raw_buffer_load_b128(rw, lane * 16, has ? (int)(at + (uint32_t)l * a.layer_step) : 0, 0);
                }
            };
            // The codes of chunk q from its words, word after word in the six steps of weight_codes(), and the sums of the codes
            uint64_t part[4];
            int ones = 0;                          // (of the lane's columns)
            auto expand = [&](int stage, int q, unsigned char *to) {
                const int t = stage / 6, o = stage & 1;
                if (stage % 6 < 2) {
                    if (o == 1 && Q == 1) return;      // (the upper or the lower four slots)
                    uint32_t p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[i] = w[4 * o + i][t];
                        if constexpr (IL) p[i] = (o == 0 && i < 2 ? p[i] ^ flip : p[i]) & (inside(q) ? mask[2 * o + i / 2] : 0u);
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
                    *reinterpret_cast<v4i *>(to + t * 2048 + o * 1024) = out;
#pragma unroll
                    for (int k = 0; k < 4; ++k) ones = __builtin_amdgcn_sdot4(out[k], 0x01010101, ones, false);
                }
            };
            u32x4 ar[2][DC];
            auto load_digits = [&](u32x4 (&dst)[DC], int step, int from) {
#pragma unroll
                for (int d = 0; d < DC; ++d)
                    dst[d] = __builtin_amdgcn_raw_buffer_load_b128(rd, (int)(doff + (from + d) * per_digit),
                                                                   (int)((uint32_t)min(step, a.cq * 8 - 1) * dstep), 0);
            };
            issue(0);
            load_digits(ar[0], 0, 0);
#pragma unroll
            for (int i = 0; i < STAGES; ++i) {
                expand(i, 0, my_codes);
                __builtin_amdgcn_sched_barrier(0);
            }
            issue(1);
            __syncthreads();
            v4i acc[ND][NT];
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[d][nt] = v4i{0, 0, 0, 0};
            for (int q = 0; q < a.cq; ++q) {
                const int here = q & 1 ? kBatchBuffer : 0;
                const unsigned char *src = operands + here;
                unsigned char *const to = my_codes + (kBatchBuffer - here);
                auto codes = [&](int th, int nt) { return *reinterpret_cast<const v4i *>(src + nt * 8192 + th * 1024); };
                v4i br[BR];
#pragma unroll
                for (int i = 0; i < BR - 1; ++i) br[i] = codes(0, i);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int k = 0; k < TURNS; ++k) {
                    // (turn k: (t, h) k / (TURNS / 8), the digits from k % (TURNS / 8) * DC on)
                    load_digits(ar[(k + 1) & 1], q * 8 + (k + 1) / (TURNS / 8), (k + 1) % (TURNS / 8) * DC);
                    if constexpr (ND == 4) {      // the third digit enters as u - 128 (see pb_imma.h)
                        if (k & 1) ar[1][0] ^= 0x80808080u;
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const int i = k * NT + nt, ahead = i + BR - 1;
                        if (ahead < TURNS * NT) br[ahead % BR] = codes(ahead / NT / (TURNS / 8), ahead % NT);
                        // (the next chunk's codes first: the words after them then have the rest of the loop to arrive)
                        if (i < STAGES) expand(i, q + 1, to);
                        if (i == 19) issue(q + 2);       // (the last word has been taken)
#pragma unroll
                        for (int d = 0; d < DC; ++d) {
                            v4i &sum = acc[k % (TURNS / 8) * DC + d][nt];
                            sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, ar[k & 1][d]), br[i % BR], sum, 0, 0, 0);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __syncthreads();
            }
            // ---- a lane has row j of every row tile and the vectors 4 kb + c ----
            ones += __shfl_xor(ones, 16);
            ones += __shfl_xor(ones, 32);
            if (lane < kTileRows) s_ones[wave][lane] = ones;
            __syncthreads();
            int at = lane;
            asm volatile("" : "+v"(at));       // (what follows is worked out here and not kept during the loop)
            const int jj = at & 15, n0 = group * kGroupVectors + (at >> 4) * 4;
            const Group g = make_group(a, f, e, s_scales);
            float *const s_out = reinterpret_cast<float *>(s_codes);
            // A gated block's sums of several groups change places among the workgroup's own, which are written after a barrier only: sixteen lanes next
            // to each other in memory, not four (4096 units, 2048 columns, 11 bitlayers, 512 vectors 62 us, 2 % more than with sums in fp32; by fours 18 % more)
            const bool turned = EPI == kGated && first_tile * 4 + 32 <= a.gate_h;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int prow = (first_tile + nt) * kTileRows + jj;
                const int row = a.gate_h ? gates_matrix_row(prow, a.gate_h) : prow;
                const bool row_ok = row >= 0 && row < a.R;
                const float bias = a.bias && row_ok ? a.bias[row] : 0.0f;
                const int sum1 = s_ones[nt][jj];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int n = n0 + c;
                    const bool live = row_ok && n < a.act.batch;
                    int d[4] = {acc[0][nt][c], acc[1][nt][c], acc[2][nt][c], 0};
                    if constexpr (ND == 4) d[3] = acc[ND - 1][nt][c];
                    double v = scaled_sum<4>(g, d, sum1, ND == 4);
                    // (the thread's own: the sum of the earlier groups of bitlayers, an fp64 value in two words)
                    const size_t o = (size_t)n * a.R + (turned ? (nt >> 1) * a.gate_h + first_tile * 4 + (nt & 1) * 16 + jj : row);
                    if (live && f > 0) v += __hiloint2double((int)__float_as_uint(high[o]), (int)__float_as_uint(low[o]));
                    if (!g.last) {
                        if (live) {
                            high[o] = __uint_as_float((uint32_t)__double2hiint(v));
                            low[o] = __uint_as_float((uint32_t)__double2loint(v));
                        }
                    } else {
                        float y = (float)(v * a.out_scale);
                        if (a.bias) y += bias;
                        if constexpr (EPI == kGated)
                            s_out[(wave * kGroupVectors + (at >> 4) * 4 + c) * kBatchRow + (jj & 3) * 33 + nt * 4 + (jj >> 2)] = y;
                        else if (live) a.Y[(size_t)n * a.R + row] = y;
                    }
                }
            }
            __syncthreads();
        }
    };
    // (the waves of a workgroup may differ: both ways pass the same barriers)
    const uint32_t wide_here = load_wide<4>(a, group * 4, lane);
    if (count == 0 || !is_wide(wide_here)) sum_up(std::integral_constant<int, 3>{});
    else sum_up(std::integral_constant<int, 4>{});

    if constexpr (EPI == kGated) {
        // gates 0 and 1 of units u and units / 2 + u, and their values (gates 2 and 3): 32 units next to each other
        const float *const s_out = reinterpret_cast<const float *>(s_codes);
        const int F = a.R / 2, lu = threadIdx.x & 31, unit = first_tile * 4 + lu;
        if (unit < a.gate_h) {
            for (int v = threadIdx.x >> 5; v < kBatchVectors; v += 16) {
                const int n = vectors * kBatchVectors + v;
                if (n >= a.act.batch) break;
                float y[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = s_out[v * kBatchRow + k * 33 + lu];
                if (a.Y) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) a.Y[(size_t)n * a.R + (size_t)k * a.gate_h + unit] = y[k];
                }
                a.h_out[(size_t)n * F + unit] = gate_act(a.gate, y[0]) * y[2];
                a.h_out[(size_t)n * F + a.gate_h + unit] = gate_act(a.gate, y[1]) * y[3];
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------

// (a gated block on the pairs layout leaves its pre-activations in memory for k_gated)
static const void *const kBatchFn[2][2] = {{reinterpret_cast<const void *>(k_batch<1, false, kStore>), reinterpret_cast<const void *>(k_batch<1, true, kStore>)},
                                           {reinterpret_cast<const void *>(k_batch<2, false, kStore>), reinterpret_cast<const void *>(k_batch<2, true, kStore>)}};
static const void *const kBatchGatedFn[2] = {reinterpret_cast<const void *>(k_batch<1, false, kGated>), reinterpret_cast<const void *>(k_batch<2, false, kGated>)};
constexpr int kBatchLds = 2 * kBatchBuffer;
static_assert(kBatchVectors * kBatchRow * 4 <= kBatchLds, "the results of a gated block in the place of the codes");

int batch_workgroups(int rt_count, int batch)
{
    return ((rt_count + kBatchTiles - 1) / kBatchTiles) * ((batch + kBatchVectors - 1) / kBatchVectors);
}

int launch_imma_batch(const I8Args &a, bool il, float *low, float *high, hipStream_t st)
{
    const int gated = a.gate >= 0, q = a.m > 4;
    const void *fn = gated ? kBatchGatedFn[q] : kBatchFn[q][il];
    static uint64_t declared[2][2][2];
    const int d = declare_lds(fn, kBatchLds, &declared[gated][q][il]);
    if (d) return d;
    BatchGrid grid;
    grid.blocks = (a.rt_count + kBatchTiles - 1) / kBatchTiles;
    grid.rows_of = (a.act.batch + kBatchVectors - 1) / kBatchVectors;
    grid.workgroups = grid.blocks * grid.rows_of;
    void *args[] = {const_cast<I8Args *>(&a), &grid, &low, &high};
    const hipError_t e = hipLaunchKernel(fn, dim3((unsigned)grid.workgroups), dim3(512), args, (size_t)kBatchLds, st);
    return (int)(e != hipSuccess ? e : hipGetLastError());
}

}  // namespace pb
