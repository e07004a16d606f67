// Low-rank adapters beside a packed layer, an adapter k per vector chosen by an index on the device:
//   Y_n += scale_k B_k (A_k x_n)                                    (pb_matmul_adapters)
//   u = A_k x_n,  t = scale_k B_k^T dy_n,  dX_n += A_k^T t,  dA_k = sum_n t x_n^T,  dB_k = scale_k sum_n dy_n u^T     (its backward pass)
// A [count][rank][cols], B [count][rows][rank], both in fp32, bf16 or fp16; everything is multiplied and added in fp32.
//
// The vectors are put in the order of their adapters (k_adapter_order), and a tile is up to sixteen vectors of one adapter: an adapter
// is read once per tile and product, whatever the order of the requests.  The products are V_MFMA_F32_16X16X4_F32: lane 16 kb + i brings
// row i (column i) of the two operands at position kb of the sum, and gets rows 4 kb .. 4 kb + 3 of column i of the result.  Which
// summand stands at which position is free as long as both operands agree, so lanes load neighbouring summands with wide loads.
// Bound: memory and latencies (the products of 2048 vectors of rank 16 with 4096 columns take 2 us of the chip's fp32 matrix rate).  us (rocprofv3):
// 8192 x 4096, six adapters of rank 32 in fp16, 2048 vectors: u beside the activations' digits 22.5 (77 MB fetched, 37 written), up 28.5 (71 fetched and 60
// written of the 134 MB of Y, 4.7 TB/s), order 7.0; 4096 x 4096, 4 of rank 16 in bf16, 2048 vectors: u and t beside the scalings 21.0 (100 MB), gradients 27.7
// (101 and 32 MB); 1024 x 1024, rank 8, one vector: down 3.7, which is little more than a launch (its up is behind the product).
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "pb_grad.h"

namespace pb {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
struct bf16 { uint16_t v; };
struct f16 { uint16_t v; };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __uint_as_float((uint32_t)v.v << 16); }
__device__ __forceinline__ float to_f32(f16 v) { return (float)__builtin_bit_cast(_Float16, v.v); }
// Four values next to each other.  Global memory takes loads and stores of 8 and 16 bytes at any multiple of a value's size.
typedef float v4f_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ v4f load4(const float *p) { return *reinterpret_cast<const v4f_at4 *>(p); }
__device__ __forceinline__ v4f load4(const bf16 *p)
{
    const u32x2 w = *reinterpret_cast<const u32x2_at2 *>(p);
    return v4f{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xFFFF0000u)};
}
__device__ __forceinline__ v4f load4(const f16 *p)
{
    const u32x2 w = *reinterpret_cast<const u32x2_at2 *>(p);
    return v4f{to_f32(f16{(uint16_t)w[0]}), to_f32(f16{(uint16_t)(w[0] >> 16)}), to_f32(f16{(uint16_t)w[1]}), to_f32(f16{(uint16_t)(w[1] >> 16)})};
}
// The values p[at .. at + 4).  Unless WHOLE some may lie behind the last of `length`: the last stands for them (ZERO: 0).  (No branch: a load in a
// branch of its own is waited for there.)
template <bool WHOLE, bool ZERO, typename T>
__device__ __forceinline__ v4f load4_of(const T *p, int at, int length)
{
    if constexpr (WHOLE) {
        return load4(p + at);
    } else {
        v4f v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = to_f32(p[min(at + e, length - 1)]);
            if (ZERO && at + e >= length) v[e] = 0.0f;
        }
        return v;
    }
}
__device__ __forceinline__ void store4_of(float *p, int at, int length, v4f v)
{
    if (at + 4 <= length) {
        *reinterpret_cast<v4f_at4 *>(p + at) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (at + i < length) p[at + i] = v[i];
    }
}
typedef std::integral_constant<bool, true> yes;
typedef std::integral_constant<bool, false> no;
__device__ __forceinline__ v4f mfma(float a, float b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// ---- the order of the vectors ----
struct Item { int adapter, length, vector[16]; };

// The r-th of the lanes that are set in `mask`, in lane r
__device__ __forceinline__ int lanes_in_order(unsigned long long mask, int lane)
{
    const bool set = mask >> lane & 1;
    const int rank = __popcll(mask & ((1ull << lane) - 1));
    // (the lanes that are not set go behind the others)
    return __builtin_amdgcn_ds_permute((set ? rank : __popcll(mask) + lane - rank) * 4, lane);
}
// The lanes with the same key as this one, of those with a key of 0 or more
__device__ __forceinline__ unsigned long long same_key(int key, int count)
{
    unsigned long long mask = __builtin_amdgcn_ballot_w64(key >= 0);
    for (int b = 0; (count - 1) >> b; ++b) {
        const unsigned long long set = __builtin_amdgcn_ballot_w64((key >> b & 1) != 0);
        mask &= (key >> b & 1) ? set : ~set;
    }
    return mask;
}

// What the kernels go by: the order of the vectors, its tiles, and where an adapter's vectors begin in it.  Without an index all vectors have
// adapter 0 and their own order.  Up to 64 vectors every wave works the order out from the index; for more k_adapter_order has left it in memory.
struct Order {
    const int32_t *index;
    const int *order;
    const Item *items;
    const int *counts;        // [0]: tiles
    const int *starts;        // [adapter], and the end
    int batch, count;

    __device__ int key_of(int n) const
    {
        const int k = n < batch ? index[n] : -1;
        return k >= 0 && k < count ? k : -1;
    }
    // Tile i: its adapter, its vectors, and vector lane % 16 of them (of a lane beyond: any of the tile)
    struct Tile { int adapter, length, vector; };
    __device__ bool tile(int i, int lane, Tile *t) const
    {
        if (!index) {
            *t = {0, min(16, batch - i * 16), min(i * 16 + (lane & 15), batch - 1)};
            return i * 16 < batch;
        }
        if (order) {
            // (all read at once; items that are none hold anything)
            const int tiles = counts[0], length = items[i].length, vector = items[i].vector[lane & 15];
            *t = {items[i].adapter, length, vector};
            if (i >= tiles) return false;
            const int last = __shfl(vector, length - 1);
            if ((lane & 15) >= length) t->vector = last;
            return true;
        }
        const int key = key_of(lane);
        const unsigned long long same = same_key(key, count), below = (1ull << lane) - 1;
        const int place = __popcll(same & below);
        const bool begins = key >= 0 && place % 16 == 0;
        const unsigned long long all = __builtin_amdgcn_ballot_w64(begins);
        if (i >= __popcll(all)) return false;
        const int first = __builtin_ctzll(__builtin_amdgcn_ballot_w64(begins && __popcll(all & below) == i));
        const unsigned long long mine =
            (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(same >> 32), first) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)same, first);
        t->adapter = __builtin_amdgcn_readlane(key, first);
        const unsigned long long left = mine >> first << first;      // (it and those behind it)
        t->length = min(16, __popcll(left));
        t->vector = __shfl(lanes_in_order(left, lane), min(lane & 15, t->length - 1));
        return true;
    }
    // The vectors of an adapter: `length` of them, number p is vector(p)
    struct Segment {
        const int *order;
        int length, list;     // list: lane r has number r, if `listed`
        bool listed;
        __device__ int vector(int p) const { return listed ? __shfl(list, p) : (order ? order[p] : p); }
    };
    __device__ Segment segment(int adapter, int lane) const
    {
        if (!index) return {nullptr, adapter ? 0 : batch, 0, false};
        if (order) return {order + starts[adapter], starts[adapter + 1] - starts[adapter], 0, false};
        const unsigned long long mine = __builtin_amdgcn_ballot_w64(key_of(lane) == adapter);
        return {nullptr, (int)__popcll(mine), lanes_in_order(mine, lane), true};
    }
};
constexpr int kListed = 64;       // vectors of which no order is left in memory

// One workgroup.  A wave finds out for 64 vectors which of them have the same adapter (a ballot per bit of its number), then the waves add to the
// adapters' counts in the order of the vectors: the order within an adapter is theirs, so that sums over its vectors are the same every time.
constexpr int kOrderThreads = 1024, kChunks = PB_MAX_BATCH / 64, kChunksPerWave = kChunks / (kOrderThreads / 64);
__global__ __launch_bounds__(kOrderThreads) void k_adapter_order(const int32_t *__restrict__ index, int batch, int count, int *__restrict__ order,
                                                                 Item *__restrict__ items, int *__restrict__ counts, int *__restrict__ starts)
{
    __shared__ int s_count[PB_MAX_ADAPTERS];
    __shared__ uint32_t s_first[PB_MAX_ADAPTERS];     // places before the adapter's, and from bit 16 on tiles before its
    __shared__ uint32_t s_wave[kOrderThreads / 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int k = threadIdx.x; k < PB_MAX_ADAPTERS; k += kOrderThreads) s_count[k] = 0;
    int key[kChunksPerWave], place[kChunksPerWave], same[kChunksPerWave];
#pragma unroll
    for (int i = 0; i < kChunksPerWave; ++i) {
        const int n = (i * (kOrderThreads / 64) + wave) * 64 + lane;
        int k = n < batch ? index[n] : -1;
        if (k < 0 || k >= count) k = -1;
        const unsigned long long mask = same_key(k, count);
        key[i] = k;
        place[i] = __popcll(mask & ((1ull << lane) - 1));
        same[i] = __popcll(mask);
    }
    const int chunks = (batch + 63) / 64;
#pragma unroll
    for (int i = 0; i < kChunksPerWave; ++i)
        for (int w = 0; w < kOrderThreads / 64 && i * (kOrderThreads / 64) + w < chunks; ++w) {
            __syncthreads();
            if (wave == w && key[i] >= 0) {
                const int before = s_count[key[i]];
                if (place[i] == 0) s_count[key[i]] = before + same[i];
                place[i] += before;
            }
        }
    __syncthreads();
    // places and tiles before each adapter: four adapters per thread
    uint32_t own[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = s_count[threadIdx.x * 4 + i];
        own[i] = sum;
        sum += (uint32_t)c + ((uint32_t)((c + 15) / 16) << 16);
    }
    uint32_t scan = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t v = (uint32_t)__shfl_up((int)scan, d);
        if (lane >= d) scan += v;
    }
    if (lane == 63) s_wave[wave] = scan;
    __syncthreads();
    uint32_t before = scan - sum;
    for (int w = 0; w < wave; ++w) before += s_wave[w];
#pragma unroll
    for (int i = 0; i < 4; ++i) s_first[threadIdx.x * 4 + i] = before + own[i];
    if (threadIdx.x == kOrderThreads - 1) {
        counts[0] = (int)((before + sum) >> 16);
        starts[count] = (int)((before + sum) & 0xFFFFu);
    }
    __syncthreads();
    for (int k = threadIdx.x; k < count; k += kOrderThreads) starts[k] = (int)(s_first[k] & 0xFFFFu);
#pragma unroll
    for (int i = 0; i < kChunksPerWave; ++i) {
        const int k = key[i], n = (i * (kOrderThreads / 64) + wave) * 64 + lane;
        if (k < 0) continue;
        const int start = (int)(s_first[k] & 0xFFFFu), at = start + place[i];
        order[at] = n;
        Item *const it = items + (s_first[k] >> 16) + place[i] / 16;
        it->vector[place[i] % 16] = n;
        if (place[i] % 16 == 0) {
            it->adapter = k;
            it->length = min(16, s_count[k] - place[i]);
        }
    }
}

// ---- u = A_k x and t = scale_k B_k^T dy ----
struct DownArgs {
    Order order;
    const void *M;            // A or B
    const float *scale;       // (t only)
    const float *V;           // [batch][length]
    float *out;               // [vector][rank, a multiple of 16][parts of the sum]
    int length, rank, ranks, slices;
};
// Parts of the sum of a tile's products go to the waves of `slices` workgroups (a power of two up to 16); a lane's result is four ranks of one
// vector.  It is kept as a part per slice, four at least; those that no slice fills are zero.
//   TURNED: the summands are the rows of the matrix (B: [length][rank]), else its columns (A: [rank][length])
// What a lane loads of ranks beyond the last is another's; they are set to zero in the end.
constexpr int kMany = 32, kPartsOfMany = 8;       // of more than 32 vectors (an adapter may have them all) eight parts at most
__host__ __device__ constexpr int down_parts(int slices) { return slices > 4 ? slices : 4; }
constexpr int kDownWaves = 8;
template <typename T, bool TURNED, int RT>
__device__ __forceinline__ void adapter_down(const DownArgs &a, int item, int part, int own, v4f (*s_part)[RT][64])
{
    const int lane = threadIdx.x & 63, kb = lane >> 4, i = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Order::Tile it;
    if (!a.order.tile(item, lane, &it)) return;
    const T *const M = static_cast<const T *>(a.M) + (size_t)it.adapter * a.rank * a.length;
    const float *const x = a.V + (size_t)it.vector * a.length;
    // (RT tiles that there are, also where this workgroup's own are fewer: all but the last are whole)
    const int rt0 = min(own, a.ranks - RT), last = min((rt0 + RT - 1) * 16 + i, a.rank - 1);
    const T *row[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) row[t] = M + (size_t)(t < RT - 1 ? (rt0 + t) * 16 + i : last) * a.length;
    v4f acc[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[t] = v4f{0, 0, 0, 0};
    // 16 Q summands from c0 on
    auto step = [&](int c0, auto whole, auto many) {
        constexpr bool WHOLE = decltype(whole)::value;
        constexpr int Q = decltype(many)::value;
        v4f v[Q], w[Q][RT];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int c = c0 + 16 * q + 4 * kb;
            v[q] = load4_of<WHOLE, true>(x, c, a.length);
            if constexpr (TURNED) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const T *const m = M + (size_t)(c0 + 16 * q + e) * a.rank;       // (the same in all lanes)
                    const int r = WHOLE ? 4 * kb : min(4 * kb, a.length - 1 - (c0 + 16 * q + e));
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        w[q][t][e] = to_f32(m[r * a.rank + (t < RT - 1 ? (rt0 + t) * 16 + i : last)]);
                        if (!WHOLE && c + e >= a.length) w[q][t][e] = 0.0f;
                    }
                }
            } else {
#pragma unroll
                for (int t = 0; t < RT; ++t) w[q][t] = load4_of<WHOLE, true>(row[t], c, a.length);
            }
        }
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t] = mfma(w[q][t][e], v[q][e], acc[t]);
    };
    for (int c0 = (part * kDownWaves + wave) * 64; c0 < a.length; c0 += a.slices * kDownWaves * 64) {
        if (c0 + 64 <= a.length) {
            step(c0, yes(), std::integral_constant<int, 4>());
        } else {
#pragma unroll 1
            for (int q = 0; q < 4; ++q) step(c0 + 16 * q, no(), std::integral_constant<int, 1>());
        }
    }
    if (wave > 0) {
#pragma unroll
        for (int t = 0; t < RT; ++t) s_part[wave - 1][t][lane] = acc[t];
    }
    __syncthreads();
    if (wave > 0 || i >= it.length) return;
    const float s = a.scale ? a.scale[it.adapter] : 1.0f;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if (rt0 + t < own) continue;
        v4f v = acc[t];
#pragma unroll
        for (int w = 0; w < kDownWaves - 1; ++w) v += s_part[w][t][lane];
        v *= s;
        // (ranks beyond the last are zero whatever the vector holds: 0 times infinity must not reach the products that follow)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if ((rt0 + t) * 16 + 4 * kb + e >= a.rank) v[e] = 0.0f;
        const int parts = down_parts(a.slices), own_parts = parts / a.slices;
        float *const out = a.out + (((size_t)it.vector * a.ranks + rt0 + t) * 16 + 4 * kb) * parts + part * own_parts;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (own_parts == 4) *reinterpret_cast<v4f *>(out + e * parts) = v4f{v[e], 0, 0, 0};
            else if (own_parts == 2) *reinterpret_cast<float2 *>(out + e * parts) = make_float2(v[e], 0.0f);
            else out[e * parts] = v[e];
        }
    }
}
// u, t or both
template <typename T, int RT>
__global__ __launch_bounds__(kDownWaves * 64) void k_adapter_down(const DownArgs u, const DownArgs t)
{
    __shared__ v4f s_part[kDownWaves - 1][RT][64];
    const int z = blockIdx.z * RT;
    if (u.V && z < u.ranks) adapter_down<T, false, RT>(u, blockIdx.x, blockIdx.y, z, s_part);
    else adapter_down<T, true, RT>(t, blockIdx.x, blockIdx.y, u.V ? z - (u.ranks + RT - 1) / RT * RT : z, s_part);
}
// u, t or both beside the scalings of dY, which the last workgroups do, a vector each.  us of the backward pass, together / one after the other:
// 4096 x 4096, 4 of rank 16 in bf16, 2048 vectors 161.7 / 168.1; 8582 x 935, 5 of 50 in fp16, 670 vectors 105.5 / 111.9; 4096 x 4096, one of 16, 48 vectors
// 35 / 38.  (With the scalings first, which are short, 164.4, 109.7, 35.)
template <typename T, int RT>
__global__ __launch_bounds__(kDownWaves * 64) void k_adapter_down_dy(const DownArgs u, const DownArgs t, const float *__restrict__ dY, int rows,
                                                                     Scaling *__restrict__ scalings, int batch, int items)
{
    __shared__ v4f s_part[kDownWaves - 1][RT][64];
    const int at = blockIdx.x, scales = gridDim.x - batch;
    if (at >= scales) {
        scale_vector<kDownWaves>(dY, rows, at - scales, scalings);
        return;
    }
    const int rest = at / items, item = at % items, part = rest % u.slices, z = rest / u.slices * RT;
    if (u.V && z < u.ranks) adapter_down<T, false, RT>(u, item, part, z, s_part);
    else adapter_down<T, true, RT>(t, item, part, u.V ? z - (u.ranks + RT - 1) / RT * RT : z, s_part);
}
// The same beside the join of a gradient's parts.  us of the backward pass, together / one after the other: 1500 x 701, 3 of rank 9 in fp32, 100 vectors
// 26.1 / 28.3; 1024 x 1024, one of 8 in fp32, one vector 16.0 / 18.6.
template <typename T, int RT>
__global__ __launch_bounds__(kDownWaves * 64) void k_adapter_down_join(const DownArgs u, const DownArgs t, const GradParts joined, int workgroups, int items)
{
    __shared__ v4f s_part[kDownWaves - 1][RT][64];
    const int at = blockIdx.x;
    if (at >= workgroups) {
        join_parts(joined, ((size_t)(at - workgroups) * (kDownWaves * 64) + threadIdx.x) * 2);
        return;
    }
    const int rest = at / items, item = at % items, part = rest % u.slices, z = rest / u.slices * RT;
    if (u.V && z < u.ranks) adapter_down<T, false, RT>(u, item, part, z, s_part);
    else adapter_down<T, true, RT>(t, item, part, u.V ? z - (u.ranks + RT - 1) / RT * RT : z, s_part);
}
// u beside the activations' digits, both of which only read x: the last workgroups do four units of the digits each
struct DigitsJob {
    ActSource act;
    uint8_t *digits, *wide;
    uint32_t turn;
    int cq, units, workgroups;
};
template <typename T, int RT>
__global__ __launch_bounds__(kDownWaves * 64) void k_adapter_down_x(const DownArgs u, const DigitsJob job, const int items)
{
    __shared__ v4f s_part[kDownWaves - 1][RT][64];
    __shared__ int s_wide[kDownWaves];
    const int at = blockIdx.x, rest = at / items, id = at - (int)(gridDim.x - job.workgroups);
    if (id >= 0) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), unit = min(id * (kDownWaves / 2) + wave / 2, job.units - 1);
        digits_unit<4>(job.act, job.cq, job.digits, job.wide, nullptr, job.turn, unit % job.cq, unit / job.cq, wave & 1, s_wide + (wave & ~1));
    } else {
        adapter_down<T, false, RT>(u, at % items, rest % u.slices, rest / u.slices * RT, s_part);
    }
}
// Rank i of rank tile `rt` of a vector: the parts added up in a fixed order
template <int PARTS>
__device__ __forceinline__ float down_at(const float *parts, int ranks, int vector, int rt, int i)
{
    const v4f *const p = reinterpret_cast<const v4f *>(parts + (((size_t)vector * ranks + rt) * 16 + i) * PARTS);
    v4f v = p[0];
#pragma unroll
    for (int k = 1; k < PARTS / 4; ++k) v += p[k];
    return (v[0] + v[1]) + (v[2] + v[3]);
}
// f(integral constant of the parts, MOST at most)
template <int MOST, typename F>
__device__ __forceinline__ void by_parts(int slices, F f)
{
    if (slices <= 4) f(std::integral_constant<int, 4>());
    else if (slices == 8 || MOST == 8) f(std::integral_constant<int, 8>());
    else f(std::integral_constant<int, MOST>());
}

// ---- Y += scale_k B_k u, dX += A_k^T t ----
struct UpArgs {
    Order order;
    const void *M;
    const float *scale;       // (Y only)
    const float *parts;       // u or t
    float *out;               // [batch][length]
    int length, rank, ranks, slices, blocks;
};
// A wave does `blocks` times 64 values of the tile's vectors.  RT rank tiles at once.  TURNED: M is A [rank][length], else B [length][rank].
// Values behind the last are computed from others' rows or columns and not stored.
constexpr int kUpRow = 20;        // floats per rank in LDS: the vectors of the tile, and room that puts neighbouring ranks on other banks
template <typename T, bool TURNED, int RT, int WAVES>
__device__ __forceinline__ void adapter_up(const UpArgs &a, int column, int item, float *s_u)
{
    const int lane = threadIdx.x & 63, kb = lane >> 4, i = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = (column * WAVES + wave) * a.blocks * 64, end = min(first + a.blocks * 64, a.length);
    Order::Tile it;
    if (!a.order.tile(item, lane, &it)) return;
    const T *const M = static_cast<const T *>(a.M) + (size_t)it.adapter * a.rank * a.length;
    const float s = a.scale ? a.scale[it.adapter] : 1.0f;
    // the parts of u (t) are added up once per workgroup: a thread of the first 256 has a rank of every rank tile of one vector
    if (wave < 4) by_parts<16>(a.slices, [&](auto parts) {
        const int v = threadIdx.x / 16, vector = __shfl(it.vector, v);
        for (int rt0 = 0; rt0 < a.ranks; rt0 += RT) {
            float sum[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                sum[t] = down_at<decltype(parts)::value>(a.parts, a.ranks, vector, min(rt0 + t, a.ranks - 1), i) * s;
                if ((rt0 + t) * 16 + i >= a.rank) sum[t] = 0.0f;      // (whatever the scale is)
            }
#pragma unroll
            for (int t = 0; t < RT; ++t)
                if (rt0 + t < a.ranks) s_u[((rt0 + t) * 16 + i) * kUpRow + v] = sum[t];
        }
    });
    __syncthreads();
    if (first >= a.length) return;
    float *const y = a.out + (size_t)it.vector * a.length;
    // a lane's values: four times four next to each other
    auto value_at = [&](int r0, int t) { return r0 + 16 * t + 4 * kb; };
    // summands of rank tile t: 4 e + kb (TURNED), 4 kb + e
    float u[RT][4];
    auto load_u = [&](int rt0) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                u[t][e] = rt0 + t < a.ranks ? s_u[((rt0 + t) * 16 + (TURNED ? 4 * e + kb : 4 * kb + e)) * kUpRow + i] : 0.0f;
    };
    load_u(0);
    auto block = [&](int r0, auto whole, auto fours) {
        constexpr bool WHOLE = decltype(whole)::value, FOURS = decltype(fours)::value;
        v4f before[4], acc[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            before[t] = load4_of<WHOLE, false>(y, value_at(r0, t), a.length);
            acc[t] = v4f{0, 0, 0, 0};
        }
        for (int rt0 = 0; rt0 < a.ranks; rt0 += RT) {
            if (a.ranks > RT) load_u(rt0);
            v4f w[RT][4];
#pragma unroll
            for (int x = 0; x < RT; ++x)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    bool inside;
                    if constexpr (TURNED) {      // t: summand 4 t + kb, four values (in the order in which a lane's results then are four and four)
                        const int j = (rt0 + x) * 16 + 4 * t + kb;
                        inside = j < a.rank;
                        w[x][t] = load4_of<WHOLE, false>(M + (size_t)min(j, a.rank - 1) * a.length, r0 + 16 * (i & 3) + 4 * (i >> 2), a.length);
                    } else {                     // t: value r0 + 16 t + i, the summands 4 kb .. 4 kb + 3
                        const int j = (rt0 + x) * 16 + 4 * kb;
                        const T *const row = M + (size_t)(WHOLE ? r0 + 16 * t + i : min(r0 + 16 * t + i, a.length - 1)) * a.rank;
                        inside = !FOURS || j < a.rank;
                        w[x][t] = load4_of<FOURS, true>(row, FOURS ? min(j, a.rank - 4) : j, a.rank);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!inside) w[x][t][e] = 0.0f;
                }
#pragma unroll
            for (int x = 0; x < RT; ++x)
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (TURNED) acc[e] = mfma(w[x][t][e], u[x][t], acc[e]);
                        else acc[t] = mfma(w[x][t][e], u[x][e], acc[t]);
                    }
        }
        if (i < it.length) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                v4f v = acc[t];
                if constexpr (TURNED) v = v4f{acc[0][t], acc[1][t], acc[2][t], acc[3][t]};
                v += before[t];
                if constexpr (WHOLE) *reinterpret_cast<v4f_at4 *>(y + value_at(r0, t)) = v;
                else store4_of(y, value_at(r0, t), a.length, v);
            }
        }
    };
    // (B's rows in fours where the rank is a multiple of four: every lane's four are ranks, or none is)
    const bool fours = TURNED || a.rank % 4 == 0;
    for (int r0 = first; r0 < end; r0 += 64) {
        if (r0 + 64 <= a.length) {
            if (fours) block(r0, yes(), yes());
            else block(r0, yes(), no());
        } else {
            block(r0, no(), no());
        }
    }
}

template <typename T, bool TURNED, int RT>
__global__ __launch_bounds__(256) void k_adapter_up(const UpArgs a)
{
    __shared__ float s_u[PB_MAX_RANK * kUpRow];
    adapter_up<T, TURNED, RT, 4>(a, blockIdx.x, blockIdx.y, s_u);
}

// ---- dA_k = sum t x^T, dB_k = scale_k sum dy u^T ----
struct OuterArgs {
    Order order;
    const float *scale;       // (dB only)
    const float *parts;       // t or u
    const float *V;           // x or dy, [batch][length]
    float *out;               // TURNED: [adapter][length][rank], else [adapter][rank][length]
    int length, rank, ranks, slices;
};
// A wave does 64 columns (rows) and RT rank tiles of an adapter.  SPLIT: the waves of a workgroup do the same ones and take the adapter's vectors by
// fours in turn, and their sums meet in LDS, where every wave adds up a part; else each has columns of its own, and u (t) comes from LDS.
constexpr int outer_waves(bool split) { return split ? 16 : 4; }
constexpr int kOuterVectors = 8;       // (not split) vectors whose ranks are in LDS at a time
constexpr int outer_lds(bool split, int rt) { return split ? outer_waves(true) * rt * 4 * 64 * 4 : rt * 16 * kOuterVectors; }      // in floats
template <bool TURNED, bool SPLIT, int RT>
__device__ __forceinline__ void adapter_outer(const OuterArgs &a, int block, int k, int own, float *lds)
{
    constexpr int WAVES = SPLIT ? outer_waves(true) : 1;
    const int lane = threadIdx.x & 63, kb = lane >> 4, i = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rt0 = own * RT, c0 = (SPLIT ? block : block * outer_waves(false) + wave) * 64, c = c0 + 4 * i;
    const Order::Segment seg = a.order.segment(k, lane);
    v4f acc[RT][4];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[t][q] = v4f{0, 0, 0, 0};
    // (several requests of vectors at once: their numbers first, then what depends on them)
    constexpr int AT_ONCE = SPLIT ? 4 : kOuterVectors / 4;
    auto sums = [&](auto whole, auto parts) {
        constexpr bool WHOLE = decltype(whole)::value;
        constexpr int PARTS = decltype(parts)::value;
        for (int p0 = SPLIT ? 4 * wave : 0; p0 < seg.length; p0 += AT_ONCE * 4 * WAVES) {
            int n[AT_ONCE];
            v4f v[AT_ONCE];
            float u[AT_ONCE][RT];
#pragma unroll
            for (int x = 0; x < AT_ONCE; ++x) n[x] = seg.vector(min(p0 + x * 4 * WAVES + kb, seg.length - 1));
#pragma unroll
            for (int x = 0; x < AT_ONCE; ++x) v[x] = load4_of<WHOLE, false>(a.V + (size_t)n[x] * a.length, c, a.length);
            if constexpr (SPLIT) {
#pragma unroll
                for (int x = 0; x < AT_ONCE; ++x)
#pragma unroll
                    for (int t = 0; t < RT; ++t) u[x][t] = down_at<PARTS>(a.parts, a.ranks, n[x], min(rt0 + t, a.ranks - 1), i);
            } else {
                // a thread brings rank i of one vector and of every second rank tile
                const int m = threadIdx.x / 16 % kOuterVectors, t0 = threadIdx.x / (16 * kOuterVectors), of = seg.vector(min(p0 + m, seg.length - 1));
                float sum[(RT + 1) / 2];
#pragma unroll
                for (int y = 0; y < (RT + 1) / 2; ++y) sum[y] = down_at<PARTS>(a.parts, a.ranks, of, min(rt0 + t0 + 2 * y, a.ranks - 1), i);
                __syncthreads();
#pragma unroll
                for (int y = 0; y < (RT + 1) / 2; ++y)
                    if (t0 + 2 * y < RT) lds[((t0 + 2 * y) * kOuterVectors + m) * 16 + i] = sum[y];
                __syncthreads();
#pragma unroll
                for (int x = 0; x < AT_ONCE; ++x)
#pragma unroll
                    for (int t = 0; t < RT; ++t) u[x][t] = lds[(t * kOuterVectors + 4 * x + kb) * 16 + i];
            }
#pragma unroll
            for (int x = 0; x < AT_ONCE; ++x) {
                if (p0 + x * 4 * WAVES + kb >= seg.length) {      // (a vector that was loaded in place of one behind the last)
                    v[x] = v4f{0, 0, 0, 0};
#pragma unroll
                    for (int t = 0; t < RT; ++t) u[x][t] = 0.0f;
                }
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[t][q] = mfma(u[x][t], v[x][q], acc[t][q]);
            }
        }
    };
    // (the same in all waves of a workgroup, which meet at barriers)
    const bool whole = (SPLIT ? c0 + 64 : (block + 1) * outer_waves(false) * 64) <= a.length;
    by_parts<SPLIT ? kPartsOfMany : 16>(a.slices, [&](auto parts) {
        if (whole) sums(yes(), parts);
        else sums(no(), parts);
    });
    const float s = a.scale ? a.scale[k] : 1.0f;
    // Part x of rank tile t, four values next to each other in memory: of column c + x the ranks j .. j + 3 (TURNED), of rank j + x the columns c .. c + 3
    auto part = [&](int t, int x) {
        if constexpr (TURNED) return acc[t][x];
        else return v4f{acc[t][0][x], acc[t][1][x], acc[t][2][x], acc[t][3][x]};
    };
    auto store = [&](int t, int x, v4f v) {
        const int j = (rt0 + t) * 16 + 4 * kb;
        if constexpr (TURNED) {
            if (c + x < a.length) store4_of(a.out + ((size_t)k * a.length + c + x) * a.rank, j, a.rank, v * s);
        } else {
            if (j + x < a.rank) store4_of(a.out + ((size_t)k * a.rank + j + x) * a.length, c, a.length, v * s);
        }
    };
    if constexpr (SPLIT) {
        v4f *const s_part = reinterpret_cast<v4f *>(lds);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int x = 0; x < 4; ++x) s_part[(wave * RT * 4 + t * 4 + x) * 64 + lane] = part(t, x);
        __syncthreads();
        if (wave >= RT * 4) return;
        v4f v = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += s_part[(w * RT * 4 + wave) * 64 + lane];
        store(wave / 4, wave % 4, v);
    } else {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int x = 0; x < 4; ++x) store(t, x, part(t, x));
    }
}

// dA, dB or both
template <bool SPLIT, int RT>
__global__ __launch_bounds__(outer_waves(SPLIT) * 64) void k_adapter_outer(const OuterArgs A, const OuterArgs B, const int of_A)
{
    __shared__ __align__(16) float lds[outer_lds(SPLIT, RT)];
    const int block = blockIdx.x;
    if (block < of_A) adapter_outer<false, SPLIT, RT>(A, block, blockIdx.y, blockIdx.z, lds);
    else adapter_outer<true, SPLIT, RT>(B, block - of_A, blockIdx.y, blockIdx.z, lds);
}
// dX += A_k^T t beside dA and dB, which do not need it: the first of_A + of_B workgroups per adapter and rank tiles do these.  us of the whole backward
// pass, in two launches / in one: 1500 x 701, 3 of rank 9 in fp32, 100 vectors 32.6 / 28.6; 4096 x 4096, 4 of 16 in bf16, 2048 vectors 165 / 162.5;
// 8698 x 6860, 36 of 42 in fp16, 25 vectors 70.5 / 67.2.
struct OuterGrid { int of_A, blocks, count, workgroups, up_blocks; };
template <typename T, bool SPLIT, int RT>
__global__ __launch_bounds__(outer_waves(SPLIT) * 64) void k_adapter_grads(const OuterArgs A, const OuterArgs B, const UpArgs up, const OuterGrid g)
{
    constexpr int OUTER_RT = SPLIT && RT > 2 ? 2 : RT, LDS = outer_lds(SPLIT, OUTER_RT), UP = PB_MAX_RANK * kUpRow;
    __shared__ __align__(16) float lds[LDS > UP ? LDS : UP];
    const int id = blockIdx.x;
    if (id >= g.workgroups) {
        const int at = id - g.workgroups;
        adapter_up<T, true, RT, outer_waves(SPLIT)>(up, at % g.up_blocks, at / g.up_blocks, lds);
        return;
    }
    const int block = id % g.blocks, rest = id / g.blocks;
    if (block < g.of_A) adapter_outer<false, SPLIT, OUTER_RT>(A, block, rest % g.count, rest / g.count, lds);
    else adapter_outer<true, SPLIT, OUTER_RT>(B, block - g.of_A, rest % g.count, rest / g.count, lds);
}

// ---------------------------------------------------------------------------------------------------------------

static int items_of(const pb_adapters &ad, int batch, bool indexed)
{
    return indexed ? (ad.count + batch / 16 < batch ? ad.count + batch / 16 : batch) : (batch + 15) / 16;
}
// Parts of the sums: about two workgroups per compute unit (one does not get more than its share of the memory's rate by much), each wave with
// 64 summands or more.  A larger batch has no more parts than a smaller one.
static int slices_of(const Layout &L, const pb_adapters &ad, int batch, bool indexed)
{
    const int most = L.rows > L.cols ? L.rows : L.cols, z = ((ad.rank + 15) / 16 + 3) / 4, items = items_of(ad, batch, indexed);
    int slices = 1;
    while (slices < (batch > kMany ? kPartsOfMany : 16) && items * z * slices < 384 && slices * 64 * kDownWaves < most) slices *= 2;
    return slices;
}
static size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
static size_t down_bytes(const pb_adapters &ad, int batch, int slices) { return up256((size_t)batch * ((ad.rank + 15) / 16) * 64 * down_parts(slices)); }

AdapterPlan adapter_plan(const Layout &L, const pb_adapters &ad, int batch, bool indexed)
{
    AdapterPlan p;
    p.items = items_of(ad, batch, indexed);
    p.ranks = (ad.rank + 15) / 16;
    p.slices = slices_of(L, ad, batch, indexed);
    p.items_off = up256((size_t)batch * 4);
    p.counts_off = up256(p.items_off + (size_t)p.items * sizeof(Item));
    p.starts_off = p.counts_off + 256;
    p.u_off = up256(p.starts_off + (size_t)(ad.count + 1) * 4);
    p.t_off = p.u_off + down_bytes(ad, batch, p.slices);
    return p;
}
// Room for this batch and every smaller one, whose sums may have more parts: the last batch of each number of parts needs most
size_t adapter_bytes(const Layout &L, const pb_adapters &ad, int batch, bool indexed)
{
    size_t most = down_bytes(ad, batch, slices_of(L, ad, batch, indexed));
    for (int parts = 16; parts > 4; parts /= 2) {
        int with = 0, without = batch + 1;      // (batches that have as many parts, and those that do not)
        while (without - with > 1) {
            const int b = (with + without) / 2;
            (slices_of(L, ad, b, indexed) >= parts ? with : without) = b;
        }
        const size_t bytes = with ? down_bytes(ad, with, parts) : 0;
        most = bytes > most ? bytes : most;
    }
    return adapter_plan(L, ad, batch, indexed).u_off + 2 * most;
}

static Order order_of(const AdapterPlan &p, const pb_adapters &ad, const int32_t *index, int batch, void *workspace)
{
    char *const ws = static_cast<char *>(workspace);
    Order o = {index, nullptr, nullptr, nullptr, nullptr, batch, ad.count};
    if (index && batch > kListed) {
        o.order = reinterpret_cast<const int *>(ws);
        o.items = reinterpret_cast<const Item *>(ws + p.items_off);
        o.counts = reinterpret_cast<const int *>(ws + p.counts_off);
        o.starts = reinterpret_cast<const int *>(ws + p.starts_off);
    }
    return o;
}

int launch_adapter_order(const AdapterPlan &p, const pb_adapters &ad, const int32_t *index, int batch, void *workspace, hipStream_t st)
{
    if (!index || batch <= kListed) return 0;
    char *const ws = static_cast<char *>(workspace);
    hipLaunchKernelGGL(k_adapter_order, dim3(1), dim3(kOrderThreads), 0, st, index, batch, ad.count, reinterpret_cast<int *>(ws),
                       reinterpret_cast<Item *>(ws + p.items_off), reinterpret_cast<int *>(ws + p.counts_off),
                       reinterpret_cast<int *>(ws + p.starts_off));
    return (int)hipGetLastError();
}

// Rank tiles that a wave takes at once, four at most and no more than it needs
static int rank_tiles(int ranks)
{
    const int turns = (ranks + 3) / 4;
    return (ranks + turns - 1) / turns;
}
// fn(T(), ...) for the type of the adapters
template <typename F>
static int by_type(int type, F fn)
{
    switch (type) {
        case PB_TYPE_F32: return fn(float());
        case PB_TYPE_BF16: return fn(bf16());
        default: return fn(f16());
    }
}
static int launch(const void *fn, dim3 grid, int threads, void *args, hipStream_t st)
{
    void *list[] = {args};
    const hipError_t e = hipLaunchKernel(fn, grid, dim3((unsigned)threads), list, 0, st);
    return (int)(e != hipSuccess ? e : hipGetLastError());
}
static int launch(const void *fn, dim3 grid, int threads, void *first, void *second, void *third, hipStream_t st)
{
    void *list[] = {first, second, third};
    const hipError_t e = hipLaunchKernel(fn, grid, dim3((unsigned)threads), list, 0, st);
    return (int)(e != hipSuccess ? e : hipGetLastError());
}

static void down_args(const AdapterPlan &p, const pb_adapters &ad, const Layout &L, const int32_t *index, const float *X, const float *dY, int batch,
                      void *workspace, DownArgs *u, DownArgs *t)
{
    char *const ws = static_cast<char *>(workspace);
    u->order = order_of(p, ad, index, batch, workspace);
    u->rank = ad.rank; u->ranks = p.ranks; u->slices = p.slices;
    *t = *u;
    u->M = ad.A; u->scale = nullptr; u->V = X; u->length = L.cols; u->out = reinterpret_cast<float *>(ws + p.u_off);
    t->M = ad.B; t->scale = ad.scale; t->V = dY; t->length = L.rows; t->out = reinterpret_cast<float *>(ws + p.t_off);
}
int launch_adapter_down(const AdapterPlan &p, const pb_adapters &ad, const Layout &L, const int32_t *index, const float *X, const float *dY, int batch,
                        void *workspace, hipStream_t st)
{
    const int rt = rank_tiles(p.ranks), z = (p.ranks + rt - 1) / rt;
    DownArgs u, t;
    down_args(p, ad, L, index, X, dY, batch, workspace, &u, &t);
    return by_type(ad.type, [&](auto type) {
        typedef decltype(type) T;
        static const void *const fn[4] = {reinterpret_cast<const void *>(k_adapter_down<T, 1>), reinterpret_cast<const void *>(k_adapter_down<T, 2>),
                                          reinterpret_cast<const void *>(k_adapter_down<T, 3>), reinterpret_cast<const void *>(k_adapter_down<T, 4>)};
        return launch(fn[rt - 1], dim3((unsigned)p.items, (unsigned)p.slices, (unsigned)(z * ((X ? 1 : 0) + (dY ? 1 : 0)))), kDownWaves * 64, &u, &t,
                      nullptr, st);
    });
}

int launch_adapter_down_scalings(AdapterDown *d, const float *dY, int batch, Scaling *scalings, hipStream_t st)
{
    const AdapterPlan &p = *d->plan;
    const pb_adapters &ad = *d->adapters;
    const int rt = rank_tiles(p.ranks), z = (p.ranks + rt - 1) / rt * ((d->X ? 1 : 0) + (d->dY ? 1 : 0));
    DownArgs u, t;
    down_args(p, ad, *d->layout, d->index, d->X, d->dY, batch, d->workspace, &u, &t);
    int rows = d->layout->rows, items = p.items;
    d->done = true;
    return by_type(ad.type, [&](auto type) {
        typedef decltype(type) T;
        static const void *const fn[4] = {reinterpret_cast<const void *>(k_adapter_down_dy<T, 1>), reinterpret_cast<const void *>(k_adapter_down_dy<T, 2>),
                                          reinterpret_cast<const void *>(k_adapter_down_dy<T, 3>), reinterpret_cast<const void *>(k_adapter_down_dy<T, 4>)};
        void *list[] = {&u, &t, &dY, &rows, &scalings, &batch, &items};
        const hipError_t e = hipLaunchKernel(fn[rt - 1], dim3((unsigned)(batch + p.items * p.slices * z)), dim3(kDownWaves * 64), list, 0, st);
        return (int)(e != hipSuccess ? e : hipGetLastError());
    });
}
int launch_adapter_down_join(AdapterDown *d, const GradParts &joined, int batch, hipStream_t st)
{
    const AdapterPlan &p = *d->plan;
    const pb_adapters &ad = *d->adapters;
    const int rt = rank_tiles(p.ranks), z = (p.ranks + rt - 1) / rt * ((d->X ? 1 : 0) + (d->dY ? 1 : 0));
    DownArgs u, t;
    down_args(p, ad, *d->layout, d->index, d->X, d->dY, batch, d->workspace, &u, &t);
    GradParts parts = joined;
    int items = p.items, workgroups = p.items * p.slices * z;
    const size_t joins = (parts.total + kDownWaves * 128 - 1) / (kDownWaves * 128);
    d->done = true;
    return by_type(ad.type, [&](auto type) {
        typedef decltype(type) T;
        static const void *const fn[4] = {reinterpret_cast<const void *>(k_adapter_down_join<T, 1>), reinterpret_cast<const void *>(k_adapter_down_join<T, 2>),
                                          reinterpret_cast<const void *>(k_adapter_down_join<T, 3>), reinterpret_cast<const void *>(k_adapter_down_join<T, 4>)};
        void *list[] = {&u, &t, &parts, &workgroups, &items};
        const hipError_t e = hipLaunchKernel(fn[rt - 1], dim3((unsigned)(workgroups + joins)), dim3(kDownWaves * 64), list, 0, st);
        return (int)(e != hipSuccess ? e : hipGetLastError());
    });
}
int launch_adapter_down_digits(AdapterDown *d, const ActSource &act, int cq, void *digits, void *wide, bool plain, hipStream_t st)
{
    const AdapterPlan &p = *d->plan;
    const pb_adapters &ad = *d->adapters;
    const int rt = rank_tiles(p.ranks), z = (p.ranks + rt - 1) / rt;
    DownArgs u, t;
    down_args(p, ad, *d->layout, d->index, d->X, nullptr, act.batch, d->workspace, &u, &t);
    DigitsJob job;
    job.act = act;
    job.digits = static_cast<uint8_t *>(digits);
    job.wide = static_cast<uint8_t *>(wide);
    job.turn = plain ? 0x80808080u : 0u;
    job.cq = cq;
    job.units = cq * ((act.batch + 3) / 4);
    job.workgroups = (job.units + kDownWaves / 2 - 1) / (kDownWaves / 2);
    int items = p.items;
    d->done = true;
    return by_type(ad.type, [&](auto type) {
        typedef decltype(type) T;
        static const void *const fn[4] = {reinterpret_cast<const void *>(k_adapter_down_x<T, 1>), reinterpret_cast<const void *>(k_adapter_down_x<T, 2>),
                                          reinterpret_cast<const void *>(k_adapter_down_x<T, 3>), reinterpret_cast<const void *>(k_adapter_down_x<T, 4>)};
        return launch(fn[rt - 1], dim3((unsigned)(job.workgroups + p.items * p.slices * z)), kDownWaves * 64, &u, &job, &items, st);
    });
}

// Y += ... with B (TURNED: dX += ... with A)
static UpArgs up_args(const AdapterPlan &p, const pb_adapters &ad, const Layout &L, const int32_t *index, int batch, float *out, void *workspace, bool turned)
{
    UpArgs a;
    a.order = order_of(p, ad, index, batch, workspace);
    a.M = turned ? ad.A : ad.B;
    a.scale = turned ? nullptr : ad.scale;
    a.parts = reinterpret_cast<const float *>(static_cast<char *>(workspace) + (turned ? p.t_off : p.u_off));
    a.out = out;
    a.length = turned ? L.cols : L.rows;
    a.rank = ad.rank; a.ranks = p.ranks; a.slices = p.slices;
    // Blocks of 64 values per wave: one while that leaves the chip room, up to four (a wave finds its tile and its ranks once)
    const long long waves = (long long)((a.length + 63) / 64) * p.items;
    a.blocks = waves < 2 * 4096 ? 1 : (waves < 4 * 4096 ? 2 : 4);
    return a;
}
template <bool TURNED>
static int launch_up(const AdapterPlan &p, const pb_adapters &ad, const Layout &L, const int32_t *index, int batch, float *out, void *workspace,
                     hipStream_t st)
{
    UpArgs a = up_args(p, ad, L, index, batch, out, workspace, TURNED);
    const int rt = rank_tiles(p.ranks);
    return by_type(ad.type, [&](auto type) {
        typedef decltype(type) T;
        static const void *const fn[4] = {reinterpret_cast<const void *>(k_adapter_up<T, TURNED, 1>), reinterpret_cast<const void *>(k_adapter_up<T, TURNED, 2>),
                                          reinterpret_cast<const void *>(k_adapter_up<T, TURNED, 3>), reinterpret_cast<const void *>(k_adapter_up<T, TURNED, 4>)};
        return launch(fn[rt - 1], dim3((unsigned)((a.length + 256 * a.blocks - 1) / (256 * a.blocks)), (unsigned)p.items), 256, &a, st);
    });
}

AdapterRows adapter_rows(const AdapterPlan &p, const pb_adapters &ad, const int32_t *index, void *workspace)
{
    return {ad.B, ad.scale, reinterpret_cast<const float *>(static_cast<char *>(workspace) + p.u_off), index, ad.rank, ad.count, ad.type,
            down_parts(p.slices)};
}

int launch_adapter_up(const AdapterPlan &p, const pb_adapters &ad, const Layout &L, const int32_t *index, int batch, float *Y, void *workspace,
                      hipStream_t st)
{
    return launch_up<false>(p, ad, L, index, batch, Y, workspace, st);
}

int launch_adapter_grads(const AdapterPlan &p, const pb_adapters &ad, const Layout &L, const int32_t *index, const float *X, const float *dY, int batch,
                         float *dX, float *dA, float *dB, void *workspace, hipStream_t st)
{
    char *const ws = static_cast<char *>(workspace);
    if (!dA && !dB) return launch_up<true>(p, ad, L, index, batch, dX, workspace, st);
    OuterArgs A, B;
    A.order = order_of(p, ad, index, batch, workspace);
    A.rank = ad.rank; A.ranks = p.ranks; A.slices = p.slices;
    B = A;
    A.scale = nullptr; A.parts = reinterpret_cast<const float *>(ws + p.t_off); A.V = X; A.out = dA; A.length = L.cols;
    B.scale = ad.scale; B.parts = reinterpret_cast<const float *>(ws + p.u_off); B.V = dY; B.out = dB; B.length = L.rows;
    // Whether the waves of a workgroup share an adapter's vectors, by an estimate in us from the mean of them (which adapters the vectors have is known on
    // the device only): rounds of workgroups, one or two on a compute unit, against the turns over the vectors of a wave alone.  us, shared / alone:
    // 6453 + 2048 rows and columns, 3 adapters of rank 50, 498 vectors 29 / 37; 8845 + 1106, 1 of 19, 1568 29 / 222; 4096 + 4096, 4 of 16, 2048 15 / 58;
    // but 8438 + 4091, 6 of 49, 471 60 / 30; 4096 + 4096, 16 of 64, 1024 91 / 26; 8 of 16, 512 16 / 12.
    const int shared_rt = p.ranks == 1 ? 1 : 2, alone_rt = rank_tiles(p.ranks);
    const long long groups = (long long)((dA ? (L.cols + 63) / 64 : 0) + (dB ? (L.rows + 63) / 64 : 0)) * ad.count * ((p.ranks + shared_rt - 1) / shared_rt);
    const double mean = (double)batch / ad.count, rounds = (double)((groups + 512 / shared_rt - 1) / (512 / shared_rt));
    const bool split = batch > kMany && rounds * (5.5 + mean / 64) < 4.0 + mean / 8 * (0.75 + 0.25 * alone_rt);
    const int rt = split ? shared_rt : alone_rt, columns = split ? 64 : 64 * outer_waves(false);
    static const void *const fns[2][4] = {{reinterpret_cast<const void *>(k_adapter_outer<false, 1>), reinterpret_cast<const void *>(k_adapter_outer<false, 2>),
                                           reinterpret_cast<const void *>(k_adapter_outer<false, 3>), reinterpret_cast<const void *>(k_adapter_outer<false, 4>)},
                                          {reinterpret_cast<const void *>(k_adapter_outer<true, 1>), reinterpret_cast<const void *>(k_adapter_outer<true, 2>)}};
    int of_A = dA ? (L.cols + columns - 1) / columns : 0;
    const int of_B = dB ? (L.rows + columns - 1) / columns : 0;
    const int z = (p.ranks + rt - 1) / rt;
    UpArgs up = up_args(p, ad, L, index, batch, dX, workspace, true);
    const int per = outer_waves(split) * 64 * up.blocks;
    OuterGrid g = {of_A, of_A + of_B, ad.count, 0, (L.cols + per - 1) / per};
    const long long workgroups = (long long)g.blocks * ad.count * z + (long long)g.up_blocks * p.items;
    // (a dimension of a grid has fewer than 2^32 threads)
    const bool together = dX && workgroups * outer_waves(split) * 64 < 1ll << 32;
    if (dX && !together) {
        const int err = launch_up<true>(p, ad, L, index, batch, dX, workspace, st);
        if (err) return err;
    }
    if (!together) return launch(fns[split][rt - 1], dim3((unsigned)(of_A + of_B), (unsigned)ad.count, (unsigned)z), outer_waves(split) * 64, &A, &B, &of_A, st);
    g.workgroups = g.blocks * ad.count * z;
    return by_type(ad.type, [&](auto type) {
        typedef decltype(type) T;
#define PB_GRADS(SPLIT) {reinterpret_cast<const void *>(k_adapter_grads<T, SPLIT, 1>), reinterpret_cast<const void *>(k_adapter_grads<T, SPLIT, 2>), \
                         reinterpret_cast<const void *>(k_adapter_grads<T, SPLIT, 3>), reinterpret_cast<const void *>(k_adapter_grads<T, SPLIT, 4>)}
        static const void *const fn[2][4] = {PB_GRADS(false), PB_GRADS(true)};
        void *list[] = {&A, &B, &up, &g};
        const hipError_t e = hipLaunchKernel(fn[split][alone_rt - 1], dim3((unsigned)workgroups),
                                             dim3((unsigned)outer_waves(split) * 64), list, 0, st);
        return (int)(e != hipSuccess ? e : hipGetLastError());
    });
}

}  // namespace pb
