// How gradients become integers (pb_grad.hip has the arithmetic): the scalings of vectors, for the kernels that work them out.
#pragma once
#include "pb_imma.h"

namespace pb {

typedef float float4_at4 __attribute__((ext_vector_type(4), aligned(4)));     // (global memory takes loads of 16 bytes at any multiple of four)

constexpr int kNotFinite = INT32_MIN;      // in the place of an exponent: the vector's results are NaN

// How a vector's gradients become integers: rint(dy 2^e4) with four digits, rint(dy 2^e3) with three
struct Scaling { int e4, e3, wide, pad; };     // wide: four digits are needed

// From the bits of the largest magnitude and the sum of squares of `count` values
__device__ __forceinline__ Scaling scaling_of(uint32_t largest, double squares, int count)
{
    if (largest >= 0x7F800000u) return {kNotFinite, kNotFinite, 0, 0};
    if (largest == 0) return {0, 0, 0, 0};
    int e;
    const double most = (double)__uint_as_float(largest);
    const float f = frexpf(__uint_as_float(largest), &e);
    // (three balanced digits hold 127 * 65536 + 127 * 256 + 127 = 8355711 < 2^23)
    const double limit = count < 2304 ? count / 16.0 : 144.0 * fmax(1.0, count / 4096.0);
    return {30 - e, 23 - e - (f * 8388608.0f > 8355000.0f ? 1 : 0), most * most * count > limit * squares ? 1 : 0, 0};
}

// The largest magnitude of a vector and the sum of its squares
struct Size {
    uint32_t most = 0;       // bits
    double squares = 0.0;
    __device__ void take(float v)
    {
        most = max(most, __float_as_uint(v) & 0x7FFFFFFFu);
        squares = fma((double)v, (double)v, squares);
    }
    // thread `first` of `threads`: its share of y[0 .. rows)
    __device__ void take(const float *y, int rows, int first, int threads)
    {
        const int fours = rows / 4;
#pragma unroll 4
        for (int i = first; i < fours; i += threads) {
            const float4_at4 v = *reinterpret_cast<const float4_at4 *>(y + 4 * i);
            take(v.x); take(v.y); take(v.z); take(v.w);
        }
        if (first < rows - 4 * fours) take(y[4 * fours + first]);
    }
    __device__ void over_wave()
    {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            most = max(most, (uint32_t)__shfl_xor((int)most, d));
            squares += __shfl_xor(squares, d);
        }
    }
    template <int WAVES>
    __device__ void over_workgroup()       // (in thread 0)
    {
        __shared__ uint32_t s_max[WAVES];
        __shared__ double s_sum[WAVES];
        over_wave();
        if ((threadIdx.x & 63) == 0) {
            s_max[threadIdx.x >> 6] = most;
            s_sum[threadIdx.x >> 6] = squares;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int w = 1; w < WAVES; ++w) {
                most = max(most, s_max[w]);
                squares += s_sum[w];
            }
        }
    }
};

// The parts of a split sum [split][total], in the order of the rows: values i and i + 1
struct GradParts {
    const float *parts;
    float *dX;
    size_t total;
    int splits;
};
__device__ __forceinline__ void join_parts(const GradParts &p, size_t i)
{
    const float *const parts = p.parts;
    float *const dX = p.dX;
    const size_t total = p.total;
    const int splits = p.splits;
    if (i >= total) return;
    if (total % 2 == 0) {
        float2 v = *reinterpret_cast<const float2 *>(parts + i);
#pragma unroll 8
        for (int s = 1; s < splits; ++s) {
            const float2 w = *reinterpret_cast<const float2 *>(parts + (size_t)s * total + i);
            v.x += w.x;
            v.y += w.y;
        }
        *reinterpret_cast<float2 *>(dX + i) = v;
    } else {
        for (size_t k = i; k < i + 2 && k < total; ++k) {
            float v = parts[k];
#pragma unroll 8
            for (int s = 1; s < splits; ++s) v += parts[(size_t)s * total + k];
            dX[k] = v;
        }
    }
}

// The scaling of vector n, by a workgroup of WAVES waves
template <int WAVES>
__device__ __forceinline__ void scale_vector(const float *__restrict__ dY, int rows, int n, Scaling *__restrict__ scalings)
{
    Size size;
    size.take(dY + (size_t)n * rows, rows, threadIdx.x, WAVES * 64);
    size.over_workgroup<WAVES>();
    if (threadIdx.x == 0) scalings[n] = scaling_of(size.most, size.squares, rows);
}

}  // namespace pb
