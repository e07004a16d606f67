// The gate of a gated block on pre-activations that the product left in memory, for the layouts and shapes whose product kernels have no such epilogue.
// Bound: the launch for what comes here (18090 x 76 values, 5.5 MB: 4.9 us), else memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pb_device.h"
#include "pb_kernels.h"

namespace pb {

__global__ __launch_bounds__(256) void k_gated(const float *__restrict__ pre, int units, int gate, float *__restrict__ H)
{
    const int r = blockIdx.x * 256 + threadIdx.x;
    if (r >= units) return;
    const float *p = pre + (size_t)blockIdx.y * 2 * units;
    H[(size_t)blockIdx.y * units + r] = gate_act(gate, p[r]) * p[units + r];
}

int launch_gated(const float *pre, int units, int gate, int batch, float *H, hipStream_t st)
{
    hipLaunchKernelGGL(k_gated, dim3((unsigned)((units + 255) / 256), (unsigned)batch), dim3(256), 0, st, pre, units, gate, H);
    return (int)hipGetLastError();
}

}  // namespace pb
