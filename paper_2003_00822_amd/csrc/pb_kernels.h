// Internal: launchers implemented by the .hip files of this library.
// Each returns a hipError_t value as int (0 = success); arguments are validated by the caller.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pb_layout.h"

namespace pb {

// More dynamic LDS than the default 64 KB is declared once per kernel and GPU, `bytes` being the most that its launches use.  `devices`: the kernel's own, a
// bit for each GPU on which it has been (beyond 64 of them: at every call).
inline int declare_lds(const void *fn, size_t bytes, uint64_t *devices)
{
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return (int)e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (__atomic_load_n(devices, __ATOMIC_RELAXED) & bit) return 0;
    e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess) __atomic_fetch_or(devices, bit, __ATOMIC_RELAXED);
    return (int)e;
}

// pb_quantize.hip
int launch_quantize_pack(const float *W, const Layout &L, int quantizer, uint32_t *packed, float *scales,
                         hipStream_t st);
int launch_unpack(const uint32_t *packed, const Layout &L, int32_t *q, hipStream_t st);

// pb_prep.hip: fp32 activations -> fixed point -> bit planes + plane statistics.
// Row n of the activations is the concatenation [X0[n][0..cols0) ; X1[n][0..cols1)] (X1 may be null with cols1 = 0).
int launch_prep(const float *X0, int cols0, const float *X1, int cols1, int batch, const Layout &L, int frac_bits,
                int act_bits, uint32_t *planes, int *meta, int32_t *xq_out, hipStream_t st);

// pb_matvec.hip: AND + popcount product against register-resident planes, one launch for all bitlayers.
// Exactly one of Y / A is non-null.
int launch_matvec(const uint32_t *packed, const float *scales, const Layout &L, int bits_used, int frac_bits,
                  const uint32_t *planes, const int *meta, int batch, float *Y, long long *A, hipStream_t st);

// What a single vector's adapter adds to it in k_mfma: scale_k B_k u, u being there in parts (pb_adapters.hip)
struct AdapterRows {
    const void *B;
    const float *scale, *parts;
    const int32_t *index;
    int rank, count, type, nparts;
};
constexpr int kAdapterRowsRank = 16;     // (32 cost scratch memory in two of the kernels)
struct AdapterDown;

// pb_mfma.hip: the whole of Algorithm 2 in one launch on the matrix cores, for ONE activation vector (the tiled layouts but
// the pairs layout).  Activations come from X0 / X1 (converted and bit-transposed inside the kernel) or, if `planes` is
// non-null, from bit planes that launch_prep left in memory.  Exactly one of Y / A is non-null.
// What follows the product in the same launch: bias and ReLU before the store of Y, or (PB_LAYOUT_TILE16_GATES_V1
// only) the LSTM cell update, which writes h_out / c_out [batch][H] instead of Y, or a gated block's act(g) u, which writes
// h_out [batch][rows / 2] and, where wanted, the pre-activations to Y.
constexpr int kBatchFrom = 64;           // the kernel for large batches takes more vectors than this
struct Epilogue {
    const float *bias = nullptr;   // [rows] or null
    int relu = 0;
    const float *c_prev = nullptr; // non-null: fused LSTM cell
    float *h_out = nullptr, *c_out = nullptr;
    int gate = -1;                 // 0 or more: fused gated block (a pb_gate)
    float *pre = nullptr;          // non-null: room for [batch][rows], and the kernel for large batches of pb_batch.hip may be taken
    float *more = nullptr;         // as much room again, where there is no Y and that kernel may be taken (more than kBatchFrom vectors)
    AdapterDown *down = nullptr;   // adapters whose u = A_k x is wanted: where the activations' digits have a launch, it does both
    const AdapterRows *adapter = nullptr;   // (one vector, tiled layouts but the pairs')
    bool fused() const { return c_prev || gate >= 0; }
};
int launch_mfma(const uint32_t *packed, const float *scales, const Layout &L, int bits_used, int frac_bits,
                int act_bits, const float *X0, int cols0, const float *X1, int cols1, const uint32_t *planes, float *Y,
                long long *A, const Epilogue &ep, hipStream_t st);

// pb_imma.hip: the same product as whole weight codes times the bytes of x_q on the 8-bit integer matrix cores, for
// batches and for PB_LAYOUT_TILE16_PAIRS_V1.  `digits` is the workspace's room for the activations' byte digits (4 bytes per
// padded column and vector at most) and `wide` a byte per four vectors (64 apart) and 512 columns, both written by
// launch_digits: before the call (`prepared`, with the third of four digits left `plain`) or, where the product kernel does not convert
// the activations itself, by the call.
// (`pairs_out`: the sums of bitlayer pairs are asked for)
inline bool takes_digits(const Layout &L, int batch, bool pairs_out = false)
{
    return is_tile16(L.layout) && (batch > 1 || is_pairs(L.layout) || pairs_out);
}
int launch_digits(const float *X0, int cols0, const float *X1, int cols1, int batch, const Layout &L, int frac_bits,
                  int act_bits, void *digits, void *wide, int32_t *xq_out, bool plain, hipStream_t st);
int launch_imma(const uint32_t *packed, const float *scales, const Layout &L, int bits_used, int frac_bits, int act_bits,
                const float *X0, int cols0, const float *X1, int cols1, void *digits, void *wide, bool prepared, int batch,
                float *Y, long long *A, bool pairs_out, const Epilogue &ep, hipStream_t st);

// logistic function of the LSTM gates in the stand-alone cell update (the fused one evaluates 0.5 tanh(v / 2) + 0.5,
// the same function, side by side with the tanh of the fourth gate)
__device__ __forceinline__ float sigmoid_f(float v) { return 1.0f / (1.0f + expf(-v)); }

// pb_lstm.hip: y = act(y + bias) in place, for the layout whose product kernel has no fused epilogue
int launch_bias_act(float *Y, const float *bias, int relu, int rows, int batch, hipStream_t st);

// pb_lstm.hip: gate nonlinearities and state update on the gate pre-activations.
int launch_lstm_pointwise(const float *gates, const float *bias, const float *c_prev, int H, int batch, float *h_out,
                          float *c_out, hipStream_t st);

// pb_gated.hip: H[n][r] = act(pre[n][r]) pre[n][units + r]
int launch_gated(const float *pre, int units, int gate, int batch, float *H, hipStream_t st);

// pb_grad.hip: dX = dY W through the packed matrix (tiled layouts).  With `gated`, dY are the gradients of the pre-activations [g; u] of
// H = act(g) u, which the call works out from dH and leaves in `dpre`.  `down`: adapters whose u and t are wanted; where the scalings or the join of
// the sum's parts have a launch, it does both.
struct GatedSource {
    const float *pre, *dH;
    float *dpre;
    int gate;
};
size_t grad_workspace_bytes(const Layout &L, int batch);      // (not less than those of a smaller batch)
int launch_grad(const uint32_t *packed, const float *scales, const Layout &L, int bits_used, const float *dY, const GatedSource *gated,
                int batch, float *dX, void *workspace, hipStream_t st, AdapterDown *down = nullptr);

// pb_adapters.hip: low-rank adapters beside a layer of rows x cols.  The plan carves the workspace up for a batch.
struct AdapterPlan {
    int items;             // tiles of up to sixteen vectors of one adapter, at most
    int ranks;             // rank tiles of sixteen
    int slices;            // parts of the sums of u and t
    size_t items_off, counts_off, starts_off, u_off, t_off;
};
AdapterPlan adapter_plan(const Layout &L, const pb_adapters &ad, int batch, bool indexed);
size_t adapter_bytes(const Layout &L, const pb_adapters &ad, int batch, bool indexed);     // (not less than those of a smaller batch)
// The order of the vectors (by adapter) and its tiles; nothing to do without an index or for few vectors
int launch_adapter_order(const AdapterPlan &p, const pb_adapters &ad, const int32_t *index, int batch, void *workspace, hipStream_t st);
// u = A_k x (and t = scale_k B_k^T dY, if dY is given) of the ordered vectors, in parts
int launch_adapter_down(const AdapterPlan &p, const pb_adapters &ad, const Layout &L, const int32_t *index, const float *X, const float *dY, int batch,
                        void *workspace, hipStream_t st);
// The same for x beside k_digits<4>, or for x and dY (where given) beside k_grad_scalings or k_grad_join, in one launch, which then is `done`
struct AdapterDown {
    const AdapterPlan *plan;
    const pb_adapters *adapters;
    const Layout *layout;
    const int32_t *index;
    const float *X, *dY;
    void *workspace;
    bool done;
};
struct ActSource;
struct Scaling;
struct GradParts;
int launch_adapter_down_join(AdapterDown *down, const GradParts &joined, int batch, hipStream_t st);
int launch_adapter_down_scalings(AdapterDown *down, const float *dY, int batch, Scaling *scalings, hipStream_t st);
int launch_adapter_down_digits(AdapterDown *down, const ActSource &act, int cq, void *digits, void *wide, bool plain, hipStream_t st);
// Y += scale_k B_k u; what launch_mfma needs to do it for one vector
AdapterRows adapter_rows(const AdapterPlan &p, const pb_adapters &ad, const int32_t *index, void *workspace);
int launch_adapter_up(const AdapterPlan &p, const pb_adapters &ad, const Layout &L, const int32_t *index, int batch, float *Y, void *workspace,
                      hipStream_t st);
// dX += A_k^T t (if dX is given), dA_k = sum t x^T, dB_k = scale_k sum dy u^T (where given)
int launch_adapter_grads(const AdapterPlan &p, const pb_adapters &ad, const Layout &L, const int32_t *index, const float *X, const float *dY, int batch,
                         float *dX, float *dA, float *dB, void *workspace, hipStream_t st);

}  // namespace pb
