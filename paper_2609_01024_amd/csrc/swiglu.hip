// SwiGLU between the experts' two products, u = SiLU(gate) * up, and its gradient. A row of gate_up holds its gate
// values before its up values. Bound by memory: 8 columns a thread, everything read and written once.
#include "eight.h"

namespace pcm {
namespace {

template <class IN, class OUT>
__global__ __launch_bounds__(256) void swiglu_kernel(const IN* __restrict__ gate_up, const int32_t* __restrict__ count, int64_t R,
                                                     int F, OUT* __restrict__ u) {
    const int64_t rows = count ? min(R, (int64_t)max(*count, 0)) : R, per = F / 8, total = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per, c = (i - r * per) * 8;
        const Eight gate = load8(gate_up + r * 2 * F + c), up = load8(gate_up + r * 2 * F + F + c);
        Eight v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v.v[j] = gated(IN(), gate.v[j], up.v[j]);
        store8(u + r * F + c, v);
    }
}

// d gate = du up sig (1 + g (1 - sig)) and d up = du g sig, sig = 1 / (1 + e^-g), float32. 1 - sig comes as e^-g sig, so
// that it keeps its bits where sig is near 1. du up is formed first (it overflows before the result does only where the
// gate is far below 0). From g = -64 down sig is e^g to float32, and e^g may be below the normal range where the result
// is not: it goes in as two factors e^(g/2).
__device__ __forceinline__ void gated_grad(float g, float up, float du, float& dgate, float& dup) {
    const bool far = g < -64.0f;
    const float e = expf(far ? 0.5f * g : -g);
    const float sig = far ? e : 1.0f / (1.0f + e), more = far ? e : 1.0f;
    const float slope = far ? 1.0f + g : 1.0f + g * (e * sig);
    dgate = du * up * sig * slope * more;
    dup = du * sig * g * more;
}

template <class IN, class OUT>
__global__ __launch_bounds__(256) void swiglu_grad_kernel(const IN* __restrict__ gate_up, const IN* __restrict__ du,
                                                          const int32_t* __restrict__ count, int64_t R, int F,
                                                          OUT* __restrict__ dgate_up) {
    const int64_t rows = count ? min(R, (int64_t)max(*count, 0)) : R, per = F / 8, total = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per, c = (i - r * per) * 8;
        const Eight gate = load8(gate_up + r * 2 * F + c), up = load8(gate_up + r * 2 * F + F + c), d = load8(du + r * F + c);
        Eight dg, dup;
#pragma unroll
        for (int j = 0; j < 8; ++j) gated_grad(gate.v[j], up.v[j], d.v[j], dg.v[j], dup.v[j]);
        store8(dgate_up + r * 2 * F + c, dg);
        store8(dgate_up + r * 2 * F + F + c, dup);
    }
}

dim3 grid_of(int64_t R, int F) {
    const int64_t blocks = ceil_div(R * (F / 8), 256);
    return dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
}

template <class IN, class OUT>
hipError_t swiglu_typed(const void* gate_up, const void* du, const int32_t* count, int64_t R, int F, void* out, hipStream_t s) {
    if (du) swiglu_grad_kernel<<<grid_of(R, F), 256, 0, s>>>((const IN*)gate_up, (const IN*)du, count, R, F, (OUT*)out);
    else swiglu_kernel<<<grid_of(R, F), 256, 0, s>>>((const IN*)gate_up, count, R, F, (OUT*)out);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_swiglu(bool bf16, bool out_bf16, const void* gate_up, const void* du, const int32_t* count, int64_t R, int F,
                         void* out, hipStream_t s) {
    if (bf16)
        return out_bf16 ? swiglu_typed<uint16_t, uint16_t>(gate_up, du, count, R, F, out, s)
                        : swiglu_typed<uint16_t, float>(gate_up, du, count, R, F, out, s);
    return out_bf16 ? swiglu_typed<float, uint16_t>(gate_up, du, count, R, F, out, s)
                    : swiglu_typed<float, float>(gate_up, du, count, R, F, out, s);
}

}  // namespace pcm
