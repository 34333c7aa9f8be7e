// SwiGLU between the experts' two products, u = SiLU(gate) * up, and its gradient. A row of gate_up holds its gate
// values before its up values. Bound by memory: 16 bytes a thread and operand, everything read and written once: 65536 rows of 2 x
// 1408 bf16 87 us, the gradient 146 (6.3 TB/s both; a copy 6.5), float32 8192 x 4096 the gradient 105 (6.4). The exponential
// and the division of the library hide behind that.
#include "columns.h"

namespace pcm {
namespace {

template <class IN, class OUT, bool STREAM>
__global__ __launch_bounds__(256) void swiglu_kernel(const IN* __restrict__ gate_up, const int32_t* __restrict__ count, int64_t R,
                                                     int F, OUT* __restrict__ u) {
    constexpr int C = kCols<IN, OUT>;
    const int64_t rows = count ? min(R, (int64_t)max(*count, 0)) : R, per = F / C, total = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per, c = (i - r * per) * C;
        Raw<IN, C> gate, up;
        read<STREAM>(gate, gate_up + r * 2 * F + c);
        read<STREAM>(up, gate_up + r * 2 * F + F + c);
        Cols<C> v;
#pragma unroll
        for (int j = 0; j < C; ++j) v.v[j] = gated(IN(), gate.at(j), up.at(j));
        store_cols<C>(u + r * F + c, v);
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

template <class IN, class OUT, bool STREAM>
__global__ __launch_bounds__(256) void swiglu_grad_kernel(const IN* __restrict__ gate_up, const IN* __restrict__ du,
                                                          const int32_t* __restrict__ count, int64_t R, int F,
                                                          OUT* __restrict__ dgate_up) {
    constexpr int C = kCols<IN, OUT>;
    const int64_t rows = count ? min(R, (int64_t)max(*count, 0)) : R, per = F / C, total = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per, c = (i - r * per) * C;
        Raw<IN, C> gate, up, d;
        read<STREAM>(gate, gate_up + r * 2 * F + c);
        read<STREAM>(up, gate_up + r * 2 * F + F + c);
        read<STREAM>(d, du + r * F + c);
        Cols<C> dg, dup;
#pragma unroll
        for (int j = 0; j < C; ++j) gated_grad(gate.at(j), up.at(j), d.at(j), dg.v[j], dup.v[j]);
        store_cols<C>(dgate_up + r * 2 * F + c, dg);
        store_cols<C>(dgate_up + r * 2 * F + F + c, dup);
    }
}

template <class IN, class OUT, bool STREAM>
hipError_t swiglu_sized(const IN* gate_up, const IN* du, const int32_t* count, int64_t R, int F, OUT* out, hipStream_t s) {
    const int64_t blocks = ceil_div(R * (F / kCols<IN, OUT>), 256);
    const dim3 grid((unsigned)(blocks < (1 << 22) ? blocks : (1 << 22)));
    if (du) swiglu_grad_kernel<IN, OUT, STREAM><<<grid, 256, 0, s>>>(gate_up, du, count, R, F, out);
    else swiglu_kernel<IN, OUT, STREAM><<<grid, 256, 0, s>>>(gate_up, count, R, F, out);
    return hipGetLastError();
}

template <class IN, class OUT>
hipError_t swiglu_typed(const void* gate_up, const void* du, const int32_t* count, int64_t R, int F, void* out, hipStream_t s) {
    return streamed((du ? 3 : 2) * R * F * (int64_t)sizeof(IN))
               ? swiglu_sized<IN, OUT, true>((const IN*)gate_up, (const IN*)du, count, R, F, (OUT*)out, s)
               : swiglu_sized<IN, OUT, false>((const IN*)gate_up, (const IN*)du, count, R, F, (OUT*)out, s);
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
