// Tokens to their experts' rows and back, and the mix along a token's paths, with their gradients:
//   dispatch        y[r] = w_ta x[t]                       for r = row_of[t, a]
//   its gradient    dx[t] = sum_a w_ta dy[r],              dw_ta = <dy[r], x[t]>
//   combine         y[t] = [y[t] +] sum_a w_ta o[r]
//   its gradient    do[r] = w_ta dy[t],                    dw_ta = <o[r], dy[t]>
//   mix             z[tgt_b] = sum_a beta_ab u[src_a]      over the token's paths (a, b)
//   its gradient    du[src_a] = sum_b beta_ab dz[tgt_b],   dbeta_ab = <dz[tgt_b], u[src_a]>
// All are bound by memory. A workgroup takes a token: the token's row numbers and weights are scalars there, and what
// the rows of a token share (its own row, or the sum) is read or written once. Sums are float32, slots ascending.
#include "eight.h"

namespace pcm {
namespace {

constexpr int kThreads = 256;

// Sum over the wavefront, on every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Rows [first, first + count) of the groups, inside [0, R).
__device__ __forceinline__ void held_rows(const int32_t* offsets, int n, int64_t R, int& first, int& count) {
    first = 0;
    count = (int)R;
    if (!offsets) return;
    const int lo = min(max(offsets[0], 0), (int)R), hi = min(max(offsets[n], lo), (int)R);
    first = lo;
    count = hi - lo;
}

// TO_ROWS: dispatch and the combine's gradient, from `tokens` to the rows of out; otherwise combine and the dispatch's
// gradient, from `rows` to the tokens of out. DOT: dweights too, from both.
template <class IN, class OUT, int KK, bool TO_ROWS, bool DOT>
__global__ __launch_bounds__(kThreads) void rows_kernel(RowsArgs g) {
    __shared__ float part[KK][kThreads / 64];
    const IN* __restrict__ tokens = (const IN*)g.tokens;
    const IN* __restrict__ rows = (const IN*)g.rows;
    OUT* __restrict__ out = (OUT*)g.out;
    int first, count;
    held_rows(g.offsets, g.n, g.R, first, count);
    for (int64_t t = blockIdx.x; t < g.T; t += gridDim.x) {
        int r[KK];
        float w[KK], dot[KK];
        bool on[KK];
#pragma unroll
        for (int a = 0; a < KK; ++a) {
            r[a] = a < g.k ? g.row_of[t * g.k + a] : -1;
            w[a] = g.weights && a < g.k ? g.weights[t * g.k + a] : 1.0f;
            dot[a] = 0.0f;
            on[a] = a < g.k && (uint32_t)r[a] - (uint32_t)first < (uint32_t)count;
        }
        for (int c = (blockIdx.y * blockDim.x + threadIdx.x) * 8; c < g.H; c += gridDim.y * blockDim.x * 8) {
            Eight x{}, v[KK];
            if (TO_ROWS || DOT) x = load8(tokens + t * g.H + c);
            if (!TO_ROWS || DOT) {
#pragma unroll
                for (int a = 0; a < KK; ++a)
                    if (on[a]) v[a] = load8(rows + (int64_t)r[a] * g.H + c);
            }
            if constexpr (DOT) {
#pragma unroll
                for (int a = 0; a < KK; ++a)
                    if (on[a]) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) dot[a] = fmaf(v[a].v[i], x.v[i], dot[a]);
                    }
            }
            if (!out) continue;
            if constexpr (TO_ROWS) {
#pragma unroll
                for (int a = 0; a < KK; ++a)
                    if (on[a]) {
                        Eight y;
#pragma unroll
                        for (int i = 0; i < 8; ++i) y.v[i] = w[a] * x.v[i];
                        store8(out + (int64_t)r[a] * g.H + c, y);
                    }
            } else {
                Eight y{};
                if (g.accumulate) y = load8(out + t * g.H + c);
                Eight s{};
#pragma unroll
                for (int a = 0; a < KK; ++a)
                    if (on[a]) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) s.v[i] = fmaf(w[a], v[a].v[i], s.v[i]);
                    }
#pragma unroll
                for (int i = 0; i < 8; ++i) y.v[i] += s.v[i];
                store8(out + t * g.H + c, y);
            }
        }
        if constexpr (DOT) {
            const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
            for (int a = 0; a < KK; ++a) {
                const float s = wave_sum(dot[a]);
                if (lane == 0) part[a][wave] = s;
            }
            __syncthreads();
            if (threadIdx.x < (unsigned)g.k) {
                float s = 0.0f;
                for (int q = 0; q < (int)blockDim.x / 64; ++q) s += part[threadIdx.x][q];
                g.dweights[t * g.k + threadIdx.x] = s;
            }
            __syncthreads();
        }
    }
}

template <class IN, class OUT, int KK, bool TO_ROWS>
hipError_t rows_by_dot(const RowsArgs& g, hipStream_t s) {
    const int64_t chunks = g.H / 8;
    const int threads = (int)(chunks >= kThreads ? kThreads : align_up(chunks, 64));
    const unsigned blocks = (unsigned)(g.T < (1 << 20) ? g.T : (1 << 20));
    if (g.dweights) {
        rows_kernel<IN, OUT, KK, TO_ROWS, true><<<dim3(blocks), threads, 0, s>>>(g);
    } else {
        const int64_t split = ceil_div(chunks, threads);
        rows_kernel<IN, OUT, KK, TO_ROWS, false><<<dim3(blocks, (unsigned)(split < 64 ? split : 64)), threads, 0, s>>>(g);
    }
    return hipGetLastError();
}

template <class IN, class OUT, bool TO_ROWS>
hipError_t rows_by_slots(const RowsArgs& g, hipStream_t s) {
    if (g.k <= 1) return rows_by_dot<IN, OUT, 1, TO_ROWS>(g, s);
    if (g.k <= 2) return rows_by_dot<IN, OUT, 2, TO_ROWS>(g, s);
    if (g.k <= 4) return rows_by_dot<IN, OUT, 4, TO_ROWS>(g, s);
    return rows_by_dot<IN, OUT, 8, TO_ROWS>(g, s);
}

template <bool TO_ROWS>
hipError_t rows_by_type(bool bf16, bool out_bf16, const RowsArgs& g, hipStream_t s) {
    if (bf16) return out_bf16 ? rows_by_slots<uint16_t, uint16_t, TO_ROWS>(g, s) : rows_by_slots<uint16_t, float, TO_ROWS>(g, s);
    return out_bf16 ? rows_by_slots<float, uint16_t, TO_ROWS>(g, s) : rows_by_slots<float, float, TO_ROWS>(g, s);
}

// The token's paths. A path counts where its bit is set and both of its rows are there.
template <int K>
struct Paths {
    uint64_t bits;
    int src[K], tgt[K];
    bool has_src[K], has_tgt[K];
};
template <int K>
__device__ __forceinline__ Paths<K> paths_of(const MixRowsArgs& g, int64_t t) {
    Paths<K> p;
    p.bits = g.bits[t];
#pragma unroll
    for (int a = 0; a < K; ++a) {
        p.src[a] = g.src_row_of[t * K + a];
        p.tgt[a] = g.tgt_row_of[t * K + a];
        p.has_src[a] = (uint32_t)p.src[a] < (uint32_t)g.R_src;
        p.has_tgt[a] = (uint32_t)p.tgt[a] < (uint32_t)g.R_tgt;
    }
    return p;
}

template <class IN, class OUT, int K>
__global__ __launch_bounds__(kThreads) void mix_rows_kernel(MixRowsArgs g) {
    const IN* __restrict__ u = (const IN*)g.u;
    OUT* __restrict__ z = (OUT*)g.out;
    for (int64_t t = blockIdx.x; t < g.T; t += gridDim.x) {
        const Paths<K> p = paths_of<K>(g, t);
        const float* beta = g.beta + t * K * K;
        for (int c = (blockIdx.y * blockDim.x + threadIdx.x) * 8; c < g.F; c += gridDim.y * blockDim.x * 8) {
            Eight v[K];
#pragma unroll
            for (int a = 0; a < K; ++a)
                if (p.has_src[a]) v[a] = load8(u + (int64_t)p.src[a] * g.F + c);
#pragma unroll
            for (int b = 0; b < K; ++b) {
                if (!p.has_tgt[b]) continue;
                Eight s{};
#pragma unroll
                for (int a = 0; a < K; ++a)
                    if (p.has_src[a] && ((p.bits >> (a * K + b)) & 1)) {
                        const float w = beta[a * K + b];
#pragma unroll
                        for (int i = 0; i < 8; ++i) s.v[i] = fmaf(w, v[a].v[i], s.v[i]);
                    }
                store8(z + (int64_t)p.tgt[b] * g.F + c, s);
            }
        }
    }
}

// A thread takes four columns: the K rows of both sides and K * K sums for dbeta stay in registers.
struct Four {
    float v[4];
};
__device__ __forceinline__ Four load4(const uint16_t* p) {
    typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
    const uintx2 w = *(const uintx2*)p;
    return Four{{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16),
                 __uint_as_float(w[1] & 0xFFFF0000u)}};
}
__device__ __forceinline__ Four load4(const float* p) {
    const floatx4 a = *(const floatx4*)p;
    return Four{{a[0], a[1], a[2], a[3]}};
}
__device__ __forceinline__ void store4(uint16_t* p, const Four& x) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *(bf16x4*)p = bf16x4{(__bf16)x.v[0], (__bf16)x.v[1], (__bf16)x.v[2], (__bf16)x.v[3]};
}
__device__ __forceinline__ void store4(float* p, const Four& x) { *(floatx4*)p = floatx4{x.v[0], x.v[1], x.v[2], x.v[3]}; }

template <class IN, class OUT, int K>
__global__ __launch_bounds__(kThreads) void mix_rows_grad_kernel(MixRowsArgs g) {
    __shared__ float part[kThreads / 64][K * K];
    const IN* __restrict__ u = (const IN*)g.u;
    const IN* __restrict__ dz = (const IN*)g.dz;
    OUT* __restrict__ du = (OUT*)g.out;
    for (int64_t t = blockIdx.x; t < g.T; t += gridDim.x) {
        const Paths<K> p = paths_of<K>(g, t);
        const float* beta = g.beta + t * K * K;
        float dot[K * K];
#pragma unroll
        for (int i = 0; i < K * K; ++i) dot[i] = 0.0f;
        for (int c = threadIdx.x * 4; c < g.F; c += blockDim.x * 4) {
            Four v[K], d[K];
#pragma unroll
            for (int a = 0; a < K; ++a) {
                if (g.dbeta && p.has_src[a]) v[a] = load4(u + (int64_t)p.src[a] * g.F + c);
                if (p.has_tgt[a]) d[a] = load4(dz + (int64_t)p.tgt[a] * g.F + c);
            }
#pragma unroll
            for (int a = 0; a < K; ++a) {
                if (!p.has_src[a]) continue;
                Four s{};
#pragma unroll
                for (int b = 0; b < K; ++b)
                    if (p.has_tgt[b] && ((p.bits >> (a * K + b)) & 1)) {
                        const float w = beta[a * K + b];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            s.v[i] = fmaf(w, d[b].v[i], s.v[i]);
                            if (g.dbeta) dot[a * K + b] = fmaf(v[a].v[i], d[b].v[i], dot[a * K + b]);
                        }
                    }
                if (du) store4(du + (int64_t)p.src[a] * g.F + c, s);
            }
        }
        if (!g.dbeta) continue;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < K * K; ++i) {
            const float s = wave_sum(dot[i]);
            if (lane == 0) part[wave][i] = s;
        }
        __syncthreads();
        if (threadIdx.x < K * K) {
            float s = 0.0f;
            for (int q = 0; q < (int)blockDim.x / 64; ++q) s += part[q][threadIdx.x];
            g.dbeta[t * K * K + threadIdx.x] = s;
        }
        __syncthreads();
    }
}

template <class IN, class OUT, int K>
hipError_t mix_sized(bool grad, const MixRowsArgs& g, hipStream_t s) {
    const unsigned blocks = (unsigned)(g.T < (1 << 20) ? g.T : (1 << 20));
    const int64_t chunks = grad ? g.F / 4 : g.F / 8;
    const int threads = (int)(chunks >= kThreads ? kThreads : align_up(chunks, 64));
    if (grad) {
        mix_rows_grad_kernel<IN, OUT, K><<<dim3(blocks), threads, 0, s>>>(g);
    } else {
        const int64_t split = ceil_div(chunks, threads);
        mix_rows_kernel<IN, OUT, K><<<dim3(blocks, (unsigned)(split < 64 ? split : 64)), threads, 0, s>>>(g);
    }
    return hipGetLastError();
}

template <class IN, class OUT>
hipError_t mix_by_slots(bool grad, const MixRowsArgs& g, hipStream_t s) {
    switch (g.k) {
        case 1: return mix_sized<IN, OUT, 1>(grad, g, s);
        case 2: return mix_sized<IN, OUT, 2>(grad, g, s);
        case 3: return mix_sized<IN, OUT, 3>(grad, g, s);
        case 4: return mix_sized<IN, OUT, 4>(grad, g, s);
        case 5: return mix_sized<IN, OUT, 5>(grad, g, s);
        case 6: return mix_sized<IN, OUT, 6>(grad, g, s);
        case 7: return mix_sized<IN, OUT, 7>(grad, g, s);
        default: return mix_sized<IN, OUT, 8>(grad, g, s);
    }
}

}  // namespace

hipError_t launch_rows(bool to_rows, bool bf16, bool out_bf16, const RowsArgs& g, hipStream_t s) {
    return to_rows ? rows_by_type<true>(bf16, out_bf16, g, s) : rows_by_type<false>(bf16, out_bf16, g, s);
}

hipError_t launch_mix_rows(bool grad, bool bf16, bool out_bf16, const MixRowsArgs& g, hipStream_t s) {
    if (bf16) return out_bf16 ? mix_by_slots<uint16_t, uint16_t>(grad, g, s) : mix_by_slots<uint16_t, float>(grad, g, s);
    return out_bf16 ? mix_by_slots<float, uint16_t>(grad, g, s) : mix_by_slots<float, float>(grad, g, s);
}

}  // namespace pcm
