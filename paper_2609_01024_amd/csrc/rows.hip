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

constexpr int kThreads = 256, kGradThreads = 256;

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

// The token's paths: those whose two rows are there, and a row to read in any case (0 for a number that is no row; a
// token without paths reads none).
template <int K>
struct Paths {
    uint64_t bits;
    int src[K], tgt[K];
    bool has_src[K], has_tgt[K];
};
template <int K>
__device__ __forceinline__ Paths<K> paths_of(const MixRowsArgs& g, int64_t t) {
    Paths<K> p;
    uint64_t from = 0, to = 0;
#pragma unroll
    for (int a = 0; a < K; ++a) {
        p.src[a] = g.src_row_of[t * K + a];
        p.tgt[a] = g.tgt_row_of[t * K + a];
    }
#pragma unroll
    for (int a = 0; a < K; ++a) {
        p.has_src[a] = (uint32_t)p.src[a] < (uint32_t)g.R_src;
        p.has_tgt[a] = (uint32_t)p.tgt[a] < (uint32_t)g.R_tgt;
        p.src[a] = p.has_src[a] ? p.src[a] : 0;
        p.tgt[a] = p.has_tgt[a] ? p.tgt[a] : 0;
        constexpr uint64_t kRow = ((uint64_t)1 << K) - 1;
        from |= p.has_src[a] ? kRow << (a * K) : 0;
#pragma unroll
        for (int q = 0; q < K; ++q) to |= p.has_tgt[a] ? (uint64_t)1 << (q * K + a) : 0;
    }
    p.bits = g.bits[t] & from & to;
    return p;
}

// C columns of a row in float32 registers.
template <int C>
struct Cols {
    float v[C];
};
template <int C>
__device__ __forceinline__ Cols<C> load_cols(const uint16_t* p) {
    typedef uint32_t words __attribute__((ext_vector_type(C / 2)));
    const words w = *(const words*)p;
    Cols<C> r;
#pragma unroll
    for (int i = 0; i < C / 2; ++i) {
        r.v[2 * i] = __uint_as_float(w[i] << 16);
        r.v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
    return r;
}
template <int C>
__device__ __forceinline__ Cols<C> load_cols(const float* p) {
    Cols<C> r;
#pragma unroll
    for (int i = 0; i < C; i += 4) {
        const floatx4 a = *(const floatx4*)(p + i);
        r.v[i] = a[0]; r.v[i + 1] = a[1]; r.v[i + 2] = a[2]; r.v[i + 3] = a[3];
    }
    return r;
}
template <int C>
__device__ __forceinline__ void store_cols(uint16_t* p, const Cols<C>& x) {
    typedef __bf16 out_t __attribute__((ext_vector_type(C)));
    out_t y;
#pragma unroll
    for (int i = 0; i < C; ++i) y[i] = (__bf16)x.v[i];
    *(out_t*)p = y;
}
template <int C>
__device__ __forceinline__ void store_cols(float* p, const Cols<C>& x) {
#pragma unroll
    for (int i = 0; i < C; i += 4) *(floatx4*)(p + i) = floatx4{x.v[i], x.v[i + 1], x.v[i + 2], x.v[i + 3]};
}

constexpr int pow2_above(int v) { return v <= 1 ? 1 : 2 * pow2_above((v + 1) / 2); }

// Sums of N values (a power of two up to 64) over the wavefront, all lanes active: lane l ends with the whole sum of value
// l * N / 64. While there are several values a step halves them: each lane gives one half away and adds what its partner,
// on the other side of the step's bit, gives it; then steps of one value. 63 additions for 64 values, where a sum each
// would take 384. Bits 5 and 4: v_permlane32_swap and 16_swap exchange a half of one register with a half of another;
// below, partners are mirrors in 16 and 8 lanes and neighbours at 2 and 1 (DPP), each of which crosses its bit.
__device__ __forceinline__ float dpp_f32(float v, const int bit) {
    const int i = __float_as_int(v);
    switch (bit) {
        case 3: return __int_as_float(__builtin_amdgcn_update_dpp(0, i, 0x140, 0xF, 0xF, true));   // row_mirror
        case 2: return __int_as_float(__builtin_amdgcn_update_dpp(0, i, 0x141, 0xF, 0xF, true));   // row_half_mirror
        case 1: return __int_as_float(__builtin_amdgcn_update_dpp(0, i, 0x4E, 0xF, 0xF, true));    // lane ^ 2
        default: return __int_as_float(__builtin_amdgcn_update_dpp(0, i, 0xB1, 0xF, 0xF, true));   // lane ^ 1
    }
}
__device__ __forceinline__ float joined32(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float joined16(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int N, int BIT = 5>
__device__ __forceinline__ float wave_sums(float (&v)[N]) {
    constexpr int H = N > 1 ? N / 2 : 1;   // values left after the step of this bit
    float w[H];
    const bool upper = (threadIdx.x >> BIT) & 1;
#pragma unroll
    for (int i = 0; i < H; ++i) {
        const float a = v[i], b = N > 1 ? v[i + H] : v[i];
        if constexpr (BIT == 5) w[i] = joined32(a, b);
        else if constexpr (BIT == 4) w[i] = joined16(a, b);
        else w[i] = (upper ? b : a) + dpp_f32(upper ? a : b, BIT);
    }
    if constexpr (BIT == 0) return w[0];
    else return wave_sums<H, BIT - 1>(w);
}

// BACK: the gradient by u alone, which is the mix of dz from the targets to the sources.
template <class IN, class OUT, int K, bool BACK>
__global__ __launch_bounds__(kThreads) void mix_rows_kernel(MixRowsArgs g) {
    const IN* __restrict__ in = (const IN*)(BACK ? g.dz : g.u);
    OUT* __restrict__ out = (OUT*)g.out;
    for (int64_t t = blockIdx.x; t < g.T; t += gridDim.x) {
        const Paths<K> p = paths_of<K>(g, t);
        float beta[K * K];
#pragma unroll
        for (int i = 0; i < K * K; ++i) beta[i] = g.beta[t * K * K + i];
        for (int c = (blockIdx.y * blockDim.x + threadIdx.x) * 8; c < g.F; c += gridDim.y * blockDim.x * 8) {
            Eight v[K];
            if (p.bits)
#pragma unroll
                for (int a = 0; a < K; ++a) v[a] = load8(in + (int64_t)(BACK ? p.tgt[a] : p.src[a]) * g.F + c);
#pragma unroll
            for (int b = 0; b < K; ++b) {
                if (!(BACK ? p.has_src[b] : p.has_tgt[b])) continue;
                Eight s{};
#pragma unroll
                for (int a = 0; a < K; ++a) {
                    const int i = BACK ? b * K + a : a * K + b;
                    if ((p.bits >> i) & 1)
#pragma unroll
                        for (int q = 0; q < 8; ++q) s.v[q] = fmaf(beta[i], v[a].v[q], s.v[q]);
                }
                store8(out + (int64_t)(BACK ? p.src[b] : p.tgt[b]) * g.F + c, s);
            }
        }
    }
}

// The waves of a workgroup are shared by its tokens, `per` to each; all lanes of a wave stay active (past the last column
// on the last ones again, as zeros), so that the sums cross the whole wave.
template <class IN, class OUT, int K, int C>
__global__ __launch_bounds__(kGradThreads) void mix_rows_grad_kernel(MixRowsArgs g, int per) {
    constexpr int N = pow2_above(K * K);
    __shared__ float part[kGradThreads / 64][N];
    const IN* __restrict__ u = (const IN*)g.u;
    const IN* __restrict__ dz = (const IN*)g.dz;
    OUT* __restrict__ du = (OUT*)g.out;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x / 64, tokens = waves / per, mine = wave / per, sub = wave - mine * per;
    for (int64_t t0 = (int64_t)blockIdx.x * tokens; t0 < g.T; t0 += (int64_t)gridDim.x * tokens) {
        const int64_t t = t0 + mine;
        float dot[N];
#pragma unroll
        for (int i = 0; i < N; ++i) dot[i] = 0.0f;
        if (t < g.T) {
            const Paths<K> p = paths_of<K>(g, t);
            float beta[K * K];
#pragma unroll
            for (int i = 0; i < K * K; ++i) beta[i] = g.beta[t * K * K + i];
            for (int c0 = sub * 64 * C; c0 < g.F; c0 += per * 64 * C) {
                const int at = c0 + lane * C, c = min(at, g.F - C);
                Cols<C> v[K], d[K];
                if (p.bits) {
#pragma unroll
                    for (int a = 0; a < K; ++a) {
                        v[a] = load_cols<C>(u + (int64_t)p.src[a] * g.F + c);
                        d[a] = load_cols<C>(dz + (int64_t)p.tgt[a] * g.F + c);
                    }
                }
                if (c0 + 64 * C > g.F) {
#pragma unroll
                    for (int a = 0; a < K; ++a)
#pragma unroll
                        for (int i = 0; i < C; ++i) {
                            v[a].v[i] = at < g.F ? v[a].v[i] : 0.0f;
                            d[a].v[i] = at < g.F ? d[a].v[i] : 0.0f;
                        }
                }
#pragma unroll
                for (int a = 0; a < K; ++a) {
                    Cols<C> s{};
#pragma unroll
                    for (int b = 0; b < K; ++b)
                        if ((p.bits >> (a * K + b)) & 1) {
#pragma unroll
                            for (int i = 0; i < C; ++i) {
                                s.v[i] = fmaf(beta[a * K + b], d[b].v[i], s.v[i]);
                                dot[a * K + b] = fmaf(v[a].v[i], d[b].v[i], dot[a * K + b]);
                            }
                        }
                    if (du && p.has_src[a] && at < g.F) store_cols<C>(du + (int64_t)p.src[a] * g.F + at, s);
                }
            }
        }
        const float sum = wave_sums<N>(dot);
        constexpr int kLanes = 64 / N;
        const int i = lane / kLanes;
        if (per == 1) {
            if (t < g.T && lane % kLanes == 0 && i < K * K) g.dbeta[t * K * K + i] = sum;
            continue;
        }
        if (lane % kLanes == 0) part[wave][i] = sum;
        __syncthreads();
        if (sub == 0 && t < g.T && lane < K * K) {
            float s = 0.0f;
            for (int q = 0; q < per; ++q) s += part[wave + q][lane];
            g.dbeta[t * K * K + lane] = s;
        }
        __syncthreads();
    }
}

template <class IN, class OUT, int K>
hipError_t mix_sized(bool grad, const MixRowsArgs& g, hipStream_t s) {
    if (grad && g.dbeta) {
        // Waves for a token: steps of 64 C columns, up to four to a wave.
        constexpr int C = K > 4 ? 4 : 8;
        const int64_t steps = ceil_div(g.F, 64 * C);
        const int per = steps <= 4 ? 1 : steps <= 8 ? 2 : 4, tokens = kGradThreads / 64 / per;
        const int64_t blocks = ceil_div(g.T, tokens);
        mix_rows_grad_kernel<IN, OUT, K, C><<<dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), kGradThreads, 0, s>>>(g, per);
        return hipGetLastError();
    }
    const unsigned blocks = (unsigned)(g.T < (1 << 20) ? g.T : (1 << 20));
    const int64_t chunks = g.F / 8;
    const int threads = (int)(chunks >= kThreads ? kThreads : align_up(chunks, 64));
    const int64_t split = ceil_div(chunks, threads);
    const dim3 grid(blocks, (unsigned)(split < 64 ? split : 64));
    if (grad) mix_rows_kernel<IN, OUT, K, true><<<grid, threads, 0, s>>>(g);
    else mix_rows_kernel<IN, OUT, K, false><<<grid, threads, 0, s>>>(g);
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
