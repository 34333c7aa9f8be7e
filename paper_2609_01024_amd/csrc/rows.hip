// Tokens to their experts' rows and back, and the mix along a token's paths, with their gradients:
//   dispatch        y[r] = w_ta x[t]                       for r = row_of[t, a]
//   its gradient    dx[t] = sum_a w_ta dy[r],              dw_ta = <dy[r], x[t]>
//   combine         y[t] = [y[t] +] sum_a w_ta o[r]
//   its gradient    do[r] = w_ta dy[t],                    dw_ta = <o[r], dy[t]>
//   mix             z[tgt_b] = sum_a beta_ab u[src_a]      over the token's paths (a, b)
//   its gradient    du[src_a] = sum_b beta_ab dz[tgt_b],   dbeta_ab = <dz[tgt_b], u[src_a]>
// All are bound by memory. A workgroup takes a token: the token's row numbers and weights are scalars there, and what
// the rows of a token share (its own row, or the sum) is read or written once. Sums are float32, slots ascending.
// Measured, bf16 (a copy of 2 GB moves 6.5 TB/s read and written, a read stream 7.1): dispatch of 8192 tokens to 8 rows of 2048 each 51
// us (6.0 TB/s), combine 52 (5.8), dispatch gradient 56 (6.0), combine gradient of 16384 x 4 99 (6.1); mix of 4096 x 2 rows of 14336
// 79 (5.9), of 8192 x 8 rows of 1024 53 (5.0), their gradients 122 (5.8) and 81 (5.0). Rows of 2 KB at eight places of a
// buffer are what costs there: one to four slots of that width move 5.6 TB/s, whatever their paths.
#include <type_traits>

#include "columns.h"

namespace pcm {
namespace {

constexpr int kThreads = 256, kGradThreads = 1024;
// Threads at most for a token where its products are summed over the workgroup: one pass over the columns where it goes (dispatch
// gradient, float32, 8192 x 4 of 2048: 512 threads 63.0 us, 256 66.8; 2048 x 8 of 7168: 51.8 / 51.6, 1024 62.5); towards the
// rows two (combine gradient, 2048 x 8 of 7168: 256 threads 96.4 us, 512 100.5; 4096 x 2 of 4096: 30.4 / 29.8).
template <bool TO_ROWS>
constexpr int kDotThreads = TO_ROWS ? 256 : 512;

constexpr int pow2_above(int v) { return v <= 1 ? 1 : 2 * pow2_above((v + 1) / 2); }

// Sums of N values (a power of two up to 64) over the wavefront, all lanes active: lane l ends with the whole sum of value
// l * N / 64. While there are several values a step halves them: each lane gives one half away and adds what its partner,
// on the other side of the step's bit, gives it; then steps of one value. 32 additions for the 32 values of a mix gradient's
// wave at eight slots, where a sum each would take 192. Bits 5 and 4: v_permlane32_swap and 16_swap exchange a half of one register with a half of another;
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

// Scalar loads of what a token's slots or paths have (the address is the same on every lane; nothing writes there while the
// kernel runs). All of them are on their way before the first wait: read under a branch or by vector loads, each waited for
// the one before (8192 tokens of 8 rows, combine 74 us, 56 with one wait).
template <class T>
using Scalar = const __attribute__((address_space(4))) T*;
template <class T>
__device__ __forceinline__ Scalar<T> scalar(const T* p) { return (Scalar<T>)p; }

// Rows [first, first + count) of the groups, inside [0, R).
__device__ __forceinline__ void held_rows(const int32_t* offsets, int n, int64_t R, int& first, int& count) {
    first = 0;
    count = (int)R;
    if (!offsets) return;
    const int lo = min(max(scalar(offsets)[0], 0), (int)R), hi = min(max(scalar(offsets)[n], lo), (int)R);
    first = lo;
    count = hi - lo;
}

// Element c of the row that starts at element `row` of p: a scalar address and 32 bits of offset.
template <class T>
__device__ __forceinline__ T* column(T* __restrict__ p, int64_t row, uint32_t c) {
    return (T*)((char*)(p + row) + c * (uint32_t)sizeof(T));
}

// TO_ROWS: dispatch and the combine's gradient, from `tokens` to the rows of out; otherwise combine and the dispatch's
// gradient, from `rows` to the tokens of out. DOT: dweights too, from both.
template <class TOKEN, class ROW, class OUT, int KK, bool TO_ROWS, bool DOT, bool STREAM>
__global__ __launch_bounds__(DOT ? kDotThreads<TO_ROWS> : kThreads) void rows_kernel(RowsArgs g) {
    constexpr int C = kCols<TOKEN, ROW, OUT>;
    __shared__ float part[kDotThreads<TO_ROWS> / 64][KK];
    const TOKEN* __restrict__ tokens = (const TOKEN*)g.tokens;
    const ROW* __restrict__ rows = (const ROW*)g.rows;
    OUT* __restrict__ out = (OUT*)g.out;
    for (int64_t item = blockIdx.x; item < g.T * g.parts; item += gridDim.x) {
        const int64_t t = g.parts == 1 ? item : item / g.parts;
        const int part0 = (int)(item - t * g.parts);
        int64_t r[KK];
        float w[KK], dot[KK];
        int row[KK];
#pragma unroll
        for (int a = 0; a < KK; ++a) {
            const int64_t slot = t * g.k + min(a, g.k - 1);
            row[a] = scalar(g.row_of)[slot];
            w[a] = 1.0f;
            if (g.weights) w[a] = scalar(g.weights)[slot];
            dot[a] = 0.0f;
        }
        int first, count;
        held_rows(g.offsets, g.n, g.R, first, count);
        uint32_t held = 0;
#pragma unroll
        for (int a = 0; a < KK; ++a) {
            const bool on = a < g.k && (uint32_t)row[a] - (uint32_t)first < (uint32_t)count;
            held |= on ? 1u << a : 0u;
            r[a] = (int64_t)(on ? row[a] : first) * g.H;   // a row to read in any case, where there are any
        }
        for (int c = (part0 * blockDim.x + threadIdx.x) * C; c < g.H; c += g.parts * blockDim.x * C) {
            Raw<TOKEN, C> x;
            Raw<ROW, C> v[KK];
            if (TO_ROWS || DOT) x.load(column(tokens, t * g.H, c));
            if ((!TO_ROWS || DOT) && held) {
#pragma unroll
                for (int a = 0; a < KK; ++a) read<STREAM>(v[a], column(rows, r[a], c));
            }
            Raw<float, C> before;
            if (!TO_ROWS && g.accumulate) before.load(column((const float*)g.out, t * g.H, c));
            if constexpr (DOT) {
#pragma unroll
                for (int a = 0; a < KK; ++a)
                    if ((held >> a) & 1) {
#pragma unroll
                        for (int i = 0; i < C; ++i) dot[a] = fmaf(v[a].at(i), x.at(i), dot[a]);
                    }
            }
            if (!out) continue;
            Cols<C> y{};
            if constexpr (TO_ROWS) {
#pragma unroll
                for (int a = 0; a < KK; ++a)
                    if ((held >> a) & 1) {
#pragma unroll
                        for (int i = 0; i < C; ++i) y.v[i] = w[a] * x.at(i);
                        store_cols<C>(column(out, r[a], c), y);
                    }
            } else {
#pragma unroll
                for (int a = 0; a < KK; ++a)
                    if ((held >> a) & 1) {
#pragma unroll
                        for (int i = 0; i < C; ++i) y.v[i] = fmaf(w[a], v[a].at(i), y.v[i]);
                    }
                if (g.accumulate)
#pragma unroll
                    for (int i = 0; i < C; ++i) y.v[i] += before.at(i);
                store_cols<C>(column(out, t * g.H, c), y);
            }
        }
        if constexpr (DOT) {
            const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
            const float sum = wave_sums<KK>(dot);
            if (lane % (64 / KK) == 0) part[wave][lane / (64 / KK)] = sum;
            __syncthreads();
            if (threadIdx.x < (unsigned)g.k) {
                float s = 0.0f;
                for (int q = 0; q < (int)blockDim.x / 64; ++q) s += part[q][threadIdx.x];
                g.dweights[t * g.k + threadIdx.x] = s;
            }
            __syncthreads();
        }
    }
}

constexpr int64_t kMostBlocks = 1 << 21;   // of up to 1024 threads, whose number is held in 32 bits
// Threads for a token's columns in `parts` workgroups, whole waves, the parts alike.
int threads_of(int64_t chunks, int parts, int most) {
    const int64_t share = ceil_div(chunks, parts);
    return (int)(share < most ? align_up(share, 64) : most);
}

template <class TOKEN, class ROW, class OUT, int KK, bool TO_ROWS, bool DOT, bool STREAM>
hipError_t rows_sized(RowsArgs g, hipStream_t s) {
    const int64_t chunks = g.H / kCols<TOKEN, ROW, OUT>;
    constexpr int kMost = DOT ? kDotThreads<TO_ROWS> : kThreads;
    const int pieces = (int)ceil_div(chunks, kMost);      // passes of a workgroup, or workgroups
    g.parts = DOT ? 1 : pieces;
    const int64_t items = g.T * g.parts;
    rows_kernel<TOKEN, ROW, OUT, KK, TO_ROWS, DOT, STREAM>
        <<<dim3((unsigned)(items < kMostBlocks ? items : kMostBlocks)), threads_of(chunks, pieces, kMost), 0, s>>>(g);
    return hipGetLastError();
}

template <class TOKEN, class ROW, class OUT, bool TO_ROWS, bool DOT, bool STREAM>
hipError_t rows_by_slots(const RowsArgs& g, hipStream_t s) {
    if (g.k <= 1) return rows_sized<TOKEN, ROW, OUT, 1, TO_ROWS, DOT, STREAM>(g, s);
    if (g.k <= 2) return rows_sized<TOKEN, ROW, OUT, 2, TO_ROWS, DOT, STREAM>(g, s);
    if (g.k <= 4) return rows_sized<TOKEN, ROW, OUT, 4, TO_ROWS, DOT, STREAM>(g, s);
    return rows_sized<TOKEN, ROW, OUT, 8, TO_ROWS, DOT, STREAM>(g, s);
}

template <class TOKEN, class ROW, class OUT, bool TO_ROWS, bool DOT>
hipError_t rows_by_size(const RowsArgs& g, hipStream_t s) {
    // (towards the rows alone none are read)
    if constexpr (TO_ROWS && !DOT) return rows_by_slots<TOKEN, ROW, OUT, TO_ROWS, DOT, false>(g, s);
    else return streamed(g.R * g.H * (int64_t)sizeof(ROW) + (DOT ? g.T * g.H * (int64_t)sizeof(TOKEN) : 0))
                    ? rows_by_slots<TOKEN, ROW, OUT, TO_ROWS, DOT, true>(g, s)
                    : rows_by_slots<TOKEN, ROW, OUT, TO_ROWS, DOT, false>(g, s);
}

// Without the products one side's rows are not read: its type is then the other's.
template <class TOKEN, class ROW, class OUT, bool TO_ROWS>
hipError_t rows_by_dot(const RowsArgs& g, hipStream_t s) {
    using ONE = std::conditional_t<TO_ROWS, TOKEN, ROW>;
    return g.dweights ? rows_by_size<TOKEN, ROW, OUT, TO_ROWS, true>(g, s) : rows_by_size<ONE, ONE, OUT, TO_ROWS, false>(g, s);
}

template <class OUT, bool TO_ROWS>
hipError_t rows_by_type(bool tokens_bf16, bool rows_bf16, const RowsArgs& g, hipStream_t s) {
    if (tokens_bf16)
        return rows_bf16 ? rows_by_dot<uint16_t, uint16_t, OUT, TO_ROWS>(g, s) : rows_by_dot<uint16_t, float, OUT, TO_ROWS>(g, s);
    return rows_bf16 ? rows_by_dot<float, uint16_t, OUT, TO_ROWS>(g, s) : rows_by_dot<float, float, OUT, TO_ROWS>(g, s);
}

// The token's paths: those whose two rows are there, and a row to read in any case (0 for a number that is no row; a
// token without paths reads none).
template <int K>
struct Paths {
    uint64_t bits;
    uint32_t srcs, tgts;     // which slots have rows
    int src[K], tgt[K];
    Scalar<float> beta;
};
template <int K>
__device__ __forceinline__ Paths<K> paths_of(const MixRowsArgs& g, int64_t t) {
    Paths<K> p;
    p.beta = scalar(g.beta) + t * (K * K);
    p.bits = scalar(g.bits)[t];
#pragma unroll
    for (int a = 0; a < K; ++a) {
        p.src[a] = scalar(g.src_row_of)[t * K + a];
        p.tgt[a] = scalar(g.tgt_row_of)[t * K + a];
    }
    p.srcs = p.tgts = 0;
    uint64_t from = 0, to = 0;
    constexpr uint64_t kRow = ((uint64_t)1 << K) - 1;
#pragma unroll
    for (int a = 0; a < K; ++a) {
        const bool s = (uint32_t)p.src[a] < (uint32_t)g.R_src, d = (uint32_t)p.tgt[a] < (uint32_t)g.R_tgt;
        p.srcs |= s ? 1u << a : 0u;
        p.tgts |= d ? 1u << a : 0u;
        p.src[a] = s ? p.src[a] : 0;
        p.tgt[a] = d ? p.tgt[a] : 0;
        from |= s ? kRow << (a * K) : 0;
    }
#pragma unroll
    for (int a = 0; a < K; ++a) to |= (uint64_t)p.tgts << (a * K);
    p.bits &= from & to;
    return p;
}

// BACK: the gradient by u alone, which is the mix of dz from the targets to the sources.
template <class IN, class OUT, int K, bool BACK, bool STREAM>
__global__ __launch_bounds__(kThreads) void mix_rows_kernel(MixRowsArgs g) {
    constexpr int C = kCols<IN, OUT>;
    const IN* __restrict__ in = (const IN*)(BACK ? g.dz : g.u);
    OUT* __restrict__ out = (OUT*)g.out;
    for (int64_t item = blockIdx.x; item < g.T * g.parts; item += gridDim.x) {
        const int64_t t = g.parts == 1 ? item : item / g.parts;
        const int part0 = (int)(item - t * g.parts);
        const Paths<K> p = paths_of<K>(g, t);
        float beta[K * K];
#pragma unroll
        for (int i = 0; i < K * K; ++i) beta[i] = p.beta[i];
        for (int c = (part0 * blockDim.x + threadIdx.x) * C; c < g.F; c += g.parts * blockDim.x * C) {
            Raw<IN, C> v[K];
            if (p.bits) {
#pragma unroll
                for (int a = 0; a < K; ++a) read<STREAM>(v[a], column(in, (int64_t)(BACK ? p.tgt[a] : p.src[a]) * g.F, c));
#pragma unroll
                for (int a = 0; a < K; ++a) v[a].arrived();
            }
#pragma unroll
            for (int b = 0; b < K; ++b) {
                if (!(((BACK ? p.srcs : p.tgts) >> b) & 1)) continue;
                Cols<C> s{};
#pragma unroll
                for (int a = 0; a < K; ++a) {
                    const int i = BACK ? b * K + a : a * K + b;
                    if ((p.bits >> i) & 1) {
                        const float w = beta[i];
#pragma unroll
                        for (int q = 0; q < C; ++q) s.v[q] = fmaf(w, v[a].at(q), s.v[q]);
                    }
                }
                store_cols<C>(column(out, (int64_t)(BACK ? p.src[b] : p.tgt[b]) * g.F, c), s);
            }
        }
    }
}

// A wave takes A of a token's K sources, all targets and every per-th step of 64 C columns: A * K sums for dbeta in registers
// next to the rows. All lanes of a wave stay active (past the last column on the last ones again, as zeros), so that the sums
// cross the whole wave. Eight sources in one wave left two waves on a SIMD, waiting (8192 tokens, F 1024: 89 us; two of four
// sources 81; four of two 88). The products on the matrix cores instead, as a corner of X X^T of all a token's rows X, took 106: rows
// in pieces of half a line, and dz a second time for du.
template <class IN, class OUT, int K, int A, int C, bool STREAM>
__global__ __launch_bounds__(kGradThreads) void mix_rows_grad_kernel(MixRowsArgs g, int per) {
    constexpr int N = pow2_above(A * K), kShares = (K + A - 1) / A;
    constexpr bool kTwice = kShares * A > K;
    __shared__ float part[kGradThreads / 64][N];
    const IN* __restrict__ u = (const IN*)g.u;
    const IN* __restrict__ dz = (const IN*)g.dz;
    OUT* __restrict__ du = (OUT*)g.out;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // waves: tokens, shares of their sources, shares of the columns
    const int group = wave / per, sub = wave - group * per, mine = group / kShares, share = group - mine * kShares, a0 = share ? K - A : 0;
    const int tokens = blockDim.x / 64 / per / kShares;
    for (int64_t t0 = (int64_t)blockIdx.x * tokens; t0 < g.T; t0 += (int64_t)gridDim.x * tokens) {
        const int64_t t = t0 + mine;
        float dot[N];
#pragma unroll
        for (int i = 0; i < N; ++i) dot[i] = 0.0f;
        if (t < g.T) {
            const Paths<K> p = paths_of<K>(g, t);
            // (of an odd number the source in the middle is the first share's)
            const uint64_t bits = share && kTwice ? p.bits >> (a0 * K) & ~(((uint64_t)1 << K) - 1) : p.bits >> (a0 * K);
            const uint32_t srcs = share && kTwice ? p.srcs >> a0 & ~1u : p.srcs >> a0;
            float beta[A * K];
#pragma unroll
            for (int i = 0; i < A * K; ++i) beta[i] = p.beta[a0 * K + i];
            int src[A];
#pragma unroll
            for (int a = 0; a < A; ++a) {
                src[a] = p.src[0];
#pragma unroll
                for (int q = 1; q < K; ++q) src[a] = a0 + a == q ? p.src[q] : src[a];
            }
            for (int c0 = sub * 64 * C; c0 < g.F; c0 += per * 64 * C) {
                const int at = c0 + lane * C, c = min(at, g.F - C);
                Raw<IN, C> v[A], d[K];
                if (p.bits) {
#pragma unroll
                    for (int a = 0; a < A; ++a) read<STREAM>(v[a], column(u, (int64_t)src[a] * g.F, c));
#pragma unroll
                    for (int b = 0; b < K; ++b) read<STREAM && kShares == 1>(d[b], column(dz, (int64_t)p.tgt[b] * g.F, c));
#pragma unroll
                    for (int a = 0; a < A; ++a) v[a].arrived();
#pragma unroll
                    for (int b = 0; b < K; ++b) d[b].arrived();
                }
                if (c0 + 64 * C > g.F) {
#pragma unroll
                    for (int a = 0; a < A; ++a) v[a].zero_unless(at < g.F);
#pragma unroll
                    for (int b = 0; b < K; ++b) d[b].zero_unless(at < g.F);
                }
#pragma unroll
                for (int a = 0; a < A; ++a) {
                    Cols<C> s{};
#pragma unroll
                    for (int b = 0; b < K; ++b)
                        if ((bits >> (a * K + b)) & 1) {
                            const float w = beta[a * K + b];
#pragma unroll
                            for (int i = 0; i < C; ++i) {
                                s.v[i] = fmaf(w, d[b].at(i), s.v[i]);
                                dot[a * K + b] = fmaf(v[a].at(i), d[b].at(i), dot[a * K + b]);
                            }
                        }
                    if (du && ((srcs >> a) & 1) && at < g.F) store_cols<C>(column(du, (int64_t)src[a] * g.F, at), s);
                }
            }
        }
        const float sum = wave_sums<N>(dot);
        constexpr int kLanes = 64 / N;
        const int i = lane / kLanes, skip = share && kTwice ? K : 0;   // elements of dbeta [skip, A K) are this wave's
        float* const out = g.dbeta + t * (K * K) + a0 * K;
        if (per == 1) {
            if (t < g.T && lane % kLanes == 0 && i >= skip && i < A * K) out[i] = sum;
            continue;
        }
        if (lane % kLanes == 0) part[wave][i] = sum;
        __syncthreads();
        if (sub == 0 && t < g.T && lane >= skip && lane < A * K) {
            float s = 0.0f;
            for (int q = 0; q < per; ++q) s += part[wave + q][lane];
            out[lane] = s;
        }
        __syncthreads();
    }
}

template <class IN, class OUT, int K, bool STREAM>
hipError_t mix_sized(bool grad, MixRowsArgs g, hipStream_t s) {
    if (grad && g.dbeta) {
        // A step of 64 C columns a wave (few experts, 7 steps / 1: 131 / 122 us; top-4, F 1408, 3 steps / 1: 107 / 104); where a
        // wave's sums are many, four (top-8, F 1024, 4 steps / 2 / 1: 82 / 85 / 113). As many tokens a workgroup as have at
        // most four waves together, one at least. Above four slots a lane takes four columns of bf16 too: eight do not fit in the
        // 128 registers of 1024 threads and go to scratch memory (top-8, 8192 tokens, F 1024, 4 columns / 8: 82 / 2665; F 2048
        // 159 / 3738).
        constexpr int A = K > 4 ? (K + 1) / 2 : K, C = K > 4 ? 4 : kCols<IN, OUT>, kShares = K > 4 ? 2 : 1, kSteps = K > 4 ? 4 : 1;
        constexpr int kMost = kGradThreads / 64 / kShares;
        const int64_t wanted = ceil_div(g.F, 64 * C * kSteps);
        const int per = (int)(wanted < kMost ? wanted : kMost), tokens = per * kShares < 4 ? 4 / (per * kShares) : 1;
        const int64_t blocks = ceil_div(g.T, tokens);
        mix_rows_grad_kernel<IN, OUT, K, A, C, STREAM>
            <<<dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks)), per * kShares * tokens * 64, 0, s>>>(g, per);
        return hipGetLastError();
    }
    const int64_t chunks = g.F / kCols<IN, OUT>;
    g.parts = (int)ceil_div(chunks, kThreads);
    const int threads = threads_of(chunks, g.parts, kThreads);
    const int64_t items = g.T * g.parts;
    const dim3 grid((unsigned)(items < kMostBlocks ? items : kMostBlocks));
    if (grad) mix_rows_kernel<IN, OUT, K, true, STREAM><<<grid, threads, 0, s>>>(g);
    else mix_rows_kernel<IN, OUT, K, false, STREAM><<<grid, threads, 0, s>>>(g);
    return hipGetLastError();
}

template <class IN, class OUT, bool STREAM>
hipError_t mix_by_slots(bool grad, const MixRowsArgs& g, hipStream_t s) {
    switch (g.k) {
        case 1: return mix_sized<IN, OUT, 1, STREAM>(grad, g, s);
        case 2: return mix_sized<IN, OUT, 2, STREAM>(grad, g, s);
        case 3: return mix_sized<IN, OUT, 3, STREAM>(grad, g, s);
        case 4: return mix_sized<IN, OUT, 4, STREAM>(grad, g, s);
        case 5: return mix_sized<IN, OUT, 5, STREAM>(grad, g, s);
        case 6: return mix_sized<IN, OUT, 6, STREAM>(grad, g, s);
        case 7: return mix_sized<IN, OUT, 7, STREAM>(grad, g, s);
        default: return mix_sized<IN, OUT, 8, STREAM>(grad, g, s);
    }
}

template <class IN, class OUT>
hipError_t mix_by_size(bool grad, const MixRowsArgs& g, hipStream_t s) {
    const int64_t bytes = ((g.u ? g.R_src : 0) + (grad ? g.R_tgt : 0)) * g.F * (int64_t)sizeof(IN);
    return streamed(bytes) ? mix_by_slots<IN, OUT, true>(grad, g, s) : mix_by_slots<IN, OUT, false>(grad, g, s);
}

}  // namespace

hipError_t launch_rows(bool to_rows, bool tokens_bf16, bool rows_bf16, bool out_bf16, const RowsArgs& g, hipStream_t s) {
    if (to_rows)
        return out_bf16 ? rows_by_type<uint16_t, true>(tokens_bf16, rows_bf16, g, s) : rows_by_type<float, true>(tokens_bf16, rows_bf16, g, s);
    return out_bf16 ? rows_by_type<uint16_t, false>(tokens_bf16, rows_bf16, g, s) : rows_by_type<float, false>(tokens_bf16, rows_bf16, g, s);
}

hipError_t launch_mix_rows(bool grad, bool bf16, bool out_bf16, const MixRowsArgs& g, hipStream_t s) {
    if (bf16) return out_bf16 ? mix_by_size<uint16_t, uint16_t>(grad, g, s) : mix_by_size<uint16_t, float>(grad, g, s);
    return out_bf16 ? mix_by_size<float, uint16_t>(grad, g, s) : mix_by_size<float, float>(grad, g, s);
}

}  // namespace pcm
