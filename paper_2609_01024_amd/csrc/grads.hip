// The router's gradient from those of the weights it gave, and the norm over all gradients with clipping.
#include "pcomoe.h"

#include "columns.h"

namespace pcm {
namespace {

// ---------------------------------------------------------------- router
// A token's weights p over its k experts are a softmax, and beta_ab follows from p (T_a: the targets of source a):
//   beta_ab = f_a p_b with   SRC_COND f_a = p_a / S_a, S_a = sum of p over T_a;   PRODUCT f_a = p_a;   GLOBAL f_a = p_a / Z,
//   Z the sum of p_a p_b over all paths.
// With G_a = sum over T_a of dbeta_ab p_b the gradient by p is
//   dp_c = dw_c + A_c + sum over a with c in T_a of f_a (dbeta_ac - h_a),
//   SRC_COND A_c = h_c = G_c / S_c;   PRODUCT A_c = G_c, h = 0;   GLOBAL h = sum_a p_a G_a / Z, A_c = (G_c - h S_c) / Z,
// and by the logits dl_a = p_a (dp_a - sum_c p_c dp_c). S_a = 0 (every p of T_a, p_a among them, below float32's range):
// what it would scale is multiplied by a zero p, so nothing is. Differences of sums that are near to each other: 64 bits.
// Bound by its launch and by writing [T, n]: 8 threads a token, the rows of 32 tokens built in LDS (16384 x 60: 5.5 us).
constexpr int kTokens = 32;

template <class OUT>
__global__ __launch_bounds__(kTokens * kMaxK) void route_grad_kernel(RouteGradArgs g) {
    __shared__ double s_p[kTokens][kMaxK], s_f[kTokens][kMaxK], s_h[kTokens][kMaxK], s_z[kTokens][kMaxK];
    extern __shared__ float tile[];   // [kTokens][n]
    const int a = threadIdx.x % kMaxK, j = threadIdx.x / kMaxK, k = g.k, n = g.n;
    for (int64_t t0 = (int64_t)blockIdx.x * kTokens; t0 < g.T; t0 += (int64_t)gridDim.x * kTokens) {
        const int64_t t = t0 + j;
        const bool mine = t < g.T && a < k;
        for (int i = threadIdx.x; i < kTokens * n; i += blockDim.x) tile[i] = 0.0f;
        const double p = mine ? (double)g.w[t * k + a] : 0.0;
        s_p[j][a] = p;
        __syncthreads();
        const uint64_t bits = mine && g.bits ? g.bits[t] : 0;
        const float* dbeta = g.dbeta + t * k * k;
        double G = 0.0, S = 0.0;
        if (mine)
            for (int b = 0; b < k; ++b)
                if ((bits >> (a * k + b)) & 1) {
                    G += (double)dbeta[a * k + b] * s_p[j][b];
                    S += s_p[j][b];
                }
        double A = G, f = p, h = 0.0;
        if (g.beta_mode == 0) {
            A = h = S > 0.0 ? G / S : 0.0;
            f = S > 0.0 ? p / S : 0.0;
        }
        if (g.beta_mode == 2) {
            s_f[j][a] = p * S;
            s_h[j][a] = p * G;
            __syncthreads();
            double Z = 0.0, D = 0.0;
            for (int c = 0; c < k; ++c) {
                Z += s_f[j][c];
                D += s_h[j][c];
            }
            __syncthreads();
            const double inv = Z > 0.0 ? 1.0 / Z : 0.0;
            h = D * inv;
            A = (G - h * S) * inv;
            f = p * inv;
        }
        s_f[j][a] = f;
        s_h[j][a] = h;
        __syncthreads();
        double dp = 0.0;
        if (mine) {
            dp = A + (g.dw ? (double)g.dw[t * k + a] : 0.0);
            for (int q = 0; q < k; ++q)
                if ((bits >> (q * k + a)) & 1) dp += s_f[j][q] * ((double)dbeta[q * k + a] - s_h[j][q]);
        }
        s_z[j][a] = p * dp;
        __syncthreads();
        if (mine) {
            double all = 0.0;
            for (int c = 0; c < k; ++c) all += s_z[j][c];
            const int e = g.ids[t * k + a];
            if ((unsigned)e < (unsigned)n) tile[j * n + e] = (float)(p * (dp - all));
        }
        __syncthreads();
        const int count = (int)min((int64_t)kTokens, g.T - t0) * n;
        OUT* out = (OUT*)g.dlogits + t0 * n;
        for (int i = threadIdx.x; i < count; i += blockDim.x) {
            if constexpr (sizeof(OUT) == 4) out[i] = tile[i];
            else out[i] = __builtin_bit_cast(uint16_t, (__bf16)tile[i]);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- all gradients
// A launch takes up to GradTable::kMost tensors, cut into chunks (of what is read) that begin at multiples of 16 bytes, wherever
// the tensor does. The vectors of 16 bytes at a tensor's ends that hold other bytes too go by elements. Squares and their
// sums are 64 bits: no gradient that float32 holds overflows or vanishes in them; nor do they cost time (1.4 G elements of bf16
// 445 us with sums of 8 in 32 bits too).
// Chunks of 4 vectors a thread for the norm, whose workgroups, six on a compute unit, all of them at once, take every so-manyeth
// chunk (1.4 G bf16, 100 M float32: 410 and 68 us, 6.9 and 5.9 TB/s; 2048 workgroups 445 and 86; 2 vectors and eight on a compute
// unit 426 and 65; 1 520 and 78), of 2 for the clipping, a chunk a workgroup: what writes runs at 6.5 TB/s read and
// written that way and at 5 with workgroups that loop (100 M float32, both passes: 2 vectors 193 us, 4 201, 1 208).
constexpr int kNormThreads = 256, kNormVectors = 4, kClipVectors = 2;
constexpr int chunk_bytes(int vectors) { return vectors * 16 * kNormThreads; }
// Sums of so many workgroups are added by every workgroup of the clipping, instead of by a launch of their own (us, without /
// with it: 8 MB 17.8 / 20.7, 16 MB 18.2 / 20.9, 24 MB 22.6 / 22.6, 48 MB, of 1536 sums, 35.4 / 33.8).
constexpr int kFewParts = kGradBlocks - 1;

__device__ __forceinline__ double block_sum(double v, double* part) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int q = 0; q < kNormThreads / 64; ++q) s += part[q];
    __syncthreads();
    return s;
}

// The tensor that holds chunk c: the last one that starts at it or before.
__device__ __forceinline__ int tensor_of(const GradTable& g, uint32_t c) {
    int lo = 0, hi = g.m - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (g.start[mid] <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <class T>
struct Vec;   // the elements of 16 bytes
template <>
struct Vec<uint16_t> {
    static constexpr int N = 8;
    float v[8];
};
template <>
struct Vec<float> {
    static constexpr int N = 4;
    float v[4];
};
__device__ __forceinline__ Vec<uint16_t> unpacked(const uint16_t*, uintx4 w) {
    Vec<uint16_t> r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.v[2 * i] = __uint_as_float(w[i] << 16);
        r.v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
    return r;
}
__device__ __forceinline__ Vec<float> unpacked(const float*, uintx4 w) {
    return Vec<float>{{__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3])}};
}
__device__ __forceinline__ float element(const uint16_t* p, int64_t i) { return bf16_bits_to_f32(p[i]); }
__device__ __forceinline__ float element(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ void put(uint16_t* p, int64_t i, float v) { p[i] = __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ void put(float* p, int64_t i, float v) { p[i] = v; }

// Chunk j of a tensor of `count` elements at p: whole(first element, vector) for each vector inside, part(element) for
// each element of the others. All vectors are loaded first.
template <int V, class T, class WHOLE, class PART>
__device__ __forceinline__ void each_vector(const T* p, int64_t count, int64_t j, WHOLE whole, PART part) {
    constexpr int N = Vec<T>::N;
    const int64_t before = ((uintptr_t)p & 15) / sizeof(T);     // elements of the first vector that lie before p
    const int64_t e0 = j * (chunk_bytes(V) / (int64_t)sizeof(T)) - before + threadIdx.x * N;
    uintx4 w[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int64_t e = e0 + i * (kNormThreads * N);
        if (e >= 0 && e + N <= count) w[i] = __builtin_nontemporal_load((const uintx4*)(p + e));
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int64_t e = e0 + i * (kNormThreads * N);
        if (e >= 0 && e + N <= count) whole(e, unpacked(p, w[i]));
        else
            for (int q = 0; q < N; ++q)
                if (e + q >= 0 && e + q < count) part(e + q);
    }
}

template <class T>
__device__ __forceinline__ double chunk_squares(const T* p, int64_t count, int64_t j) {
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    each_vector<kNormVectors>(
        p, count, j,
        [&](int64_t, const Vec<T>& x) {
#pragma unroll
            for (int i = 0; i < Vec<T>::N; ++i) s[i % 4] = fma((double)x.v[i], (double)x.v[i], s[i % 4]);
        },
        [&](int64_t e) {
            const double v = (double)element(p, e);
            s[0] = fma(v, v, s[0]);
        });
    return (s[0] + s[1]) + (s[2] + s[3]);
}

__global__ __launch_bounds__(kNormThreads) void norm_kernel(GradTable g, double* __restrict__ parts) {
    __shared__ double red[kNormThreads / 64];
    const uint32_t chunks = g.start[g.m];
    double sum = 0.0;
    int i = tensor_of(g, blockIdx.x);
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        while (c >= g.start[i + 1]) ++i;
        const int64_t j = c - g.start[i];
        sum += g.type[i] & 1 ? chunk_squares((const uint16_t*)g.src[i], g.count[i], j) : chunk_squares((const float*)g.src[i], g.count[i], j);
    }
    sum = block_sum(sum, red);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

// The norm from the workgroups' sums, added in one order by every workgroup that needs it.
__device__ __forceinline__ float norm_of(const double* parts, int count, double* red) {
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += kNormThreads) s += parts[i];
    return (float)sqrt(block_sum(s, red));
}

__global__ __launch_bounds__(kNormThreads) void norm_join_kernel(const double* __restrict__ parts, int count, float* __restrict__ norm) {
    __shared__ double red[kNormThreads / 64];
    const float v = norm_of(parts, count, red);
    if (threadIdx.x == 0) *norm = v;
}

template <class IN, class OUT>
__device__ __forceinline__ void chunk_scaled(const IN* p, OUT* q, int64_t count, int64_t j, float f) {
    constexpr int N = Vec<IN>::N, kBytes = N * (int)sizeof(OUT) < 16 ? N * (int)sizeof(OUT) : 16;
    // (an output whose elements lie otherwise than the input's to multiples of a vector)
    const bool aligned = (((uintptr_t)q - ((uintptr_t)p & 15) / sizeof(IN) * sizeof(OUT)) & (kBytes - 1)) == 0;
    each_vector<kClipVectors>(
        p, count, j,
        [&](int64_t e, const Vec<IN>& x) {
            if (!aligned) {
#pragma unroll
                for (int i = 0; i < N; ++i) put(q, e + i, x.v[i] * f);
                return;
            }
            Cols<N> y;
#pragma unroll
            for (int i = 0; i < N; ++i) y.v[i] = x.v[i] * f;
            if constexpr (N * sizeof(OUT) <= 16) {
                store_cols<N>(q + e, y);
            } else {   // two stores of neighbouring halves: their lines fill up in the cache (100 M bf16 147 us; not kept 164)
#pragma unroll
                for (int i = 0; i < N; i += 4) *(floatx4*)(q + e + i) = floatx4{y.v[i], y.v[i + 1], y.v[i + 2], y.v[i + 3]};
            }
        },
        [&](int64_t e) { put(q, e, element(p, e) * f); });
}

// parts: the norm is formed from them here (and written by the first workgroup); otherwise it is read.
__global__ __launch_bounds__(kNormThreads) void clip_kernel(GradTable g, const double* parts, int count, float* norm, int write_norm,
                                                            float max_norm) {
    __shared__ double red[kNormThreads / 64];
    const float v = parts ? norm_of(parts, count, red) : *norm;
    if (parts && write_norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = v;
    // A norm that is not finite leaves the gradients as they are.
    const bool clip = v > max_norm && v < __builtin_inff();
    const float f = clip ? (float)((double)max_norm / (double)v) : 1.0f;
    const uint32_t chunks = g.start[g.m];
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int i = tensor_of(g, c);
        if (!clip && g.dst[i] == g.src[i]) continue;
        const int64_t j = c - g.start[i], n = g.count[i];
        switch (g.type[i]) {
            case 0: chunk_scaled((const float*)g.src[i], (float*)g.dst[i], n, j, f); break;
            case 1: chunk_scaled((const uint16_t*)g.src[i], (float*)g.dst[i], n, j, f); break;
            case 2: chunk_scaled((const float*)g.src[i], (uint16_t*)g.dst[i], n, j, f); break;
            default: chunk_scaled((const uint16_t*)g.src[i], (uint16_t*)g.dst[i], n, j, f); break;
        }
    }
}

// The table of grads[0, m); false where its chunks are too many to count.
bool table_of(const pcm_tensor* in, const pcm_tensor* out, int m, int chunk, GradTable* g) {
    uint64_t chunks = 0;
    g->m = m;
    for (int i = 0; i < m; ++i) {
        const int64_t size = in[i].dtype == PCM_BF16 ? 2 : 4;
        g->src[i] = in[i].data;
        g->dst[i] = out ? out[i].data : in[i].data;
        g->count[i] = in[i].count;
        g->type[i] = (uint8_t)((in[i].dtype == PCM_BF16 ? 1 : 0) | ((out ? out[i] : in[i]).dtype == PCM_BF16 ? 2 : 0));
        g->start[i] = (uint32_t)chunks;
        if (in[i].count) chunks += (uint64_t)ceil_div((int64_t)((uintptr_t)in[i].data & 15) + in[i].count * size, chunk);
        if (chunks >> 31) return false;
    }
    g->start[m] = (uint32_t)chunks;
    return true;
}

}  // namespace

hipError_t launch_route_grad(bool out_bf16, const RouteGradArgs& g, hipStream_t s) {
    const int64_t blocks = ceil_div(g.T, kTokens);
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), block(kTokens * kMaxK);
    const size_t lds = (size_t)kTokens * g.n * sizeof(float);
    if (out_bf16) route_grad_kernel<uint16_t><<<grid, block, lds, s>>>(g);
    else route_grad_kernel<float><<<grid, block, lds, s>>>(g);
    return hipGetLastError();
}

size_t grad_norm_ws_bytes(int64_t m) { return (size_t)ceil_div(m > 0 ? m : 1, GradTable::kMost) * kGradBlocks * sizeof(double); }

hipError_t launch_grad_norm(const pcm_tensor* in, const pcm_tensor* out, int m, bool clip, float max_norm, float* norm, double* parts,
                            hipStream_t s) {
    constexpr int kMost = GradTable::kMost;
    int count = 0;
    GradTable g;
    if (parts) {
        for (int at = 0; at < m; at += kMost) {
            if (!table_of(in + at, nullptr, m - at < kMost ? m - at : kMost, chunk_bytes(kNormVectors), &g)) return hipErrorInvalidValue;
            const uint32_t chunks = g.start[g.m], blocks = chunks < kGradBlocks ? chunks : kGradBlocks;
            if (!blocks) continue;
            norm_kernel<<<blocks, kNormThreads, 0, s>>>(g, parts + count);
            count += (int)blocks;
        }
        if (!clip || count > kFewParts || !count) {
            norm_join_kernel<<<1, kNormThreads, 0, s>>>(parts, count, norm);
            if (!clip) return hipGetLastError();
            parts = nullptr;
        }
    }
    bool first = true;
    for (int at = 0; at < m; at += kMost) {
        if (!table_of(in + at, out ? out + at : nullptr, m - at < kMost ? m - at : kMost, chunk_bytes(kClipVectors), &g))
            return hipErrorInvalidValue;
        const uint32_t chunks = g.start[g.m], blocks = chunks < (1u << 22) ? chunks : (1u << 22);
        if (!blocks) continue;
        clip_kernel<<<blocks, kNormThreads, 0, s>>>(g, parts, count, norm, first, max_norm);
        first = false;
    }
    return hipGetLastError();
}

}  // namespace pcm
