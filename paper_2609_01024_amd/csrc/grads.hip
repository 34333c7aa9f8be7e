// The router's gradient from those of the weights it gave, and the norm over all gradients with clipping.
#include "pcomoe.h"

#include "eight.h"

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
// Bound by its launch and by writing [T, n]: 8 threads a token, the rows of 32 tokens built in LDS.
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
// A launch takes up to GradTable::kMost tensors, cut into chunks of kChunk elements; a workgroup takes a run of
// neighbouring chunks. Squares and their sums are 64 bits: no gradient that float32 holds overflows or vanishes in them.
constexpr int kChunk = 4096, kNormThreads = 256;

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

__device__ __forceinline__ float element(const uint16_t* p, int64_t i) { return bf16_bits_to_f32(p[i]); }
__device__ __forceinline__ float element(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ void put(uint16_t* p, int64_t i, float v) { p[i] = __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ void put(float* p, int64_t i, float v) { p[i] = v; }

template <class IN>
__device__ __forceinline__ double chunk_squares(const IN* p, int64_t lo, int64_t hi) {
    double s = 0.0;
    for (int64_t i = lo + threadIdx.x; i < hi; i += kNormThreads) {
        const double v = (double)element(p, i);
        s = fma(v, v, s);
    }
    return s;
}

__global__ __launch_bounds__(kNormThreads) void norm_kernel(GradTable g, uint32_t per, double* __restrict__ parts) {
    __shared__ double red[kNormThreads / 64];
    const uint32_t chunks = g.start[g.m];
    const uint32_t from = blockIdx.x * per, to = min(chunks, from + per);
    double sum = 0.0;
    int i = from < to ? tensor_of(g, from) : 0;
    for (uint32_t c = from; c < to; ++c) {
        while (c >= g.start[i + 1]) ++i;
        const int64_t lo = (int64_t)(c - g.start[i]) * kChunk, hi = min(g.count[i], lo + kChunk);
        sum += g.type[i] & 1 ? chunk_squares((const uint16_t*)g.src[i], lo, hi) : chunk_squares((const float*)g.src[i], lo, hi);
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
__device__ __forceinline__ void chunk_scaled(const IN* p, OUT* q, int64_t lo, int64_t hi, float f) {
    for (int64_t i = lo + threadIdx.x; i < hi; i += kNormThreads) put(q, i, element(p, i) * f);
}

// parts: the norm is formed from them here (and written by the first workgroup); otherwise it is read.
__global__ __launch_bounds__(kNormThreads) void clip_kernel(GradTable g, uint32_t per, const double* parts, int count, float* norm,
                                                            int write_norm, float max_norm) {
    __shared__ double red[kNormThreads / 64];
    const float v = parts ? norm_of(parts, count, red) : *norm;
    if (parts && write_norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = v;
    // A norm that is not finite leaves the gradients as they are.
    const bool clip = v > max_norm && v < __builtin_inff();
    const float f = clip ? (float)((double)max_norm / (double)v) : 1.0f;
    const uint32_t chunks = g.start[g.m];
    const uint32_t from = blockIdx.x * per, to = min(chunks, from + per);
    int i = from < to ? tensor_of(g, from) : 0;
    for (uint32_t c = from; c < to; ++c) {
        while (c >= g.start[i + 1]) ++i;
        if (!clip && g.dst[i] == g.src[i]) continue;
        const int64_t lo = (int64_t)(c - g.start[i]) * kChunk, hi = min(g.count[i], lo + kChunk);
        switch (g.type[i]) {
            case 0: chunk_scaled((const float*)g.src[i], (float*)g.dst[i], lo, hi, f); break;
            case 1: chunk_scaled((const uint16_t*)g.src[i], (float*)g.dst[i], lo, hi, f); break;
            case 2: chunk_scaled((const float*)g.src[i], (uint16_t*)g.dst[i], lo, hi, f); break;
            default: chunk_scaled((const uint16_t*)g.src[i], (uint16_t*)g.dst[i], lo, hi, f); break;
        }
    }
}

// The table of grads[0, m), and the workgroups that share its chunks.
struct Launch {
    GradTable table;
    uint32_t per, blocks;
};
bool launch_of(const pcm_tensor* in, const pcm_tensor* out, int m, Launch* l) {
    uint64_t chunks = 0;
    l->table.m = m;
    for (int i = 0; i < m; ++i) {
        l->table.src[i] = in[i].data;
        l->table.dst[i] = out ? out[i].data : in[i].data;
        l->table.count[i] = in[i].count;
        l->table.type[i] = (uint8_t)((in[i].dtype == PCM_BF16 ? 1 : 0) | ((out ? out[i] : in[i]).dtype == PCM_BF16 ? 2 : 0));
        l->table.start[i] = (uint32_t)chunks;
        chunks += (uint64_t)ceil_div(in[i].count, kChunk);
        if (chunks >> 31) return false;
    }
    l->table.start[m] = (uint32_t)chunks;
    l->per = (uint32_t)ceil_div((int64_t)chunks, kGradBlocks);
    l->blocks = chunks ? (uint32_t)ceil_div((int64_t)chunks, l->per) : 0;
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
    int count = 0;
    Launch l;
    if (parts) {
        for (int at = 0; at < m; at += GradTable::kMost) {
            if (!launch_of(in + at, nullptr, m - at < GradTable::kMost ? m - at : GradTable::kMost, &l)) return hipErrorInvalidValue;
            if (!l.blocks) continue;
            norm_kernel<<<l.blocks, kNormThreads, 0, s>>>(l.table, l.per, parts + count);
            count += (int)l.blocks;
        }
        if (!clip || !count) {
            norm_join_kernel<<<1, kNormThreads, 0, s>>>(parts, count, norm);
            return hipGetLastError();
        }
    }
    bool first = true;
    for (int at = 0; at < m; at += GradTable::kMost) {
        if (!launch_of(in + at, out ? out + at : nullptr, m - at < GradTable::kMost ? m - at : GradTable::kMost, &l))
            return hipErrorInvalidValue;
        if (!l.blocks) continue;
        clip_kernel<<<l.blocks, kNormThreads, 0, s>>>(l.table, l.per, parts, count, norm, first, max_norm);
        first = false;
    }
    return hipGetLastError();
}

}  // namespace pcm
