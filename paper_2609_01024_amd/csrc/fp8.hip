// 8-bit floating point (e4m3) with a float32 scale for each block of 128: the quantisers and the product.
// A block with largest finite magnitude m has a = max(m, 2^-100), scale = a / 448 and values
// e4m3(x * (448 / a)), to nearest even: every finite value lands within e4m3's largest, 448. The floor
// keeps 448 / a finite. What is not finite becomes NaN and has no part in the scale.
// The quantisers are bound by memory: rows 16384 x 7168 bf16 65 us (5.5 TB/s read and written), SwiGLU of 32768 x
// 2 x 1408 41 us (5.7), 64 weights of 2048 x 1024 with their transposes 104 us (5.1 of the 5.1 TB/s that a
// copy has). The product: 8192^3 2060 TF into bf16; 8 experts of 14336 x 4096 with 8192 rows 560-580 us; 256
// of 2048 x 7168 with one row each 345-360 us (weights at 6.7-7 TB/s).
#include "columns.h"
#include "grouped.h"

namespace pcm {
namespace {

constexpr float kE4m3Max = 448.0f;
constexpr float kFloor = 0x1p-100f;

typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));

// magnitude bits of v, 0 for infinities and NaN
__device__ __forceinline__ uint32_t finite_bits(float v) {
    const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}

template <bool FINITE>
__device__ __forceinline__ uint32_t block_max(const Eight& x) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, FINITE ? finite_bits(x.v[i]) : __float_as_uint(x.v[i]) & 0x7FFFFFFFu);
    return m;
}
// largest of the 16 lanes of a DPP row, on each of them
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
    v = max(v, dpp_u32<0xB1>(v));
    v = max(v, dpp_u32<0x4E>(v));
    v = max(v, dpp_u32<0x141>(v));
    return max(v, dpp_u32<0x140>(v));
}

// The block's largest finite magnitude: all values first, the finite ones again where that finds another.
__device__ __forceinline__ uint32_t row16_block_max(const Eight& x) {
    const uint32_t m = row16_max(block_max<false>(x));
    return __any(m >= 0x7F800000u) ? row16_max(block_max<true>(x)) : m;
}

__device__ __forceinline__ uint32_t four_e4m3(float a, float b, float c, float d) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ uintx2 eight_e4m3(const Eight& x, float inv) {
    return uintx2{four_e4m3(x.v[0] * inv, x.v[1] * inv, x.v[2] * inv, x.v[3] * inv),
                  four_e4m3(x.v[4] * inv, x.v[5] * inv, x.v[6] * inv, x.v[7] * inv)};
}

// Rows in blocks of 128 columns: 16 lanes take a block, 8 values each; the maximum stays in registers.
template <class IN, bool SWIGLU>
__global__ __launch_bounds__(256) void quant_rows_kernel(const IN* __restrict__ x, const int32_t* __restrict__ count,
                                                         int64_t R, int K, uint8_t* __restrict__ q,
                                                         float* __restrict__ scale) {
    const int kb = (K + 127) / 128, part = threadIdx.x & 15;
    int64_t rows = R;
    if (count) rows = min(R, (int64_t)max(*count, 0));
    const int64_t total = rows * kb;
    for (int64_t b = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); b < total; b += (int64_t)gridDim.x * 16) {
        const int64_t r = b / kb;
        const int c = (int)(b - r * kb) * 128 + part * 8;
        Eight v{};
        if (c < K) {
            if constexpr (SWIGLU) {
                const Eight g = load8(x + r * 2 * K + c), u = load8(x + r * 2 * K + K + c);
#pragma unroll
                for (int i = 0; i < 8; ++i) v.v[i] = gated(IN(), g.v[i], u.v[i]);
            } else {
                v = load8(x + r * K + c);
            }
        }
        const float a = fmaxf(__uint_as_float(row16_block_max(v)), kFloor);
        if (c < K) *(uintx2*)(q + r * K + c) = eight_e4m3(v, kE4m3Max / a);
        if (part == 0) scale[b] = a / kE4m3Max;
    }
}

// One 128 x 128 block of a weight per workgroup: 16 rows at a time, 8 passes, all values in registers
// until the block's maximum is known. The transposed codes go through LDS.
template <class IN>
__global__ __launch_bounds__(256) void quant_weights_kernel(const IN* __restrict__ w, int N, int K, uint8_t* __restrict__ q,
                                                            float* __restrict__ scale, uint8_t* __restrict__ q_t,
                                                            float* __restrict__ scale_t) {
    constexpr int kPitch = 132;
    __shared__ uint32_t s_max[4];
    __shared__ __attribute__((aligned(16))) uint8_t codes[128 * kPitch];
    const int nb = (N + 127) / 128, kb = (K + 127) / 128;
    const int64_t b = blockIdx.x, e = b / (nb * kb);
    const int ib = (int)(b - e * nb * kb) / kb, jb = (int)(b - e * nb * kb) % kb;
    const int part = threadIdx.x & 15, r0 = threadIdx.x >> 4, c = jb * 128 + part * 8;
    w += e * N * K;
    Eight v[8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = ib * 128 + i * 16 + r0;
        v[i] = Eight{};
        if (r < N && c < K) v[i] = load8(w + (int64_t)r * K + c);
        m = max(m, block_max<true>(v[i]));
    }
    m = wave_max_u32(m);
    if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    const float a = fmaxf(__uint_as_float(m), kFloor), inv = kE4m3Max / a;
    if (threadIdx.x == 0) {
        scale[b] = a / kE4m3Max;
        if (scale_t) scale_t[e * nb * kb + (int64_t)jb * nb + ib] = a / kE4m3Max;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = ib * 128 + i * 16 + r0;
        const uintx2 eight = eight_e4m3(v[i], inv);
        if (r < N && c < K) *(uintx2*)(q + (e * N + r) * K + c) = eight;
        if (q_t) {
            uint32_t* p = (uint32_t*)(codes + (i * 16 + r0) * kPitch + part * 8);
            p[0] = eight[0];
            p[1] = eight[1];
        }
    }
    if (!q_t) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {   // row k of W^T: 8 values of n from 8 rows
        const int k = i * 16 + r0, n = ib * 128 + part * 8;
        if (jb * 128 + k >= K || n >= N) continue;
        uint32_t t[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j / 4] |= (uint32_t)codes[(part * 8 + j) * kPitch + k] << (8 * (j % 4));
        *(uintx2*)(q_t + (e * K + jb * 128 + k) * N + n) = uintx2{t[0], t[1]};
    }
}

using Narrow = TileCfg<32, 64, 2, 2, 4>;     // three workgroups on a compute unit
using Small = TileCfg<64, 64, 2, 2, 3>;      // three
using Middle = TileCfg<64, 128, 2, 2, 3>;    // two
using Square = TileCfg<128, 128, 2, 2, 2>;   // two
using Wide = TileCfg<128, 256, 2, 4, 3>;     // one, eight waves of 64 x 64

// Tiles as for 16-bit products, measured on both sides of every bound (one group, a contraction of 4096, us, this
// tile / the next smaller):
//   into bf16     128 x 256  112 tiles 29.3 / 39.7, 96 tiles 29.0 / 26.1, 64 tiles 28.7 / 22.2. (8192^3, an earlier
//                            step: 128 x 256 1780 TF, 256 x 128 1590, 128 x 128 1650; 256 x 256 does not fit the
//                            registers.) Many groups of few rows do not need a bound of their own (4096 columns, a
//                            contraction of 2048, this / 64 x 64): 64 groups of 17 rows 109 / 108, 32 114 / 113, 64
//                            122 / 146, 96 128 / 172; 128 groups of 32 218 / 220, 48 223 / 231
//                 64 x 64    320 tiles 21.7 / 20.9 (32 x 64), 512 tiles 22.2 / 29.8; 256 tiles 19.4 / 17.2
//   into float32  128 x 128  448 tiles 71.2 / 82.0, 256 tiles 49.6 / 44.1; groups of fewer than 96 rows leave much of
//                            such a tile empty (64 groups of 32: 87 / 66)
//                 64 x 128   448 tiles 43.1 / 50.9, 512 tiles 44.1 / 50.8, 384 tiles 43.3 / 38.7
//   16 rows of 64 columns, per-wave rings: float32, 512 tiles 17.2, 32 x 64 18.3; bf16, 256 tiles 10.0, 64 x
//   64 18.9; 512 tiles 14.7, 32 x 64 14.7
template <class E, class OUT>
hipError_t fp8_by_shape(const GroupArgs& g, hipStream_t s) {
    if (!near(g, 1)) return launch_rows<E, Small, Small, false, OUT, int64_t>(g, 8, s);
    auto tiles = [&](int bm, int bn) { return expected_row_tiles(g, bm) * ceil_div(g.cols, bn); };
    if (few_rows(g, 1, E::PAIRS ? 14 : 16) || tiles(16, 64) <= (E::PAIRS ? 256 : 512)) return launch_thin<E, OUT>(g, 8, weights_once(g, 1), s);
    if (tiles(64, 64) <= 256) return launch_rows<E, Narrow, Narrow, false, OUT>(g, 8, s);
    if constexpr (E::PAIRS) {
        if (tiles(128, 256) >= 100) return launch_rows<E, Wide, Wide, false, OUT>(g, 8, s);
    } else {
        if (tiles(128, 128) >= 400 && mean_rows(g) >= 96) return launch_rows<E, Square, Square, false, OUT>(g, 8, s);
        if (tiles(64, 128) >= 400) return launch_rows<E, Middle, Middle, false, OUT>(g, 8, s);
    }
    return launch_rows<E, Small, Small, false, OUT>(g, 8, s);
}

}  // namespace

hipError_t launch_quant_rows(bool bf16, bool swiglu, const void* x, const int32_t* count, int64_t R, int K, uint8_t* q,
                             float* scale, hipStream_t s) {
    const int64_t blocks = ceil_div(R * ceil_div(K, 128), 16);
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), block(256);
    if (bf16) {
        const uint16_t* p = (const uint16_t*)x;
        if (swiglu) quant_rows_kernel<uint16_t, true><<<grid, block, 0, s>>>(p, count, R, K, q, scale);
        else quant_rows_kernel<uint16_t, false><<<grid, block, 0, s>>>(p, count, R, K, q, scale);
    } else {
        const float* p = (const float*)x;
        if (swiglu) quant_rows_kernel<float, true><<<grid, block, 0, s>>>(p, count, R, K, q, scale);
        else quant_rows_kernel<float, false><<<grid, block, 0, s>>>(p, count, R, K, q, scale);
    }
    return hipGetLastError();
}

hipError_t launch_quant_weights(bool bf16, const void* w, int n, int N, int K, uint8_t* q, float* scale, uint8_t* q_t,
                                float* scale_t, hipStream_t s) {
    const int64_t blocks = (int64_t)n * ceil_div(N, 128) * ceil_div(K, 128);
    if (blocks >= int64_t(1) << 31) return hipErrorInvalidValue;
    if (bf16)
        quant_weights_kernel<<<dim3((unsigned)blocks), dim3(256), 0, s>>>((const uint16_t*)w, N, K, q, scale, q_t, scale_t);
    else
        quant_weights_kernel<<<dim3((unsigned)blocks), dim3(256), 0, s>>>((const float*)w, N, K, q, scale, q_t, scale_t);
    return hipGetLastError();
}

hipError_t launch_grouped_fp8(bool out_bf16, const GroupArgs& g, hipStream_t s) {
    return out_bf16 ? fp8_by_shape<TE4m3, __bf16>(g, s) : fp8_by_shape<TE4m3AsBf16, float>(g, s);
}

}  // namespace pcm
