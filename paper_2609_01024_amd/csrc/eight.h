// Eight neighbouring columns in float32 registers, read from and written to rows of bf16 (uint16_t) or float32,
// and SiLU(gate) * up of them.
#pragma once
#include "internal.h"

namespace pcm {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

struct Eight {
    float v[8];
};
__device__ __forceinline__ Eight load8(const uint16_t* p) {
    const uintx4 w = *(const uintx4*)p;
    Eight r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.v[2 * i] = __uint_as_float(w[i] << 16);
        r.v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
    return r;
}
__device__ __forceinline__ Eight load8(const float* p) {
    const floatx4 a = *(const floatx4*)p, b = *(const floatx4*)(p + 4);
    return Eight{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
// bf16: one rounding to nearest even
__device__ __forceinline__ void store8(uint16_t* p, const Eight& x) {
    *(bf16x8*)p = bf16x8{(__bf16)x.v[0], (__bf16)x.v[1], (__bf16)x.v[2], (__bf16)x.v[3],
                         (__bf16)x.v[4], (__bf16)x.v[5], (__bf16)x.v[6], (__bf16)x.v[7]};
}
__device__ __forceinline__ void store8(float* p, const Eight& x) {
    *(floatx4*)p = floatx4{x.v[0], x.v[1], x.v[2], x.v[3]};
    *(floatx4*)(p + 4) = floatx4{x.v[4], x.v[5], x.v[6], x.v[7]};
}

// SiLU(g) u in float32, near to correctly rounded: an error of some units in the last place would move as many
// more codes across a border between two. g / (1 + e^-g) alone would lose the gates from -88.8 down, whose
// exponential is infinite, and with the reciprocal instruction, whose results are never below the normal range, those
// from -87.4; SiLU(g) u is a plain number there where u is large.
// bf16 inputs (this is what the kernel has time for next to its memory traffic): e^-g = 2^i 2^f with i whole and f
// from fused multiply-adds (2^(-g log2 e) at once is off by |g| units), the hardware reciprocal (about 1 ulp), and
// both terms of the sum smaller by 2^60. i - 60 comes in the low bits of a sum with 1.5 2^23 and is added to the
// exponent; the bounds keep that exponent in range and do not change the result (e^-40 is nothing beside 1, and
// from g = -120 down the result is 0). 32768 x 2 x 1408: 40 us, as with neither; a choice between two forms 42.7.
// float32 inputs: the library exponential and an IEEE division; below -80 1 + e^g is 1 and SiLU(g) = g e^g.
__device__ __forceinline__ float gated(uint16_t, float g, float u) {
    constexpr float kLog2e = 1.44269504088896340736f, kWhole = 0x1.8p23f - 60.0f, kDown = 0x1p-60f;
    const float c = __builtin_amdgcn_fmed3f(-g, -40.0f, 120.0f);
    const float n = fmaf(c, kLog2e, kWhole), f = fmaf(c, kLog2e, kWhole - n);
    const float e = __uint_as_float(__float_as_uint(__builtin_amdgcn_exp2f(f)) + (__float_as_uint(n) << 23));
    return g * (__builtin_amdgcn_rcpf(kDown + e) * kDown) * u;
}
__device__ __forceinline__ float gated(float, float g, float u) {
    const bool far = g < -80.0f;
    const float e = expf(far ? g : -g);
    return (far ? g * e : g / (1.0f + e)) * u;
}

}  // namespace pcm
