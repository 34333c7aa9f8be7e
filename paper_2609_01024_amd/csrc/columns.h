// Neighbouring columns of rows of bf16 (uint16_t) or float32, read, widened to float32 and written, and SiLU(gate) * up.
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

// C neighbouring columns as they are read. They stay so until they are used, so that all of a thread's loads are on their
// way before the first wait. arrived(): waits for them here. Where they are used under branches, with stores between, the
// compiler waits again at every use, and a wait for a load is one for the stores before it too.
template <class T, int C>
struct Raw;
template <int C>
struct Raw<uint16_t, C> {
    typedef uint32_t words __attribute__((ext_vector_type(C / 2)));
    words w;
    __device__ __forceinline__ void load(const uint16_t* p) { w = *(const words*)p; }
    __device__ __forceinline__ void stream(const uint16_t* p) { w = __builtin_nontemporal_load((const words*)p); }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16); }
    __device__ __forceinline__ void zero_unless(bool keep) {
#pragma unroll
        for (int i = 0; i < C / 2; ++i) w[i] = keep ? w[i] : 0u;
    }
    __device__ __forceinline__ void arrived() { asm volatile("" : "+v"(w)); }
};
template <int C>
struct Raw<float, C> {
    floatx4 w[C / 4];
    __device__ __forceinline__ void load(const float* p) {
#pragma unroll
        for (int i = 0; i < C / 4; ++i) w[i] = *(const floatx4*)(p + 4 * i);
    }
    __device__ __forceinline__ void stream(const float* p) {
#pragma unroll
        for (int i = 0; i < C / 4; ++i) w[i] = __builtin_nontemporal_load((const floatx4*)(p + 4 * i));
    }
    __device__ __forceinline__ float at(int i) const { return w[i / 4][i % 4]; }
    __device__ __forceinline__ void zero_unless(bool keep) {
#pragma unroll
        for (int i = 0; i < C; ++i) w[i / 4][i % 4] = keep ? w[i / 4][i % 4] : 0.0f;
    }
    __device__ __forceinline__ void arrived() {
#pragma unroll
        for (int i = 0; i < C / 4; ++i) asm volatile("" : "+v"(w[i]));
    }
};
template <bool STREAM, class T, int C>
__device__ __forceinline__ void read(Raw<T, C>& r, const T* p) {
    if constexpr (STREAM) r.stream(p);
    else r.load(p);
}
// From 96 MB read on operands are loaded non-temporally: they are then hardly in the 256 MB of the last cache level, which the
// kernel that wrote them and this one's results share. us, non-temporally / plainly, tensors used in turn: SwiGLU 64 MB read 17.4 /
// 15.6, 128 MB 32.6 / 34.3, its gradient 48 MB 15.7 / 14.5, 96 MB 27.8 / 29.4; combine 64 MB 15.1 / 14.2, 128 MB 28.5 / 31.1, its
// gradient 80 MB 26.8 / 24.1, 160 MB 48.8 / 56.0; mix 64 MB 26.0 / 22.4, 128 MB 48.2 / 52.0, its gradient 64 MB 19.8 / 18.2, 128 MB
// 39.8 / 42.3.
inline bool streamed(int64_t bytes) { return bytes >= (int64_t)96 << 20; }
// Columns a thread takes: 16 bytes of float32, where there is any, or of bf16, so that a wave's access is one piece.
template <class... T>
constexpr int kCols = ((sizeof(T) == 2) && ...) ? 8 : 4;

// C columns of a result, in float32; bf16 is rounded once, to nearest even. Results are stored non-temporally: they are
// written once and read by a later kernel (dispatch of 8192 tokens to 8 rows of 2048 each 63 us -> 51).
template <int C>
struct Cols {
    float v[C];
};
template <int C>
__device__ __forceinline__ void store_cols(uint16_t* p, const Cols<C>& x) {
    typedef __bf16 out_t __attribute__((ext_vector_type(C)));
    out_t y;
#pragma unroll
    for (int i = 0; i < C; ++i) y[i] = (__bf16)x.v[i];
    __builtin_nontemporal_store(y, (out_t*)p);
}
template <int C>
__device__ __forceinline__ void store_cols(float* p, const Cols<C>& x) {
#pragma unroll
    for (int i = 0; i < C; i += 4)
        __builtin_nontemporal_store(floatx4{x.v[i], x.v[i + 1], x.v[i + 2], x.v[i + 3]}, (floatx4*)(p + i));
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
