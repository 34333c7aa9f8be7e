// Products grouped by expert, their gradients and their 8-bit form: one tile loop for every operand
// layout and element type, and the search for a workgroup's tile.
//
// A tile is C[i, j] = sum_k A[i, k] B[j, k] over the contraction k. Each operand lies in memory
//   along k (KC: a row i holds consecutive k; x and dy rows, and w rows of the forward product), or
//   across k (KS: a row k holds consecutive i; w of the input gradient, dy and x of the weight's).
// Both come through LDS in slices of 128 bytes of k for every i (64 bf16, 32 float32 or 128 8-bit
// values), NS slices in a ring of global -> LDS loads of 1 KB each, one barrier per slice.
//   KC rows are 128 bytes, the 16-byte chunk c of row r at c ^ ((r >> 1) & 7): fragment reads (16 rows,
//      4 chunks) touch every bank once.
//   KS rows k hold the tile's columns; units of 16 columns (32 bytes of bf16, 64 of float32) sit at
//      u ^ f(k), so that the rows one read touches lie in different banks. bf16 fragments are read
//      with the transposing LDS load (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 columns, lane i
//      gets column i of the four rows), float32 ones value by value.
// The MFMA takes B as its first operand: a lane's four sums are four consecutive columns j of one row i.
// The last slice of a contraction that is no multiple of the slice: loads past the end repeat the last
// valid data, and fragments are cleared there in registers, both operands (a NaN or an infinity times a
// cleared value would still be NaN).
#pragma once
#include "gemm_common.h"

namespace pcm {
namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));

// Bounds of group e, held inside [0, R] whatever the offsets are.
__device__ __forceinline__ void clamp_group(int R, int& lo, int& cnt) {
    const int hi = min(max(lo + cnt, 0), R);
    lo = min(max(lo, 0), R);
    cnt = max(hi - lo, 0);
}

template <int BM_, int BN_, int WM_, int WN_, int NS_>
struct TileCfg {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NS = NS_;
    static constexpr int NW = WM * WN, NT = NW * 64;
    static constexpr int WTM = BM / WM, WTN = BN / WN, MB = WTM / 16, NBK = WTN / 16;
    static constexpr int QA = BM / 8 / NW, QB = BN / 8 / NW;   // loads per wave and slice
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "every wave issues the same loads");
    static_assert(WTM % 16 == 0 && WTN % 16 == 0 && 128 % WTN == 0, "whole MFMA blocks within one scale block");
};

// A workgroup barrier that neither the compiler's nor its scheduler's reordering crosses.
__device__ __forceinline__ void tile_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// ------------------------------------------------------------------------ element types
// KB: values of k per slice. UNIT: bytes of a KS unit. Frag: a lane's values of one fragment (of two a slice).
struct TBf16 {
    static constexpr int SIZE = 2, KB = 64, UNIT = 32;
    static constexpr bool SCALED = false;
    using Frag = bf16x8;
    // f(k) of the KS layout: the rows that 32 lanes read together (k = 0-3 and 8-11 of their block) in
    // different units; rows of 128 bytes alternate banks by themselves.
    __device__ static int swizzle(int k, int rb) {
        return rb >= 256 ? (k & 3) | ((k >> 3) & 1) << 2 : ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
    }
    __device__ static Frag kc(const char* p) { return *(const Frag*)p; }
    // rows k = 32 s + 8 kg + 0..7 of column unit u
    template <int RB>
    __device__ static Frag ks(const char* tile, int s, int u, int lane) {
        const int i = lane & 15, kg = lane >> 4, f = swizzle((kg & 1) * 8 + (i >> 2), RB);
        const char* p = tile + (8 * kg + (i >> 2)) * RB + (u ^ f) * UNIT + (i & 3) * 8;
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PCM_LDS shortx4*)(p + 32 * s * RB));
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PCM_LDS shortx4*)(p + (32 * s + 4) * RB));
        return __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // clears the values at k >= rem
    __device__ static Frag head(Frag v, int s, int kg, int rem) {
        intx4 w = __builtin_bit_cast(intx4, v);
        const int k0 = 32 * s + 8 * kg;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] &= k0 + 2 * i + 1 < rem ? -1 : k0 + 2 * i < rem ? 0xFFFF : 0;
        return __builtin_bit_cast(Frag, w);
    }
    __device__ static floatx4 step(const Frag& b, const Frag& a, floatx4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, c, 0, 0, 0);
    }
};

struct TF32 {
    static constexpr int SIZE = 4, KB = 32, UNIT = 64;
    static constexpr bool SCALED = false;
    using Frag = floatx4;
    __device__ static int swizzle(int k, int rb) { return (k >> 2) & (rb >= 256 ? 3 : 1); }
    __device__ static Frag kc(const char* p) { return *(const Frag*)p; }
    // rows k = 16 s + 4 kg + 0..3 of column unit u
    template <int RB>
    __device__ static Frag ks(const char* tile, int s, int u, int lane) {
        const int i = lane & 15, kg = lane >> 4;
        const char* p = tile + (16 * s + 4 * kg) * RB + (u ^ swizzle(4 * kg, RB)) * UNIT + i * 4;
        return Frag{*(const float*)p, *(const float*)(p + RB), *(const float*)(p + 2 * RB), *(const float*)(p + 3 * RB)};
    }
    __device__ static Frag head(Frag v, int s, int kg, int rem) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 16 * s + 4 * kg + i < rem ? v[i] : 0.0f;
        return v;
    }
    __device__ static floatx4 step(const Frag& b, const Frag& a, floatx4 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(b[j], a[j], c, 0, 0, 0);
        return c;
    }
};

// e4m3 values with scales. A lane's 32 values of a row are the chunks kg and kg + 4 of the slice; which k
// they are does not matter, as both operands are read alike.
struct E4m3 {
    static constexpr int SIZE = 1, KB = 128, UNIT = 32;
    static constexpr bool SCALED = true;
    using Frag = intx8;
    __device__ static Frag kc2(const char* p0, const char* p1) {
        const intx4 lo = *(const intx4*)p0, hi = *(const intx4*)p1;
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    __device__ static Frag head(Frag v, int kg, int rem) {   // rem: a multiple of 16
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = 16 * kg < rem ? v[i] : 0;
            v[i + 4] = 64 + 16 * kg < rem ? v[i + 4] : 0;
        }
        return v;
    }
};
// Results in bf16: one 8-bit MFMA of 128 k per slice. It aligns the products of neighbouring k to the
// largest of them and cuts what lies below 2^-13 of that (as measured with pairs of powers of two; the
// 16x16x32 8-bit MFMA does the same): 1.3e-5 of the result's norm on normal values, against 1.7e-3 of the
// rounding to bf16.
struct TE4m3 : E4m3 {
    using Value = intx8;
    __device__ static Value value(const Frag& v) { return v; }
    __device__ static floatx4 product(const Value& b, const Value& a) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
    }
};
// Results in float32: the values as bf16 (exact), four bf16 MFMAs, float32 sums to the last bit.
struct TE4m3Wide : E4m3 {
    struct Value {
        bf16x8 v[4];
    };
    __device__ static Value value(const Frag& f) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        Value r;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[i], 1.0f, false);
            const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[i], 1.0f, true);
            const int j = (i & 1) * 4;
            r.v[i / 2][j] = lo[0];
            r.v[i / 2][j + 1] = lo[1];
            r.v[i / 2][j + 2] = hi[0];
            r.v[i / 2][j + 3] = hi[1];
        }
        return r;
    }
    __device__ static floatx4 product(const Value& b, const Value& a) {
        floatx4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[i], a.v[i], c, 0, 0, 0);
        return c;
    }
};

template <class E, class C>
struct Slots {   // LDS: a ring of slices (A rows, B rows, then, for 8-bit operands, one scale per row and wave)
    static constexpr int SA = C::BM * 128, SB = C::BN * 128;
    static constexpr int SLICE = SA + SB + (E::SCALED ? C::NW * 256 : 0);
    static constexpr int BYTES = C::NS * SLICE;
    static_assert(BYTES <= 160 * 1024 && C::BM <= C::NW * 64, "LDS; a scale load per wave covers the rows");
};

// One operand of a tile: where this lane's loads of a slice come from.
template <class E, class C, int B_, int Q_, bool KS>
struct Side {
    static constexpr int RB = B_ * E::SIZE;
    static_assert(!KS || (RB >= 128 && RB <= 1024), "KS: four or more units of bf16 columns, two or more of float32");
    const char* p[Q_];
    int64_t step;   // bytes from a slice to the next
    int64_t ld;     // KS: bytes of a row k

    __device__ static int blk(int q, int wave) { return q * C::NW + wave; }
    __device__ static int row(int q, int wave, int lane) {   // KC: row of the tile; KS: row k of the slice
        return KS ? (blk(q, wave) * 1024 + lane * 16) / RB : blk(q, wave) * 8 + (lane >> 3);
    }
    __device__ static int chunk(int q, int wave, int lane) {   // KC: byte offset of this lane's 16 bytes in the row
        return ((lane & 7) ^ ((row(q, wave, lane) >> 1) & 7)) * 16;
    }
    __device__ static int column(int q, int wave, int lane) {   // KS: byte offset of the 16 bytes among the columns
        const int c = (blk(q, wave) * 1024 + lane * 16) % RB;
        return ((c / E::UNIT) ^ E::swizzle(row(q, wave, lane), RB)) * E::UNIT + c % E::UNIT;
    }
    // how far load q of a slice with rem valid k has to step back to stay inside
    __device__ int64_t over(int q, int wave, int lane, int rem) const {
        if (KS) return (int64_t)max(row(q, wave, lane) - (rem - 1), 0) * ld;
        return max(chunk(q, wave, lane) - (rem * E::SIZE - 16), 0);
    }
};

// Fragments of one slice, and their products into the accumulators.
template <class E, class C, bool A_KS, bool B_KS>
__device__ __forceinline__ void slice_products(const char* S, int wm, int wn, int lane, bool tail, int rem,
                                               floatx4 (&acc)[C::NBK][C::MB], float ws) {
    const int r16 = lane & 15, kg = lane >> 4;
    const char* SB = S + Slots<E, C>::SA;
    auto at = [&](int s) { return r16 * 128 + (((4 * s + kg) ^ ((r16 >> 1) & 7)) * 16); };
    if constexpr (E::SCALED) {
        typename E::Frag bf[C::NBK], af[C::MB];
        float scale[C::MB];
#pragma unroll
        for (int nb = 0; nb < C::NBK; ++nb) {
            const char* p = SB + (wn * C::WTN + nb * 16) * 128;
            bf[nb] = E::kc2(p + at(0), p + at(1));
        }
#pragma unroll
        for (int mb = 0; mb < C::MB; ++mb) {
            const int r = wm * C::WTM + mb * 16;
            af[mb] = E::kc2(S + r * 128 + at(0), S + r * 128 + at(1));
            scale[mb] = *(const float*)(SB + Slots<E, C>::SB + (r + r16) * 4) * ws;
        }
        if (tail) {
#pragma unroll
            for (int nb = 0; nb < C::NBK; ++nb) bf[nb] = E::head(bf[nb], kg, rem);
#pragma unroll
            for (int mb = 0; mb < C::MB; ++mb) af[mb] = E::head(af[mb], kg, rem);
        }
        typename E::Value av[C::MB];
#pragma unroll
        for (int mb = 0; mb < C::MB; ++mb) av[mb] = E::value(af[mb]);
#pragma unroll
        for (int nb = 0; nb < C::NBK; ++nb) {
            const typename E::Value bv = E::value(bf[nb]);
#pragma unroll
            for (int mb = 0; mb < C::MB; ++mb) {
                const floatx4 p = E::product(bv, av[mb]);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nb][mb][i] = fmaf(p[i], scale[mb], acc[nb][mb][i]);
            }
        }
    } else {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            typename E::Frag bf[C::NBK], af[C::MB];
#pragma unroll
            for (int nb = 0; nb < C::NBK; ++nb) {
                const int r = wn * C::WTN + nb * 16;
                if constexpr (B_KS) bf[nb] = E::template ks<C::BN * E::SIZE>(SB, s, r / 16, lane);
                else bf[nb] = E::kc(SB + r * 128 + at(s));
            }
#pragma unroll
            for (int mb = 0; mb < C::MB; ++mb) {
                const int r = wm * C::WTM + mb * 16;
                if constexpr (A_KS) af[mb] = E::template ks<C::BM * E::SIZE>(S, s, r / 16, lane);
                else af[mb] = E::kc(S + r * 128 + at(s));
            }
            if (tail) {
#pragma unroll
                for (int nb = 0; nb < C::NBK; ++nb) bf[nb] = E::head(bf[nb], s, kg, rem);
#pragma unroll
                for (int mb = 0; mb < C::MB; ++mb) af[mb] = E::head(af[mb], s, kg, rem);
            }
#pragma unroll
            for (int nb = 0; nb < C::NBK; ++nb)
#pragma unroll
                for (int mb = 0; mb < C::MB; ++mb) acc[nb][mb] = E::step(bf[nb], af[mb], acc[nb][mb]);
        }
    }
}

// The tile's sums over a contraction of `len` (>= 1) values. GATHER: the B rows k of slice t are the rows
// gather[t * KB + ..] of b_base (clamped to x_rows), plus this lane's column offset, B.p; their indices are
// loaded a slice ahead. sa: this lane's scale of the first slice (8-bit operands), wsc: the wave's.
template <class E, class C, bool A_KS, bool B_KS, bool GATHER>
__device__ __forceinline__ void tile_loop(Side<E, C, C::BM, C::QA, A_KS>& A, Side<E, C, C::BN, C::QB, B_KS>& B, int len,
                                          char* lds, floatx4 (&acc)[C::NBK][C::MB], const int32_t* gather,
                                          int64_t x_rows, const float* sa, const float* wsc) {
    using L = Slots<E, C>;
    static_assert(!GATHER || B_KS, "rows k are gathered");
    constexpr int PER = C::QA + C::QB + (GATHER ? C::QB : 0) + (E::SCALED ? 1 : 0);   // memory operations per slice
    static_assert((C::NS - 2) * PER <= 62, "vmcnt range");
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / C::WN, wn = wave % C::WN;
    const int KT = (len + E::KB - 1) / E::KB;
    int idx[C::QB];
    auto index = [&](int q, int kt) { return gather[min(kt * E::KB + B.row(q, wave, lane), len - 1)]; };
    if constexpr (GATHER)
#pragma unroll
        for (int q = 0; q < C::QB; ++q) idx[q] = index(q, 0);
    auto issue = [&](int slot, int kt) {
        char* S = lds + slot * L::SLICE;
        const int rem = len - kt * E::KB;
        const bool tail = rem < E::KB;   // uniform
        int next[C::QB];
        if constexpr (GATHER)
#pragma unroll
            for (int q = 0; q < C::QB; ++q) next[q] = index(q, kt + 1);
#pragma unroll
        for (int q = 0; q < C::QA; ++q) {
            const char* p = A.p[q];
            if (tail) p -= A.over(q, wave, lane, rem);
            __builtin_amdgcn_global_load_lds((const PCM_GLOBAL void*)p, (PCM_LDS void*)(S + A.blk(q, wave) * 1024), 16, 0, 0);
            A.p[q] += A.step;
        }
#pragma unroll
        for (int q = 0; q < C::QB; ++q) {
            const char* p = B.p[q];
            if constexpr (GATHER) {
                const int64_t r = idx[q];
                p += (r < 0 ? 0 : r >= x_rows ? x_rows - 1 : r) * B.ld;
                idx[q] = next[q];
            } else {
                if (tail) p -= B.over(q, wave, lane, rem);
                B.p[q] += B.step;
            }
            __builtin_amdgcn_global_load_lds((const PCM_GLOBAL void*)p,
                                             (PCM_LDS void*)(S + L::SA + B.blk(q, wave) * 1024), 16, 0, 0);
        }
        if constexpr (E::SCALED) {
            __builtin_amdgcn_global_load_lds((const PCM_GLOBAL void*)sa, (PCM_LDS void*)(S + L::SA + L::SB + wave * 256), 4, 0, 0);
            ++sa;
        }
    };
#pragma unroll
    for (int s = 0; s < C::NS - 1; ++s)
        if (s < KT) issue(s, s);
    for (int base = 0; base < KT; base += C::NS) {
#pragma unroll
        for (int j = 0; j < C::NS; ++j) {
            const int kt = base + j;
            if (kt >= KT) break;
            // slice kt has landed (this wave's loads of it; the barrier covers the others'), and
            // every wave is done with slice kt - 1, whose slot takes slice kt + NS - 1
            if (kt + C::NS - 2 < KT) __builtin_amdgcn_s_waitcnt(waitcnt_imm((C::NS - 2) * PER, 0));
            else __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
            tile_barrier();
            if (kt + C::NS - 1 < KT) issue((j + C::NS - 1) % C::NS, kt + C::NS - 1);
            const int rem = len - kt * E::KB;
            float ws = 1.0f;
            if constexpr (E::SCALED) ws = wsc[kt];
            slice_products<E, C, A_KS, B_KS>(lds + j * L::SLICE, wm, wn, lane, rem < E::KB, rem, acc, ws);
        }
    }
}

// ------------------------------------------------------------------------ output
__device__ __forceinline__ void store4(float* p, floatx4 v) { *(floatx4*)p = v; }
// bf16: one rounding to nearest even of the float32 sum
__device__ __forceinline__ void store4(__bf16* p, floatx4 v) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *(bf16x4*)p = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
}

// acc[nb][mb] holds C[row = .. + (lane & 15)][columns .. + 4 (lane >> 4) + 0..3] (columns: a multiple of 16).
template <class C, class OUT, bool ADD>
__device__ __forceinline__ void store_tile(OUT* out, int64_t row0, int rows, int col0, int cols, int wave, int lane,
                                           const floatx4 (&acc)[C::NBK][C::MB]) {
    const int wm = wave / C::WN, wn = wave % C::WN;
#pragma unroll
    for (int mb = 0; mb < C::MB; ++mb) {
        const int r = wm * C::WTM + mb * 16 + (lane & 15);
        if (r >= rows) continue;
#pragma unroll
        for (int nb = 0; nb < C::NBK; ++nb) {
            const int c = col0 + wn * C::WTN + nb * 16 + (lane >> 4) * 4;
            if (c >= cols) continue;
            OUT* p = out + (row0 + r) * cols + c;
            floatx4 v = acc[nb][mb];
            if constexpr (ADD) v += *(const floatx4*)p;
            store4(p, v);
        }
    }
}

// ------------------------------------------------------------------------ which tile
// Tile of this workgroup among ceil(rows / BM) x nt tiles of every group, expert-major: a group's tiles
// in blocks of max(1, window / row tiles) column tiles, the row tile varying slowest in a block; each XCD
// (workgroup id % 8) takes a contiguous eighth of the list. s_item: group, row0, row1, column tile, found.
// Groups 4 * lane .. 4 * lane + 3 of wave 0 count; n <= 256.
template <int BM>
__device__ bool group_item(const GroupArgs& g, int nt, int window, int* s_item) {
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        int lo[4], cnt[4], m[4], local = 0;
        group_bounds(g.offsets, g.n, g.R, lane, lo, cnt);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            clamp_group((int)g.R, lo[j], cnt[j]);
            m[j] = (cnt[j] + BM - 1) / BM;
            local += m[j] * nt;
        }
        const int incl = wave_incl_scan_i32(local);
        const int total = __builtin_amdgcn_readlane(incl, 63);
        const int x8 = (int)(blockIdx.x % 8), j8 = (int)(blockIdx.x / 8);
        const int l0 = (int)((int64_t)x8 * total / 8), l1 = (int)((int64_t)(x8 + 1) * total / 8);
        const bool valid = j8 < l1 - l0;
        if (lane == 0) s_item[4] = valid ? 1 : 0;
        if (valid) {
            const int id = l0 + j8;
            int start = incl - local, hit = -1, l = 0, mm_ = 1, lo_ = 0, cnt_ = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in = id >= start && id < start + m[j] * nt;
                hit = in ? j : hit;
                l = in ? id - start : l;
                mm_ = in ? m[j] : mm_;
                lo_ = in ? lo[j] : lo_;
                cnt_ = in ? cnt[j] : cnt_;
                start += m[j] * nt;
            }
            if (hit >= 0) {
                int gn = window / mm_;
                gn = gn < 1 ? 1 : (gn > nt ? nt : gn);
                const int gsize = gn * mm_;
                const int grp = l / gsize, in = l - grp * gsize;
                const int gcols = min(gn, nt - grp * gn);
                const int mm = in / gcols;
                const int r0 = lo_ + mm * BM;
                s_item[0] = lane * 4 + hit;
                s_item[1] = r0;
                s_item[2] = min(lo_ + cnt_, r0 + BM);
                s_item[3] = grp * gn + (in - mm * gcols);
            }
        }
    }
    __syncthreads();
    return s_item[4] != 0;
}

// Most row tiles of BM rows that R rows make in n groups.
inline int64_t most_row_tiles(const GroupArgs& g, int BM) {
    if (!g.offsets) return ceil_div(g.R, BM);
    return (g.R + (int64_t)(BM - 1) * (g.R < g.n ? g.R : g.n)) / BM;
}

// ------------------------------------------------------------------------ kernels
// out[r, :] = x[s(r), :] . b[e]^T (DX false: b [n, cols, len]) or dy[r, :] . b[e] (DX true: b [n, len, cols]),
// rows r of group e.
template <class E, class C, bool DX, class OUT>
__global__ __launch_bounds__(C::NT) void group_rows_kernel(GroupArgs g, int nt, int window) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    int* const s_item = (int*)lds;   // read into registers before the first loads overwrite it
    if (!group_item<C::BM>(g, nt, window, s_item)) return;   // workgroup-uniform
    const int e = __builtin_amdgcn_readfirstlane(s_item[0]), row0 = __builtin_amdgcn_readfirstlane(s_item[1]);
    const int row1 = __builtin_amdgcn_readfirstlane(s_item[2]), ntile = __builtin_amdgcn_readfirstlane(s_item[3]);
    __syncthreads();
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t lenb = (int64_t)g.len * E::SIZE, colb = (int64_t)g.cols * E::SIZE;
    auto source = [&](int r) -> int64_t {   // rows past row1 repeat the last (never stored)
        r = min(r, row1 - 1);
        if (!g.gather) return r;
        const int64_t t = g.gather[r];
        return t < 0 ? 0 : t >= g.x_rows ? g.x_rows - 1 : t;
    };
    Side<E, C, C::BM, C::QA, false> A;
    Side<E, C, C::BN, C::QB, DX> B;
    int64_t src[C::QA];   // every row index is loaded before any is used
#pragma unroll
    for (int q = 0; q < C::QA; ++q) src[q] = source(row0 + A.row(q, wave, lane));
#pragma unroll
    for (int q = 0; q < C::QA; ++q) A.p[q] = (const char*)g.a + src[q] * lenb + A.chunk(q, wave, lane);
    A.step = 128;
    A.ld = 0;
    const char* bg = (const char*)g.b + (int64_t)e * g.len * colb;
    const int col0 = ntile * C::BN;
#pragma unroll
    for (int q = 0; q < C::QB; ++q) {
        if constexpr (DX)   // columns past the end repeat the last 16 bytes (never stored)
            B.p[q] = bg + B.row(q, wave, lane) * colb + min((int64_t)col0 * E::SIZE + B.column(q, wave, lane), colb - 16);
        else
            B.p[q] = bg + (int64_t)min(col0 + B.row(q, wave, lane), g.cols - 1) * lenb + B.chunk(q, wave, lane);
    }
    B.step = DX ? E::KB * colb : 128;
    B.ld = colb;
    const float *sa = nullptr, *wsc = nullptr;
    if constexpr (E::SCALED) {
        const int kb = (g.len + 127) / 128, nb = (g.cols + 127) / 128;
        sa = g.a_scale + source(row0 + (wave * 64 + lane) % C::BM) * kb;
        wsc = g.b_scale + ((int64_t)e * nb + min((col0 + wave % C::WN * C::WTN) / 128, nb - 1)) * kb;
    }
    floatx4 acc[C::NBK][C::MB];
#pragma unroll
    for (int i = 0; i < C::NBK; ++i)
#pragma unroll
        for (int j = 0; j < C::MB; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    tile_loop<E, C, false, DX, false>(A, B, g.len, lds, acc, nullptr, 0, sa, wsc);
    store_tile<C, OUT, false>((OUT*)g.out, row0, row1 - row0, col0, g.cols, wave, lane, acc);
}

// out[e] [rows, cols] = sum over the rows r of group e of a[r, :]^T b[s(r), :].
template <class E, class C, bool GATHER, class OUT, bool ADD>
__global__ __launch_bounds__(C::NT) void group_outer_kernel(GroupArgs g, int mt, int nt) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t total = (int64_t)g.n * mt * nt;
    const int64_t per = (total + 7) / 8, id = (int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8;
    if ((int64_t)(blockIdx.x / 8) >= per || id >= total) return;
    const int e = (int)(id / ((int64_t)mt * nt)), in = (int)(id - (int64_t)e * mt * nt);
    const int mtile = in / nt, ntile = in - mtile * nt;
    int lo = 0, cnt = (int)g.R;
    if (g.offsets) {
        lo = g.offsets[e];
        cnt = g.offsets[e + 1] - lo;
        clamp_group((int)g.R, lo, cnt);
    }
    if (ADD && cnt == 0) return;
    const int64_t ab = (int64_t)g.rows * E::SIZE, bb = (int64_t)g.cols * E::SIZE;
    Side<E, C, C::BM, C::QA, true> A;
    Side<E, C, C::BN, C::QB, true> B;
#pragma unroll
    for (int q = 0; q < C::QA; ++q)
        A.p[q] = (const char*)g.a + (lo + A.row(q, wave, lane)) * ab +
                 min((int64_t)mtile * C::BM * E::SIZE + A.column(q, wave, lane), ab - 16);
    A.step = E::KB * ab;
    A.ld = ab;
#pragma unroll
    for (int q = 0; q < C::QB; ++q)
        B.p[q] = (const char*)g.b + (GATHER ? 0 : (lo + B.row(q, wave, lane)) * bb) +
                 min((int64_t)ntile * C::BN * E::SIZE + B.column(q, wave, lane), bb - 16);
    B.step = E::KB * bb;
    B.ld = bb;
    floatx4 acc[C::NBK][C::MB];
#pragma unroll
    for (int i = 0; i < C::NBK; ++i)
#pragma unroll
        for (int j = 0; j < C::MB; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (cnt > 0)
        tile_loop<E, C, true, true, GATHER>(A, B, cnt, lds, acc, GATHER ? g.gather + lo : nullptr, g.x_rows, nullptr, nullptr);
    store_tile<C, OUT, ADD>((OUT*)g.out + (int64_t)e * g.rows * g.cols, mtile * C::BM, g.rows - mtile * C::BM,
                            ntile * C::BN, g.cols, wave, lane, acc);
}

template <class K>
hipError_t allow_lds(K kernel, int bytes) {   // set on every launch (idempotent; the library keeps no state)
    return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <class E, class C, bool DX, class OUT>
hipError_t launch_rows(const GroupArgs& g, int window, hipStream_t s) {
    const int nt = (int)ceil_div(g.cols, C::BN);
    const int64_t grid = ceil_div(most_row_tiles(g, C::BM) * nt, 8) * 8;
    if (grid >= int64_t(1) << 28) return hipErrorInvalidValue;   // counted in 32 bits
    const hipError_t err = allow_lds(group_rows_kernel<E, C, DX, OUT>, Slots<E, C>::BYTES);
    if (err != hipSuccess) return err;
    group_rows_kernel<E, C, DX, OUT><<<dim3((unsigned)grid), dim3(C::NT), Slots<E, C>::BYTES, s>>>(g, nt, window);
    return hipGetLastError();
}

template <class E, class C, bool GATHER, class OUT, bool ADD>
hipError_t launch_outer_(const GroupArgs& g, hipStream_t s) {
    const int mt = (int)ceil_div(g.rows, C::BM), nt = (int)ceil_div(g.cols, C::BN);
    const int64_t grid = ceil_div((int64_t)g.n * mt * nt, 8) * 8;
    if (grid >= int64_t(1) << 28) return hipErrorInvalidValue;
    const hipError_t err = allow_lds(group_outer_kernel<E, C, GATHER, OUT, ADD>, Slots<E, C>::BYTES);
    if (err != hipSuccess) return err;
    group_outer_kernel<E, C, GATHER, OUT, ADD><<<dim3((unsigned)grid), dim3(C::NT), Slots<E, C>::BYTES, s>>>(g, mt, nt);
    return hipGetLastError();
}
template <class E, class C, class OUT, bool ADD>
hipError_t launch_outer(const GroupArgs& g, hipStream_t s) {
    return g.gather ? launch_outer_<E, C, true, OUT, ADD>(g, s) : launch_outer_<E, C, false, OUT, ADD>(g, s);
}

}  // namespace
}  // namespace pcm
