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
#include <type_traits>

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

// Tile BM x BN on WM x WN waves; NSA slices of the rows side and NSB (NSA or NSA + 1) of the columns side
// in LDS.
template <int BM_, int BN_, int WM_, int WN_, int NSA_, int NSB_ = NSA_>
struct TileCfg {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NSA = NSA_, NSB = NSB_;
    static constexpr int NW = WM * WN, NT = NW * 64;
    static constexpr int WTM = BM / WM, WTN = BN / WN, MB = WTM / 16, NBK = WTN / 16;
    static constexpr int QA = BM / 8 / NW, QB = BN / 8 / NW;   // loads per wave and slice
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "every wave issues the same loads");
    static_assert(WTM % 16 == 0 && WTN % 16 == 0 && 128 % WTN == 0, "whole MFMA blocks within one scale block");
    static_assert(NSA >= 2 && (NSB == NSA || NSB == NSA + 1), "ring");
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
    static constexpr bool SCALED = false, PAIRS = false;
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
    static constexpr bool SCALED = false, PAIRS = false;
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
    __device__ static Frag head(Frag v, int, int kg, int rem) {   // rem: a multiple of 16
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
    static constexpr bool PAIRS = true;
    using Value = intx8;
    __device__ static Value value(const Frag& v) { return v; }
    __device__ static floatx4 product(const Value& b, const Value& a) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
    }
};
// Results in float32: the values as bf16 (exact), four bf16 MFMAs, float32 sums to the last bit.
struct TE4m3AsBf16 : E4m3 {
    static constexpr bool PAIRS = false;
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
struct Slots {   // LDS: NSA slices of A rows, NSB of B rows, then, for 8-bit operands, A's scales of 2 x 8 slices
    static constexpr int SA = C::BM * 128, SB = C::BN * 128, SS = C::BM * 32;
    static constexpr int B0 = C::NSA * SA, S0 = B0 + C::NSB * SB, BYTES = S0 + (E::SCALED ? 2 * SS : 0);
    static_assert(BYTES <= 160 * 1024, "LDS");
};

// A weight block's scales, the same for a wave, come by scalar loads: a vector load's wait would cover the
// slices on their way.
typedef const __attribute__((address_space(4))) float* ScalarPtr;

// Scales of A's rows (those of its loads), fetched for 8 slices at a time: one load a slice would touch a
// cache line for every row.
template <class C>
struct RowScales {
    const float* base;      // [x_rows, kb]
    int64_t off[C::QA];     // elements from base to this lane's row of load q
    int kb;
};

// 16 bytes a lane into 1 KB of LDS at `to`, from base (uniform) + voff + soff (uniform), or from p. Written as
// assembly because the compiler makes each transposing LDS load wait for every direct load before it,
// whatever slot that fills; tile_loop waits for slices itself. (They write no registers, and any vmcnt wait
// that the compiler counts without them is only the stricter for them.) "m0" takes the LDS address.
template <bool NT>
__device__ __forceinline__ void buffer_to_lds(const char* base, uint32_t voff, int soff, char* to) {
    const uint64_t b = (uint64_t)base;
    const intx4 r = {(int)b, (int)((b >> 32) & 0xFFFF), -1, 0x00020000};
    if constexpr (NT)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
                     :: "s"((uint32_t)(uintptr_t)(PCM_LDS char*)to), "v"(voff), "s"(r), "s"(soff) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :: "s"((uint32_t)(uintptr_t)(PCM_LDS char*)to), "v"(voff), "s"(r), "s"(soff) : "memory", "m0");
}
__device__ __forceinline__ void global_to_lds(const char* p, char* to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"((uint32_t)(uintptr_t)(PCM_LDS char*)to), "v"(p) : "memory", "m0");
}

// One operand of a tile: where this lane's loads of a slice come from: a uniform address that advances
// with the slices, and a fixed offset per lane (and, for KC rows, per load; KS loads are whole rows k apart).
// OFF: uint32_t, or int64_t where 32 bits do not reach.
template <class E, class C, int B_, int Q_, bool KS, class OFF>
struct Side {
    static constexpr int RB = B_ * E::SIZE;
    static_assert(!KS || (RB >= 128 && RB <= 1024), "KS: four or more units of bf16 columns, two or more of float32");
    static constexpr int QROWS = KS ? C::NW * 1024 / RB : 0;   // KS: rows k from a load to the next
    const char* base;
    OFF off[KS ? 1 : Q_];
    int64_t ld;     // KS: bytes of a row k

    __device__ static int blk(int q, int wave) { return q * C::NW + wave; }
    __device__ static int row(int q, int wave, int lane) {   // KC: row of the tile; KS: row k of the slice
        return KS ? (blk(q, wave) * 1024 + lane * 16) / RB : blk(q, wave) * 8 + (lane >> 3);
    }
    __device__ static int chunk(int q, int wave, int lane) {   // KC: byte offset of this lane's 16 bytes in the row
        return ((lane & 7) ^ ((row(q, wave, lane) >> 1) & 7)) * 16;
    }
    __device__ static int column(int wave, int lane) {   // KS: byte offset of the 16 bytes among the columns
        static_assert(!KS || QROWS % 16 == 0, "the same column for every load");
        const int c = (wave * 1024 + lane * 16) % RB;
        return ((c / E::UNIT) ^ E::swizzle(row(0, wave, lane), RB)) * E::UNIT + c % E::UNIT;
    }
    __device__ __forceinline__ void advance(int slices = 1) { base += slices * (KS ? E::KB * ld : 128); }
    // how far load q of a slice with rem < KB valid k steps back, to the last valid data again
    __device__ __forceinline__ int64_t back(int q, int wave, int lane, int rem) const {
        if (KS) return (int64_t)max(row(q, wave, lane) - (rem - 1), 0) * ld;
        return max(chunk(q, wave, lane) - (rem * E::SIZE - 16), 0);
    }
    // load q of the slice into LDS at `to` (1 KB a wave)
    template <bool NT = false>
    __device__ __forceinline__ void load(int q, char* to) const {
        if constexpr (sizeof(OFF) == 4) {
            buffer_to_lds<NT>(base, off[KS ? 0 : q], (int)(q * QROWS * ld), to);
        } else {
            const char* p = KS ? base + q * QROWS * ld + off[0] : base + off[KS ? 0 : q];
            global_to_lds(p, to);
        }
    }
    __device__ __forceinline__ void load_last(int q, char* to, int wave, int lane, int rem) const {
        const char* p = (KS ? base + q * QROWS * ld + off[0] : base + off[KS ? 0 : q]) - back(q, wave, lane, rem);
        global_to_lds(p, to);
    }
};

// The fragments of one step (half a slice; 8-bit operands: a slice) and their products.
template <class E, class C>
struct Step {
    typename E::Frag b[C::NBK], a[C::MB];
    float scale[E::SCALED ? C::MB : 1];

    static constexpr int N = C::NBK + C::MB;   // fragments, B's first
    template <bool A_KS, bool B_KS, int SCALE_STRIDE = 32>
    __device__ __forceinline__ void read(int j, const char* S, const char* SB, const char* SC, int s, int wm, int wn, int lane) {
        const int r16 = lane & 15, kg = lane >> 4;
        auto at = [&](int s) { return r16 * 128 + (((4 * s + kg) ^ ((r16 >> 1) & 7)) * 16); };
        if (j < C::NBK) {
            const int nb = j, r = wn * C::WTN + nb * 16;
            if constexpr (E::SCALED) b[nb] = E::kc2(SB + r * 128 + at(0), SB + r * 128 + at(1));
            else if constexpr (B_KS) b[nb] = E::template ks<C::BN * E::SIZE>(SB, s, r / 16, lane);
            else b[nb] = E::kc(SB + r * 128 + at(s));
        } else {
            const int mb = j - C::NBK, r = wm * C::WTM + mb * 16;
            if constexpr (E::SCALED) a[mb] = E::kc2(S + r * 128 + at(0), S + r * 128 + at(1));
            else if constexpr (A_KS) a[mb] = E::template ks<C::BM * E::SIZE>(S, s, r / 16, lane);
            else a[mb] = E::kc(S + r * 128 + at(s));
            if constexpr (E::SCALED) scale[mb] = *(const float*)(SC + (r + r16) * SCALE_STRIDE);
        }
    }
    __device__ __forceinline__ void head(int s, int kg, int rem) {   // clears what lies at k >= rem
#pragma unroll
        for (int nb = 0; nb < C::NBK; ++nb) b[nb] = E::head(b[nb], s, kg, rem);
#pragma unroll
        for (int mb = 0; mb < C::MB; ++mb) a[mb] = E::head(a[mb], s, kg, rem);
    }
    __device__ __forceinline__ void multiply(floatx4 (&acc)[C::NBK][C::MB], float ws) const {
        if constexpr (E::SCALED) {
            typename E::Value av[C::MB];
            float f[C::MB];
#pragma unroll
            for (int mb = 0; mb < C::MB; ++mb) {
                av[mb] = E::value(a[mb]);
                f[mb] = scale[mb] * ws;   // (one product a row; scaling the sums twice would double what stands beside an MFMA)
            }
#pragma unroll
            for (int nb = 0; nb < C::NBK; ++nb) {
                const typename E::Value bv = E::value(b[nb]);
#pragma unroll
                for (int mb = 0; mb < C::MB; ++mb) {
                    const floatx4 p = E::product(bv, av[mb]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[nb][mb][i] = fmaf(p[i], f[mb], acc[nb][mb][i]);
                }
            }
        } else {
#pragma unroll
            for (int nb = 0; nb < C::NBK; ++nb)
#pragma unroll
                for (int mb = 0; mb < C::MB; ++mb) acc[nb][mb] = E::step(b[nb], a[mb], acc[nb][mb]);
        }
    }
};

// The tile's sums over a contraction of `len` (>= 1) values. GATHER: the B rows k of slice t are the rows
// gather[t * KB + ..] of B.base (clamped to x_rows); their indices are loaded a slice ahead. rs, wsc: the scales of
// 8-bit operands, A's by row and the wave's of B by slice.
template <class E, class C, bool A_KS, bool B_KS, bool GATHER, class OFF>
__device__ __forceinline__ void tile_loop(Side<E, C, C::BM, C::QA, A_KS, OFF>& A, Side<E, C, C::BN, C::QB, B_KS, OFF>& B,
                                          int len, char* lds, floatx4 (&acc)[C::NBK][C::MB], const int32_t* gather,
                                          int64_t x_rows, const RowScales<C>* rs, ScalarPtr wsc) {
    using L = Slots<E, C>;
    static_assert(!GATHER || B_KS, "rows k are gathered");
    // A gather's load covers GR rows k in turn. Two of them: their indices come by scalar loads, for the wait on a
    // vector load drains the direct loads behind it (256 x 256 tiles: 64 groups of 2048 x 2048 664 -> 559 us,
    // as without a gather); four or more: selecting costs more than that (128 x 128 26 -> 46, float32 164 -> 179).
    constexpr int GR = GATHER ? 1024 / (C::BN * E::SIZE) : 1;
    constexpr bool GS = GATHER && GR <= 2;
    constexpr int PA = C::QA, PB = C::QB + (GATHER && !GS ? C::QB : 0), PER = PA + PB;
    // memory operations after those of slices kt + 1 when slice kt + NSA (A) and kt + NSB (B) are next
    constexpr int LATER = (C::NSA - 2) * PER + (C::NSB > C::NSA ? PB : 0);
    static_assert(LATER <= 62, "vmcnt range");
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / C::WN, wn = wave % C::WN, kg = lane >> 4;
    const int KT = (len + E::KB - 1) / E::KB, rem = len - (KT - 1) * E::KB;   // slices; values of the last
    char* const ldsb = lds + L::B0;
    typedef const __attribute__((address_space(4))) int32_t* ScalarInts;
    int idx[C::QB][GS ? GR : 1];
    auto index = [&](int q, int kt) {
        if constexpr (GS)
#pragma unroll
            for (int j = 0; j < GR; ++j) idx[q][j] = ((ScalarInts)gather)[min(kt * E::KB + B.blk(q, wave) * GR + j, len - 1)];
        else
            idx[q][0] = gather[min(kt * E::KB + B.row(q, wave, lane), len - 1)];
    };
    if constexpr (GATHER)
#pragma unroll
        for (int q = 0; q < C::QB; ++q) index(q, 0);
    // One load of A's next slice into its slot (8-bit operands: the last one also the scales), or of B's.
    auto load_a = [&](int q, int slot, bool last) {
        char* S = lds + slot * L::SA;
        if (last) A.load_last(q, S + A.blk(q, wave) * 1024, wave, lane, rem);
        else A.load(q, S + A.blk(q, wave) * 1024);
        if (q == C::QA - 1) A.advance();
    };
    auto load_b = [&](int q, int slot, bool last, int kt) {
        char* S = ldsb + slot * L::SB + B.blk(q, wave) * 1024;
        if constexpr (GATHER) {
            int r = idx[q][0];
            if constexpr (GS && GR == 2) r = lane >= 32 ? idx[q][1] : r;
            r = min(max(r, 0), (int)x_rows - 1);
            global_to_lds(B.base + (int64_t)r * B.ld + B.off[0], S);
            index(q, kt + 1);
        } else {
            if (last) B.load_last(q, S, wave, lane, rem);
            else B.load(q, S);
            if (q == C::QB - 1) B.advance();
        }
    };
    auto issue_a = [&](int slot, bool last) {
#pragma unroll
        for (int q = 0; q < C::QA; ++q) load_a(q, slot, last);
    };
    auto issue_b = [&](int slot, bool last, int kt) {
#pragma unroll
        for (int q = 0; q < C::QB; ++q) load_b(q, slot, last, kt);
    };
    // The scales of slices 8 c .. 8 c + 7 (past the end: the last again). They are issued ahead of a slice's
    // loads and not counted in the waits, which are the stricter for it.
    auto load_scales = [&](int c) {
        if constexpr (E::SCALED)
#pragma unroll
            for (int q = 0; q < C::QA; ++q)
                __builtin_amdgcn_global_load_lds((const PCM_GLOBAL void*)(rs->base + rs->off[q] + min(8 * c + (lane & 7), rs->kb - 1)),
                                                 (PCM_LDS void*)(lds + L::S0 + (c & 1) * L::SS + A.blk(q, wave) * 256), 4, 0, 0);
    };
    auto scales_of = [&](int kt) { return lds + L::S0 + ((kt >> 3) & 1) * L::SS + (kt & 7) * 4; };
    const bool part = rem < E::KB;   // the last slice is not whole
    auto is_last = [&](int kt) { return part && kt == KT - 1; };
    Step<E, C> f0, f1;
    load_scales(0);
    if (KT > 8) load_scales(1);
    issue_a(0, is_last(0));
    issue_b(0, is_last(0), 0);
#pragma unroll
    for (int s = 1; s < C::NSB; ++s) {
        if (s < C::NSA && s < KT) issue_a(s, is_last(s));
        if (s < KT) issue_b(s, is_last(s), s);
    }
    // slice 0 has landed: whatever was issued after it may be in flight
    constexpr int AFTER0 = (C::NSA - 1) * PER + (C::NSB - C::NSA) * PB;
    if (KT >= C::NSB) __builtin_amdgcn_s_waitcnt(waitcnt_imm(AFTER0 <= 62 ? AFTER0 : 62, 0));
    else __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
    tile_barrier();
    int sla = 0, slb = 0;
    auto up_a = [](int v) { return v + 1 == C::NSA ? 0 : v + 1; };
    auto up_b = [](int v) { return v + 1 == C::NSB ? 0 : v + 1; };
    auto read = [&](Step<E, C>& f, int s, int kt) {
#pragma unroll
        for (int j = 0; j < Step<E, C>::N; ++j) f.template read<A_KS, B_KS>(j, lds + sla * L::SA, ldsb + slb * L::SB, scales_of(kt), s, wm, wn, lane);
    };
    // The products of f, with the reads of g (half s of the slices in sla, slb) and, LOADS, the loads of
    // slices kt + NSA and kt + NSB into slots la and lb spread between them, in this order.
    auto half = [&](Step<E, C>& f, Step<E, C>& g, int s, auto loads, int la, int lb, int kt) {
        constexpr int M = C::MB * C::NBK, NR = Step<E, C>::N, NL = decltype(loads)::value ? C::QA + C::QB : 0;
        constexpr int R_EVERY = M > NR ? M / NR : 1, L_EVERY = M > NL && NL > 0 ? M / (NL > 0 ? NL : 1) : 1;
        int r = 0, l = 0;
#pragma unroll
        for (int i = 0; i < M; ++i) {
            bool any = false;
            const int rr = i % R_EVERY == 0 ? (M < NR ? (NR + M - 1) / M : 1) : 0;
            const int ll = i % L_EVERY == L_EVERY / 2 ? (M < NL ? (NL + M - 1) / M : 1) : 0;
#pragma unroll
            for (int j = 0; j < rr; ++j)
                if (r < NR) {
                    g.template read<A_KS, B_KS>(r++, lds + sla * L::SA, ldsb + slb * L::SB, nullptr, s, wm, wn, lane);
                    any = true;
                }
#pragma unroll
            for (int j = 0; j < ll; ++j)
                if (l < NL) {
                    if (l < C::QA) load_a(l, la, false);
                    else load_b(l - C::QA, lb, false, kt + C::NSB);
                    ++l;
                    any = true;
                }
            if constexpr (!E::SCALED) acc[i / C::MB][i % C::MB] = E::step(f.b[i / C::MB], f.a[i % C::MB], acc[i / C::MB][i % C::MB]);
            if (any) __builtin_amdgcn_sched_barrier(0);
        }
    };
    // One slice: its second half's fragments are read during the first half's products, then slice kt + 1
    // has landed (this wave's loads of it; the barrier covers the others') and every wave holds its last
    // fragments of slice kt, whose slots take slices kt + NSA and kt + NSB; the next slice's first fragments
    // are read during the second half's products. MORE: both those slices exist.
    auto slice = [&](int kt, auto more) {
        constexpr bool MORE = decltype(more)::value;
        if constexpr (!E::SCALED) half(f0, f1, 1, std::false_type{}, 0, 0, 0);
        __builtin_amdgcn_s_waitcnt(waitcnt_imm(MORE ? LATER : 0, 0));
        tile_barrier();
        const int la = sla, lb = slb;
        sla = up_a(sla);
        slb = up_b(slb);
        if (E::SCALED && kt % 8 == 0 && kt > 0 && kt + 8 < KT) load_scales(kt / 8 + 1);
        if constexpr (!MORE || E::SCALED) {
            if (kt + C::NSA < KT) issue_a(la, is_last(kt + C::NSA));
            if (kt + C::NSB < KT) issue_b(lb, is_last(kt + C::NSB), kt + C::NSB);
        }
        if constexpr (E::SCALED) {
            f0.multiply(acc, wsc[kt]);
            read(f0, 0, kt + 1);
        } else {
            half(f1, f0, 0, more, la, lb, kt);
        }
    };
    if constexpr (E::SCALED && C::MB % 4 == 0 && E::PAIRS) {
        // 8-bit MFMAs take 128 k each, so a slice is one step and its fragments are twice as large: B's stay
        // in registers for the slice, A's come two at a time, a pair ahead. The next slice has to have
        // landed before the last pair, in which every B fragment is replaced by the next slice's right
        // after its last use. Products are scaled and added while the next two run.
        using Frag = typename E::Frag;
        constexpr int NP = C::MB / 2, NL = C::QA + C::QB, NG = NP * C::NBK;
        static_assert(C::NBK >= 2, "the last two groups are of the last pair");
        floatx4 held[2][2] = {};
        float held_f[2] = {0.f, 0.f};
        const int r16 = lane & 15;
        const int at0 = r16 * 128 + ((kg ^ ((r16 >> 1) & 7)) * 16), at1 = r16 * 128 + (((4 + kg) ^ ((r16 >> 1) & 7)) * 16);
        Frag b[C::NBK], a[2][2];
        float sc[2][2];
        auto read_b = [&](int nb, int slot) {
            const char* p = ldsb + slot * L::SB + (wn * C::WTN + nb * 16) * 128;
            b[nb] = E::kc2(p + at0, p + at1);
        };
        auto read_a = [&](int mb, int slot, int kt) {
            const int r = wm * C::WTM + mb * 16;
            const char* p = lds + slot * L::SA;
            a[(mb / 2) & 1][mb & 1] = E::kc2(p + r * 128 + at0, p + r * 128 + at1);
            sc[(mb / 2) & 1][mb & 1] = *(const float*)(scales_of(kt) + (r + r16) * 32);
        };
        float ws = wsc[0];
        auto slice = [&](int kt, auto more, auto last) {
            constexpr bool MORE = decltype(more)::value, LAST = decltype(last)::value;
            const float ws_next = wsc[LAST ? kt : kt + 1];
            const int la = sla, lb = slb;
            floatx4 q[NG][2];     // products, scaled and added two groups later
            float f[2][2];
            auto add = [&](const floatx4& v, float g, int nb, int mb) {
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nb][mb][i] = fmaf(v[i], g, acc[nb][mb][i]);
            };
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const bool tail = p == NP - 1;
                f[p & 1][0] = sc[p & 1][0] * ws;
                f[p & 1][1] = sc[p & 1][1] * ws;
                if (tail && !LAST) {
                    __builtin_amdgcn_s_waitcnt(waitcnt_imm(MORE ? LATER : 0, 0));
                    tile_barrier();
                    sla = up_a(sla);
                    slb = up_b(slb);
                    if (kt % 8 == 0 && kt > 0 && kt + 8 < KT) load_scales(kt / 8 + 1);
                    if constexpr (!MORE) {
                        if (kt + C::NSA < KT) issue_a(la, is_last(kt + C::NSA));
                        if (kt + C::NSB < KT) issue_b(lb, is_last(kt + C::NSB), kt + C::NSB);
                    }
                }
#pragma unroll
                for (int nb = 0; nb < C::NBK; ++nb) {
                    const int G = p * C::NBK + nb;
                    if (!tail && nb < 2) {
                        read_a(2 * (p + 1) + nb, sla, kt);
                        if (LAST && part) a[(p + 1) & 1][nb] = E::head(a[(p + 1) & 1][nb], 0, kg, rem);
                    }
                    q[G][0] = E::product(b[nb], a[p & 1][0]);
                    q[G][1] = E::product(b[nb], a[p & 1][1]);
                    if (tail && !LAST) {
                        read_b(nb, slb);
                        if (nb < 2) read_a(nb, sla, kt + 1);
                        if constexpr (MORE)
#pragma unroll
                            for (int l = 0; l < NL; ++l) {
                                if (l * C::NBK / NL != nb) continue;
                                if (l < C::QA) load_a(l, la, false);
                                else load_b(l - C::QA, lb, false, 0);
                            }
                    }
                    if (G < 2) {   // the last two of the slice before
                        add(held[G][0], held_f[0], C::NBK - 2 + G, C::MB - 2);
                        add(held[G][1], held_f[1], C::NBK - 2 + G, C::MB - 1);
                    } else {
                        const int gp = (G - 2) / C::NBK, gn = (G - 2) % C::NBK;
                        add(q[G - 2][0], f[gp & 1][0], gn, 2 * gp);
                        add(q[G - 2][1], f[gp & 1][1], gn, 2 * gp + 1);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                held[i][0] = q[NG - 2 + i][0];
                held[i][1] = q[NG - 2 + i][1];
                held_f[i] = f[(NP - 1) & 1][i];
            }
            ws = ws_next;
        };
#pragma unroll
        for (int nb = 0; nb < C::NBK; ++nb) read_b(nb, 0);
        read_a(0, 0, 0);
        read_a(1, 0, 0);
        int kt = 0;
        for (; kt + C::NSB < KT - 1; ++kt) slice(kt, std::true_type{}, std::false_type{});
        for (; kt < KT - 1; ++kt) slice(kt, std::false_type{}, std::false_type{});
        if (part) {
#pragma unroll
            for (int nb = 0; nb < C::NBK; ++nb) b[nb] = E::head(b[nb], 0, kg, rem);
            a[0][0] = E::head(a[0][0], 0, kg, rem);
            a[0][1] = E::head(a[0][1], 0, kg, rem);
        }
        slice(kt, std::false_type{}, std::true_type{});
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    acc[C::NBK - 2 + i][C::MB - 2 + j][k] = fmaf(held[i][j][k], held_f[j], acc[C::NBK - 2 + i][C::MB - 2 + j][k]);
    } else {
        read(f0, 0, 0);
        int kt = 0;
        for (; kt + C::NSB < KT - 1; ++kt) slice(kt, std::true_type{});   // whole slices to come
        for (; kt < KT - 1; ++kt) slice(kt, std::false_type{});
        if constexpr (E::SCALED) {
            if (part) f0.head(0, kg, rem);
            f0.multiply(acc, wsc[KT - 1]);
        } else {
            read(f1, 1, 0);
            if (part) {
                f0.head(0, kg, rem);
                f1.head(1, kg, rem);
            }
            f0.multiply(acc, 1.0f);
            f1.multiply(acc, 1.0f);
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

// acc[nb][mb] holds C[row = .. + (lane & 15)][columns .. + 4 (lane >> 4) + 0..3] (columns: a multiple of
// 16, pointers 16-byte aligned). Each wave turns its block through LDS, so that a store covers whole rows of
// the block (128 bytes of bf16, 256 of float32 for 64 columns) instead of parts of 16 rows. LDS row r holds
// the 16-byte chunk c at c ^ (r % chunks).
template <class C, class OUT, bool ADD, int LDS_BYTES>
__device__ __forceinline__ void store_tile(OUT* out, int64_t row0, int rows, int col0, int cols, int wave, int lane,
                                           char* lds, const floatx4 (&acc)[C::NBK][C::MB]) {
    constexpr int WB = C::WTN * (int)sizeof(OUT), CH = WB / 16, RPI = 64 / CH;   // bytes and chunks of a row, rows a store
    constexpr int FIT = LDS_BYTES / C::NW / (16 * WB);
    constexpr int PM = FIT >= C::MB ? C::MB : FIT >= 4 ? 4 : FIT >= 2 ? 2 : 1;    // 16-row blocks a pass
    static_assert(FIT >= 1 && C::MB % PM == 0 && CH >= 1 && CH <= 64, "LDS");
    const int wm = wave / C::WN, wn = wave % C::WN;
    char* const wl = lds + wave * PM * 16 * WB;
    tile_barrier();   // every wave holds its last fragments
#pragma unroll
    for (int ps = 0; ps < C::MB / PM; ++ps) {
#pragma unroll
        for (int ml = 0; ml < PM; ++ml) {
            const int r = ml * 16 + (lane & 15);
#pragma unroll
            for (int nb = 0; nb < C::NBK; ++nb) {
                const int byte = (nb * 16 + (lane >> 4) * 4) * (int)sizeof(OUT);
                store4((OUT*)(wl + r * WB + (((byte / 16) ^ (r % CH)) * 16) + byte % 16), acc[nb][ps * PM + ml]);
            }
        }
#pragma unroll
        for (int i = 0; i < PM * 16 / RPI; ++i) {
            const int r = i * RPI + lane / CH, c = lane % CH;
            floatx4 v = *(const floatx4*)(wl + r * WB + ((c ^ (r % CH)) * 16));
            const int tr = wm * C::WTM + ps * PM * 16 + r, tc = col0 + wn * C::WTN + c * (16 / (int)sizeof(OUT));
            if (tr < rows && tc < cols) {
                floatx4* p = (floatx4*)(out + (row0 + tr) * cols + tc);
                if constexpr (ADD) v += *p;
                *p = v;
            }
        }
    }
}

// ------------------------------------------------------------------------ which tile
// Tile of this workgroup among ceil(rows / BM) x nt tiles of every group, expert-major: a group's tiles
// in blocks of max(1, window / row tiles) column tiles, the row tile varying slowest in a block; each XCD
// (workgroup id % 8) takes a contiguous eighth of the list. s_item: group, row0, row1, column tile, found, rows
// of the group.
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
                // a band of at most `window` row tiles, its column tiles in blocks of gn
                const int band = l / (window * nt), lb = l - band * window * nt;
                const int bm = min(window, mm_ - band * window);
                int gn = window / bm;
                gn = gn > nt ? nt : gn;
                const int gsize = gn * bm;
                const int grp = lb / gsize, in = lb - grp * gsize;
                const int gcols = min(gn, nt - grp * gn);
                const int mm = in / gcols;
                const int r0 = lo_ + (band * window + mm) * BM;
                s_item[0] = lane * 4 + hit;
                s_item[1] = r0;
                s_item[2] = min(lo_ + cnt_, r0 + BM);
                s_item[3] = grp * gn + (in - mm * gcols);
                s_item[5] = cnt_;
            }
        }
    }
    __syncthreads();
    return s_item[4] != 0;
}

// The same with each XCD's eighth of the row tiles of more than TBM rows before its eighth of the shorter ones,
// which then fill the last round instead of lengthening it: for products of few rounds (Mixtral-shaped down
// projection, 576 tiles: 954 -> 847 us; with more rounds, or a row tile or two a group, the order above shares
// operands better: 256 rows each in 64 groups 176 -> 212 us). Both sides of launch_rows' bounds (a contraction of 4096,
// 8 to 32 groups, us, this order / the one above): a mean of 256 rows, 384 tiles 207-210 / 206-207, 768 tiles 348-358 /
// 332-340; of 400, 528 tiles 228-238 / 219-222; of 512, 320 tiles 156-171 / 177-199, 640 tiles 286-299 / 290-305, 1280
// tiles 550-585 / 522-550; of 700, 400 to 1650 tiles within 2% of each other; of 1000, 560 tiles 245-266 / 269-299. (Past
// the bound of 1024 tiles a mean of 1000 and more would still gain: 1120 tiles 457-468 / 469-489.)
template <int BM, int TBM>
__device__ bool group_item_long_first(const GroupArgs& g, int nt, int window, int* s_item) {
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        int lo[4], cnt[4], m[4], tail[4], nl = 0, ns = 0;   // m: long row tiles, tail: 0 or 1 short one
        group_bounds(g.offsets, g.n, g.R, lane, lo, cnt);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            clamp_group((int)g.R, lo[j], cnt[j]);
            const int rem = cnt[j] % BM;
            m[j] = cnt[j] / BM + (rem > TBM ? 1 : 0);
            tail[j] = rem > 0 && rem <= TBM ? 1 : 0;
            nl += m[j] * nt;
            ns += tail[j] * nt;
        }
        const int incl = wave_incl_scan_i32(nl), incs = wave_incl_scan_i32(ns);
        const int total = __builtin_amdgcn_readlane(incl, 63), totals = __builtin_amdgcn_readlane(incs, 63);
        const int x8 = (int)(blockIdx.x % 8), j8 = (int)(blockIdx.x / 8);
        const int l0 = (int)((int64_t)x8 * total / 8), l1 = (int)((int64_t)(x8 + 1) * total / 8);
        const int s0 = (int)((int64_t)x8 * totals / 8), s1 = (int)((int64_t)(x8 + 1) * totals / 8);
        const bool is_long = j8 < l1 - l0, valid = is_long || j8 - (l1 - l0) < s1 - s0;
        if (lane == 0) s_item[4] = valid ? 1 : 0;
        if (valid) {
            const int id = is_long ? l0 + j8 : s0 + j8 - (l1 - l0);
            int start = is_long ? incl - nl : incs - ns;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int mm = is_long ? m[j] : tail[j];
                if (id >= start && id < start + mm * nt) {
                    const int l = id - start;
                    const int band = l / (window * nt), lb = l - band * window * nt;
                    const int bm = min(window, mm - band * window);
                    int gn = window / bm;
                    gn = gn > nt ? nt : gn;
                    const int gsize = gn * bm, grp = lb / gsize, in = lb - grp * gsize;
                    const int gcols = min(gn, nt - grp * gn), row = in / gcols;
                    const int r0 = lo[j] + (is_long ? band * window + row : cnt[j] / BM) * BM;
                    s_item[0] = lane * 4 + j;
                    s_item[1] = r0;
                    s_item[2] = min(lo[j] + cnt[j], r0 + BM);
                    s_item[3] = grp * gn + (in - row * gcols);
                }
                start += mm * nt;
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

// Row tiles of BM rows to expect: whole tiles and, for each group with rows, half a tile.
inline int64_t expected_row_tiles(const GroupArgs& g, int64_t BM) {
    if (g.n == 1) return ceil_div(g.R, BM);
    return g.R / BM + ((g.R < g.n ? g.R : g.n) + 1) / 2;
}
inline int64_t mean_rows(const GroupArgs& g) {
    const int64_t groups = g.offsets ? (g.R < g.n ? g.R : g.n) : 1;
    return ceil_div(g.R, groups);
}
// Whether a mean of few rows a group makes the per-wave rings faster than 64 x 64 tiles and more: enough slices of
// 128 bytes of the contraction for the rings to run (64 groups, 4096 columns: bf16 54 against 56 us at 8
// slices, 38 against 31 at 4; 8 bits, mean of 8 rows: 110 against 108 us at 16, 78 against 64 at 8; a mean of 16 rows
// needs twice as many, the second row tile of some groups reading the weights again). The bound of the mean, 16, and 14
// where 8-bit values make results in bf16, whose tiles are the faster ones: random counts, 2048 columns, a contraction
// of 7168, rings / tiles, us: 256 groups, 8 bits into bf16, mean of 12 622 / 666, 14 679 / 677, 16 755 / 677; into
// float32 14 695 / 747, 16 759 / 751; bf16 12 1097 / 1220, 16 1210 / 1223; 64 groups, 8 bits into bf16 12 166 / 171, 16
// 198 / 172, into float32 14 190 / 187, 16 204 / 188, bf16 14 302 / 311, 16 314 / 311. (A contraction of 4096 in 64
// groups is the one found where bf16 results of a mean of 16 would keep the rings: 120 / 131; 256 groups 450 / 399.)
// The counts are the device's, the host has their mean only: where nine tenths of the rows lie in one group, rings take
// up to 1.4 times the tiles' time (256 groups of 2048 x 2048, bf16, mean of 16 453 / 349, of 8 298 / 253).
inline bool few_rows(const GroupArgs& g, int64_t size, int most = 16) {
    const int64_t mean = mean_rows(g);
    return mean <= most && ceil_div(g.len * size, 128) >= (size == 1 ? 2 : 1) * (mean > 8 ? 16 : 8);
}
// Whether the weights are worth reading non-temporally by groups of one row tile, which read them once:
// together they are more than half of the 256 MB MALL.
inline bool weights_once(const GroupArgs& g, int64_t size) {
    return (g.offsets ? (g.R < g.n ? g.R : g.n) : 1) * size * g.len * g.cols >= ((int64_t)128 << 20);
}
// Whether 32-bit offsets reach every row of a tile (a gather's from the start of x).
inline bool near(const GroupArgs& g, int64_t size) {
    const int64_t far = (int64_t)1 << 31, row = g.len * size, col = g.cols * size, out = g.rows * size;
    return 256 * row < far && 64 * col < far && 64 * out < far && !(g.gather && g.len > 0 && g.x_rows * row >= far);
}

// ------------------------------------------------------------------------ kernels
// A tile of out[r, :] = x[s(r), :] . b[e]^T (DX false: b [n, cols, len]) or dy[r, :] . b[e] (DX true: b [n,
// len, cols]): rows row0 .. row1 - 1 of group e, column tile ntile.
template <class E, class C, bool DX, class OUT, class OFF, int LDS_BYTES>
__device__ __forceinline__ void rows_tile(const GroupArgs& g, char* lds, int e, int row0, int row1, int ntile) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t lenb = (int64_t)g.len * E::SIZE, colb = (int64_t)g.cols * E::SIZE;
    auto source = [&](int r) -> int64_t {   // rows past row1 repeat the last (never stored)
        r = min(r, row1 - 1);
        if (!g.gather) return r;
        const int64_t t = g.gather[r];
        return t < 0 ? 0 : t >= g.x_rows ? g.x_rows - 1 : t;
    };
    Side<E, C, C::BM, C::QA, false, OFF> A;
    Side<E, C, C::BN, C::QB, DX, OFF> B;
    const int64_t first = g.gather ? 0 : row0;
    int64_t src[C::QA];   // every row index is loaded before any is used
#pragma unroll
    for (int q = 0; q < C::QA; ++q) src[q] = source(row0 + A.row(q, wave, lane)) - first;
#pragma unroll
    for (int q = 0; q < C::QA; ++q) A.off[q] = (OFF)(src[q] * lenb + A.chunk(q, wave, lane));
    A.base = (const char*)g.a + first * lenb;
    A.ld = 0;
    const char* bg = (const char*)g.b + (int64_t)e * g.len * colb;
    const int col0 = ntile * C::BN;
    if constexpr (DX) {   // columns past the end repeat the last 16 bytes (never stored)
        B.base = bg;
        B.off[0] = (OFF)(B.row(0, wave, lane) * colb + min((int64_t)col0 * E::SIZE + B.column(wave, lane), colb - 16));
    } else {
        B.base = bg + col0 * lenb;
#pragma unroll
        for (int q = 0; q < C::QB; ++q)
            B.off[q] = (OFF)(min(B.row(q, wave, lane), g.cols - 1 - col0) * lenb + B.chunk(q, wave, lane));
    }
    B.ld = colb;
    RowScales<C> rs;
    ScalarPtr wsc = nullptr;
    if constexpr (E::SCALED) {
        const int kb = (g.len + 127) / 128, nb = (g.cols + 127) / 128;
        rs.base = g.a_scale + first * kb;
        rs.kb = kb;
#pragma unroll
        for (int q = 0; q < C::QA; ++q) rs.off[q] = src[q] * kb;
        wsc = (ScalarPtr)(g.b_scale + ((int64_t)e * nb + min((col0 + wave % C::WN * C::WTN) / 128, nb - 1)) * kb);
    }
    floatx4 acc[C::NBK][C::MB];
#pragma unroll
    for (int i = 0; i < C::NBK; ++i)
#pragma unroll
        for (int j = 0; j < C::MB; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    tile_loop<E, C, false, DX, false, OFF>(A, B, g.len, lds, acc, nullptr, 0, &rs, wsc);
    store_tile<C, OUT, false, LDS_BYTES>((OUT*)g.out, row0, row1 - row0, col0, g.cols, wave, lane, lds, acc);
}

// A row tile of at most CT::BM rows runs as the smaller tile CT (the same columns and waves; CT = C: none).
template <class E, class C, class CT, bool DX, class OUT, class OFF>
__global__ __launch_bounds__(C::NT) void group_rows_kernel(GroupArgs g, int nt, int window, bool long_first) {
    static_assert(CT::NT == C::NT && CT::BN == C::BN && CT::BM <= C::BM, "tail tile");
    constexpr int BYTES = Slots<E, C>::BYTES;
    static_assert(Slots<E, CT>::BYTES <= BYTES, "tail tile");
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    int* const s_item = (int*)lds;   // read into registers before the first loads overwrite it
    if (CT::BM < C::BM && long_first) {   // workgroup-uniform branches and returns
        if (!group_item_long_first<C::BM, CT::BM>(g, nt, window, s_item)) return;
    } else if (!group_item<C::BM>(g, nt, window, s_item)) {
        return;
    }
    const int e = __builtin_amdgcn_readfirstlane(s_item[0]), row0 = __builtin_amdgcn_readfirstlane(s_item[1]);
    const int row1 = __builtin_amdgcn_readfirstlane(s_item[2]), ntile = __builtin_amdgcn_readfirstlane(s_item[3]);
    __syncthreads();
    if (CT::BM < C::BM && row1 - row0 <= CT::BM) rows_tile<E, CT, DX, OUT, OFF, BYTES>(g, lds, e, row0, row1, ntile);
    else rows_tile<E, C, DX, OUT, OFF, BYTES>(g, lds, e, row0, row1, ntile);
}

// out[e] [rows, cols] = sum over the rows r of group e of a[r, :]^T b[s(r), :]. gridDim.y > 1: the rows in that
// many parts, each with sums of its own, out [parts, n, rows, cols].
template <class E, class C, bool GATHER, class OUT, bool ADD, class OFF>
__global__ __launch_bounds__(C::NT) void group_outer_kernel(GroupArgs g, int mt, int nt, int cm, int cn) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Chunks of cm x cn tiles (about as many as an XCD's 32 compute units run at once, so that they share
    // operand tiles), dealt to the XCDs (workgroup id % 8) in turn, so that a group with many rows does not
    // keep one of them busy alone (64 groups of very different size 1051 -> 852 us, now 720; contiguous eighths of the
    // tiles are 0-3% faster where all groups are alike; the groups sorted by rows first gave 769 us there
    // and cost 5-10% elsewhere, a search in front of every tile).
    const int slots = cm * cn, mc = (mt + cm - 1) / cm, nc = (nt + cn - 1) / cn;
    const int j8 = (int)(blockIdx.x / 8), x8 = (int)((blockIdx.x + blockIdx.y) % 8);
    const int chunk = j8 / slots * 8 + x8, slot = j8 % slots;
    const int e = chunk / (mc * nc), in = chunk - e * (mc * nc);
    const int mtile = in % mc * cm + slot % cm, ntile = in / mc * cn + slot / cm;
    if (e >= g.n || mtile >= mt || ntile >= nt) return;   // workgroup-uniform
    int lo = 0, cnt = (int)g.R;
    if (g.offsets) {
        lo = g.offsets[e];
        cnt = g.offsets[e + 1] - lo;
        clamp_group((int)g.R, lo, cnt);
    }
    int64_t out = (int64_t)e * g.rows * g.cols;
    if (gridDim.y > 1) {   // this part of the group's rows, whole slices, into its own sums
        const int part = ((cnt + E::KB - 1) / E::KB + (int)gridDim.y - 1) / (int)gridDim.y * E::KB;
        const int skip = min((int)blockIdx.y * part, cnt);
        lo += skip;
        cnt = min(part, cnt - skip);
        out += (int64_t)blockIdx.y * g.n * g.rows * g.cols;
    }
    if (ADD && cnt == 0) return;
    const int64_t ab = (int64_t)g.rows * E::SIZE, bb = (int64_t)g.cols * E::SIZE;
    Side<E, C, C::BM, C::QA, true, OFF> A;
    Side<E, C, C::BN, C::QB, true, OFF> B;
    A.base = (const char*)g.a + lo * ab;
    A.off[0] = (OFF)(A.row(0, wave, lane) * ab + min((int64_t)mtile * C::BM * E::SIZE + A.column(wave, lane), ab - 16));
    A.ld = ab;
    const int64_t bcol = min((int64_t)ntile * C::BN * E::SIZE + B.column(wave, lane), bb - 16);
    B.base = (const char*)g.b + (GATHER ? 0 : lo * bb);
    B.off[0] = (OFF)((GATHER ? 0 : B.row(0, wave, lane) * bb) + bcol);
    B.ld = bb;
    floatx4 acc[C::NBK][C::MB];
#pragma unroll
    for (int i = 0; i < C::NBK; ++i)
#pragma unroll
        for (int j = 0; j < C::MB; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (cnt > 0)
        tile_loop<E, C, true, true, GATHER, OFF>(A, B, cnt, lds, acc, GATHER ? g.gather + lo : nullptr, g.x_rows, nullptr, nullptr);
    store_tile<C, OUT, ADD, Slots<E, C>::BYTES>((OUT*)g.out + out, mtile * C::BM,
                                                g.rows - mtile * C::BM, ntile * C::BN, g.cols, wave, lane, lds, acc);
}

// Few rows a group: the weights are what there is to read, so a compute unit has to keep many of their
// bytes in flight. A workgroup takes 16 rows and 64 columns, and each of its four waves its own
// slices of the contraction (every fourth) through a ring of its own, with no barrier until the waves' sums
// are added, in order, at the end.
template <class E>
struct ThinCfg {
    static constexpr int BM = 16, NW = 4, NS = 2;   // rows, waves, slices of a ring
    using C = TileCfg<BM, 64, 1, 1, 2>;   // the layout of one wave
    static constexpr int SLOT = (BM + 64) * 128 + (E::SCALED ? 256 : 0), WAVE = NS * SLOT;
    static constexpr int BYTES = NW * WAVE, PER = C::QA + C::QB + (E::SCALED ? 1 : 0);
    static_assert(NW == C::NBK, "each wave adds one block of columns");
    static_assert(BYTES <= 160 * 1024 && (NS - 1) * PER <= 62 && BM * 256 <= WAVE, "LDS, vmcnt range, sums");
};
template <class E, class OUT>
__global__ __launch_bounds__(ThinCfg<E>::NW * 64) void group_thin_kernel(GroupArgs g, int nt, int window, bool once) {
    using T = ThinCfg<E>;
    using C = typename T::C;
    constexpr int BM = T::BM, NW = T::NW, NS = T::NS;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    int* const s_item = (int*)lds;
    if (!group_item<BM>(g, nt, window, s_item)) return;   // workgroup-uniform
    const int e = __builtin_amdgcn_readfirstlane(s_item[0]), row0 = __builtin_amdgcn_readfirstlane(s_item[1]);
    const int row1 = __builtin_amdgcn_readfirstlane(s_item[2]), ntile = __builtin_amdgcn_readfirstlane(s_item[3]);
    const bool alone = once && __builtin_amdgcn_readfirstlane(s_item[5]) <= BM;   // weights read once: non-temporal
    __syncthreads();
    const int lane = threadIdx.x & 63, r16 = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char* const ring = lds + wave * T::WAVE;
    const int64_t lenb = (int64_t)g.len * E::SIZE;
    const int col0 = ntile * 64, KT = (g.len + E::KB - 1) / E::KB, rem = g.len - (KT - 1) * E::KB;
    const int mine = KT > wave ? (KT - wave + NW - 1) / NW : 0;   // this wave's slices: wave + i NW
    auto source = [&](int r) -> int64_t {   // rows past row1 repeat the last (never stored)
        r = min(r, row1 - 1);
        if (!g.gather) return r;
        const int64_t t = g.gather[r];
        return t < 0 ? 0 : t >= g.x_rows ? g.x_rows - 1 : t;
    };
    const int64_t first = g.gather ? 0 : row0;
    Side<E, C, C::BM, C::QA, false, uint32_t> A;
    Side<E, C, C::BN, C::QB, false, uint32_t> B;
    int64_t src[C::QA];
#pragma unroll
    for (int q = 0; q < C::QA; ++q) src[q] = source(row0 + A.row(q, 0, lane)) - first;
    const int64_t scale_row = E::SCALED ? source(row0 + lane % BM) : 0;
#pragma unroll
    for (int q = 0; q < C::QA; ++q) A.off[q] = (uint32_t)(src[q] * lenb + A.chunk(q, 0, lane));
    A.base = (const char*)g.a + first * lenb + wave * 128;
#pragma unroll
    for (int q = 0; q < C::QB; ++q)
        B.off[q] = (uint32_t)(min(B.row(q, 0, lane), g.cols - 1 - col0) * lenb + B.chunk(q, 0, lane));
    B.base = (const char*)g.b + ((int64_t)e * g.cols + col0) * lenb + wave * 128;
    A.ld = B.ld = 0;
    const int kb = (g.len + 127) / 128, nb128 = (g.cols + 127) / 128;
    const float* xs = E::SCALED ? g.a_scale + scale_row * kb + wave : nullptr;
    const ScalarPtr ws = E::SCALED ? (ScalarPtr)(g.b_scale + ((int64_t)e * nb128 + col0 / 128) * kb + wave) : nullptr;
    auto issue = [&](int i, int slot) {
        char* S = ring + slot * T::SLOT;
        if (rem < E::KB && wave + i * NW == KT - 1) {   // the slice that is not whole
#pragma unroll
            for (int q = 0; q < C::QB; ++q) B.load_last(q, S + BM * 128 + q * 1024, 0, lane, rem);
#pragma unroll
            for (int q = 0; q < C::QA; ++q) A.load_last(q, S + q * 1024, 0, lane, rem);
        } else {
            if (alone)
#pragma unroll
                for (int q = 0; q < C::QB; ++q) B.template load<true>(q, S + BM * 128 + q * 1024);
            else
#pragma unroll
                for (int q = 0; q < C::QB; ++q) B.load(q, S + BM * 128 + q * 1024);
#pragma unroll
            for (int q = 0; q < C::QA; ++q) A.load(q, S + q * 1024);
        }
        if constexpr (E::SCALED) {
            __builtin_amdgcn_global_load_lds((const PCM_GLOBAL void*)xs, (PCM_LDS void*)(S + (BM + 64) * 128), 4, 0, 0);
            xs += NW;
        }
        A.advance(NW);
        B.advance(NW);
    };
    floatx4 acc[C::NBK][C::MB];
#pragma unroll
    for (int i = 0; i < C::NBK; ++i)
#pragma unroll
        for (int j = 0; j < C::MB; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    // 8-bit operands: one step of both halves a slice
    Step<E, C> f0, f1;
    auto finish = [&](int i, int slot, bool more) {   // slice i has landed
        const char* S = ring + slot * T::SLOT;
        const char* SC = S + (BM + 64) * 128;
#pragma unroll
        for (int j = 0; j < Step<E, C>::N; ++j) f0.template read<false, false, 4>(j, S, S + BM * 128, SC, 0, 0, 0, lane);
        if constexpr (!E::SCALED) {
#pragma unroll
            for (int j = 0; j < Step<E, C>::N; ++j) f1.template read<false, false>(j, S, S + BM * 128, SC, 1, 0, 0, lane);
        }
        float w = 1.0f;
        if constexpr (E::SCALED) w = ws[i * NW];
        __builtin_amdgcn_s_waitcnt(waitcnt_imm(kNoVm, 0));   // the fragments are held: the slot is free
        __builtin_amdgcn_sched_barrier(0);
        if (more) issue(i + NS, slot);
        if (rem < E::KB && wave + i * NW == KT - 1) {
            f0.head(0, kg, rem);
            if constexpr (!E::SCALED) f1.head(1, kg, rem);
        }
        f0.multiply(acc, w);
        if constexpr (!E::SCALED) f1.multiply(acc, w);
    };
#pragma unroll
    for (int s = 0; s < NS; ++s)
        if (s < mine) issue(s, s);
    int slot = 0, i = 0;
    for (; i + NS <= mine; ++i) {
        __builtin_amdgcn_s_waitcnt(waitcnt_imm((NS - 1) * T::PER, kNoLgkm));
        asm volatile("" ::: "memory");
        finish(i, slot, i + NS < mine);
        slot = slot + 1 == NS ? 0 : slot + 1;
    }
    if (i < mine) {
        __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, kNoLgkm));
        asm volatile("" ::: "memory");
        for (; i < mine; ++i) {
            finish(i, slot, false);
            slot = slot + 1 == NS ? 0 : slot + 1;
        }
    }
    // every wave's sums, then wave w adds column block w of all of them, in order
    tile_barrier();
#pragma unroll
    for (int nb = 0; nb < C::NBK; ++nb)
#pragma unroll
        for (int mb = 0; mb < C::MB; ++mb)
            *(floatx4*)(lds + ((wave * C::NBK + nb) * C::MB + mb) * 1024 + lane * 16) = acc[nb][mb];
    __syncthreads();
    const int c = col0 + wave * 16 + kg * 4;
#pragma unroll
    for (int mb = 0; mb < C::MB; ++mb) {
        floatx4 sum = *(const floatx4*)(lds + (wave * C::MB + mb) * 1024 + lane * 16);
#pragma unroll
        for (int w = 1; w < NW; ++w) sum += *(const floatx4*)(lds + ((w * C::NBK + wave) * C::MB + mb) * 1024 + lane * 16);
        const int r = row0 + mb * 16 + r16;
        if (r < row1 && c < g.cols) store4((OUT*)g.out + (int64_t)r * g.cols + c, sum);
    }
}

template <class K>
hipError_t allow_lds(K kernel, int bytes) {   // set on every launch (idempotent; the library keeps no state)
    return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <class E, class C, class CT, bool DX, class OUT, class OFF = uint32_t>
hipError_t launch_rows(const GroupArgs& g, int window, hipStream_t s) {
    const int nt = (int)ceil_div(g.cols, C::BN);
    // (groups of few row tiles read their weights once for all of them in the other order)
    const bool long_first = CT::BM < C::BM && g.offsets && mean_rows(g) >= 512 && expected_row_tiles(g, C::BM) * nt < 4 * 256;
    // An eighth of the long tiles and one of the short ones, each rounded up, can be one more than an eighth of both.
    const int64_t grid = ceil_div(most_row_tiles(g, C::BM) * nt, 8) * 8 + (long_first ? 8 : 0);
    if (grid >= int64_t(1) << 28) return hipErrorInvalidValue;   // counted in 32 bits
    const auto kernel = group_rows_kernel<E, C, CT, DX, OUT, OFF>;
    const hipError_t err = allow_lds(kernel, Slots<E, C>::BYTES);
    if (err != hipSuccess) return err;
    kernel<<<dim3((unsigned)grid), dim3(C::NT), Slots<E, C>::BYTES, s>>>(g, nt, window, long_first);
    return hipGetLastError();
}

template <class E, class OUT>
hipError_t launch_thin(const GroupArgs& g, int window, bool once, hipStream_t s) {
    using T = ThinCfg<E>;
    const int nt = (int)ceil_div(g.cols, 64);
    const int64_t grid = ceil_div(most_row_tiles(g, T::BM) * nt, 8) * 8;
    if (grid >= int64_t(1) << 28) return hipErrorInvalidValue;
    const auto kernel = group_thin_kernel<E, OUT>;
    const hipError_t err = allow_lds(kernel, T::BYTES);
    if (err != hipSuccess) return err;
    kernel<<<dim3((unsigned)grid), dim3(T::NW * 64), T::BYTES, s>>>(g, nt, window, once);
    return hipGetLastError();
}

template <class E, class C, bool GATHER, class OUT, bool ADD, class OFF>
hipError_t launch_outer_(const GroupArgs& g, int parts, hipStream_t s) {
    const int mt = (int)ceil_div(g.rows, C::BM), nt = (int)ceil_div(g.cols, C::BN);
    // chunks of up to 32 tiles, fewer where that would make less than 64 of them
    const int64_t some = (int64_t)g.n * mt * nt / 64, most = some < 1 ? 1 : some > 32 ? 32 : some;
    int cm = 1;   // rows by columns about two to one
    while (cm < mt && 4 * cm * cm <= 2 * most) cm *= 2;
    cm = cm < mt ? cm : mt;
    const int across = (int)ceil_div((int64_t)nt * cm, most), cn = (int)ceil_div(nt, across);
    const int64_t chunks = g.n * ceil_div(mt, cm) * ceil_div(nt, cn), grid = ceil_div(chunks, 8) * 8 * cm * cn;
    if (grid >= int64_t(1) << 28) return hipErrorInvalidValue;
    const auto kernel = group_outer_kernel<E, C, GATHER, OUT, ADD, OFF>;
    const hipError_t err = allow_lds(kernel, Slots<E, C>::BYTES);
    if (err != hipSuccess) return err;
    kernel<<<dim3((unsigned)grid, (unsigned)parts), dim3(C::NT), Slots<E, C>::BYTES, s>>>(g, mt, nt, cm, cn);
    return hipGetLastError();
}
template <class E, class C, class OUT, bool ADD, class OFF = uint32_t>
hipError_t launch_outer(const GroupArgs& g, hipStream_t s, int parts = 1) {
    return g.gather ? launch_outer_<E, C, true, OUT, ADD, OFF>(g, parts, s) : launch_outer_<E, C, false, OUT, ADD, OFF>(g, parts, s);
}

}  // namespace
}  // namespace pcm
