// Products grouped by expert with ragged row counts, and their gradients (bf16 and float32 operands,
// float32 sums):
//   forward          y[r, :]  = x[s(r), :] W[e]^T          W [n, N, K], rows r of group e
//   input gradient   dx[r, :] = dy[r, :] W[e]              (then summed over the rows of a token)
//   weight gradient  dW[e]    = sum_r dy[r, :]^T x[s(r), :]
// Large ones are bound by the matrix cores and the loads that feed them (8192^3 bf16: 1470 TF forward, 1444 and
// 1450 for the gradients), few rows in many groups by reading every weight once (256 groups of 7168 x
// 2048, one row each: 676 us, 7.0 TB/s), a large gradient of few rows by writing it. A token's gradient adds the
// rows of its groups in slot order in a second launch (slot_sum_kernel: the rows in float32, written and read
// once; 32768 rows of 2048 take 52 us there, 5.8 TB/s), not with atomics, whose order would change results.
#include "grouped.h"

namespace pcm {
namespace {

using Small = TileCfg<64, 64, 2, 2, 3>;          // three workgroups on a compute unit
using Narrow = TileCfg<32, 64, 2, 2, 4>;         // three
using Middle = TileCfg<64, 128, 2, 2, 3>;        // two
using Square = TileCfg<128, 128, 2, 2, 2, 3>;    // two
using Large = TileCfg<256, 256, 2, 4, 2, 3>;     // one, eight waves of 128 x 64
using LargeTail = TileCfg<128, 256, 2, 4, 2, 3>;

// The larger the tile the fewer bytes a product loads (a compute unit takes in about 50 GB/s from its L2 and
// beyond: 64 x 64 tiles stop at 700 TF, 64 x 128 at 890, 128 x 128 at 1110, 256 x 256 at 1480), but each
// fills the 256 compute units from a number of tiles on. Measured on both sides of every bound, one group, a
// contraction of 4096, bf16 (us, this tile / the next smaller):
//   256 x 256  224 tiles 94 / 117, 128 tiles 78 / 64
//   128 x 128  224 tiles 38.2 / 39.0 (input gradient 38.4 / 41.5), 128 tiles 34.0 / 24.6
//   64 x 128   256 tiles 24.6 / 27.4, 128 tiles 33 / 19.1
//   64 x 64    192 tiles 18.5 / 20.6 (32 x 64), 128 tiles 18.2 / 13.9
//   16 rows    of 64 columns, per-wave rings: 256 tiles 10.5, 64 x 64 18.1; 384 tiles 16.0, 32 x 64 13.8
// float32: 64 x 64 / 32 x 64, 1024 columns, a contraction of 1024. Each step of a few hundred tiles is a round of
// workgroups, in which now the one and now the other is ahead; the bounds are where neither is by much on both sides:
//   one group         384 tiles 38.6 / 31.5, 448 38.4 / 41.3, 512 38.8 / 41.2, 640 53.6 / 49.0, 768 54.4 / 57.6, 2048 135 / 145
//   8 and 16 groups   368 tiles 38.1 / 30.6, 496 38.5 / 41.0, 560-624 53.4 / 48.3, 752 54.2 / 56.9, 1008 71.5 / 74.4, 2032 135 / 145
//   64 groups (row tiles that are not full)   752 tiles 82 / 64, 1008 82 / 72, 1264 84 / 90, 1520 123 / 106, 2032 147 / 135
// 64 x 64 reaches 128 TF in 2048 tiles. 128 x 128 would bring 4% to one large group (8192 x 4096 x 4096 1964 / 2043) and
// cost 13% in 8 groups of 1024 rows (624 / 552), 64 x 128 1% and 5%; the input gradient's layout has no such tiles.
template <class E, bool DX, class OUT>
hipError_t rows_by_shape(const GroupArgs& g, hipStream_t s) {
    if (!near(g, E::SIZE)) return launch_rows<E, Small, Small, DX, OUT, int64_t>(g, 8, s);
    auto tiles = [&](int bm, int bn) { return expected_row_tiles(g, bm) * ceil_div(g.cols, bn); };
    if constexpr (E::SIZE == 4) {
        if (tiles(64, 64) < (g.n == 1 ? 512 : 1024)) return launch_rows<E, Narrow, Narrow, DX, OUT>(g, 8, s);
        return launch_rows<E, Small, Small, DX, OUT>(g, 8, s);
    } else {
        if constexpr (!DX)
            if (few_rows(g, E::SIZE) || tiles(16, 64) <= 256)
                return launch_thin<E, OUT>(g, 8, weights_once(g, E::SIZE), s);
        if (tiles(64, 64) <= 128) return launch_rows<E, Narrow, Narrow, DX, OUT>(g, 8, s);
        if (tiles(256, 256) >= 192) return launch_rows<E, Large, LargeTail, DX, OUT>(g, 8, s);
        if (tiles(128, 128) >= 192) return launch_rows<E, Square, Square, DX, OUT>(g, 8, s);
        if (tiles(64, 128) >= 256) return launch_rows<E, Middle, Middle, DX, OUT>(g, 8, s);
        return launch_rows<E, Small, Small, DX, OUT>(g, 8, s);
    }
}

template <bool DX>
hipError_t rows_by_type(bool bf16, bool out_bf16, const GroupArgs& g, hipStream_t s) {
    if (!bf16) return rows_by_shape<TF32, DX, float>(g, s);
    return out_bf16 ? rows_by_shape<TBf16, DX, __bf16>(g, s) : rows_by_shape<TBf16, DX, float>(g, s);
}

// The same for the weight gradient (4096 rows, one group, bf16, us, this tile / the next smaller):
//   256 x 256  224 tiles 98 / 119, 128 tiles 80 / 66
//              (64 groups of 2048 x 2048 with 8 rows each, bound by writing them, 132 / 163; with 1024, 651 / 853)
//   128 x 128  224 tiles 38.7 / 55.4, 128 tiles 33.7 / 30.0, 64 tiles 26.9 / 19.9
template <class E, class OUT, bool ADD>
hipError_t outer_by_shape(const GroupArgs& g, hipStream_t s) {
    if (!near(g, E::SIZE)) return launch_outer<E, Small, OUT, ADD, int64_t>(g, s);
    auto tiles = [&](int bm, int bn) { return g.n * ceil_div(g.rows, bm) * ceil_div(g.cols, bn); };
    if constexpr (E::SIZE == 2) {
        if (tiles(256, 256) >= 192) return launch_outer<E, Large, OUT, ADD>(g, s);
        if (tiles(128, 128) >= 160) return launch_outer<E, Square, OUT, ADD>(g, s);
    }
    return launch_outer<E, Small, OUT, ADD>(g, s);
}

// out = [out +] the parts' sums, in order.
template <class OUT>
__global__ __launch_bounds__(256) void part_sum_kernel(const float* __restrict__ parts, int count, int64_t size,
                                                       OUT* __restrict__ out, int add) {
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size; i += (int64_t)gridDim.x * 1024) {
        floatx4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < count; p += 8) {   // eight loads in flight; past the end the last again, not added
            floatx4 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = *(const floatx4*)(parts + min(p + j, count - 1) * size + i);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (p + j < count) sum += v[j];
        }
        if constexpr (sizeof(OUT) == 4)
            if (add) sum += *(const floatx4*)(out + i);
        store4(out + i, sum);
    }
}

// A thread adds four columns of a token's rows, slots ascending, in float32. Rows of no group are not added: the
// product has not written them. Bound by reading the rows: all indices, then all rows, are loaded before any is
// used.
template <class OUT>
__global__ __launch_bounds__(256) void slot_sum_kernel(const float* __restrict__ rows, const int32_t* __restrict__ row_of,
                                                       const int32_t* __restrict__ offsets, int n, int64_t T, int k,
                                                       int64_t R, int K, OUT* __restrict__ out) {
    int first = 0, count = (int)R;   // the groups' rows
    if (offsets) {
        first = offsets[0];
        count = offsets[n] - first;
        clamp_group((int)R, first, count);
    }
    const int64_t per = K / 4, total = T * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / per, c = (i - t * per) * 4;
        int r[kMaxK];
        floatx4 v[kMaxK];
#pragma unroll
        for (int a = 0; a < kMaxK; ++a) r[a] = a < k ? row_of[t * k + a] : -1;
#pragma unroll
        for (int a = 0; a < kMaxK; ++a)
            if ((uint32_t)r[a] - (uint32_t)first < (uint32_t)count) v[a] = *(const floatx4*)(rows + (int64_t)r[a] * K + c);
        floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int a = 0; a < kMaxK; ++a)
            if ((uint32_t)r[a] - (uint32_t)first < (uint32_t)count) sum += v[a];
        store4(out + t * K + c, sum);
    }
}

}  // namespace

hipError_t launch_grouped(bool bf16, bool out_bf16, const GroupArgs& g, hipStream_t s) {
    return rows_by_type<false>(bf16, out_bf16, g, s);
}

hipError_t launch_grouped_dx(bool bf16, bool out_bf16, const GroupArgs& g, hipStream_t s) {
    return rows_by_type<true>(bf16, out_bf16, g, s);
}

// Long sums over rows in few tiles (a router's weight, one small matrix) would leave most compute units idle:
// their rows are cut into parts of at least 256, for at most about two workgroups on each. 256 x 2048 of 65536 rows:
// 164 us in parts, 363 without. Both sides of the bounds (in parts / without): 128 tiles 4096 rows 15.9 / 19.6, 2600
// rows 14.7 / 14.4, 2048 rows, where the second launch costs more than the rows, 14.6 / 12.2; 64 tiles 2600 rows 13.9
// / 15.1, 2048 rows 13.7 / 12.8; 160 tiles 4096 rows 21.2 / 21.2, 8192 rows 33.9 / 37.2; 256 tiles 4096 rows 23.6
// / 20.9, 16384 rows 68.3 / 67.2.
int dw_parts(int64_t R, int N, int K, int n) {
    const int64_t tiles = n * ceil_div(N, 64) * ceil_div(K, 64), mean = R / n;
    if (tiles > 128 || mean < 3000) return 1;
    const int64_t parts = 512 / tiles;
    return (int)(parts < mean / 256 ? parts : mean / 256);
}

hipError_t launch_grouped_dw(bool bf16, bool out_bf16, const GroupArgs& g, float* ws, hipStream_t s) {
    const int parts = dw_parts(g.R, g.rows, g.cols, g.n);
    if (parts > 1 && near(g, bf16 ? 2 : 4)) {
        GroupArgs p = g;
        p.out = ws;
        const hipError_t err = bf16 ? launch_outer<TBf16, Small, float, false>(p, s, parts)
                                    : launch_outer<TF32, Small, float, false>(p, s, parts);
        if (err != hipSuccess) return err;
        const int64_t size = (int64_t)g.n * g.rows * g.cols;
        const dim3 grid((unsigned)ceil_div(size, 1024));
        if (out_bf16) part_sum_kernel<<<grid, dim3(256), 0, s>>>(ws, parts, size, (__bf16*)g.out, 0);
        else part_sum_kernel<<<grid, dim3(256), 0, s>>>(ws, parts, size, (float*)g.out, g.accumulate);
        return hipGetLastError();
    }
    if (!bf16) return g.accumulate ? outer_by_shape<TF32, float, true>(g, s) : outer_by_shape<TF32, float, false>(g, s);
    if (out_bf16) return outer_by_shape<TBf16, __bf16, false>(g, s);
    return g.accumulate ? outer_by_shape<TBf16, float, true>(g, s) : outer_by_shape<TBf16, float, false>(g, s);
}

hipError_t launch_slot_sum(const float* rows, const int32_t* row_of, const int32_t* offsets, int n, int64_t T, int k,
                           int64_t R, int K, void* out, bool out_bf16, hipStream_t s) {
    const int64_t blocks = ceil_div(T * (K / 4), 256);
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
    if (out_bf16) slot_sum_kernel<<<grid, dim3(256), 0, s>>>(rows, row_of, offsets, n, T, k, R, K, (__bf16*)out);
    else slot_sum_kernel<<<grid, dim3(256), 0, s>>>(rows, row_of, offsets, n, T, k, R, K, (float*)out);
    return hipGetLastError();
}

}  // namespace pcm
