// C ABI of libpcomoe: host-side validation, workspace layout and launch sequencing.
// Every check runs before anything is enqueued; the library never allocates, frees or
// synchronises.
#include "pcomoe.h"

#include <algorithm>
#include <mutex>

#include "internal.h"

using namespace pcm;

// Scratch of pcm_project_combine_noalloc: z, its row scales and o live here instead of in a
// caller workspace. Each GPU the library runs on holds its own copy until the process ends.
// Host code never uses the array's name as an address: the device address of this GPU's copy
// comes from hipGetSymbolAddress (scratch_on_current_device).
static __device__ __align__(256) unsigned char scratch[PCM_NOALLOC_SCRATCH_BYTES];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mutex;
void* g_scratch_ptr[kMaxDevices];   // device address of `scratch` per device (set once)

// The address of the current device's scratch array, looked up on the first call made with
// that device current.
pcm_status scratch_on_current_device(void** out) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return PCM_ERR_HIP;
    if (dev < 0 || dev >= kMaxDevices) return PCM_ERR_UNSUPPORTED;
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_ptr[dev]) {
        void* p = nullptr;
        if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) return PCM_ERR_HIP;
        g_scratch_ptr[dev] = p;
    }
    *out = g_scratch_ptr[dev];
    return PCM_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

pcm_status check_shape(int64_t T, int n, int k) {
    if (T < 0 || n < 1 || k < 1 || k > n) return PCM_ERR_ARG;
    if (k > kMaxK || n > kMaxN) return PCM_ERR_UNSUPPORTED;
    if (T * (int64_t)k >= ((int64_t)1 << 31)) return PCM_ERR_UNSUPPORTED;
    return PCM_OK;
}

pcm_status check_dims(int H, int F) {
    if (H < 1 || F < 1) return PCM_ERR_ARG;
    if (H % 64 || F % 64) return PCM_ERR_UNSUPPORTED;
    return PCM_OK;
}

pcm_status check_paths(const pcm_paths* p) {
    if (!p || !p->path_bits || !p->beta || !p->expert_offsets || !p->row_token || !p->row_slot ||
        !p->row_of)
        return PCM_ERR_ARG;
    return PCM_OK;
}

// The experts' products: sizes, then types.
constexpr int64_t kMaxGroupedRows = (int64_t)1 << 30;
constexpr int kMaxGroupedWidth = INT32_MAX - 127;   // kernels count blocks as (width + 127) / 128
pcm_status check_grouped(int64_t T, int64_t R, int K, int N, int n) {
    if (T < 0 || R < 0 || K < 1 || N < 1 || n < 1) return PCM_ERR_ARG;
    if (K % 16 || N % 16 || K > kMaxGroupedWidth || N > kMaxGroupedWidth) return PCM_ERR_UNSUPPORTED;
    if (n > kMaxN || T >= kMaxGroupedRows || R >= kMaxGroupedRows) return PCM_ERR_UNSUPPORTED;
    return PCM_OK;
}
bool plain_dtype(pcm_dtype d) { return d == PCM_F32 || d == PCM_BF16; }
bool grouped_types(pcm_dtype dtype, pcm_dtype out) {
    return plain_dtype(dtype) && plain_dtype(out) && (dtype == PCM_BF16 || out == PCM_F32);
}
// The rows of a product: without offsets one group, without a gather the rows themselves.
bool grouped_rows(const int32_t* offsets, const int32_t* row_token, int64_t T, int64_t R, int n) {
    if (!offsets && (n != 1 || row_token)) return false;
    if (!row_token && T != R) return false;
    return !(row_token && T == 0 && R > 0) && aligned16(offsets) && aligned16(row_token);
}

// Training around the products: sizes, then what the calls on rows share.
constexpr int kMaxRowWidth = 1 << 28;   // a column's offset in bytes, and the next step's column, fit in 32 bits
pcm_status check_rows(int64_t T, int64_t R, int k, int H, int n) {
    const pcm_status st = check_grouped(T, R, H, 16, n);
    if (st != PCM_OK) return st;
    if (k < 1) return PCM_ERR_ARG;
    if (H > kMaxRowWidth) return PCM_ERR_UNSUPPORTED;
    return k > kMaxK ? PCM_ERR_UNSUPPORTED : PCM_OK;
}
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }   // any element of an array of 32-bit numbers

constexpr int kMaxTensors = 4096;
constexpr int64_t kMaxTensor = (int64_t)1 << 36;
pcm_status check_tensors(const pcm_tensor* t, int m) {
    for (int i = 0; i < m; ++i) {
        if (!plain_dtype(t[i].dtype) || t[i].count < 0) return PCM_ERR_ARG;
        if (t[i].count > kMaxTensor) return PCM_ERR_UNSUPPORTED;
        const uintptr_t size = t[i].dtype == PCM_BF16 ? 2 : 4;
        if (t[i].count && (!t[i].data || (uintptr_t)t[i].data % size)) return PCM_ERR_ARG;
    }
    return PCM_OK;
}
struct Range {
    uintptr_t from, to;
};
Range range_of(const pcm_tensor& t) {
    const uintptr_t from = (uintptr_t)t.data;
    return Range{from, from + (uintptr_t)t.count * (t.dtype == PCM_BF16 ? 2 : 4)};
}
template <class ITEM, class RANGE>
bool any_shared(ITEM* items, int count, RANGE range) {
    std::sort(items, items + count, [=](const ITEM& a, const ITEM& b) { return range(a).from < range(b).from; });
    for (int i = 1; i < count; ++i)
        if (range(items[i]).from < range(items[i - 1]).to) return true;
    return false;
}
// Whether two tensors of a call share memory, an output with its own gradient aside (then of the same type). 16 KB of stack:
// a caller's thread may have little. Up to 1024 ranges are sorted themselves, more of them by number (those of `out` from
// kMaxTensors on). 8192 ranges in any order take 0.65 ms that way, 0.45 as 128 KB of ranges; in address order 0.15 and 0.1.
bool overlapping(const pcm_tensor* in, const pcm_tensor* out, int m) {
    constexpr int kFew = 1024;
    union {
        Range ranges[kFew];
        uint16_t numbers[2 * kMaxTensors];
    } s;
    const auto tensor = [=](uint16_t i) -> const pcm_tensor& { return i < kMaxTensors ? in[i] : out[i - kMaxTensors]; };
    const auto each = [=](auto take) {
        for (int i = 0; i < m; ++i)
            if (in[i].count) take((uint16_t)i);
        for (int i = 0; out && i < m; ++i)
            if (in[i].count && (out[i].data != in[i].data || out[i].dtype != in[i].dtype)) take((uint16_t)(kMaxTensors + i));
    };
    int count = 0;
    if ((out ? 2 : 1) * m <= kFew) {
        each([&](uint16_t i) { s.ranges[count++] = range_of(tensor(i)); });
        return any_shared(s.ranges, count, [](const Range& r) { return r; });
    }
    each([&](uint16_t i) { s.numbers[count++] = i; });
    return any_shared(s.numbers, count, [=](uint16_t i) { return range_of(tensor(i)); });
}
// Whether `bytes` at p share memory with a tensor of a call.
bool on_tensors(const pcm_tensor* in, const pcm_tensor* out, int m, const void* p, size_t bytes) {
    const uintptr_t from = (uintptr_t)p, to = from + bytes;
    for (const pcm_tensor* t : {in, out})
        for (int i = 0; t && i < m; ++i) {
            const Range r = range_of(t[i]);
            if (t[i].count && r.from < to && from < r.to) return true;
        }
    return false;
}
pcm_status check_clip(const pcm_tensor* grads, const pcm_tensor* out, int m, float max_norm) {
    if (m < 0 || !(max_norm >= 0.0f)) return PCM_ERR_ARG;
    if (m > kMaxTensors) return PCM_ERR_UNSUPPORTED;
    if (m == 0) return PCM_OK;
    if (!grads) return PCM_ERR_ARG;
    pcm_status st = check_tensors(grads, m);
    if (st == PCM_OK && out) st = check_tensors(out, m);
    if (st != PCM_OK) return st;
    for (int i = 0; out && i < m; ++i)
        if (out[i].count != grads[i].count) return PCM_ERR_ARG;
    return overlapping(grads, out == grads ? nullptr : out, m) ? PCM_ERR_ARG : PCM_OK;
}

pcm_status from_hip(hipError_t e) { return e == hipSuccess ? PCM_OK : PCM_ERR_HIP; }

pcm_status check_scored(const pcm_scored_paths* p) {
    if (!p || !p->sel_pair || !p->sel_score || !p->n_src || !p->src_expert || !p->n_tgt ||
        !p->tgt_expert || !p->path_bits || !p->beta || !p->src_offsets || !p->src_row_token ||
        !p->src_row_slot || !p->src_row_of || !p->tgt_offsets || !p->tgt_row_token ||
        !p->tgt_row_slot || !p->tgt_row_of)
        return PCM_ERR_ARG;
    return PCM_OK;
}

pcm_status check_layout(const pcm_path_layout* l) {
    if (!l || !l->count || !l->pair || !l->bias) return PCM_ERR_ARG;
    return PCM_OK;
}

// The kernel choices of a pcm_tuning (NULL: every default) for the expansion or the
// projection side; PCM_ERR_ARG for a value outside the documented set.
pcm_status to_tune(const pcm_tuning* t, bool expansion, GemmTune* out) {
    *out = GemmTune();
    if (!t) return PCM_OK;
    if (t->tile != 0 && t->tile != 'S' && t->tile != 'M' && t->tile != 'L' && t->tile != 'W')
        return PCM_ERR_ARG;
    if (t->order_expand < -1 || t->order_expand > 2 || t->order_down < -1 || t->order_down > 2)
        return PCM_ERR_ARG;
    if (t->em_window < 0 || t->group_n < 0) return PCM_ERR_ARG;
    const int d = t->stream_depth;
    if (d != -1 && d != 0 && d != 2 && d != 3 && d != 4 && d != 6) return PCM_ERR_ARG;
    out->tile = (char)t->tile;
    out->order = expansion ? t->order_expand : t->order_down;
    out->window = t->em_window;
    out->group_n = t->group_n;
    out->stream_depth = d;
    return PCM_OK;
}

// Records stage event i of a tuning (if any) on the stream.
hipError_t stage_event(const pcm_tuning* t, int i, hipStream_t s) {
    if (!t || !t->stage_events[i]) return hipSuccess;
    return hipEventRecord((hipEvent_t)t->stage_events[i], s);
}

// Layer dtypes: PCM_BF16_F16DOWN is a bf16 layer whose projection weights are float16.
bool dtype_ok(pcm_dtype d) { return d == PCM_F32 || d == PCM_BF16 || d == PCM_BF16_F16DOWN; }
bool is_bf16(pcm_dtype d) { return d == PCM_BF16 || d == PCM_BF16_F16DOWN; }

// Workspace of the projection of R rows of n groups: z [R,F] (f16 for bf16 layers, f32
// otherwise), the per-row inverse scales [R] f32 (bf16 layers), then, when `with_o`, the
// projected rows o [ksplit, R, H] f32 (K slices of the projection); parts 256-byte aligned.
struct ProjWs {
    size_t zscale_off, o_off, total;
    int ksplit;
};
ProjWs proj_ws(size_t R, int n, int H, int F, pcm_dtype dt, bool with_o, char tile = 0) {
    ProjWs w;
    w.ksplit = (with_o && is_bf16(dt)) ? down_ksplit((int64_t)R, n, H, F, tile) : 1;
    const size_t z = align_up(R * F * (is_bf16(dt) ? 2 : 4), 256);
    w.zscale_off = z;
    w.o_off = z + (is_bf16(dt) ? align_up(R * sizeof(float), 256) : 0);
    w.total = w.o_off + (with_o ? align_up((size_t)w.ksplit * R * H * sizeof(float), 256) : 0);
    return w;
}

// Workspace of the per-path execution (baseline), P = T*k*k rows at most:
//   c, start [R] i32; path offsets [n+1] x2; path_token [P] x2; path_row_of [T*k*k] x2;
//   path_gather [P]; U [P or R, F] f32; z [P or R, F] (f16 + scales [P] for bf16); o [P, H] f32.
struct PathWs {
    size_t c, start, off_t, off_s, tok_t, tok_s, rof_t, rof_s, gather, u, z, zscale, o, total;
};
PathWs path_ws(int64_t T, int H, int F, int n, int k, pcm_dtype dt) {
    PathWs w{};
    const size_t R = (size_t)T * k, P = (size_t)T * k * k;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    w.c = take(R * 4);
    w.start = take(R * 4);
    w.off_t = take((size_t)(n + 1) * 4);
    w.off_s = take((size_t)(n + 1) * 4);
    w.tok_t = take(P * 4);
    w.tok_s = take(P * 4);
    w.rof_t = take(P * 4);
    w.rof_s = take(P * 4);
    w.gather = take(P * 4);
    w.u = take(P * F * 4);
    w.z = take(P * F * (is_bf16(dt) ? 2 : 4));
    w.zscale = take(is_bf16(dt) ? P * 4 : 0);
    w.o = take(P * H * 4);
    w.total = at;
    return w;
}

}  // namespace

extern "C" {

int pcm_abi_version(void) { return 123; }

const char* pcm_status_string(pcm_status s) {
    switch (s) {
        case PCM_OK: return "PCM_OK: success";
        case PCM_ERR_ARG: return "PCM_ERR_ARG: invalid argument (null or misaligned pointer, bad size, k > n)";
        case PCM_ERR_UNSUPPORTED: return "PCM_ERR_UNSUPPORTED: outside the supported limits (k <= 8, n <= 256, H and F multiples of 64, T*k < 2^31; experts' products: K and N multiples of 16 up to 2^31 - 128, T and R < 2^30)";
        case PCM_ERR_WORKSPACE: return "PCM_ERR_WORKSPACE: workspace smaller than pcm_workspace_bytes()";
        case PCM_ERR_HIP: return "PCM_ERR_HIP: a HIP launch failed";
    }
    return "unknown pcm_status";
}

size_t pcm_workspace_bytes(pcm_op op, int64_t T, int H, int F, int n, int k, pcm_dtype dtype) {
    if (T < 0 || n < 1 || k < 1) return 0;
    switch (op) {
        case PCM_OP_BUILD_PATHS: return build_paths_ws_bytes(T, n);
        case PCM_OP_ROUTE_PATHS: return route_paths_ws_bytes(T, n);
        case PCM_OP_EXPAND: return 0;
        case PCM_OP_PROJECT_COMBINE:
            if (H < 1 || F < 1) return 0;
            return proj_ws((size_t)T * k, n, H, F, dtype, true).total;
        case PCM_OP_ROUTE_LOGITS:
            if (H < 1 || H % 64) return 0;
            return is_bf16(dtype) ? router_ws_bytes(T, H, n) : 0;
        case PCM_OP_LAYER_PER_PATH:
            if (H < 1 || F < 1) return 0;
            return path_ws(T, H, F, n, k, dtype).total;
        case PCM_OP_GROUPED_DX:  // the rows' gradients [T*k, K] f32, K in the place of H
            if (H < 1) return 0;
            return align_up((size_t)T * k * H * sizeof(float), 256);
        case PCM_OP_GROUPED_DW: {  // T*k rows, K and N in the places of H and F: the parts' sums
            if (H < 1 || F < 1) return 0;
            const int parts = dw_parts(T * k, F, H, n);
            return parts > 1 ? (size_t)parts * n * H * F * sizeof(float) : 0;
        }
        case PCM_OP_GRAD_NORM: return grad_norm_ws_bytes(T);  // T tensors: the workgroups' sums
        case PCM_OP_ROUTE_SCORED:  // block counts of the source and the target dispatch
            return 2 * build_paths_ws_bytes(T, n);
        case PCM_OP_DENSE_SWIGLU:  // the SwiGLU output u [T,F] f32, then a projection input
            if (H < 1 || F < 1) return 0;
            return align_up((size_t)T * F * sizeof(float), 256) +
                   (is_bf16(dtype) ? proj_ws((size_t)T, 1, H, F, dtype, false).total : 0);
    }
    return 0;
}

pcm_status pcm_route(const float* logits, int64_t T, int n, int k, int32_t* topk_ids,
                     float* topk_w, void* stream) {
    pcm_status st = check_shape(T, n, k);
    if (st != PCM_OK) return st;
    if (T == 0) return PCM_OK;
    if (!logits || !topk_ids || !topk_w) return PCM_ERR_ARG;
    if (!aligned16(logits) || !aligned16(topk_ids) || !aligned16(topk_w)) return PCM_ERR_ARG;
    return from_hip(launch_route(logits, T, n, k, topk_ids, topk_w, (hipStream_t)stream));
}

pcm_status pcm_route_logits(pcm_dtype dtype, const void* x, const void* w_router, int64_t T,
                            int H, int n, int k, float* logits, int32_t* topk_ids, float* topk_w,
                            void* ws, size_t ws_bytes, void* stream) {
    pcm_status st = check_shape(T, n, k);
    if (st != PCM_OK) return st;
    if (H < 1) return PCM_ERR_ARG;
    if (H % 64) return PCM_ERR_UNSUPPORTED;
    if (!dtype_ok(dtype)) return PCM_ERR_ARG;
    if (T == 0) return PCM_OK;
    if (!x || !w_router || !topk_ids || !topk_w) return PCM_ERR_ARG;
    if (!aligned16(x) || !aligned16(w_router) || !aligned16(topk_ids) || !aligned16(topk_w) ||
        (logits && !aligned16(logits)))
        return PCM_ERR_ARG;
    const size_t need = is_bf16(dtype) ? router_ws_bytes(T, H, n) : 0;
    if (ws_bytes < need || (need && !ws)) return PCM_ERR_WORKSPACE;
    if (need && !aligned16(ws)) return PCM_ERR_ARG;
    return from_hip(launch_router(is_bf16(dtype), x, w_router, T, H, n, k, logits, topk_ids,
                                  topk_w, (float*)ws, (hipStream_t)stream));
}

pcm_status pcm_residual_add(pcm_dtype dtype, void* h, const float* y, int64_t T, int H,
                            void* stream) {
    if (T < 0 || H < 1) return PCM_ERR_ARG;
    if (H % 64) return PCM_ERR_UNSUPPORTED;
    if (!dtype_ok(dtype)) return PCM_ERR_ARG;
    if (T == 0) return PCM_OK;
    if (!h || !y || !aligned16(h) || !aligned16(y)) return PCM_ERR_ARG;
    return from_hip(launch_residual(h, y, T * (int64_t)H, is_bf16(dtype), (hipStream_t)stream));
}

pcm_status pcm_widen_f16(const void* w_bf16, int64_t count, void* w_f16, void* stream) {
    if (count < 0) return PCM_ERR_ARG;
    if (count == 0) return PCM_OK;
    if (!w_bf16 || !w_f16 || !aligned16(w_bf16) || !aligned16(w_f16)) return PCM_ERR_ARG;
    return from_hip(launch_widen_f16((const uint16_t*)w_bf16, count, (uint16_t*)w_f16,
                                     (hipStream_t)stream));
}

pcm_status pcm_build_paths(const int32_t* topk_ids, const float* topk_w, const uint8_t* mask,
                           int64_t T, int n, int k, pcm_beta_mode beta_mode, const pcm_paths* out,
                           void* ws, size_t ws_bytes, void* stream) {
    pcm_status st = check_shape(T, n, k);
    if (st != PCM_OK) return st;
    if (beta_mode < PCM_BETA_SRC_COND || beta_mode > PCM_BETA_GLOBAL) return PCM_ERR_ARG;
    if (T == 0) return PCM_OK;
    if (!topk_ids || !topk_w || !mask || check_paths(out) != PCM_OK) return PCM_ERR_ARG;
    if (!aligned16(topk_ids) || !aligned16(topk_w) || !aligned16(mask) ||
        !aligned16(out->path_bits) || !aligned16(out->beta) || !aligned16(out->expert_offsets) ||
        !aligned16(out->row_token) || !aligned16(out->row_slot) || !aligned16(out->row_of))
        return PCM_ERR_ARG;
    const size_t need = build_paths_ws_bytes(T, n);
    if (ws_bytes < need || (need && !ws)) return PCM_ERR_WORKSPACE;
    if (need && !aligned16(ws)) return PCM_ERR_ARG;
    return from_hip(launch_build_paths(topk_ids, topk_w, mask, T, n, k, (int)beta_mode,
                                       out->path_bits, out->beta, out->expert_offsets,
                                       out->row_token, out->row_slot, out->row_of, (int32_t*)ws,
                                       (hipStream_t)stream));
}

pcm_status pcm_mask_pack(const uint8_t* mask, int n, uint64_t* packed, void* stream) {
    if (n < 1) return PCM_ERR_ARG;
    if (n > kMaxN) return PCM_ERR_UNSUPPORTED;
    if (!mask || !packed || !aligned16(mask) || !aligned16(packed)) return PCM_ERR_ARG;
    return from_hip(launch_mask_pack(mask, n, packed, (hipStream_t)stream));
}

pcm_status pcm_route_paths(const float* logits, const uint64_t* packed_mask, int64_t T, int n,
                           int k, pcm_beta_mode beta_mode, int32_t* topk_ids, float* topk_w,
                           const pcm_paths* out, void* ws, size_t ws_bytes, void* stream) {
    pcm_status st = check_shape(T, n, k);
    if (st != PCM_OK) return st;
    if (beta_mode < PCM_BETA_SRC_COND || beta_mode > PCM_BETA_GLOBAL) return PCM_ERR_ARG;
    if (T == 0) return PCM_OK;
    if (!logits || !packed_mask || !topk_ids || !topk_w || check_paths(out) != PCM_OK)
        return PCM_ERR_ARG;
    if (!aligned16(logits) || !aligned16(packed_mask) || !aligned16(topk_ids) ||
        !aligned16(topk_w) || !aligned16(out->path_bits) || !aligned16(out->beta) ||
        !aligned16(out->expert_offsets) || !aligned16(out->row_token) ||
        !aligned16(out->row_slot) || !aligned16(out->row_of))
        return PCM_ERR_ARG;
    const size_t need = route_paths_ws_bytes(T, n);
    if (ws_bytes < need || !ws) return PCM_ERR_WORKSPACE;
    if (!aligned16(ws)) return PCM_ERR_ARG;
    return from_hip(launch_route_paths(logits, packed_mask, T, n, k, (int)beta_mode, topk_ids,
                                       topk_w, out->path_bits, out->beta, out->expert_offsets,
                                       out->row_token, out->row_slot, out->row_of, ws,
                                       (hipStream_t)stream));
}

pcm_status pcm_expand_tuned(pcm_dtype dtype, const void* x, const void* w_gate, const void* w_up,
                            const pcm_paths* paths, int64_t T, int H, int F, int n, int k, void* u,
                            void* ws, size_t ws_bytes, void* stream, const pcm_tuning* tuning) {
    (void)ws;
    (void)ws_bytes;
    pcm_status st = check_shape(T, n, k);
    if (st != PCM_OK) return st;
    if ((st = check_dims(H, F)) != PCM_OK) return st;
    if (!dtype_ok(dtype)) return PCM_ERR_ARG;
    GemmTune tune;
    if ((st = to_tune(tuning, true, &tune)) != PCM_OK) return st;
    if (T == 0) return PCM_OK;
    if (!x || !w_gate || !w_up || !u || check_paths(paths) != PCM_OK) return PCM_ERR_ARG;
    if (!aligned16(x) || !aligned16(w_gate) || !aligned16(w_up) || !aligned16(u)) return PCM_ERR_ARG;
    GemmArgs g{};
    g.a = x;
    g.b0 = w_gate;
    g.b1 = w_up;
    g.out = u;
    g.offsets = paths->expert_offsets;
    g.gather = paths->row_token;
    g.a_rows = T;
    g.n = n;
    g.K = H;
    g.N = F;
    const int64_t R = T * k;
    hipStream_t s = (hipStream_t)stream;
    return from_hip(is_bf16(dtype) ? launch_gemm_bf16(kExpand, g, R, s, tune)
                                      : launch_gemm_f32(kExpand, g, R, s));
}

pcm_status pcm_expand(pcm_dtype dtype, const void* x, const void* w_gate, const void* w_up,
                      const pcm_paths* paths, int64_t T, int H, int F, int n, int k, void* u,
                      void* ws, size_t ws_bytes, void* stream) {
    return pcm_expand_tuned(dtype, x, w_gate, w_up, paths, T, H, F, n, k, u, ws, ws_bytes, stream,
                            nullptr);
}

pcm_status pcm_project_combine_tuned(pcm_dtype dtype, const void* u, const void* w_down,
                                     const pcm_paths* paths, int64_t T, int H, int F, int n, int k,
                                     float* y, int accumulate, void* ws, size_t ws_bytes,
                                     void* stream, const pcm_tuning* tuning) {
    pcm_status st = check_shape(T, n, k);
    if (st != PCM_OK) return st;
    if ((st = check_dims(H, F)) != PCM_OK) return st;
    if (!dtype_ok(dtype)) return PCM_ERR_ARG;
    GemmTune tune;
    if ((st = to_tune(tuning, false, &tune)) != PCM_OK) return st;
    if (T == 0) return PCM_OK;
    if (!u || !w_down || !y || check_paths(paths) != PCM_OK) return PCM_ERR_ARG;
    if (!aligned16(u) || !aligned16(w_down) || !aligned16(y)) return PCM_ERR_ARG;
    const int64_t R = T * k;
    const ProjWs w = proj_ws((size_t)R, n, H, F, dtype, true, tune.tile);
    if (!ws || ws_bytes < w.total) return PCM_ERR_WORKSPACE;
    if (!aligned16(ws)) return PCM_ERR_ARG;
    void* z = ws;
    const bool bf16 = is_bf16(dtype);
    float* zscale = bf16 ? (float*)((char*)ws + w.zscale_off) : nullptr;
    float* o = (float*)((char*)ws + w.o_off);
    hipStream_t s = (hipStream_t)stream;
    MixMap m{};
    m.bits = paths->path_bits;
    m.beta = paths->beta;
    m.src_row = m.tgt_row = paths->row_of;
    m.K = k;
    m.R_src = m.R_tgt = R;
    hipError_t e = stage_event(tuning, 0, s);
    if (e == hipSuccess) e = launch_mix((const float*)u, z, zscale, m, T, F, s);
    if (e == hipSuccess) e = stage_event(tuning, 1, s);
    if (e != hipSuccess) return PCM_ERR_HIP;
    GemmArgs g{};
    g.a = z;
    g.b0 = w_down;
    g.b_f16 = dtype == PCM_BF16_F16DOWN;
    g.out = o;
    g.row_scale = zscale;
    g.offsets = paths->expert_offsets;
    g.a_rows = R;
    g.n = n;
    g.K = F;
    g.N = H;
    g.ksplit = w.ksplit;
    g.rows_total = R;
    e = bf16 ? launch_gemm_bf16(kDownStore, g, R, s, tune) : launch_gemm_f32(kDownStore, g, R, s);
    if (e == hipSuccess) e = stage_event(tuning, 2, s);
    if (e != hipSuccess) return PCM_ERR_HIP;
    e = launch_combine(o, w.ksplit, m, T, H, y, accumulate, s);
    if (e == hipSuccess) e = stage_event(tuning, 3, s);
    return from_hip(e);
}

pcm_status pcm_project_combine(pcm_dtype dtype, const void* u, const void* w_down,
                               const pcm_paths* paths, int64_t T, int H, int F, int n, int k,
                               float* y, int accumulate, void* ws, size_t ws_bytes, void* stream) {
    return pcm_project_combine_tuned(dtype, u, w_down, paths, T, H, F, n, k, y, accumulate, ws,
                                     ws_bytes, stream, nullptr);
}

pcm_status pcm_project_combine_noalloc(pcm_dtype dtype, const void* u, const void* w_down,
                                      const pcm_paths* paths, int64_t T, int H, int F, int n,
                                      int k, float* y, int accumulate, void* stream) {
    // the same checks, in the same order, as pcm_project_combine_tuned, before the scratch
    // size (so that bad arguments report PCM_ERR_ARG / UNSUPPORTED as there)
    pcm_status st = check_shape(T, n, k);
    if (st != PCM_OK) return st;
    if ((st = check_dims(H, F)) != PCM_OK) return st;
    if (!dtype_ok(dtype)) return PCM_ERR_ARG;
    if (T == 0) return PCM_OK;
    if (!u || !w_down || !y || check_paths(paths) != PCM_OK) return PCM_ERR_ARG;
    if (!aligned16(u) || !aligned16(w_down) || !aligned16(y)) return PCM_ERR_ARG;
    const size_t need = proj_ws((size_t)(T * k), n, H, F, dtype, true).total;
    if (need > (size_t)PCM_NOALLOC_SCRATCH_BYTES) return PCM_ERR_UNSUPPORTED;
    void* ws = nullptr;
    if ((st = scratch_on_current_device(&ws)) != PCM_OK) return st;
    // every byte of z, the scales and o that the combine reads is written earlier in the same
    // call (one z row per (token, target) by the mix, every o element by the projection), so
    // nothing is cleared
    return pcm_project_combine_tuned(dtype, u, w_down, paths, T, H, F, n, k, y, accumulate, ws,
                                     need, stream, nullptr);
}

pcm_status pcm_project_workspace_layout(pcm_dtype dtype, int64_t T, int H, int F, int n, int k,
                                        const pcm_tuning* tuning, size_t* z_off,
                                        size_t* zscale_off, size_t* o_off, int* ksplit) {
    pcm_status st = check_shape(T, n, k);
    if (st != PCM_OK) return st;
    if ((st = check_dims(H, F)) != PCM_OK) return st;
    if (!dtype_ok(dtype)) return PCM_ERR_ARG;
    GemmTune tune;
    if ((st = to_tune(tuning, false, &tune)) != PCM_OK) return st;
    if (!z_off || !zscale_off || !o_off || !ksplit) return PCM_ERR_ARG;
    const ProjWs w = proj_ws((size_t)(T * k), n, H, F, dtype, true, tune.tile);
    *z_off = 0;
    *zscale_off = is_bf16(dtype) ? w.zscale_off : 0;
    *o_off = w.o_off;
    *ksplit = w.ksplit;
    return PCM_OK;
}

pcm_status pcm_dense_swiglu_tuned(pcm_dtype dtype, const void* x, const void* w_gate,
                                  const void* w_up, const void* w_down, int64_t T, int H, int Fs,
                                  float* y, int accumulate, void* ws, size_t ws_bytes, void* stream,
                                  const pcm_tuning* tuning) {
    if (T < 0) return PCM_ERR_ARG;
    pcm_status st = check_dims(H, Fs);
    if (st != PCM_OK) return st;
    if (!dtype_ok(dtype)) return PCM_ERR_ARG;
    GemmTune tune_up, tune_down;
    if ((st = to_tune(tuning, true, &tune_up)) != PCM_OK) return st;
    if ((st = to_tune(tuning, false, &tune_down)) != PCM_OK) return st;
    if (T >= ((int64_t)1 << 31)) return PCM_ERR_UNSUPPORTED;
    if (T == 0) return PCM_OK;
    if (!x || !w_gate || !w_up || !w_down || !y) return PCM_ERR_ARG;
    if (!aligned16(x) || !aligned16(w_gate) || !aligned16(w_up) || !aligned16(w_down) || !aligned16(y))
        return PCM_ERR_ARG;
    const bool bf16 = is_bf16(dtype);
    const size_t u_bytes = align_up((size_t)T * Fs * sizeof(float), 256);
    const ProjWs w = proj_ws((size_t)T, 1, H, Fs, dtype, false);
    const size_t need = u_bytes + (bf16 ? w.total : 0);
    if (!ws || ws_bytes < need) return PCM_ERR_WORKSPACE;
    if (!aligned16(ws)) return PCM_ERR_ARG;
    hipStream_t s = (hipStream_t)stream;
    float* u = (float*)ws;
    GemmArgs g{};
    g.a = x;
    g.b0 = w_gate;
    g.b1 = w_up;
    g.out = u;
    g.offsets = nullptr;
    g.gather = nullptr;
    g.a_rows = T;
    g.n = 1;
    g.K = H;
    g.N = Fs;
    hipError_t e = bf16 ? launch_gemm_bf16(kExpand, g, T, s, tune_up) : launch_gemm_f32(kExpand, g, T, s);
    if (e != hipSuccess) return PCM_ERR_HIP;
    void* z = u;
    float* zscale = nullptr;
    if (bf16) {  // row-scaled float16 projection input
        z = (char*)ws + u_bytes;
        zscale = (float*)((char*)z + w.zscale_off);
        MixMap id{};  // identity: z_t = u_t
        id.K = 1;
        id.R_src = id.R_tgt = T;
        e = launch_mix(u, z, zscale, id, T, Fs, s);
        if (e != hipSuccess) return PCM_ERR_HIP;
    }
    GemmArgs d{};
    d.a = z;
    d.row_scale = zscale;
    d.b0 = w_down;
    d.b_f16 = dtype == PCM_BF16_F16DOWN;
    d.out = y;
    d.offsets = nullptr;
    d.a_rows = T;
    d.n = 1;
    d.K = Fs;
    d.N = H;
    d.accumulate = accumulate;
    e = bf16 ? launch_gemm_bf16(kDownAccum, d, T, s, tune_down) : launch_gemm_f32(kDownAccum, d, T, s);
    return from_hip(e);
}

pcm_status pcm_dense_swiglu(pcm_dtype dtype, const void* x, const void* w_gate, const void* w_up,
                            const void* w_down, int64_t T, int H, int Fs, float* y, int accumulate,
                            void* ws, size_t ws_bytes, void* stream) {
    return pcm_dense_swiglu_tuned(dtype, x, w_gate, w_up, w_down, T, H, Fs, y, accumulate, ws,
                                  ws_bytes, stream, nullptr);
}

pcm_status pcm_layer_per_path(pcm_dtype dtype, const void* x, const void* w_gate,
                              const void* w_up, const void* w_down, const pcm_paths* paths,
                              int64_t T, int H, int F, int n, int k, int reuse, float* y,
                              int accumulate, void* ws, size_t ws_bytes, void* stream) {
    pcm_status st = check_shape(T, n, k);
    if (st != PCM_OK) return st;
    if ((st = check_dims(H, F)) != PCM_OK) return st;
    if (!dtype_ok(dtype)) return PCM_ERR_ARG;
    if (T * (int64_t)k * k >= ((int64_t)1 << 31)) return PCM_ERR_UNSUPPORTED;
    if (T == 0) return PCM_OK;
    if (!x || !w_gate || !w_up || !w_down || !y || check_paths(paths) != PCM_OK) return PCM_ERR_ARG;
    if (!aligned16(x) || !aligned16(w_gate) || !aligned16(w_up) || !aligned16(w_down) || !aligned16(y))
        return PCM_ERR_ARG;
    const PathWs w = path_ws(T, H, F, n, k, dtype);
    if (!ws || ws_bytes < w.total) return PCM_ERR_WORKSPACE;
    if (!aligned16(ws)) return PCM_ERR_ARG;
    char* b = (char*)ws;
    auto i32 = [&](size_t off) { return (int32_t*)(b + off); };
    const int64_t R = T * k, P = T * (int64_t)k * k;
    const bool bf16 = is_bf16(dtype);
    hipStream_t s = (hipStream_t)stream;
    float* u = (float*)(b + w.u);
    void* z = b + w.z;
    float* zscale = bf16 ? (float*)(b + w.zscale) : nullptr;
    float* o = (float*)(b + w.o);
    hipError_t e;
    GemmArgs g{};
    g.a = x;
    g.b0 = w_gate;
    g.b1 = w_up;
    g.out = u;
    g.a_rows = T;
    g.n = n;
    g.K = H;
    g.N = F;
    int64_t u_rows;
    const int32_t* gather_src = nullptr;
    if (reuse) {  // one expansion row per (token, source): the top-k dispatch itself
        g.offsets = paths->expert_offsets;
        g.gather = paths->row_token;
        u_rows = R;
    } else {      // one expansion row per path, keyed by its source
        e = launch_path_rows(paths->path_bits, paths->expert_offsets, paths->row_token,
                             paths->row_slot, paths->row_of, R, n, k, 0, nullptr, i32(w.c),
                             i32(w.start), i32(w.off_s), i32(w.tok_s), i32(w.rof_s), nullptr, s);
        if (e != hipSuccess) return PCM_ERR_HIP;
        g.offsets = i32(w.off_s);
        g.gather = i32(w.tok_s);
        u_rows = P;
        gather_src = i32(w.rof_s);
    }
    e = bf16 ? launch_gemm_bf16(kExpand, g, u_rows, s, GemmTune()) : launch_gemm_f32(kExpand, g, u_rows, s);
    if (e != hipSuccess) return PCM_ERR_HIP;
    if (bf16) {  // U rows as row-scaled float16, no mixing
        MixMap id{};
        id.K = 1;
        id.R_src = id.R_tgt = u_rows;
        id.live = reuse ? nullptr : i32(w.off_s) + n;
        e = launch_mix(u, z, zscale, id, u_rows, F, s);
        if (e != hipSuccess) return PCM_ERR_HIP;
    } else {
        z = u;
    }
    // one projection row per path, keyed by its target, gathering its source's z row
    e = launch_path_rows(paths->path_bits, paths->expert_offsets, paths->row_token,
                         paths->row_slot, paths->row_of, R, n, k, 1, gather_src, i32(w.c),
                         i32(w.start), i32(w.off_t), i32(w.tok_t), i32(w.rof_t), i32(w.gather), s);
    if (e != hipSuccess) return PCM_ERR_HIP;
    GemmArgs d{};
    d.a = z;
    d.b0 = w_down;
    d.b_f16 = dtype == PCM_BF16_F16DOWN;
    d.out = o;
    d.row_scale = zscale;
    d.offsets = i32(w.off_t);
    d.gather = i32(w.gather);
    d.a_rows = u_rows;
    d.n = n;
    d.K = F;
    d.N = H;
    d.ksplit = 1;
    d.rows_total = P;
    e = bf16 ? launch_gemm_bf16(kDownStore, d, P, s, GemmTune()) : launch_gemm_f32(kDownStore, d, P, s);
    if (e != hipSuccess) return PCM_ERR_HIP;
    return from_hip(launch_combine_paths(o, paths->path_bits, paths->beta, i32(w.rof_t), T, k, H, P,
                                         y, accumulate, s));
}

pcm_status pcm_path_layout_build(const uint8_t* mask, const float* bias, int n,
                                 const pcm_path_layout* out, void* stream) {
    if (n < 1) return PCM_ERR_ARG;
    if (n > kMaxN) return PCM_ERR_UNSUPPORTED;
    if (!mask || !bias || check_layout(out) != PCM_OK) return PCM_ERR_ARG;
    return from_hip(launch_path_layout(mask, bias, n, out->count, out->pair, out->bias,
                                       (hipStream_t)stream));
}

pcm_status pcm_route_scored(const float* g_base, const float* g_tgt, float lambda,
                            const pcm_path_layout* layout, int64_t T, int n, int K,
                            const pcm_scored_paths* out, void* ws, size_t ws_bytes, void* stream) {
    pcm_status st = check_shape(T, n, K);
    if (st != PCM_OK) return st;
    if (!(lambda == lambda) || lambda - lambda != 0.0f) return PCM_ERR_ARG;  // NaN or inf
    if (T == 0) return PCM_OK;
    if (!g_base || !g_tgt || check_layout(layout) != PCM_OK || check_scored(out) != PCM_OK)
        return PCM_ERR_ARG;
    const size_t one = build_paths_ws_bytes(T, n);
    if (ws_bytes < 2 * one || (one && !ws)) return PCM_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    hipError_t e = launch_route_scored(g_base, g_tgt, lambda, layout->count, layout->pair,
                                       layout->bias, T, n, K, out->sel_pair, out->sel_score,
                                       out->n_src, out->src_expert, out->n_tgt, out->tgt_expert,
                                       out->path_bits, out->beta, s);
    if (e != hipSuccess) return PCM_ERR_HIP;
    const DispatchSides d = {{{out->src_expert, out->n_src, out->src_offsets, out->src_row_token,
                               out->src_row_slot, out->src_row_of, (int32_t*)ws},
                              {out->tgt_expert, out->n_tgt, out->tgt_offsets, out->tgt_row_token,
                               out->tgt_row_slot, out->tgt_row_of,
                               one ? (int32_t*)((char*)ws + one) : nullptr}}};
    return from_hip(launch_dispatch(d, T, n, K, s));
}

pcm_status pcm_expand_scored_tuned(pcm_dtype dtype, const void* x, const void* w_gate,
                                   const void* w_up, const pcm_scored_paths* paths, int64_t T,
                                   int H, int F, int n, int K, void* u, void* ws, size_t ws_bytes,
                                   void* stream, const pcm_tuning* tuning) {
    (void)ws;
    (void)ws_bytes;
    pcm_status st = check_shape(T, n, K);
    if (st != PCM_OK) return st;
    if ((st = check_dims(H, F)) != PCM_OK) return st;
    if (!dtype_ok(dtype)) return PCM_ERR_ARG;
    GemmTune tune;
    if ((st = to_tune(tuning, true, &tune)) != PCM_OK) return st;
    if (T == 0) return PCM_OK;
    if (!x || !w_gate || !w_up || !u || check_scored(paths) != PCM_OK) return PCM_ERR_ARG;
    if (!aligned16(x) || !aligned16(w_gate) || !aligned16(w_up) || !aligned16(u)) return PCM_ERR_ARG;
    GemmArgs g{};
    g.a = x;
    g.b0 = w_gate;
    g.b1 = w_up;
    g.out = u;
    g.offsets = paths->src_offsets;
    g.gather = paths->src_row_token;
    g.a_rows = T;
    g.n = n;
    g.K = H;
    g.N = F;
    const int64_t R = T * K;  // upper bound: the rows in use are src_offsets[n]
    hipStream_t s = (hipStream_t)stream;
    return from_hip(is_bf16(dtype) ? launch_gemm_bf16(kExpand, g, R, s, tune)
                                      : launch_gemm_f32(kExpand, g, R, s));
}

pcm_status pcm_expand_scored(pcm_dtype dtype, const void* x, const void* w_gate, const void* w_up,
                             const pcm_scored_paths* paths, int64_t T, int H, int F, int n, int K,
                             void* u, void* ws, size_t ws_bytes, void* stream) {
    return pcm_expand_scored_tuned(dtype, x, w_gate, w_up, paths, T, H, F, n, K, u, ws, ws_bytes,
                                   stream, nullptr);
}

pcm_status pcm_project_combine_scored_tuned(pcm_dtype dtype, const void* u, const void* w_down,
                                            const pcm_scored_paths* paths, int64_t T, int H, int F,
                                            int n, int K, float* y, int accumulate, void* ws,
                                            size_t ws_bytes, void* stream,
                                            const pcm_tuning* tuning) {
    pcm_status st = check_shape(T, n, K);
    if (st != PCM_OK) return st;
    if ((st = check_dims(H, F)) != PCM_OK) return st;
    if (!dtype_ok(dtype)) return PCM_ERR_ARG;
    GemmTune tune;
    if ((st = to_tune(tuning, false, &tune)) != PCM_OK) return st;
    if (T == 0) return PCM_OK;
    if (!u || !w_down || !y || check_scored(paths) != PCM_OK) return PCM_ERR_ARG;
    if (!aligned16(u) || !aligned16(w_down) || !aligned16(y)) return PCM_ERR_ARG;
    const int64_t R = T * K;  // row bound of U, z and o
    const ProjWs w = proj_ws((size_t)R, n, H, F, dtype, true, tune.tile);
    if (!ws || ws_bytes < w.total) return PCM_ERR_WORKSPACE;
    if (!aligned16(ws)) return PCM_ERR_ARG;
    void* z = ws;
    const bool bf16 = is_bf16(dtype);
    float* zscale = bf16 ? (float*)((char*)ws + w.zscale_off) : nullptr;
    float* o = (float*)((char*)ws + w.o_off);
    hipStream_t s = (hipStream_t)stream;
    MixMap m{};
    m.bits = paths->path_bits;
    m.beta = paths->beta;
    m.src_row = paths->src_row_of;
    m.tgt_row = paths->tgt_row_of;
    m.n_src = paths->n_src;
    m.n_tgt = paths->n_tgt;
    m.K = K;
    m.R_src = m.R_tgt = R;
    hipError_t e = stage_event(tuning, 0, s);
    if (e == hipSuccess) e = launch_mix((const float*)u, z, zscale, m, T, F, s);
    if (e == hipSuccess) e = stage_event(tuning, 1, s);
    if (e != hipSuccess) return PCM_ERR_HIP;
    GemmArgs g{};
    g.a = z;
    g.b0 = w_down;
    g.b_f16 = dtype == PCM_BF16_F16DOWN;
    g.out = o;
    g.row_scale = zscale;
    g.offsets = paths->tgt_offsets;
    g.a_rows = R;
    g.n = n;
    g.K = F;
    g.N = H;
    g.ksplit = w.ksplit;
    g.rows_total = R;
    e = bf16 ? launch_gemm_bf16(kDownStore, g, R, s, tune) : launch_gemm_f32(kDownStore, g, R, s);
    if (e == hipSuccess) e = stage_event(tuning, 2, s);
    if (e != hipSuccess) return PCM_ERR_HIP;
    e = launch_combine(o, w.ksplit, m, T, H, y, accumulate, s);
    if (e == hipSuccess) e = stage_event(tuning, 3, s);
    return from_hip(e);
}

pcm_status pcm_project_combine_scored(pcm_dtype dtype, const void* u, const void* w_down,
                                      const pcm_scored_paths* paths, int64_t T, int H, int F, int n,
                                      int K, float* y, int accumulate, void* ws, size_t ws_bytes,
                                      void* stream) {
    return pcm_project_combine_scored_tuned(dtype, u, w_down, paths, T, H, F, n, K, y, accumulate,
                                            ws, ws_bytes, stream, nullptr);
}

pcm_status pcm_grouped_gemm(pcm_dtype dtype, pcm_dtype out_dtype, const void* x, const void* w,
                            const int32_t* offsets, const int32_t* row_token, int64_t T, int64_t R,
                            int K, int N, int n, void* y, void* stream) {
    const pcm_status st = check_grouped(T, R, K, N, n);
    if (st != PCM_OK) return st;
    if (!grouped_types(dtype, out_dtype)) return PCM_ERR_ARG;
    if (!grouped_rows(offsets, row_token, T, R, n)) return PCM_ERR_ARG;
    if (R == 0) return PCM_OK;
    if (!x || !w || !y || !aligned16(x) || !aligned16(w) || !aligned16(y)) return PCM_ERR_ARG;
    GroupArgs g{};
    g.a = x;
    g.b = w;
    g.out = y;
    g.offsets = offsets;
    g.gather = row_token;
    g.x_rows = T;
    g.R = R;
    g.n = n;
    g.len = K;
    g.cols = N;
    return from_hip(launch_grouped(dtype == PCM_BF16, out_dtype == PCM_BF16, g, (hipStream_t)stream));
}

pcm_status pcm_grouped_gemm_dx(pcm_dtype dtype, pcm_dtype out_dtype, const void* dy, const void* w,
                               const int32_t* offsets, const int32_t* row_of, int64_t T, int k,
                               int64_t R, int K, int N, int n, void* dx, void* ws, size_t ws_bytes,
                               void* stream) {
    const pcm_status st = check_grouped(T, R, K, N, n);
    if (st != PCM_OK) return st;
    if (!grouped_types(dtype, out_dtype) || k < 1) return PCM_ERR_ARG;
    if (k > kMaxK) return PCM_ERR_UNSUPPORTED;
    if (!grouped_rows(offsets, nullptr, R, R, n)) return PCM_ERR_ARG;
    if (row_of ? R > T * k : T != R || k != 1) return PCM_ERR_ARG;
    if (T == 0) return PCM_OK;
    if (!dx || !aligned16(dx) || !aligned16(row_of)) return PCM_ERR_ARG;
    if (R > 0 && (!dy || !w || !aligned16(dy) || !aligned16(w))) return PCM_ERR_ARG;
    if (row_of) {
        const size_t need = pcm_workspace_bytes(PCM_OP_GROUPED_DX, T, K, 0, n, k, dtype);
        if (ws_bytes < need || !ws) return PCM_ERR_WORKSPACE;
        if (!aligned16(ws)) return PCM_ERR_ARG;
    }
    GroupArgs g{};
    g.a = dy;
    g.b = w;
    g.out = row_of ? ws : dx;
    g.offsets = offsets;
    g.x_rows = R;
    g.R = R;
    g.n = n;
    g.len = N;
    g.cols = K;
    hipStream_t s = (hipStream_t)stream;
    if (R > 0) {
        const hipError_t err = launch_grouped_dx(dtype == PCM_BF16, !row_of && out_dtype == PCM_BF16, g, s);
        if (err != hipSuccess) return PCM_ERR_HIP;
    }
    if (!row_of) return PCM_OK;
    return from_hip(launch_slot_sum((const float*)ws, row_of, offsets, n, T, k, R, K, dx, out_dtype == PCM_BF16, s));
}

pcm_status pcm_grouped_gemm_dw(pcm_dtype dtype, pcm_dtype out_dtype, const void* x, const void* dy,
                               const int32_t* offsets, const int32_t* row_token, int64_t T, int64_t R,
                               int K, int N, int n, void* dw, int accumulate, void* ws, size_t ws_bytes,
                               void* stream) {
    const pcm_status st = check_grouped(T, R, K, N, n);
    if (st != PCM_OK) return st;
    if (!grouped_types(dtype, out_dtype) || (accumulate && out_dtype != PCM_F32)) return PCM_ERR_ARG;
    if (!grouped_rows(offsets, row_token, T, R, n)) return PCM_ERR_ARG;
    if (!dw || !aligned16(dw)) return PCM_ERR_ARG;
    if (R > 0 && (!x || !dy || !aligned16(x) || !aligned16(dy))) return PCM_ERR_ARG;
    if (R == 0 && accumulate) return PCM_OK;
    const size_t need = pcm_workspace_bytes(PCM_OP_GROUPED_DW, R, K, N, n, 1, dtype);
    if (ws_bytes < need || (need && !ws)) return PCM_ERR_WORKSPACE;
    if (need && !aligned16(ws)) return PCM_ERR_ARG;
    GroupArgs g{};
    g.a = dy;
    g.b = x;
    g.out = dw;
    g.offsets = R > 0 ? offsets : nullptr;
    g.gather = R > 0 ? row_token : nullptr;
    g.x_rows = T;
    g.R = R;
    g.n = n;
    g.rows = N;
    g.cols = K;
    g.accumulate = accumulate != 0;
    return from_hip(launch_grouped_dw(dtype == PCM_BF16, out_dtype == PCM_BF16, g, (float*)ws,
                                      (hipStream_t)stream));
}

static pcm_status quant_rows(pcm_dtype dtype, bool swiglu, const void* x, const int32_t* count, int64_t R,
                             int K, uint8_t* q, float* scale, void* stream) {
    const pcm_status st = check_grouped(0, R, K, 16, 1);
    if (st != PCM_OK) return st;
    if (!plain_dtype(dtype)) return PCM_ERR_ARG;
    if (R == 0) return PCM_OK;
    // count may be any element of an offsets array
    if (!x || !q || !scale || !aligned16(x) || !aligned16(q) || !aligned16(scale) || ((uintptr_t)count & 3u))
        return PCM_ERR_ARG;
    return from_hip(launch_quant_rows(dtype == PCM_BF16, swiglu, x, count, R, K, q, scale, (hipStream_t)stream));
}

pcm_status pcm_quant_fp8_rows(pcm_dtype dtype, const void* x, const int32_t* count, int64_t R, int K,
                              uint8_t* q, float* scale, void* stream) {
    return quant_rows(dtype, false, x, count, R, K, q, scale, stream);
}

pcm_status pcm_swiglu_quant_fp8(pcm_dtype dtype, const void* gate_up, const int32_t* count, int64_t R,
                                int F, uint8_t* q, float* scale, void* stream) {
    return quant_rows(dtype, true, gate_up, count, R, F, q, scale, stream);
}

pcm_status pcm_quant_fp8_weights(pcm_dtype dtype, const void* w, int n, int N, int K, uint8_t* q,
                                 float* scale, uint8_t* q_t, float* scale_t, void* stream) {
    const pcm_status st = check_grouped(0, 0, K, N, n);
    if (st != PCM_OK) return st;
    if (!plain_dtype(dtype)) return PCM_ERR_ARG;
    if (!w || !q || !scale || !aligned16(w) || !aligned16(q) || !aligned16(scale)) return PCM_ERR_ARG;
    if (!q_t != !scale_t || !aligned16(q_t) || !aligned16(scale_t)) return PCM_ERR_ARG;
    return from_hip(launch_quant_weights(dtype == PCM_BF16, w, n, N, K, q, scale, q_t, scale_t, (hipStream_t)stream));
}

pcm_status pcm_grouped_gemm_fp8(pcm_dtype out_dtype, const uint8_t* x, const float* x_scale,
                                const uint8_t* w, const float* w_scale, const int32_t* offsets,
                                const int32_t* row_token, int64_t T, int64_t R, int K, int N, int n,
                                void* y, void* stream) {
    const pcm_status st = check_grouped(T, R, K, N, n);
    if (st != PCM_OK) return st;
    if (!plain_dtype(out_dtype) || !grouped_rows(offsets, row_token, T, R, n)) return PCM_ERR_ARG;
    if (R == 0) return PCM_OK;
    if (!x || !x_scale || !w || !w_scale || !y) return PCM_ERR_ARG;
    if (!aligned16(x) || !aligned16(x_scale) || !aligned16(w) || !aligned16(w_scale) || !aligned16(y))
        return PCM_ERR_ARG;
    GroupArgs g{};
    g.a = x;
    g.b = w;
    g.a_scale = x_scale;
    g.b_scale = w_scale;
    g.out = y;
    g.offsets = offsets;
    g.gather = row_token;
    g.x_rows = T;
    g.R = R;
    g.n = n;
    g.len = K;
    g.cols = N;
    return from_hip(launch_grouped_fp8(out_dtype == PCM_BF16, g, (hipStream_t)stream));
}

static pcm_status rows_call(bool to_rows, pcm_dtype tokens_dtype, pcm_dtype rows_dtype, pcm_dtype out_dtype,
                            const void* tokens, const void* rows,
                            const int32_t* row_of, const float* weights, const int32_t* offsets, int64_t T, int k,
                            int64_t R, int H, int n, void* out, float* dweights, bool dot, int accumulate, void* stream) {
    const pcm_status st = check_rows(T, R, k, H, n);
    if (st != PCM_OK) return st;
    if (!plain_dtype(tokens_dtype) || !plain_dtype(rows_dtype) || !plain_dtype(out_dtype) || (!offsets && n != 1))
        return PCM_ERR_ARG;
    if (accumulate && out_dtype != PCM_F32) return PCM_ERR_ARG;
    if (!aligned16(tokens) || !aligned16(rows) || !aligned16(row_of) || !aligned16(weights) || !aligned4(offsets) ||
        !aligned16(out) || !aligned16(dweights))
        return PCM_ERR_ARG;
    // (row buffers without rows may be NULL)
    if (T == 0 || (to_rows && R == 0 && !dweights)) return PCM_OK;
    if (!row_of || (!out && !dweights) || (!dot && !out)) return PCM_ERR_ARG;
    if (!tokens && ((to_rows && R > 0) || dweights)) return PCM_ERR_ARG;
    if (!rows && R > 0 && (!to_rows || dweights)) return PCM_ERR_ARG;
    RowsArgs g{};
    g.tokens = tokens;
    g.rows = rows;
    g.out = out;
    g.row_of = row_of;
    g.weights = weights;
    g.dweights = dweights;
    g.offsets = offsets;
    g.T = T;
    g.R = R;
    g.k = k;
    g.H = H;
    g.n = n;
    g.accumulate = accumulate != 0;
    return from_hip(launch_rows(to_rows, tokens_dtype == PCM_BF16, rows_dtype == PCM_BF16, out_dtype == PCM_BF16, g,
                                (hipStream_t)stream));
}

pcm_status pcm_dispatch_rows(pcm_dtype dtype, pcm_dtype out_dtype, const void* x, const int32_t* row_of,
                             const float* weights, const int32_t* offsets, int64_t T, int k, int64_t R,
                             int H, int n, void* y, void* stream) {
    return rows_call(true, dtype, dtype, out_dtype, x, nullptr, row_of, weights, offsets, T, k, R, H, n, y, nullptr, false, 0, stream);
}

pcm_status pcm_dispatch_rows_grad(pcm_dtype dtype, pcm_dtype x_dtype, pcm_dtype out_dtype, const void* dy, const void* x,
                                  const int32_t* row_of, const float* weights, const int32_t* offsets,
                                  int64_t T, int k, int64_t R, int H, int n, void* dx, float* dweights,
                                  void* stream) {
    return rows_call(false, x_dtype, dtype, out_dtype, x, dy, row_of, weights, offsets, T, k, R, H, n, dx, dweights, true, 0, stream);
}

pcm_status pcm_combine_rows(pcm_dtype dtype, pcm_dtype out_dtype, const void* o, const int32_t* row_of,
                            const float* weights, const int32_t* offsets, int64_t T, int k, int64_t R,
                            int H, int n, void* y, int accumulate, void* stream) {
    return rows_call(false, dtype, dtype, out_dtype, nullptr, o, row_of, weights, offsets, T, k, R, H, n, y, nullptr, false, accumulate,
                     stream);
}

pcm_status pcm_combine_rows_grad(pcm_dtype dtype, pcm_dtype o_dtype, pcm_dtype out_dtype, const void* dy, const void* o,
                                 const int32_t* row_of, const float* weights, const int32_t* offsets,
                                 int64_t T, int k, int64_t R, int H, int n, void* d_o, float* dweights,
                                 void* stream) {
    return rows_call(true, dtype, o_dtype, out_dtype, dy, o, row_of, weights, offsets, T, k, R, H, n, d_o, dweights, true, 0, stream);
}

static pcm_status swiglu_call(pcm_dtype dtype, pcm_dtype out_dtype, const void* gate_up, const void* du, bool grad,
                              const int32_t* count, int64_t R, int F, void* out, void* stream) {
    const pcm_status st = check_rows(0, R, 1, F, 1);
    if (st != PCM_OK) return st;
    if (!plain_dtype(dtype) || !plain_dtype(out_dtype)) return PCM_ERR_ARG;
    if (R == 0) return PCM_OK;
    if (!gate_up || !out || (grad && !du) || !aligned16(gate_up) || !aligned16(du) || !aligned16(out) || !aligned4(count))
        return PCM_ERR_ARG;
    return from_hip(launch_swiglu(dtype == PCM_BF16, out_dtype == PCM_BF16, gate_up, du, count, R, F, out, (hipStream_t)stream));
}

pcm_status pcm_swiglu(pcm_dtype dtype, pcm_dtype out_dtype, const void* gate_up, const int32_t* count,
                      int64_t R, int F, void* u, void* stream) {
    return swiglu_call(dtype, out_dtype, gate_up, nullptr, false, count, R, F, u, stream);
}

pcm_status pcm_swiglu_grad(pcm_dtype dtype, pcm_dtype out_dtype, const void* gate_up, const void* du,
                           const int32_t* count, int64_t R, int F, void* dgate_up, void* stream) {
    return swiglu_call(dtype, out_dtype, gate_up, du, true, count, R, F, dgate_up, stream);
}

static pcm_status mix_call(bool grad, pcm_dtype dtype, pcm_dtype out_dtype, const void* u, const void* dz,
                           const uint64_t* path_bits, const float* beta, const int32_t* src_row_of,
                           const int32_t* tgt_row_of, int64_t T, int k, int64_t R_src, int64_t R_tgt, int F, void* out,
                           float* dbeta, void* stream) {
    pcm_status st = check_rows(T, R_src, k, F, 1);
    if (st == PCM_OK) st = check_rows(T, R_tgt, k, F, 1);
    if (st != PCM_OK) return st;
    if (!plain_dtype(dtype) || !plain_dtype(out_dtype)) return PCM_ERR_ARG;
    if (!aligned16(u) || !aligned16(dz) || !aligned16(path_bits) || !aligned16(beta) || !aligned16(src_row_of) ||
        !aligned16(tgt_row_of) || !aligned16(out) || !aligned16(dbeta))
        return PCM_ERR_ARG;
    if (T == 0 || ((grad ? R_src : R_tgt) == 0 && !dbeta)) return PCM_OK;   // (buffers without rows may be NULL)
    if (!path_bits || !beta || !src_row_of || !tgt_row_of || (!out && !dbeta)) return PCM_ERR_ARG;
    if (!u && R_src > 0 && (!grad || dbeta)) return PCM_ERR_ARG;
    if (!dz && grad && R_tgt > 0) return PCM_ERR_ARG;
    MixRowsArgs g{};
    g.u = u;
    g.dz = dz;
    g.out = out;
    g.dbeta = dbeta;
    g.bits = path_bits;
    g.beta = beta;
    g.src_row_of = src_row_of;
    g.tgt_row_of = tgt_row_of;
    g.T = T;
    g.R_src = R_src;
    g.R_tgt = R_tgt;
    g.k = k;
    g.F = F;
    return from_hip(launch_mix_rows(grad, dtype == PCM_BF16, out_dtype == PCM_BF16, g, (hipStream_t)stream));
}

pcm_status pcm_mix_rows(pcm_dtype dtype, pcm_dtype out_dtype, const void* u, const uint64_t* path_bits,
                        const float* beta, const int32_t* src_row_of, const int32_t* tgt_row_of, int64_t T,
                        int k, int64_t R_src, int64_t R_tgt, int F, void* z, void* stream) {
    return mix_call(false, dtype, out_dtype, u, nullptr, path_bits, beta, src_row_of, tgt_row_of, T, k, R_src, R_tgt, F, z,
                    nullptr, stream);
}

pcm_status pcm_mix_rows_grad(pcm_dtype dtype, pcm_dtype out_dtype, const void* dz, const void* u,
                             const uint64_t* path_bits, const float* beta, const int32_t* src_row_of,
                             const int32_t* tgt_row_of, int64_t T, int k, int64_t R_src, int64_t R_tgt, int F,
                             void* du, float* dbeta, void* stream) {
    return mix_call(true, dtype, out_dtype, u, dz, path_bits, beta, src_row_of, tgt_row_of, T, k, R_src, R_tgt, F, du, dbeta,
                    stream);
}

pcm_status pcm_route_grad(pcm_dtype out_dtype, const int32_t* topk_ids, const float* topk_w,
                          const uint64_t* path_bits, const float* dbeta, pcm_beta_mode beta_mode,
                          const float* dw, int64_t T, int n, int k, void* dlogits, void* stream) {
    const pcm_status st = check_shape(T, n, k);
    if (st != PCM_OK) return st;
    if (!plain_dtype(out_dtype) || beta_mode < PCM_BETA_SRC_COND || beta_mode > PCM_BETA_GLOBAL) return PCM_ERR_ARG;
    if (T >= kMaxGroupedRows) return PCM_ERR_UNSUPPORTED;
    if (!aligned16(topk_ids) || !aligned16(topk_w) || !aligned16(path_bits) || !aligned16(dbeta) || !aligned16(dw) ||
        !aligned16(dlogits) || !path_bits != !dbeta)
        return PCM_ERR_ARG;
    if (T == 0) return PCM_OK;
    if (!topk_ids || !topk_w || !dlogits || (!dbeta && !dw)) return PCM_ERR_ARG;
    RouteGradArgs g{};
    g.ids = topk_ids;
    g.w = topk_w;
    g.bits = path_bits;
    g.dbeta = dbeta;
    g.dw = dw;
    g.dlogits = dlogits;
    g.T = T;
    g.n = n;
    g.k = k;
    g.beta_mode = (int)beta_mode;
    return from_hip(launch_route_grad(out_dtype == PCM_BF16, g, (hipStream_t)stream));
}

static pcm_status check_norm(const pcm_tensor* grads, const pcm_tensor* out, int m, const float* norm, const void* ws,
                             size_t ws_bytes) {
    if (!norm || !aligned4(norm)) return PCM_ERR_ARG;
    const size_t need = pcm_workspace_bytes(PCM_OP_GRAD_NORM, m, 0, 0, 1, 1, PCM_F32);
    if (ws_bytes < need || !ws) return PCM_ERR_WORKSPACE;
    if (!aligned16(ws)) return PCM_ERR_ARG;
    const uintptr_t in_ws = (uintptr_t)norm - (uintptr_t)ws;
    if (in_ws < need || on_tensors(grads, out, m, norm, sizeof(float)) || on_tensors(grads, out, m, ws, need)) return PCM_ERR_ARG;
    return PCM_OK;
}

pcm_status pcm_grad_norm(const pcm_tensor* grads, int m, float* norm, void* ws, size_t ws_bytes, void* stream) {
    if (m < 0 || (m && !grads)) return PCM_ERR_ARG;
    if (m > kMaxTensors) return PCM_ERR_UNSUPPORTED;
    pcm_status st = check_tensors(grads, m);
    if (st == PCM_OK) st = check_norm(grads, nullptr, m, norm, ws, ws_bytes);
    if (st != PCM_OK) return st;
    return from_hip(launch_grad_norm(grads, nullptr, m, false, 0.0f, norm, (double*)ws, (hipStream_t)stream));
}

pcm_status pcm_clip_grads(const pcm_tensor* grads, const pcm_tensor* out, int m, const float* norm,
                          float max_norm, void* stream) {
    const pcm_status st = check_clip(grads, out, m, max_norm);
    if (st != PCM_OK) return st;
    if (m == 0) return PCM_OK;
    if (!norm || !aligned4(norm) || on_tensors(out ? out : grads, nullptr, m, norm, sizeof(float))) return PCM_ERR_ARG;
    return from_hip(launch_grad_norm(grads, out, m, true, max_norm, (float*)norm, nullptr, (hipStream_t)stream));
}

pcm_status pcm_clip_grad_norm(const pcm_tensor* grads, const pcm_tensor* out, int m, float max_norm,
                              float* norm, void* ws, size_t ws_bytes, void* stream) {
    pcm_status st = check_clip(grads, out, m, max_norm);
    if (st == PCM_OK) st = check_norm(grads, out, m, norm, ws, ws_bytes);
    if (st != PCM_OK) return st;
    return from_hip(launch_grad_norm(grads, out, m, true, max_norm, norm, (double*)ws, (hipStream_t)stream));
}

}  // extern "C"
