// C ABI of the operators around the experts' weights: argument checks and launches.  No kernels here.
#include <stdio.h>

#include <initializer_list>

#include "moe_ops.h"
#include "moe_overlap.h"

namespace {

constexpr int kMaxRows = 1 << 24, kMaxExperts = 256, kMaxWidth = 1 << 17;
constexpr int64_t kMaxLd = 1 << 21;  // 256 rows of that many values stay inside a 2 GB buffer descriptor

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
// a tensor of `rows` rows: it may be null where there are none
inline bool bad(const void* p, size_t a, int64_t rows) { return (p == nullptr && rows > 0) || !aligned(p, a); }
inline bool bad_ld(int64_t ld, int64_t width, int unit) { return ld < width || ld % unit != 0 || ld > kMaxLd; }
inline bool bad_width(int w, int unit) { return w < unit || w % unit != 0 || w > kMaxWidth; }

moe_status from_hip(hipError_t e) {
    if (e == hipSuccess) return MOE_OK;
    char text[200];
    snprintf(text, sizeof(text), "kernel launch: %s", hipGetErrorString(e));
    moe_note_error(text);
    return MOE_ERR_DEVICE;
}

// rows, experts and widths of a grouped product; `unit`: what K has to be a multiple of
moe_status check_grouped(const int32_t* offsets, int32_t rows, int32_t E, int32_t K, int32_t N, int unit) {
    if (rows < 0 || rows > kMaxRows || E < 1) return MOE_ERR_INVALID_ARG;
    if (offsets == nullptr || !aligned(offsets, 4)) return MOE_ERR_INVALID_ARG;
    if (E > kMaxExperts || bad_width(K, unit) || bad_width(N, 8)) return MOE_ERR_UNSUPPORTED_SHAPE;
    return MOE_OK;
}

// a workspace of at least `need` bytes
moe_status check_workspace(const void* workspace, size_t bytes, size_t need) {
    if (need == 0) return MOE_OK;
    if (bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
    return workspace == nullptr || !aligned(workspace, 16) ? MOE_ERR_INVALID_ARG : MOE_OK;
}

// An output that shares bytes with one of the others: results would depend on which workgroup ran when.
bool over(const Rows& out, std::initializer_list<Rows> others) {
    for (const Rows& o : others)
        if (overlap(out, o)) return true;
    return false;
}

// The same for calls whose lanes read what they need of a place before they write there: an output may be exactly an input.
bool partly_over(const Rows& out, std::initializer_list<Rows> inputs) {
    for (const Rows& i : inputs)
        if (!same_place(out, i) && overlap(out, i)) return true;
    return false;
}

bool grouped_shape_ok(int32_t rows, int32_t E, int32_t K, int32_t N, int unit) {
    return rows >= 0 && rows <= kMaxRows && E >= 1 && E <= kMaxExperts && !bad_width(K, unit) && !bad_width(N, 8);
}

moe_status check_list(const void* const* grads, void* const* outs, bool with_outs, const int64_t* counts, const int32_t* types, int32_t n,
                      const void* workspace, size_t workspace_bytes, const float* norm) {
    if (n < 0 || norm == nullptr || !aligned(norm, 4) || workspace == nullptr || !aligned(workspace, 8)) return MOE_ERR_INVALID_ARG;
    if (n > 0 && (grads == nullptr || counts == nullptr || types == nullptr || (with_outs && outs == nullptr))) return MOE_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n; ++i) {
        if (types[i] != MOE_BF16 && types[i] != MOE_F32) return MOE_ERR_INVALID_ARG;
        const size_t size = types[i] == MOE_F32 ? 4 : 2;
        if (counts[i] < 0 || counts[i] > (int64_t)1 << 38 || bad(grads[i], size, counts[i])) return MOE_ERR_INVALID_ARG;
        if (with_outs && bad(outs[i], size, counts[i])) return MOE_ERR_INVALID_ARG;
    }
    if (workspace_bytes < grad_norm_workspace(n)) return MOE_ERR_WORKSPACE_TOO_SMALL;
    return MOE_OK;
}

}  // namespace

extern "C" {

size_t moe_grouped_gemm_workspace_bytes(int32_t n_rows_cap, int32_t E, int32_t K, int32_t N, int32_t transpose_w) {
    return grouped_shape_ok(n_rows_cap, E, K, N, 8) ? grouped_workspace(grouped_rows_plan(n_rows_cap, E, K * 2, N, transpose_w == 0, false), (int64_t)n_rows_cap * N) : 0;
}

moe_status moe_grouped_gemm(const void* x, int64_t ldx, const void* w, int32_t transpose_w, const int32_t* offsets, int32_t n_rows_cap,
                            int32_t E, int32_t K, int32_t N, void* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    moe_status st = check_grouped(offsets, n_rows_cap, E, K, N, 8);
    if (st != MOE_OK) return st;
    if (bad(x, 16, n_rows_cap) || bad(w, 16, 1) || bad(y, 16, n_rows_cap)) return MOE_ERR_INVALID_ARG;
    if (bad_ld(ldx, K, 8) || bad_ld(ldy, N, 8)) return MOE_ERR_INVALID_ARG;
    if (n_rows_cap == 0) return MOE_OK;
    const GroupedPlan plan = grouped_rows_plan(n_rows_cap, E, K * 2, N, transpose_w == 0, false);
    st = check_workspace(workspace, workspace_bytes, grouped_workspace(plan, (int64_t)n_rows_cap * N));
    if (st != MOE_OK) return st;
    if (over({y, n_rows_cap, ldy * 2, (int64_t)N * 2}, {{x, n_rows_cap, ldx * 2, (int64_t)K * 2}, {w, 1, 0, (int64_t)E * K * N * 2}, {offsets, 1, 0, (E + 1) * 4}}))
        return MOE_ERR_INVALID_ARG;
    return from_hip(launch_grouped_gemm(x, ldx, w, transpose_w != 0, offsets, n_rows_cap, E, K, N, y, ldy, plan, workspace, (hipStream_t)stream));
}

size_t moe_grouped_gemm_wgrad_workspace_bytes(int32_t n_rows_cap, int32_t E, int32_t K, int32_t N) {
    return grouped_shape_ok(n_rows_cap, E, K, N, 8) ? grouped_workspace(grouped_weights_plan(n_rows_cap, E, K, N), (int64_t)E * K * N) : 0;
}

moe_status moe_grouped_gemm_wgrad(const void* x, int64_t ldx, const void* dy, int64_t lddy, const int32_t* offsets, int32_t n_rows_cap,
                                  int32_t E, int32_t K, int32_t N, void* dw, int32_t type, int32_t accumulate, void* workspace,
                                  size_t workspace_bytes, void* stream) {
    moe_status st = check_grouped(offsets, n_rows_cap, E, K, N, 8);
    if (st != MOE_OK) return st;
    if (bad(x, 16, n_rows_cap) || bad(dy, 16, n_rows_cap) || bad(dw, 16, 1)) return MOE_ERR_INVALID_ARG;
    if (bad_ld(ldx, K, 8) || bad_ld(lddy, N, 8)) return MOE_ERR_INVALID_ARG;
    if (type != MOE_BF16 && type != MOE_F32) return MOE_ERR_INVALID_ARG;
    if (accumulate != 0 && type != MOE_F32) return MOE_ERR_INVALID_ARG;
    const GroupedPlan plan = grouped_weights_plan(n_rows_cap, E, K, N);
    st = check_workspace(workspace, workspace_bytes, grouped_workspace(plan, (int64_t)E * K * N));
    if (st != MOE_OK) return st;
    if (over({dw, 1, 0, (int64_t)E * K * N * (type == MOE_F32 ? 4 : 2)},
             {{x, n_rows_cap, ldx * 2, (int64_t)K * 2}, {dy, n_rows_cap, lddy * 2, (int64_t)N * 2}, {offsets, 1, 0, (E + 1) * 4}}))
        return MOE_ERR_INVALID_ARG;
    return from_hip(launch_grouped_wgrad(x, ldx, dy, lddy, offsets, n_rows_cap, E, K, N, dw, type == MOE_F32, accumulate != 0, plan, workspace,
                                         (hipStream_t)stream));
}

moe_status moe_swiglu(const void* gu, int64_t ldgu, const int32_t* n_rows, int32_t n_rows_cap, int32_t f, void* h, int64_t ldh,
                      void* stream) {
    if (n_rows_cap < 0 || n_rows_cap > kMaxRows || !aligned(n_rows, 4)) return MOE_ERR_INVALID_ARG;
    if (bad_width(f, 8)) return MOE_ERR_UNSUPPORTED_SHAPE;
    if (bad(gu, 16, n_rows_cap) || bad(h, 16, n_rows_cap)) return MOE_ERR_INVALID_ARG;
    if (bad_ld(ldgu, 2 * (int64_t)f, 8) || bad_ld(ldh, f, 8)) return MOE_ERR_INVALID_ARG;
    if (n_rows_cap == 0) return MOE_OK;
    const Rows g(gu, n_rows_cap, ldgu * 2, (int64_t)f * 2), u((const char*)gu + (int64_t)f * 2, n_rows_cap, ldgu * 2, (int64_t)f * 2), live(n_rows, 1, 0, 4);
    const Rows out(h, n_rows_cap, ldh * 2, (int64_t)f * 2);
    if (partly_over(out, {g, u}) || over(out, {live})) return MOE_ERR_INVALID_ARG;
    return from_hip(launch_swiglu(gu, ldgu, n_rows, n_rows_cap, f, h, ldh, (hipStream_t)stream));
}

moe_status moe_swiglu_backward(const void* dh, int64_t lddh, const void* gu, int64_t ldgu, const int32_t* n_rows, int32_t n_rows_cap,
                               int32_t f, void* dgu, int64_t lddgu, void* h, int64_t ldh, void* stream) {
    if (n_rows_cap < 0 || n_rows_cap > kMaxRows || !aligned(n_rows, 4)) return MOE_ERR_INVALID_ARG;
    if (bad_width(f, 8)) return MOE_ERR_UNSUPPORTED_SHAPE;
    if (bad(dh, 16, n_rows_cap) || bad(gu, 16, n_rows_cap) || bad(dgu, 16, n_rows_cap) || !aligned(h, 16)) return MOE_ERR_INVALID_ARG;
    if (bad_ld(lddh, f, 8) || bad_ld(ldgu, 2 * (int64_t)f, 8) || bad_ld(lddgu, 2 * (int64_t)f, 8)) return MOE_ERR_INVALID_ARG;
    if (h != nullptr && bad_ld(ldh, f, 8)) return MOE_ERR_INVALID_ARG;
    if (n_rows_cap == 0) return MOE_OK;
    const int64_t n = n_rows_cap, width = (int64_t)f * 2;
    const Rows d(dh, n, lddh * 2, width), g(gu, n, ldgu * 2, width), u((const char*)gu + width, n, ldgu * 2, width), live(n_rows, 1, 0, 4);
    const Rows dg(dgu, n, lddgu * 2, width), du((const char*)dgu + width, n, lddgu * 2, width), again(h, n, ldh * 2, width);
    if (partly_over(dg, {d, g, u}) || partly_over(du, {d, g, u}) || partly_over(again, {d, g, u})) return MOE_ERR_INVALID_ARG;
    if (over(again, {dg, du}) || over(live, {dg, du, again})) return MOE_ERR_INVALID_ARG;
    return from_hip(launch_swiglu_backward(dh, lddh, gu, ldgu, n_rows, n_rows_cap, f, dgu, lddgu, h, ldh, (hipStream_t)stream));
}

size_t moe_grad_norm_workspace_bytes(int32_t n) { return n < 0 ? 0 : grad_norm_workspace(n); }

moe_status moe_grad_norm(const void* const* grads, const int64_t* counts, const int32_t* types, int32_t n, void* workspace,
                         size_t workspace_bytes, float* norm, void* stream) {
    const moe_status st = check_list(grads, nullptr, false, counts, types, n, workspace, workspace_bytes, norm);
    if (st != MOE_OK) return st;
    return from_hip(launch_grad_norm(grads, counts, types, n, (double*)workspace, norm, (hipStream_t)stream));
}

moe_status moe_clip_grad_norm(const void* const* grads, void* const* outs, const int64_t* counts, const int32_t* types, int32_t n,
                              float max_norm, void* workspace, size_t workspace_bytes, float* norm, void* stream) {
    if (!(max_norm >= 0.f)) return MOE_ERR_INVALID_ARG;  // (a NaN too)
    const moe_status st = check_list(grads, outs, true, counts, types, n, workspace, workspace_bytes, norm);
    if (st != MOE_OK) return st;
    return from_hip(launch_clip_grads(grads, outs, counts, types, n, max_norm, (double*)workspace, norm, (hipStream_t)stream));
}

int32_t moe_mxfp4_scale_cols(int32_t K) { return K < 32 || K % 32 != 0 || K > kMaxWidth ? 0 : mx_scale_cols(K); }

moe_status moe_mxfp4_quantize(const void* x, int32_t type, int64_t ldx, const int32_t* n_rows, int32_t n_rows_cap, int32_t K, void* values,
                              void* scales, void* stream) {
    if (n_rows_cap < 0 || n_rows_cap > kMaxRows || !aligned(n_rows, 4)) return MOE_ERR_INVALID_ARG;
    if (type != MOE_BF16 && type != MOE_F32) return MOE_ERR_INVALID_ARG;
    if (bad_width(K, 32)) return MOE_ERR_UNSUPPORTED_SHAPE;
    if (bad(x, 16, n_rows_cap) || bad(values, 16, n_rows_cap) || bad(scales, 16, n_rows_cap)) return MOE_ERR_INVALID_ARG;
    if (bad_ld(ldx, K, type == MOE_F32 ? 4 : 8)) return MOE_ERR_INVALID_ARG;
    if (n_rows_cap == 0) return MOE_OK;
    const Rows q(values, 1, 0, (int64_t)n_rows_cap * (K / 2)), s(scales, 1, 0, (int64_t)n_rows_cap * mx_scale_cols(K));
    const int64_t size = type == MOE_F32 ? 4 : 2;
    if (over(q, {s}) || over({x, n_rows_cap, ldx * size, K * size}, {q, s}) || over({n_rows, 1, 0, 4}, {q, s})) return MOE_ERR_INVALID_ARG;
    return from_hip(launch_mx_quantize(x, type == MOE_F32, ldx, n_rows, n_rows_cap, K, values, scales, (hipStream_t)stream));
}

moe_status moe_mxfp4_quantize_weights(const void* w, int32_t E, int32_t K, int32_t N, void* values, void* scales, void* stream) {
    if (E < 1) return MOE_ERR_INVALID_ARG;
    if (E > kMaxExperts || bad_width(K, 32) || bad_width(N, 8)) return MOE_ERR_UNSUPPORTED_SHAPE;
    if (bad(w, 16, 1) || bad(values, 16, 1) || bad(scales, 16, 1)) return MOE_ERR_INVALID_ARG;
    const Rows q(values, 1, 0, (int64_t)E * N * (K / 2)), s(scales, 1, 0, (int64_t)E * N * mx_scale_cols(K));
    if (over(q, {s}) || over({w, 1, 0, (int64_t)E * K * N * 2}, {q, s})) return MOE_ERR_INVALID_ARG;
    return from_hip(launch_mx_quantize_weights(w, E, K, N, values, scales, (hipStream_t)stream));
}

moe_status moe_mxfp4_dequantize(const void* values, const void* scales, int64_t rows, int32_t K, void* x, int64_t ldx, void* stream) {
    if (rows < 0 || rows > (int64_t)kMaxExperts * kMaxWidth) return MOE_ERR_INVALID_ARG;
    if (bad_width(K, 32)) return MOE_ERR_UNSUPPORTED_SHAPE;
    if (bad(values, 16, rows) || bad(scales, 16, rows) || bad(x, 16, rows) || bad_ld(ldx, K, 8)) return MOE_ERR_INVALID_ARG;
    if (rows == 0) return MOE_OK;
    if (over({x, rows, ldx * 2, (int64_t)K * 2}, {{values, 1, 0, rows * (K / 2)}, {scales, 1, 0, rows * mx_scale_cols(K)}})) return MOE_ERR_INVALID_ARG;
    return from_hip(launch_mx_dequantize(values, scales, rows, K, x, ldx, (hipStream_t)stream));
}

size_t moe_mxfp4_grouped_gemm_workspace_bytes(int32_t n_rows_cap, int32_t E, int32_t K, int32_t N) {
    return grouped_shape_ok(n_rows_cap, E, K, N, 32) ? grouped_workspace(grouped_rows_plan(n_rows_cap, E, K / 2, N, false, true), (int64_t)n_rows_cap * N) : 0;
}

moe_status moe_mxfp4_grouped_gemm(const void* x_values, const void* x_scales, const void* w_values, const void* w_scales,
                                  const int32_t* offsets, int32_t n_rows_cap, int32_t E, int32_t K, int32_t N, void* y, int64_t ldy,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    moe_status st = check_grouped(offsets, n_rows_cap, E, K, N, 32);
    if (st != MOE_OK) return st;
    if (bad(x_values, 16, n_rows_cap) || bad(x_scales, 16, n_rows_cap) || bad(w_values, 16, 1) || bad(w_scales, 16, 1)) return MOE_ERR_INVALID_ARG;
    if (bad(y, 16, n_rows_cap) || bad_ld(ldy, N, 8)) return MOE_ERR_INVALID_ARG;
    if (n_rows_cap == 0) return MOE_OK;
    const GroupedPlan plan = grouped_rows_plan(n_rows_cap, E, K / 2, N, false, true);
    st = check_workspace(workspace, workspace_bytes, grouped_workspace(plan, (int64_t)n_rows_cap * N));
    if (st != MOE_OK) return st;
    const int64_t cols = mx_scale_cols(K);
    if (over({y, n_rows_cap, ldy * 2, (int64_t)N * 2}, {{x_values, 1, 0, (int64_t)n_rows_cap * (K / 2)}, {x_scales, 1, 0, n_rows_cap * cols},
                                                      {w_values, 1, 0, (int64_t)E * N * (K / 2)}, {w_scales, 1, 0, (int64_t)E * N * cols}, {offsets, 1, 0, (E + 1) * 4}}))
        return MOE_ERR_INVALID_ARG;
    return from_hip(launch_grouped_mx(x_values, x_scales, w_values, w_scales, offsets, n_rows_cap, E, K, N, y, ldy, plan, workspace, (hipStream_t)stream));
}

}  // extern "C"
