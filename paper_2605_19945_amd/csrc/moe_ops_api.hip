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

// ---- norms around a block ----
inline bool type_ok(int32_t t) { return t == MOE_BF16 || t == MOE_F32; }
inline int64_t size_of(int32_t t) { return t == MOE_F32 ? 4 : 2; }
inline bool bad_rows(const void* p, int64_t rows, int64_t ld, int64_t d, int32_t type) { return bad(p, 16, rows) || bad_ld(ld, d, type == MOE_F32 ? 4 : 8); }

moe_status check_norm(int32_t x_type, int32_t y_type, const void* w, const void* w_next, int32_t w_type, float eps, const int32_t* n_rows, int32_t rows, int32_t d) {
    if (rows < 0 || rows > kMaxRows || !aligned(n_rows, 4) || !(eps >= 0.f) || eps > 3e38f) return MOE_ERR_INVALID_ARG;
    if (!type_ok(x_type) || !type_ok(y_type) || (x_type == MOE_BF16 && y_type == MOE_F32)) return MOE_ERR_INVALID_ARG;
    if ((w != nullptr || w_next != nullptr) && !type_ok(w_type)) return MOE_ERR_INVALID_ARG;
    if (!aligned(w, 16) || !aligned(w_next, 16)) return MOE_ERR_INVALID_ARG;
    return d < 8 || d % 8 != 0 || d > NORM_MAX_WIDTH ? MOE_ERR_UNSUPPORTED_SHAPE : MOE_OK;
}

// ---- orthogonalised updates ----
// Two stacks of E matrices that share bytes
bool stacks_overlap(const char* a, int64_t a_matrix, int64_t a_ld, int64_t a_width, const char* b, int64_t b_matrix, int64_t b_ld, int64_t b_width, int E, int rows) {
    const Rows whole_a(a, 1, 0, (E - 1) * a_matrix + (rows - 1) * a_ld + a_width), whole_b(b, 1, 0, (E - 1) * b_matrix + (rows - 1) * b_ld + b_width);
    if (!overlap(whole_a, whole_b)) return false;
    for (int i = 0; i < E; ++i)
        for (int j = 0; j < E; ++j)
            if (overlap({a + i * a_matrix, rows, a_ld, a_width}, {b + j * b_matrix, rows, b_ld, b_width})) return true;
    return false;
}
inline bool orth_shape_ok(int32_t E, int32_t rows, int32_t cols) {
    return E >= 1 && E <= kMaxExperts && rows >= 1 && rows <= kMaxWidth && cols >= 1 && cols <= kMaxWidth && (int64_t)rows * cols <= (int64_t)1 << 29;
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

moe_status moe_rms_norm(const void* x, int32_t x_type, int64_t ldx, const void* w, int32_t w_type, float eps, const int32_t* n_rows,
                        int32_t n_rows_cap, int32_t d, void* h, int32_t h_type, int64_t ldh, void* stream) {
    const moe_status st = check_norm(x_type, h_type, w, nullptr, w_type, eps, n_rows, n_rows_cap, d);
    if (st != MOE_OK) return st;
    const int64_t n = n_rows_cap;
    if (bad_rows(x, n, ldx, d, x_type) || bad_rows(h, n, ldh, d, h_type)) return MOE_ERR_INVALID_ARG;
    if (n == 0) return MOE_OK;
    const Rows out(h, n, ldh * size_of(h_type), d * size_of(h_type));
    if (partly_over(out, {{x, n, ldx * size_of(x_type), d * size_of(x_type)}}) || over(out, {{w, 1, 0, d * size_of(w_type)}, {n_rows, 1, 0, 4}})) return MOE_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = x, a.ldx = ldx, a.w_next = w, a.h = h, a.ldh = ldh, a.n_rows = n_rows, a.rows = n_rows_cap, a.d = d, a.eps = eps, a.scale = 1.f;
    a.x_f32 = x_type == MOE_F32, a.y_f32 = h_type == MOE_F32, a.w_f32 = w_type == MOE_F32;
    return from_hip(launch_norm(a, (hipStream_t)stream));
}

size_t moe_norm_backward_workspace_bytes(int32_t n_rows_cap, int32_t d) {
    if (n_rows_cap < 0 || n_rows_cap > kMaxRows || d < 8 || d % 8 != 0 || d > NORM_MAX_WIDTH) return 0;
    return (size_t)norm_grad_groups(n_rows_cap, d) * d * 4 * 2;
}

moe_status moe_rms_norm_backward(const void* dh, int32_t h_type, int64_t lddh, const void* x, int32_t x_type, int64_t ldx, const void* w,
                                 int32_t w_type, float eps, const void* dres, int64_t lddres, const int32_t* n_rows, int32_t n_rows_cap,
                                 int32_t d, void* dx, int64_t lddx, float* dw, void* workspace, size_t workspace_bytes, void* stream) {
    moe_status st = check_norm(x_type, h_type, w, nullptr, w_type, eps, n_rows, n_rows_cap, d);
    if (st != MOE_OK) return st;
    const int64_t n = n_rows_cap, xs = size_of(x_type), hs = size_of(h_type);
    if (bad_rows(dh, n, lddh, d, h_type) || bad_rows(x, n, ldx, d, x_type) || bad_rows(dx, n, lddx, d, x_type) || !aligned(dw, 16)) return MOE_ERR_INVALID_ARG;
    if (dres != nullptr && bad_rows(dres, n, lddres, d, x_type)) return MOE_ERR_INVALID_ARG;
    if (n == 0 && dw == nullptr) return MOE_OK;
    const size_t need = dw != nullptr ? moe_norm_backward_workspace_bytes(n_rows_cap, d) : 0;
    st = check_workspace(workspace, workspace_bytes, need);
    if (st != MOE_OK) return st;
    const Rows rh(dh, n, lddh * hs, d * hs), rx(x, n, ldx * xs, d * xs), rr(dres, n, lddres * xs, d * xs), out(dx, n, lddx * xs, d * xs);
    const Rows rw(w, 1, 0, d * size_of(w_type)), live(n_rows, 1, 0, 4), rdw(dw, 1, 0, (int64_t)d * 4), ws(need > 0 ? workspace : nullptr, 1, 0, (int64_t)need);
    if (partly_over(out, {rh, rx, rr}) || over(out, {rw, live}) || over(rdw, {rh, rx, rr, out, rw, live}) || over(ws, {rh, rx, rr, out, rw, live, rdw})) return MOE_ERR_INVALID_ARG;
    NormGradArgs a = {};
    a.dout = dres, a.lddout = lddres, a.dh = dh, a.lddh = lddh, a.o = x, a.ldo = ldx, a.w_next = w, a.dx = dx, a.lddx = lddx, a.n_rows = n_rows;
    a.rows = n_rows_cap, a.d = d, a.eps = eps, a.scale = 1.f, a.x_f32 = x_type == MOE_F32, a.y_f32 = h_type == MOE_F32, a.w_f32 = w_type == MOE_F32;
    return from_hip(launch_norm_backward(a, nullptr, dw, (float*)workspace, (hipStream_t)stream));
}

moe_status moe_residual_norm(const void* x, int32_t x_type, int64_t ldx, const void* y, int32_t y_type, int64_t ldy, const void* w,
                             int32_t w_type, int32_t norm, const void* gate, int64_t ldgate, float scale, const void* w_next, float eps,
                             const int32_t* n_rows, int32_t n_rows_cap, int32_t d, void* out, int64_t ldout, void* h, int64_t ldh,
                             void* stream) {
    const moe_status st = check_norm(x_type, y_type, w, w_next, w_type, eps, n_rows, n_rows_cap, d);
    if (st != MOE_OK) return st;
    const int64_t n = n_rows_cap, xs = size_of(x_type), ys = size_of(y_type);
    if (bad_rows(x, n, ldx, d, x_type) || bad_rows(y, n, ldy, d, y_type) || bad_rows(out, n, ldout, d, x_type)) return MOE_ERR_INVALID_ARG;
    if (h != nullptr ? bad_rows(h, n, ldh, d, y_type) : w_next != nullptr && n > 0) return MOE_ERR_INVALID_ARG;
    if (gate == nullptr ? ldgate != 0 : ldgate != 0 ? bad_rows(gate, n, ldgate, d, y_type) : !aligned(gate, 4)) return MOE_ERR_INVALID_ARG;
    if (n == 0) return MOE_OK;
    const Rows rx(x, n, ldx * xs, d * xs), ry(y, n, ldy * ys, d * ys), full(ldgate != 0 ? gate : nullptr, n, ldgate * ys, d * ys);
    const Rows each(ldgate == 0 ? gate : nullptr, 1, 0, n * 4), rw(w, 1, 0, d * size_of(w_type)), rn(w_next, 1, 0, d * size_of(w_type)), live(n_rows, 1, 0, 4);
    const Rows ro(out, n, ldout * xs, d * xs), rh(h, n, ldh * ys, d * ys);
    if (partly_over(ro, {rx, ry, full}) || over(ro, {each, rw, rn, live, rh}) || partly_over(rh, {rx, ry, full}) || over(rh, {each, rw, rn, live})) return MOE_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = x, a.ldx = ldx, a.y = y, a.ldy = ldy, a.w = w, a.w_next = w_next, a.gate = gate, a.ldgate = ldgate, a.out = out, a.ldout = ldout, a.h = h, a.ldh = ldh;
    a.n_rows = n_rows, a.rows = n_rows_cap, a.d = d, a.scale = scale, a.eps = eps, a.norm = norm != 0;
    a.x_f32 = x_type == MOE_F32, a.y_f32 = y_type == MOE_F32, a.w_f32 = w_type == MOE_F32;
    return from_hip(launch_norm(a, (hipStream_t)stream));
}

moe_status moe_residual_norm_backward(const void* dout, int64_t lddout, const void* dh, int64_t lddh, const void* out, int32_t x_type,
                                      int64_t ldout, const void* y, int32_t y_type, int64_t ldy, const void* w, int32_t w_type, int32_t norm,
                                      const void* gate, int64_t ldgate, float scale, const void* w_next, float eps, const int32_t* n_rows,
                                      int32_t n_rows_cap, int32_t d, void* dx, int64_t lddx, void* dy, int64_t lddy, void* dgate,
                                      int64_t lddgate, float* dw, float* dw_next, void* workspace, size_t workspace_bytes, void* stream) {
    moe_status st = check_norm(x_type, y_type, w, w_next, w_type, eps, n_rows, n_rows_cap, d);
    if (st != MOE_OK) return st;
    const int64_t n = n_rows_cap, xs = size_of(x_type), ys = size_of(y_type);
    if (dout != nullptr && bad_rows(dout, n, lddout, d, x_type)) return MOE_ERR_INVALID_ARG;
    if (dh != nullptr ? bad_rows(dh, n, lddh, d, y_type) || bad_rows(out, n, ldout, d, x_type) : n > 0 && (w_next != nullptr || dw_next != nullptr)) return MOE_ERR_INVALID_ARG;
    if (bad_rows(y, n, ldy, d, y_type) || bad_rows(dx, n, lddx, d, x_type) || bad_rows(dy, n, lddy, d, y_type)) return MOE_ERR_INVALID_ARG;
    if (gate == nullptr ? ldgate != 0 || dgate != nullptr : ldgate != 0 ? bad_rows(gate, n, ldgate, d, y_type) : !aligned(gate, 4)) return MOE_ERR_INVALID_ARG;
    if (dgate != nullptr && (ldgate != 0 ? bad_rows(dgate, n, lddgate, d, y_type) : !aligned(dgate, 4))) return MOE_ERR_INVALID_ARG;
    if (!aligned(dw, 16) || !aligned(dw_next, 16)) return MOE_ERR_INVALID_ARG;
    if (n == 0 && dw == nullptr && dw_next == nullptr) return MOE_OK;
    const size_t need = dw != nullptr || dw_next != nullptr ? moe_norm_backward_workspace_bytes(n_rows_cap, d) : 0;
    st = check_workspace(workspace, workspace_bytes, need);
    if (st != MOE_OK) return st;
    const void* o = dh != nullptr ? out : nullptr;
    const Rows rd(dout, n, lddout * xs, d * xs), rh(dh, n, lddh * ys, d * ys), ro(o, n, ldout * xs, d * xs), ry(y, n, ldy * ys, d * ys);
    const Rows full(ldgate != 0 ? gate : nullptr, n, ldgate * ys, d * ys), each(ldgate == 0 ? gate : nullptr, 1, 0, n * 4);
    const Rows rw(w, 1, 0, d * size_of(w_type)), rn(w_next, 1, 0, d * size_of(w_type)), live(n_rows, 1, 0, 4);
    const Rows gx(dx, n, lddx * xs, d * xs), gy(dy, n, lddy * ys, d * ys), gf(ldgate != 0 ? dgate : nullptr, n, lddgate * ys, d * ys);
    const Rows ge(ldgate == 0 ? dgate : nullptr, 1, 0, n * 4), gw(dw, 1, 0, (int64_t)d * 4), gn(dw_next, 1, 0, (int64_t)d * 4), ws(need > 0 ? workspace : nullptr, 1, 0, (int64_t)need);
    for (const Rows* g : {&gx, &gy, &gf})
        if (partly_over(*g, {rd, rh, ro, ry, full}) || over(*g, {each, rw, rn, live, ge, gw, gn, ws})) return MOE_ERR_INVALID_ARG;
    if (over(gx, {gy, gf}) || over(gy, {gf}) || over(gw, {gn})) return MOE_ERR_INVALID_ARG;
    for (const Rows* g : {&ge, &gw, &gn, &ws})
        if (over(*g, {rd, rh, ro, ry, full, each, rw, rn, live})) return MOE_ERR_INVALID_ARG;
    if (over(ge, {gw, gn, ws}) || over(ws, {gw, gn})) return MOE_ERR_INVALID_ARG;
    NormGradArgs a = {};
    a.dout = dout, a.lddout = lddout, a.dh = dh, a.lddh = lddh, a.o = o, a.ldo = ldout, a.y = y, a.ldy = ldy, a.w = w, a.w_next = w_next, a.gate = gate, a.ldgate = ldgate;
    a.dx = dx, a.lddx = lddx, a.dy = dy, a.lddy = lddy, a.dgate = dgate, a.lddgate = lddgate, a.n_rows = n_rows, a.rows = n_rows_cap, a.d = d;
    a.scale = scale, a.eps = eps, a.norm = norm != 0, a.x_f32 = x_type == MOE_F32, a.y_f32 = y_type == MOE_F32, a.w_f32 = w_type == MOE_F32;
    return from_hip(launch_norm_backward(a, dw, dw_next, (float*)workspace, (hipStream_t)stream));
}

size_t moe_orthogonalize_workspace_bytes(int32_t E, int32_t rows, int32_t cols) { return orth_shape_ok(E, rows, cols) ? orth_workspace(E, rows, cols) : 0; }

moe_status moe_orthogonalize(const void* g, int32_t type, int64_t stride_g, int64_t ldg, int32_t E, int32_t rows, int32_t cols,
                             const float* coefficients, int32_t steps, float eps, float scale, void* out, int32_t out_type,
                             int64_t stride_out, int64_t ldout, void* workspace, size_t workspace_bytes, void* stream) {
    if (E < 1 || rows < 1 || cols < 1 || !type_ok(type) || !type_ok(out_type)) return MOE_ERR_INVALID_ARG;
    if (!orth_shape_ok(E, rows, cols)) return MOE_ERR_UNSUPPORTED_SHAPE;
    if (g == nullptr || out == nullptr || !aligned(g, size_of(type)) || !aligned(out, size_of(out_type))) return MOE_ERR_INVALID_ARG;
    if (coefficients == nullptr || steps < 1 || steps > ORTH_MAX_STEPS || !(eps >= 0.f) || eps > 3e38f || !(scale >= -3e38f && scale <= 3e38f)) return MOE_ERR_INVALID_ARG;
    for (int32_t i = 0; i < 3 * steps; ++i)
        if (const float most = i % 3 == 0 ? ORTH_MOST_A : 1e6f; !(coefficients[i] >= -most && coefficients[i] <= most)) return MOE_ERR_INVALID_ARG;
    const int64_t most = (int64_t)1 << 40;
    if (ldg < cols || ldout < cols || ldg > kMaxLd || ldout > kMaxLd) return MOE_ERR_INVALID_ARG;
    // matrices of a stack lie one behind the other, or side by side in the same rows
    auto apart = [&](int64_t stride, int64_t ld) { return E == 1 || (stride <= most && (stride >= (rows - 1) * ld + cols || (stride >= cols && (E - 1) * stride + cols <= ld))); };
    if (!apart(stride_g, ldg) || !apart(stride_out, ldout)) return MOE_ERR_INVALID_ARG;
    const size_t need = orth_workspace(E, rows, cols);
    if (workspace_bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
    if (workspace == nullptr || !aligned(workspace, 256)) return MOE_ERR_INVALID_ARG;
    if (E == 1) stride_g = stride_out = 0;
    const int64_t gs = size_of(type), os = size_of(out_type);
    const bool same = g == out && type == out_type && stride_g == stride_out && (rows == 1 || ldg == ldout);
    if (!same && stacks_overlap((const char*)g, stride_g * gs, ldg * gs, cols * gs, (const char*)out, stride_out * os, ldout * os, cols * os, E, rows)) return MOE_ERR_INVALID_ARG;
    const Rows ws(workspace, 1, 0, (int64_t)need);
    for (int32_t e = 0; e < E; ++e)
        if (over(ws, {{(const char*)g + e * stride_g * gs, rows, ldg * gs, cols * gs}, {(const char*)out + e * stride_out * os, rows, ldout * os, cols * os}})) return MOE_ERR_INVALID_ARG;
    OrthTask t = {};
    t.g = g, t.out = out, t.g_matrix = stride_g, t.g_ld = ldg, t.out_matrix = stride_out, t.out_ld = ldout, t.E = E, t.rows = rows, t.cols = cols;
    t.steps = steps, t.coefficients = coefficients, t.scale = scale, t.eps = eps, t.in_f32 = type == MOE_F32, t.out_f32 = out_type == MOE_F32;
    return from_hip(launch_orth(t, workspace, (hipStream_t)stream));
}

}  // extern "C"
