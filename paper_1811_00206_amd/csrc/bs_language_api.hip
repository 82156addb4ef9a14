// C-ABI entry points of the calls on 4-bit matrices and logits: argument validation on the host, then the launchers.
#include "bs_mx4.h"

namespace bs {

bool rows_meet(const Rows& a, const Rows& b) {
    if (!a.fit() || !b.fit()) return true;
    const int64_t d = (int64_t)(b.at - a.at);
    if (d >= (a.count - 1) * a.pitch + a.bytes || -d >= (b.count - 1) * b.pitch + b.bytes) return false;
    // rows of a to look at: where both are equally far apart the same distances come again, so that one with all b beside it will do
    const auto meets = [&](int64_t i) {
        const int64_t to = i * a.pitch - d, j = to >= 0 ? to / b.pitch : -1;      // the last row of b that starts at or before it
        return (j >= 0 && j < b.count && to - j * b.pitch < b.bytes) || (j + 1 < b.count && (j + 1) * b.pitch - to < a.bytes);
    };
    if (a.pitch == b.pitch && a.count == b.count) return meets(d >= 0 ? a.count - 1 : 0);
    for (int64_t i = 0; i < a.count; ++i)
        if (meets(i)) return true;
    return false;
}

}  // namespace bs

namespace {

constexpr int64_t kMost = (int64_t)1 << 24;      // rows, columns

constexpr int64_t kMostOutputs = (int64_t)1 << 36;      // of an MX product

bool type_ok(int dtype) { return dtype == BS_F32 || dtype == BS_F16 || dtype == BS_BF16; }
bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool matrix_ok(int64_t M, int64_t K) { return M >= 1 && K >= 1; }
bool limits_ok(int64_t M, int64_t K, int group) { return M <= kMost && K <= kMost && bs::q4_group_ok(group); }

int check_codes(const uint8_t* codes, const uint16_t* scales, int64_t M, int64_t K, int group) {
    if (!codes || !scales) return BS_ERR_NULL;
    if (!matrix_ok(M, K)) return BS_ERR_SHAPE;
    if (!limits_ok(M, K, group)) return BS_ERR_UNSUPPORTED;
    return aligned(codes, 16) && aligned(scales, 2) ? BS_OK : BS_ERR_ALIGN;
}

int check_logits(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld, const int64_t* targets) {
    if (!logits || !targets) return BS_ERR_NULL;
    if (T < 1 || V < 1 || ld < V) return BS_ERR_SHAPE;
    if (!type_ok(dtype) || V >= ((int64_t)1 << 31) - 64) return BS_ERR_UNSUPPORTED;
    return aligned(logits, bs::dtype_bytes(dtype)) && aligned(targets, 8) ? BS_OK : BS_ERR_ALIGN;
}

int check_mx4(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K) {
    if (!codes || !scales) return BS_ERR_NULL;
    if (!matrix_ok(M, K)) return BS_ERR_SHAPE;
    if (M > kMost || K > kMost) return BS_ERR_UNSUPPORTED;
    return aligned(codes, 16) && aligned(scales, 4) ? BS_OK : BS_ERR_ALIGN;
}

bool aligned4(const void* a, const void* b, const void* c, const void* d) {
    return aligned(a, 4) && aligned(b, 4) && aligned(c, 4) && aligned(d, 4);
}

using bs::mx4_codes_place;
using bs::mx4_scales_place;
using bs::Rows;
using bs::rows_meet;

}  // namespace

extern "C" {

size_t bs_q4_codes_bytes(int64_t M, int64_t K) {
    return matrix_ok(M, K) && limits_ok(M, K, 32) ? (size_t)M * bs::q4_row_bytes(K) : 0;
}

size_t bs_q4_scales_bytes(int64_t M, int64_t K, int group) {
    return matrix_ok(M, K) && limits_ok(M, K, group) ? (size_t)M * bs::q4_groups(K, group) * 2 : 0;
}

int bs_q4_pack(const void* W, int dtype, int64_t M, int64_t K, int group, uint8_t* codes, uint16_t* scales, void* stream) {
    if (!W) return BS_ERR_NULL;
    const int st = check_codes(codes, scales, M, K, group);
    if (st) return st;
    if (!type_ok(dtype)) return BS_ERR_UNSUPPORTED;
    if (!aligned(W, bs::dtype_bytes(dtype))) return BS_ERR_ALIGN;
    return bs::launch_q4_pack(W, dtype, M, K, group, codes, scales, nullptr, static_cast<hipStream_t>(stream));
}

int bs_q4_unpack(const uint8_t* codes, const uint16_t* scales, int64_t M, int64_t K, int group, void* W, int dtype, void* stream) {
    if (!W) return BS_ERR_NULL;
    const int st = check_codes(codes, scales, M, K, group);
    if (st) return st;
    if (!type_ok(dtype)) return BS_ERR_UNSUPPORTED;
    if (!aligned(W, bs::dtype_bytes(dtype))) return BS_ERR_ALIGN;
    return bs::launch_q4_pack(nullptr, dtype, M, K, group, const_cast<uint8_t*>(codes), const_cast<uint16_t*>(scales), W,
                              static_cast<hipStream_t>(stream));
}

size_t bs_q4_gemv_workspace_bytes(int dtype, int64_t M, int64_t K, int group, int64_t N) {
    if (!matrix_ok(M, K) || !limits_ok(M, K, group) || !type_ok(dtype) || N < 1 || N > 65535) return 0;
    return bs::q4_gemv_workspace_bytes(dtype, M, K, N);
}

int bs_q4_gemv(const uint8_t* codes, const uint16_t* scales, int64_t M, int64_t K, int group, const void* x, int dtype, int64_t N,
               int64_t ldx, void* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x || !y) return BS_ERR_NULL;
    const int st = check_codes(codes, scales, M, K, group);
    if (st) return st;
    if (N < 1 || ldx < K || ldy < M) return BS_ERR_SHAPE;
    if (!type_ok(dtype) || N > 65535) return BS_ERR_UNSUPPORTED;
    const size_t size = bs::dtype_bytes(dtype);
    if (!aligned(x, size) || !aligned(y, size)) return BS_ERR_ALIGN;
    return bs::launch_q4_gemv(codes, scales, M, K, group, x, dtype, N, ldx, y, ldy, workspace, workspace_bytes,
                              static_cast<hipStream_t>(stream));
}

size_t bs_q4_moe_workspace_bytes(int dtype, int64_t T, int64_t D, int64_t F, int E, int top_k, int group) {
    if (T < 1 || T > BS_MOE_TOKENS_MAX || !matrix_ok(D, F) || F > kMost / 2 || !limits_ok(D, F, group) || !type_ok(dtype)) return 0;
    if (E < 1 || E > BS_MOE_EXPERTS_MAX || top_k < 1 || top_k > E || top_k > BS_MOE_TOP_K_MAX) return 0;
    return bs::q4_moe_workspace_bytes(dtype, T, D, F, E, top_k);
}

int bs_q4_moe(const void* x, int dtype, int64_t T, int64_t ldx, int64_t D, const void* router, int E, const uint8_t* w1,
              const uint16_t* s1, const uint8_t* w2, const uint16_t* s2, int64_t F, int group, int top_k, int renormalise, void* y,
              int64_t ldy, int32_t* ids, float* weights, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x || !router || !w1 || !s1 || !w2 || !s2 || !y || !ids || !weights) return BS_ERR_NULL;
    if (T < 1 || !matrix_ok(D, F) || E < 1 || top_k < 1 || top_k > E || ldx < D || ldy < D) return BS_ERR_SHAPE;
    if (!type_ok(dtype) || T > BS_MOE_TOKENS_MAX || E > BS_MOE_EXPERTS_MAX || top_k > BS_MOE_TOP_K_MAX || F > kMost / 2 ||
        !limits_ok(D, F, group))
        return BS_ERR_UNSUPPORTED;
    const size_t size = bs::dtype_bytes(dtype);
    if (!aligned(x, size) || !aligned(router, size) || !aligned(y, size) || !aligned(w1, 16) || !aligned(w2, 16) ||
        !aligned(s1, 2) || !aligned(s2, 2) || !aligned(ids, 4) || !aligned(weights, 4))
        return BS_ERR_ALIGN;
    return bs::launch_q4_moe(x, dtype, T, ldx, D, router, E, w1, s1, w2, s2, F, group, top_k, renormalise, y, ldy, ids, weights,
                             workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

size_t bs_logprobs_workspace_bytes(int dtype, int64_t T, int64_t V, int top_n) {
    if (T < 1 || V < 1 || V >= ((int64_t)1 << 31) - 64 || !type_ok(dtype) || top_n < 0 || top_n > V || top_n > BS_LOGPROBS_TOP_MAX)
        return 0;
    return bs::logprobs_workspace_bytes(dtype, T, V, top_n);
}

int bs_logprobs(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld, const int64_t* targets, int top_n, float* logprob,
                float* entropy, float* lse, float* top_values, int32_t* top_ids, void* workspace, size_t workspace_bytes,
                void* stream) {
    if (!logprob || !entropy || !lse || (top_n > 0 && (!top_values || !top_ids))) return BS_ERR_NULL;
    const int st = check_logits(logits, dtype, T, V, ld, targets);
    if (st) return st;
    if (top_n < 0 || top_n > V) return BS_ERR_SHAPE;
    if (top_n > BS_LOGPROBS_TOP_MAX) return BS_ERR_UNSUPPORTED;
    if (!aligned4(logprob, entropy, lse, top_values) || !aligned(top_ids, 4)) return BS_ERR_ALIGN;
    return bs::launch_logprobs(logits, dtype, T, V, ld, targets, top_n, logprob, entropy, lse, top_values, top_ids, workspace,
                               workspace_bytes, static_cast<hipStream_t>(stream));
}

int bs_logprobs_backward(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld, const int64_t* targets, const float* lse,
                         const float* entropy, const float* g_logprob, const float* g_entropy, void* grad, int64_t ldg, void* stream) {
    if (!lse || !g_logprob || !grad || !entropy != !g_entropy) return BS_ERR_NULL;
    const int st = check_logits(logits, dtype, T, V, ld, targets);
    if (st) return st;
    if (ldg < V) return BS_ERR_SHAPE;
    const int64_t size = bs::dtype_bytes(dtype);
    if (!aligned(grad, size)) return BS_ERR_ALIGN;
    if ((grad != logits || ldg != ld) && rows_meet(Rows(logits, T, V, ld, size), Rows(grad, T, V, ldg, size))) return BS_ERR_UNSUPPORTED;
    if (!aligned4(lse, entropy, g_logprob, g_entropy)) return BS_ERR_ALIGN;
    return bs::launch_logprobs_backward(logits, dtype, T, V, ld, targets, lse, entropy, g_logprob, g_entropy, grad, ldg,
                                        static_cast<hipStream_t>(stream));
}

size_t bs_mx4_codes_bytes(int64_t M, int64_t K) {
    return matrix_ok(M, K) && M <= kMost && K <= kMost ? (size_t)M * bs::mx4_row_bytes(K) : 0;
}

size_t bs_mx4_scales_bytes(int64_t M, int64_t K) {
    return matrix_ok(M, K) && M <= kMost && K <= kMost ? (size_t)M * bs::mx4_scale_pitch(K) : 0;
}

int bs_mx4_pack(const void* W, int dtype, int64_t M, int64_t K, int64_t ld, uint8_t* codes, uint8_t* scales, void* stream) {
    if (!W) return BS_ERR_NULL;
    const int st = check_mx4(codes, scales, M, K);
    if (st) return st;
    if (ld < K) return BS_ERR_SHAPE;
    if (!type_ok(dtype)) return BS_ERR_UNSUPPORTED;
    if (!aligned(W, bs::dtype_bytes(dtype))) return BS_ERR_ALIGN;
    const Rows from(W, M, K, ld, bs::dtype_bytes(dtype)), c = mx4_codes_place(codes, M, K), sc = mx4_scales_place(scales, M, K);
    if (rows_meet(c, from) || rows_meet(sc, from) || rows_meet(c, sc)) return BS_ERR_UNSUPPORTED;
    return bs::launch_mx4_pack(W, dtype, M, K, ld, codes, scales, static_cast<hipStream_t>(stream));
}

int bs_mx4_unpack(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K, void* W, int dtype, void* stream) {
    if (!W) return BS_ERR_NULL;
    const int st = check_mx4(codes, scales, M, K);
    if (st) return st;
    if (!type_ok(dtype)) return BS_ERR_UNSUPPORTED;
    if (!aligned(W, bs::dtype_bytes(dtype))) return BS_ERR_ALIGN;
    const Rows to(W, 1, M * K, 0, bs::dtype_bytes(dtype));
    if (rows_meet(mx4_codes_place(codes, M, K), to) || rows_meet(mx4_scales_place(scales, M, K), to)) return BS_ERR_UNSUPPORTED;
    return bs::launch_mx4_unpack(codes, scales, M, K, W, dtype, static_cast<hipStream_t>(stream));
}

size_t bs_mx4_gemm_workspace_bytes(int dtype, int64_t M, int64_t K, int64_t N) {
    if (!matrix_ok(M, K) || M > kMost || K > kMost || !type_ok(dtype) || N < 1 || N > kMost || M * N > kMostOutputs) return 0;
    return bs::mx4_gemm_workspace_bytes(false, M, K, N);
}

size_t bs_mx4_gemm_packed_workspace_bytes(int dtype, int64_t M, int64_t K, int64_t N) {
    if (!matrix_ok(M, K) || M > kMost || K > kMost || !type_ok(dtype) || N < 1 || N > kMost || M * N > kMostOutputs) return 0;
    return bs::mx4_gemm_workspace_bytes(true, M, K, N);
}

int bs_mx4_gemm(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K, const void* x, int dtype, int64_t N, int64_t ldx,
                const float* bias, void* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x || !y) return BS_ERR_NULL;
    const int st = check_mx4(codes, scales, M, K);
    if (st) return st;
    if (N < 1 || ldx < K || ldy < M) return BS_ERR_SHAPE;
    if (!type_ok(dtype) || N > kMost || M * N > kMostOutputs) return BS_ERR_UNSUPPORTED;
    const size_t size = bs::dtype_bytes(dtype);
    if (!aligned(x, size) || !aligned(y, size) || !aligned(bias, 4)) return BS_ERR_ALIGN;
    if (rows_meet(Rows(x, N, K, ldx, size), Rows(y, N, M, ldy, size))) return BS_ERR_UNSUPPORTED;
    return bs::launch_mx4_gemm(codes, scales, M, K, x, ldx, nullptr, nullptr, dtype, N, bias, y, ldy, workspace, workspace_bytes,
                               static_cast<hipStream_t>(stream));
}

int bs_mx4_gemm_packed(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K, const uint8_t* x_codes,
                       const uint8_t* x_scales, int64_t N, const float* bias, void* y, int dtype, int64_t ldy, void* workspace,
                       size_t workspace_bytes, void* stream) {
    if (!y) return BS_ERR_NULL;
    int st = check_mx4(codes, scales, M, K);
    if (st) return st;
    st = check_mx4(x_codes, x_scales, N, K);
    if (st) return st;
    if (ldy < M) return BS_ERR_SHAPE;
    if (!type_ok(dtype) || M * N > kMostOutputs) return BS_ERR_UNSUPPORTED;
    if (!aligned(y, bs::dtype_bytes(dtype)) || !aligned(bias, 4)) return BS_ERR_ALIGN;
    return bs::launch_mx4_gemm(codes, scales, M, K, nullptr, 0, x_codes, x_scales, dtype, N, bias, y, ldy, workspace, workspace_bytes,
                               static_cast<hipStream_t>(stream));
}

int bs_mx4_gemm_plan(int64_t M, int64_t K, int64_t N, int64_t* out, int n_out) {
    if (!out) return BS_ERR_NULL;
    if (!matrix_ok(M, K) || N < 1 || n_out < 1) return BS_ERR_SHAPE;
    if (M > kMost || K > kMost || N > kMost || M * N > kMostOutputs) return BS_ERR_UNSUPPORTED;
    bs::mx4_gemm_plan_describe(M, K, N, out, n_out);
    return BS_OK;
}

size_t bs_beam_step_workspace_bytes(int dtype, int64_t B, int W, int64_t V, int n) {
    if (B < 1 || B > kMost || W < 1 || W > BS_BEAM_WIDTH_MAX || n < 1 || n > BS_BEAM_WIDTH_MAX || V < 1 ||
        V >= ((int64_t)1 << 31) - 64 || !type_ok(dtype))
        return 0;
    return bs::beam_step_workspace_bytes(dtype, B, W, V, n);
}

int bs_beam_step(const void* logits, int dtype, int64_t B, int W, int64_t V, int64_t ld, const float* scores, const uint8_t* finished,
                 int64_t end, int n, float* out_scores, int32_t* out_tokens, int32_t* out_parents, uint8_t* out_finished,
                 void* workspace, size_t workspace_bytes, void* stream) {
    if (!logits || !scores || !out_scores || !out_tokens || !out_parents || !out_finished) return BS_ERR_NULL;
    if (B < 1 || W < 1 || V < 1 || n < 1 || ld < V || end >= V) return BS_ERR_SHAPE;
    if (!type_ok(dtype) || B > kMost || W > BS_BEAM_WIDTH_MAX || n > BS_BEAM_WIDTH_MAX || V >= ((int64_t)1 << 31) - 64)
        return BS_ERR_UNSUPPORTED;
    if (!aligned(logits, bs::dtype_bytes(dtype)) || !aligned4(scores, out_scores, out_tokens, out_parents)) return BS_ERR_ALIGN;
    return bs::launch_beam_step(logits, dtype, B, W, V, ld, scores, finished, end < 0 ? -1 : end, n, out_scores, out_tokens, out_parents,
                                out_finished, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

int bs_beam_reorder(int count, const void* const* states, void* const* outs, const int64_t* row_bytes, const int64_t* pitch,
                    const int64_t* out_pitch, int64_t B, int W, const int32_t* parents, void* stream) {
    if (!states || !outs || !row_bytes || !pitch || !out_pitch || !parents) return BS_ERR_NULL;
    if (count < 1 || B < 1 || W < 1) return BS_ERR_SHAPE;
    if (count > BS_REORDER_STATES_MAX || W > BS_BEAM_WIDTH_MAX || B > kMost) return BS_ERR_UNSUPPORTED;
    constexpr int64_t kMostBytes = (int64_t)1 << 30;      // of a beam, all its states
    int64_t bytes = 0;
    for (int i = 0; i < count; ++i) {
        if (!states[i] || !outs[i]) return BS_ERR_NULL;
        if (row_bytes[i] < 1 || pitch[i] < row_bytes[i] || out_pitch[i] < row_bytes[i]) return BS_ERR_SHAPE;
        if (row_bytes[i] > kMostBytes - bytes || pitch[i] >= (int64_t)1 << 32 || out_pitch[i] >= (int64_t)1 << 32) return BS_ERR_UNSUPPORTED;
        bytes += row_bytes[i];
    }
    if (!aligned(parents, 4)) return BS_ERR_ALIGN;
    const Rows chosen(parents, 1, B * W, B * W, 4);
    for (int i = 0; i < count; ++i) {
        const Rows out(outs[i], B * W, row_bytes[i], out_pitch[i], 1);
        if (rows_meet(chosen, out)) return BS_ERR_UNSUPPORTED;
        for (int j = 0; j < count; ++j) {
            const bool itself = i == j && states[j] == outs[i] && pitch[j] == out_pitch[i];
            if (!itself && rows_meet(Rows(states[j], B * W, row_bytes[j], pitch[j], 1), out)) return BS_ERR_UNSUPPORTED;
            if (j < i && rows_meet(Rows(outs[j], B * W, row_bytes[j], out_pitch[j], 1), out)) return BS_ERR_UNSUPPORTED;
        }
    }
    return bs::launch_beam_reorder(count, states, outs, row_bytes, pitch, out_pitch, B, W, parents, static_cast<hipStream_t>(stream));
}

}  // extern "C"
