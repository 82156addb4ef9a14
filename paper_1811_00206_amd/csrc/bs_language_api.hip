// C-ABI entry points of the calls on 4-bit matrices and logits: argument validation on the host, then the launchers.
#include "bs_q4.h"

namespace {

constexpr int64_t kMost = (int64_t)1 << 24;      // rows, columns

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

bool aligned4(const void* a, const void* b, const void* c, const void* d) {
    return aligned(a, 4) && aligned(b, 4) && aligned(c, 4) && aligned(d, 4);
}

// Whether a row at a + i * pa and one at b + j * pb, of n bytes each, share any: rows of one tensor do not, and n <= pa, pb.
bool rows_meet(uintptr_t a, int64_t pa, uintptr_t b, int64_t pb, int64_t rows, int64_t n) {
    const int64_t d = (int64_t)(b - a);
    if (d >= (rows - 1) * pa + n || -d >= (rows - 1) * pb + n) return false;
    // rows of a to look at: where both are equally far apart the same distances come again, so that one with all b beside it will do
    const auto meets = [&](int64_t i) {
        const int64_t to = i * pa - d, j = to >= 0 ? to / pb : -1;      // the last row of b that starts at or before it
        return (j >= 0 && j < rows && to - j * pb < n) || (j + 1 < rows && (j + 1) * pb - to < n);
    };
    if (pa == pb) return meets(d >= 0 ? rows - 1 : 0);
    for (int64_t i = 0; i < rows; ++i)
        if (meets(i)) return true;
    return false;
}

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
    if ((grad != logits || ldg != ld) &&
        rows_meet(reinterpret_cast<uintptr_t>(logits), ld * size, reinterpret_cast<uintptr_t>(grad), ldg * size, T, V * size))
        return BS_ERR_UNSUPPORTED;
    if (!aligned4(lse, entropy, g_logprob, g_entropy)) return BS_ERR_ALIGN;
    return bs::launch_logprobs_backward(logits, dtype, T, V, ld, targets, lse, entropy, g_logprob, g_entropy, grad, ldg,
                                        static_cast<hipStream_t>(stream));
}

}  // extern "C"
