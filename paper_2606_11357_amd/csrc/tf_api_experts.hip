// C-ABI entry points of the 8-bit linear layers and the layers made of experts:
// argument checks, always before any HIP call, and dispatch to the launchers.  Sizes
// are looked at before pointers: tensors without elements have none.
#include "tf_route.h"
#include "tf_w8a8.h"

namespace tf {
int launch_quantize_rows(bool bf, const void* x, int64_t stride, int64_t M, int64_t N, bool gated, int8_t* q,
                         float* scale, hipStream_t s);
int launch_pack_w8a8(const int8_t* w, const void* scales, int scale_dtype, int64_t K, int64_t N, int64_t experts,
                     void* packed, hipStream_t s);
int launch_w8a8(W8Args a, void* ws, int64_t ws_bytes, hipStream_t s);
int64_t w8a8_workspace_bytes(int64_t M, int64_t K, int64_t N);
int launch_route_experts(const RouteArgs& a, int32_t* offsets, int32_t* tokens, int32_t* places, hipStream_t s);
int launch_combine_experts(const CombineArgs& a, bool bf, hipStream_t s);
}  // namespace tf

namespace {

bool misaligned(const void* p, uintptr_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
bool bad_dtype(int dtype) { return dtype != TF_F16 && dtype != TF_BF16; }
// A launch has fewer than 2^32 threads.
bool too_many(int64_t threads) { return threads > (int64_t)UINT32_MAX; }
bool bad_kn(int64_t K, int64_t N) {
    return K <= 0 || N <= 0 || K % 16 != 0 || N % 8 != 0 || K > TF_MAX_DIM || N > TF_MAX_DIM;
}

}  // namespace

extern "C" {

int tf_quantize_rows(int dtype, const void* X, int64_t x_stride, int64_t M, int64_t N, int gated, int8_t* codes,
                     float* scales, void* stream) {
    if (bad_dtype(dtype)) return TF_ERR_ARG;
    if (M < 1 || M > TF_MAX_SLOTS || N <= 0 || N > TF_MAX_DIM || N % 16 != 0) return TF_ERR_SHAPE;
    if (x_stride < (gated ? 2 * N : N) || x_stride % 8 != 0 || x_stride > (int64_t(1) << 40)) return TF_ERR_SHAPE;
    if (too_many(M * (N <= 512 ? 64 : N <= 1024 ? 128 : N <= 4096 ? 256 : N <= 8192 ? 512 : 1024) + 255))
        return TF_ERR_SHAPE;
    if (!X || !codes || !scales) return TF_ERR_NULL;
    if (misaligned(X) || misaligned(codes) || misaligned(scales, 4)) return TF_ERR_ALIGN;
    return tf::launch_quantize_rows(dtype == TF_BF16, X, x_stride, M, N, gated != 0, codes, scales,
                                    static_cast<hipStream_t>(stream));
}

int64_t tf_w8a8_packed_bytes(int64_t K, int64_t N) {
    if (bad_kn(K, N)) return TF_ERR_SHAPE;
    return tf::w8_layout(K, N).total;
}

int tf_pack_w8a8(const int8_t* qweight, const void* scales, int scale_dtype, int64_t K, int64_t N, int64_t experts,
                 void* packed, void* stream) {
    if (bad_dtype(scale_dtype) && scale_dtype != TF_F32) return TF_ERR_ARG;
    if (bad_kn(K, N) || experts < 1 || experts > TF_MAX_EXPERTS) return TF_ERR_SHAPE;
    if (!qweight || !scales || !packed) return TF_ERR_NULL;
    if (misaligned(qweight) || misaligned(scales) || misaligned(packed, 256)) return TF_ERR_ALIGN;
    return tf::launch_pack_w8a8(qweight, scales, scale_dtype, K, N, experts, packed, static_cast<hipStream_t>(stream));
}

int64_t tf_w8a8_workspace_bytes(int64_t M, int64_t K, int64_t N) {
    if (bad_kn(K, N) || M < 1 || M > TF_MAX_M) return TF_ERR_SHAPE;
    return tf::w8a8_workspace_bytes(M, K, N);
}

int tf_w8a8_gemm(int dtype, const int8_t* A, const float* a_scales, const void* packed, void* C, int64_t M, int64_t K,
                 int64_t N, void* workspace, size_t workspace_bytes, void* stream) {
    if (bad_dtype(dtype)) return TF_ERR_ARG;
    if (bad_kn(K, N) || M < 1 || M > TF_MAX_M) return TF_ERR_SHAPE;
    if (!A || !a_scales || !packed || !C) return TF_ERR_NULL;
    if (workspace && (int64_t)workspace_bytes < tf::w8a8_workspace_bytes(M, K, N)) return TF_ERR_ARG;
    if (misaligned(A) || misaligned(C) || misaligned(packed, 256) || misaligned(a_scales, 4) || misaligned(workspace))
        return TF_ERR_ALIGN;
    const tf::W8Layout L = tf::w8_layout(K, N);
    const tf::W8Args a{A, a_scales, static_cast<const uint8_t*>(packed), static_cast<uint16_t*>(C), nullptr, nullptr,
                       M, M, K, N, L.total, L.s_off, (int)L.na, (int)L.np, 0, dtype == TF_BF16, 1, nullptr};
    const auto turn = tf::workspace_turn(workspace);
    return tf::launch_w8a8(a, workspace, (int64_t)workspace_bytes, static_cast<hipStream_t>(stream));
}

int tf_route_experts(int dtype, const void* logits, int64_t stride, const float* bias, int64_t T, int experts,
                     int top_k, int scoring, int groups, int top_groups, int group_score, int renormalize, float scale,
                     float* weights, int32_t* chosen, int32_t* offsets, int32_t* tokens, int32_t* places,
                     void* stream) {
    if ((bad_dtype(dtype) && dtype != TF_F32) || scoring < 0 || scoring > 1 || group_score < 0 || group_score > 1)
        return TF_ERR_ARG;
    if (!(scale > 0.f) || scale > 1e30f) return TF_ERR_ARG;
    if (T < 1 || T > TF_MAX_M || experts < 1 || experts > TF_MAX_EXPERTS) return TF_ERR_SHAPE;
    if (stride < experts || stride > (int64_t(1) << 40)) return TF_ERR_SHAPE;
    if (groups < 1 || groups > 64 || experts % groups != 0 || top_groups < 1 || top_groups > groups) return TF_ERR_SHAPE;
    if (top_k < 1 || top_k > TF_MAX_TOP_K || top_k > experts / groups * top_groups) return TF_ERR_SHAPE;
    if (!logits || !weights || !chosen || !offsets || !tokens || !places) return TF_ERR_NULL;
    if (misaligned(logits, dtype == TF_F32 ? 4 : 2)) return TF_ERR_ALIGN;
    for (const void* p : {(const void*)bias, (const void*)weights, (const void*)chosen, (const void*)offsets,
                          (const void*)tokens, (const void*)places})
        if (misaligned(p, 4)) return TF_ERR_ALIGN;
    int per = 1;
    while (2 * per <= 64 / groups) per *= 2;
    const tf::RouteArgs a{logits, bias, weights, chosen, T, stride, dtype, experts, top_k, groups, top_groups, per,
                          scoring == 1, group_score == 1, renormalize != 0, scale};
    return tf::launch_route_experts(a, offsets, tokens, places, static_cast<hipStream_t>(stream));
}

int tf_w8a8_expert_gemm(int dtype, const int8_t* A, const float* a_scales, int64_t a_rows, const void* packed,
                        const int32_t* offsets, const int32_t* rows, void* C, int64_t slots, int64_t K, int64_t N,
                        int64_t experts, void* stream) {
    if (bad_dtype(dtype)) return TF_ERR_ARG;
    if (bad_kn(K, N) || experts < 1 || experts > TF_MAX_EXPERTS) return TF_ERR_SHAPE;
    if (slots < 1 || slots > TF_MAX_SLOTS || a_rows < 1 || a_rows > TF_MAX_SLOTS) return TF_ERR_SHAPE;
    if (rows && a_rows * K >= 0xFFFFFF00ll) return TF_ERR_SHAPE;      // gathered rows have 32-bit offsets
    if (!A || !a_scales || !packed || !offsets || !C) return TF_ERR_NULL;
    if (misaligned(A) || misaligned(C) || misaligned(packed, 256) || misaligned(a_scales, 4) ||
        misaligned(offsets, 4) || misaligned(rows, 4))
        return TF_ERR_ALIGN;
    const tf::W8Layout L = tf::w8_layout(K, N);
    const tf::W8Args a{A, a_scales, static_cast<const uint8_t*>(packed), static_cast<uint16_t*>(C), offsets, rows,
                       slots, a_rows, K, N, L.total, L.s_off, (int)L.na, (int)L.np, (int)experts, dtype == TF_BF16, 1, nullptr};
    return tf::launch_w8a8(a, nullptr, 0, static_cast<hipStream_t>(stream));
}

int tf_combine_experts(int dtype, const void* Y, int64_t slots, const float* weights, const int32_t* places,
                       const void* add, int64_t T, int top_k, int64_t N, void* out, void* stream) {
    if (bad_dtype(dtype)) return TF_ERR_ARG;
    if (T < 1 || T > TF_MAX_M || slots < 1 || slots > TF_MAX_SLOTS || N <= 0 || N > TF_MAX_DIM || N % 8 != 0 ||
        top_k < 1 || top_k > TF_MAX_TOP_K)
        return TF_ERR_SHAPE;
    if (too_many(T * (N / 8) + 255)) return TF_ERR_SHAPE;
    if (!Y || !weights || !places || !out) return TF_ERR_NULL;
    for (const void* p : {Y, add, (const void*)out})
        if (misaligned(p)) return TF_ERR_ALIGN;
    if (misaligned(weights, 4) || misaligned(places, 4)) return TF_ERR_ALIGN;
    const tf::CombineArgs a{static_cast<const uint16_t*>(Y), static_cast<const uint16_t*>(add), weights, places,
                            static_cast<uint16_t*>(out), T, slots, top_k, (int)N};
    return tf::launch_combine_experts(a, dtype == TF_BF16, static_cast<hipStream_t>(stream));
}

}  // extern "C"
