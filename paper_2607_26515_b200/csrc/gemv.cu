// *_w4a16_gemv: Y[m, n] = sum_k X[m, k] deq(W)[n, k] for at most RESQ_GEMV_MAX_TOKENS token rows.
//
// One warp per weight row: a lane takes eight codes (one 32-bit word) at a time, decodes them to fp32 and multiplies them
// with the eight activations of every token; the 32 partial sums are added at the end.
#include "common.cuh"
#include "quant_device.cuh"
#include "row_common.cuh"

namespace resq {
namespace {

constexpr int kGemvThreads = 256;

template <int FMT, int MT>
__global__ void __launch_bounds__(kGemvThreads) gemv_kernel(const __nv_bfloat16* __restrict__ X, int M, int64_t K, int64_t ldx,
                                                            const uint8_t* __restrict__ codes, const void* __restrict__ side,
                                                            int64_t N, void* __restrict__ Y, int out_dtype, int64_t ldy) {
    pdl_wait();
    pdl_trigger();
    const int64_t n = (int64_t)blockIdx.x * (kGemvThreads / 32) + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (n >= N) return;
    float acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = 0.0f;
    for (int64_t k = lane * 8; k < K; k += 256) {
        const uint32_t c = *reinterpret_cast<const uint32_t*>(codes + n * (K / 2) + k / 2);
        float w[8];
        if (FMT == kHiF4)
            hif4_decode_lane(c, reinterpret_cast<const uint32_t*>(side)[n * (K / kHif4Block) + k / kHif4Block], (int)((k / 8) & 7), w);
        else
            mxfp4_decode_lane(c, reinterpret_cast<const uint8_t*>(side)[n * (K / kMxBlock) + k / kMxBlock], w);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (m >= M) break;
            Raw8<__nv_bfloat16> r;
            r.load(X + m * ldx + k, 8);
            float x[8];
            r.get(x);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[m] = fmaf(x[i], w[i], acc[m]);
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if (m >= M) break;
        float v = acc[m];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        if (lane == 0) {
            if (out_dtype == RESQ_OUT_BF16) reinterpret_cast<__nv_bfloat16*>(Y)[m * ldy + n] = __float2bfloat16_rn(v);
            else reinterpret_cast<float*>(Y)[m * ldy + n] = v;
        }
    }
}

template <int FMT>
int launch_gemv(const __nv_bfloat16* X, int M, int64_t K, int64_t ldx, const uint8_t* codes, const void* side, int64_t N, void* Y,
                int out_dtype, int64_t ldy, cudaStream_t stream) {
    const int64_t grid = (N + kGemvThreads / 32 - 1) / (kGemvThreads / 32);
    LaunchScope scope(kKindGemm, stream);
    auto kern = M <= 1 ? gemv_kernel<FMT, 1> : M <= 4 ? gemv_kernel<FMT, 4> : gemv_kernel<FMT, RESQ_GEMV_MAX_TOKENS>;
    return cuda_fail(launch_kernel(kern, dim3((unsigned)grid), dim3(kGemvThreads), 0, stream, X, M, K, ldx, codes, side, N, Y, out_dtype, ldy),
                     "gemv_kernel launch");
}

int gemv(int fmt, const void* X, int64_t M, int64_t K, int64_t ldx, const void* w_codes, const void* w_side, int64_t N, void* Y,
         int out_dtype, int64_t ldy, void* stream) {
    const int block = fmt == kHiF4 ? kHif4Block : kMxBlock;
    if (!X || !w_codes || !w_side || !Y) return fail(RESQ_ERR_NULL, "gemv", "X, the packed weight and Y must not be NULL");
    if (M <= 0 || N <= 0 || K <= 0 || K % block != 0 || M > RESQ_GEMV_MAX_TOKENS || N > INT32_MAX || K > INT32_MAX) {
        set_last_error("gemv: M=%lld N=%lld K=%lld (1 <= M <= %d, K a positive multiple of %d, N and K below 2^31)", (long long)M,
                       (long long)N, (long long)K, RESQ_GEMV_MAX_TOKENS, block);
        return RESQ_ERR_SHAPE;
    }
    if (out_dtype != RESQ_OUT_BF16 && out_dtype != RESQ_OUT_F32) {
        set_last_error("unknown output type %d", out_dtype);
        return RESQ_ERR_PATTERN;
    }
    if (!rows_aligned(X, ldx, K, RESQ_OUT_BF16))
        return fail(RESQ_ERR_ALIGN, "gemv", "X needs a 16-byte aligned base and ldx >= K, ldx % 8 == 0");
    if (!is_aligned(w_codes, 16) || !is_aligned(w_side, 16) || !rows_aligned(Y, ldy, N, out_dtype))
        return fail(RESQ_ERR_ALIGN, "gemv", "Y / weights need 16-byte aligned bases, ldy >= N and 16-byte aligned rows");
    const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(X);
    const uint8_t* c = static_cast<const uint8_t*>(w_codes);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return fmt == kHiF4 ? launch_gemv<kHiF4>(x, (int)M, K, ldx, c, w_side, N, Y, out_dtype, ldy, st)
                        : launch_gemv<kMXFP4>(x, (int)M, K, ldx, c, w_side, N, Y, out_dtype, ldy, st);
}

}  // namespace
}  // namespace resq

using namespace resq;

extern "C" {
int hif4_w4a16_gemv(const void* X, int64_t M, int64_t K, int64_t ldx, const void* w_codes, const void* w_meta, int64_t N, void* Y,
                    int out_dtype, int64_t ldy, void* stream) {
    return gemv(kHiF4, X, M, K, ldx, w_codes, w_meta, N, Y, out_dtype, ldy, stream);
}
int mxfp4_w4a16_gemv(const void* X, int64_t M, int64_t K, int64_t ldx, const void* w_codes, const void* w_scale, int64_t N, void* Y,
                     int out_dtype, int64_t ldy, void* stream) {
    return gemv(kMXFP4, X, M, K, ldx, w_codes, w_scale, N, Y, out_dtype, ldy, stream);
}
}
