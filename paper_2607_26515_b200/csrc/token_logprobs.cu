// resq_token_logprobs: log-probabilities of given tokens, entropy and the largest alternatives of every row of logits, and
// the gradient of the logits.
//
//   log p_j = (x_j - peak) / T - log_sum,  peak = max_j x_j,  log_sum = log sum_j exp((x_j - peak) / T),
//   logp = log p_tok,  entropy = -sum_j p_j log p_j
//
// The largest logit's own term is exactly 1 and is left out of the running sum: with s the sum of the other terms and
// t = sum_j e_j (x_j - peak), e_j = exp((x_j - peak) / T),
//   log_sum = log1p(s),   entropy = log1p(s) - t / (T (1 + s)),
// so a log-probability or an entropy near 0 keeps its digits.  The backward pass takes peak and log_sum, not their sum:
// in a row of very low values the sum would lose log_sum altogether.
#include "row_common.cuh"

namespace resq {
namespace {

constexpr int kLpThreads = 256;
constexpr float kInf = __builtin_huge_valf();
constexpr float kLowest = -3.4028234663852886e38f;  // differences are cut here: 0 * -inf is no term of a sum

struct LpArgs {
    const void* x;
    int64_t ld;
    const int64_t* tokens;
    float* logp;
    float* entropy;
    float* peak;
    float* log_sum;
    int32_t* top_ids;
    float* top_logp;
    int V, top;
    float inv_t;  // 1 / T
};

// Running sums of a set of logits: m its largest value (-inf: the set has no finite term), s the sum of exp((x - m) / T)
// without one term of value 1, t the sum of exp((x - m) / T) (x - m).
struct Stat {
    float m, s, t;
};
__device__ __forceinline__ void stat_add(Stat& a, float x, float c) {
    if (x == -kInf) return;
    if (x > a.m) {
        if (a.m != -kInf) {
            const float d = fmaxf(a.m - x, kLowest), f = exp2f(d * c);
            a.t = f * (a.t + d * (a.s + 1.0f));
            a.s = (a.s + 1.0f) * f;
        }
        a.m = x;
    } else {
        const float d = fmaxf(x - a.m, kLowest), e = exp2f(d * c);
        a.s += e;
        a.t = fmaf(e, d, a.t);
    }
}
__device__ __forceinline__ Stat stat_join(const Stat& p, const Stat& q, float c) {
    const bool p_first = p.m >= q.m;
    Stat a = p_first ? p : q;
    const Stat& b = p_first ? q : p;
    if (b.m == -kInf) return a.m != -kInf ? a : Stat{a.m, p.s + q.s, 0.0f};
    const float d = fmaxf(b.m - a.m, kLowest), f = exp2f(d * c);
    a.s += f * (b.s + 1.0f);
    a.t += f * (b.t + d * (b.s + 1.0f));
    return a;
}

__device__ __forceinline__ float load_logit(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load_logit(const float* p) { return *p; }

// Orders logits by value (NaN above +inf, -0 equal to 0), equal values by lower index first.
__device__ __forceinline__ uint64_t top_key(float x, int j) {
    uint32_t u;
    if (x != x) u = 0xFFFFFFFFu;
    else {
        const uint32_t b = __float_as_uint(x + 0.0f);
        u = (b & 0x80000000u) ? ~b : b | 0x80000000u;
    }
    return ((uint64_t)u << 32) | (uint32_t)~j;
}

template <typename T>
__global__ void __launch_bounds__(kLpThreads) logprobs_kernel(const __grid_constant__ LpArgs a) {
    __shared__ Stat st[kLpThreads / 32];
    __shared__ uint64_t best[2][kLpThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t m = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + m * a.ld;
    const float c = a.inv_t * 1.4426950408889634f;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    Stat s{-kInf, 0.0f, 0.0f};
    bool bad = false;
    for (int j = threadIdx.x; j < a.V; j += kLpThreads) {
        const float v = load_logit(x + j);
        bad |= !(v < kInf);
        stat_add(s, v, c);
    }
    bad = __syncthreads_or(bad);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s = stat_join(s, Stat{__shfl_xor_sync(~0u, s.m, o), __shfl_xor_sync(~0u, s.s, o), __shfl_xor_sync(~0u, s.t, o)}, c);
    if (lane == 0) st[w] = s;
    __syncthreads();
    s = st[0];
    for (int i = 1; i < kLpThreads / 32; ++i) s = stat_join(s, st[i], c);
    const float log_s = bad ? __int_as_float(0x7FC00000) : log1pf(s.s);
    const bool empty = s.m == -kInf;
    if (threadIdx.x == 0) {
        if (a.logp) {
            const int64_t tok = a.tokens[m];
            float v = 0.0f;
            if (tok >= 0 && tok < a.V) {
                const float xt = load_logit(x + tok);
                v = bad ? log_s : xt == -kInf ? -kInf : (xt - s.m) * a.inv_t - log_s;
            }
            a.logp[m] = v;
        }
        if (a.entropy) a.entropy[m] = bad ? log_s : empty ? 0.0f : log_s - s.t * a.inv_t / (1.0f + s.s);
        if (a.peak) a.peak[m] = bad ? log_s : s.m;
        if (a.log_sum) a.log_sum[m] = log_s;
    }
    uint64_t last = ~0ull;
    for (int r = 0; r < a.top; ++r) {
        uint64_t b = 0;
        for (int j = threadIdx.x; j < a.V; j += kLpThreads) {
            const uint64_t key = top_key(load_logit(x + j), j);
            if ((r == 0 || key < last) && key > b) b = key;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const uint64_t q = __shfl_xor_sync(~0u, b, o);
            b = q > b ? q : b;
        }
        if (lane == 0) best[r & 1][w] = b;
        __syncthreads();
        b = best[r & 1][0];
        for (int i = 1; i < kLpThreads / 32; ++i) b = best[r & 1][i] > b ? best[r & 1][i] : b;
        last = b;
        if (threadIdx.x == 0) {
            const int j = (int)~(uint32_t)b;
            const float v = load_logit(x + j);
            a.top_ids[m * a.top + r] = j;
            a.top_logp[m * a.top + r] = bad ? log_s : v == -kInf ? -kInf : (v - s.m) * a.inv_t - log_s;
        }
    }
}

struct LpBwdArgs {
    const void* x;
    void* dx;
    int64_t ld, ldd;
    const int64_t* tokens;
    const float* logp;
    const float* peak;
    const float* log_sum;
    const float* entropy;
    const float* dlogp;
    const float* dentropy;
    int V;
    float inv_t;
    unsigned chunks;  // blocks per row
};

// dx_j = (1 / T) [dlogp (1[j = tok] - p_j) - dentropy p_j (log p_j + entropy)].  At the token itself 1 - p comes from the
// forward call's logp (-expm1), which keeps its digits when p is near 1.
template <typename T>
__global__ void __launch_bounds__(kLpThreads) logprobs_bwd_kernel(const __grid_constant__ LpBwdArgs a) {
    pdl_wait();
    pdl_trigger();
    const int64_t m = blockIdx.x / a.chunks;
    const int k = (int)((blockIdx.x % a.chunks) * kLpThreads + threadIdx.x) * 8, n = a.V - k;
    if (n <= 0) return;
    const float peak = a.peak[m], log_sum = a.log_sum[m], H = a.dentropy ? a.entropy[m] : 0.0f, de = a.dentropy ? a.dentropy[m] * a.inv_t : 0.0f;
    const int64_t tok = a.tokens[m];
    const bool there = tok >= 0 && tok < a.V;
    const float dl = there ? a.dlogp[m] * a.inv_t : 0.0f;
    Raw8<T> r;
    float v[8];
    r.load(static_cast<const T*>(a.x) + m * a.ld + k, n);
    r.get(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool hot = there && k + i == tok;
        const float z = hot ? a.logp[m] : fmaf(v[i] - peak, a.inv_t, -log_sum);
        const float p = exp2f(z * 1.4426950408889634f);
        float g = hot ? -expm1f(z) * dl : -p * dl;
        if (a.dentropy && p != 0.0f) g -= p * (z + H) * de;
        v[i] = peak == -kInf ? 0.0f : g;
    }
    store8(static_cast<T*>(a.dx) + m * a.ldd + k, v, n);
}

int check_logits(const char* what, const void* x, int dtype, int64_t M, int64_t V, int64_t ld, float temperature) {
    if (!x) return fail(RESQ_ERR_NULL, what, "logits is NULL");
    if (M <= 0 || V <= 0 || M > INT32_MAX || V > RESQ_MAX_VOCAB) {
        set_last_error("%s: M=%lld V=%lld (1 <= M < 2^31, 1 <= V <= %d)", what, (long long)M, (long long)V, RESQ_MAX_VOCAB);
        return RESQ_ERR_SHAPE;
    }
    if (dtype != RESQ_OUT_BF16 && dtype != RESQ_OUT_F32) return fail(RESQ_ERR_PATTERN, what, "unknown type of the logits");
    if (!(temperature >= 1e-6f && temperature <= 1e6f)) return fail(RESQ_ERR_SHAPE, what, "the temperature must lie in 1e-6 .. 1e6");
    if (!rows_aligned(x, ld, V, dtype)) return fail(RESQ_ERR_ALIGN, what, "logits need a 16-byte aligned base and rows, ld >= V");
    return RESQ_OK;
}

}  // namespace
}  // namespace resq

using namespace resq;

extern "C" {

int resq_token_logprobs(const void* logits, int dtype, int64_t M, int64_t V, int64_t ld, const int64_t* tokens, float temperature, int top,
                        float* logp, float* entropy, float* peak, float* log_sum, int32_t* top_ids, float* top_logp, void* stream) {
    const char* what = "token_logprobs";
    int rc = check_logits(what, logits, dtype, M, V, ld, temperature);
    if (rc) return rc;
    if (top < 0 || top > RESQ_MAX_TOP || top > V) {
        set_last_error("token_logprobs: top=%d (0 <= top <= %d and top <= V)", top, RESQ_MAX_TOP);
        return RESQ_ERR_SHAPE;
    }
    if (!logp && !entropy && !peak && !log_sum && top == 0) return fail(RESQ_ERR_NULL, what, "no output is asked for");
    if ((logp && !tokens) || (top > 0 && (!top_ids || !top_logp))) return fail(RESQ_ERR_NULL, what, "logp needs tokens, top needs top_ids and top_logp");
    if (!is_aligned(tokens, 8) || !is_aligned(logp, 4) || !is_aligned(entropy, 4) || !is_aligned(peak, 4) || !is_aligned(log_sum, 4) || !is_aligned(top_ids, 4) ||
        !is_aligned(top_logp, 4))
        return fail(RESQ_ERR_ALIGN, what, "tokens must be 8-byte aligned, the outputs 4-byte aligned");
    LpArgs a{logits, ld, tokens, logp, entropy, peak, log_sum, top_ids, top_logp, (int)V, top, 1.0f / temperature};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    LaunchScope scope(kKindRow, st);
    auto kern = dtype == RESQ_OUT_F32 ? logprobs_kernel<float> : logprobs_kernel<__nv_bfloat16>;
    return cuda_fail(launch_kernel(kern, dim3((unsigned)M), dim3(kLpThreads), 0, st, a), "logprobs_kernel launch");
}

int resq_token_logprobs_backward(const void* logits, int dtype, int64_t M, int64_t V, int64_t ld, const int64_t* tokens, float temperature,
                                 const float* logp, const float* peak, const float* log_sum, const float* entropy, const float* dlogp,
                                 const float* dentropy, void* dlogits, int64_t ldd, void* stream) {
    const char* what = "token_logprobs_backward";
    int rc = check_logits(what, logits, dtype, M, V, ld, temperature);
    if (rc) return rc;
    if (!tokens || !logp || !peak || !log_sum || !dlogp || !dlogits || (dentropy && !entropy))
        return fail(RESQ_ERR_NULL, what, "tokens, logp, peak, log_sum, dlogp and dlogits must not be NULL, dentropy needs entropy");
    if (!rows_aligned(dlogits, ldd, V, dtype)) return fail(RESQ_ERR_ALIGN, what, "dlogits needs a 16-byte aligned base and rows, ldd >= V");
    if (!is_aligned(tokens, 8) || !is_aligned(logp, 4) || !is_aligned(peak, 4) || !is_aligned(log_sum, 4) || !is_aligned(entropy, 4) ||
        !is_aligned(dlogp, 4) ||
        !is_aligned(dentropy, 4))
        return fail(RESQ_ERR_ALIGN, what, "tokens must be 8-byte aligned, the row values 4-byte aligned");
    const int64_t chunks = (V + kLpThreads * 8 - 1) / (kLpThreads * 8);
    if (M * chunks > INT32_MAX) return fail(RESQ_ERR_SHAPE, what, "M x V is too large for one call");
    LpBwdArgs a{logits, dlogits, ld, ldd, tokens, logp, peak, log_sum, entropy, dlogp, dentropy, (int)V, 1.0f / temperature, (unsigned)chunks};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    LaunchScope scope(kKindRow, st);
    auto kern = dtype == RESQ_OUT_F32 ? logprobs_bwd_kernel<float> : logprobs_bwd_kernel<__nv_bfloat16>;
    return cuda_fail(launch_kernel(kern, dim3((unsigned)(M * chunks)), dim3(kLpThreads), 0, st, a),
                     "logprobs_bwd_kernel launch");
}
}
