// resq_block_join: the residual stream between two blocks, forward and backward.
//
//   p  = B rp gamma_post,  rp = 1 / sqrt(mean(B^2) + eps)      (p = B without gamma_post)
//   H' = H + alpha g p,    g = 1 | gate | sigmoid(gate)
//   X  = H' r gamma_pre,   r  = 1 / sqrt(mean(H'^2) + eps)
//
// Forward: one CTA per row, the row stays in registers between the two row sums, so every tensor crosses HBM once.
// Backward: persistent CTAs walk rows m = b, b + P, ... (P CTAs or clusters); a thread owns eight columns and keeps their
// sums over the rows (the gradients of gamma_pre, gamma_post and a channel gate) in registers; at the end each CTA writes its
// sums as one fp32 partial row and a second kernel adds the P partial rows in a fixed order (bit-identical run to run).
#include "row_common.cuh"

#include <algorithm>

namespace resq {
namespace {

constexpr int kMaxThreadsFwd = 1024;  // one row: up to 4 vectors of 8 per thread
constexpr int kMaxThreadsBwd = 512;   // eight columns per thread; longer rows are split over a cluster of CTAs
constexpr int kMaxClusterBwd = 8;
static_assert(kMaxThreadsFwd * 8 * 4 >= RESQ_JOIN_MAX_K && kMaxThreadsBwd * 8 * kMaxClusterBwd >= RESQ_JOIN_MAX_K, "row length");

struct JoinFwd {
    const void* H;
    const __nv_bfloat16* B;
    const __nv_bfloat16* gate;
    const __nv_bfloat16* gamma_post;
    const __nv_bfloat16* gamma_pre;
    void* H_out;
    __nv_bfloat16* X;
    int64_t ldh, ldb, ldg, ldho, ldx;
    int K, sigmoid;
    float alpha, eps;
};

__device__ __forceinline__ float sigmoid_of(float g) { return __fdividef(1.0f, 1.0f + __expf(-g)); }

template <typename S, int VPT>
__global__ void __launch_bounds__(kMaxThreadsFwd) join_fwd_kernel(const __grid_constant__ JoinFwd a) {
    __shared__ float red[2][32];
    pdl_wait();
    pdl_trigger();
    const int64_t m = blockIdx.x;
    const S* hrow = static_cast<const S*>(a.H) + m * a.ldh;
    const __nv_bfloat16* brow = a.B + m * a.ldb;
    Raw8<S> rh[VPT];
    Raw8<__nv_bfloat16> rb[VPT], rg[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int k = (threadIdx.x + j * blockDim.x) * 8, n = a.K - k;
        if (n <= 0) continue;
        rh[j].load(hrow + k, n);
        rb[j].load(brow + k, n);
        if (a.gate) rg[j].load(a.gate + m * a.ldg + k, n);
    }
    float rp = 1.0f;
    if (a.gamma_post) {
        float s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            if ((int)(threadIdx.x + j * blockDim.x) * 8 >= a.K) continue;
            float b[8];
            rb[j].get(b);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] = fmaf(b[i], b[i], s[0]);
        }
        block_sum<1>(s, red[0]);
        rp = 1.0f / sqrtf(s[0] / (float)a.K + a.eps);
    }
    float h[VPT][8];
    float s[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int k = (threadIdx.x + j * blockDim.x) * 8, n = a.K - k;
        if (n <= 0) continue;
        float p[8];
        rb[j].get(p);
        if (a.gamma_post) {
            Raw8<__nv_bfloat16> r;
            float w[8];
            r.load(a.gamma_post + k, n);
            r.get(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = p[i] * rp * w[i];
        }
        if (a.gate) {
            float g[8];
            rg[j].get(g);
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] *= a.sigmoid ? sigmoid_of(g[i]) : g[i];
        }
        rh[j].get(h[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[j][i] = fmaf(a.alpha, p[i], h[j][i]);
            if (i < n) s[0] = fmaf(h[j][i], h[j][i], s[0]);
        }
        store8(static_cast<S*>(a.H_out) + m * a.ldho + k, h[j], n);
    }
    if (!a.X) return;
    // X comes from the 32-bit sum, not from its rounding to the stream's type
    block_sum<1>(s, red[1]);
    const float r = 1.0f / sqrtf(s[0] / (float)a.K + a.eps);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int k = (threadIdx.x + j * blockDim.x) * 8, n = a.K - k;
        if (n <= 0) continue;
        Raw8<__nv_bfloat16> rw;
        float w[8];
        rw.load(a.gamma_pre + k, n);
        rw.get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = h[j][i] * r * w[i];
        store8(a.X + m * a.ldx + k, w, n);
    }
}

struct JoinBwd {
    const void* dHo;             // gradient of H_out, or null
    const __nv_bfloat16* dX;     // gradient of X, or null
    const void* H;               // H_out of the forward call
    const __nv_bfloat16* B;
    const __nv_bfloat16* gate;
    const __nv_bfloat16* gamma_post;
    const __nv_bfloat16* gamma_pre;
    void* dH;
    __nv_bfloat16* dB;
    __nv_bfloat16* dgate;        // a gate per token: [M, K]; null with a channel gate or none
    float* part;                 // [P][ncol][kp]: gamma_pre (if dX), gamma_post (if given), channel gate (if given)
    int64_t kp;                  // K rounded up to a multiple of 8
    int ncol;
    int64_t lddho, lddx, ldh, ldb, ldg, lddh, lddb, lddg;
    int64_t M;
    int K, sigmoid;
    float alpha, eps;
};

// Sum over the block, then over the cluster's blocks in rank order (the same bits in every thread).
template <int NV, int CS>
__device__ __forceinline__ void row_sum(float (&v)[NV], float* buf, float* xbuf) {
    block_sum<NV>(v, buf);
    if (CS == 1) return;
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    if (threadIdx.x < CS) {  // thread t hands this block's sums to block t
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            uint32_t remote;
            const uint32_t local = (uint32_t)__cvta_generic_to_shared(xbuf + rank * NV + i);
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(threadIdx.x));
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote), "f"(v[i]) : "memory");
        }
    }
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float t = 0.0f;
#pragma unroll
        for (int c = 0; c < CS; ++c) t += xbuf[c * NV + i];
        v[i] = t;
    }
}

template <typename S, int CS>
__global__ void __launch_bounds__(kMaxThreadsBwd) join_bwd_kernel(const __grid_constant__ JoinBwd a) {
    __shared__ float red[2][3 * 32];
    __shared__ float xred[2][3 * CS];
    pdl_wait();
    pdl_trigger();
    const int64_t group = blockIdx.x / CS, groups = gridDim.x / CS;
    const int k = (int)((blockIdx.x % CS) * blockDim.x + threadIdx.x) * 8;
    const int n = a.K - k;  // <= 0: no column of its own, but it takes part in the sums
    const float inv_k = 1.0f / (float)a.K;
    float wpre[8], wpost[8], acc_pre[8], acc_post[8], acc_gate[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) wpre[i] = 0.0f, wpost[i] = 1.0f, acc_pre[i] = acc_post[i] = acc_gate[i] = 0.0f;
    if (n > 0) {
        Raw8<__nv_bfloat16> r;
        if (a.dX) r.load(a.gamma_pre + k, n), r.get(wpre);
        if (a.gamma_post) r.load(a.gamma_post + k, n), r.get(wpost);
    }
    int flip = 0;
    for (int64_t m = group; m < a.M; m += groups) {
        float h[8], u[8], d[8], b[8], G[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = u[i] = d[i] = b[i] = 0.0f, G[i] = 1.0f;
        if (n > 0) {
            Raw8<S> rs;
            Raw8<__nv_bfloat16> r;
            rs.load(static_cast<const S*>(a.H) + m * a.ldh + k, n), rs.get(h);
            if (a.dHo) rs.load(static_cast<const S*>(a.dHo) + m * a.lddho + k, n), rs.get(d);
            if (a.dX) r.load(a.dX + m * a.lddx + k, n), r.get(u);
            r.load(a.B + m * a.ldb + k, n), r.get(b);
            if (a.gate) r.load(a.gate + m * a.ldg + k, n), r.get(G);
        }
        float s[3] = {0.0f, 0.0f, 0.0f};  // sum h^2, sum dX gamma_pre h, sum b^2
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[0] = fmaf(h[i], h[i], s[0]);
            s[1] = fmaf(u[i] * wpre[i], h[i], s[1]);
            s[2] = fmaf(b[i], b[i], s[2]);
        }
        row_sum<3, CS>(s, red[flip], xred[flip]);
        const float r = 1.0f / sqrtf(s[0] * inv_k + a.eps);
        const float c = s[1] * r * inv_k * r;  // mean(u xhat) r, per unit of h
        const float rp = a.gamma_post ? 1.0f / sqrtf(s[2] * inv_k + a.eps) : 1.0f;
        float t[1] = {0.0f};
        float dg[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (a.dX) {
                acc_pre[i] = fmaf(u[i], h[i] * r, acc_pre[i]);
                d[i] = fmaf(r, u[i] * wpre[i] - h[i] * c, d[i]);
            }
            const float nb = b[i] * rp;            // normalised branch (or the branch itself)
            float g = G[i], slope = 1.0f;
            if (a.gate && a.sigmoid) g = sigmoid_of(g), slope = g * (1.0f - g);
            const float dp = a.alpha * d[i];
            dg[i] = dp * nb * wpost[i] * slope;
            acc_gate[i] += dg[i];
            acc_post[i] = fmaf(dp * g, nb, acc_post[i]);
            b[i] = dp * g * wpost[i];              // gradient of the normalised branch
            h[i] = nb;
            t[0] = fmaf(b[i], nb, t[0]);
        }
        if (a.gamma_post) {
            row_sum<1, CS>(t, red[1], xred[1]);
            const float q = t[0] * inv_k;
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = rp * (b[i] - h[i] * q);
        } else {
            flip ^= 1;  // one sum per row: alternate the buffers from row to row
        }
        if (n > 0) {
            store8(static_cast<S*>(a.dH) + m * a.lddh + k, d, n);
            store8(a.dB + m * a.lddb + k, b, n);
            if (a.dgate) store8(a.dgate + m * a.lddg + k, dg, n);
        }
    }
    if (n > 0) {
        float* out = a.part + group * a.ncol * a.kp + k;
        if (a.dX) store8(out, acc_pre, n), out += a.kp;
        if (a.gamma_post) store8(out, acc_post, n), out += a.kp;
        if (a.gate && a.ldg == 0) store8(out, acc_gate, n);
    }
    if (CS > 1) {  // no CTA leaves while a peer may still write its shared memory
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
}

// Sum of the P partial rows: a block owns 32 columns, each of its eight warps adds a contiguous run of rows, and the eight
// sums are added in order.
struct JoinSum {
    const float* part;
    float* out[3];
    int64_t kp;
    int P, ncol, K;
};
__global__ void __launch_bounds__(256) join_sum_kernel(const __grid_constant__ JoinSum a) {
    __shared__ float buf[8][32];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, col = blockIdx.x * 32 + lane, which = blockIdx.y;
    const int per = (a.P + 7) / 8, p0 = w * per, p1 = min(a.P, p0 + per);
    float s = 0.0f;
    if (col < a.K) {
        const float* src = a.part + (int64_t)which * a.kp + col;
        for (int p = p0; p < p1; ++p) s += src[(int64_t)p * a.ncol * a.kp];
    }
    buf[w][lane] = s;
    __syncthreads();
    if (w == 0 && col < a.K) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += buf[i][lane];
        a.out[which][col] = t;
    }
}

// ---- host side -----------------------------------------------------------------------------------
constexpr int kSms = 148;

int bwd_cluster(int64_t K) {
    int cs = 1;
    while ((K + 7) / 8 > (int64_t)cs * kMaxThreadsBwd) cs *= 2;
    return cs;
}
int bwd_threads(int64_t K, int cs) { return (int)(((K + 7) / 8 + cs * 32 - 1) / (cs * 32) * 32); }
int64_t bwd_groups(int64_t M, int64_t K) {
    const int cs = bwd_cluster(K), per_sm = std::min(16, std::max(1, 1024 / bwd_threads(K, cs)));
    return std::min<int64_t>(M, std::max(1, kSms * per_sm / cs));
}

int check_join(const char* what, int64_t M, int64_t K, int dtype, const void* B, int64_t ldb, const void* gate, int64_t ldg, int gate_act,
               const void* gamma_post, float alpha, float eps) {
    if (!B) return fail(RESQ_ERR_NULL, what, "B is NULL");
    if (M <= 0 || K <= 0 || K > RESQ_JOIN_MAX_K || M > INT32_MAX) {
        set_last_error("%s: M=%lld K=%lld (1 <= K <= %d, 1 <= M < 2^31)", what, (long long)M, (long long)K, RESQ_JOIN_MAX_K);
        return RESQ_ERR_SHAPE;
    }
    if (dtype != RESQ_OUT_BF16 && dtype != RESQ_OUT_F32) return fail(RESQ_ERR_PATTERN, what, "unknown type of the residual stream");
    if (gate_act != RESQ_GATE_LINEAR && gate_act != RESQ_GATE_SIGMOID) return fail(RESQ_ERR_PATTERN, what, "unknown gate function");
    if (!(eps >= 0.0f) || eps > 3.0e38f || !(alpha >= -3.0e38f && alpha <= 3.0e38f))
        return fail(RESQ_ERR_SHAPE, what, "eps must be finite and >= 0, alpha finite");
    if (!rows_aligned(B, ldb, K, RESQ_OUT_BF16) || (gate && ldg != 0 && !rows_aligned(gate, ldg, K, RESQ_OUT_BF16)) ||
        (gate && !is_aligned(gate, 16)) || (gamma_post && !is_aligned(gamma_post, 16)))
        return fail(RESQ_ERR_ALIGN, what, "B, gate and the norm weights need 16-byte aligned bases and rows, ld >= K (a channel gate: ldg = 0)");
    return RESQ_OK;
}

}  // namespace
}  // namespace resq

using namespace resq;

extern "C" {

int resq_block_join(const void* H, int stream_dtype, const void* B, int64_t M, int64_t K, int64_t ldh, int64_t ldb, const void* gate,
                    int64_t ldg, int gate_act, const void* gamma_post, const void* gamma_pre, float alpha, float eps, void* H_out,
                    int64_t ldho, void* X, int64_t ldx, void* stream) {
    const char* what = "block_join";
    if (!H || !H_out) return fail(RESQ_ERR_NULL, what, "H and H_out must not be NULL");
    if (X && !gamma_pre) return fail(RESQ_ERR_NULL, what, "X needs gamma_pre");
    int rc = check_join(what, M, K, stream_dtype, B, ldb, gate, ldg, gate_act, gamma_post, alpha, eps);
    if (rc) return rc;
    if (!rows_aligned(H, ldh, K, stream_dtype) || !rows_aligned(H_out, ldho, K, stream_dtype))
        return fail(RESQ_ERR_ALIGN, what, "H and H_out need 16-byte aligned bases and rows, ld >= K");
    if (X && (!rows_aligned(X, ldx, K, RESQ_OUT_BF16) || !is_aligned(gamma_pre, 16)))
        return fail(RESQ_ERR_ALIGN, what, "X and gamma_pre need 16-byte aligned bases and rows, ldx >= K");
    JoinFwd a;
    a.H = H;
    a.B = static_cast<const __nv_bfloat16*>(B);
    a.gate = static_cast<const __nv_bfloat16*>(gate);
    a.gamma_post = static_cast<const __nv_bfloat16*>(gamma_post);
    a.gamma_pre = static_cast<const __nv_bfloat16*>(gamma_pre);
    a.H_out = H_out;
    a.X = static_cast<__nv_bfloat16*>(X);
    a.ldh = ldh, a.ldb = ldb, a.ldg = ldg, a.ldho = ldho, a.ldx = ldx;
    a.K = (int)K, a.sigmoid = gate_act == RESQ_GATE_SIGMOID, a.alpha = alpha, a.eps = eps;
    const int64_t vecs = (K + 7) / 8;
    const int vpt = vecs <= kMaxThreadsFwd ? 1 : vecs <= 2 * kMaxThreadsFwd ? 2 : 4;
    const unsigned threads = (unsigned)((vecs + vpt * 32 - 1) / (vpt * 32) * 32);
    const bool f32 = stream_dtype == RESQ_OUT_F32;
    auto kern = vpt == 1   ? (f32 ? join_fwd_kernel<float, 1> : join_fwd_kernel<__nv_bfloat16, 1>)
                : vpt == 2 ? (f32 ? join_fwd_kernel<float, 2> : join_fwd_kernel<__nv_bfloat16, 2>)
                           : (f32 ? join_fwd_kernel<float, 4> : join_fwd_kernel<__nv_bfloat16, 4>);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    LaunchScope scope(kKindRow, st);
    return cuda_fail(launch_kernel(kern, dim3((unsigned)M), dim3(threads), 0, st, a), "join_fwd_kernel launch");
}

size_t resq_block_join_backward_workspace_bytes(int64_t M, int64_t K) {
    if (M <= 0 || K <= 0 || K > RESQ_JOIN_MAX_K) return 0;
    return align_up((size_t)bwd_groups(M, K) * 3 * (size_t)((K + 7) / 8 * 8) * sizeof(float), 256);
}

int resq_block_join_backward(const void* dH_out, const void* dX, const void* H_out, int stream_dtype, const void* B, int64_t M, int64_t K,
                             int64_t lddho, int64_t lddx, int64_t ldho, int64_t ldb, const void* gate, int64_t ldg, int gate_act,
                             const void* gamma_post, const void* gamma_pre, float alpha, float eps, void* dH, int64_t lddh, void* dB,
                             int64_t lddb, void* dgate, int64_t lddg, float* dgamma_post, float* dgamma_pre, void* workspace,
                             size_t ws_bytes, void* stream) {
    const char* what = "block_join_backward";
    if (!H_out || !dH || !dB || (!dH_out && !dX)) return fail(RESQ_ERR_NULL, what, "H_out, dH, dB and one of dH_out and dX must not be NULL");
    if (dX && (!gamma_pre || !dgamma_pre)) return fail(RESQ_ERR_NULL, what, "dX needs gamma_pre and dgamma_pre");
    if ((gamma_post && !dgamma_post) || (gate && !dgate)) return fail(RESQ_ERR_NULL, what, "gamma_post needs dgamma_post, a gate needs dgate");
    int rc = check_join(what, M, K, stream_dtype, B, ldb, gate, ldg, gate_act, gamma_post, alpha, eps);
    if (rc) return rc;
    if (!rows_aligned(H_out, ldho, K, stream_dtype) || !rows_aligned(dH, lddh, K, stream_dtype) ||
        (dH_out && !rows_aligned(dH_out, lddho, K, stream_dtype)) || !rows_aligned(dB, lddb, K, RESQ_OUT_BF16))
        return fail(RESQ_ERR_ALIGN, what, "dH_out, H_out, dH and dB need 16-byte aligned bases and rows, ld >= K");
    if (dX && (!rows_aligned(dX, lddx, K, RESQ_OUT_BF16) || !is_aligned(gamma_pre, 16) || !is_aligned(dgamma_pre, 4)))
        return fail(RESQ_ERR_ALIGN, what, "dX and gamma_pre need 16-byte aligned bases and rows, lddx >= K");
    if (gate && (ldg == 0 ? !is_aligned(dgate, 4) : !rows_aligned(dgate, lddg, K, RESQ_OUT_BF16)))
        return fail(RESQ_ERR_ALIGN, what, "dgate needs a 16-byte aligned base and rows, lddg >= K (a channel gate: fp32 [K])");
    if (gamma_post && !is_aligned(dgamma_post, 4)) return fail(RESQ_ERR_ALIGN, what, "dgamma_post is not aligned");
    const size_t need = resq_block_join_backward_workspace_bytes(M, K);
    if (!workspace || !is_aligned(workspace, 256) || ws_bytes < need) {
        set_last_error("workspace: need %zu bytes, 256-byte aligned (have %zu at %p)", need, ws_bytes, workspace);
        return RESQ_ERR_WORKSPACE;
    }
    JoinBwd a;
    a.dHo = dH_out;
    a.dX = static_cast<const __nv_bfloat16*>(dX);
    a.H = H_out;
    a.B = static_cast<const __nv_bfloat16*>(B);
    a.gate = static_cast<const __nv_bfloat16*>(gate);
    a.gamma_post = static_cast<const __nv_bfloat16*>(gamma_post);
    a.gamma_pre = static_cast<const __nv_bfloat16*>(gamma_pre);
    a.dH = dH;
    a.dB = static_cast<__nv_bfloat16*>(dB);
    a.dgate = gate && ldg != 0 ? static_cast<__nv_bfloat16*>(dgate) : nullptr;
    a.part = static_cast<float*>(workspace);
    a.kp = (K + 7) / 8 * 8;
    a.lddho = lddho, a.lddx = lddx, a.ldh = ldho, a.ldb = ldb, a.ldg = ldg, a.lddh = lddh, a.lddb = lddb, a.lddg = lddg;
    a.M = M, a.K = (int)K, a.sigmoid = gate_act == RESQ_GATE_SIGMOID, a.alpha = alpha, a.eps = eps;
    JoinSum s;
    s.ncol = 0;
    if (dX) s.out[s.ncol++] = dgamma_pre;
    if (gamma_post) s.out[s.ncol++] = dgamma_post;
    if (gate && ldg == 0) s.out[s.ncol++] = static_cast<float*>(dgate);
    a.ncol = s.ncol;
    const int cs = bwd_cluster(K);
    const int64_t groups = bwd_groups(M, K);
    const bool f32 = stream_dtype == RESQ_OUT_F32;
    using bf = __nv_bfloat16;
    auto kern = cs == 1   ? (f32 ? join_bwd_kernel<float, 1> : join_bwd_kernel<bf, 1>)
                : cs == 2 ? (f32 ? join_bwd_kernel<float, 2> : join_bwd_kernel<bf, 2>)
                : cs == 4 ? (f32 ? join_bwd_kernel<float, 4> : join_bwd_kernel<bf, 4>)
                          : (f32 ? join_bwd_kernel<float, 8> : join_bwd_kernel<bf, 8>);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    {
        LaunchScope scope(kKindRow, st);
        rc = cuda_fail(launch_clusters(kern, (unsigned)(groups * cs), (unsigned)bwd_threads(K, cs), 0, cs, st, a), "join_bwd_kernel launch");
    }
    if (rc || s.ncol == 0) return rc;
    s.part = a.part, s.kp = a.kp, s.P = (int)groups, s.K = (int)K;
    LaunchScope scope(kKindRow, st);
    return cuda_fail(launch_kernel(join_sum_kernel, dim3((unsigned)((K + 31) / 32), (unsigned)s.ncol), dim3(256), 0, st, s),
                     "join_sum_kernel launch");
}
}
