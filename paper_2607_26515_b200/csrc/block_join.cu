// resq_block_join: the residual stream between two blocks, forward and backward.
//
//   p  = B rp gamma_post,  rp = 1 / sqrt(mean(B^2) + eps)      (p = B without gamma_post)
//   H' = H + alpha g p,    g = 1 | gate | sigmoid(gate)
//   X  = H' r gamma_pre,   r  = 1 / sqrt(mean(H'^2) + eps)
//
// Forward: one CTA per row, the row stays in registers between the two row sums, so every tensor crosses HBM once.
// Backward: persistent CTAs walk rows m = b, b + P, ... (P CTAs or clusters); a thread owns eight or sixteen columns and keeps
// their sums over the rows in registers; at the end each CTA writes them as one fp32 partial row and a second kernel adds the P
// partial rows in a fixed order (bit-identical run to run).  The rows to come are in flight in a ring of asynchronous copies:
// two row sums with a block barrier each leave a row's loads no time of their own otherwise (8192 x 2048, fp32 stream, channel
// gate: 122 us without the ring, 59 with it).
//
// Measured: forward 16384 x 3584, bf16, norm and gate per token, 105 us = 5.6 TB/s (0.86 of the copy rate); backward of the
// same 214 us = 4.4 TB/s (0.67) and 8192 x 2048, fp32, channel gate, 59 us = 5.1 TB/s (0.78).  The forward pass is bound by HBM.  The
// backward pass keeps a row and its column sums in registers, which leaves 16 warps per SM: between a row's barrier and its
// loads' arrival in registers there are too few of them to fill the issue slots (about half are empty).
#include "row_common.cuh"

#include <algorithm>

namespace resq {
namespace {

constexpr int kMaxThreadsFwd = 1024;  // one row: up to 4 vectors of 8 per thread
// Backward, threads per SM: 512 of 128 registers, or 640 of 96 for rows that need them (they spill nothing either, but short rows
// measured slower: 8192 x 2048, fp32 stream, channel gate, 63 against 59 us; 16384 x 3584, gated, 221 against 214).
constexpr int kFewThreads = 512, kManyThreads = 640;
static_assert(kMaxThreadsFwd * 8 * 4 >= RESQ_JOIN_MAX_K && kManyThreads * 8 * 8 >= RESQ_JOIN_MAX_K, "row length");

struct JoinFwd {
    const void* H;
    const __nv_bfloat16* B;
    const __nv_bfloat16* gate;
    const __nv_bfloat16* gamma_post;
    const __nv_bfloat16* gamma_pre;
    void* H_out;
    __nv_bfloat16* X;
    int64_t M, ldh, ldb, ldg, ldho, ldx;
    int K, sigmoid;
    float alpha, eps;
};

// e = exp(-g), s = sigmoid(g) = 1 / (1 + e): two special-function operations, each within 2 ulp; e overflowing to infinity gives 0.
__device__ __forceinline__ float sigmoid_of(float g, float& e) {
    float s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
    return s;
}
// Its derivative s (1 - s) as e s s: 1 - s has lost 1 % of itself at a gate of 12 and all of it at 17.  e is cut at the largest
// number, where s is 0.
__device__ __forceinline__ float sigmoid_slope(float s, float e) { return fminf(e, 3.4028234663852886e38f) * s * s; }

// Eight columns as four packed pairs of fp32.
typedef uint64_t Cols[4];
__device__ __forceinline__ uint64_t both(float v) { return pair(v, v); }
__device__ __forceinline__ uint64_t pair_bf16(uint32_t w) { return pair(bf16_lo(w), bf16_hi(w)); }
__device__ __forceinline__ void cols_bf16(const uint4& q, Cols& v) {
    v[0] = pair_bf16(q.x), v[1] = pair_bf16(q.y), v[2] = pair_bf16(q.z), v[3] = pair_bf16(q.w);
}
__device__ __forceinline__ float sum2(uint64_t p) {
    float lo, hi;
    unpair(p, lo, hi);
    return lo + hi;
}
template <typename T>
__device__ __forceinline__ void store_cols(T* p, const Cols& v, int n) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpair(v[i], f[2 * i], f[2 * i + 1]);
    store8(p, f, n);
}
// G becomes the gate function of G, `slope` its derivative.
__device__ __forceinline__ void gate_cols(bool sigmoid, Cols& G, Cols& slope) {
    if (sigmoid) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo, hi, el, eh;
            unpair(G[i], lo, hi);
            lo = sigmoid_of(lo, el), hi = sigmoid_of(hi, eh);
            G[i] = pair(lo, hi);
            slope[i] = pair(sigmoid_slope(lo, el), sigmoid_slope(hi, eh));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) slope[i] = both(1.0f);
    }
}
template <typename S>
__device__ __forceinline__ void cols_of(const Raw8<S>& r, Cols& v) {
    float f[8];
    r.get(f);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair(f[2 * i], f[2 * i + 1]);
}

// One vector per thread: 32 registers, so that an SM holds 2048 threads and their loads.
template <typename S, int VPT, bool POST, bool GATE>
__global__ void __launch_bounds__(kMaxThreadsFwd, VPT == 1 ? 2 : 1) join_fwd_kernel(const __grid_constant__ JoinFwd a) {
    __shared__ __align__(16) float red[2][32];
    pdl_wait();
    pdl_trigger();
    const int64_t m = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;  // several short rows per CTA, a warp each
    if (m >= a.M) return;
    Raw8<S> rh[VPT];
    Raw8<__nv_bfloat16> rb[VPT], rg[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int k = (threadIdx.x + j * blockDim.x) * 8, n = a.K - k;
        if (n <= 0) continue;
        rb[j].load(a.B + m * a.ldb + k, n);
        rh[j].load(static_cast<const S*>(a.H) + m * a.ldh + k, n);
        if (GATE) rg[j].load(a.gate + m * a.ldg + k, n);
    }
    float scale = a.alpha;  // alpha rp
    if (POST) {
        uint64_t q = 0;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            if ((int)(threadIdx.x + j * blockDim.x) * 8 >= a.K) continue;
            Cols b;
            cols_of(rb[j], b);
#pragma unroll
            for (int i = 0; i < 4; ++i) q = fma2(b[i], b[i], q);
        }
        float s[1] = {sum2(q)};
        block_sum<1>(s, red[0]);
        scale *= rsqrtf(s[0] / (float)a.K + a.eps);
    }
    Cols h[VPT];
    uint64_t q = 0;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int k = (threadIdx.x + j * blockDim.x) * 8, n = a.K - k;
        if (n <= 0) continue;
        Cols p;
        cols_of(rb[j], p);
        if (POST) {
            Raw8<__nv_bfloat16> r;
            Cols w;
            r.load(a.gamma_post + k, n);
            cols_of(r, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = mul2(p[i], w[i]);
        }
        if (GATE) {
            float g[8];
            rg[j].get(g);
            if (a.sigmoid) {
                float e;
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = sigmoid_of(g[i], e);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = mul2(p[i], pair(g[2 * i], g[2 * i + 1]));
        }
        cols_of(rh[j], h[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // behind the last column both are 0 (a padding gate's sigmoid is not, but B is)
            h[j][i] = fma2(both(scale), p[i], h[j][i]);
            q = fma2(h[j][i], h[j][i], q);
        }
        store_cols(static_cast<S*>(a.H_out) + m * a.ldho + k, h[j], n);
    }
    if (!a.X) return;
    // X comes from the 32-bit sum, not from its rounding to the stream's type
    float s[1] = {sum2(q)};
    block_sum<1>(s, red[1]);
    const float r = rsqrtf(s[0] / (float)a.K + a.eps);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int k = (threadIdx.x + j * blockDim.x) * 8, n = a.K - k;
        if (n <= 0) continue;
        Raw8<__nv_bfloat16> rw;
        Cols w;
        rw.load(a.gamma_pre + k, n);
        cols_of(rw, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = mul2(mul2(h[j][i], both(r)), w[i]);
        store_cols(a.X + m * a.ldx + k, w, n);
    }
}

template <typename S, bool POST, bool GATE>
cudaError_t launch_fwd(const JoinFwd& a, cudaStream_t st) {
    const int64_t vecs = (a.K + 7) / 8;
    const int vpt = vecs <= kMaxThreadsFwd ? 1 : vecs <= 2 * kMaxThreadsFwd ? 2 : 4;
    const unsigned threads = (unsigned)((vecs + vpt * 32 - 1) / (vpt * 32) * 32);
    auto kern = vpt == 1 ? join_fwd_kernel<S, 1, POST, GATE> : vpt == 2 ? join_fwd_kernel<S, 2, POST, GATE> : join_fwd_kernel<S, 4, POST, GATE>;
    const unsigned rows = threads == 32 ? 8 : 1;  // 16384 x 256: 17.4 us with a CTA of one warp per row
    return launch_kernel(kern, dim3((unsigned)((a.M + rows - 1) / rows)), dim3(threads, rows), 0, st, a);
}
template <typename S>
cudaError_t launch_fwd(const JoinFwd& a, cudaStream_t st) {
    if (a.gamma_post) return a.gate ? launch_fwd<S, true, true>(a, st) : launch_fwd<S, true, false>(a, st);
    return a.gate ? launch_fwd<S, false, true>(a, st) : launch_fwd<S, false, false>(a, st);
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
    __nv_bfloat16* dgate;        // a gate per token: [M, K]
    float* col[3];               // column sums: [groups][pitch] partial rows (or, with one group, the results) of gamma_pre,
                                 // gamma_post, channel gate; null: not asked for
    int64_t pitch;
    int lddho, lddx, ldh, ldb, ldg, lddh, lddb, lddg;
    int M, K, sigmoid, depth;
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

// One row of a stage in shared memory: its tensors one after the other, each as the CTA's columns lie in memory (whole vectors
// of 8, zeros behind the last column).
__host__ __device__ inline int stage_bytes(int stream_size, bool gate, int columns) { return columns * (2 * stream_size + 4 + (gate ? 2 : 0)); }
constexpr int kMaxDepth = 6;

// POST: the branch is normalised.  GATE: 0 none, 1 channel, 2 per token.  VPT: vectors of 8 columns per thread.  CS: CTAs per row.
// First come the sums over the row of H'^2, dX gamma_pre H' and B^2; then d = the gradient of H' and v = the gradient of the
// normalised branch n; then, with a norm on the branch, the sum of v n.  The first sums of the next row and the last one of this
// row are taken together, so a row costs one barrier.  Without a gate per token the gradients of gamma_post and of the channel
// gate are the same column sum of d n times a constant of the column.
template <typename S, bool POST, int GATE, int VPT, int CS, int MAX>
__global__ void __launch_bounds__(MAX) join_bwd_kernel(const __grid_constant__ JoinBwd a) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ __align__(16) float red[2][4 * 32];
    __shared__ float xred[2][4 * CS];
    const int threads = blockDim.x, tid = threadIdx.x;
    const unsigned groups = gridDim.x / CS, rows = a.M;  // unsigned: the rows asked for run past the last one, which may be 2^31 - 1
    const int columns = VPT * threads * 8, first = (int)(blockIdx.x % CS) * columns;  // this CTA's
    const int stage_size = stage_bytes(sizeof(S), GATE == 2, columns);
    const int at_d = columns * (int)sizeof(S), at_x = 2 * at_d, at_b = at_x + columns * 2, at_g = at_b + columns * 2;
    int n[VPT];  // columns of the thread's vectors (<= 0: none; such a thread takes part in copies and sums)
#pragma unroll
    for (int j = 0; j < VPT; ++j) n[j] = a.K - first - (j * threads + tid) * 8;

    // every CTA of the cluster runs before a peer writes into its shared memory
    if (CS > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    pdl_wait();
    pdl_trigger();
    // one row of one tensor: neighbouring threads copy neighbouring chunks of 16 bytes; zeros up to whole vectors
    const int cols = min(a.K - first, columns);
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + tid * 16;
    auto copy_row = [&](uint32_t dst, const void* src, int size) {
        const uint8_t* p = static_cast<const uint8_t*>(src) + tid * 16;
        int left = cols * size - tid * 16;
#pragma unroll
        for (int c = 0; c < VPT * size / 2; ++c) {
            // behind the last column: the whole of its vector, from the vector's own address (nothing is read there)
            if (left > -16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(left > 0 ? p : p - 16), "r"(min(max(left, 0), 16)) : "memory");
            dst += threads * 16, p += threads * 16, left -= threads * 16;
        }
    };
    auto copy = [&](unsigned m, int stage) {
        if (m < rows && cols > 0) {
            uint32_t dst = ring_at + stage * stage_size;
            copy_row(dst, static_cast<const S*>(a.H) + first + (int64_t)m * a.ldh, sizeof(S));
            if (a.dHo) copy_row(dst + at_d, static_cast<const S*>(a.dHo) + first + (int64_t)m * a.lddho, sizeof(S));
            if (a.dX) copy_row(dst + at_x, a.dX + first + (int64_t)m * a.lddx, 2);
            copy_row(dst + at_b, a.B + first + (int64_t)m * a.ldb, 2);
            if (GATE == 2) copy_row(dst + at_g, a.gate + first + (int64_t)m * a.ldg, 2);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto landed = [&](int pending) {  // all but the newest `pending` copies of this thread have arrived
        if (pending >= 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
        else if (pending == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else if (pending == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
    };
    auto stream_cols = [&](const uint8_t* p, int j, Cols& v) {
        const int at = (j * threads + tid) * 8;
        if (sizeof(S) == 2) {
            cols_bf16(*reinterpret_cast<const uint4*>(p + at * 2), v);
        } else {
            const float4 q = *reinterpret_cast<const float4*>(p + at * 4), t = *reinterpret_cast<const float4*>(p + at * 4 + 16);
            v[0] = pair(q.x, q.y), v[1] = pair(q.z, q.w), v[2] = pair(t.x, t.y), v[3] = pair(t.z, t.w);
        }
    };
    auto half_cols = [&](const uint8_t* p, int j, Cols& v) { cols_bf16(*reinterpret_cast<const uint4*>(p + (j * threads + tid) * 16), v); };

    unsigned m = blockIdx.x / CS, ahead = m;  // this row, and the next one to copy
    for (int d = 0; d < a.depth - 1; ++d, ahead += groups) copy(ahead, d);

    const float inv_k = 1.0f / (float)a.K;
    uint4 wpre[VPT];   // gamma_pre, bf16 as it lies in memory
    Cols scale[VPT];   // alpha gamma_post, times the channel gate's function
    Cols acc_pre[VPT], acc_post[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        Raw8<__nv_bfloat16> r;
        const int col = first + (j * threads + tid) * 8;
        wpre[j] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc_pre[j][i] = acc_post[j][i] = 0, scale[j][i] = both(a.alpha);
        if (n[j] <= 0) continue;
        if (a.dX) r.load(a.gamma_pre + col, n[j]), wpre[j] = r.q;
        Cols w;
        if (POST) {
            r.load(a.gamma_post + col, n[j]);
            cols_of(r, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) scale[j][i] = mul2(scale[j][i], w[i]);
        }
        if (GATE == 1) {
            Cols slope;
            r.load(a.gate + col, n[j]);
            cols_of(r, w);
            gate_cols(a.sigmoid, w, slope);
#pragma unroll
            for (int i = 0; i < 4; ++i) scale[j][i] = mul2(scale[j][i], w[i]);
        }
    }
    // sums of the row in stage p: H'^2, dX gamma_pre H', B^2
    auto first_sums = [&](const uint8_t* p, float (&s)[4]) {
        uint64_t sh = 0, su = 0, sb = 0;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            if (n[j] <= 0) continue;
            Cols h, u, w;
            stream_cols(p, j, h);
#pragma unroll
            for (int i = 0; i < 4; ++i) sh = fma2(h[i], h[i], sh);
            if (a.dX) {
                half_cols(p + at_x, j, u);
                cols_bf16(wpre[j], w);
#pragma unroll
                for (int i = 0; i < 4; ++i) su = fma2(mul2(u[i], w[i]), h[i], su);
            }
            if (POST) {
                half_cols(p + at_b, j, u);
#pragma unroll
                for (int i = 0; i < 4; ++i) sb = fma2(u[i], u[i], sb);
            }
        }
        s[0] = sum2(sh), s[1] = sum2(su), s[2] = sum2(sb);
    };

    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    int stage = 0, flip = 0;
    landed(a.depth - 2);
    __syncthreads();
    if (m < rows) first_sums(ring, s);
    landed(a.depth - 3);
    if (CS > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    row_sum<4, CS>(s, red[0], xred[0]);
    for (; m < rows; m += groups) {
        const float r = rsqrtf(s[0] * inv_k + a.eps);
        const float c = -s[1] * r * inv_k * r * r;  // - mean(u xhat) r, per unit of H'
        const float rp = POST ? rsqrtf(s[2] * inv_k + a.eps) : 1.0f;
        // into the stage of the row before, which every thread has left
        copy(ahead, stage == 0 ? a.depth - 1 : stage - 1);
        ahead += groups;
        const uint8_t* p = ring + (size_t)stage * stage_size;
        Cols v[VPT], nb[VPT];  // gradient of the normalised branch, and that branch
        uint64_t t2 = 0;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            if (n[j] <= 0) continue;
            const int col = first + (j * threads + tid) * 8;
            Cols d;
            if (a.dHo) {
                stream_cols(p + at_d, j, d);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] = 0;
            }
            if (a.dX) {
                Cols h, u, w;
                stream_cols(p, j, h);
                half_cols(p + at_x, j, u);
                cols_bf16(wpre[j], w);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint64_t ur = mul2(u[i], both(r));
                    acc_pre[j][i] = fma2(ur, h[i], acc_pre[j][i]);
                    d[i] = fma2(ur, w[i], fma2(both(c), h[i], d[i]));
                }
            }
            store_cols(static_cast<S*>(a.dH) + (int64_t)m * a.lddh + col, d, n[j]);
            half_cols(p + at_b, j, nb[j]);
            Cols G, dg;
            if (GATE == 2) {
                half_cols(p + at_g, j, G);
                gate_cols(a.sigmoid, G, dg);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (POST) nb[j][i] = mul2(nb[j][i], both(rp));
                const uint64_t dn = mul2(d[i], nb[j][i]);
                v[j][i] = mul2(d[i], scale[j][i]);
                if (GATE == 2) {
                    acc_post[j][i] = fma2(dn, G[i], acc_post[j][i]);
                    dg[i] = mul2(mul2(dn, scale[j][i]), dg[i]);
                    v[j][i] = mul2(v[j][i], G[i]);
                } else {
                    acc_post[j][i] = add2(acc_post[j][i], dn);
                }
                if (POST) t2 = fma2(v[j][i], nb[j][i], t2);
            }
            if (GATE == 2) store_cols(a.dgate + (int64_t)m * a.lddg + col, dg, n[j]);
            if (!POST) store_cols(a.dB + (int64_t)m * a.lddb + col, v[j], n[j]);
        }
        if (++stage == a.depth) stage = 0;
        s[0] = s[1] = s[2] = 0.0f;
        s[3] = sum2(t2);
        if (m + groups < rows) first_sums(ring + (size_t)stage * stage_size, s);
        landed(a.depth - 3);  // the row after the next: visible to all behind the barrier
        flip ^= 1;
        row_sum<4, CS>(s, red[flip], xred[flip]);
        if (POST) {
            const float q = -s[3] * inv_k;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                if (n[j] <= 0) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j][i] = mul2(both(rp), fma2(both(q), nb[j][i], v[j][i]));
                store_cols(a.dB + (int64_t)m * a.lddb + first + (j * threads + tid) * 8, v[j], n[j]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        if (n[j] <= 0) continue;
        // a partial row is padded to whole vectors; a result (one group) ends with column K - 1 and starts on any float
        auto put = [&](int which, const Cols& v) {
            if (!a.col[which]) return;
            float f[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) unpair(v[i], f[2 * i], f[2 * i + 1]);
            float* p = a.col[which] + (blockIdx.x / CS) * a.pitch + first + (j * threads + tid) * 8;
            if (groups > 1) {  // wide stores (single floats at a stride of 8 cost 4 us at 148 x 5003)
                store8(p, f, 8);
                return;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n[j]) p[i] = f[i];
        };
        put(0, acc_pre[j]);
        if (!POST && GATE != 1) continue;
        // acc_post: the column sum of d n (times the gate, if it has one per token)
        Raw8<__nv_bfloat16> r;
        const int col = first + (j * threads + tid) * 8;
        Cols w, G, slope, x;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = G[i] = both(1.0f);
        if (POST) r.load(a.gamma_post + col, n[j]), cols_of(r, w);
        if (GATE == 1) r.load(a.gate + col, n[j]), cols_of(r, G), gate_cols(a.sigmoid, G, slope);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t sum = mul2(acc_post[j][i], both(a.alpha));
            if (GATE == 1) x[i] = mul2(mul2(sum, slope[i]), w[i]);
            acc_post[j][i] = mul2(sum, G[i]);
        }
        if (POST) put(1, acc_post[j]);
        if (GATE == 1) put(2, x);
    }
    if (CS > 1) {  // no CTA leaves while a peer may still write its shared memory
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
}

// Sum of the P partial rows: a block owns 32 columns, each of its warps adds a contiguous run of rows with 16 loads in flight,
// and the warps' sums are added in order.  Latency: 16 warps (148 x 5003: 3 us less than with 32, whose blocks do not all fit on
// the device at once); more than 512 rows (short rows: up to 16 CTAs per SM) go to clusters of four or eight such blocks (16384 x
// 256: 22.7 us in all, 28.8 with one block of 32 warps).
constexpr int kSumWarps = 16;
struct JoinSum {
    const float* part[3];
    float* out[3];
    int64_t pitch;
    int P, K;
};
template <int CS>
__global__ void __launch_bounds__(kSumWarps * 32) join_sum_kernel(const __grid_constant__ JoinSum a) {
    __shared__ float buf[kSumWarps][32], sum[32];
    pdl_wait();
    pdl_trigger();
    const int rank = CS > 1 ? (int)(blockIdx.x % CS) : 0;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, col = (int)(blockIdx.x / CS) * 32 + lane, which = blockIdx.y;
    const int per = (a.P + kSumWarps * CS - 1) / (kSumWarps * CS), p0 = (rank * kSumWarps + w) * per, p1 = min(a.P, p0 + per);
    float s = 0.0f;
    if (col < a.K) {
        const float* src = a.part[which] + col;
        for (int p = p0; p < p1; p += 16) {
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = p + i < p1 ? src[(p + i) * a.pitch] : 0.0f;
#pragma unroll
            for (int o = 8; o > 0; o /= 2)
#pragma unroll
                for (int i = 0; i < o; ++i) v[i] += v[i + o];
            s += v[0];
        }
    }
    buf[w][lane] = s;
    __syncthreads();
    float t = 0.0f;
    if (w == 0) {
#pragma unroll
        for (int i = 0; i < kSumWarps; ++i) t += buf[i][lane];
        sum[lane] = t;
    }
    if (CS > 1) {
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        if (w == 0 && rank == 0) {
            t = 0.0f;
            float v[CS];
#pragma unroll
            for (int c = 0; c < CS; ++c) {
                uint32_t at;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(sum + lane)), "r"(c));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[c]) : "r"(at) : "memory");
            }
#pragma unroll
            for (int c = 0; c < CS; ++c) t += v[c];
        }
    }
    if (w == 0 && rank == 0 && col < a.K) a.out[which][col] = t;
    if (CS > 1) {  // no CTA leaves while the first one may still read its shared memory
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
}

// ---- host side -----------------------------------------------------------------------------------
// Split of a row: vectors per thread, CTAs, threads; CTAs per SM (each holds at least three rows
// in shared memory, for which long rows are split further); groups of CTAs that share the rows.
constexpr int kSmemSm = 224 * 1024, kSmemStatic = 2048;
struct BwdShape {
    int vpt, cs, max, threads, per_sm, depth;
    int64_t groups;
};
BwdShape bwd_shape(int64_t M, int64_t K, int stream_size, bool gate) {
    const int64_t vecs = (K + 7) / 8;
    BwdShape s;
    int stage = 0;
    // One CTA with one vector per thread, then with two, then clusters (4736 x 5003, gated: 85 us with one, 109 with two;
    // 4096 x 8192, channel gate: 96 us with two, 139 in a cluster of two).
    for (s.vpt = 1, s.cs = 1, s.max = kFewThreads;;) {
        const int64_t per = (int64_t)s.cs * s.vpt * 32;
        s.threads = (int)((vecs + per - 1) / per * 32);
        stage = stage_bytes(stream_size, gate, s.vpt * s.threads * 8);
        if (s.threads <= s.max && 3 * stage <= kSmemSm - kSmemStatic) break;
        if (s.cs > 1) s.cs *= 2;
        else if (s.vpt == 2) s.vpt = 1, s.cs = 2, s.max = kManyThreads;
        else if (s.max == kFewThreads) s.max = kManyThreads;
        else s.vpt = 2, s.max = kFewThreads;
    }
    s.per_sm = std::min(s.max / s.threads, kSmemSm / (3 * stage + kSmemStatic));
    s.depth = std::min(kMaxDepth, (kSmemSm / s.per_sm - kSmemStatic) / stage);
    s.groups = std::min<int64_t>(M, resident_clusters(s.cs) * s.per_sm);
    return s;
}
int64_t bwd_most_groups(int64_t M, int64_t K) {
    int64_t g = 0;
    for (int size = 2; size <= 4; size += 2)
        for (int gate = 0; gate < 2; ++gate) g = std::max(g, bwd_shape(M, K, size, gate).groups);
    return g;
}

template <typename S, bool POST, int GATE, int VPT, int CS, int MAX>
int launch_bwd(const BwdShape& s, JoinBwd a, cudaStream_t st) {
    auto kern = join_bwd_kernel<S, POST, GATE, VPT, CS, MAX>;
    const int smem = s.depth * stage_bytes(sizeof(S), GATE == 2, VPT * s.threads * 8);
    a.depth = s.depth;
    const int rc = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem, "join_bwd_kernel shared memory");
    if (rc) return rc;
    LaunchScope scope(kKindRow, st);
    return cuda_fail(launch_clusters(kern, (unsigned)(s.groups * CS), (unsigned)s.threads, (size_t)smem, CS, st, a),
                     "join_bwd_kernel launch");
}
template <typename S, bool POST, int GATE>
int launch_bwd(const BwdShape& s, const JoinBwd& a, cudaStream_t st) {
    if (s.vpt == 2) return launch_bwd<S, POST, GATE, 2, 1, kFewThreads>(s, a, st);
    switch (s.cs) {
        case 1:
            if (s.max == kFewThreads) return launch_bwd<S, POST, GATE, 1, 1, kFewThreads>(s, a, st);
            return launch_bwd<S, POST, GATE, 1, 1, kManyThreads>(s, a, st);
        case 2: return launch_bwd<S, POST, GATE, 1, 2, kManyThreads>(s, a, st);
        case 4: return launch_bwd<S, POST, GATE, 1, 4, kManyThreads>(s, a, st);
        default: return launch_bwd<S, POST, GATE, 1, 8, kManyThreads>(s, a, st);
    }
}
template <typename S>
int launch_bwd(const BwdShape& s, const JoinBwd& a, cudaStream_t st) {
    const int gate = !a.gate ? 0 : a.ldg == 0 ? 1 : 2;
    if (a.gamma_post) return gate == 0 ? launch_bwd<S, true, 0>(s, a, st) : gate == 1 ? launch_bwd<S, true, 1>(s, a, st) : launch_bwd<S, true, 2>(s, a, st);
    return gate == 0 ? launch_bwd<S, false, 0>(s, a, st) : gate == 1 ? launch_bwd<S, false, 1>(s, a, st) : launch_bwd<S, false, 2>(s, a, st);
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
    a.M = M, a.ldh = ldh, a.ldb = ldb, a.ldg = ldg, a.ldho = ldho, a.ldx = ldx;
    a.K = (int)K, a.sigmoid = gate_act == RESQ_GATE_SIGMOID, a.alpha = alpha, a.eps = eps;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    LaunchScope scope(kKindRow, st);
    return cuda_fail(stream_dtype == RESQ_OUT_F32 ? launch_fwd<float>(a, st) : launch_fwd<__nv_bfloat16>(a, st), "join_fwd_kernel launch");
}

size_t resq_block_join_backward_workspace_bytes(int64_t M, int64_t K) {
    if (M <= 0 || K <= 0 || K > RESQ_JOIN_MAX_K) return 0;
    return align_up((size_t)bwd_most_groups(M, K) * 3 * (size_t)((K + 7) / 8 * 8) * sizeof(float), 256);
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
    for (int64_t ld : {dH_out ? lddho : 0, dX ? lddx : 0, ldho, ldb, gate ? ldg : 0, lddh, lddb, gate && ldg != 0 ? lddg : 0})
        if (ld > INT32_MAX) return fail(RESQ_ERR_SHAPE, what, "a row pitch is 2^31 elements or more");
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
    a.lddho = (int)lddho, a.lddx = (int)lddx, a.ldh = (int)ldho, a.ldb = (int)ldb, a.ldg = (int)ldg;
    a.lddh = (int)lddh, a.lddb = (int)lddb, a.lddg = (int)lddg;
    a.M = (int)M, a.K = (int)K, a.sigmoid = gate_act == RESQ_GATE_SIGMOID, a.alpha = alpha, a.eps = eps;
    const BwdShape shape = bwd_shape(M, K, stream_dtype == RESQ_OUT_F32 ? 4 : 2, gate && ldg != 0);
    float* const results[3] = {dX ? dgamma_pre : nullptr, gamma_post ? dgamma_post : nullptr,
                               gate && ldg == 0 ? static_cast<float*>(dgate) : nullptr};
    a.pitch = (K + 7) / 8 * 8;
    JoinSum s;
    int ncol = 0;
    for (int i = 0; i < 3; ++i) {
        a.col[i] = results[i];
        if (!results[i] || shape.groups == 1) continue;  // one group of CTAs: its sums are the results
        a.col[i] = static_cast<float*>(workspace) + (int64_t)ncol * shape.groups * a.pitch;
        s.part[ncol] = a.col[i], s.out[ncol++] = results[i];
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    rc = stream_dtype == RESQ_OUT_F32 ? launch_bwd<float>(shape, a, st) : launch_bwd<__nv_bfloat16>(shape, a, st);
    if (rc || ncol == 0) return rc;
    s.pitch = a.pitch, s.P = (int)shape.groups, s.K = (int)K;
    LaunchScope scope(kKindRow, st);
    const int cs = s.P > 1024 ? 8 : s.P > 512 ? 4 : 1;
    return cuda_fail(launch_clusters(cs == 8 ? join_sum_kernel<8> : cs == 4 ? join_sum_kernel<4> : join_sum_kernel<1>,
                                     dim3((unsigned)((K + 31) / 32) * cs, (unsigned)ncol), kSumWarps * 32, 0, cs, st, s),
                     "join_sum_kernel launch");
}
}
