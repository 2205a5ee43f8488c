// resq_rope_append: from the qkv projection's rows to rotated queries and to keys and values in their slots of a paged cache.
//
//   x = qkv + bias;  token i of sequence b stands at pos = kv_len[b] - n_b + i;  pair (a, b) of frequency j turns by pos inv_freq_j:
//   a' = a cos - b sin,  b' = b cos + a sin;  values and elements from `rot` on are copied
//
// Angles.  pos inv_freq in fp32 is off by 0.03 rad half a million tokens into a sequence.  inv_freq / 2 pi is turned into a 64-bit
// fraction of a turn instead (once per angle; a product of fp64 numbers keeps 53 bits, too few times a position of 2^31, so its
// second half and that of 1 / 2 pi are added), within 2 2^-64, and pos times that fraction modulo 2^64 is the angle within 2^-32 of a
// turn.  Its top 32 bits, as a signed number of half turns, go to sincospi in fp32: 2^-26 of a turn, or 1.6 2^-24 rad, at every position.
//
// Bound by HBM: every element is read and written once.  A block takes one to eight tokens; its threads first compute the tokens'
// sines and cosines (two each for eight tokens of 128-wide heads, shared by all heads), with their first elements already on the
// way, then take 16 elements each: the two runs of 8 that turn into each other.  Measured: 16384 tokens of 28 + 2 x 4 heads of 128, bf16 with
// bias, 54.5 us = 5.5 TB/s (0.85 of the copy rate); one token 2.9 us.
#include "paged.cuh"

#include <algorithm>

namespace resq {
namespace {

constexpr int kThreads = 256, kMaxTokens = 8;  // a warp looks up each token

struct RopeArgs {
    SeqArgs seq;
    const void* qkv;
    const __nv_bfloat16* bias;  // or null
    const double* inv_freq;     // [rot / 2]
    const int32_t* positions;   // [T] or null
    __nv_bfloat16 *q, *k, *v;
    int64_t ldqkv, ldq, k_page, k_row, k_head, v_page, v_row, v_head;
    int Hq, Hkv, rot, pairs, tokens;  // tokens per block
    FastDiv by_token;                 // shares per token
};

struct Place {
    int there;  // the row belongs to a sequence
    int pos;    // position that the rotation takes
    int page;   // of the token's slot; -1: none
    int row;    // in the page
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) rope_append_kernel(const __grid_constant__ RopeArgs a) {
    constexpr int C = D / 16;  // threads' shares per head
    __shared__ Place place[kMaxTokens];
    __shared__ int owner[kMaxTokens];
    __shared__ __align__(16) float cs[kMaxTokens][D / 2], sn[kMaxTokens][D / 2];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int64_t t0 = (int64_t)blockIdx.x * a.tokens;
    const int nt = (int)min((int64_t)a.tokens, a.seq.T - t0);
    pdl_wait();
    pdl_trigger();
    // ---- whose token it is: up to 128 sequences are all asked, by a warp per token
    const bool few = a.seq.B <= 128;
    bool lost = false;
    auto place_of = [&](int b) {  // of token t0 + w, if it is sequence b's
        Place p{0, 0, -1, 0};
        if (b >= a.seq.B) return p;
        const Seq s = load_seq(a.seq, b);
        const int tok = (int)t0 + w, i = tok - s.q0;
        if (i < 0 || i >= s.n) return p;
        const int slot = s.kv - s.n + i;
        p.there = 1;
        p.pos = a.positions ? a.positions[tok] : slot;
        if (slot >= 0) p.page = page_of(a.seq, b, slot, p.row);
        return p;
    };
    if (w < nt && few) {
        int from[4], to[4], b = a.seq.B;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            from[k] = to[k] = 0;
            if (k * 32 + lane < a.seq.B) from[k] = a.seq.q_start[k * 32 + lane], to[k] = a.seq.q_start[k * 32 + lane + 1];
        }
#pragma unroll
        for (int k = 3; k >= 0; --k) {
            const unsigned here = __ballot_sync(~0u, t0 + w >= from[k] && t0 + w < to[k]);
            if (here) b = k * 32 + __ffs(here) - 1;
        }
        const Place p = place_of(b);
        if (lane == 0) place[w] = p;
    } else if (w < nt) {  // more are searched, 32 starts at a time
        const int tok = (int)t0 + w;
        int lo = 0, hi = a.seq.B;  // the last b in lo .. hi with q_start[b] <= tok
        while (hi > lo) {
            const int step = (hi - lo + 31) / 32, b = min(lo + 1 + lane * step, hi);
            // Starts out of order make the answers disagree: only their first run counts here.
            const unsigned upto = __ballot_sync(~0u, a.seq.q_start[b] <= tok);
            const int n = upto == ~0u ? 32 : __ffs(~upto) - 1;
            const int at = n == 0 ? lo : min(lo + 1 + (n - 1) * step, hi);
            hi = n == 32 ? hi : min(lo + n * step, hi);
            if (step == 1 || at == hi) {
                lo = at;
                break;
            }
            lo = at;
        }
        const Place p = place_of(lo);
        lost = !p.there;
        if (lane == 0) place[w] = p;
    }
    // Starts out of order, or rows of no sequence (a padded batch has them): then all are asked, once for the block's tokens (1.5 us of 8 at
    // 256 sequences and 4096 tokens, nearly all of them padding).
    if (few) __syncthreads();
    else if (__syncthreads_or(lost)) {
        if (tid < kMaxTokens) owner[tid] = a.seq.B;
        __syncthreads();
        for (int b0 = tid; b0 < a.seq.B; b0 += 4 * kThreads) {
            int from[4], to[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int b = min(b0 + k * kThreads, a.seq.B - 1);
                from[k] = a.seq.q_start[b], to[k] = a.seq.q_start[b + 1];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                for (int64_t t = max((int64_t)from[k] - t0, (int64_t)0); t < nt && t0 + t < to[k]; ++t)
                    atomicMin(&owner[t], min(b0 + k * kThreads, a.seq.B - 1));
        }
        __syncthreads();
        if (lost) {
            const Place p = place_of(owner[w]);
            if (lane == 0) place[w] = p;
        }
        __syncthreads();
    }
    const int heads = a.Hq + 2 * a.Hkv, per_token = heads * C, items = nt * per_token;
    const int half = a.rot / 2, turning = a.rot / 16;
    // the two runs of 8 elements of a share, within its head
    auto runs = [&](int head, int c, int& e0, int& e1) {
        const bool far = !a.pairs && head < a.Hq + a.Hkv && c < turning;
        e0 = far ? c * 8 : c * 16;
        e1 = far ? half + c * 8 : c * 16 + 8;
    };
    auto fetch = [&](int it, Raw8<T>& x, Raw8<T>& y) {
        const int tok = (int)div_by((uint32_t)it, a.by_token), r = it - tok * per_token, head = r / C;
        int e0, e1;
        runs(head, r % C, e0, e1);
        const T* row = static_cast<const T*>(a.qkv) + (t0 + tok) * a.ldqkv + head * D;
        x.load(row + e0, 8);
        y.load(row + e1, 8);
    };
    constexpr int N = sizeof(T) == 2 ? 3 : 2;  // shares whose loads are in flight
    Raw8<T> x[N], y[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (tid + i * kThreads < items) fetch(tid + i * kThreads, x[i], y[i]);
    // ---- sines and cosines
    for (int i = tid; i < nt * half; i += kThreads) {
        const int tok = i / half, j = i - tok * half;
        const double inv = a.inv_freq[j], mag = fabs(inv), k2Pi = 0.15915494309189535, kLow2Pi = -9.839338337591243e-18;  // 1 / 2 pi
        const double f = mag * k2Pi, low = fma(mag, k2Pi, -f) + mag * kLow2Pi, k64 = 18446744073709551616.0;
        const unsigned long long part = (unsigned long long)((f - floor(f)) * k64) + (unsigned long long)(long long)(low * k64);
        const unsigned long long turn = (inv < 0.0 ? 0ull - part : part) * (unsigned long long)(long long)place[tok].pos;
        sincospif((float)(int)(unsigned)(turn >> 32) * 4.656612873077393e-10f, &sn[tok][j], &cs[tok][j]);  // 2^-31: in half turns
    }
    __syncthreads();
    for (int base = tid; base < items; base += N * kThreads) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int it = base + i * kThreads;
            if (it >= items) break;
            const int tok = (int)div_by((uint32_t)it, a.by_token), r = it - tok * per_token, head = r / C, c = r % C;
            int e0, e1;
            runs(head, c, e0, e1);
            const Place p = place[tok];
            float u[8], v[8];
            x[i].get(u);
            y[i].get(v);
            if (it + N * kThreads < items) fetch(it + N * kThreads, x[i], y[i]);
            if (!p.there) continue;
            if (a.bias) {
                float b0[8], b1[8];
                Raw8<__nv_bfloat16> rb;
                rb.load(a.bias + head * D + e0, 8);
                rb.get(b0);
                rb.load(a.bias + head * D + e1, 8);
                rb.get(b1);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] += b0[e], v[e] += b1[e];
            }
            if (head < a.Hq + a.Hkv && c < turning) {
                float co[8], si[8];
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    const float4 p4 = *reinterpret_cast<const float4*>(&cs[tok][c * 8 + e]), s4 = *reinterpret_cast<const float4*>(&sn[tok][c * 8 + e]);
                    co[e] = p4.x, co[e + 1] = p4.y, co[e + 2] = p4.z, co[e + 3] = p4.w;
                    si[e] = s4.x, si[e + 1] = s4.y, si[e + 2] = s4.z, si[e + 3] = s4.w;
                }
                if (a.pairs) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float f = u[2 * e], g = u[2 * e + 1];
                        u[2 * e] = f * co[e] - g * si[e], u[2 * e + 1] = g * co[e] + f * si[e];
                        f = v[2 * e], g = v[2 * e + 1];
                        v[2 * e] = f * co[4 + e] - g * si[4 + e], v[2 * e + 1] = g * co[4 + e] + f * si[4 + e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float f = u[e], g = v[e];
                        u[e] = f * co[e] - g * si[e], v[e] = g * co[e] + f * si[e];
                    }
                }
            }
            __nv_bfloat16* dst;
            if (head < a.Hq) dst = a.q + (t0 + tok) * a.ldq + head * D;
            else if (p.page < 0) continue;
            else if (head < a.Hq + a.Hkv) dst = a.k + (int64_t)p.page * a.k_page + (int64_t)p.row * a.k_row + (int64_t)(head - a.Hq) * a.k_head;
            else dst = a.v + (int64_t)p.page * a.v_page + (int64_t)p.row * a.v_row + (int64_t)(head - a.Hq - a.Hkv) * a.v_head;
            store8(dst + e0, u, 8);
            store8(dst + e1, v, 8);
        }
    }
}

}  // namespace
}  // namespace resq

using namespace resq;

extern "C" int resq_rope_append(const void* QKV, int dtype, int64_t T, int64_t ldqkv, int64_t Hq, int64_t Hkv, int64_t D, const void* bias_bf16,
                                const double* inv_freq, int64_t rot, int pairs, const int32_t* positions, const resq_paged_cache* cache,
                                const resq_sequences* seqs, void* Q, int64_t ldq, void* stream) {
    const char* what = "rope_append";
    if (!QKV || !Q || (rot > 0 && !inv_freq)) return fail(RESQ_ERR_NULL, what, "QKV, Q and inv_freq must not be NULL");
    if (dtype != RESQ_OUT_BF16 && dtype != RESQ_OUT_F32) return fail(RESQ_ERR_PATTERN, what, "unknown type of QKV");
    int rc = check_paged(what, cache, seqs, T, Hq, Hkv, D);
    if (rc) return rc;
    // Slots that share memory would be written by several threads: slots of one kind lie D apart or more.
    auto apart = [&](int64_t page, int64_t row, int64_t head) {
        return (cache->pages == 1 || page >= D) && (cache->page_size == 1 || row >= D) && (Hkv == 1 || head >= D);
    };
    if (!apart(cache->k_page, cache->k_row, cache->k_head) || !apart(cache->v_page, cache->v_row, cache->v_head))
        return fail(RESQ_ERR_ALIGN, what, "pages, rows and heads of a cache that is written to must not share memory");
    if (rot < 0 || rot > D || rot % 16) return fail(RESQ_ERR_SHAPE, what, "rot must be a multiple of 16 up to the head's width");
    if ((Hq + 2 * Hkv) * D > INT32_MAX / 8) return fail(RESQ_ERR_SHAPE, what, "too many heads");
    if (!rows_aligned(QKV, ldqkv, (Hq + 2 * Hkv) * D, dtype) || !rows_aligned(Q, ldq, Hq * D, RESQ_OUT_BF16))
        return fail(RESQ_ERR_ALIGN, what, "QKV and Q need 16-byte aligned bases and rows that hold their heads");
    if (!is_aligned(bias_bf16, 16) || !is_aligned(inv_freq, 8) || !is_aligned(positions, 4))
        return fail(RESQ_ERR_ALIGN, what, "bias must be 16-byte aligned, inv_freq 8-byte, positions 4-byte");
    using bf = __nv_bfloat16;
    RopeArgs a;
    a.seq = seq_args(*cache, *seqs, T);
    a.qkv = QKV, a.bias = static_cast<const bf*>(bias_bf16), a.inv_freq = inv_freq, a.positions = positions;
    a.q = static_cast<bf*>(Q), a.k = static_cast<bf*>(cache->k), a.v = static_cast<bf*>(cache->v);
    a.ldqkv = ldqkv, a.ldq = ldq;
    a.k_page = cache->k_page, a.k_row = cache->k_row, a.k_head = cache->k_head;
    a.v_page = cache->v_page, a.v_row = cache->v_row, a.v_head = cache->v_head;
    a.Hq = (int)Hq, a.Hkv = (int)Hkv, a.rot = (int)rot, a.pairs = pairs != 0;
    // One token per block until the device is full, then up to eight: fewer blocks to start and an even number of shares per thread
    // (16384 tokens of 36 heads: 85 us with two, 58.8 with four, 54.4 with eight).
    a.tokens = (int)std::min<int64_t>(kMaxTokens, std::max<int64_t>(1, T / (148 * 4)));
    a.by_token = fast_div((uint32_t)((Hq + 2 * Hkv) * (D / 16)));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    LaunchScope scope(kKindRow, st);
    auto kern = dtype == RESQ_OUT_F32 ? (D == 128 ? rope_append_kernel<float, 128> : rope_append_kernel<float, 64>)
                                      : (D == 128 ? rope_append_kernel<bf, 128> : rope_append_kernel<bf, 64>);
    return cuda_fail(launch_kernel(kern, dim3((unsigned)((T + a.tokens - 1) / a.tokens)), dim3(kThreads), 0, st, a), "rope_append_kernel launch");
}
