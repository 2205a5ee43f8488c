// resq_verify_drafts: which drafted tokens a sequence keeps, and the token that takes the place of the first one it does not keep.
//
//   row r of a sequence: target p = softmax(logits_r / T), draft x_r proposed with q = exp((draft_logits - draft_peak) / T -
//   draft_log_sum), or with certainty; x_r is kept while all before it are and u_r q(x_r) < p(x_r)
//   at the first row that is not kept (the last row proposes nothing): argmax_j w_j / e_j over w = max(p - q, 0), or w = p where
//   nothing was proposed; e are exponential variates, so token j is drawn with probability w_j / sum w
//
// The rows' sums are resq_token_logprobs' kernel, one pass over the logits, which is what the call is bound by.  This file's kernel
// then needs one row per sequence again (of the logits, the draft's logits and e): a cluster of 1 to 8 CTAs per sequence finds the
// row and takes the largest w / e of its slices.  Measured: 64 sequences of 5 rows of 131072, bf16, 43.8 us (rows and
// both launches 28.7, the deciding row 2, the drawing 13 for 67 MB, 10.2 of them at the copy rate); one such sequence 13.6 us, latency of
// both.
//
// Decisions that 32 bits leave open are made in 64 bits: a probability next to its border, and a drawing where another ratio may be
// the largest, or where nothing may be left of p - q.  What 32 bits can be off by is below.
#include "row_common.cuh"

#include <algorithm>
#include <cmath>

namespace resq {
namespace {

constexpr float kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 512;  // at most
// The argument of an exponential of 2 is a sum of two terms of one sign with six roundings of 2^-24 at most on the way of each, and
// weights down to 2^-126 count: it is off by 6 * 127 * 2^-24 = 4.6e-5 at most, and a fast exponential and log_sum / ln 2 add
// 1.3e-6.  kSlack, 2^-14 in the exponent, is above that: 2^(y + kSlack) is an upper bound of p, 2^(y - kSlack) a lower one.
constexpr float kSlack = 6.103515625e-05f;
// Ratios p / e, off by less than 2^-14.5 of themselves each: the largest is the largest if the next one is this far below.
constexpr float kNear = 6.103515625e-05f;
// Ratios (p - q) / e have no such bound, since little may be left of p.  The pass takes upper bounds of p - q, leaves out what lies
// more than kWide below the largest, and the largest's lower bound then says whether another one reaches it (or one left out may).
// Where more than 1/370 of p is left it is mostly clear; with less the row is read again.
constexpr float kWide = 0.0625f, kFold = 1.9073486328125e-06f;  // 2^-19: what the quotients and their bounds are rounded by, several times over
// log p and log q are off by at most 7 * 2^-24 of themselves and of each other, which matters where both are far below 0.
constexpr float kNearLog = 4.76837158203125e-07f;  // 2^-21

struct VerifyArgs {
    const void *logits, *draft_logits;
    int64_t ld, ldd, lde;
    const int32_t* row_start;
    const int64_t* drafts;
    const float *u, *e, *draft_peak, *draft_log_sum;
    const float *logp, *peak, *log_sum;        // of the target's rows for the drafts
    const int32_t* best;                       // greedy: the largest logit of every row, and its log-probability
    const float* best_logp;
    int32_t* accepted;
    int64_t* tokens;
    float* out_logp;
    DeviceStatus* status;
    int B, R, V, slice;  // slice: vectors of 8 per CTA
    float inv_t;
    double inv_t64;
};

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {  // NaN is passed over
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float warp_max(float v) {  // NaN is passed over
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float value(const float* p) { return *p; }

struct Best {
    float s;     // largest ratio; 0: none
    int j;       // its lowest place
    float next;  // the largest of the others
};
__device__ __forceinline__ Best join(const Best& p, const Best& q) {
    const bool p_first = p.s > q.s || (p.s == q.s && p.j < q.j);
    Best r = p_first ? p : q;
    r.next = fmaxf(fmaxf(p.next, q.next), p_first ? q.s : p.s);
    return r;
}
struct Best64 {
    double s;
    int j;
};
__device__ __forceinline__ Best64 join(const Best64& p, const Best64& q) { return p.s > q.s || (p.s == q.s && p.j < q.j) ? p : q; }

__device__ __forceinline__ Best shuffle(const Best& b, int o) {
    return Best{__shfl_xor_sync(~0u, b.s, o), __shfl_xor_sync(~0u, b.j, o), __shfl_xor_sync(~0u, b.next, o)};
}
__device__ __forceinline__ Best64 shuffle(const Best64& b, int o) { return Best64{__shfl_xor_sync(~0u, b.s, o), __shfl_xor_sync(~0u, b.j, o)}; }

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
template <typename W>
__device__ __forceinline__ W remote(const W* p, int rank) {
    static_assert(sizeof(W) % 4 == 0, "");
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    W v;
    uint32_t* dst = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int i = 0; i < (int)sizeof(W) / 4; ++i)
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(dst[i]) : "r"(at + 4 * i) : "memory");
    return v;
}
// The largest over the cluster, the same in all threads.  `warps` and `mine` in shared memory, not used by the call before.
template <typename W>
__device__ W cluster_best(W b, W* warps, W* mine, int cs) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) b = join(b, shuffle(b, o));
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = b;
    __syncthreads();
    b = warps[0];
    for (int i = 1; i < (int)(blockDim.x >> 5); ++i) b = join(b, warps[i]);
    if (cs == 1) return b;
    if (threadIdx.x == 0) *mine = b;
    cluster_sync();
    b = remote(mine, threadIdx.x & (cs - 1));  // cs is a power of two
    for (int o = 1; o < cs; o <<= 1) b = join(b, shuffle(b, o));
    return b;
}

// This thread's largest ratio in 64 bits, among the places from j0 to j1 - 1 of row r whose ratio in 32 bits reaches `low`.  Rare:
// kept out of the pass, whose registers it would take.
template <typename T, bool DRAFT>
__device__ __noinline__ Best64 best64(const VerifyArgs& a, int r, int b, int j0, int j1, bool minus, int skip, float low) {
    const T* const x = static_cast<const T*>(a.logits) + (int64_t)r * a.ld;
    const T* const xd = DRAFT ? static_cast<const T*>(a.draft_logits) + (int64_t)r * a.ldd : nullptr;
    const float* const e = a.e + (int64_t)b * a.lde;
    const float c = a.inv_t * kLog2e, peak = a.peak[r], log_sum = a.log_sum[r];
    const float dpeak = DRAFT && minus ? a.draft_peak[r] : 0.0f, dlog_sum = DRAFT && minus ? a.draft_log_sum[r] : 0.0f;
    const float add = -log_sum * kLog2e + kSlack, dadd = -dlog_sum * kLog2e - kSlack;
    Best64 best{0.0, a.V};
#pragma unroll 4
    for (int j = j0 + (int)threadIdx.x; j < j1; j += (int)blockDim.x) {
        const float z = value(x + j), zd = DRAFT && minus ? value(xd + j) : 0.0f, ev = e[j];
        float w = ex2(fmaf(z - peak, c, add));
        if (DRAFT && minus) w -= ex2(fmaf(zd - dpeak, c, dadd));
        if (!(w >= low * ev) || j == skip) continue;
        double w64 = exp(((double)z - (double)peak) * a.inv_t64 - (double)log_sum);
        if (DRAFT && minus) w64 -= exp(((double)zd - (double)dpeak) * a.inv_t64 - (double)dlog_sum);
        if (w64 > 0.0) best = join(best, Best64{w64 / (double)ev, j});
    }
    return best;
}

template <typename T, bool DRAFT, bool GREEDY>
__global__ void __launch_bounds__(kThreads, 2) verify_kernel(const __grid_constant__ VerifyArgs a) {
    __shared__ Best warp_best[kThreads / 32], cta_best;
    __shared__ Best64 warp_best64[kThreads / 32], cta_best64;
    uint32_t cs, rank = 0;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
    if (cs > 1) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x, b = blockIdx.x / cs;
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && tid == 0) *a.status = DeviceStatus{RESQ_OK, 0, 0, 0};
    const int r0 = min(max(a.row_start[b], 0), a.R), n = max(min(max(a.row_start[b + 1], 0), a.R) - r0, 0);
    if (n == 0) {  // the cluster's CTAs alike
        if (rank == 0 && tid == 0) a.accepted[b] = 0;
        return;
    }
    const float c = a.inv_t * kLog2e;
    // ---- the first row that is not kept; every warp for itself
    int kept = 0;
    bool proposed = false;  // something was proposed at that row
    for (int i0 = 0;; i0 += 32) {
        const int i = i0 + lane, r = r0 + i;
        bool keep = false, some = false;
        if (i < n - 1) {
            const int64_t x = a.drafts[r];
            some = x >= 0 && x < a.V;
            if (some && GREEDY) keep = x == a.best[r] && a.best_logp[r] > -kInf;  // not of a row of NaN
            else if (some) {
                const float logp = a.logp[r], u = a.u[r];
                float logq = 0.0f, xd = 0.0f;
                if (DRAFT) {
                    xd = value(static_cast<const T*>(a.draft_logits) + (int64_t)r * a.ldd + x);
                    logq = (xd - a.draft_peak[r]) * a.inv_t - a.draft_log_sum[r];
                }
                const float ratio = ex2((logp - logq) * kLog2e);
                keep = u < ratio && logp > -kInf;
                if (fabsf(u - ratio) <= (kNear + kNearLog * (fabsf(logp) + fabsf(logq))) * ratio) {
                    const double lp = ((double)value(static_cast<const T*>(a.logits) + (int64_t)r * a.ld + x) - (double)a.peak[r]) * a.inv_t64 - (double)a.log_sum[r];
                    const double lq = DRAFT ? ((double)xd - (double)a.draft_peak[r]) * a.inv_t64 - (double)a.draft_log_sum[r] : 0.0;
                    keep = (double)u < exp(lp - lq) && logp > -kInf;
                }
            }
        }
        const unsigned all = __ballot_sync(~0u, keep), had = __ballot_sync(~0u, some);
        if (all != ~0u) {
            const int at = __ffs(~all) - 1;
            kept = i0 + at;
            proposed = (had >> at) & 1;
            break;
        }
    }
    const int r = r0 + kept;
    // ---- the token at that row
    int64_t token = -1;
    float token_logp = 0.0f;
    if (GREEDY) {
        const float lp = a.best_logp[r];
        if (lp == lp && lp > -kInf) token = a.best[r], token_logp = lp;
    } else {
        const T* const x = static_cast<const T*>(a.logits) + (int64_t)r * a.ld;
        const T* const xd = DRAFT ? static_cast<const T*>(a.draft_logits) + (int64_t)r * a.ldd : nullptr;
        const float* const e = a.e + (int64_t)b * a.lde;
        const bool less = DRAFT && proposed;
        const float peak = a.peak[r], log_sum = a.log_sum[r], add = -log_sum * kLog2e + (less ? kSlack : 0.0f);
        const float dpeak = DRAFT ? a.draft_peak[r] : 0.0f, dadd = DRAFT ? -a.draft_log_sum[r] * kLog2e - kSlack : 0.0f;
        const int sure = !DRAFT && proposed ? (int)a.drafts[r] : -1;  // q is 1 there
        const int v0 = min((int)rank * a.slice, (a.V + 7) / 8), v1 = min(v0 + a.slice, (a.V + 7) / 8);
        const uint64_t c2 = pair(c, c), peak2 = pair(-peak, -peak), add2c = pair(add, add), dpeak2 = pair(-dpeak, -dpeak), dadd2 = pair(dadd, dadd);
        const uint64_t minus1 = pair(-1.0f, -1.0f);
        auto weights = [&](uint64_t z, uint64_t zd) {  // of two places; of p - q upper bounds, below 0 where p < q
            float l, h;
            unpair(fma2(add2(z, peak2), c2, add2c), l, h);
            const uint64_t p = pair(ex2(l), ex2(h));
            if (!less) return p;
            unpair(fma2(add2(zd, dpeak2), c2, dadd2), l, h);
            return fma2(pair(ex2(l), ex2(h)), minus1, p);
        };
        // take(j, weights, e) for eight of this thread's places after the other, the next ones' loads ahead; all lanes of a warp the
        // same number of times, and only where a ratio of the warp reaches `floor` (w >= floor e, without a division).  Places
        // behind the row's end and the one to be left out have a logit of -inf.
        auto visit = [&](const float& floor, auto&& take) {
            Raw8<T> rz, rd;
            Raw8<float> re;
            const int whole = min(v1, a.V / 8);
            auto fetch = [&](int v, int m) {
                rz.load(x + (int64_t)v * 8, m);
                if (less) rd.load(xd + (int64_t)v * 8, m);
                re.load(e + (int64_t)v * 8, m);
            };
            auto step = [&](int v, int m, int next) {
                float z[8], zd[8] = {}, ev[8], w[8];
                rz.get(z);
                if (less) rd.get(zd);
                re.get(ev);
                if (next < whole) fetch(next, 8);
                if (m < 8 || sure >> 3 == v) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i >= m || v * 8 + i == sure) z[i] = -kInf, ev[i] = 1.0f;
                }
                const uint64_t floor2 = pair(-floor, -floor);
                float t[8];
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const uint64_t w2 = weights(pair(z[i], z[i + 1]), pair(zd[i], zd[i + 1]));
                    unpair(w2, w[i], w[i + 1]);
                    unpair(fma2(pair(ev[i], ev[i + 1]), floor2, w2), t[i], t[i + 1]);
                }
                if (__any_sync(~0u, max3(max3(t[0], t[1], t[2]), max3(t[3], t[4], t[5]), fmaxf(t[6], t[7])) >= 0.0f)) take(v * 8, w, ev);
            };
            if (v0 + tid < whole) fetch(v0 + tid, 8);
            for (int vw = v0 + (tid & ~31); vw < whole; vw += threads) step(vw + lane, vw + lane < whole ? 8 : 0, vw + lane + threads);
            if (whole < v1 && tid < 32) {  // the ragged end of the row
                if (lane == 0) fetch(whole, a.V - whole * 8);
                step(whole, lane == 0 ? a.V - whole * 8 : 0, whole);
            }
        };
        Best best{0.0f, a.V, 0.0f};
        const float window = 1.0f - (less ? kWide : 2.0f * kNear);
        // most are far below the largest that the warp has seen, and are not looked at one by one
        float seen = 0.0f, floor = 0.0f;
        visit(floor, [&](int j, const float (&w)[8], const float (&ev)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float s = w[i] * rcp(ev[i]);
                best.next = fmaxf(best.next, fminf(s, best.s));
                best.j = s > best.s ? j + i : best.j;  // in the order of places: equal ones keep the first
                best.s = fmaxf(best.s, s);
            }
            seen = fmaxf(seen, warp_max(best.s));
            floor = fminf(seen, 1e38f) * window;
        });
        best = cluster_best(best, warp_best, &cta_best, (int)cs);
        const int j0 = v0 * 8, j1 = min(v1 * 8, a.V);
        if (best.j < a.V) {
            // any place that reaches `low` may be the largest
            float low = fminf(best.s, 1e38f) * window;
            bool open = best.next >= best.s * (1.0f - kNear);
            if (less) {
                const float least = ex2(fmaf(value(x + best.j) - peak, c, add) - 2.0f * kSlack) - ex2(fmaf(value(xd + best.j) - dpeak, c, dadd) + 2.0f * kSlack);
                const float reach = least > 0.0f ? fminf(least * rcp(e[best.j]), 1e38f) * (1.0f - kFold) : 0.0f;
                open = best.next >= reach || low > reach;
                low = reach;
            }
            if (open) best.j = cluster_best(best64<T, DRAFT>(a, r, b, j0, j1, less, sure, low), warp_best64, &cta_best64, (int)cs).j;
        }
        if (best.j == a.V && (less || sure >= 0)) {  // nothing is left of p - q (p = q up to rounding): drawn from p
            if (cs > 1) cluster_sync();
            __syncthreads();
            best.j = cluster_best(best64<T, DRAFT>(a, r, b, j0, j1, false, -1, 0.0f), warp_best64, &cta_best64, (int)cs).j;
        }
        if (best.j < a.V) token = best.j, token_logp = (value(x + best.j) - peak) * a.inv_t - log_sum;
        if (cs > 1) cluster_sync();  // a CTA's shared memory stays until the others have read it
    }
    if (rank != 0) return;
    if (tid == 0) a.accepted[b] = kept;
    for (int i = tid; i < n; i += threads) {
        const bool k = i < kept;
        a.tokens[r0 + i] = k ? a.drafts[r0 + i] : i == kept ? token : -1;
        a.out_logp[r0 + i] = k ? (GREEDY ? a.best_logp[r0 + i] : a.logp[r0 + i]) : i == kept ? token_logp : 0.0f;
    }
}

struct Layout {
    size_t logp, peak, log_sum, ids, bytes;
};
Layout layout(int64_t R) {
    const size_t one = align_up((size_t)R * 4, 256);
    return Layout{kWsHeader, kWsHeader + one, kWsHeader + 2 * one, kWsHeader + 3 * one, kWsHeader + 4 * one};
}

}  // namespace
}  // namespace resq

using namespace resq;

extern "C" {

size_t resq_verify_drafts_workspace_bytes(int64_t R) { return R > 0 ? layout(R).bytes : 0; }

int resq_verify_drafts(const void* logits, int dtype, int64_t R, int64_t V, int64_t ld, const int32_t* row_start, int64_t count, const int64_t* drafts,
                       const float* u, const float* noise, int64_t lde, const void* draft_logits, int64_t ldd, const float* draft_peak,
                       const float* draft_log_sum, float temperature, int32_t* accepted, int64_t* tokens, float* logp, void* workspace,
                       size_t ws_bytes, void* stream) {
    const char* what = "verify_drafts";
    const bool greedy = temperature == 0.0f, draft = draft_logits != nullptr && !greedy;
    if (!logits || !row_start || !drafts || !accepted || !tokens || !logp || (!greedy && (!u || !noise)) || (draft && (!draft_peak || !draft_log_sum)))
        return fail(RESQ_ERR_NULL, what, "logits, row_start, drafts and the outputs must not be NULL, nor u and noise where tokens are drawn, nor a draft's peak and log_sum");
    if (dtype != RESQ_OUT_BF16 && dtype != RESQ_OUT_F32) return fail(RESQ_ERR_PATTERN, what, "unknown type of the logits");
    if (R <= 0 || R > INT32_MAX || V <= 0 || V > RESQ_MAX_VOCAB || count <= 0 || count > RESQ_MAX_SEQUENCES) {
        set_last_error("verify_drafts: %lld rows of %lld, %lld sequences (1 or more, V <= %d, 1 .. %d sequences)", (long long)R, (long long)V, (long long)count,
                       RESQ_MAX_VOCAB, RESQ_MAX_SEQUENCES);
        return RESQ_ERR_SHAPE;
    }
    if (!greedy && !(temperature >= 1e-6f && temperature <= 1e6f)) return fail(RESQ_ERR_SHAPE, what, "temperature must be 0 or lie in 1e-6 .. 1e6");
    if (!rows_aligned(logits, ld, V, dtype) || (draft && !rows_aligned(draft_logits, ldd, V, dtype)) || (!greedy && !rows_aligned(noise, lde, V, RESQ_OUT_F32)))
        return fail(RESQ_ERR_ALIGN, what, "logits, draft_logits and noise need 16-byte aligned bases and rows of at least V elements");
    if (!is_aligned(row_start, 4) || !is_aligned(drafts, 8) || !is_aligned(u, 4) || !is_aligned(draft_peak, 4) || !is_aligned(draft_log_sum, 4) ||
        !is_aligned(accepted, 4) || !is_aligned(tokens, 8) || !is_aligned(logp, 4))
        return fail(RESQ_ERR_ALIGN, what, "drafts and tokens must be 8-byte aligned, the other row values 4-byte aligned");
    const Layout l = layout(R);
    if (!workspace || !is_aligned(workspace, 256) || ws_bytes < l.bytes) {
        set_last_error("verify_drafts: workspace needs %zu bytes (256-byte aligned), got %zu", l.bytes, ws_bytes);
        return RESQ_ERR_WORKSPACE;
    }
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    float *wl = reinterpret_cast<float*>(ws + l.logp), *wp = reinterpret_cast<float*>(ws + l.peak), *ws_sum = reinterpret_cast<float*>(ws + l.log_sum);
    int32_t* ids = reinterpret_cast<int32_t*>(ws + l.ids);
    const int64_t vecs = (V + 7) / 8;
    // (Rows cut into two or four slices so that the SMs' shares are even gain 1 to 4 us at 150 and 160 rows of 131072 and lose 8 at 180 and
    // 300: 33.2 against 24.7 us for the largest logit, bf16, at 180, 48.6 against 40.0 for fp32 rows to draw from.)
    int rc = greedy ? resq_token_logprobs(logits, dtype, R, V, ld, nullptr, 1.0f, 1, nullptr, nullptr, nullptr, nullptr, ids, wl, stream)
                    : resq_token_logprobs(logits, dtype, R, V, ld, drafts, temperature, 0, wl, nullptr, wp, ws_sum, nullptr, nullptr, stream);
    if (rc) return rc;
    // Few sequences: their row over a cluster, not below 4096 logits a CTA.  The 1024 threads that an SM holds are shared by the CTAs
    // it gets, and the clusters are as large as it takes to keep most of them busy on the average: 64 sequences of 131072 take 43.4
    // us by four CTAs of 512 threads each, 49.9 by eight of 256 (clusters of eight leave SMs of a GPC over) and 51.0 by four of
    // 256; 100 sequences 54.6 by four of 320, 56.6 by two of 512; one sequence 13.6 by eight of 512, 13.3 by eight of 256.  Short
    // rows get no more threads than vectors.
    int cs = 1;
    unsigned threads = 128;
    int64_t busy = 0;
    for (int n = 1; n <= (greedy ? 1 : 8) && (n == 1 || (count * n <= 148 * 8 && vecs / n >= 512)); n *= 2) {
        const int64_t per_sm = std::min<int64_t>(8, (count * n + 147) / 148), most = std::min<int64_t>(kThreads, 1024 / per_sm / 32 * 32);
        if (n > 1 && count * n * most * 100 < busy * 106) continue;
        busy = std::max(busy, count * n * most), cs = n;
        if (!greedy) threads = (unsigned)std::min<int64_t>(most, std::max<int64_t>(64, ((vecs + n - 1) / n + 31) / 32 * 32));
    }
    const int64_t slice = (vecs + cs - 1) / cs;
    VerifyArgs a{logits, draft ? draft_logits : nullptr, ld, ldd, lde, row_start, drafts, u, noise, draft_peak, draft_log_sum, wl, wp, ws_sum, ids, wl,
                 accepted, tokens, logp, reinterpret_cast<DeviceStatus*>(ws), (int)count, (int)R, (int)V, (int)slice, greedy ? 1.0f : 1.0f / temperature,
                 greedy ? 1.0 : 1.0 / (double)temperature};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    using bf = __nv_bfloat16;
    auto kern = dtype == RESQ_OUT_F32 ? (greedy ? verify_kernel<float, false, true> : draft ? verify_kernel<float, true, false> : verify_kernel<float, false, false>)
                                      : (greedy ? verify_kernel<bf, false, true> : draft ? verify_kernel<bf, true, false> : verify_kernel<bf, false, false>);
    LaunchScope scope(kKindRow, st);
    return cuda_fail(launch_clusters(kern, dim3((unsigned)(count * cs)), threads, 0, cs, st, a), "verify_kernel launch");
}

}  // extern "C"
