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
//
// Forward: one pass over the logits.  A row belongs to a cluster of 1 to 8 CTAs (as many as it takes to fill the device), each
// with a contiguous slice.  The lanes of a warp share the running maximum, so rescaling is rare; per element that leaves a
// subtraction, a multiplication, the exponential and two additions.  It is bound by HBM, with the exponentials (16 per clock and
// SM) at 0.7 of their rate beside it.  Measured: 4096 x 131072, bf16, 184 us = 5.8 TB/s (0.89 of the copy rate); 512 x 131072,
// fp32, 42 us (0.97); one row of 131072 5.1 us, with 20 alternatives 11.4 (latency: launch, loads, three exchanges in the cluster).
// Backward: 2048 x 131072, bf16, read and written, 169 us = 6.35 TB/s (0.97).
//
// Top alternatives: every lane remembers its largest logit, the group of 16 it was in, and the largest of its other groups.  The
// k-th largest of the lanes' values (taken over sets of lanes) is a lower bound of the k-th largest logit, and only the lanes
// that reach it can hold anything above it: that group is read again, or all of the lane's groups if a second one reaches the
// bound too, and the few dozen logits that pass are ranked.  Bounds and ranks are on (value, lower index) keys, so ties need no
// care.  (4096 x 131072, top 32: 245 us; 310 when all groups of such lanes were read again, since their sectors
// come from DRAM.)
#include "row_common.cuh"

#include <algorithm>

namespace resq {
namespace {

constexpr float kInf = __builtin_huge_valf();
constexpr float kLowest = -3.4028234663852886e38f;  // differences are cut here: 0 * -inf is no term of a sum
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxLpThreads = 512;
constexpr int kV = 2, kGroup = 8 * kV;  // vectors of 8 per lane and iteration (four need 96 registers: 2 instead of 4 CTAs per SM)
constexpr int kBuckets = 64;            // sets of lanes whose largest logits bound the k-th largest
constexpr int kMaxCluster = 8;
constexpr int kCandidates = 2048;  // logits that may pass the bound before the selection falls back to repeated passes
static_assert(kCandidates >= kMaxLpThreads / kBuckets * RESQ_MAX_TOP * 8, "a row of equal logits");

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
    int slice;    // vectors of 8 per CTA of a cluster
    float inv_t;  // 1 / T
};

// Sums of a set of logits: m its largest value (-inf: the set has no finite term), s the sum of exp((x - m) / T) without one
// term of value 1, t the sum of exp((x - m) / T) (x - m).
struct Stat {
    float m, s, t;
};
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
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
__device__ __forceinline__ Stat stat_join(const Stat& p, const Stat& q, float c) {
    const bool p_first = p.m >= q.m;
    Stat a = p_first ? p : q;
    const Stat& b = p_first ? q : p;
    if (b.m == -kInf) {
        a.s += b.s;  // nothing, or the NaN of its logits
        return a;
    }
    const float d = max_nan(b.m - a.m, kLowest), f = ex2(d * c);
    a.s += f * (b.s + 1.0f);
    a.t += f * b.t + (f * d) * (b.s + 1.0f);
    return a;
}

__device__ __forceinline__ float load_logit(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load_logit(const float* p) { return *p; }

// Eight logits of a row from element k on; -inf behind its end.
template <typename T>
__device__ __forceinline__ void get_logits(const Raw8<T>& r, int n, float (&v)[8]) {
    r.get(v);
    if (n < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= n) v[i] = -kInf;
    }
}

// Orders logits by value (NaN above +inf, -0 equal to 0), equal values by lower index first.
__device__ __forceinline__ uint64_t top_key(float x, int j) {
    uint32_t u;
    if (x != x) u = 0xFFFFFFFEu;  // below the key that stands for no bound
    else {
        const uint32_t b = __float_as_uint(x + 0.0f);
        u = (b & 0x80000000u) ? ~b : b | 0x80000000u;
    }
    return ((uint64_t)u << 32) | (uint32_t)~j;
}

__device__ __forceinline__ float key_value(uint64_t key) {  // of a logit that is not NaN
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float((u & 0x80000000u) ? u & 0x7FFFFFFFu : ~u);
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote_addr(const void* p, int rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float remote_f32(const float* p, int rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote_addr(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ uint64_t remote_u64(const uint64_t* p, int rank) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(remote_addr(p, rank)) : "memory");
    return v;
}

// The block's largest key below `last` among vectors v0 .. v1 - 1 of the row, the same in every thread.
template <typename T>
__device__ uint64_t next_key(const T* x, int V, int v0, int v1, uint64_t last, uint64_t* buf) {
    uint64_t b = 0;
    for (int j = v0 * 8 + threadIdx.x; j < min(v1 * 8, V); j += blockDim.x) {
        const uint64_t key = top_key(load_logit(x + j), j);
        if (key < last && key > b) b = key;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const uint64_t q = __shfl_xor_sync(~0u, b, o);
        b = q > b ? q : b;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = b;
    __syncthreads();
    for (int i = 0; i < (int)((blockDim.x + 31) >> 5); ++i) b = buf[i] > b ? buf[i] : b;
    return b;
}

// Keys in descending order: those of rank < k go to out[rank].  All keys differ.
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, int k, uint64_t* out) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const uint64_t mine = keys[i];
        int r = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) r += keys[j] > mine;
        if (r < k) out[r] = mine;
    }
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(kMaxLpThreads, 2) logprobs_kernel(const __grid_constant__ LpArgs a) {
    __shared__ Stat warp_stat[kMaxLpThreads / 32], cta_stat;
    __shared__ uint64_t cand[TOP ? kCandidates : 1], best[TOP ? RESQ_MAX_TOP : 1];
    __shared__ __align__(16) uint32_t bucket_order[kBuckets];
    __shared__ uint16_t hot[TOP ? kMaxLpThreads : 1];
    __shared__ int count[2];
    uint32_t cs;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(cs));
    const int rank = cs > 1 ? (int)cluster_rank() : 0;
    pdl_wait();
    pdl_trigger();
    const int64_t m = blockIdx.x / cs;
    const T* const x = static_cast<const T*>(a.x) + m * a.ld;
    const float c = a.inv_t * kLog2e;
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31, w = tid >> 5, warps = threads >> 5;
    const int v0 = min(rank * a.slice, (a.V + 7) / 8), v1 = min(v0 + a.slice, (a.V + 7) / 8);

    float x_tok = 0.0f;  // thread 0 of the row: asked for before the pass, needed behind it
    bool named = false;
    if (a.logp && tid == 0 && rank == 0) {
        const int64_t tok = a.tokens[m];
        named = tok >= 0 && tok < a.V;
        if (named) x_tok = load_logit(x + tok);
    }

    // ---- one pass
    float ms = -kInf;                  // the warp's maximum
    uint64_t s2 = 0, t2 = 0;           // the lane's sums relative to it, in two halves (bits of 0.0f, 0.0f)
    bool one = false;                  // the lane holds the maximum's own term, which s leaves out
    bool cut = false;                  // the warp has met a difference of -inf: differences are cut at the lowest number
    float lane_max = -kInf, lane_second = -kInf;  // of the lane's groups
    int lane_it = 0;
    auto take = [&](float (&y)[kGroup], int it) {
        float top = y[0];
#pragma unroll
        for (int i = 1; i + 1 < kGroup; i += 2) top = max3(top, y[i], y[i + 1]);
        top = fmaxf(top, y[kGroup - 1]);
        if (TOP) {
            lane_second = fmaxf(lane_second, fminf(top, lane_max));
            if (top > lane_max || it == 0) lane_max = top, lane_it = it;
        }
        const float all = warp_max(top);
        if (all > ms) {  // warp-uniform
            if (ms != -kInf) {
                const float d = max_nan(ms - all, kLowest), f = ex2(d * c);
                float sl, sh, tl, th;
                unpair(s2, sl, sh), unpair(t2, tl, th);
                const float held = sl + sh + (one ? 1.0f : 0.0f);
                t2 = pair(f * (tl + th) + (f * d) * held, 0.0f);  // f * d first: d may be the lowest number
                s2 = pair(f * held, 0.0f);
            }
            ms = all;
            const unsigned who = __ballot_sync(~0u, top == all);
            one = lane == __ffs(who) - 1;
            if (one) {  // its own term stays out: that element becomes one whose term is 0
                const float none = fabsf(all) < 1e29f ? -1e30f : all > 0.0f ? 0.0f : -kInf;
                bool done = false;
#pragma unroll
                for (int i = 0; i < kGroup; ++i) {
                    const bool hit = !done && y[i] == all;
                    done |= hit;
                    if (hit) y[i] = none;
                }
            }
        }
        const float ref = fmaxf(ms, kLowest);
        const uint64_t ref2 = pair(-ref, -ref), c2 = pair(c, c);
        uint64_t gs = 0, gt = 0;
        // 0 * -inf (a masked logit) shows as NaN in gt: then the group is done again with its differences cut, and so are the
        // warp's later ones
        if (!cut) {
#pragma unroll
            for (int i = 0; i < kGroup; i += 2) {
                const uint64_t d = add2(pair(y[i], y[i + 1]), ref2), q = mul2(d, c2);
                float ql, qh;
                unpair(q, ql, qh);
                const uint64_t e = pair(ex2(ql), ex2(qh));
                gs = add2(gs, e);
                gt = fma2(e, d, gt);
            }
            float tl, th;
            unpair(gt, tl, th);
            cut = __any_sync(~0u, !(tl + th <= 0.0f));
        }
        if (cut) {
            gs = gt = 0;
#pragma unroll
            for (int i = 0; i < kGroup; i += 2) {
                const float dl = max_nan(y[i] - ref, kLowest), dh = max_nan(y[i + 1] - ref, kLowest);
                const uint64_t e = pair(ex2(dl * c), ex2(dh * c));
                gs = add2(gs, e);
                gt = fma2(e, pair(dl, dh), gt);
            }
        }
        s2 = add2(s2, gs), t2 = add2(t2, gt);
    };
    // All lanes of a warp make the same number of iterations: first those whose vectors are all whole, the next one's loads
    // ahead of the sums, then the one or two at the end of the row or slice.
    const int step = kV * threads, whole = min(v1, a.V / 8) - (v0 + w * 32 + 31 + (kV - 1) * threads);
    const int its = whole > 0 ? (whole + step - 1) / step : 0;
    const T* p = x + (int64_t)(v0 + tid) * 8;
    // iterations whose loads are in flight: two of 32 bytes per lane for bf16 (4096 x 131072: 184 against 192 us), which the
    // selection of alternatives has no registers for
    constexpr int kAheadIts = sizeof(T) == 2 && !TOP ? 2 : 1;
    Raw8<T> raw[kAheadIts][kV];
    auto fetch = [&](int b) {
#pragma unroll
        for (int h = 0; h < kV; ++h) raw[b][h].load(p + (int64_t)h * threads * 8, 8);
        p += (int64_t)step * 8;
    };
#pragma unroll
    for (int b = 0; b < kAheadIts; ++b)
        if (b < its) fetch(b);
    for (int it0 = 0; it0 < its; it0 += kAheadIts) {
#pragma unroll
        for (int b = 0; b < kAheadIts; ++b) {
            if (it0 + b >= its) break;
            float y[kGroup];
#pragma unroll
            for (int h = 0; h < kV; ++h) {
                float z[8];
                raw[b][h].get(z);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[h * 8 + i] = z[i];
            }
            if (it0 + b + kAheadIts < its) fetch(b);
            take(y, it0 + b);
        }
    }
    for (int it = its, vw = v0 + w * 32 + its * step; vw < v1; vw += step, ++it) {
        float y[kGroup];
#pragma unroll
        for (int h = 0; h < kV; ++h) {
            const int v = vw + lane + h * threads, n = v < v1 ? a.V - v * 8 : 0;
            float z[8];
            Raw8<T> r;
            if (n > 0) r.load(x + (int64_t)v * 8, n);
            get_logits(r, n, z);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[h * 8 + i] = z[i];
        }
        take(y, it);
    }
    float s, t;
    {
        float sl, sh, tl, th;
        unpair(s2, sl, sh), unpair(t2, tl, th);
        s = sl + sh, t = tl + th;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o), t += __shfl_xor_sync(~0u, t, o);
    if (lane == 0) warp_stat[w] = Stat{ms, s, t};
    if (TOP && tid < 2) count[tid] = 0;
    __syncthreads();
    if (w == 0) {
        Stat q = lane < warps ? warp_stat[lane] : Stat{-kInf, 0.0f, 0.0f};
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            q = stat_join(q, Stat{__shfl_xor_sync(~0u, q.m, o), __shfl_xor_sync(~0u, q.s, o), __shfl_xor_sync(~0u, q.t, o)}, c);
        if (lane == 0) cta_stat = q;
    }
    __syncthreads();

    // ---- this slice's largest keys, in order, into best[]
    const int have = min(a.V - v0 * 8, (v1 - v0) * 8), k = TOP ? max(0, min(a.top, have)) : 0;
    if (TOP) {
        const Stat q = cta_stat;
        const bool strange = q.m == kInf || q.s != q.s;  // +inf or NaN: by repeated passes, which order them too
        int found = kCandidates + 1;
        if (!strange && k > 0) {
            // Buckets of neighbouring lanes, ranked by their largest value (cut to make room for the bucket's number: any k
            // buckets give a valid bound).  Leaders of the first k: their exact keys, the smallest of which is the bound.
            int per_bucket = 1;  // a power of two; 32 to 64 buckets
            while (threads > kBuckets * per_bucket) per_bucket *= 2;
            const int buckets = threads / per_bucket;
            float bmax = lane_max;
            for (int o = 1; o < per_bucket; o *= 2) bmax = fmaxf(bmax, __shfl_xor_sync(~0u, bmax, o));
            const unsigned tied = __ballot_sync(~0u, lane_max == bmax) >> (lane & ~(per_bucket - 1));
            const bool leader = (lane & (per_bucket - 1)) == __ffs(tied & ((2u << (per_bucket - 1)) - 1u)) - 1;
            const int mine = tid / per_bucket;
            const uint32_t order = ((uint32_t)(top_key(bmax, 0) >> 32) & ~(uint32_t)(kBuckets - 1)) | (uint32_t)(kBuckets - 1 - mine);
            if (leader) bucket_order[mine] = order;
            __syncthreads();
            int r = kBuckets;
            if (leader) {
                r = 0;
                for (int j = 0; j < buckets; j += 4) {
                    const uint4 o = *reinterpret_cast<const uint4*>(bucket_order + j);
                    r += (o.x > order) + (o.y > order) + (o.z > order) + (o.w > order);
                }
                if (r < k) best[r] = top_key(lane_max, 0) & ~0xFFFFFFFFull;
            }
            // First with the leaders' values alone; a row with too many equal logits goes by their places too, which takes
            // reading the leaders' groups again.
            for (int exact = 0; exact < 2; ++exact) {
                if (exact && r < k) {
                    uint64_t key = 0;  // a lane without elements: no bound
#pragma unroll
                    for (int h = kV - 1; h >= 0; --h) {
                        const int v = v0 + (lane_it * kV + h) * threads + tid;
                        if (v >= v1) continue;
                        Raw8<T> g;
                        float z[8];
                        g.load(x + (int64_t)v * 8, a.V - v * 8);
                        get_logits(g, a.V - v * 8, z);
#pragma unroll
                        for (int i = 7; i >= 0; --i)
                            if (z[i] == lane_max) key = top_key(z[i], v * 8 + i);
                    }
                    best[r] = key;
                }
                __syncthreads();
                uint64_t low = lane < k ? best[lane] : ~0ull;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const uint64_t q8 = __shfl_xor_sync(~0u, low, o);
                    low = q8 < low ? q8 : low;
                }
                // lanes that may hold keys from the bound on: the group of their largest logit again, or all their groups
                const float lv = low == 0 ? -kInf : key_value(low);
                auto pass = [&](const Raw8<T>& g, int v) {
                    float z[8];
                    get_logits(g, a.V - v * 8, z);
                    unsigned mask = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (z[e] >= lv && v * 8 + e < a.V && top_key(z[e], v * 8 + e) >= low) mask |= 1u << e;
                    if (mask == 0) return;
                    int at = atomicAdd(&count[1], __popc(mask));
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (!(mask >> e & 1)) continue;
                        if (at < kCandidates) cand[at] = top_key(z[e], v * 8 + e);
                        ++at;
                    }
                };
                // one place in the code takes them all (it runs once per row: its length costs time)
                const int per = (v1 - v0 + threads - 1) / threads;  // vectors of a lane
                const bool any = v0 + tid < v1 && lane_max >= lv, all = any && per > kV && lane_second >= lv;
                if (all) hot[atomicAdd(&count[0], 1)] = (uint16_t)tid;
                __syncthreads();
                const int items = count[0] * per;
                // step 0 to kV - 1: the lane's own group; then the vectors of the lanes on the list, 32 per warp and step
                auto fetch = [&](int n, Raw8<T>& g) {
                    int v = v1;
                    if (n < kV) {
                        if (any && !all) v = v0 + (lane_it * kV + n) * threads + tid;
                    } else {
                        const int i = (n - kV) * threads + tid;
                        if (i < items) v = v0 + i % per * threads + hot[i / per];
                    }
                    if (v < v1) g.load(x + (int64_t)v * 8, a.V - v * 8);
                    return v;
                };
                constexpr int kFlight = 2;  // three cost registers that 32-bit logits do not have
                Raw8<T> g[kFlight];
                int at[kFlight];
#pragma unroll
                for (int b = 0; b < kFlight; ++b) at[b] = fetch(b, g[b]);
#pragma unroll 1
                for (int n = 0; n < kV || (n - kV) * threads + w * 32 < items; ++n) {
                    if (at[0] < v1) pass(g[0], at[0]);
#pragma unroll
                    for (int b = 0; b + 1 < kFlight; ++b) g[b] = g[b + 1], at[b] = at[b + 1];
                    at[kFlight - 1] = fetch(n + kFlight, g[kFlight - 1]);
                }
                __syncthreads();
                found = count[1];
                if (found <= kCandidates || exact) break;
                __syncthreads();
                if (tid < 2) count[tid] = 0;
            }
            // many equal logits: the k-th largest key itself, by bisection, and the k keys from there on
            if (found > 128 && found <= kCandidates) {
                uint64_t bound = 0;
                int n = found;
                for (int bit = 63; bit >= 0 && n != k; --bit) {
                    const uint64_t trial = bound | (1ull << bit);
                    int reach = 0;
                    for (int i = 0; i < found; i += threads) reach += __syncthreads_count(i + tid < found && cand[i + tid] >= trial);
                    if (reach >= k) bound = trial, n = reach;
                }
                __syncthreads();
                if (tid == 0) count[0] = 0;
                __syncthreads();
                for (int i = tid; i < found; i += threads)
                    if (cand[i] >= bound) best[atomicAdd(&count[0], 1)] = cand[i];
                __syncthreads();
                if (tid < k) cand[tid] = best[tid];
                __syncthreads();
                found = k;
            }
        }
        if (found <= kCandidates) {
            rank_keys(cand, found, k, best);
        } else {
            uint64_t last = ~0ull;
            for (int r = 0; r < k; ++r) {
                last = next_key(x, a.V, v0, v1, last, cand);
                if (tid == 0) best[r] = last;
            }
        }
        if (tid < RESQ_MAX_TOP && tid >= k) best[tid] = 0;
    }

    // ---- the row's values
    if (cs > 1) cluster_sync();
    if (rank == 0) {
        if (cs > 1) {
            if (w == 0) {
                Stat q{-kInf, 0.0f, 0.0f};
                if (lane < (int)cs) q = Stat{remote_f32(&cta_stat.m, lane), remote_f32(&cta_stat.s, lane), remote_f32(&cta_stat.t, lane)};
#pragma unroll
                for (int o = kMaxCluster / 2; o > 0; o >>= 1)
                    q = stat_join(q, Stat{__shfl_xor_sync(~0u, q.m, o), __shfl_xor_sync(~0u, q.s, o), __shfl_xor_sync(~0u, q.t, o)}, c);
                if (lane == 0) warp_stat[0] = q;
            }
            if (TOP)
                for (int i = tid; i < (int)cs * a.top; i += threads) cand[i] = remote_u64(&best[i % a.top], i / a.top);
            __syncthreads();
        } else if (TOP) {
            __syncthreads();
        }
        const Stat q = cs > 1 ? warp_stat[0] : cta_stat;
        const bool bad = q.m == kInf || q.s != q.s, empty = q.m == -kInf;
        const float nan = __int_as_float(0x7FC00000), log_s = bad ? nan : log1pf(q.s);
        if (tid == 0) {
            if (a.logp) a.logp[m] = !named ? 0.0f : bad ? nan : x_tok == -kInf ? -kInf : (x_tok - q.m) * a.inv_t - log_s;
            if (a.entropy) a.entropy[m] = bad ? nan : empty ? 0.0f : log_s - q.t * a.inv_t / (1.0f + q.s);
            if (a.peak) a.peak[m] = bad ? nan : q.m;
            if (a.log_sum) a.log_sum[m] = log_s;
        }
        if (TOP) {
            auto put = [&](int r, uint64_t key) {
                const float v = key_value(key);
                a.top_ids[m * a.top + r] = (int)~(uint32_t)key;
                a.top_logp[m * a.top + r] = bad ? nan : v == -kInf ? -kInf : (v - q.m) * a.inv_t - log_s;
            };
            if (cs > 1) {  // the slices' best together; entries behind a slice's own count are 0 and rank behind every key
                for (int i = tid; i < (int)cs * a.top; i += threads) {
                    const uint64_t mine = cand[i];
                    int r = 0;
                    for (int j = 0; j < (int)cs * a.top; ++j) r += cand[j] > mine;
                    if (mine != 0 && r < a.top) put(r, mine);
                }
            } else if (tid < a.top) {
                put(tid, best[tid]);
            }
        }
    }
    if (cs > 1) cluster_sync();  // no CTA leaves while rank 0 may still read its shared memory
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

// dx_j = (1 / T) [dlogp (1[j = tok] - p_j) - dentropy p_j (log p_j + entropy)] = -p_j (A + B log2 p_j) but for the token itself,
// where 1 - p comes from the forward call's logp (-expm1), which keeps its digits when p is near 1.  One read and one write of
// the row: HBM-bound.
constexpr int kBwdThreads = 256, kBwdVecs = 4;
template <typename T>
__global__ void __launch_bounds__(kBwdThreads) logprobs_bwd_kernel(const __grid_constant__ LpBwdArgs a) {
    pdl_wait();
    pdl_trigger();
    const int64_t m = blockIdx.x / a.chunks;
    const int base = (int)(blockIdx.x % a.chunks) * ((int)blockDim.x * kBwdVecs * 8) + threadIdx.x * 8;
    Raw8<T> r[kBwdVecs];
#pragma unroll
    for (int h = 0; h < kBwdVecs; ++h) {
        const int k = base + h * (int)blockDim.x * 8;
        if (k < a.V) r[h].load(static_cast<const T*>(a.x) + m * a.ld + k, a.V - k);
    }
    const float peak = a.peak[m], log_sum = a.log_sum[m];
    const float H = a.dentropy ? a.entropy[m] : 0.0f, de = a.dentropy ? a.dentropy[m] * a.inv_t : 0.0f;
    const int64_t tok = a.tokens[m];
    const bool there = tok >= 0 && tok < a.V;
    const float dl = there ? a.dlogp[m] * a.inv_t : 0.0f;
    const float c = a.inv_t * kLog2e, shift = -log_sum * kLog2e, A = -(dl + H * de), B = -de * 0.6931471805599453f;
    const bool empty = peak == -kInf;
    const float ref = empty ? 0.0f : peak;
#pragma unroll
    for (int h = 0; h < kBwdVecs; ++h) {
        const int k = base + h * (int)blockDim.x * 8, n = a.V - k;
        if (n <= 0) continue;
        float v[8];
        r[h].get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float z = max_nan(fmaf(v[i] - ref, c, shift), -1e5f);  // log2 p; 2^-1e5 is 0
            v[i] = ex2(z) * fmaf(B, z, A);
        }
        if (there && tok >= k && tok < k + 8) {
            const float z = a.logp[m];
            float g = -expm1f(z) * dl;
            const float p = expf(z);
            if (p != 0.0f) g -= p * (z + H) * de;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i == tok) v[i] = g;
        }
        if (empty) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        }
        store8(static_cast<T*>(a.dx) + m * a.ldd + k, v, n);
    }
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
    // Few rows are sliced, up to 256 CTAs and not below 16384 logits a slice: 1 x 131072 takes 5.2 us in eight slices and 9.8
    // in one, but 512 x 131072 33 us in two and 31 in one, and 8000 logits a slice lose (a cluster's launch costs more than
    // its CTAs').
    const int64_t vecs = (V + 7) / 8;
    int cs = 1;
    while (cs < kMaxCluster && M * cs * 2 <= 256 && vecs / (2 * cs) >= 2048) cs *= 2;
    const int64_t slice = (vecs + cs - 1) / cs;
    // An SM holds 1024 of these threads.  Up to eight CTAs per SM share them, so that all rows are under way at once (740 x
    // 131072, fp32: 59 us with 192 threads, 71 with 256, which leave 148 rows to a second wave); beyond, the number of CTAs
    // per SM whose waves come out best.
    const int64_t ctas = M * cs;
    int per_sm = 2;
    if (ctas <= 8 * 148) {
        while (ctas > per_sm * 148) per_sm = per_sm == 6 ? 8 : per_sm + 1;
    } else {
        per_sm = 4;
        auto rows_sm = [&](int n) { return (ctas + 148 * n - 1) / (148 * n) * n; };
        for (int n = 5; n <= 6; ++n)
            if (rows_sm(n) < rows_sm(per_sm)) per_sm = n;
    }
    // With alternatives rows of up to 64 vectors get a thread for each: the bound wants `top` lanes with logits (4000 x 500, top
    // 32: 30 against 79 us; 4000 x 1000 would lose, 30 against 27 us for one alternative).
    const int64_t most = 1024 / per_sm / 32 * 32, per_lane = top && slice <= 64 ? 1 : kV;
    const unsigned threads = (unsigned)std::min<int64_t>(most, ((slice + per_lane - 1) / per_lane + 31) / 32 * 32);
    if (M * cs > INT32_MAX) return fail(RESQ_ERR_SHAPE, what, "too many rows for one call");
    LpArgs a{logits, ld, tokens, logp, entropy, peak, log_sum, top_ids, top_logp, (int)V, top, (int)slice, 1.0f / temperature};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    using bf = __nv_bfloat16;
    auto kern = dtype == RESQ_OUT_F32 ? (top ? logprobs_kernel<float, true> : logprobs_kernel<float, false>)
                                      : (top ? logprobs_kernel<bf, true> : logprobs_kernel<bf, false>);
    LaunchScope scope(kKindRow, st);
    return cuda_fail(launch_clusters(kern, (unsigned)(M * cs), threads, 0, cs, st, a), "logprobs_kernel launch");
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
    // a row in equal chunks with as few threads as they need (4000 x 1000: 5.2 us; 9.1 with 256 threads whatever V is)
    const int64_t vecs = (V + 7) / 8, parts = (vecs + kBwdThreads * kBwdVecs - 1) / (kBwdThreads * kBwdVecs);
    const unsigned threads = (unsigned)((vecs + parts * kBwdVecs * 32 - 1) / (parts * kBwdVecs * 32) * 32);
    const int64_t chunks = (vecs + threads * kBwdVecs - 1) / (threads * kBwdVecs);
    if (M * chunks > INT32_MAX) return fail(RESQ_ERR_SHAPE, what, "M x V is too large for one call");
    LpBwdArgs a{logits, dlogits, ld, ldd, tokens, logp, peak, log_sum, entropy, dlogp, dentropy, (int)V, 1.0f / temperature, (unsigned)chunks};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    LaunchScope scope(kKindRow, st);
    auto kern = dtype == RESQ_OUT_F32 ? logprobs_bwd_kernel<float> : logprobs_bwd_kernel<__nv_bfloat16>;
    return cuda_fail(launch_kernel(kern, dim3((unsigned)(M * chunks)), dim3(threads), 0, st, a),
                     "logprobs_bwd_kernel launch");
}
}
