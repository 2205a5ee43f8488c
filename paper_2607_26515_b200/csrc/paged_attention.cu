// resq_paged_attention: softmax attention of the new tokens of several sequences over their keys and values in a paged cache.
//
//   O_i = sum_{j <= pos_i} p_ij v_j,   p_ij = exp(scale q_i.k_j - lse_i),   lse_i = log sum_{j <= pos_i} exp(scale q_i.k_j)
//
// One pass over the keys with a running reference m (the largest score so far): p = 2^(s c - m) with c = scale log2(e), the sums
// l and O multiplied by 2^(m_old - m_new) when m grows, O / l at the end.  P is rounded to bf16 for its product with V, since the
// instruction takes both operands in the type that V has (off by at most 2^-8 of each weight, as the output is by its own rounding); l is
// of the weights before that, which lse needs.  Scores, sums and O are fp32.
//
// Three kernels, by the query rows that share a kv head (tokens times heads of a group):
//   attn_rows_kernel, up to 32 (decoded tokens): bound by reading the cache once.  The queries are the rows of one register-operand
//     tensor instruction (m16n8k16), so each key is read once for all of them.  The four warps of a CTA take 16 keys each of a tile of
//     64, with a ring of asynchronous copies of their own and their own running sums, and meet only when the item is finished:
//     nothing in the loop waits for another warp.  64 sequences of 2000 to 12000 keys, 28 heads on 4 of 128: 176 us = 6.0 TB/s (0.92 of the
//     copy rate); one sequence of 4000 keys 11.5 us, latency (lengths, page numbers, keys, sums, and the join of 63 parts).
//   attn_wide_kernel, up to 64 (drafted tokens): bound by latencies.  That instruction does 1024 products of a row, a key and a
//     channel per clock and SM, a quarter of what tensor memory allows, and is busy 39 % of the time, as issue slots and DRAM are 35 %:
//     products, maxima, exponentials and products follow one another in a warp, and rows that do not exist are multiplied too.  24
//     sequences of up to 9000 keys, 2 to 6 tokens, 16 heads on 2: 39.6 us for 91 MB; the chunk kernel takes 44, and 31 instead of 23
//     for 64 sequences of 100 to 600 keys (larger fixed parts).
//   attn_chunk_kernel (paged_chunk.cu), beyond.
// Work is dealt out over the keys of all items evenly (paged.cuh), and what was cut is joined by a second kernel.
#include "paged.cuh"

#include <algorithm>
#include <cmath>

namespace resq {

int check_paged(const char* what, const resq_paged_cache* c, const resq_sequences* s, int64_t T, int64_t Hq, int64_t Hkv, int64_t D) {
    if (!c || !s || !c->k || !c->v || !s->q_start || !s->kv_len || !s->page_table) return fail(RESQ_ERR_NULL, what, "cache, sequences and their arrays must not be NULL");
    if (T <= 0 || s->count <= 0 || s->count > kMaxSeqs) {
        set_last_error("%s: %lld token rows, %lld sequences (1 or more rows, 1 .. %d sequences)", what, (long long)T, (long long)s->count, RESQ_MAX_SEQUENCES);
        return RESQ_ERR_SHAPE;
    }
    if (c->kv_heads != Hkv || c->head_dim != D || Hkv <= 0 || Hq <= 0 || Hq % Hkv || Hq / Hkv > RESQ_MAX_GROUP_HEADS || (D != 64 && D != 128)) {
        set_last_error("%s: %lld query heads, %lld kv heads of %lld (heads of 64 or 128, 1 .. %d query heads per kv head)", what, (long long)Hq,
                       (long long)Hkv, (long long)D, RESQ_MAX_GROUP_HEADS);
        return RESQ_ERR_SHAPE;
    }
    if (T > INT32_MAX / Hq || Hkv > INT32_MAX / D / 2) return fail(RESQ_ERR_SHAPE, what, "too many rows or heads for one call");
    if (c->pages <= 0 || c->pages > INT32_MAX || c->page_size <= 0 || c->page_size % 8 || c->page_size > 65536 || s->max_pages <= 0 ||
        s->max_pages > (INT32_MAX - 65536) / c->page_size) {
        set_last_error("%s: %lld pages of %lld, %lld per sequence (pages of a multiple of 8 up to 65536 keys, fewer than 2^31 keys per sequence)", what,
                       (long long)c->pages, (long long)c->page_size, (long long)s->max_pages);
        return RESQ_ERR_SHAPE;
    }
    const int64_t strides[6] = {c->k_page, c->k_row, c->k_head, c->v_page, c->v_row, c->v_head};
    for (int64_t v : strides)
        if (v < 0 || v % 8 || v >= (int64_t)1 << 36) return fail(RESQ_ERR_ALIGN, what, "cache strides must be multiples of 8 elements, below 2^36");
    if (!is_aligned(c->k, 16) || !is_aligned(c->v, 16)) return fail(RESQ_ERR_ALIGN, what, "the cache must be 16-byte aligned");
    if (!is_aligned(s->q_start, 4) || !is_aligned(s->kv_len, 4) || !is_aligned(s->page_table, 4) || s->ld_table < s->max_pages)
        return fail(RESQ_ERR_ALIGN, what, "q_start, kv_len and page_table must be 4-byte aligned, ld_table >= max_pages");
    return RESQ_OK;
}

namespace {

constexpr float kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWarps = 4, kKeys = 64, kWarpKeys = kKeys / kWarps;  // of attn_rows_kernel
constexpr int kRowsCtasPerSm = 2;

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes to shared memory; zeros where !there (nothing is read then).
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A share of a row's keys has a reference and a sum (and a product).  One without weights is none: its product may not even be
// written.  Any other counts, also where its weight is 0 beside a far larger reference: what it holds may be NaN or infinite, and
// which keys share a part must not decide whether a row is.
__device__ __forceinline__ bool no_share(float2 q) { return q.x == -kInf && q.y == 0.0f; }
__device__ __forceinline__ float join_weight(float2 q, float ref) {
    return q.x == -kInf ? (q.y == 0.0f ? 0.0f : 1.0f) : ex2(q.x - ref);  // a sum without a reference is one of NaN scores
}

template <int D>
constexpr int rows_stages() { return D == 128 ? 3 : 6; }  // 24 KB of ring per warp
template <int D, int MT>
constexpr int rows_smem() { return MT * 16 * D * 2 + kWarps * rows_stages<D>() * kWarpKeys * D * 4 + kWarps * MT * 16 * 8; }

template <int D, int MT>
__global__ void __launch_bounds__(kWarps * 32, kRowsCtasPerSm) attn_rows_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int R = MT * 16, CH = D / 8, S = rows_stages<D>(), kStage = kWarpKeys * D * 4, kHalf = kWarpKeys * D * 2;
    constexpr int KS = D / 16, NT = D / 8;
    static_assert(S * kStage >= R * D * 4, "the ring holds a warp's sums at the end");
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int64_t sums[kWarps];
    __shared__ DealStart found;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, cta = blockIdx.x;
    unsigned char* const ring = smem + R * D * 2 + w * S * kStage;
    float2* const ml = reinterpret_cast<float2*>(smem + R * D * 2 + kWarps * S * kStage);  // [warp][R]
    const uint32_t q_base = (uint32_t)__cvta_generic_to_shared(smem), ring_base = (uint32_t)__cvta_generic_to_shared(ring);
    pdl_wait();
    if (cta == 0 && tid == 0) *a.status = DeviceStatus{RESQ_OK, 0, 0, 0};
    const Deal& d = a.deal;
    const DealStart start = deal_start(a.seq, d, cta, gridDim.x, a.min_chunk, sums, &found);
    DealWalk walk;
    walk.init(a.seq, d, start);
    bool first = true;
    Segment seg;
    while (walk.next(a.seq, d, seg)) {
        const int f0 = seg.t * R, rows = min(R, seg.s.n * d.g - f0), k_end = deal_k_end(seg.s, d, seg.t), past = seg.s.kv - seg.s.n;
        __syncthreads();  // the sums of the segment before have been read
        // ---- queries, on their way with the first keys
        for (int i = tid; i < R * CH; i += kWarps * 32) {
            const int r = i / CH, ch = i % CH;
            const bool there = r < rows;
            const int f = f0 + (there ? r : 0), tok = (int)div_by((uint32_t)f, d.by_g), head = seg.h * d.g + (f - tok * d.g);
            copy16(q_base + r * D * 2 + ((ch ^ (r & 7)) * 16), a.q + (int64_t)(seg.s.q0 + tok) * a.ldq + head * D + ch * 8, there);
        }
        int pos[MT][2];  // of the rows this thread holds; rows behind the tile see what the last one does
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                pos[mt][i] = past + (int)div_by((uint32_t)(f0 + min(mt * 16 + i * 8 + lane / 4, rows - 1)), d.by_g);
        const int first_pos = past + (int)div_by((uint32_t)f0, d.by_g);  // keys up to here are seen by all rows

        const int key_first = seg.k0 * kKeys + w * kWarpKeys;
        // tiles of this warp that hold a key
        const int tiles = min(seg.k1 - seg.k0, max(0, (k_end - key_first + kKeys - 1) / kKeys));
        auto issue = [&](int i) {
            if (i < tiles) {
                const int key0 = key_first + i * kKeys;
                const uint32_t dst = ring_base + (i % S) * kStage;
                constexpr int kPass = 32 / CH;  // rows per pass of the warp
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    int in_page = 0;
                    const int page = key0 + half * 8 < k_end ? page_of(a.seq, seg.b, key0 + half * 8, in_page) : -1;
                    const __nv_bfloat16* kp = a.k + (int64_t)max(page, 0) * a.k_page + seg.h * a.k_head;
                    const __nv_bfloat16* vp = a.v + (int64_t)max(page, 0) * a.v_page + seg.h * a.v_head;
#pragma unroll
                    for (int p = 0; p < 8 / kPass; ++p) {
                        const int r = p * kPass + lane / CH, ch = lane % CH, rr = half * 8 + r;
                        const bool there = page >= 0 && key0 + rr < k_end;
                        const uint32_t at = dst + rr * D * 2 + ((ch ^ (rr & 7)) * 16);
                        copy16(at, kp + (there ? (int64_t)(in_page + r) * a.k_row + ch * 8 : 0), there);
                        copy16(at + kHalf, vp + (there ? (int64_t)(in_page + r) * a.v_row + ch * 8 : 0), there);
                    }
                }
            }
            copy_commit();
        };
        float o[MT][NT][4], m[MT][2], l[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int n = 0; n < NT; ++n) o[mt][n][0] = o[mt][n][1] = o[mt][n][2] = o[mt][n][3] = 0.0f;
            m[mt][0] = m[mt][1] = -kInf, l[mt][0] = l[mt][1] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < S - 1; ++i) issue(i);
        copy_wait<S - 2>();
        __syncthreads();  // the queries, whoever brought them
        for (int i = 0; i < tiles; ++i) {
            copy_wait<S - 2>();
            __syncwarp();
            const uint32_t kb = ring_base + (i % S) * kStage, vb = kb + kHalf;
            const int key0 = key_first + i * kKeys;
            float s[MT][2][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int n = 0; n < 2; ++n) s[mt][n][0] = s[mt][n][1] = s[mt][n][2] = s[mt][n][3] = 0.0f;
            const int lr = lane & 7, lm = lane >> 3;  // row and matrix of an ldmatrix address
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                uint32_t kf[4];
                {
                    const int r = (lm >> 1) * 8 + lr, ch = ks * 2 + (lm & 1);
                    ldsm4(kf, kb + r * D * 2 + ((ch ^ (r & 7)) * 16));
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    uint32_t qf[4];
                    const int r = mt * 16 + (lm & 1) * 8 + lr, ch = ks * 2 + (lm >> 1);
                    ldsm4(qf, q_base + r * D * 2 + ((ch ^ (r & 7)) * 16));
                    mma(s[mt][0], qf, kf[0], kf[1]);
                    mma(s[mt][1], qf, kf[2], kf[3]);
                }
            }
            const bool masked = key0 + kWarpKeys - 1 > first_pos;  // some row does not see all of these keys
            if (masked) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (key0 + n * 8 + (lane & 3) * 2 + (e & 1) > pos[mt][e >> 1]) s[mt][n][e] = -kInf;
            }
            uint32_t pf[MT][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                float top[2], ref[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = fmaxf(fmaxf(s[mt][0][2 * e], s[mt][0][2 * e + 1]), fmaxf(s[mt][1][2 * e], s[mt][1][2 * e + 1]));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
                    top[e] = fmaxf(m[mt][e], x * a.c);
                }
                if (__any_sync(~0u, top[0] > m[mt][0] || top[1] > m[mt][1])) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float f = top[e] > m[mt][e] ? ex2(m[mt][e] - top[e]) : 1.0f;
                        m[mt][e] = top[e];
                        l[mt][e] *= f;
#pragma unroll
                        for (int n = 0; n < NT; ++n) o[mt][n][2 * e] *= f, o[mt][n][2 * e + 1] *= f;
                    }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) ref[e] = m[mt][e] == -kInf ? 0.0f : m[mt][e];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[mt][n][e] = ex2(fmaf(s[mt][n][e], a.c, -ref[e >> 1]));
                        l[mt][e >> 1] += s[mt][n][e];
                    }
                pf[mt][0] = pack_bf16(s[mt][0][0], s[mt][0][1]);
                pf[mt][1] = pack_bf16(s[mt][0][2], s[mt][0][3]);
                pf[mt][2] = pack_bf16(s[mt][1][0], s[mt][1][1]);
                pf[mt][3] = pack_bf16(s[mt][1][2], s[mt][1][3]);
            }
            // A weight of 0 must not meet an infinity or NaN: in a tile with masked keys (those of tokens that came later; keys
            // from k_end on are zeros here) such values take the way element by element.
            bool strange = false;
            if (masked && k_end - 1 > first_pos) {
                for (int j = lane; j < kWarpKeys * CH; j += 32) {
                    const uint4 v = *reinterpret_cast<const uint4*>(ring + (i % S) * kStage + kHalf + j * 16);
                    const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) strange |= (x[e] & 0x7F80u) == 0x7F80u || (x[e] & 0x7F800000u) == 0x7F800000u;
                }
                strange = __any_sync(~0u, strange);
            }
            if (!strange) {
#pragma unroll
                for (int n = 0; n < NT; n += 2) {
                    uint32_t vf[4];
                    const int r = (lm & 1) * 8 + lr, ch = n + (lm >> 1);
                    ldsm4_t(vf, vb + r * D * 2 + ((ch ^ (r & 7)) * 16));
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        mma(o[mt][n], pf[mt], vf[0], vf[1]);
                        mma(o[mt][n + 1], pf[mt], vf[2], vf[3]);
                    }
                }
            } else {
                for (int j = 0; j < kWarpKeys; ++j) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        float p[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float x0 = (j & 8) ? s[mt][1][2 * e] : s[mt][0][2 * e], x1 = (j & 8) ? s[mt][1][2 * e + 1] : s[mt][0][2 * e + 1];
                            p[e] = __shfl_sync(~0u, (j & 1) ? x1 : x0, (lane & ~3) | ((j & 7) >> 1));
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint32_t v = *reinterpret_cast<const uint32_t*>(ring + (i % S) * kStage + kHalf + j * D * 2 + ((n ^ (j & 7)) * 16) + (lane & 3) * 4);
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (key0 + j <= pos[mt][e]) {
                                    o[mt][n][2 * e] = fmaf(p[e], bf16_lo(v), o[mt][n][2 * e]);
                                    o[mt][n][2 * e + 1] = fmaf(p[e], bf16_hi(v), o[mt][n][2 * e + 1]);
                                }
                        }
                    }
                }
            }
            __syncwarp();
            issue(i + S - 1);
        }
        copy_wait<0>();
        __syncwarp();
        // ---- the warps' sums, into their rings
        float* const mine = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float x = l[mt][e];
                x += __shfl_xor_sync(~0u, x, 1);
                x += __shfl_xor_sync(~0u, x, 2);
                const int r = mt * 16 + e * 8 + lane / 4;
                if ((lane & 3) == 0) ml[w * R + r] = make_float2(m[mt][e], x);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    *reinterpret_cast<float2*>(mine + r * D + ((n ^ (r & 7)) * 8) + (lane & 3) * 2) = make_float2(o[mt][n][2 * e], o[mt][n][2 * e + 1]);
            }
        __syncthreads();
        const bool whole = seg.u0 == 0 && seg.u1 == seg.units;
        const int slot = 2 * cta + (seg.u0 == 0 ? 1 : 0);
        for (int i = tid; i < rows * NT; i += kWarps * 32) {
            const int r = i / NT, n = i % NT;
            float ref = -kInf;
#pragma unroll
            for (int x = 0; x < kWarps; ++x) ref = fmaxf(ref, ml[x * R + r].x);
            float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0}, sum = 0.0f;
#pragma unroll
            for (int x = 0; x < kWarps; ++x) {
                const float2 p = ml[x * R + r];
                if (no_share(p)) continue;
                const float f = join_weight(p, ref);
                sum = fmaf(f, p.y, sum);
                const float* src = reinterpret_cast<const float*>(smem + R * D * 2 + x * S * kStage) + r * D + ((n ^ (r & 7)) * 8);
                const float4 u = *reinterpret_cast<const float4*>(src), v = *reinterpret_cast<const float4*>(src + 4);
                acc[0] = fmaf(f, u.x, acc[0]), acc[1] = fmaf(f, u.y, acc[1]), acc[2] = fmaf(f, u.z, acc[2]), acc[3] = fmaf(f, u.w, acc[3]);
                acc[4] = fmaf(f, v.x, acc[4]), acc[5] = fmaf(f, v.y, acc[5]), acc[6] = fmaf(f, v.z, acc[6]), acc[7] = fmaf(f, v.w, acc[7]);
            }
            if (whole) {
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] *= inv;
                const int tok = (int)div_by((uint32_t)(f0 + r), d.by_g), head = seg.h * d.g + (f0 + r - tok * d.g);
                const int64_t row = seg.s.q0 + tok;
                store8(a.out + row * a.ldo + head * D + n * 8, acc, 8);
                if (a.lse && n == 0) a.lse[row * a.Hq + head] = sum == 0.0f ? -kInf : (ref + log2f(sum)) * kLn2;
            } else {
                const int64_t at = (int64_t)slot * R + r;
                store8(a.part_o + at * D + n * 8, acc, 8);
                if (n == 0) a.part_ml[at] = make_float2(ref, sum);
            }
        }
        if (first && tid == 0) a.notes[cta] = join_note(seg, start, cta, f0);
        first = false;
    }
    if (first && tid == 0) a.notes[cta].parts = 0;
    pdl_trigger();
}

// The form for 33 to 64 query rows per kv head (drafted tokens): the four warps share each tile of 64 keys and take 16 rows each, so
// that a warp's sums fit its registers (keys apart, as above, would take 256 of them) and nothing is to be joined at the end; the
// price is a barrier per tile and four reads of it from shared memory.
template <int D>
constexpr int wide_stages() { return D == 128 ? 3 : 6; }
template <int D>
constexpr int wide_smem() { return 64 * D * 2 + wide_stages<D>() * kKeys * D * 4; }

template <int D>
__global__ void __launch_bounds__(kWarps * 32, kRowsCtasPerSm) attn_wide_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int R = 64, CH = D / 8, S = wide_stages<D>(), kHalf = kKeys * D * 2, kStage = 2 * kHalf, KS = D / 16, NT = D / 8;
    constexpr int kTiles = 3;  // key tiles that can hold keys of the item's own tokens
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int64_t sums[kWarps];
    __shared__ DealStart found;
    __shared__ uint32_t strange[kTiles][2];  // a bit per key whose value row holds an infinity or NaN
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, cta = blockIdx.x;
    unsigned char* const ring = smem + R * D * 2;
    const uint32_t q_base = (uint32_t)__cvta_generic_to_shared(smem), ring_base = q_base + R * D * 2;
    pdl_wait();
    if (cta == 0 && tid == 0) *a.status = DeviceStatus{RESQ_OK, 0, 0, 0};
    const Deal& d = a.deal;
    const DealStart start = deal_start(a.seq, d, cta, gridDim.x, a.min_chunk, sums, &found);
    DealWalk walk;
    walk.init(a.seq, d, start);
    bool first = true;
    Segment seg;
    const int lr = lane & 7, lm = lane >> 3;  // row and matrix of an ldmatrix address
    while (walk.next(a.seq, d, seg)) {
        const int f0 = seg.t * R, rows = min(R, seg.s.n * d.g - f0), k_end = deal_k_end(seg.s, d, seg.t), past = seg.s.kv - seg.s.n;
        const int key_first = seg.k0 * kKeys, tiles = min(seg.k1 - seg.k0, max(0, (k_end - key_first + kKeys - 1) / kKeys));
        const int first_pos = past + (int)div_by((uint32_t)f0, d.by_g);  // keys up to here are seen by all rows
        const int first_cut = max(seg.k0, (max(first_pos, -1) + 1) / kKeys);  // the first tile with a key that some row does not see
        __syncthreads();  // the segment before has read its buffers
        if (tid < kTiles * 2) strange[tid / 2][tid % 2] = 0;
        auto issue = [&](int i) {
            if (i < tiles) {
                const int key0 = key_first + i * kKeys;
                const uint32_t dst = ring_base + (i % S) * kStage;
                // lanes 0-7 look up the pages of eight keys each
                int in_page = 0;
                const int key = key0 + (lane & 7) * 8, found_page = key < k_end ? page_of(a.seq, seg.b, key, in_page) : -1;
                constexpr int kPass = 128 / CH;  // rows per pass of the block: 8 or 16
#pragma unroll
                for (int p = 0; p < kKeys / kPass; ++p) {
                    const int r = p * kPass + tid / CH, ch = tid % CH, group = r / 8;  // the same group for all lanes of a warp
                    const int page = __shfl_sync(~0u, found_page, group), row = __shfl_sync(~0u, in_page, group) + r % 8;
                    const bool there = page >= 0 && key0 + r < k_end;
                    const uint32_t at = dst + r * D * 2 + ((ch ^ (r & 7)) * 16);
                    const int64_t pg = there ? page : 0, rw = there ? row : 0;
                    copy16(at, a.k + pg * a.k_page + rw * a.k_row + seg.h * a.k_head + (there ? ch * 8 : 0), there);
                    copy16(at + kHalf, a.v + pg * a.v_page + rw * a.v_row + seg.h * a.v_head + (there ? ch * 8 : 0), there);
                }
            }
            copy_commit();
        };
        // ---- queries with the first tile
        for (int i = tid; i < R * CH; i += kWarps * 32) {
            const int r = i / CH, ch = i % CH;
            const bool there = r < rows;
            const int tok = (int)div_by((uint32_t)(f0 + (there ? r : 0)), d.by_g), head = seg.h * d.g + (f0 + (there ? r : 0) - tok * d.g);
            copy16(q_base + r * D * 2 + ((ch ^ (r & 7)) * 16), a.q + (int64_t)(seg.s.q0 + tok) * a.ldq + head * D + ch * 8, there);
        }
#pragma unroll
        for (int i = 0; i < S - 1; ++i) issue(i);
        int pos[2];  // of the rows this thread holds; rows behind the tile see what the last one does
#pragma unroll
        for (int i = 0; i < 2; ++i) pos[i] = past + (int)div_by((uint32_t)(f0 + min(w * 16 + i * 8 + lane / 4, rows - 1)), d.by_g);
        float o[NT][4], m[2] = {-kInf, -kInf}, l[2] = {0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < NT; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;
        uint32_t qf[KS][4];
        for (int i = 0; i < tiles; ++i) {
            copy_wait<S - 2>();
            __syncthreads();  // the tile is there, and all have done with the one before, whose room the next copies take
            issue(i + S - 1);
            if (i == 0) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int r = w * 16 + (lm & 1) * 8 + lr, ch = ks * 2 + (lm >> 1);
                    ldsm4(qf[ks], q_base + r * D * 2 + ((ch ^ (r & 7)) * 16));
                }
            }
            const uint32_t kb = ring_base + (i % S) * kStage, vb = kb + kHalf;
            const int key0 = key_first + i * kKeys;
            const bool masked = seg.k0 + i >= first_cut;
            if (masked && k_end - 1 > first_pos) {
                // A weight of 0 must not meet an infinity or NaN: keys that some row does not see give theirs up, and the rows that do
                // see them get them at the end.  (Keys from k_end on are zeros here.)
                const int lo = max(0, first_pos + 1 - key0), n = min(kKeys, k_end - key0) - lo;
                for (int j = tid; j < n * CH; j += kWarps * 32) {
                    uint4* const at = reinterpret_cast<uint4*>(ring + (i % S) * kStage + kHalf + (lo + j / CH) * D * 2 + j % CH * 16);
                    uint32_t x[4] = {at->x, at->y, at->z, at->w};
                    bool bad = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((x[e] & 0x7F80u) == 0x7F80u) x[e] &= 0xFFFF0000u, bad = true;
                        if ((x[e] & 0x7F800000u) == 0x7F800000u) x[e] &= 0xFFFFu, bad = true;
                    }
                    if (bad) {
                        *at = make_uint4(x[0], x[1], x[2], x[3]);
                        const int t = min(seg.k0 + i - first_cut, kTiles - 1), r = lo + j / CH;
                        atomicOr(&strange[t][r / 32], 1u << (r & 31));
                    }
                }
                __syncthreads();
            }
            float s[8][4];
#pragma unroll
            for (int n = 0; n < 8; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int n = 0; n < 8; n += 2) {
                    uint32_t kf[4];
                    const int r = n * 8 + (lm >> 1) * 8 + lr, ch = ks * 2 + (lm & 1);
                    ldsm4(kf, kb + r * D * 2 + ((ch ^ (r & 7)) * 16));
                    mma(s[n], qf[ks], kf[0], kf[1]);
                    mma(s[n + 1], qf[ks], kf[2], kf[3]);
                }
            if (masked) {
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (key0 + n * 8 + (lane & 3) * 2 + (e & 1) > pos[e >> 1]) s[n][e] = -kInf;
            }
            float top[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float x = fmaxf(s[0][2 * e], s[0][2 * e + 1]);
#pragma unroll
                for (int n = 1; n < 8; ++n) x = fmaxf(x, fmaxf(s[n][2 * e], s[n][2 * e + 1]));
                x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
                x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
                top[e] = fmaxf(m[e], x * a.c);
            }
            if (__any_sync(~0u, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float f = top[e] > m[e] ? ex2(m[e] - top[e]) : 1.0f;
                    m[e] = top[e];
                    l[e] *= f;
#pragma unroll
                    for (int n = 0; n < NT; ++n) o[n][2 * e] *= f, o[n][2 * e + 1] *= f;
                }
            }
            const float ref[2] = {m[0] == -kInf ? 0.0f : m[0], m[1] == -kInf ? 0.0f : m[1]};
#pragma unroll
            for (int k = 0; k < 4; ++k) {  // 16 keys at a time: their weights, and their product with the values
                uint32_t pf[4];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    float* const x = s[2 * k + n];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = ex2(fmaf(x[e], a.c, -ref[e >> 1]));
                        l[e >> 1] += x[e];
                    }
                    pf[2 * n] = pack_bf16(x[0], x[1]), pf[2 * n + 1] = pack_bf16(x[2], x[3]);
                }
#pragma unroll
                for (int n = 0; n < NT; n += 2) {
                    uint32_t vf[4];
                    const int r = k * 16 + (lm & 1) * 8 + lr, ch = n + (lm >> 1);
                    ldsm4_t(vf, vb + r * D * 2 + ((ch ^ (r & 7)) * 16));
                    mma(o[n], pf, vf[0], vf[1]);
                    mma(o[n + 1], pf, vf[2], vf[3]);
                }
            }
        }
        copy_wait<0>();
        const bool whole = seg.u0 == 0 && seg.u1 == seg.units;
        const int slot = 2 * cta + (seg.u0 == 0 ? 1 : 0);
        uint32_t any = 0;
        if (tiles > 0) {
#pragma unroll
            for (int t = 0; t < kTiles * 2; ++t) any |= strange[t / 2][t % 2];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float sum = l[e];
            sum += __shfl_xor_sync(~0u, sum, 1);
            sum += __shfl_xor_sync(~0u, sum, 2);
            const int r = w * 16 + e * 8 + lane / 4;
            if (r >= rows) continue;
            const float inv = whole ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f;
#pragma unroll
            for (int n = 0; n < NT; ++n) o[n][2 * e] *= inv, o[n][2 * e + 1] *= inv;
            if (any) {  // rare
                for (int t = 0; t < kTiles * 2; ++t)
                    for (uint32_t bits = strange[t / 2][t % 2]; bits; bits &= bits - 1) {
                        const int key = (first_cut + t / 2) * kKeys + t % 2 * 32 + __ffs(bits) - 1;
                        int in_page = 0;
                        const int page = key <= pos[e] ? page_of(a.seq, seg.b, key, in_page) : -1;
                        if (page < 0) continue;
                        const __nv_bfloat16* src = a.v + (int64_t)page * a.v_page + (int64_t)in_page * a.v_row + (int64_t)seg.h * a.v_head + (lane & 3) * 2;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const float x = __bfloat162float(src[n * 8]), y = __bfloat162float(src[n * 8 + 1]);
                            if (!(fabsf(x) < kInf)) o[n][2 * e] += x;
                            if (!(fabsf(y) < kInf)) o[n][2 * e + 1] += y;
                        }
                    }
            }
            if (whole) {
                const int tok = (int)div_by((uint32_t)(f0 + r), d.by_g), head = seg.h * d.g + (f0 + r - tok * d.g);
                const int64_t row = seg.s.q0 + tok;
                uint32_t* const dst = reinterpret_cast<uint32_t*>(a.out + row * a.ldo + head * D + (lane & 3) * 2);
#pragma unroll
                for (int n = 0; n < NT; ++n) dst[n * 4] = pack_bf16(o[n][2 * e], o[n][2 * e + 1]);
                if (a.lse && (lane & 3) == 0) a.lse[row * a.Hq + head] = sum == 0.0f ? -kInf : (m[e] + log2f(sum)) * kLn2;
            } else {
                const int64_t at = (int64_t)slot * R + r;
                float* const dst = a.part_o + at * D + (lane & 3) * 2;
#pragma unroll
                for (int n = 0; n < NT; ++n) *reinterpret_cast<float2*>(dst + n * 8) = make_float2(o[n][2 * e], o[n][2 * e + 1]);
                if ((lane & 3) == 0) a.part_ml[at] = make_float2(m[e], sum);
            }
        }
        if (first && tid == 0) a.notes[cta] = join_note(seg, start, cta, f0);
        first = false;
    }
    if (first && tid == 0) a.notes[cta].parts = 0;
    pdl_trigger();
}

// Where part p of an item lies whose second CTA is `cta`, row r.
__device__ __forceinline__ int64_t join_slot(int cta, int p, int R, int r) { return (int64_t)(p == 0 ? 2 * (cta - 1) + 1 : 2 * (cta - 1 + p)) * R + r; }
__device__ __forceinline__ void join_place(const AttnArgs& a, const JoinNote& note, int f, int64_t& row, int& head) {
    const int tok = (int)div_by((uint32_t)f, a.deal.by_g);
    head = note.h * a.deal.g + (f - tok * a.deal.g);
    row = note.q0 + tok;
}

// A row's parts p0 .. p1 - 1 by one warp, kDeep loads in flight: reference, sum and this lane's columns.
template <int D, int E, int kDeep>
__device__ __forceinline__ void join_parts(const AttnArgs& a, int cta, int p0, int p1, int R, int r, float& ref, float& sum, float (&acc)[E]) {
    const int lane = threadIdx.x & 31;
    ref = -kInf, sum = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
    for (int b = p0; b < p1; b += kDeep) {
        float2 q[kDeep];
        float x[kDeep][E];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            q[i] = make_float2(-kInf, 0.0f);
            if (b + i >= p1) continue;
            const int64_t at = join_slot(cta, b + i, R, r);
            q[i] = a.part_ml[at];
            if (E == 4) {
                const float4 v = *reinterpret_cast<const float4*>(a.part_o + at * D + lane * E);
                x[i][0] = v.x, x[i][1] = v.y, x[i][2 % E] = v.z, x[i][3 % E] = v.w;
            } else {
                const float2 v = *reinterpret_cast<const float2*>(a.part_o + at * D + lane * E);
                x[i][0] = v.x, x[i][1] = v.y;
            }
        }
        float top = ref;
#pragma unroll
        for (int i = 0; i < kDeep; ++i) top = fmaxf(top, q[i].x);
        const float f0 = join_weight(make_float2(ref, sum), top);
        ref = top, sum *= f0;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= f0;
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            if (no_share(q[i])) continue;
            const float f = join_weight(q[i], ref);
            sum = fmaf(f, q[i].y, sum);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(f, x[i][e], acc[e]);
        }
    }
}

// Joins the parts of the items that attn_rows_kernel had to cut, in a fixed order: block (i, y) those of the item whose second CTA
// is i, rows 8 y .. 8 y + 7, a warp per row.  An item of many parts (a long sequence by itself is cut into as many as the device
// has CTAs) has its rows one by one, y, y + grid.y, ..., and the eight warps share a row's parts.
template <int D>
__global__ void __launch_bounds__(256) attn_join_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int E = D / 32, W = 8, kDeep = 8;
    __shared__ float2 warp_ml[W];
    __shared__ float warp_o[W][D];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, cta = blockIdx.x;
    pdl_wait();
    pdl_trigger();
    const JoinNote note = a.notes[cta];
    if (note.parts == 0) return;
    const int R = a.deal.rows, rows = min(R, note.n * a.deal.g - note.f0);
    float ref, sum, acc[E];
    auto write = [&](int r) {
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        int64_t row;
        int head;
        join_place(a, note, note.f0 + r, row, head);
        uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + row * a.ldo + head * D + lane * E);
#pragma unroll
        for (int e = 0; e < E; e += 2) dst[e / 2] = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
        if (a.lse && lane == 0) a.lse[row * a.Hq + head] = sum == 0.0f ? -kInf : (ref + log2f(sum)) * kLn2;
    };
    if (note.parts <= 3 * kDeep) {
        const int r = blockIdx.y * W + w;
        if (r >= rows) return;
        join_parts<D, E, kDeep>(a, cta, 0, note.parts, R, r, ref, sum, acc);
        write(r);
        return;
    }
    const int per = (note.parts + W - 1) / W, p0 = min(w * per, note.parts), p1 = min(p0 + per, note.parts);
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        join_parts<D, E, kDeep>(a, cta, p0, p1, R, r, ref, sum, acc);
        if (lane == 0) warp_ml[w] = make_float2(ref, sum);
#pragma unroll
        for (int e = 0; e < E; ++e) warp_o[w][lane * E + e] = acc[e];
        __syncthreads();
        if (w == 0) {
            ref = -kInf, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) ref = fmaxf(ref, warp_ml[i].x);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (no_share(warp_ml[i])) continue;
                const float f = join_weight(warp_ml[i], ref);
                sum = fmaf(f, warp_ml[i].y, sum);
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = fmaf(f, warp_o[i][lane * E + e], acc[e]);
            }
            write(r);
        }
        __syncthreads();
    }
}

// The same for attn_chunk_kernel, whose parts lie with the rows of a column side by side: block (i, y) rows 32 y .. + 31 of the item,
// a row per lane, 16 columns per warp.
template <int D>
__global__ void __launch_bounds__(D * 2) attn_join_tiles_kernel(const __grid_constant__ AttnArgs a) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, cta = blockIdx.x;
    pdl_wait();
    pdl_trigger();
    const JoinNote note = a.notes[cta];
    const int R = a.deal.rows, r = blockIdx.y * 32 + lane, f = note.f0 + r;
    if (note.parts == 0 || r >= R || f >= note.n * a.deal.g) return;
    float ref = -kInf, sum = 0.0f, acc[16] = {};
    constexpr int kDeep = 4;
    for (int b = 0; b < note.parts; b += kDeep) {
        float2 q[kDeep];
        float x[kDeep][16];
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            q[k] = make_float2(-kInf, 0.0f);
            if (b + k >= note.parts) continue;
            const int64_t at = join_slot(cta, b + k, R, r);
            q[k] = a.part_ml[at];
            const float* const src = a.part_o + ((at - r) * D + (int64_t)w * 16 * R) + r;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[k][i] = src[i * R];
        }
        float top = ref;
#pragma unroll
        for (int k = 0; k < kDeep; ++k) top = fmaxf(top, q[k].x);
        const float f0 = join_weight(make_float2(ref, sum), top);
        ref = top, sum *= f0;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] *= f0;
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            if (no_share(q[k])) continue;
            const float weight = join_weight(q[k], ref);
            sum = fmaf(weight, q[k].y, sum);
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[i] = fmaf(weight, x[k][i], acc[i]);
        }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    int64_t row;
    int head;
    join_place(a, note, f, row, head);
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] *= inv;
    const float lo[8] = {acc[0], acc[1], acc[2], acc[3], acc[4], acc[5], acc[6], acc[7]}, hi[8] = {acc[8], acc[9], acc[10], acc[11], acc[12], acc[13], acc[14], acc[15]};
    __nv_bfloat16* const dst = a.out + row * a.ldo + head * D + w * 16;
    store8(dst, lo, 8);
    store8(dst + 8, hi, 8);
    if (a.lse && w == 0) a.lse[row * a.Hq + head] = chunk_lse(ref, sum);
}

// Workspace: notes, then the partial sums of two slots per CTA.
struct Layout {
    int ctas, rows;
    size_t ml, o, bytes;
};
Layout layout(int64_t D, int rows, int ctas) {
    Layout l;
    l.ctas = ctas, l.rows = rows;
    l.ml = kWsHeader + align_up((size_t)ctas * sizeof(JoinNote), 256);
    l.o = l.ml + align_up((size_t)2 * ctas * rows * sizeof(float2), 256);
    l.bytes = l.o + (size_t)2 * ctas * rows * (size_t)D * 4;
    return l;
}
// The kernel and its tiles, from what the host knows of a sequence's query rows per kv head: up to 16 or 32 rows are one or two
// tiles of the register-operand instruction, more go to the tensor-memory form.
struct Choice {
    bool chunk;
    int rows, ctas;
};
constexpr int kPlanSms = 148;  // the workspace query answers without a device
Choice choose(int64_t T, int64_t Hq, int64_t Hkv, int64_t max_new) {
    const int64_t n = max_new > 0 ? std::min(max_new, T) : T, rows = n * (Hq / Hkv);
    if (rows > 64) return Choice{true, attn_chunk_rows((int)(Hq / Hkv)), kPlanSms};
    return Choice{false, rows <= 16 ? 16 : rows <= 32 ? 32 : 64, kPlanSms * kRowsCtasPerSm};
}

}  // namespace
}  // namespace resq

using namespace resq;

extern "C" {

size_t resq_paged_attention_workspace_bytes(int64_t T, int64_t count, int64_t Hq, int64_t Hkv, int64_t D, int64_t max_new) {
    if (T <= 0 || count <= 0 || Hkv <= 0 || Hq <= 0 || Hq % Hkv || Hq / Hkv > RESQ_MAX_GROUP_HEADS || (D != 64 && D != 128)) return 0;
    const Choice c = choose(T, Hq, Hkv, max_new);
    return layout(D, c.rows, c.ctas).bytes;
}

int resq_paged_attention(const void* Q, int64_t T, int64_t ldq, int64_t Hq, int64_t Hkv, int64_t D, const resq_paged_cache* cache,
                         const resq_sequences* seqs, int64_t max_new, float scale, void* O, int64_t ldo, float* lse, void* workspace, size_t ws_bytes,
                         void* stream) {
    const char* what = "paged_attention";
    if (!Q || !O) return fail(RESQ_ERR_NULL, what, "Q and O must not be NULL");
    int rc = check_paged(what, cache, seqs, T, Hq, Hkv, D);
    if (rc) return rc;
    if (!(scale > 0.0f) || !std::isfinite(scale * kLog2e)) return fail(RESQ_ERR_SHAPE, what, "scale must be positive and below 2.3e38");
    if (!rows_aligned(Q, ldq, Hq * D, RESQ_OUT_BF16) || !rows_aligned(O, ldo, Hq * D, RESQ_OUT_BF16) || !is_aligned(lse, 4))
        return fail(RESQ_ERR_ALIGN, what, "Q and O need 16-byte aligned bases and rows of at least Hq * D elements, lse 4-byte alignment");
    Choice ch = choose(T, Hq, Hkv, max_new);
    Layout l = layout(D, ch.rows, ch.ctas);
    if (!workspace || !is_aligned(workspace, 256) || ws_bytes < l.bytes) {
        set_last_error("paged_attention: workspace needs %zu bytes (256-byte aligned), got %zu", l.bytes, ws_bytes);
        return RESQ_ERR_WORKSPACE;
    }
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    using bf = __nv_bfloat16;
    AttnArgs a;
    a.seq = seq_args(*cache, *seqs, T);
    a.deal = make_deal(l.rows, ch.chunk ? kChunkKeys : kKeys, (int)Hkv, (int)(Hq / Hkv), ch.chunk ? kChunkExtra : 0);
    a.q = static_cast<const bf*>(Q), a.k = static_cast<const bf*>(cache->k), a.v = static_cast<const bf*>(cache->v);
    a.ldq = ldq, a.ldo = ldo;
    a.k_page = cache->k_page, a.k_row = cache->k_row, a.k_head = cache->k_head;
    a.v_page = cache->v_page, a.v_row = cache->v_row, a.v_head = cache->v_head;
    // Tiles a CTA takes at least: with up to 32 rows a part costs less than the tile it saves (one decoded token at 4000 keys: 12.1 us with
    // one, 13.3 with two); with more, joining does (40 rows at 4000 keys: 20.6 us with one, 15.9 with three, 18.7 with four).
    a.out = static_cast<bf*>(O), a.lse = lse, a.Hq = (int)Hq, a.c = scale * kLog2e, a.min_chunk = ch.rows == 64 ? 3 : 1;
    if (ch.chunk && !attn_chunk_supported(a)) {  // a stride of 0: no tensor map takes it; this workspace is smaller
        ch = Choice{false, 32, kPlanSms * kRowsCtasPerSm};
        l = layout(D, ch.rows, ch.ctas);
        a.deal = make_deal(l.rows, kKeys, (int)Hkv, (int)(Hq / Hkv), 0);
    }
    a.status = reinterpret_cast<DeviceStatus*>(ws);
    a.notes = reinterpret_cast<JoinNote*>(ws + kWsHeader);
    a.part_ml = reinterpret_cast<float2*>(ws + l.ml);
    a.part_o = reinterpret_cast<float*>(ws + l.o);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (ch.chunk) {
        rc = launch_attn_chunk(a, (int)D, l.ctas, st);
        if (rc) return rc;
        LaunchScope scope(kKindRow, st);
        return cuda_fail(launch_kernel(D == 128 ? attn_join_tiles_kernel<128> : attn_join_tiles_kernel<64>, dim3((unsigned)l.ctas, (unsigned)((l.rows + 31) / 32)),
                                       dim3((unsigned)(2 * D)), 0, st, a),
                         "attn_join_tiles_kernel launch");
    }
    auto kern = D == 128 ? (l.rows == 16 ? attn_rows_kernel<128, 1> : l.rows == 32 ? attn_rows_kernel<128, 2> : attn_wide_kernel<128>)
                         : (l.rows == 16 ? attn_rows_kernel<64, 1> : l.rows == 32 ? attn_rows_kernel<64, 2> : attn_wide_kernel<64>);
    const int smem = D == 128 ? (l.rows == 16 ? rows_smem<128, 1>() : l.rows == 32 ? rows_smem<128, 2>() : wide_smem<128>())
                              : (l.rows == 16 ? rows_smem<64, 1>() : l.rows == 32 ? rows_smem<64, 2>() : wide_smem<64>());
    rc = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem, "attn_rows_kernel shared memory");
    if (rc) return rc;
    {
        LaunchScope scope(kKindRow, st);
        rc = cuda_fail(launch_kernel(kern, dim3((unsigned)l.ctas), dim3(kWarps * 32), (size_t)smem, st, a), "attn_rows_kernel launch");
        if (rc) return rc;
    }
    LaunchScope scope(kKindRow, st);
    return cuda_fail(launch_kernel(D == 128 ? attn_join_kernel<128> : attn_join_kernel<64>, dim3((unsigned)l.ctas, 8), dim3(256), 0, st, a),
                     "attn_join_kernel launch");
}

}  // extern "C"
