// Attention of chunks of new tokens over a paged cache: the tensor-core form of resq_paged_attention (formulas in
// paged_attention.cu), for sequences with more query rows per kv head than attn_rows_kernel takes.
//
// A tile is two halves of up to 128 query rows (tokens times the heads that share a kv head, whole tokens per half), the keys come
// in tiles of 128.  Scores S = Q K^T of a half fill 128 columns of tensor memory, its softmax warps replace them by the weights P
// (bf16, in the same columns), which are the A operand of O += P V from there; S and O of both halves are all 512 columns.  While the
// warps of one half are at their exponentials the tensor cores have the other half's products to do, with K and V read into
// shared memory once for both.  An item with rows for one half only is worked on by both halves, on every second key tile each,
// and their sums are joined at its end.
//
// Warps: 0-3 and 4-7 softmax of a half (a row per thread, so maxima and sums need no exchange), 8 and 9 issue a half's products, 10
// deals out segments and loads (a page's rows per copy, page numbers looked up by its lanes), 11 repairs the value tiles that reach
// past the first row's last key: rows behind the last key become zeros (0 times what a page holds there may be NaN), and
// infinities and NaN are taken out and added by those rows that do see them.
//
// O is rescaled only when a row's maximum has grown by more than 20 in the exponent of 2 since its reference was set.  The reference
// lies those 20 above the maximum that it was set by: weights are at most 1, so that sums with large values overflow no sooner than
// they have to, lose nothing in bf16 or fp32 by being 2^-20, and the final division takes the reference out.
//
// Measured: 8192 tokens from the beginning, 28 heads on 4 of 128, 562 us = 856 TFLOP/s (0.52 of the burst rate of a library product);
// 512 tokens behind 31500 keys, 16 heads on 2, two sequences, 299 us = 880 TFLOP/s.  The products alone, with the weights left
// as they lie, take 379 and 214 us: S = Q K^T is bound by the reads of both operands from shared memory (115 cycles an
// instruction instead of 64).  The rest is the way from scores to weights: 512 cycles for a half's scores out of tensor memory and
// their maxima, 1024 for its 16384 exponentials (16 a clock), 600 of hand-overs, of which the other half hides the part that its
// own phase allows.
#include "paged.cuh"
#include "ptx.cuh"

namespace resq {
namespace {

constexpr float kInf = __builtin_huge_valf();
constexpr int kKeys = kChunkKeys, kHalf = 128;
constexpr int kMmaWarp = 8, kLoadWarp = 10, kFixWarp = 11, kThreads = 384;  // products: warps 8 and 9
constexpr int kDescs = 4;    // segments described ahead of the slowest reader
constexpr int kStrange = 4;  // key tiles of a segment that can hold keys of its own tokens (at most 256)
// Registers per thread: 168 at the launch; the eight softmax warps take what the other four give up.
constexpr int kSoftmaxRegs = 200, kOtherRegs = 104;
static_assert(256 * kSoftmaxRegs + 128 * kOtherRegs <= kThreads * 168, "");

template <int D>
constexpr int stages() { return D == 128 ? 5 : 10; }  // 160 KB of key and value tiles
template <int D>
constexpr int tile_bytes() { return kKeys * D * 2; }

struct ChunkMaps {
    CUtensorMap q, k, v;
};
struct ChunkArgs {
    AttnArgs a;
    int half_rows, half_tokens;  // of a half tile
    int box;                     // keys per copy: a power of two that divides the page and the tile
    int wide;                    // rows of the output start on 32-byte boundaries
    int expire;                  // test hook: the repairs wait for what does not come
};

struct ChunkSeg {
    int b, q0, n, h, f0, past, k_end, first_pos;
    int u0, end, slot;           // key tiles u0 .. end - 1 are to be read; slot: of the partial result, -1: the whole item
    int rows[2], stop[2];        // per half: rows, key tiles u0 .. stop - 1
    int split;                   // rows for one half only: both work on them, on every second key tile each
};
struct ChunkShared {
    uint64_t desc_full[kDescs], desc_empty[kDescs], strange_full[kDescs];
    uint64_t q_full[2], q_empty[2], s_full[2], p_full[2][2], o_full[2], merge_full, merge_free, done[2], never;
    uint64_t kv_full[10], kv_empty[10], raw_full[10];
    ChunkSeg seg[kDescs];
    float2 other[kHalf];                    // of a split segment's second half: reference and sum of each row
    uint32_t strange[kDescs][kStrange][4];  // a bit per key whose value row holds an infinity or NaN
    int64_t sums[kThreads / 32];
    DealStart found;
    uint32_t tmem;
    int abort;
};

static_assert(2 * kHalf * 128 * 2 + stages<128>() * tile_bytes<128>() + sizeof(ChunkShared) <= 232448, "227 KB");

__device__ __forceinline__ void chunk_timeout(DeviceStatus* st, int where) {
    st->where = where;
    st->block = (int)blockIdx.x;
    st->code = RESQ_ERR_TIMEOUT;
}
// A wait of all lanes with one answer for them all: lanes that gave up apart would part the warp.  It does not let the warp sleep:
// every role's answer is on the way of the next product.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint32_t polls = 1u << 24) {
    return __all_sync(~0u, ptx::mbar_wait_spin(bar, parity, abort_flag, polls));
}
// Polls of a wait that may take as long as `tiles` key tiles do: 250 are 6000 cycles, twice what a tile takes.
__device__ __forceinline__ uint32_t long_wait(int tiles) { return (1u << 24) + 250u * (uint32_t)tiles; }
// Waits for what is under way in any case, without a look at the others: 0.4 ms at most.
__device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity) {
    for (int i = 0; i < 4096 && !ptx::mbar_test_wait(bar, parity); ++i) __nanosleep(100);
}
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {  // NaN if one of them is
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
template <int N>
__device__ __forceinline__ void more_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void fewer_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
__device__ __forceinline__ bool strange_pair(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }

template <int D>
__global__ void __launch_bounds__(kThreads, 1) attn_chunk_kernel(const __grid_constant__ ChunkArgs p, const __grid_constant__ ChunkMaps maps) {
    constexpr int ST = stages<D>(), TILE = tile_bytes<D>(), CG = D / 64, QH = kHalf * D * 2;  // column groups of 64
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* const q_smem = smem;                // [half][column group][128 rows][128 bytes]
    unsigned char* const ring = smem + 2 * QH;         // [stage][column group][128 keys][128 bytes]
    ChunkShared& sh = *reinterpret_cast<ChunkShared*>(ring + ST * TILE);
    const AttnArgs& a = p.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
    volatile int* const abort_flag = &sh.abort;

    if (tid == 0) {
        for (int i = 0; i < kDescs; ++i) {
            ptx::mbar_init(&sh.desc_full[i], 1);
            ptx::mbar_init(&sh.desc_empty[i], 11);  // eight softmax warps, products of two halves, repairs
            ptx::mbar_init(&sh.strange_full[i], 1);
        }
        for (int h = 0; h < 2; ++h) {
            ptx::mbar_init(&sh.q_full[h], 1);
            ptx::mbar_init(&sh.q_empty[h], h == 0 ? 2 : 1);  // the first half's queries: the products of both halves
            ptx::mbar_init(&sh.s_full[h], 1);
            ptx::mbar_init(&sh.p_full[h][0], 4);  // the weights of the first 64 keys, of the others
            ptx::mbar_init(&sh.p_full[h][1], 4);
            ptx::mbar_init(&sh.o_full[h], 1);
            ptx::mbar_init(&sh.done[h], 1);
        }
        ptx::mbar_init(&sh.merge_full, 4);
        ptx::mbar_init(&sh.merge_free, 4);
        ptx::mbar_init(&sh.never, 1);
        for (int i = 0; i < ST; ++i) {
            ptx::mbar_init(&sh.kv_full[i], 1);
            ptx::mbar_init(&sh.kv_empty[i], 2);  // the products of both halves
            ptx::mbar_init(&sh.raw_full[i], 1);
        }
        ptx::mbar_fence_init();
        sh.abort = 0;
    }
    if (warp == kMmaWarp) ptx::tmem_alloc(&sh.tmem, 512);
    if (warp == kLoadWarp && lane == 0) {
        ptx::tma_prefetch_desc(&maps.q);
        ptx::tma_prefetch_desc(&maps.k);
        ptx::tma_prefetch_desc(&maps.v);
    }
    pdl_wait();
    if (cta == 0 && tid == 0) *a.status = DeviceStatus{RESQ_OK, 0, 0, 0};
    ptx::tc_fence_before();
    const DealStart start = deal_start(a.seq, a.deal, cta, gridDim.x, a.min_chunk, sh.sums, &sh.found);  // orders the block
    ptx::tc_fence_after();
    const uint32_t tmem = sh.tmem;

    // (The four warps of a group change their registers together, before they part.)
    if (warp >= kMmaWarp) {
        fewer_registers<kOtherRegs>();
        if (warp == kLoadWarp) {
            // ------------------------------------------------------------------ segments, queries, keys and values
            DealWalk walk;
            walk.init(a.seq, a.deal, start);
            Segment s;
            int count = 0, q_uses[2] = {0, 0}, q_loads[2] = {0, 0};
            uint32_t pos = 0;                // key and value tiles so far
            uint32_t raw = 0, raw_turn = 0;  // per stage: its tile goes to the repairs; parity of those that did
            bool ok = true;
            while (ok && walk.next(a.seq, a.deal, s)) {
                const int e = count % kDescs;
                if (!(ok = warp_wait(&sh.desc_empty[e], ((count / kDescs) & 1) ^ 1, abort_flag))) break;
                ChunkSeg g;
                g.b = s.b, g.q0 = s.s.q0, g.n = s.s.n, g.h = s.h, g.f0 = s.t * a.deal.rows;
                g.past = s.s.kv - s.s.n, g.k_end = deal_k_end(s.s, a.deal, s.t);
                const int tok0 = (int)div_by((uint32_t)g.f0, a.deal.by_g);
                g.first_pos = g.past + tok0;
                g.u0 = s.k0, g.end = s.k0;
                g.slot = s.u0 == 0 && s.u1 == s.units ? -1 : 2 * cta + (s.u0 == 0 ? 1 : 0);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    g.rows[h] = max(0, min(p.half_rows, s.s.n * a.deal.g - g.f0 - h * p.half_rows));
                    const int last = min(tok0 + (h + 1) * p.half_tokens, s.s.n) - 1;  // last token of the half
                    const int k_end = max(0, min(g.past + last + 1, s.s.kv));
                    g.stop[h] = g.rows[h] == 0 ? s.k0 : max(s.k0, min(s.k1, (k_end + kKeys - 1) / kKeys));
                    g.end = max(g.end, g.stop[h]);
                }
                g.split = g.rows[1] == 0;
                if (g.split) g.stop[1] = g.stop[0];
                if (lane == 0) {
                    if (count == 0) a.notes[cta] = join_note(s, start, cta, g.f0);
                    sh.seg[e] = g;
                    for (int i = 0; i < kStrange * 4; ++i) sh.strange[e][i / 4][i % 4] = 0;
                    ptx::mbar_arrive(&sh.desc_full[e]);
                }
                __syncwarp();
                // where this lane's piece of key tile u lies; asked for a tile ahead, since the answer takes as long as a copy
                int page = 0, within = 0, next_page = 0, next_within = 0;
                auto look = [&](int u) {
                    const int key = u * kKeys + lane * p.box;
                    if (lane * p.box < kKeys && key < g.k_end) {
                        next_page = page_of(a.seq, g.b, key, next_within);
                        if (next_page < 0) next_page = a.seq.pages;  // outside the cache: zeros
                    }
                };
                // one tile of keys or values
                auto load = [&](int u, const CUtensorMap* m, bool special) {
                    const int st = pos % ST;
                    if (!warp_wait(&sh.kv_empty[st], ((pos / ST) & 1) ^ 1, abort_flag)) return false;
                    ++pos;
                    raw = special ? raw | 1u << st : raw & ~(1u << st);
                    raw_turn ^= (uint32_t)special << st;
                    uint64_t* const bar = special ? &sh.raw_full[st] : &sh.kv_full[st];
                    const int pieces = min(kKeys / p.box, (g.k_end - u * kKeys + p.box - 1) / p.box);
                    if (lane == 0) ptx::mbar_arrive_expect_tx(bar, (uint32_t)(pieces * p.box * D * 2));
                    __syncwarp();
                    if (lane < pieces) {
                        unsigned char* const dst = ring + st * TILE + lane * p.box * 128;
#pragma unroll
                        for (int c = 0; c < CG; ++c) ptx::tma_load_4d(dst + c * kKeys * 128, m, bar, c * 64, within, g.h, page);
                    }
                    __syncwarp();
                    return true;
                };
                auto special = [&](int u) { return u * kKeys + kKeys - 1 > g.first_pos; };
                if (g.end > g.u0) {
                    look(g.u0);
                    page = next_page, within = next_within;
                    look(g.u0 + 1);
                    ok = load(g.u0, &maps.k, false);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // (a split segment's second half has no queries of its own; where it has keys, its sums use their room at the end)
                    if (!ok || g.stop[h] <= g.u0 + (h == 1 && g.split)) continue;
                    if (!(ok = warp_wait(&sh.q_empty[h], (q_uses[h] & 1) ^ 1, abort_flag))) continue;
                    ++q_uses[h];
                    if (h == 1 && g.split) continue;
                    ++q_loads[h];
                    if (lane == 0) {
                        ptx::mbar_arrive_expect_tx(&sh.q_full[h], (uint32_t)(p.half_rows * D * 2));
#pragma unroll
                        for (int c = 0; c < CG; ++c)
                            ptx::tma_load_3d(q_smem + h * QH + c * kHalf * 128, &maps.q, &sh.q_full[h], c * 64, g.h * a.deal.g, g.q0 + tok0 + h * p.half_tokens);
                    }
                    __syncwarp();
                }
                for (int u = g.u0; ok && u < g.end; ++u) {
                    ok = load(u, &maps.v, special(u));
                    if (!ok || u + 1 == g.end) continue;
                    page = next_page, within = next_within;
                    look(u + 2);
                    ok = load(u + 1, &maps.k, false);
                }
                ++count;
            }
            if (lane == 0) {
                if (count == 0 && ok) a.notes[cta].parts = 0;
                if (!ok) {
                    chunk_timeout(a.status, 1);
                } else {
                    // an empty description ends the others' loops
                    const int e = count % kDescs;
                    if (ptx::mbar_wait_spin(&sh.desc_empty[e], ((count / kDescs) & 1) ^ 1, abort_flag)) {
                        sh.seg[e].b = -1;
                        ptx::mbar_arrive(&sh.desc_full[e]);
                    } else chunk_timeout(a.status, 2);
                }
                // Copies in flight write to this CTA's shared memory: whoever has given up, they are waited for, with a limit.
                for (int h = 0; h < 2; ++h)
                    if (q_loads[h] > 0) drain(&sh.q_full[h], (q_loads[h] - 1) & 1);
                for (uint32_t q = pos > ST ? pos - ST : 0; q < pos; ++q) {
                    const int st = q % ST;
                    if ((raw >> st) & 1) drain(&sh.raw_full[st], ((raw_turn >> st) & 1) ^ 1);
                    else drain(&sh.kv_full[st], (q / ST) & 1);
                }
            }
        } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
            // ------------------------------------------------------------------ products of a half
            // Few products are taken ahead of their execution: a thread that waits leaves the tensor cores idle unless another one has
            // products for them.  So each half has a thread of its own.
            if (lane == 0) {
                const int h = warp - kMmaWarp;
                constexpr uint32_t s_idesc = ptx::idesc_bf16_f32(128, kKeys), o_idesc = ptx::idesc_bf16_f32_bmn(128, D);
                const uint64_t q_desc = ptx::smem_desc_sw128_kmajor(ptx::smem_u32(q_smem));
                const uint64_t k_desc = ptx::smem_desc_sw128_kmajor(ptx::smem_u32(ring)), v_desc = ptx::smem_desc_sw128_mnmajor(ptx::smem_u32(ring), kKeys * 128);
                const uint32_t s_at = tmem + h * 128, o_at = tmem + 256 + h * D;
                uint32_t pos = 0;  // of the segment's first key tile; tile i's values are at pos + 2 i + 1, tile i + 1's keys behind them
                uint32_t q_uses[2] = {0, 0}, p_uses = 0;
                bool ok = true;
                auto wait = [&](uint64_t* bar, uint32_t parity) { return ptx::mbar_wait_spin(bar, parity, abort_flag); };
                auto full = [&](uint32_t at) { return wait(&sh.kv_full[at % ST], (at / ST) & 1); };
                auto scores = [&](uint64_t q_desc, uint32_t k_pos) {
                    const uint64_t kd = k_desc + (uint64_t)((k_pos % ST) * (TILE >> 4));
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t off = (uint64_t)(((k / 4) * kHalf * 128 + (k % 4) * 32) >> 4);
                        ptx::umma_bf16(s_at, q_desc + off, kd + off, s_idesc, k > 0);
                    }
                    ptx::umma_commit(&sh.s_full[h]);
                };
                auto values = [&](uint32_t v_pos, int part, bool add) {  // keys 64 part .. + 63 of the tile
                    const uint64_t vd = v_desc + (uint64_t)((v_pos % ST) * (TILE >> 4));
#pragma unroll
                    for (int k = part * 4; k < part * 4 + 4; ++k)
                        ptx::umma_bf16_ta(o_at, s_at + k * 8, vd + (uint64_t)((k * 2048) >> 4), o_idesc, add || k > part * 4);
                };
                // tiles this half has no use for: given back once they are there (before, the arrival could count for the buffer's turn before)
                auto skip = [&](uint32_t from, uint32_t to) {
                    for (; from < to; ++from) {
                        if (!full(from)) return false;
                        ptx::mbar_arrive(&sh.kv_empty[from % ST]);
                    }
                    return true;
                };
                for (int count = 0; ok; ++count) {
                    const int e = count % kDescs;
                    if (!(ok = wait(&sh.desc_full[e], (count / kDescs) & 1))) break;
                    if (sh.seg[e].b < 0) break;
                    const int u0 = sh.seg[e].u0, tiles = sh.seg[e].end - u0, split = sh.seg[e].split;
                    const int step = split ? 2 : 1, first = split ? h : 0, end = sh.seg[e].stop[h] - u0;  // tiles first, first + step .. below end
                    const int from = split ? 0 : h;                                                        // whose queries
                    const uint64_t qd = q_desc + (uint64_t)(from * (QH >> 4));
                    // the other half's queries
                    if (h == 1 && (!split || first >= end) && sh.seg[e].stop[0] > u0) {
                        if (!(ok = wait(&sh.q_full[0], q_uses[0] & 1))) break;
                        ptx::mbar_arrive(&sh.q_empty[0]);
                    }
                    uint32_t done = pos;  // tiles up to here are given back, or will be when the products with them are done
                    if (first < end) {
                        const uint32_t at = pos + 2 * first;
                        if (!(ok = skip(done, at) && full(at) && wait(&sh.q_full[from], q_uses[from] & 1))) break;
                        ptx::tc_fence_after();
                        scores(qd, at);
                        if (first + step >= end) ptx::umma_commit(&sh.q_empty[from]);
                        ptx::umma_commit(&sh.kv_empty[at % ST]);
                        done = at + 1;
                    }
                    for (int i = first; ok && i < end; i += step) {
                        const uint32_t v_pos = pos + 2 * i + 1, k_pos = v_pos + 2 * step - 1;
                        const bool more = i + step < end;
                        // The tiles first: they are there by then, and asking costs time that the weights would wait for.  (The next keys of a
                        // split segment are four tiles on, which may have to wait for the room of these values.)
                        if (!(ok = full(v_pos) && (!more || split || full(k_pos)))) break;
                        if (!(ok = wait(&sh.p_full[h][0], p_uses & 1))) break;
                        ptx::tc_fence_after();
                        values(v_pos, 0, i > first);
                        if (!(ok = wait(&sh.p_full[h][1], p_uses & 1))) break;
                        ++p_uses;
                        ptx::tc_fence_after();
                        values(v_pos, 1, true);
                        if (more && !split) {
                            scores(qd, k_pos);
                            if (i + 2 * step >= end) ptx::umma_commit(&sh.q_empty[from]);
                            ptx::umma_commit(&sh.kv_empty[v_pos % ST]);
                            ptx::umma_commit(&sh.kv_empty[k_pos % ST]);
                            done = k_pos + 1;
                            continue;
                        }
                        if (!more) ptx::umma_commit(&sh.o_full[h]);
                        ptx::umma_commit(&sh.kv_empty[v_pos % ST]);
                        done = v_pos + 1;
                        if (!more) break;
                        if (!(ok = skip(done, k_pos) && full(k_pos))) break;
                        ptx::tc_fence_after();
                        scores(qd, k_pos);
                        if (i + 2 * step >= end) ptx::umma_commit(&sh.q_empty[from]);
                        ptx::umma_commit(&sh.kv_empty[k_pos % ST]);
                        done = k_pos + 1;
                    }
                    ok = ok && skip(done, pos + 2 * tiles);
                    if (sh.seg[e].stop[0] > u0) ++q_uses[0];
                    if (!split && sh.seg[e].stop[1] > u0) ++q_uses[1];
                    pos += 2 * tiles;
                    if (ok) ptx::mbar_arrive(&sh.desc_empty[e]);
                }
                if (!ok) chunk_timeout(a.status, 3);
            }
        } else if (warp == kFixWarp) {
            // ------------------------------------------------------------------ repairs of value tiles
            uint32_t pos = 0, raw_turn = 0;  // parity of the next repaired tile of each stage
            uint32_t polls = long_wait(0);  // this warp waits for the end of the segment that the others are at
            bool ok = !p.expire || warp_wait(&sh.never, 0, abort_flag, 1u << 12);
            for (int count = 0; ok; ++count) {
                const int e = count % kDescs;
                if (!(ok = warp_wait(&sh.desc_full[e], (count / kDescs) & 1, abort_flag, polls))) break;
                const ChunkSeg g = sh.seg[e];
                if (g.b < 0) break;
                polls = long_wait(g.end - g.u0);
                const int us = max(g.u0, (max(g.first_pos, -1) + 1) / kKeys);  // first tile that reaches past the first row's last key
                for (int u = us; ok && u < g.end; ++u) {
                    const uint32_t at = pos + 2 * (u - g.u0) + 1;
                    const int st = at % ST;
                    if (!(ok = warp_wait(&sh.raw_full[st], (raw_turn >> st) & 1, abort_flag, polls))) break;
                    raw_turn ^= 1u << st;
                    unsigned char* const tile = ring + st * TILE;
                    const int key0 = u * kKeys, valid = min(kKeys, g.k_end - key0);
                    for (int i = lane; i < (kKeys - valid) * CG * 8; i += 32) {
                        const int r = valid + i / (CG * 8), c = i % (CG * 8);
                        *reinterpret_cast<uint4*>(tile + (c / 8) * kKeys * 128 + r * 128 + (c % 8) * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    const int lo = max(0, g.first_pos + 1 - key0);
                    const int chunks = (valid - lo) * CG * 8;
                    for (int base = lane; base < chunks; base += 32 * 8) {
                        uint4 x[8];
                        auto place = [&](int n) {
                            const int i = base + n * 32, r = lo + i / (CG * 8), c = i % (CG * 8);
                            return reinterpret_cast<uint4*>(tile + (c / 8) * kKeys * 128 + r * 128 + (c % 8) * 16);
                        };
#pragma unroll
                        for (int n = 0; n < 8; ++n) x[n] = base + n * 32 < chunks ? *place(n) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                        for (int n = 0; n < 8; ++n)
                            if (strange_pair(x[n].x) || strange_pair(x[n].y) || strange_pair(x[n].z) || strange_pair(x[n].w)) {
                                const int r = lo + (base + n * 32) / (CG * 8);
                                auto clean = [](uint32_t v) {
                                    if ((v & 0x7F80u) == 0x7F80u) v &= 0xFFFF0000u;
                                    if ((v & 0x7F800000u) == 0x7F800000u) v &= 0xFFFFu;
                                    return v;
                                };
                                *place(n) = make_uint4(clean(x[n].x), clean(x[n].y), clean(x[n].z), clean(x[n].w));
                                if (u - us < kStrange) atomicOr(&sh.strange[e][u - us][r >> 5], 1u << (r & 31));
                            }
                    }
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sh.kv_full[st]);
                }
                pos += 2 * (g.end - g.u0);
                __syncwarp();
                if (ok && lane == 0) {
                    ptx::mbar_arrive(&sh.strange_full[e]);
                    ptx::mbar_arrive(&sh.desc_empty[e]);
                }
            }
            if (!ok && lane == 0) chunk_timeout(a.status, 4);
        }
    } else {
        more_registers<kSoftmaxRegs>();
        // ------------------------------------------------------------------ softmax: a row per thread
        const int h = warp >> 2, row = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_at = tmem + lanes + h * 128, o_at = tmem + lanes + 256 + h * D;
        uint32_t s_uses = 0, o_uses = 0;
        bool ok = true;
        for (int count = 0; ok; ++count) {
            const int e = count % kDescs;
            if (!(ok = warp_wait(&sh.desc_full[e], (count / kDescs) & 1, abort_flag))) break;
            const ChunkSeg& g = sh.seg[e];
            if (g.b < 0) break;
            const int split = g.split, u0 = g.u0 + (split ? h : 0), stop = g.stop[h], rows = g.rows[split ? 0 : h], step = split ? 2 : 1;
            const int half_row = (split ? 0 : h * p.half_rows) + row;  // in the tile
            const int f = g.f0 + half_row - row + min(row, max(rows - 1, 0)), tok = (int)div_by((uint32_t)f, a.deal.by_g), pos = g.past + tok;
            float ref = -kInf;             // reference of the weights, in the exponent of 2
            uint64_t sum2 = 0, sum3 = 0;   // sums of the weights, in four parts
            for (int u = u0; u < stop; u += step) {
                if (!(ok = warp_wait(&sh.s_full[h], s_uses & 1, abort_flag))) break;
                ++s_uses;
                ptx::tc_fence_after();
                uint32_t s[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) ptx::tmem_ld_32x32(s_at + i * 32, s[i]);
                ptx::tmem_ld_wait();
                const int seen = pos - u * kKeys;  // columns up to here
                if (__any_sync(~0u, seen < kKeys - 1)) {
#pragma unroll
                    for (int i = 0; i < 128; ++i)
                        if (i > seen) s[i / 32][i % 32] = __float_as_uint(-kInf);
                }
                float top[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    top[i] = max3(__uint_as_float(s[i][0]), __uint_as_float(s[i][1]), __uint_as_float(s[i][2]));
#pragma unroll
                    for (int j = 3; j + 1 < 32; j += 2) top[i] = max3(top[i], __uint_as_float(s[i][j]), __uint_as_float(s[i][j + 1]));
                    top[i] = max_nan(top[i], __uint_as_float(s[i][31]));
                }
                // what the reference would be; a score of NaN or +inf makes the row NaN by way of it
                float m = fmaf(max3(max_nan(top[0], top[1]), top[2], top[3]), a.c, kChunkGrowth);
                if (m == kInf) m = __int_as_float(0x7FFFFFFF);
                if (u == u0) ref = m;
                bool again = false;
                auto weights = [&](int part, uint32_t (&w)[32], uint64_t& a2, uint64_t& b2) {  // of keys 64 part .. + 63, and their sums
                    const float r = ref == -kInf ? 0.0f : -ref;
                    const uint64_t c2 = pair(a.c, a.c), r2 = pair(r, r);
                    a2 = b2 = 0;
#pragma unroll
                    for (int i = 0; i < 64; i += 2) {
                        const uint32_t* const v = &s[part * 2 + i / 32][i % 32];
                        float x, y;
                        unpair(fma2(pair(__uint_as_float(v[0]), __uint_as_float(v[1])), c2, r2), x, y);
                        x = ex2(x), y = ex2(y);
                        if (i & 2) b2 = add2(b2, pair(x, y));
                        else a2 = add2(a2, pair(x, y));
                        w[i / 2] = pack_bf16(x, y);
                    }
                };
                auto deliver = [&](int part, const uint32_t (&w)[32]) {
                    ptx::tmem_st_32x32(s_at + part * 32, w);
                    ptx::tmem_st_wait();
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sh.p_full[h][part]);
                };
                uint32_t w[32];
                uint64_t a2, b2;
                // The weights by the reference as it is; the maximum is wanted only to see that it will do, and comes meanwhile.
                for (;;) {
                    weights(0, w, a2, b2);
                    const bool grown = row < rows && !(m <= ref + kChunkGrowth) && !again;  // (rows behind the last hold anything)
                    if (!__any_sync(~0u, grown)) break;
                    // the products before this tile's scores are done: O is this warp's
                    const float f2 = grown ? ex2(ref - m) : 1.0f;
                    if (grown) ref = m;
                    again = true;  // once: a reference of NaN would never do
                    sum2 = mul2(sum2, pair(f2, f2)), sum3 = mul2(sum3, pair(f2, f2));
                    if (u == u0) continue;
#pragma unroll 1
                    for (int i = 0; i < D / 16; ++i) {
                        uint32_t o[16];
                        ptx::tmem_ld_32x16(o_at + i * 16, o);
                        ptx::tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f2);
                        ptx::tmem_st_32x16(o_at + i * 16, o);
                    }
                }
                sum2 = add2(sum2, a2), sum3 = add2(sum3, b2);
                deliver(0, w);
                weights(1, w, a2, b2);
                sum2 = add2(sum2, a2), sum3 = add2(sum3, b2);
                deliver(1, w);
            }
            if (!ok) break;
            const bool some = stop > u0;
            if (some) {
                if (!(ok = warp_wait(&sh.o_full[h], o_uses & 1, abort_flag))) break;
                ++o_uses;
                ptx::tc_fence_after();
            }
            if (!(ok = warp_wait(&sh.strange_full[e], (count / kDescs) & 1, abort_flag))) break;
            float sum;
            {
                float x, y, z, w;
                unpair(sum2, x, y), unpair(sum3, z, w);
                sum = (x + y) + (z + w);
            }
            // A split segment: the second half's sums go through the room of the second half's queries, half of the columns at a time
            // ([column][row], a row per thread), and the first half joins them to its own.
            const bool merge = split && g.u0 + 1 < stop, any_row = (warp & 3) * 32 < rows;  // of the warp
            float* const room = reinterpret_cast<float*>(q_smem + QH) + row;
            if (merge && h == 1) {
                sh.other[row] = make_float2(ref, sum);
#pragma unroll 1
                for (int r = 0; r < 2; ++r) {
#pragma unroll 1
                    for (int i = 0; any_row && i < D / 64; ++i) {
                        uint32_t o[32];
                        ptx::tmem_ld_32x32(o_at + r * (D / 2) + i * 32, o);
                        ptx::tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 32; ++j) room[(i * 32 + j) * kHalf] = __uint_as_float(o[j]);
                    }
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sh.merge_full);
                    if (!(ok = warp_wait(&sh.merge_free, r, abort_flag))) break;
                }
                if (!ok) break;
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (warp == 4 && lane == 0) ptx::mbar_arrive(&sh.q_empty[1]);
            }
            float f_own = 1.0f, f_other = 0.0f;
            const bool writes = !split || h == 0;
            if (merge && h == 0) {
                if (!(ok = warp_wait(&sh.merge_full, 0, abort_flag))) break;
                const float2 q = sh.other[row];
                // (a reference of -inf with a sum that is not 0 is one of NaN scores)
                const float top = max_nan(ref, q.x);
                f_own = ref == top || ref == -kInf ? 1.0f : ex2(ref - top), f_other = q.x == top || q.x == -kInf ? 1.0f : ex2(q.x - top);
                sum = sum * f_own + q.y * f_other;
                ref = top;
            }
            const int slot = g.slot, head = g.h * a.deal.g + (f - tok * a.deal.g);
            const int64_t out_row = g.q0 + tok, at = (int64_t)max(slot, 0) * a.deal.rows + half_row;
            const float inv = slot < 0 ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f;
            f_own *= inv, f_other *= inv;
            const int us = max(g.u0, (max(g.first_pos, -1) + 1) / kKeys);
            uint32_t any = 0;
#pragma unroll
            for (int i = 0; i < kStrange * 4; ++i) any |= sh.strange[e][i / 4][i % 4];
#pragma unroll 1
            for (int i = 0; writes && i < D / 32; ++i) {
                uint32_t o[32];
                if (merge && i == D / 64) {  // on to the second half of the columns
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&sh.merge_free);
                    if (!(ok = warp_wait(&sh.merge_full, 1, abort_flag))) break;
                }
                if (!any_row) continue;
                if (some) {
                    ptx::tmem_ld_32x32(o_at + i * 32, o);
                    ptx::tmem_ld_wait();
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) o[j] = 0;
                }
                if (row < rows && (some || slot < 0)) {
                    const int col = i * 32;
                    float v[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(o[j]) * f_own;
                    if (merge) {
                        const float* const x = room + (i % (D / 64)) * 32 * kHalf;
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = fmaf(x[j * kHalf], f_other, v[j]);
                    }
                    if (any && some) {  // rare: infinities and NaN of the keys that this row sees
                        for (int w = 0; w < kStrange * 4; ++w)
                            for (uint32_t bits = sh.strange[e][w / 4][w % 4]; bits; bits &= bits - 1) {
                                const int key = (us + w / 4) * kKeys + (w % 4) * 32 + __ffs(bits) - 1;
                                int within = 0;
                                const int page = key <= pos ? page_of(a.seq, g.b, key, within) : -1;
                                if (page < 0) continue;
                                const __nv_bfloat16* src = a.v + (int64_t)page * a.v_page + (int64_t)within * a.v_row + (int64_t)g.h * a.v_head + col;
#pragma unroll
                                for (int j = 0; j < 32; ++j) {
                                    const float x = __bfloat162float(src[j]);
                                    if (!(fabsf(x) < kInf)) v[j] += x;
                                }
                            }
                    }
                    if (slot >= 0) {  // [column][row]: the lanes' rows lie side by side
                        float* const dst = a.part_o + ((int64_t)slot * D + i * 32) * a.deal.rows + half_row;
#pragma unroll
                        for (int j = 0; j < 32; ++j) dst[j * a.deal.rows] = v[j];
                    } else {
                        __nv_bfloat16* const dst = a.out + out_row * a.ldo + head * D + i * 32;
                        uint32_t x[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) x[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
                        if (p.wide) {  // whole sectors
                            ptx::st_global_v8(dst, x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]);
                            ptx::st_global_v8(dst + 16, x[8], x[9], x[10], x[11], x[12], x[13], x[14], x[15]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; j += 4) reinterpret_cast<uint4*>(dst)[j / 4] = make_uint4(x[j], x[j + 1], x[j + 2], x[j + 3]);
                        }
                    }
                }
                __syncwarp();
            }
            if (!ok) break;
            if (merge && h == 0) {
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sh.merge_free);
            }
            if (writes && row < rows) {
                if (slot >= 0) a.part_ml[at] = make_float2(ref, sum);
                else if (a.lse) a.lse[out_row * a.Hq + head] = chunk_lse(ref, sum);
            }
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sh.desc_empty[e]);
        }
        if (!ok && lane == 0) chunk_timeout(a.status, 5);
    }
    // Products in flight read shared memory, write tensor memory and report to barriers.  (In the products' own branch this costs its
    // loop 3 % of a prefill.)
    if ((warp == kMmaWarp || warp == kMmaWarp + 1) && lane == 0) {
        ptx::umma_commit(&sh.done[warp - kMmaWarp]);
        drain(&sh.done[warp - kMmaWarp], 0);
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) ptx::tmem_dealloc(tmem, 512);
    pdl_trigger();
}

}  // namespace

bool attn_chunk_supported(const AttnArgs& a) {
    auto ok = [](int64_t stride, int64_t extent) { return extent == 1 || stride > 0; };
    return ok(a.k_row, a.seq.page) && ok(a.v_row, a.seq.page) && ok(a.k_head, a.deal.Hkv) && ok(a.v_head, a.deal.Hkv) && ok(a.k_page, a.seq.pages) &&
           ok(a.v_page, a.seq.pages) && (a.seq.T == 1 || a.ldq > 0);
}

int attn_chunk_rows(int g) { return 2 * (kHalf / g) * g; }

int launch_attn_chunk(const AttnArgs& args, int D, int ctas, cudaStream_t stream) {
    ChunkArgs p;
    p.a = args;
    const int g = args.deal.g;
    p.half_tokens = kHalf / g;
    p.half_rows = p.half_tokens * g;
    p.wide = reinterpret_cast<uintptr_t>(args.out) % 32 == 0 && args.ldo % 16 == 0;
    p.expire = take_expire_request(2);
    p.box = 8;
    while (p.box < kKeys && args.seq.page % (2 * p.box) == 0) p.box *= 2;
    ChunkMaps maps;
    const uint64_t d = (uint64_t)D;
    auto stride = [](int64_t s, int64_t extent) { return extent == 1 ? (uint64_t)16 : (uint64_t)s * 2; };  // of a single one: any
    {
        const uint64_t dims[3] = {d, (uint64_t)args.Hq, (uint64_t)args.seq.T}, strides[2] = {d * 2, args.seq.T == 1 ? d * 2 * args.Hq : (uint64_t)args.ldq * 2};
        const uint32_t box[3] = {64, (uint32_t)g, (uint32_t)p.half_tokens};
        int rc = make_tmap_bf16(&maps.q, args.q, 3, dims, strides, box);
        if (rc) return rc;
    }
    const uint64_t dims[4] = {d, (uint64_t)args.seq.page, (uint64_t)args.deal.Hkv, (uint64_t)args.seq.pages};
    const uint32_t box[4] = {64, (uint32_t)p.box, 1, 1};
    const uint64_t ks[3] = {stride(args.k_row, args.seq.page), stride(args.k_head, args.deal.Hkv), stride(args.k_page, args.seq.pages)};
    const uint64_t vs[3] = {stride(args.v_row, args.seq.page), stride(args.v_head, args.deal.Hkv), stride(args.v_page, args.seq.pages)};
    int rc = make_tmap_bf16(&maps.k, args.k, 4, dims, ks, box);
    if (rc) return rc;
    rc = make_tmap_bf16(&maps.v, args.v, 4, dims, vs, box);
    if (rc) return rc;
    auto kern = D == 128 ? attn_chunk_kernel<128> : attn_chunk_kernel<64>;
    const int smem = 2 * kHalf * D * 2 + (D == 128 ? stages<128>() * tile_bytes<128>() : stages<64>() * tile_bytes<64>()) + (int)sizeof(ChunkShared);
    rc = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem, "attn_chunk_kernel shared memory");
    if (rc) return rc;
    LaunchScope scope(kKindRow, stream);
    return cuda_fail(launch_kernel(kern, dim3((unsigned)ctas), dim3(kThreads), (size_t)smem, stream, p, maps), "attn_chunk_kernel launch");
}

}  // namespace resq
