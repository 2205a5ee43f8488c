// What the operators on a paged cache share (rope_append.cu, paged_attention.cu, paged_chunk.cu): argument checks, where a
// token's key lies, and how attention over ragged sequences is dealt out to CTAs.  Internal.
#pragma once
#include "row_common.cuh"

namespace resq {

constexpr int64_t kMaxSeqs = RESQ_MAX_SEQUENCES;
constexpr float kLn2 = 0.6931471805599453f;

// n / d for 0 <= n < 2^31 by one multiplication (Granlund and Montgomery: m = ceil(2^(32 + s) / d), s = ceil(log2 d) - 1 bits of
// shift are enough for 31-bit n; d = 1 is apart).
struct FastDiv {
    uint32_t d, m, s;
};
inline FastDiv fast_div(uint32_t d) {
    FastDiv f{d, 0, 0};
    if (d == 1) return f;
    while ((1ull << (f.s + 1)) < d) ++f.s;
    f.m = (uint32_t)(((1ull << (32 + f.s)) + d - 1) / d);
    return f;
}
__host__ __device__ inline uint32_t div_by(uint32_t n, const FastDiv& f) {
#ifdef __CUDA_ARCH__
    return f.d == 1 ? n : __umulhi(n, f.m) >> f.s;
#else
    return f.d == 1 ? n : (uint32_t)(((uint64_t)n * f.m) >> 32) >> f.s;
#endif
}

// Checks of the cache and the sequences that rope_append and paged_attention share; T: token rows of the call.
int check_paged(const char* what, const resq_paged_cache* cache, const resq_sequences* seqs, int64_t T, int64_t Hq, int64_t Hkv, int64_t D);

// The sequences as kernels read them.  Whatever the device arrays hold, no access leaves the tensors: starts are cut to 0 .. T and
// kept in order, lengths to 0 .. max_keys, and a page outside the cache is no page.
struct SeqArgs {
    const int32_t* q_start;
    const int32_t* kv_len;
    const int32_t* table;
    int64_t ld_table;
    int B, T, max_keys, page, pages;
    FastDiv by_page;
};
inline SeqArgs seq_args(const resq_paged_cache& c, const resq_sequences& s, int64_t T) {
    return SeqArgs{s.q_start, s.kv_len, s.page_table, s.ld_table, (int)s.count, (int)T, (int)(s.max_pages * c.page_size), (int)c.page_size,
                   (int)c.pages, fast_div((uint32_t)c.page_size)};
}

// How attention is dealt out (below): rows and keys (a power of two) per tile, heads.
struct Deal {
    int rows, keys, Hkv, g;
    int extra;  // what an item costs besides its keys, in units
    int key_bits;
    FastDiv by_g, by_rows;
};
inline Deal make_deal(int rows, int keys, int Hkv, int g, int extra) {
    Deal d{rows, keys, Hkv, g, extra, 0, fast_div((uint32_t)g), fast_div((uint32_t)rows)};
    while ((1 << d.key_bits) < keys) ++d.key_bits;
    return d;
}
// Where partial results lie: a CTA's first segment, when its item began in an earlier CTA, in slot 2 * cta; one whose item goes on
// in the next CTA otherwise in slot 2 * cta + 1.  The CTA that begins inside an item says so in its entry of `notes`: the CTAs
// before it that the item covers, and all of them.
struct JoinNote {
    int parts;   // CTAs of the item (0: this CTA does not begin inside an item, or is not the item's second one)
    int q0, n;   // the item's sequence: first token row, new tokens
    int h, f0;   // kv head, first row
    int pad[3];
};
struct AttnArgs {
    SeqArgs seq;
    Deal deal;
    const __nv_bfloat16 *q, *k, *v;
    int64_t ldq, ldo, k_page, k_row, k_head, v_page, v_row, v_head;
    __nv_bfloat16* out;
    float* lse;       // [T, Hq] or null
    int Hq;
    float c;          // scale log2(e)
    int min_chunk;
    float* part_o;    // [2 ctas][rows][D] (attn_chunk_kernel: [2 ctas][D][rows]), unnormalised
    float2* part_ml;  // [2 ctas][rows]: reference, sum
    JoinNote* notes;  // [ctas]
    DeviceStatus* status;
};

// paged_chunk.cu: the tensor-core form for chunks of new tokens.  Rows of its tiles for g query heads per kv head, whether it takes
// these strides, and its launch (args.deal.rows and .keys as it wants them).
constexpr int kChunkKeys = 128, kChunkExtra = 6;
constexpr float kChunkGrowth = 20.0f;  // its references lie this far above the maximum that they were set by, in the exponent of 2
int attn_chunk_rows(int g);
bool attn_chunk_supported(const AttnArgs& args);
int launch_attn_chunk(const AttnArgs& args, int D, int ctas, cudaStream_t stream);

#ifdef __CUDACC__

// Log of a row's sum relative to such a reference.  The 20 are taken out of both first (exactly): the sum of the two would round to
// the digits of a number of 20.
__device__ __forceinline__ float chunk_lse(float ref, float sum) {
    return sum == 0.0f ? -__builtin_huge_valf() : ((ref - kChunkGrowth) + log2f(sum * 1048576.0f)) * kLn2;
}
static_assert(kChunkGrowth == 20.0f, "2^20 above");

struct Seq {
    int q0, n, kv;  // first token row, new tokens, keys (the new tokens' among them)
};
__device__ __forceinline__ Seq load_seq(const SeqArgs& a, int b) {
    Seq s;
    s.q0 = min(max(a.q_start[b], 0), a.T);
    s.n = max(min(max(a.q_start[b + 1], 0), a.T) - s.q0, 0);
    s.kv = min(max(a.kv_len[b], 0), a.max_keys);
    return s;
}
// Page of key j of sequence b (0 <= j < max_keys); -1: none.
__device__ __forceinline__ int page_of(const SeqArgs& a, int b, int j, int& within) {
    const int i = (int)div_by((uint32_t)j, a.by_page);
    within = j - i * a.page;
    const int id = a.table[b * a.ld_table + i];
    return (unsigned)id < (unsigned)a.pages ? id : -1;
}

// ---- how attention is dealt out ------------------------------------------------------------------------------------------------
// The queries of a sequence that share a kv head are rows f = token * g + head, cut into tiles of `rows`; an item is one tile, and
// its units are `extra` ones for its beginning and end, then tiles of `keys` keys up to the last one that its last token sees (one
// at least: an item without keys still writes its rows).  Items are ordered by sequence, kv head, tile; all units in this order are cut into equal ranges, one per CTA,
// so that ragged lengths need no plan from the host and a captured call follows the lengths on the device.  A CTA's first item may
// have begun in an earlier CTA and its last one may go on in a later one: those are left as partial results.
__device__ __forceinline__ int deal_tiles(const Seq& s, const Deal& d) { return (int)div_by((uint32_t)max(s.n * d.g - 1, 0), d.by_rows) + (s.n > 0); }
__device__ __forceinline__ int deal_k_end(const Seq& s, const Deal& d, int t) {  // keys that tile t sees
    const uint32_t f = min((uint32_t)(t + 1) * (uint32_t)d.rows, (uint32_t)(s.n * d.g)) - 1u;  // n g < 2^31, and the last tile ends below 2^32
    const int last = (int)div_by(f, d.by_g);
    return max(0, min(s.kv - s.n + last + 1, s.kv));
}
__device__ __forceinline__ int deal_units(const Seq& s, const Deal& d, int t) { return max(1, (deal_k_end(s, d, t) + d.keys - 1) >> d.key_bits) + d.extra; }

// Where a CTA's range begins, and how long it is.
struct DealStart {
    int64_t unit, units;  // first unit of the range, units in it (0: none)
    int64_t chunk;        // units per CTA
    int64_t before;       // first unit of sequence b
    int64_t per_head;     // units of one kv head of sequence b
    int b;
};
// Units of one kv head of sequence s; all lanes of the warp, each with a sequence of its own: short ones a lane by itself, long
// ones (many tiles) together.
__device__ __forceinline__ int64_t deal_head_units(const Seq& s, const Deal& d) {
    const int tiles = deal_tiles(s, d), lane = threadIdx.x & 31;
    int64_t sum = 0;
    const bool longer = tiles > 4;
    if (!longer)
        for (int t = 0; t < tiles; ++t) sum += deal_units(s, d, t);
    unsigned todo = __ballot_sync(~0u, longer);
    while (todo) {
        const int src = __ffs(todo) - 1;
        todo &= todo - 1;
        Seq q;
        q.q0 = 0;
        q.n = __shfl_sync(~0u, s.n, src), q.kv = __shfl_sync(~0u, s.kv, src);
        const int nt = deal_tiles(q, d);
        unsigned long long part = 0;
        for (int t = lane; t < nt; t += 32) part += (unsigned)deal_units(q, d, t);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(~0u, part, o);
        if (lane == src) sum = (int64_t)part;
    }
    return sum;
}
// The whole block; `sums` (one int64 per warp) and `found` in shared memory.  Thread i owns the sequences i * per .. + per - 1.
__device__ __forceinline__ DealStart deal_start(const SeqArgs& a, const Deal& d, int cta, int ctas, int min_chunk, int64_t* sums, DealStart* found) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, nw = blockDim.x >> 5;
    const int per = (a.B + (int)blockDim.x - 1) / (int)blockDim.x;
    // visit(i, units of a head): this thread's sequences in order, four loads in flight
    auto each = [&](auto&& visit) {
        for (int i0 = 0; i0 < per; i0 += 4) {
            Seq s[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[i] = Seq{0, 0, 0};
                if (i0 + i < per && tid * per + i0 + i < a.B) s[i] = load_seq(a, tid * per + i0 + i);
            }
#pragma unroll 1
            for (int i = 0; i < 4 && i0 + i < per; ++i) visit(tid * per + i0 + i, deal_head_units(i == 0 ? s[0] : i == 1 ? s[1] : i == 2 ? s[2] : s[3], d));
        }
    };
    int64_t mine = 0;
    each([&](int, int64_t per_head) { mine += per_head * d.Hkv; });
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(~0u, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31) sums[w] = upto;
    if (tid == 0) found->units = 0;
    __syncthreads();
    int64_t base = 0, total = 0;
    for (int i = 0; i < nw; ++i) {
        if (i == w) base = total;
        total += sums[i];
    }
    upto += base;
    const int64_t chunk = max((total + ctas - 1) / ctas, (int64_t)min_chunk), unit = (int64_t)cta * chunk;
    // the owner of the sequence that unit lies in looks for it; its warp helps (deal_head_units is the warp's)
    const bool owner = unit >= upto - mine && unit < upto;
    if (__any_sync(~0u, owner)) {
        int64_t at = upto - mine;
        bool open = owner;
        each([&](int b, int64_t per_head) {
            if (open && unit < at + per_head * d.Hkv) {
                *found = DealStart{unit, min(chunk, total - unit), chunk, at, per_head, b};
                open = false;
            }
            at += per_head * d.Hkv;
        });
    }
    __syncthreads();
    return *found;
}

// One item's share of a CTA's range.
struct Segment {
    int b, h, t;        // sequence, kv head, tile
    int u0, u1, units;  // units u0 .. u1 - 1 of the item's `units`
    int k0, k1;         // their tiles of keys, k0 .. k1 - 1
    Seq s;
};
// Walks a CTA's range item by item; one warp at a time, all lanes alike.
struct DealWalk {
    DealStart at;
    int64_t left;  // units still to hand out
    int b, h, t, u;
    Seq s, ahead;  // of sequence b, and of the next one, asked for early
    int tiles;
    __device__ __forceinline__ void init(const SeqArgs& a, const Deal& d, const DealStart& start) {
        at = start, left = start.units;
        if (left <= 0) return;
        b = start.b;
        s = load_seq(a, b);
        ahead = load_seq(a, min(b + 1, a.B - 1));
        tiles = deal_tiles(s, d);
        int64_t off = start.unit - start.before;
        h = (int)(off / start.per_head);
        off -= h * start.per_head;
        // the tile in which unit `off` of the head lies: 32 tiles at a time
        t = 0;
        const int lane = threadIdx.x & 31;
        for (;;) {
            const int n = t + lane < tiles ? deal_units(s, d, t + lane) : 0;
            int64_t upto = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t v = __shfl_up_sync(~0u, upto, o);
                if (lane >= o) upto += v;
            }
            const unsigned past = __ballot_sync(~0u, upto > off);
            if (past) {
                const int src = __ffs(past) - 1;
                u = (int)(off - __shfl_sync(~0u, upto - n, src));
                t += src;
                return;
            }
            off -= __shfl_sync(~0u, upto, 31);
            t += 32;
        }
    }
    __device__ __forceinline__ bool next(const SeqArgs& a, const Deal& d, Segment& out) {
        if (left <= 0) return false;
        while (t >= tiles) {  // on to the next head, or the next sequence with new tokens
            t = 0;
            if (tiles == 0 || ++h == d.Hkv) {
                h = 0;
                if (++b >= a.B) return false;
                s = ahead;
                ahead = load_seq(a, min(b + 1, a.B - 1));
                tiles = deal_tiles(s, d);
            }
        }
        out.b = b, out.h = h, out.t = t, out.s = s;
        out.units = deal_units(s, d, t);
        out.u0 = u;
        out.u1 = (int)min((int64_t)out.units, u + left);
        left -= out.u1 - u;
        out.k0 = max(out.u0 - d.extra, 0), out.k1 = max(out.u1 - d.extra, 0);
        u = 0;
        ++t;
        return true;
    }
};

// The note of a CTA whose first segment is `seg`: the item that it begins inside of, if it is that item's second CTA.
__device__ __forceinline__ JoinNote join_note(const Segment& seg, const DealStart& start, int cta, int f0) {
    JoinNote note{0, seg.s.q0, seg.s.n, seg.h, f0, {0, 0, 0}};
    if (seg.u0 > 0) {
        const int64_t item = start.unit - seg.u0;
        const int i0 = (int)(item / start.chunk), i1 = (int)((item + seg.units - 1) / start.chunk);
        if (i0 == cta - 1) note.parts = i1 - i0 + 1;
    }
    return note;
}

#endif  // __CUDACC__

}  // namespace resq
