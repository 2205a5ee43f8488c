// *_w4a16_gemv: Y[m, n] = sum_k X[m, k] deq(W)[n, k] for at most RESQ_GEMV_MAX_TOKENS token rows.
//
// What it has to do is stream the packed weights (4.5 or 4.25 bits each) once; the arithmetic next to that is the expansion
// of the codes.  At 6.5 TB/s an SM receives about 41 weights per clock, so an expansion may cost three instructions a weight
// and the multiplications must cost next to none: they go to the register-operand tensor instruction (m16n8k16, bf16 in, fp32
// out), whose A fragment is 16 weight rows in exactly the layout a lane can expand in registers, and whose 8 columns are
// tokens.  (The tensor-memory instruction would need the expanded weights written to shared memory and read back, which is
// what bounds the decode GEMM.)  The order of k inside a fragment is free as long as both operands use the same one, so
// a lane owns 32 consecutive k of rows g and g + 8 (one 16-byte load each), and pairs elements i and i + 4 of a 32-bit word:
// their nibbles lie 16 bits apart, so one mask takes both.
//
// Work: a unit is 16 weight rows x 128 k (1 KB of codes).  A CTA (12 warps, one CTA per SM, so that the activations are staged
// once) owns T row tiles and one of CS slices of K; its T x units are dealt out evenly and contiguously to its warps.  The codes
// come by asynchronous copies into a ring of two steps of up to four units per warp, each lane fetching what it will expand
// itself; loads into registers measured up to 1.4 times slower (11 tokens, 3584 -> 100003: 102 against 73 us), because their
// lines in flight have to fit into what the staged activations leave of the L1.  Tiles that a warp has to itself are written from
// its registers; the parts of a tile that several warps (or slices) share go to shared memory and are added in a fixed order.
// Twelve warps with four units at a time are faster than sixteen with two (the same case: 65 against 73 us) or eight (68).
//
// Measured, weights from HBM: 3584 -> 37888, HiF4, 23 us for one token and 25 for eight (3.3 TB/s, 0.50 of the copy rate); MXFP4
// 24 us; 11 tokens 3584 -> 100003 65 us (3.1 TB/s); 2048 -> 2048 4.0 us, of which the launch and the chain load, expand, sum
// are all.  It is bound by the arithmetic of the expansion: without it (the codes taken as they are) 3584 -> 37888 takes 17 us,
// without the copies 19.5.
#include "common.cuh"
#include "row_common.cuh"

#include <algorithm>
#include <type_traits>

namespace resq {
namespace {

constexpr int kWarps = 12, kThreads = kWarps * 32;
constexpr int kUnitK = 128, kTileN = 16;
// STEP: units of a tile per step (512 or 256 k), which has one wait and one set of copies: four, or two where the staged
// activations leave no room for more or a warp's run is too short for them (plan_gemv; one token 2048 -> 2048: 4.0 against 4.1 us,
// 3584 -> 37888: 26.5 us with two for eight tokens, 25.0 with four).
constexpr int kRing = 2;        // steps in flight per warp: 96 or 48 KB per SM (three of two units: no faster, and it costs the tiles room)
// words per row of a step's scales: HiF4 two per unit and one against bank conflicts, MXFP4 one per unit and one because rows
// start on any byte
__host__ __device__ constexpr int side_row(int fmt, int step) { return fmt == kHiF4 ? 2 * step + 1 : step + 1; }
constexpr int kMaxTiles = 64;   // row tiles per CTA (int arithmetic on units x warps)
constexpr int kXPad = 64;       // bytes behind a token's staged row: neighbouring tokens use the other half of the banks

struct GemvArgs {
    const __nv_bfloat16* X;
    const uint8_t* codes;
    const uint8_t* side;
    void* Y;
    int64_t ldx, ldy;
    int M, K, N, out_dtype;
    int tiles;        // row tiles in all
    int tiles_cta;    // row tiles per CTA (and cluster)
    int units_slice;  // units of 128 k per slice
};

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t mad(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("mad.lo.u32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
// ZERO: the sum starts here
template <bool ZERO>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (ZERO)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
template <int BYTES>
__device__ __forceinline__ void copy_scales(uint32_t dst, const void* src) {
    static_assert(BYTES == 8 || BYTES == 16);
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
// the first `n` bytes of a word (0 to 4), zeros behind them
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, int n) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// What a lane needs to expand its 32 codes of one row: HiF4 half a block (four level-2 groups), MXFP4 one whole block.
//
// Both element formats are small floating-point numbers, and their magnitude bits are bf16 numbers as they stand once they
// sit at the right place: S1P2 (= E1M2) at bits 7:5 is the bf16 number q/4 * 2^-126 (q < 4 as a subnormal), E2M1 at bits
// 8:6 is value * 2^-126.  So an element is moved into place together with its sign, and one packed multiplication by
// 2^126 times its scale gives the exact weight (at most 6 significant bits).
template <int FMT>
struct Scale;
template <>
struct Scale<kHiF4> {
    // 2^126 S1 2^2 may pass the range of bf16, so the weights are formed as w * 2^-16 and the sums take 2^16 at the end; only
    // products below 2^-110 lose bits by that.
    static constexpr float kBack = 65536.0f;
    uint32_t base, e;  // e: exponents, two bits for every group of four: of words 0 to 3 in bits 0 to 7, of their upper halves in 16 to 23
    // odd: the lane's half of the 64-block
    __device__ __forceinline__ void set(uint32_t meta, int odd) {
        base = (meta & 255u) * 0x00200020u + 0x5E805E80u;  // bf16 bits of 2^110 S1 in both halves (s << 5 is (E << 7) | (Mn << 5))
        // a level-2 bit counts for both halves of its word, two level-3 bits belong to a word (the lower to its lower half)
        const uint32_t e3 = __byte_perm(meta, 0u, odd ? 0x4443 : 0x4442), e2 = meta >> (8 + 4 * odd);
        const uint32_t spread = (e2 & 0x03u) | ((e2 << 2) & 0x30u);
        e = mad((spread | (spread << 1)) & 0x55u, 0x00010001u, (e3 * 0x8001u) & 0x00550055u);
    }
    // v[i]: elements i (low half) and i + 4.  Element 2j is the low, 2j + 1 the high nibble of byte j; the sign goes to bit 7
    // of the upper byte, the magnitude to bits 7:5 of the lower byte of a half.
    template <bool TWO>
    __device__ __forceinline__ void expand(uint32_t w, int group, uint32_t (&v)[4]) const {
        // both exponents to bit 7 of their half, as a multiply-add: it runs beside the integer pipe, which the element work fills
        const uint32_t c = mad(e & (0x00030003u << (2 * group)), 128u >> (2 * group), base);
        const uint32_t w1 = w << 1, w4 = w << 4, w5 = w << 5;
        v[0] = mul_bf16x2(__byte_perm(w4, w5, 0x2604) & 0x80E080E0u, c);
        v[1] = mul_bf16x2(__byte_perm(w, w1, 0x2604) & 0x80E080E0u, c);
        v[2] = mul_bf16x2(__byte_perm(w4, w5, 0x3715) & 0x80E080E0u, c);
        v[3] = mul_bf16x2(__byte_perm(w, w1, 0x3715) & 0x80E080E0u, c);
    }
};
template <>
struct Scale<kMXFP4> {
    static constexpr float kBack = 1.0f;
    uint32_t c, sc;
    __device__ __forceinline__ void set(uint32_t code, bool none) {
        sc = none ? 0u : code;
        c = none ? 0u : min(code + 126u, 254u) * 0x00800080u;  // 2^126 2^(code - 127), at most 2^127
    }
    // TWO: a scale code above 128 has a second factor 2^(code - 128)
    template <bool TWO>
    __device__ __forceinline__ void expand(uint32_t w, int, uint32_t (&v)[4]) const {
        // a code times 2^6 + 2^12 has its magnitude at bits 8:6 and its sign at bit 15: one multiply-add instead of two shifts
        const uint32_t u = w >> 8;
        v[0] = mul_bf16x2(((w & 0x000F000Fu) * 0x1040u) & 0x81C081C0u, c);
        v[1] = mul_bf16x2(((w & 0x00F000F0u) * 0x0104u) & 0x81C081C0u, c);
        v[2] = mul_bf16x2(((u & 0x000F000Fu) * 0x1040u) & 0x81C081C0u, c);
        v[3] = mul_bf16x2(((u & 0x00F000F0u) * 0x0104u) & 0x81C081C0u, c);
        if (TWO) {
            const uint32_t c2 = sc > 128u ? (sc == 255u ? 0x7F807F80u : (sc - 1u) * 0x00800080u) : 0x3F803F80u;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = mul_bf16x2(v[i], c2);
        }
    }
};

// One unit of 16 rows x 128 k: a chain of 8 instructions from zero for each token group, then one rounded addition to each sum
// (the tensor cores cut their sums instead of rounding them).
template <int FMT, int NT, bool TWO>
__device__ __forceinline__ void unit(const uint4& qa, const uint4& qb, const Scale<FMT>& fa, const Scale<FMT>& fb,
                                     const uint8_t* const (&xs)[NT], int at, float (&acc)[NT][4]) {
    float c[NT][4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t va[4], vb[4];
        fa.template expand<TWO>(w == 0 ? qa.x : w == 1 ? qa.y : w == 2 ? qa.z : qa.w, w, va);
        fb.template expand<TWO>(w == 0 ? qb.x : w == 1 ? qb.y : w == 2 ? qb.z : qb.w, w, vb);
#pragma unroll
        for (int q = 0; q < NT; ++q) {
            const uint4 x = *reinterpret_cast<const uint4*>(xs[q] + at + w * 64);
            if (w == 0) mma16816<true>(c[q], va[0], vb[0], va[1], vb[1], x.x, x.y);
            else mma16816<false>(c[q], va[0], vb[0], va[1], vb[1], x.x, x.y);
            mma16816<false>(c[q], va[2], vb[2], va[3], vb[3], x.z, x.w);
        }
    }
#pragma unroll
    for (int q = 0; q < NT; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[q][j] += c[q][j];
}

__device__ __forceinline__ void store_out(const GemvArgs& a, int m, int n, float v) {
    if (a.out_dtype == RESQ_OUT_BF16) static_cast<__nv_bfloat16*>(a.Y)[m * a.ldy + n] = __float2bfloat16_rn(v);
    else static_cast<float*>(a.Y)[m * a.ldy + n] = v;
}

// Slots of 8 NT tokens x 16 rows of partial sums.  Without slices two per warp (the tile its run starts in and the one it ends
// in), with slices one per (tile, warp) of a run, at tile + warp (both only grow along the runs).  Token pairs lie 32 floats
// apart and a pair's rows are turned by four places from pair to pair, so that a warp's stores from the accumulator layout and
// its loads of neighbouring rows meet no bank twice.
__device__ __forceinline__ int part_at(int token, int row) {
    return (token >> 1) * 32 + ((row + 4 * (token >> 1)) & 15) * 2 + (token & 1);
}
__host__ __device__ constexpr size_t ring_bytes(int fmt, int step) {
    return (size_t)kWarps * kRing * (step * 1024 + kTileN * side_row(fmt, step) * 4);
}
__host__ __device__ inline size_t part_bytes(int cs, int tiles, int nt) {
    return (size_t)(cs == 1 ? 2 * kWarps : tiles + kWarps) * kTileN * 8 * nt * sizeof(float);
}

// NT: groups of 8 tokens; CS: CTAs of a cluster, each with its slice of K.
template <int FMT, int NT, int STEP, int CS>
__global__ void __launch_bounds__(kThreads, 1) gemv_kernel(const __grid_constant__ GemvArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int rank = CS > 1 ? (int)(blockIdx.x % CS) : 0;
    const int tile0 = (int)(blockIdx.x / CS) * a.tiles_cta;
    const int tiles = min(a.tiles_cta, a.tiles - tile0);
    const int units_all = (a.K + kUnitK - 1) / kUnitK;
    const int units = max(0, min(a.units_slice, units_all - rank * a.units_slice));
    const int k0 = rank * a.units_slice * kUnitK;
    const int xrow = a.units_slice * 256 + kXPad;
    constexpr int kSideRow = side_row(FMT, STEP), kSideBytes = kTileN * kSideRow * 4;
    uint8_t* const ring = smem + (size_t)a.M * xrow + warp * (kRing * STEP * 1024);
    uint8_t* const sides = smem + (size_t)a.M * xrow + kWarps * (kRing * STEP * 1024) + warp * (kRing * kSideBytes);
    float* const part = reinterpret_cast<float*>(smem + (size_t)a.M * xrow + ring_bytes(FMT, STEP));
    constexpr int kSlot = kTileN * 8 * NT;

    pdl_wait();

    // ---- the warp's run of (tile, unit) pairs: its first copies are under way while the activations are staged
    const int total = tiles * units;
    const int first = total * warp / kWarps, last = total * (warp + 1) / kWarps;  // below 64 x 384 x 12
    const int64_t row_codes = a.K / 2, row_side = FMT == kHiF4 ? (int64_t)a.K / 64 * 4 : (int64_t)a.K / 32;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + lane * 16, side_at = (uint32_t)__cvta_generic_to_shared(sides);
    // The last unit of K may hold one, two or three blocks of 32: a lane beyond the end reads the start of its row instead
    // and multiplies it with zeros (its activations are staged as zeros; an MXFP4 scale, which may be infinite, is zeroed).
    const bool beyond = k0 + (units - 1) * kUnitK + t * 32 >= a.K;
    auto step_units = [&](int u, int i) { return min(min(STEP - (u & (STEP - 1)), units - u), last - i); };
    int lu = units > 0 ? first % units : 0, lt = units > 0 ? first / units : 0, li = first, lslot = 0;  // copy cursor
    const uint8_t *pa = a.codes, *pb = a.codes, *tside = a.side;  // the lane's two rows at its first k; the tile's first row
    int rows_left = 0;
    const uint32_t lane_k = (uint32_t)(k0 / 2 + t * 16);
    auto point = [&]() {
        const int n0 = (tile0 + lt) * kTileN;
        rows_left = a.N - 1 - n0;
        const uint8_t* tcodes = a.codes + n0 * row_codes + lane_k;
        tside = a.side + n0 * row_side;
        pa = tcodes + (uint32_t)min(g, rows_left) * (uint32_t)row_codes, pb = tcodes + (uint32_t)min(g + 8, rows_left) * (uint32_t)row_codes;
    };
    const bool ragged = a.K % kUnitK != 0;
    const bool even = FMT == kMXFP4 && (row_side | (k0 / 32)) % (STEP * 4) == 0;  // a step's scales of a row are one aligned piece
    const uint32_t lane_side = lane / (2 * STEP) * (uint32_t)row_side + lane % (2 * STEP) * 4;  // HiF4: the lane's first word of scales
    const uint32_t lane_word = (lane / (2 * STEP) * kSideRow + lane % (2 * STEP)) * 4;
    auto copy = [&]() {
        if (li < last) {
            const int n = step_units(lu, li), j0 = lu & (STEP - 1);
            const uint32_t to = ring_at + lslot * (STEP * 1024);
            const uint8_t *ca = pa + (lu - j0) * 64, *cb = pb + (lu - j0) * 64;
            if (n == STEP && !(ragged && lu + n == units)) {
#pragma unroll
                for (int j = 0; j < STEP; ++j) copy16(to + j * 1024, ca + j * 64), copy16(to + j * 1024 + 512, cb + j * 64);
            } else {
#pragma unroll 1
                for (int j = j0; j < j0 + n; ++j) {
                    const bool out = beyond && lu - j0 + j == units - 1;
                    copy16(to + j * 1024, out ? pa - lane_k : ca + j * 64);
                    copy16(to + j * 1024 + 512, out ? pb - lane_k : cb + j * 64);
                }
            }
            const uint32_t dst = side_at + lslot * kSideBytes;
            if (FMT == kHiF4) {
                constexpr int kWords = 2 * STEP, kRows = 32 / kWords;  // of one copy of the warp
                const int b0 = k0 / 64 + (lu - j0) * 2, b = b0 + lane % kWords, nb = a.K / 64;
                if (rows_left >= kTileN - 1 && b0 + kWords <= nb) {
                    const uint8_t* from = tside + lane_side + b0 * 4;
#pragma unroll
                    for (int i = 0; i < kTileN / kRows; ++i) copy4(dst + lane_word + i * kRows * kSideRow * 4, from + i * kRows * (uint32_t)row_side);
                } else {
#pragma unroll
                    for (int i = 0; i < kTileN / kRows; ++i) {
                        const uint32_t r = min(i * kRows + lane / kWords, rows_left);
                        copy4(dst + lane_word + i * kRows * kSideRow * 4, tside + r * (uint32_t)row_side + min(b, nb - 1) * 4, b < nb ? 4 : 0);
                    }
                }
            } else if (even) {  // one copy per row
                const uint8_t* from = tside + (uint32_t)min(lane, rows_left) * (uint32_t)row_side + (k0 / 32 + (lu - j0) * 4);
                if (lane < kTileN) copy_scales<STEP * 4>(dst + lane * (STEP * 4), from);
            } else {
                // whole aligned words over the bytes of a row, of which the first may belong to the row before; the array
                // may end within a word
                const uint8_t* const end = a.side + a.N * row_side;
#pragma unroll
                for (int i = 0; i < (kTileN * kSideRow + 31) / 32; ++i) {
                    const int j = i * 32 + lane, r = j / kSideRow;
                    if (j < kTileN * kSideRow) {
                        const uint8_t* p = tside + (uint32_t)min(r, rows_left) * (uint32_t)row_side + (k0 / 32 + (lu - j0) * 4);
                        p = reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)3) + (j - r * kSideRow) * 4;
                        const int have = (int)max((int64_t)0, min((int64_t)4, (int64_t)(end - p)));
                        copy4(dst + j * 4, have > 0 ? p : a.side, have);
                    }
                }
            }
            if (++lslot == kRing) lslot = 0;
            li += n, lu += n;
            if (lu == units && li < last) lu = 0, ++lt, point();
        }
        copies_commit();
    };
    if (first < last) point();
#pragma unroll
    for (int d = 0; d < kRing; ++d) copy();

    // ---- activations of this slice: chunks of 8, pairs (i, i + 4) side by side, chunk (lane t, word w) of a unit at
    // (4 w + t) * 16 bytes, so that the four lanes of a quad read 64 consecutive bytes
    constexpr int kBatch = 8;  // loads in flight per thread: the staging is latency, not bandwidth
    const int lg = a.M > 4 ? 3 : a.M > 2 ? 2 : a.M > 1 ? 1 : 0, chunks = a.units_slice * 16;  // 2^lg tokens x 8 / 2^lg chunks
    for (int m0 = 0; m0 < a.M; m0 += kBatch) {
        for (int j0 = threadIdx.x; j0 < chunks; j0 += kThreads << (3 - lg)) {
            uint4 v[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int j = j0 + (b >> lg) * kThreads, m = m0 + (b & ((1 << lg) - 1)), k = k0 + j * 8;
                v[b] = make_uint4(0u, 0u, 0u, 0u);
                if (m < a.M && j < chunks && k < a.K) v[b] = *reinterpret_cast<const uint4*>(a.X + m * a.ldx + k);
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int j = j0 + (b >> lg) * kThreads, m = m0 + (b & ((1 << lg) - 1));
                if (m >= a.M || j >= chunks) continue;
                *reinterpret_cast<uint4*>(smem + m * xrow + (j >> 4) * 256 + ((j & 3) * 4 + ((j >> 2) & 3)) * 16) =
                    make_uint4(__byte_perm(v[b].x, v[b].z, 0x5410), __byte_perm(v[b].x, v[b].z, 0x7632), __byte_perm(v[b].y, v[b].w, 0x5410),
                               __byte_perm(v[b].y, v[b].w, 0x7632));
            }
        }
    }
    __syncthreads();
    pdl_trigger();

    // ---- units in order
    float acc[NT][4];
#pragma unroll
    for (int q = 0; q < NT; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[q][i] = 0.0f;
    int cu = units > 0 ? first % units : 0, ct = units > 0 ? first / units : 0, slot = 0;
    bool whole = cu == 0;  // the run holds the tile's first unit
    const uint8_t* xs[NT];  // the lane's token of each group (columns behind the last token repeat it; they are not stored)
#pragma unroll
    for (int q = 0; q < NT; ++q) xs[q] = smem + min(q * 8 + g, a.M - 1) * xrow + t * 16;
    const int side_pitch = even ? STEP * 4 : kSideRow * 4;
    const uint8_t *side_a = sides + g * side_pitch, *side_b = side_a + 8 * side_pitch;
    int shift_a = 0, shift_b = 0;  // the byte of its word that a row's MXFP4 scales start on
    auto tile_sides = [&]() {
        if (FMT == kMXFP4) {
            const int n0 = (tile0 + ct) * kTileN, left = a.N - 1 - n0;
            shift_a = t + (int)(((n0 + min(g, left)) * row_side) & 3), shift_b = t + (int)(((n0 + min(g + 8, left)) * row_side) & 3);
        } else {
            shift_a = shift_b = (t >> 1) * 4;
        }
    };
    tile_sides();
    for (int i = first; i < last;) {
        const int n = step_units(cu, i), j0 = cu & (STEP - 1);
        copies_wait<kRing - 1>();
        __syncwarp();  // the scales were copied by other lanes
        const uint8_t* codes = ring + slot * (STEP * 1024) + lane * 16;
        const uint8_t *sa = side_a + slot * kSideBytes + shift_a, *sb = side_b + slot * kSideBytes + shift_b;
        const int xat = (cu - j0) * 256;
        bool two = false;
        if (FMT == kMXFP4) {
#pragma unroll
            for (int j = 0; j < STEP; ++j) two |= max(sa[j * 4], sb[j * 4]) > 128;
            two = __any_sync(0xFFFFFFFFu, two);
        }
        auto one = [&](int j, auto with_second) {
            const uint4 qa = *reinterpret_cast<const uint4*>(codes + j * 1024);
            const uint4 qb = *reinterpret_cast<const uint4*>(codes + j * 1024 + 512);
            Scale<FMT> fa, fb;
            if (FMT == kHiF4) {
                fa.set(*reinterpret_cast<const uint32_t*>(sa + j * 8), t & 1);
                fb.set(*reinterpret_cast<const uint32_t*>(sb + j * 8), t & 1);
            } else {
                const bool none = beyond && cu - j0 + j >= units - 1;
                fa.set(sa[j * 4], none), fb.set(sb[j * 4], none);
            }
            unit<FMT, NT, decltype(with_second)::value>(qa, qb, fa, fb, xs, xat + j * 256, acc);
        };
        if (FMT == kMXFP4 && two) {
#pragma unroll 1
            for (int j = j0; j < j0 + n; ++j) one(j, std::true_type());
        } else if (n == STEP) {
#pragma unroll
            for (int j = 0; j < STEP; ++j) one(j, std::false_type());
        } else {
#pragma unroll 1
            for (int j = j0; j < j0 + n; ++j) one(j, std::false_type());
        }
        if (++slot == kRing) slot = 0;
        __syncwarp();  // every lane has read the scales
        copy();        // into the slot that was just read
        i += n, cu += n;
        if (cu == units || i == last) {
            if (CS == 1 && whole && cu == units) {
                const int row = (tile0 + ct) * kTileN + g;
#pragma unroll
                for (int q = 0; q < NT; ++q)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int m = q * 8 + t * 2 + (j & 1);
                        if (m < a.M && row + (j >> 1) * 8 < a.N) store_out(a, m, row + (j >> 1) * 8, acc[q][j] * Scale<FMT>::kBack);
                    }
            } else {
                float* out = part + (size_t)(CS > 1 ? ct + warp : warp * 2 + (i - cu > first ? 1 : 0)) * kSlot;
#pragma unroll
                for (int q = 0; q < NT; ++q) {
                    *reinterpret_cast<float2*>(out + part_at(q * 8 + t * 2, g)) = make_float2(acc[q][0], acc[q][1]);
                    *reinterpret_cast<float2*>(out + part_at(q * 8 + t * 2, g + 8)) = make_float2(acc[q][2], acc[q][3]);
                }
            }
#pragma unroll
            for (int q = 0; q < NT; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[q][j] = 0.0f;
            cu = 0, ++ct, whole = true;
            tile_sides();
        }
    }

    // ---- tiles that several warps (and slices) share, in order
    __syncthreads();
    auto first_of = [&](int w) { return total * w / kWarps; };
    // the parts of the warps from w on whose runs start before unit `end`, four loads at a time
    auto sum_parts = [&](const float* src, int pitch, int w, int end) {
        float s = 0.0f;
        for (; w < kWarps && first_of(w) < end; w += 4) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int f = first_of(w + i);
                v[i] = w + i < kWarps && f < end && f < first_of(w + i + 1) ? src[(w + i) * pitch] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s += v[i];
        }
        return s;
    };
    // element o: row o % 16 of tile (o / 16) % tiles, token o / 16 / tiles
    const int outs = tiles * kTileN * a.M;
    if (CS == 1) {
        // A tile is shared if a warp's run starts inside it; the first such warp adds its parts.
        const int tile = units > 0 ? first / units : 0, u0 = tile * units, u1 = u0 + units;
        int w0 = warp - 1;
        while (w0 >= 0 && first_of(w0) == first_of(w0 + 1)) --w0;  // runs without units
        if (first < last && w0 >= 0 && first > u0 && first_of(w0) <= u0) {
            for (int m = lane >> 4; m < a.M; m += 2) {
                const float* src = part + part_at(m, lane & 15);
                const float s = src[(w0 * 2 + (first_of(w0) < u0 ? 1 : 0)) * kSlot] + sum_parts(src, 2 * kSlot, warp, u1);
                const int n = (tile0 + tile) * kTileN + (lane & 15);
                if (n < a.N) store_out(a, m, n, s * Scale<FMT>::kBack);
            }
        }
    } else {
        // this slice's sum replaces the first warp's part, of which nobody else reads this element
        for (int o = threadIdx.x; o < outs && units > 0; o += kThreads) {
            const int m = (o >> 4) / tiles, tile = (o >> 4) - m * tiles, u0 = tile * units, u1 = u0 + units;
            float* const src = part + part_at(m, o & 15) + tile * kSlot;
            const int w0 = ((u0 + 1) * kWarps + total - 1) / total - 1;  // the warp that has its first unit
            src[w0 * kSlot] += sum_parts(src, kSlot, w0 + 1, u1);
        }
    }
    if (CS > 1) {
        // every slice's sum, in order; a slice without units (the last ones of a short K) has none
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        for (int o = rank * kThreads + threadIdx.x; o < outs; o += CS * kThreads) {
            const int m = (o >> 4) / tiles, tile = (o >> 4) - m * tiles, n = (tile0 + tile) * kTileN + (o & 15);
            if (n >= a.N) continue;
            float v[CS], s = 0.0f;
#pragma unroll
            for (int c = 0; c < CS; ++c) {
                const int cunits = max(0, min(a.units_slice, units_all - c * a.units_slice)), ctotal = tiles * cunits;
                v[c] = 0.0f;
                if (cunits == 0) continue;
                // the first warp of that slice with a part of the tile: the one that has its first unit
                const int w0 = ((tile * cunits + 1) * kWarps + ctotal - 1) / ctotal - 1;
                uint32_t at;
                const uint32_t local = (uint32_t)__cvta_generic_to_shared(part + (size_t)(tile + w0) * kSlot + part_at(m, o & 15));
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(local), "r"(c));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[c]) : "r"(at));
            }
#pragma unroll
            for (int c = 0; c < CS; ++c) s += v[c];
            store_out(a, m, n, s * Scale<FMT>::kBack);
        }
        // no CTA leaves while a peer may still read its shared memory
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
}

// ---- host side -----------------------------------------------------------------------------------
struct GemvPlan {
    int cs, tiles_cta, units_slice, step;
    size_t smem;
};

constexpr size_t kSmemMax = 227 * 1024;

// Splits the K range over cs CTAs and gives each cluster T row tiles so that the busiest SM finishes first.  Cycles per unit, for
// staging the activations and for joining the sums are rough measurements (4 tokens 11008 -> 2048: 9.2 us in four slices and
// 10.3 in one; 16 tokens 3584 -> 3584: 9.9 in two, 11.9 in one; 16 tokens 2048 -> 22016: 21.8 in two, 16.0 in one).
constexpr double kExchange[4] = {0, 1300, 2300, 4500};
GemvPlan plan_gemv(int fmt, int M, int64_t N, int64_t K) {
    const int tiles = (int)((N + kTileN - 1) / kTileN), units = (int)((K + kUnitK - 1) / kUnitK), nt = M > 8 ? 2 : 1;
    GemvPlan best{0, 0, 0, 0, 0};
    double best_cost = 0;
    for (int step = 2; step <= 4; step += 2) {
        for (int lg = 0; lg < 4; ++lg) {
            const int cs = 1 << lg, us = (units + cs - 1) / cs;
            const size_t x = (size_t)M * (us * 256 + kXPad), ring = ring_bytes(fmt, step);
            // MXFP4 scales that come word by word
            const double odd = fmt == kMXFP4 && (K / 32 % (step * 4) || (cs > 1 && us % step)) ? 1.05 : 1.0;
            // the fewest waves that shared memory and kMaxTiles allow, and up to three more: the smallest T for each
            const int slots = resident_clusters(cs);
            int most = std::min(kMaxTiles, tiles);
            if (x + ring + part_bytes(cs, 1, nt) > kSmemMax) continue;
            if (cs > 1) most = std::min(most, 1 + (int)((kSmemMax - x - ring - part_bytes(cs, 1, nt)) / (kTileN * 8 * nt * sizeof(float))));
            for (int waves = (tiles + slots * most - 1) / (slots * most), tried = 0; tried < 4; ++waves, ++tried) {
                const int T = (tiles + slots * waves - 1) / (slots * waves);
                const double units_warp = (T * us + kWarps - 1) / kWarps;
                const double sums = cs == 1 ? 120.0 * M : kExchange[lg] + 2.9 * (T * kTileN * M);
                const double cost = waves * (units_warp * (step == 4 ? 1000 : 1080) * odd + (step == 4 ? 3700 : 3000) + (double)x / 16 + sums);
                if (best.cs == 0 || cost < best_cost) best = GemvPlan{cs, T, us, step, x + ring + part_bytes(cs, T, nt)}, best_cost = cost;
                if (T == 1) break;
            }
        }
    }
    return best;
}

template <int FMT, int NT, int STEP, int CS>
int launch_gemv(const GemvArgs& a, const GemvPlan& p, cudaStream_t stream) {
    auto kern = gemv_kernel<FMT, NT, STEP, CS>;
    int rc = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), (int)kSmemMax, "gemv_kernel shared memory");
    if (rc) return rc;
    const unsigned clusters = (unsigned)((a.tiles + p.tiles_cta - 1) / p.tiles_cta);
    LaunchScope scope(kKindGemm, stream);
    return cuda_fail(launch_clusters(kern, clusters * CS, kThreads, p.smem, CS, stream, a), "gemv_kernel launch");
}
template <int FMT, int NT, int STEP>
int launch_gemv(const GemvArgs& a, const GemvPlan& p, cudaStream_t stream) {
    switch (p.cs) {
        case 1: return launch_gemv<FMT, NT, STEP, 1>(a, p, stream);
        case 2: return launch_gemv<FMT, NT, STEP, 2>(a, p, stream);
        case 4: return launch_gemv<FMT, NT, STEP, 4>(a, p, stream);
        default: return launch_gemv<FMT, NT, STEP, 8>(a, p, stream);
    }
}
template <int FMT>
int launch_gemv(const GemvArgs& a, const GemvPlan& p, cudaStream_t stream) {
    if (a.M > 8) return p.step == 4 ? launch_gemv<FMT, 2, 4>(a, p, stream) : launch_gemv<FMT, 2, 2>(a, p, stream);
    return p.step == 4 ? launch_gemv<FMT, 1, 4>(a, p, stream) : launch_gemv<FMT, 1, 2>(a, p, stream);
}

int gemv(int fmt, const void* X, int64_t M, int64_t K, int64_t ldx, const void* w_codes, const void* w_side, int64_t N, void* Y,
         int out_dtype, int64_t ldy, void* stream) {
    const int block = fmt == kHiF4 ? kHif4Block : kMxBlock;
    if (!X || !w_codes || !w_side || !Y) return fail(RESQ_ERR_NULL, "gemv", "X, the packed weight and Y must not be NULL");
    if (M <= 0 || N <= 0 || K <= 0 || K % block != 0 || M > RESQ_GEMV_MAX_TOKENS || N > INT32_MAX - 65536 || K > RESQ_GEMV_MAX_K) {
        set_last_error("gemv: M=%lld N=%lld K=%lld (1 <= M <= %d, K a positive multiple of %d up to %d, N below 2^31 - 65536)", (long long)M,
                       (long long)N, (long long)K, RESQ_GEMV_MAX_TOKENS, block, RESQ_GEMV_MAX_K);
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
    // Nine to sixteen tokens of very long rows (K beyond about 24000) do not fit in shared memory even in eight slices: they
    // take two passes over the weights.
    GemvPlan p = plan_gemv(fmt, (int)M, N, K);
    const int64_t pass = p.cs ? M : 8;
    if (!p.cs) p = plan_gemv(fmt, 8, N, K);
    GemvArgs a;
    a.codes = static_cast<const uint8_t*>(w_codes);
    a.side = static_cast<const uint8_t*>(w_side);
    a.ldx = ldx, a.ldy = ldy, a.K = (int)K, a.N = (int)N, a.out_dtype = out_dtype;
    a.tiles = (int)((N + kTileN - 1) / kTileN), a.tiles_cta = p.tiles_cta, a.units_slice = p.units_slice;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    for (int64_t m = 0; m < M; m += pass) {
        a.M = (int)std::min(pass, M - m);
        a.X = static_cast<const __nv_bfloat16*>(X) + m * ldx;
        a.Y = static_cast<uint8_t*>(Y) + m * ldy * (out_dtype == RESQ_OUT_BF16 ? 2 : 4);
        const int rc = fmt == kHiF4 ? launch_gemv<kHiF4>(a, p, st) : launch_gemv<kMXFP4>(a, p, st);
        if (rc) return rc;
    }
    return RESQ_OK;
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
