// Shared pieces of the operators that walk rows of plain tensors (block_join.cu, token_logprobs.cu, gemv.cu): host-side
// argument checks and 8-element vector access.  Internal.
#pragma once
#include "common.cuh"

namespace resq {

inline bool is_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int fail(int status, const char* what, const char* why) {
    set_last_error("%s: %s", what, why);
    return status;
}
// Rows of bf16 or fp32 values: 16-byte aligned base, rows that start on 16-byte boundaries, ld >= cols.
inline bool rows_aligned(const void* p, int64_t ld, int64_t cols, int dtype) {
    return is_aligned(p, 16) && ld >= cols && ld % (dtype == RESQ_OUT_BF16 ? 8 : 4) == 0;
}

// Clusters of cs CTAs that are resident at once with one CTA per SM, as the occupancy query answers on a B200: larger clusters
// leave SMs of a GPC unused.  Plans only choose splits by it, and the workspace query has to answer without a device: a device with
// other counts gets right results at another speed.
inline int resident_clusters(int cs) { return cs == 1 ? 148 : cs == 2 ? 74 : cs == 4 ? 33 : 15; }

#ifdef __CUDACC__

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Eight consecutive elements as they lie in memory.  `n` < 8 at the ragged end of a row: only those are touched (the
// row's padding is neither read nor written).
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
    uint4 q;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int n) {
        if (n >= 8) {
            q = *reinterpret_cast<const uint4*>(p);
            return;
        }
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        const unsigned short* s = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) w[i / 2] |= (uint32_t)s[i] << (16 * (i & 1));
        q = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = bf16_lo(q.x), v[1] = bf16_hi(q.x), v[2] = bf16_lo(q.y), v[3] = bf16_hi(q.y);
        v[4] = bf16_lo(q.z), v[5] = bf16_hi(q.z), v[6] = bf16_lo(q.w), v[7] = bf16_hi(q.w);
    }
};
template <>
struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p, int n) {
        if (n >= 8) {
            a = reinterpret_cast<const float4*>(p)[0];
            b = reinterpret_cast<const float4*>(p)[1];
            return;
        }
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.0f;
        a = make_float4(v[0], v[1], v[2], v[3]);
        b = make_float4(v[4], v[5], v[6], v[7]);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
};

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8], int n) {
    if (n >= 8) {
        *reinterpret_cast<uint4*>(p) =
            make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = __float2bfloat16_rn(v[i]);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8], int n) {
    if (n >= 8) {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = v[i];
}

// Pairs of fp32 values in one instruction.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Sums of NV (1 or 4) values over the block, the same bits in every thread; fixed order.  `buf` holds NV * 32 floats (16-byte
// aligned) and must not be the buffer of the previous call (two alternate, which saves a barrier).  Four values share their
// shuffles: after two exchanges a lane carries one of them (6 shuffles instead of 20).
// It is a barrier of the block for shared memory too, which callers rely on: what a thread has read, written or waited for before
// it is ordered before what the others do behind it.
template <int NV>
__device__ __forceinline__ void block_sum(float (&v)[NV], float* buf) {
    static_assert(NV == 1 || NV == 4, "");
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = (blockDim.x + 31) >> 5;
    float x = v[0];
    if (NV == 4) {
        const bool up = lane & 16;
        const float a = (up ? v[2 % NV] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, up ? v[0] : v[2 % NV], 16);
        const float b = (up ? v[3 % NV] : v[1 % NV]) + __shfl_xor_sync(0xFFFFFFFFu, up ? v[1 % NV] : v[3 % NV], 16);
        x = (lane & 8 ? b : a) + __shfl_xor_sync(0xFFFFFFFFu, lane & 8 ? a : b, 8);
    } else {
        x += __shfl_xor_sync(0xFFFFFFFFu, x, 16);
        x += __shfl_xor_sync(0xFFFFFFFFu, x, 8);
    }
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 4);
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 2);
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
    if (nw == 1) {
        __syncwarp();  // shuffles order no memory
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = NV == 1 ? x : __shfl_sync(0xFFFFFFFFu, x, i * 8);
        return;
    }
    if (NV == 1 ? lane == 0 : (lane & 7) == 0) buf[(lane >> 3) * 32 + w] = x;
    __syncthreads();
    if (nw <= 8) {  // read back whole: less latency than five more shuffles
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const float4 p = *reinterpret_cast<const float4*>(buf + i * 32), q = *reinterpret_cast<const float4*>(buf + i * 32 + 4);
            v[i] = (((nw > 0 ? p.x : 0.0f) + (nw > 1 ? p.y : 0.0f)) + ((nw > 2 ? p.z : 0.0f) + (nw > 3 ? p.w : 0.0f))) +
                   (((nw > 4 ? q.x : 0.0f) + (nw > 5 ? q.y : 0.0f)) + ((nw > 6 ? q.z : 0.0f) + (nw > 7 ? q.w : 0.0f)));
        }
        return;
    }
    if (NV == 4) {  // eight lanes per value
        float y = 0.0f;
        for (int j = lane & 7; j < nw; j += 8) y += buf[(lane >> 3) * 32 + j];
        y += __shfl_xor_sync(0xFFFFFFFFu, y, 4);
        y += __shfl_xor_sync(0xFFFFFFFFu, y, 2);
        y += __shfl_xor_sync(0xFFFFFFFFu, y, 1);
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = __shfl_sync(0xFFFFFFFFu, y, i * 8);
        return;
    }
    v[0] = lane < nw ? buf[lane] : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], o);
}

// launch_kernel() with clusters of `cs` CTAs.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_clusters(void (*kern)(KArgs...), dim3 grid, unsigned block, size_t smem, int cs, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cs;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, KArgs(args)...);
}

#endif  // __CUDACC__

}  // namespace resq
