// Element types of the token operators (embedding, dropout, token log probabilities): loads to and stores from fp32.
#pragma once

#include <cuda_fp16.h>

#include <atomic>

#include "common.cuh"

namespace parle {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

// One rounding, to nearest with ties to even, of a value computed in fp32.
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Eight consecutive elements as fp32; p is aligned to 16 bytes.  (16 bytes of a 16-bit type, 2 x 16 bytes of fp32.)
__device__ __forceinline__ void unpack8(const float4 &a, const float4 &b, float (&v)[8]) {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <typename T> struct Pack8;                      // the raw form of eight elements, so that loads can be issued early
template <> struct Pack8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = reinterpret_cast<const float4 *>(p)[0];
        b = reinterpret_cast<const float4 *>(p)[1];
    }
    __device__ __forceinline__ void get(float (&v)[8]) const { unpack8(a, b, v); }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        a = make_float4(v[0], v[1], v[2], v[3]);
        b = make_float4(v[4], v[5], v[6], v[7]);
    }
    __device__ __forceinline__ void store(float *p) const {
        reinterpret_cast<float4 *>(p)[0] = a;
        reinterpret_cast<float4 *>(p)[1] = b;
    }
};
template <> struct Pack8<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { a = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {                    // a bf16 is the upper half of the fp32 word
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        __nv_bfloat162 h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        a = *reinterpret_cast<const uint4 *>(h);
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = a; }
};
template <> struct Pack8<__half> {
    uint4 a;
    __device__ __forceinline__ void load(const __half *p) { a = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        __half2 h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        a = *reinterpret_cast<const uint4 *>(h);
    }
    __device__ __forceinline__ void store(__half *p) const { *reinterpret_cast<uint4 *>(p) = a; }
};

// Moves the N words from byte `at` of w on (0 .. 15; even; a multiple of 4 but for HALVES) to its beginning.
template <int N, bool HALVES> __device__ __forceinline__ void skip_bytes(uint32_t (&w)[N + 4], int at) {
    if (at & 8) {
#pragma unroll
        for (int i = 0; i < N + 2; ++i) w[i] = w[i + 2];
    }
    if (at & 4) {
#pragma unroll
        for (int i = 0; i < N + 1; ++i) w[i] = w[i + 1];
    }
    if (HALVES && (at & 2)) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
}

inline bool valid_dtype(int dtype) { return dtype == PARLE_F32 || dtype == PARLE_BF16 || dtype == PARLE_F16; }
inline int dtype_bytes(int dtype) { return dtype == PARLE_F32 ? 4 : 2; }
// Whether p lies on a boundary of its element type.
inline bool element_aligned(const void *p, int dtype) { return reinterpret_cast<uintptr_t>(p) % dtype_bytes(dtype) == 0; }
// Whether rows of this pitch, starting at p, all start on 16-byte boundaries.
inline bool rows_aligned16(const void *p, long long ld, int dtype) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * dtype_bytes(dtype)) % 16 == 0;
}

// Calls f with a null pointer of the element type as a tag.
template <typename F> int with_dtype(int dtype, F f) {
    switch (dtype) {
        case PARLE_F32: return f((float *)nullptr);
        case PARLE_BF16: return f((__nv_bfloat16 *)nullptr);
        case PARLE_F16: return f((__half *)nullptr);
    }
    return PARLE_EINVAL;
}

// a / b, by 32-bit division where both fit (a 64-bit one is four times as long).
__device__ __forceinline__ long long quotient(long long a, long long b) {
    if (((a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
    return a / b;
}

// SMs of the current device; -1 if it cannot be asked.
inline int current_sms() {
    static std::atomic<int> known[64];
    int dev = -1, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return -1;
    if (dev < 64 && (sms = known[dev].load(std::memory_order_relaxed)) > 0) return sms;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return -1;
    if (dev < 64) known[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

// ---- thread-block clusters ----

__device__ __forceinline__ int cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return (int)r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// Says that this thread is done with the other blocks' shared memory; cluster_wait() then waits until all are.  (Relaxed: it orders
// no memory, so nobody's stores in flight are waited for.)
__device__ __forceinline__ void cluster_done() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
// Address of another block's copy of a shared variable.
template <typename V> __device__ __forceinline__ V *at_rank(V *p, int rank) {
    uint64_t r;
    asm volatile("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
    return reinterpret_cast<V *>(r);
}

// A launch of blocks in clusters of `cluster` along x (1: none).  attr: room for the attribute.
inline cudaLaunchConfig_t cluster_config(dim3 grid, int threads, size_t shared_bytes, int cluster, cudaLaunchAttribute *attr, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared_bytes;
    cfg.stream = stream;
    attr->id = cudaLaunchAttributeClusterDimension;
    attr->val.clusterDim.x = cluster;
    attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 1 : 0;
    return cfg;
}

inline int launch_status() { return cudaGetLastError() == cudaSuccess ? PARLE_OK : PARLE_ECUDA; }

}  // namespace parle
