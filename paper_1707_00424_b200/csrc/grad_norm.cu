// parle_grad_norm: the norm of all elements of a list of tensors, sqrt(sum g^2).  One read of every element: bound by DRAM (243 M fp32 137 us, the
// copy rate and 10 % more; 60 M bf16 23 us, 0.8 of it; two launches, 4 to 6 us, where there is little).
//
// Squares and sums are fp64, over the whole range of the types, and the result is the correctly rounded norm but where a tie is as near
// as the sums' roundings (a conversion and a fused operation an element, beside DRAM: squares and sums of eight in fp32 were up to 2 units of the
// last place off where there is little to average, and no faster at 243 M fp32, 3 % at as many bf16).  A chunk's sum depends on its elements alone, and
// chunks are added in one fixed order: the same inputs give the same bits.
#include <math.h>

#include <type_traits>

#include "tensor_list.cuh"

using namespace parle;

namespace {

constexpr int kThreads = 256;
constexpr int kFlight = 4;                               // groups of a thread in flight
constexpr int kSteps = 2;
constexpr int kChunk = kThreads * 8 * kFlight * kSteps;
constexpr int kFinish = 1024;

struct Entry {
    const void *grad;
    long long size_shift;                                // size << 4 | shift << 1 | 1
};
template <int CAP> struct List {
    int count;
    uint32_t first[CAP];
    Entry entry[CAP];
};
constexpr int kFew = 96, kSome = 400, kMany = 1600;      // a launch takes 32764 bytes of arguments at most, and 2 us more with that many

// The sum of a block's numbers, in thread 0; the same order always.
template <int THREADS> __device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[THREADS / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    if (threadIdx.x >= 32) return 0.0;
    v = threadIdx.x < THREADS / 32 ? part[threadIdx.x] : 0.0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
    return v;
}

template <typename G, class L> __global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ L list, double *partial) {
    const int index = entry_of(list, blockIdx.x);
    const Entry &t = list.entry[index];
    const long long n = t.size_shift >> 4;
    const G *const grad = static_cast<const G *>(t.grad);
    long long e0 = (long long)(blockIdx.x - list.first[index]) * kChunk + threadIdx.x * 8 - ((t.size_shift >> 1) & 7);
    double sum = 0.0;
#pragma unroll
    for (int step = 0; step < kSteps; ++step) {
        Pack8<G> x[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const long long e = e0 + u * kThreads * 8;
            if (e >= 0 && e + 8 <= n) x[u].load(grad + e);
        }
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const long long e = e0 + u * kThreads * 8;
            if (e >= n) break;
            float v[8];
            if (e >= 0 && e + 8 <= n) x[u].get(v);
            else load_some(grad, e, n, v);
            double group = 0.0;
#pragma unroll
            for (int i = 0; i < 8; ++i) group = fma((double)v[i], (double)v[i], group);
            sum += group;
        }
        e0 += kFlight * kThreads * 8;
    }
    sum = block_sum<kThreads>(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(kFinish) norm_finish_kernel(const double *partial, long long count, float *norm) {
    double sum = 0.0;
    for (long long i = threadIdx.x; i < count; i += kFinish) sum += partial[i];
    sum = block_sum<kFinish>(sum);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

long long chunks_of(long long size) { return (size + 7 + kChunk - 1) / kChunk; }      // wherever the tensor begins

template <int CAP, typename G> int launch_all(const parle_grad_tensor *tensors, int count, double *partial, long long *written, cudaStream_t stream) {
    List<CAP> list;
    list.count = 0;
    unsigned chunks = 0;
    for (int i = 0;; ++i) {
        const bool end = i == count;
        const long long n = end ? 0 : tensors[i].size;
        if (list.count && (end || list.count == CAP || chunks + chunks_of(n) >= 1LL << 31)) {
            norm_kernel<G><<<chunks, kThreads, 0, stream>>>(list, partial + *written);
            const int rc = launch_status();
            if (rc != PARLE_OK) return rc;
            *written += chunks;
            list.count = 0;
            chunks = 0;
        }
        if (end) return PARLE_OK;
        if (n == 0) continue;
        const int shift = group_shift(tensors[i].grad, sizeof(G));
        list.first[list.count] = chunks;
        list.entry[list.count++] = {tensors[i].grad, n << 4 | shift << 1 | 1};
        chunks += (unsigned)((n + shift + kChunk - 1) / kChunk);
    }
}

}  // namespace

extern "C" size_t parle_grad_norm_workspace_bytes(const parle_grad_tensor *tensors, int count) {
    if (count <= 0 || !tensors) return 0;
    long long chunks = 0;
    for (int i = 0; i < count; ++i) {
        if (tensors[i].size < 0 || tensors[i].size > PARLE_TOKEN_MAX_ELEMENTS) return 0;
        if (tensors[i].size) chunks += chunks_of(tensors[i].size);
    }
    return round_up((size_t)chunks * sizeof(double), 128);
}

extern "C" int parle_grad_norm(const parle_grad_tensor *tensors, int count, int grad_dtype, float *norm, void *workspace, size_t workspace_bytes,
                               void *cuda_stream) {
    if (count < 0 || (count && !tensors) || !valid_dtype(grad_dtype) || !norm) return PARLE_EINVAL;
    long long chunks = 0;
    for (int i = 0; i < count; ++i) {
        const parle_grad_tensor &t = tensors[i];
        if (t.size < 0) return PARLE_EINVAL;
        if (t.size == 0) continue;
        if (t.size > PARLE_TOKEN_MAX_ELEMENTS) return PARLE_ETOOBIG;
        if (!t.grad) return PARLE_EINVAL;
        if (!element_aligned(t.grad, grad_dtype)) return PARLE_EALIGN;
        chunks += chunks_of(t.size);
    }
    if (reinterpret_cast<uintptr_t>(norm) % 4) return PARLE_EALIGN;
    if (chunks && !workspace) return PARLE_EINVAL;
    if (reinterpret_cast<uintptr_t>(workspace) % 128) return PARLE_EALIGN;
    if (workspace_bytes < (size_t)chunks * sizeof(double)) return PARLE_EWORKSPACE;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    double *const partial = static_cast<double *>(workspace);
    long long written = 0;
    const int rc = with_dtype(grad_dtype, [&](auto *g) {
        using G = std::remove_pointer_t<decltype(g)>;
        return count <= kFew ? launch_all<kFew, G>(tensors, count, partial, &written, stream)
             : count <= kSome ? launch_all<kSome, G>(tensors, count, partial, &written, stream) : launch_all<kMany, G>(tensors, count, partial, &written, stream);
    });
    if (rc != PARLE_OK) return rc;
    norm_finish_kernel<<<1, kFinish, 0, stream>>>(partial, written, norm);
    return launch_status();
}
