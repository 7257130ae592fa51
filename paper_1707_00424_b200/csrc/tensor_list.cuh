// Kernels over a list of tensors (AdamW, gradient norm): the list travels in the launch's own arguments, so that a call needs no table in
// device memory, no copy to fill it and nothing that two calls could share.  (A launch with 32 KB of arguments takes 2 us more of the host's time
// than one with 2 KB, so there are kernels for short lists.)  A block takes one chunk of one tensor.
#pragma once

#include "token_types.cuh"

namespace parle {

// Elements of 16-bit or wider arrays are taken in groups of eight.  A tensor may begin anywhere: its groups are cut where memory's are, so
// that only the first and the last one are partial.  This is the distance of `p` from such a cut, in elements.
inline int group_shift(const void *p, int bytes) { return (int)(reinterpret_cast<uintptr_t>(p) / bytes % 8); }

// Entry of the list that chunk `chunk` belongs to: the last whose first chunk is not behind it.  first[0] = 0; every entry has a chunk.
template <class List> __device__ __forceinline__ int entry_of(const List &list, uint32_t chunk) {
    int low = 0, high = list.count;
    while (high - low > 1) {
        const int mid = (low + high) / 2;
        if (list.first[mid] <= chunk) low = mid; else high = mid;
    }
    return low;
}

// Elements e0 .. e0 + 7 of [0, n) at base + e0 as fp32, one by one; 0 outside.
template <typename T> __device__ __forceinline__ void load_some(const T *base, long long e0, long long n, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e0 + i >= 0 && e0 + i < n ? to_float(base[e0 + i]) : 0.f;
}
template <typename T> __device__ __forceinline__ void store_some(T *base, long long e0, long long n, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (e0 + i >= 0 && e0 + i < n) base[e0 + i] = from_float<T>(v[i]);
}

}  // namespace parle
