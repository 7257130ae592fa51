// parle_dropout: dropout whose mask is a function of (seed, offset, element number) and is never stored.
//
// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): the
// counter of eight consecutive elements is (element / 8, offset), the key is the seed; each of the four output words gives
// two 16-bit fields, low half first, one per element.  An element is kept when its field is at least
// t = round(65536 p), i.e. with probability exactly 1 - t/65536, and then multiplied by 65536 / (65536 - t), so the
// expectation is x.  16 bits an element instead of 32 halve the integer work: 20 wide multiplications for eight elements.
#include <math.h>

#include <type_traits>

#include "token_types.cuh"

using namespace parle;

namespace {

struct DropoutArgs {
    const void *x, *residual;
    void *y;
    long long ld_x, ld_r, ld_y;
    long long rows, cols;
    uint32_t threshold;                                  // 0 .. 65536
    float scale;
    unsigned long long seed, offset;
    const unsigned long long *offset_dev;
};

__device__ __forceinline__ uint4 philox4x32_10(unsigned long long group, unsigned long long offset, unsigned long long seed) {
    uint32_t c0 = (uint32_t)group, c1 = (uint32_t)(group >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// Bit i: element i of the group is kept.
__device__ __forceinline__ uint32_t keep_bits(const uint4 &w, uint32_t threshold) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bits |= (v[i] & 0xffffu) >= threshold ? 1u << (2 * i) : 0u;
        bits |= (v[i] >> 16) >= threshold ? 2u << (2 * i) : 0u;
    }
    return bits;
}

__device__ __forceinline__ unsigned long long call_offset(const DropoutArgs &p) {
    return p.offset + (p.offset_dev ? *p.offset_dev : 0ull);
}

// A dropped element is zero whatever its value was (a selection: NaN and Inf do not pass through the product).
__device__ __forceinline__ float dropped(float x, bool keep, float scale) { return keep ? x * scale : 0.f; }

constexpr int kThreads = 256;

// Groups of eight elements that lie in one row and start on 16-byte boundaries in every operand: one thread per group, `U`
// groups in flight.  `per_row` groups a row; rows == 1 stands for a wholly contiguous array.
template <typename T, bool RES, int U>
__global__ void __launch_bounds__(kThreads) dropout_groups_kernel(const DropoutArgs p, long long groups, long long per_row) {
    const long long first = (long long)blockIdx.x * (kThreads * U) + threadIdx.x;
    const unsigned long long offset = call_offset(p);
    Pack8<T> x[U], r[U];
    long long at_y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long g = first + u * kThreads;
        if (g >= groups) break;
        long long row = 0, col = g * 8;
        if (p.rows > 1) { row = g / per_row; col = (g - row * per_row) * 8; }
        x[u].load(static_cast<const T *>(p.x) + row * p.ld_x + col);
        if (RES) r[u].load(static_cast<const T *>(p.residual) + row * p.ld_r + col);
        at_y[u] = row * p.ld_y + col;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long g = first + u * kThreads;
        if (g >= groups) break;
        const uint32_t keep = keep_bits(philox4x32_10((unsigned long long)g, offset, p.seed), p.threshold);
        float v[8], w[8];
        x[u].get(v);
        if (RES) r[u].get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = dropped(v[i], (keep >> i) & 1u, p.scale);
            if (RES) v[i] += w[i];
        }
        Pack8<T> out;
        out.set(v);
        out.store(static_cast<T *>(p.y) + at_y[u]);
    }
}

// Any pitch and alignment: a warp takes 32 consecutive groups (256 elements in row-major order); every lane draws one group's
// numbers, then the warp walks over the 256 elements 32 at a time, so that its accesses are consecutive, and each lane
// fetches its element's keep bit from the lane that drew it.
template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_elements_kernel(const DropoutArgs p, long long first_group, long long elements) {
    const int lane = threadIdx.x % 32;
    const long long warp = (long long)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    const long long group0 = first_group + warp * 32;
    const long long e0 = group0 * 8;
    if (e0 >= elements) return;
    const uint32_t keep = keep_bits(philox4x32_10((unsigned long long)(group0 + lane), call_offset(p), p.seed), p.threshold);
    const long long row0 = e0 / p.cols, col0 = e0 - row0 * p.cols;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int o = i * 32 + lane;                     // element of the warp's 256
        const uint32_t bits = __shfl_sync(0xffffffffu, keep, o / 8);
        if (e0 + o >= elements) continue;
        long long row = row0, col = col0 + o;
        if (col >= p.cols) {
            const long long down = col / p.cols;
            row += down;
            col -= down * p.cols;
        }
        const float x = to_float(static_cast<const T *>(p.x)[row * p.ld_x + col]);
        float v = dropped(x, (bits >> (o % 8)) & 1u, p.scale);
        if (p.residual) v += to_float(static_cast<const T *>(p.residual)[row * p.ld_r + col]);
        static_cast<T *>(p.y)[row * p.ld_y + col] = from_float<T>(v);
    }
}

template <typename T> int launch_dropout(const DropoutArgs &a, int dtype, cudaStream_t stream) {
    DropoutArgs p = a;
    const long long elements = p.rows * p.cols;
    const bool contiguous = p.rows == 1 || (p.ld_x == p.cols && p.ld_y == p.cols && (!p.residual || p.ld_r == p.cols));
    if (contiguous) { p.rows = 1; p.cols = p.ld_x = p.ld_r = p.ld_y = elements; }
    const bool aligned = contiguous
        ? rows_aligned16(p.x, 0, dtype) && rows_aligned16(p.y, 0, dtype) && rows_aligned16(p.residual, 0, dtype)
        : p.cols % 8 == 0 && rows_aligned16(p.x, p.ld_x, dtype) && rows_aligned16(p.y, p.ld_y, dtype) &&
              (!p.residual || rows_aligned16(p.residual, p.ld_r, dtype));
    long long done = 0;                                  // elements covered by whole aligned groups
    if (aligned) {
        constexpr int U = 2;
        const long long groups = elements / 8;
        done = groups * 8;
        if (groups) {
            const long long blocks = (groups + kThreads * U - 1) / (kThreads * U);
            if (p.residual) dropout_groups_kernel<T, true, U><<<(unsigned)blocks, kThreads, 0, stream>>>(p, groups, p.cols / 8);
            else dropout_groups_kernel<T, false, U><<<(unsigned)blocks, kThreads, 0, stream>>>(p, groups, p.cols / 8);
            const int rc = launch_status();
            if (rc != PARLE_OK) return rc;
        }
    }
    if (done < elements) {
        const long long groups = (elements - done + 7) / 8, blocks = (groups + kThreads - 1) / kThreads;
        dropout_elements_kernel<T><<<(unsigned)blocks, kThreads, 0, stream>>>(p, done / 8, elements);
        return launch_status();
    }
    return PARLE_OK;
}

}  // namespace

extern "C" int parle_dropout(const void *x, long long ld_x, const void *residual, long long ld_r, void *y, long long ld_y,
                             int dtype, long long rows, long long cols, double p, uint64_t seed, uint64_t offset,
                             const uint64_t *offset_dev, void *cuda_stream) {
    if (!valid_dtype(dtype) || rows < 0 || cols < 0 || !(p >= 0.0 && p <= 1.0)) return PARLE_EINVAL;
    if (rows > 1 && (ld_x < 0 || ld_y < cols || (residual && ld_r < 0))) return PARLE_EINVAL;
    if (rows > 1 && ((x == y && ld_x != ld_y) || (residual == y && ld_r != ld_y))) return PARLE_EINVAL;
    if (rows == 0 || cols == 0) return PARLE_OK;
    if (!x || !y) return PARLE_EINVAL;
    if (rows > PARLE_TOKEN_MAX_ELEMENTS / cols) return PARLE_ETOOBIG;
    if (!element_aligned(x, dtype) || !element_aligned(y, dtype) || !element_aligned(residual, dtype) ||
        reinterpret_cast<uintptr_t>(offset_dev) % 8) return PARLE_EALIGN;
    DropoutArgs a = {};
    a.x = x; a.residual = residual; a.y = y;
    a.ld_x = ld_x; a.ld_r = ld_r; a.ld_y = ld_y;
    a.rows = rows; a.cols = cols;
    a.threshold = (uint32_t)floor(p * 65536.0 + 0.5);
    a.scale = a.threshold < 65536u ? (float)(65536.0 / (65536.0 - (double)a.threshold)) : 0.f;
    a.seed = seed; a.offset = offset;
    a.offset_dev = reinterpret_cast<const unsigned long long *>(offset_dev);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return with_dtype(dtype, [&](auto *tag) { return launch_dropout<std::remove_pointer_t<decltype(tag)>>(a, dtype, stream); });
}
