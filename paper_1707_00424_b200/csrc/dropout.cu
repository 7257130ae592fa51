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
    uint32_t upper_threshold;                            // t << 16; t = 65536: all dropped, see drop_all
    int drop_all;
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

// Whether element i of a group is kept: its field against the threshold, both in the upper half of a word.
__device__ __forceinline__ bool kept(const uint4 &w, int i, uint32_t upper_threshold) {
    const uint32_t v = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
    return (i % 2 ? v : v << 16) >= upper_threshold;
}

__device__ __forceinline__ unsigned long long call_offset(const DropoutArgs &p) {
    return p.offset + (p.offset_dev ? *p.offset_dev : 0ull);
}

// A dropped element is zero whatever its value was (a selection: NaN and Inf do not pass through the product).
__device__ __forceinline__ float dropped(float x, bool keep, float scale) { return keep ? x * scale : 0.f; }

// A group's fields.  (All zero, below any threshold but 0, where everything is dropped: 65536 << 16 does not fit.)
__device__ __forceinline__ uint4 fields(const DropoutArgs &p, unsigned long long group, unsigned long long offset) {
    return p.drop_all ? make_uint4(0, 0, 0, 0) : philox4x32_10(group, offset, p.seed);
}

constexpr int kThreads = 256;

// One group: x and r as loaded, group number g.
template <typename T, bool RES> __device__ __forceinline__ Pack8<T> drop_group(const DropoutArgs &p, const Pack8<T> &x, const Pack8<T> &r, unsigned long long g, unsigned long long offset) {
    const uint4 w = fields(p, g, offset);
    float v[8], e[8];
    x.get(v);
    if (RES) r.get(e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = dropped(v[i], kept(w, i, p.upper_threshold), p.scale);
        if (RES) v[i] += e[i];
    }
    Pack8<T> out;
    out.set(v);
    return out;
}

// Contiguous arrays on 16-byte boundaries: kFlight groups of eight elements of a thread in flight.  16384 x 4096 bf16: with a
// residual 61 us, the copy rate; without 45 us, 0.91 of it: there the integer work of the generator (20 wide multiplications and as
// many three-way xors for eight elements) takes most of the issue slots.
constexpr int kFlight = 4;
template <typename T, bool RES>
__global__ void __launch_bounds__(kThreads) dropout_flat_kernel(const DropoutArgs p, long long groups, int rest) {
    const long long first = (long long)blockIdx.x * (kThreads * kFlight) + threadIdx.x;
    Pack8<T> x[kFlight], r[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
        const long long g = first + u * kThreads;
        if (g >= groups) break;
        x[u].load(static_cast<const T *>(p.x) + g * 8);
        if (RES) r[u].load(static_cast<const T *>(p.residual) + g * 8);
    }
    const unsigned long long offset = call_offset(p);
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
        const long long g = first + u * kThreads;
        if (g >= groups) break;
        drop_group<T, RES>(p, x[u], r[u], (unsigned long long)g, offset).store(static_cast<T *>(p.y) + g * 8);
    }
    if (blockIdx.x == gridDim.x - 1 && (int)threadIdx.x < rest) {      // the elements behind the last whole group, a thread each
        const long long e = groups * 8 + threadIdx.x;
        const uint4 w = fields(p, (unsigned long long)groups, offset);
        const uint32_t word = threadIdx.x < 2 ? w.x : threadIdx.x < 4 ? w.y : threadIdx.x < 6 ? w.z : w.w;
        float v = dropped(to_float(static_cast<const T *>(p.x)[e]), (threadIdx.x % 2 ? word : word << 16) >= p.upper_threshold, p.scale);
        if (RES) v += to_float(static_cast<const T *>(p.residual)[e]);
        static_cast<T *>(p.y)[e] = from_float<T>(v);
    }
}

// Rows of whole groups on 16-byte boundaries, at any pitch: 1 << log_per_row threads of a block take a row, in col_blocks blocks
// if it is long.
template <typename T, bool RES>
__global__ void __launch_bounds__(kThreads) dropout_rows_kernel(const DropoutArgs p, int log_per_row, unsigned col_blocks) {
    const int per_row = (int)(p.cols / 8);
    const unsigned row_block = blockIdx.x / col_blocks, col_block = blockIdx.x - row_block * col_blocks;
    const long long row = (long long)row_block * (kThreads >> log_per_row) + (threadIdx.x >> log_per_row);
    if (row >= p.rows) return;
    const int first = (int)(col_block * kFlight << log_per_row) + (threadIdx.x & ((1 << log_per_row) - 1));
    const T *px = static_cast<const T *>(p.x) + row * p.ld_x, *pr = static_cast<const T *>(p.residual) + row * p.ld_r;
    T *py = static_cast<T *>(p.y) + row * p.ld_y;
    Pack8<T> x[kFlight], r[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
        const int c = first + (u << log_per_row);
        if (c >= per_row) break;
        x[u].load(px + (long long)c * 8);
        if (RES) r[u].load(pr + (long long)c * 8);
    }
    const unsigned long long offset = call_offset(p);
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
        const int c = first + (u << log_per_row);
        if (c >= per_row) break;
        drop_group<T, RES>(p, x[u], r[u], (unsigned long long)row * per_row + c, offset).store(py + (long long)c * 8);
    }
}

// Eight elements as words.
template <typename T> struct Words {
    static constexpr int N = 2 * sizeof(T);               // words of eight elements
    // N words of w from byte `at` on, the same in the whole warp
    __device__ __forceinline__ static Pack8<T> from(uint32_t (&w)[N + 4], int at) {
        skip_bytes<N, sizeof(T) == 2>(w, at);
        Pack8<T> v;
        uint32_t *to = reinterpret_cast<uint32_t *>(&v);
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = w[i];
        return v;
    }
};

// A row, for a warp that takes some of it from `base` on.  Places are relative to that; the row lies at [low, high).
template <typename T> struct Shifted {
    const T *at;                                          // element `base` (may lie before the row)
    int skew;                                             // bytes of it behind a 16-byte boundary
    __device__ __forceinline__ Shifted(const void *array, long long ld, long long row, long long base) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(array) + (uintptr_t)((row * ld + base) * (long long)sizeof(T));
        at = reinterpret_cast<const T *>(a);
        skew = (int)(a & 15);
    }
    // Elements o .. o + 7: from the 16-byte pieces that hold them, where those lie in the row; else one by one.
    __device__ __forceinline__ Pack8<T> load(int o, int low, int high) const {
        constexpr int S = sizeof(T);
        if ((o - low) * S >= skew && (high - o - 8) * S >= ((16 - skew) & 15)) {
            uint32_t w[Words<T>::N + 4];
            const uint4 *from = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(at + o) - skew);
#pragma unroll
            for (int i = 0; i < Words<T>::N / 4 + 1; ++i) {
                const uint4 q = i < Words<T>::N / 4 || skew ? from[i] : make_uint4(0, 0, 0, 0);
                w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
            }
            return Words<T>::from(w, skew);
        }
        Pack8<T> v = {};
        T *e = reinterpret_cast<T *>(&v);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (o + i >= low && o + i < high) e[i] = at[o + i];
        return v;
    }
};

constexpr int kSteps = 4, kShifted = 96;                  // steps where there are many parts; shortest rows for many elements
constexpr long long kFew = 1 << 18;
// Any pitch and alignment: a warp takes 32 groups of a row at a time, a lane each, `steps` times.  Groups lie anywhere against 16-byte
// boundaries, by the same number of bytes in all lanes: a lane loads the pieces that hold its group and shifts them, and stores the
// piece that ends its left neighbour's group and begins its own.  Only at the ends of the row and of the 32 groups elements go one by one.
// Bound by issue slots (shifting costs as much as the generator).  8192 x 4095 bf16 of pitch 4127 to 4095: 42 us, element by element 86;
// with a residual, 4096 to 4095, 57 against 96; in one step a warp instead of four 54 and 66; 77 x 1001 2.4 against 3.3.
template <typename T, bool RES>
__global__ void __launch_bounds__(kThreads, 6) dropout_shifted_kernel(const DropoutArgs p, long long parts, long long per_row, int steps) {
    const int lane = threadIdx.x % 32;
    const long long s = (long long)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (s >= parts) return;
    const long long row = quotient(s, per_row), e0 = row * p.cols;
    const long long base = (s - row * per_row) * steps * 256 - e0 % 8;
    const Shifted<T> x(p.x, p.ld_x, row, base), r(p.residual, p.ld_r, row, base), y(p.y, p.ld_y, row, base);
    const int shifted = y.skew / (int)sizeof(T);          // elements at a group's end that lie in the next lane's piece
    const unsigned long long offset = call_offset(p);
    const unsigned long long group = (unsigned long long)(e0 + base) / 8;
    const int low = (int)max(-base, -1024LL), high = (int)min(p.cols - base, kSteps * 256 + 1024LL);      // (clipped where it does not matter)
    for (int first = 0; first < min(steps * 256, high); first += 256) {
        const int o = first + lane * 8;
        const Pack8<T> in = x.load(o, low, high);
        Pack8<T> add;
        if (RES) add = r.load(o, low, high);
        const Pack8<T> out = drop_group<T, RES>(p, in, add, group + o / 8, offset);
        T *const to = const_cast<T *>(y.at) + o;
        const bool whole = o >= low && o + 8 <= high;
        if (y.skew == 0 && whole) {
            out.store(to);
            continue;
        }
        bool joined = false, joined_next = false;
        if (y.skew) {
            const unsigned wholes = __ballot_sync(0xffffffffu, whole);
            const uint32_t *own = reinterpret_cast<const uint32_t *>(&out);
            constexpr int N = Words<T>::N;
            uint32_t w[N + 4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __shfl_up_sync(0xffffffffu, own[N - 4 + i], 1);
#pragma unroll
            for (int i = 0; i < N; ++i) w[4 + i] = own[i];
            const unsigned both = wholes & (wholes << 1); // lanes whose piece is all theirs and their neighbour's
            joined = (both >> lane) & 1u;
            joined_next = lane < 31 && ((both >> (lane + 1)) & 1u);
            const Pack8<T> piece = Words<T>::from(w, 16 - y.skew);
            if (joined) piece.store(to - shifted);
        }
        const T *e = reinterpret_cast<const T *>(&out);
        const int from = joined ? 8 - shifted : 0, until = joined_next ? 8 - shifted : 8;
        if (from < until) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= from && i < until && o + i >= low && o + i < high) to[i] = e[i];
        }
    }
}

// The same for many elements of fp32, whose single accesses are wide enough: a warp takes kSegment elements of a row, which lie in
// at most 32 groups; every lane draws one group's numbers, then the warp walks over the elements 32 at a time, so that its accesses are
// consecutive, and each lane fetches its element's keep bit from the lane that drew it.  All loads come before the stores (y may
// be x).
constexpr int kSegment = 248;
template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_segments_kernel(const DropoutArgs p, long long segments, unsigned per_row) {
    const int lane = threadIdx.x % 32;
    const long long s = (long long)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (s >= segments) return;
    const long long row = quotient(s, per_row), col = (s - row * per_row) * kSegment, e0 = row * p.cols + col;
    const int count = (int)min((long long)kSegment, p.cols - col);
    const T *px = static_cast<const T *>(p.x) + row * p.ld_x + col, *pr = static_cast<const T *>(p.residual) + row * p.ld_r + col;
    T *py = static_cast<T *>(p.y) + row * p.ld_y + col;
    float x[8], r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int o = i * 32 + lane;
        if (o >= count) break;
        x[i] = to_float(px[o]);
        if (p.residual) r[i] = to_float(pr[o]);
    }
    const uint4 w = fields(p, (unsigned long long)(e0 / 8 + lane), call_offset(p));
    uint32_t keep = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) keep |= kept(w, i, p.upper_threshold) ? 1u << i : 0u;
    const int shift = (int)(e0 % 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int o = i * 32 + lane;
        const uint32_t bits = __shfl_sync(0xffffffffu, keep, (o + shift) / 8);
        if (o >= count) continue;
        float v = dropped(x[i], (bits >> ((o + shift) % 8)) & 1u, p.scale);
        if (p.residual) v += r[i];
        py[o] = from_float<T>(v);
    }
}

// Many shorter rows: the same over 32 consecutive groups (256 elements in row-major order).
template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_elements_kernel(const DropoutArgs p, long long elements) {
    const int lane = threadIdx.x % 32;
    const long long first = ((long long)blockIdx.x * (kThreads / 32) + threadIdx.x / 32) * 32, e0 = first * 8;
    if (e0 >= elements) return;
    const long long row0 = quotient(e0, p.cols), col0 = e0 - row0 * p.cols;
    float x[8], r[8];
    long long at_y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int o = i * 32 + lane;
        if (e0 + o >= elements) break;
        long long row = row0, col = col0 + o;
        if (col >= p.cols) {
            const int down = p.cols >= 256 ? 1 : (int)col / (int)p.cols;
            row += down;
            col -= down * p.cols;
        }
        x[i] = to_float(static_cast<const T *>(p.x)[row * p.ld_x + col]);
        if (p.residual) r[i] = to_float(static_cast<const T *>(p.residual)[row * p.ld_r + col]);
        at_y[i] = row * p.ld_y + col;
    }
    const uint4 w = fields(p, (unsigned long long)(first + lane), call_offset(p));
    uint32_t keep = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) keep |= kept(w, i, p.upper_threshold) ? 1u << i : 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int o = i * 32 + lane;
        const uint32_t bits = __shfl_sync(0xffffffffu, keep, o / 8);
        if (e0 + o >= elements) continue;
        float v = dropped(x[i], (bits >> (o % 8)) & 1u, p.scale);
        if (p.residual) v += r[i];
        static_cast<T *>(p.y)[at_y[i]] = from_float<T>(v);
    }
}

template <typename T> int launch_dropout(const DropoutArgs &p, int dtype, cudaStream_t stream) {
    const long long elements = p.rows * p.cols;
    const bool flat = p.rows == 1 || (p.ld_x == p.cols && p.ld_y == p.cols && (!p.residual || p.ld_r == p.cols));
    const bool starts = rows_aligned16(p.x, 0, dtype) && rows_aligned16(p.y, 0, dtype) && rows_aligned16(p.residual, 0, dtype);
    bool done = false;
    if (flat) {
        if (starts) {
            const long long groups = elements / 8;
            const int rest = (int)(elements % 8);
            const unsigned blocks = (unsigned)(groups / (kThreads * kFlight) + 1);
            if (p.residual) dropout_flat_kernel<T, true><<<blocks, kThreads, 0, stream>>>(p, groups, rest);
            else dropout_flat_kernel<T, false><<<blocks, kThreads, 0, stream>>>(p, groups, rest);
            done = true;
        }
    } else if (starts && p.cols % 8 == 0 && rows_aligned16(p.x, p.ld_x, dtype) && rows_aligned16(p.y, p.ld_y, dtype) &&
               (!p.residual || rows_aligned16(p.residual, p.ld_r, dtype)) && p.cols < (1LL << 31)) {
        const long long per_row = p.cols / 8;
        int log_per_row = 0;
        while (log_per_row < 8 && (1LL << log_per_row) * kFlight < per_row) ++log_per_row;
        const long long col_blocks = (per_row + ((long long)kFlight << log_per_row) - 1) / ((long long)kFlight << log_per_row);
        const long long row_blocks = (p.rows + (kThreads >> log_per_row) - 1) / (kThreads >> log_per_row);
        if (row_blocks * col_blocks < (1LL << 31)) {
            const unsigned blocks = (unsigned)(row_blocks * col_blocks);
            if (p.residual) dropout_rows_kernel<T, true><<<blocks, kThreads, 0, stream>>>(p, log_per_row, (unsigned)col_blocks);
            else dropout_rows_kernel<T, false><<<blocks, kThreads, 0, stream>>>(p, log_per_row, (unsigned)col_blocks);
            done = true;
        }
    }
    DropoutArgs a = p;
    if (flat) { a.rows = 1; a.cols = elements; }
    // Measured, shifted / element by element: 4096 x 33 bf16 with a residual 4.5 / 4.8 us, 8192 x 33 6.6 / 4.8, 8192 x 90 6.7 / 6.0, 8192 x 129
    // fp16 5.6 / 6.8; fp32, 4096 x 4095 with a residual, shifted 39, by segments 31 (the floor).
    const bool few = elements <= kFew;
    if (!done && (few || (sizeof(T) == 2 && a.cols >= kShifted))) {
        const int steps = a.rows * ((a.cols + 7 + 255) / 256) >= 20000 ? kSteps : 1;
        const long long each = 256LL * steps, per_row = (a.cols + 7 + each - 1) / each, parts = per_row * a.rows, blocks = (parts + kThreads / 32 - 1) / (kThreads / 32);
        if (blocks < (1LL << 31)) {
            if (p.residual) dropout_shifted_kernel<T, true><<<(unsigned)blocks, kThreads, 0, stream>>>(a, parts, per_row, steps);
            else dropout_shifted_kernel<T, false><<<(unsigned)blocks, kThreads, 0, stream>>>(a, parts, per_row, steps);
            done = true;
        }
    } else if (!done && sizeof(T) == 4 && a.cols >= kSegment && a.cols < (1LL << 31)) {
        const long long per_row = (a.cols + kSegment - 1) / kSegment, segments = per_row * a.rows, blocks = (segments + kThreads / 32 - 1) / (kThreads / 32);
        if (blocks < (1LL << 31)) {
            dropout_segments_kernel<T><<<(unsigned)blocks, kThreads, 0, stream>>>(a, segments, (unsigned)per_row);
            done = true;
        }
    }
    if (!done) {
        const long long groups = (elements + 7) / 8;
        dropout_elements_kernel<T><<<(unsigned)((groups + kThreads - 1) / kThreads), kThreads, 0, stream>>>(a, elements);
    }
    return launch_status();
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
    const uint32_t threshold = (uint32_t)floor(p * 65536.0 + 0.5);
    a.drop_all = threshold == 65536u;
    a.upper_threshold = a.drop_all ? 1u : threshold << 16;
    a.scale = a.drop_all ? 0.f : (float)(65536.0 / (65536.0 - (double)threshold));
    a.seed = seed; a.offset = offset;
    a.offset_dev = reinterpret_cast<const unsigned long long *>(offset_dev);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return with_dtype(dtype, [&](auto *tag) { return launch_dropout<std::remove_pointer_t<decltype(tag)>>(a, dtype, stream); });
}
