// parle_embedding, parle_embedding_grad: rows of n tables by token, scaled, and the gradient of the tables.
//
//   out[g, t, :] = scale * table[g, token[g, t], :]
//   dtable[g, v, :] = scale * sum over t with token[g, t] = v of dout[g, t, :]      (t in ascending order, fp32)
//
// The gradient is formed by sorted tokens: positions are sorted by (token, position), the sorted sequence is cut into chunks of
// kChunk positions, a block sums the runs of equal tokens in its chunk and writes the rows of those that begin and end there;
// a run that crosses a chunk's border leaves one partial row per chunk, which a second kernel joins.  No floating-point
// atomics: the same inputs give the same bits.
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "token_types.cuh"

using namespace parle;

namespace {

constexpr int kThreads = 256;

// ---- lookup -------------------------------------------------------------------------------------------------------------------

struct LookupArgs {
    const void *table;
    void *out;
    const int32_t *tokens;
    long long table_gs, ld_table, out_gs, ld_out;
    long long length, rows;                              // rows = n * length
    int vocab, dim;
    float scale;
    int32_t *flags;
};

// E elements per access (8: everything on 16-byte boundaries; 1: any pitch and alignment).  `per_row` threads of a block
// (a power of two) share a row.
template <typename TI, typename TO, int E>
__global__ void __launch_bounds__(kThreads) embedding_kernel(const LookupArgs p, int per_row) {
    const int lane = threadIdx.x % per_row;
    const long long row = (long long)blockIdx.x * (kThreads / per_row) + threadIdx.x / per_row;
    if (row >= p.rows) return;
    const int token = p.tokens[row];
    const long long g = row / p.length, t = row - g * p.length;
    TO *out = static_cast<TO *>(p.out) + g * p.out_gs + t * p.ld_out;
    const bool real = token >= 0 && token < p.vocab;
    if (!real && token != PARLE_NO_TOKEN && lane == 0 && p.flags) atomicOr(p.flags, PARLE_FLAG_BAD_LABEL);
    const TI *in = static_cast<const TI *>(p.table) + g * p.table_gs + (real ? (long long)token * p.ld_table : 0);
    const int steps = p.dim / E;
    if constexpr (E == 8) {
        constexpr int U = 2;
        for (int j0 = lane; j0 < steps; j0 += per_row * U) {
            Pack8<TI> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (real && j0 + u * per_row < steps) v[u].load(in + (long long)(j0 + u * per_row) * 8);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * per_row;
                if (j >= steps) break;
                float f[8];
                if (real) {
                    v[u].get(f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] *= p.scale;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = 0.f;
                }
                Pack8<TO> o;
                o.set(f);
                o.store(out + (long long)j * 8);
            }
        }
    } else {
        for (int j = lane; j < steps; j += per_row) out[j] = from_float<TO>(real ? to_float(in[j]) * p.scale : 0.f);
    }
}

int threads_per_row(int steps) {
    int t = 1;
    while (t < steps && t < kThreads) t *= 2;
    return t;
}

// ---- gradient: sorting ---------------------------------------------------------------------------------------------------------

constexpr int kChunk = 32;              // sorted positions a block of the reduction sums
constexpr int kRankedMost = 8192;       // longest sequence ranked by counting
constexpr int kDigits = 256;            // of a radix pass (8 bits)
constexpr int kTile = 4096;             // positions a block of a radix pass moves
constexpr int kSplit = 8;               // threads that share the counting for one position

// A position without a token sorts behind all others: key = vocab.
__device__ __forceinline__ int sort_key(int token, int vocab) { return token >= 0 && token < vocab ? token : vocab; }

__device__ __forceinline__ void note_bad_token(int token, int vocab, int32_t *flags) {
    if (flags && token != PARLE_NO_TOKEN && (token < 0 || token >= vocab)) atomicOr(flags, PARLE_FLAG_BAD_LABEL);
}

// Short sequences: the place of position t in the sorted order is the number of positions s with key(s) < key(t), or equal and
// s < t.  length^2 comparisons, no passes; kSplit threads share one t.
__global__ void __launch_bounds__(kThreads)
rank_tokens_kernel(const int32_t *tokens, int length, int vocab, int *keys, int *places, int32_t *flags) {
    __shared__ int tile[kThreads * 4];
    const int g = blockIdx.y;
    tokens += (long long)g * length;
    const int t = blockIdx.x * (kThreads / kSplit) + threadIdx.x / kSplit, part = threadIdx.x % kSplit;
    const int token = t < length ? tokens[t] : PARLE_NO_TOKEN;
    const int key = sort_key(token, vocab);
    int before = 0;
    for (int s0 = 0; s0 < length; s0 += kThreads * 4) {
        __syncthreads();
        for (int i = threadIdx.x; i < kThreads * 4; i += kThreads) tile[i] = s0 + i < length ? sort_key(tokens[s0 + i], vocab) : INT_MAX;
        __syncthreads();
#pragma unroll 8
        for (int i = part; i < kThreads * 4; i += kSplit) before += tile[i] < key + (s0 + i < t ? 1 : 0);
    }
    for (int o = kSplit / 2; o > 0; o >>= 1) before += __shfl_down_sync(0xffffffffu, before, o, kSplit);
    if (t < length && part == 0) {
        keys[(long long)g * length + before] = key;
        places[(long long)g * length + before] = t;
        note_bad_token(token, vocab, flags);
    }
}

// One pass of a stable radix sort, least significant digit first.  First: how often each digit occurs in a tile.
__global__ void __launch_bounds__(kThreads)
radix_count_kernel(const int32_t *keys, int length, int vocab, int shift, int first_pass, int *counts, int32_t *flags) {
    __shared__ int hist[kDigits];
    const int g = blockIdx.y;
    keys += (long long)g * length;
    hist[threadIdx.x] = 0;
    __syncthreads();
    const long long t0 = (long long)blockIdx.x * kTile;
    for (int i = threadIdx.x; i < kTile && t0 + i < length; i += kThreads) {
        int key = keys[t0 + i];
        if (first_pass) { note_bad_token(key, vocab, flags); key = sort_key(key, vocab); }
        atomicAdd(&hist[(key >> shift) & (kDigits - 1)], 1);
    }
    __syncthreads();
    counts[((long long)g * gridDim.x + blockIdx.x) * kDigits + threadIdx.x] = hist[threadIdx.x];
}

// Then: every position moves to (positions with a lower digit) + (same digit, earlier tile) + (same digit, earlier in the tile).
// A warp owns kTile / 8 consecutive positions and ranks 32 at a time by matching digits.
__global__ void __launch_bounds__(kThreads)
radix_move_kernel(const int32_t *keys, const int *places, int length, int vocab, int shift, int first_pass, const int *counts,
                  int *keys_out, int *places_out) {
    constexpr int kWarps = kThreads / 32;
    __shared__ int warp_count[kWarps][kDigits];
    __shared__ int scan[kWarps];
    const int g = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const long long base = (long long)g * length;
    const int t0 = blockIdx.x * kTile + warp * (kTile / kWarps);
    for (int w = 0; w < kWarps; ++w) warp_count[w][threadIdx.x] = 0;
    __syncthreads();
    auto key_at = [&](int t) { return first_pass ? sort_key(keys[base + t], vocab) : keys[base + t]; };
    for (int i = 0; i < kTile / kWarps; i += 32) {       // how often each digit occurs in the warp's positions
        const int t = t0 + i + lane;
        if (t < length) atomicAdd(&warp_count[warp][(key_at(t) >> shift) & (kDigits - 1)], 1);
    }
    // thread = digit: its total over all tiles, and over the tiles before this one
    int total = 0, earlier = 0;
    const int *c = counts + (long long)g * gridDim.x * kDigits + threadIdx.x;
    for (int b = 0; b < (int)gridDim.x; ++b) {
        const int v = c[(long long)b * kDigits];
        total += v;
        if (b < (int)blockIdx.x) earlier += v;
    }
    int sum = total;                                      // inclusive scan over the digits
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += v;
    }
    if (lane == 31) scan[warp] = sum;
    __syncthreads();                                      // (also: warp_count is complete)
    int start = sum - total + earlier;
    for (int w = 0; w < warp; ++w) start += scan[w];
    for (int w = 0; w < kWarps; ++w) {                    // where each warp's first position with this digit goes
        const int v = warp_count[w][threadIdx.x];
        warp_count[w][threadIdx.x] = start;
        start += v;
    }
    __syncthreads();
    for (int i = 0; i < kTile / kWarps; i += 32) {
        const int t = t0 + i + lane;
        const bool in = t < length;
        const int key = in ? key_at(t) : 0;
        const int digit = in ? (key >> shift) & (kDigits - 1) : kDigits;
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        const int rank = __popc(same & ((1u << lane) - 1u));
        int to = 0;
        if (in) to = warp_count[warp][digit] + rank;
        __syncwarp();
        if (in && rank == 0) warp_count[warp][digit] += __popc(same);
        __syncwarp();
        if (in) {
            keys_out[base + to] = key;
            places_out[base + to] = first_pass ? t : places[base + t];
        }
    }
}

// ---- gradient: sums ------------------------------------------------------------------------------------------------------------

struct GradArgs {
    const void *dout;
    float *dtable;
    const int *keys, *places;                             // sorted
    float *partial;                                       // [n][chunks][2][dim]: a chunk's first run (if it began before), last run (if it goes on)
    long long dout_gs, ld_dout, dtable_gs, ld_dtable;
    int length, vocab, dim, chunks;
    float scale;
    int accumulate;
};

// E columns; E == 8: on a 16-byte boundary.
template <int E> __device__ __forceinline__ void store_columns(float *to, const float (&v)[E]) {
    if constexpr (E == 8) {
        Pack8<float> p;
        p.set(v);
        p.store(to);
    } else {
        to[0] = v[0];
    }
}

// Sum of one run's rows inside a chunk and where it goes.  E columns per thread; grid (chunks, column tiles, n).
template <typename T, int E>
__global__ void __launch_bounds__(kThreads) embedding_grad_kernel(const GradArgs p) {
    __shared__ int key[kChunk + 2], place[kChunk];        // key[0]: the position before the chunk, key[kChunk + 1]: the one after
    const int g = blockIdx.z, chunk = blockIdx.x;
    const int first = chunk * kChunk, count = min(kChunk, p.length - first);
    if (threadIdx.x < kChunk + 2) {
        const int s = first + (int)threadIdx.x - 1;
        key[threadIdx.x] = s >= 0 && s < p.length ? p.keys[(long long)g * p.length + s] : -1;
    }
    if (threadIdx.x < count) place[threadIdx.x] = p.places[(long long)g * p.length + first + threadIdx.x];
    __syncthreads();
    const int col = (blockIdx.y * kThreads + threadIdx.x) * E;
    if (col >= p.dim) return;
    const T *dout = static_cast<const T *>(p.dout) + (long long)g * p.dout_gs + col;
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    int run = 0;                                          // where the current run begins in the chunk
    constexpr int U = 8;
    for (int i0 = 0; i0 < count; i0 += U) {
        float v[U][E];
        if constexpr (E == 8) {
            Pack8<T> raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u < count && key[i0 + u + 1] < p.vocab) raw[u].load(dout + (long long)place[i0 + u] * p.ld_dout);
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u].get(v[u]);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u < count && key[i0 + u + 1] < p.vocab) v[u][0] = to_float(dout[(long long)place[i0 + u] * p.ld_dout]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u;
            if (i >= count) break;
            const int k = key[i + 1];
            if (k >= p.vocab) return;                     // the rest has no token
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += v[u][e];
            if (i + 1 < count && key[i + 2] == k) continue;
            // the run's last position in this chunk
            const bool before = run == 0 && key[0] == k, after = i + 1 == count && key[i + 2] == k;
            if (before || after) {
                // (a run that fills the chunk and goes on both ways counts as "began before")
                store_columns<E>(p.partial + (((long long)g * p.chunks + chunk) * 2 + (before ? 0 : 1)) * p.dim + col, acc);
            } else {
                float *to = p.dtable + (long long)g * p.dtable_gs + (long long)k * p.ld_dtable + col;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = p.accumulate ? fmaf(p.scale, acc[e], to[e]) : p.scale * acc[e];
                store_columns<E>(to, acc);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = 0.f;
            run = i + 1;
        }
    }
}

// Runs that cross a border: the block of the chunk in which such a run begins adds up its partial rows.  32 columns per block
// and step; the eight warps take an eighth of the partial rows each, in order, and their sums are added in order.
__global__ void __launch_bounds__(kThreads) embedding_grad_join_kernel(const GradArgs p) {
    constexpr int kWarps = kThreads / 32;
    __shared__ float sums[kWarps][32];
    __shared__ int end_of_run;
    const int g = blockIdx.z, chunk = blockIdx.x, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int *keys = p.keys + (long long)g * p.length;
    const int first = chunk * kChunk, next = first + kChunk;
    if (next >= p.length) return;
    const int k = keys[next - 1];
    if (k >= p.vocab || keys[next] != k) return;          // no run crosses the border behind this chunk
    if (first > 0 && keys[first - 1] == k) return;        // it began in an earlier one
    if (threadIdx.x == 0) end_of_run = p.chunks;
    __syncthreads();
    for (int c0 = chunk + 1; c0 < p.chunks; c0 += kThreads) {     // first chunk that begins with another token
        const int c = c0 + threadIdx.x;
        const bool other = c < p.chunks && keys[(long long)c * kChunk] != k;
        if (other) atomicMin(&end_of_run, c);
        if (__syncthreads_or(other)) break;
    }
    __syncthreads();
    const int parts = end_of_run - chunk;                 // this chunk's last run, then the first runs of the following chunks
    const int per_warp = (parts + kWarps - 1) / kWarps;
    const float *partial = p.partial + ((long long)g * p.chunks + chunk) * 2 * p.dim;
    for (int c0 = blockIdx.y * 32; c0 < p.dim; c0 += gridDim.y * 32) {
        const int col = c0 + lane;
        float s = 0.f;
        if (col < p.dim) {
            const int to = min(parts, (warp + 1) * per_warp);
#pragma unroll 8
            for (int i = warp * per_warp; i < to; ++i) s += partial[((long long)i * 2 + (i == 0 ? 1 : 0)) * p.dim + col];
        }
        sums[warp][lane] = s;
        __syncthreads();
        if (warp == 0 && col < p.dim) {
            for (int w = 1; w < kWarps; ++w) s += sums[w][lane];
            float *to = p.dtable + (long long)g * p.dtable_gs + (long long)k * p.ld_dtable + col;
            *to = p.accumulate ? fmaf(p.scale, s, *to) : p.scale * s;
        }
        __syncthreads();
    }
}

// Rows of tokens that do not occur: zero.  A block takes kZeroRows rows and finds their tokens in the sorted keys.
constexpr int kZeroRows = 32;
template <int E>
__global__ void __launch_bounds__(kThreads) embedding_grad_zero_kernel(const GradArgs p) {
    __shared__ uint32_t present;
    const int g = blockIdx.y, v0 = blockIdx.x * kZeroRows;
    const int *keys = p.keys + (long long)g * p.length;
    if (threadIdx.x == 0) present = 0;
    __syncthreads();
    int lo = 0, hi = p.length;                            // first sorted position with a key >= v0
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (keys[mid] < v0) lo = mid + 1; else hi = mid;
    }
    const int limit = min(v0 + kZeroRows, p.vocab);
    for (int s = lo;; s += kThreads) {
        const int k = s + (int)threadIdx.x < p.length ? keys[s + threadIdx.x] : p.vocab;
        if (k < limit) atomicOr(&present, 1u << (k - v0));
        if (!__syncthreads_and(k < limit)) break;
    }
    for (int r = 0; r < limit - v0; ++r) {
        if ((present >> r) & 1u) continue;
        float *row = p.dtable + (long long)g * p.dtable_gs + (long long)(v0 + r) * p.ld_dtable;
        for (int j = threadIdx.x * E; j < p.dim; j += kThreads * E) {
            if constexpr (E == 4) *reinterpret_cast<float4 *>(row + j) = make_float4(0.f, 0.f, 0.f, 0.f);
            else row[j] = 0.f;
        }
    }
}

// ---- workspace -----------------------------------------------------------------------------------------------------------------

struct GradPlan {
    int chunks, tiles, passes;
    size_t keys[2], places[2], counts, partial, bytes;
};

GradPlan plan_grad(int n, long long length, int vocab, int dim) {
    GradPlan p = {};
    p.chunks = (int)((length + kChunk - 1) / kChunk);
    const size_t ints = round_up((size_t)n * length * sizeof(int), 128);
    if (length > kRankedMost) {
        p.tiles = (int)((length + kTile - 1) / kTile);
        int bits = 1;
        while (bits < 31 && (vocab >> bits)) ++bits;      // keys 0 .. vocab
        p.passes = (bits + 7) / 8;
    }
    size_t at = 0;
    for (int i = 0; i < (p.passes ? 2 : 1); ++i) { p.keys[i] = at; at += ints; p.places[i] = at; at += ints; }
    p.counts = at;
    at += round_up((size_t)n * p.tiles * kDigits * sizeof(int), 128);
    p.partial = at;
    at += round_up((size_t)n * p.chunks * 2 * dim * sizeof(float), 128);
    p.bytes = at;
    return p;
}

bool valid_sizes(int n, long long length, int vocab, int dim) {
    return n >= 1 && n <= PARLE_MAX_REPLICAS && length >= 0 && vocab >= 1 && dim >= 1;
}

// Whether n groups of `rows` rows of dim elements, at these pitches, do not overlap: group after group, or row by row with the
// groups side by side.
bool separate_rows(int n, long long rows, int dim, long long gs, long long ld) {
    if (ld < dim && rows > 1) return false;
    if (n == 1) return true;
    return gs >= dim && (rows <= 1 || gs / ld >= rows || (gs / ld == rows - 1 && gs % ld >= dim) || ld / gs >= n || (ld / gs == n - 1 && ld % gs >= dim));
}

}  // namespace

extern "C" int parle_embedding(const void *table, int table_dtype, long long table_gs, long long ld_table, int n, int vocab, int dim,
                               const int32_t *tokens, long long length, double scale, void *out, int out_dtype,
                               long long out_gs, long long ld_out, int32_t *flags, void *cuda_stream) {
    if (!valid_sizes(n, length, vocab, dim) || !valid_dtype(table_dtype) || !valid_dtype(out_dtype) || !isfinite((float)scale)) return PARLE_EINVAL;
    if (length > PARLE_TOKEN_MAX_ROWS / n) return PARLE_ETOOBIG;
    if (ld_table < 0 || (n > 1 && table_gs < 0) || !separate_rows(n, length, dim, out_gs, ld_out)) return PARLE_EINVAL;
    if (length == 0) return PARLE_OK;
    if (!table || !tokens || !out) return PARLE_EINVAL;
    if (!element_aligned(table, table_dtype) || !element_aligned(out, out_dtype) || !element_aligned(tokens, PARLE_F32) ||
        !element_aligned(flags, PARLE_F32)) return PARLE_EALIGN;
    LookupArgs a = {};
    a.table = table; a.out = out; a.tokens = tokens; a.flags = flags;
    a.table_gs = table_gs; a.ld_table = ld_table; a.out_gs = out_gs; a.ld_out = ld_out;
    a.length = length; a.rows = (long long)n * length;
    a.vocab = vocab; a.dim = dim; a.scale = (float)scale;
    const bool wide = dim % 8 == 0 && rows_aligned16(table, ld_table, table_dtype) && rows_aligned16(out, ld_out, out_dtype) &&
                      (n == 1 || (rows_aligned16(table, table_gs, table_dtype) && rows_aligned16(out, out_gs, out_dtype)));
    const int per_row = threads_per_row(wide ? dim / 8 : dim);
    const long long rows_per_block = kThreads / per_row;
    const unsigned blocks = (unsigned)((a.rows + rows_per_block - 1) / rows_per_block);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return with_dtype(table_dtype, [&](auto *ti) {
        return with_dtype(out_dtype, [&](auto *to) {
            using TI = std::remove_pointer_t<decltype(ti)>;
            using TO = std::remove_pointer_t<decltype(to)>;
            if (wide) embedding_kernel<TI, TO, 8><<<blocks, kThreads, 0, stream>>>(a, per_row);
            else embedding_kernel<TI, TO, 1><<<blocks, kThreads, 0, stream>>>(a, per_row);
            return launch_status();
        });
    });
}

extern "C" size_t parle_embedding_grad_workspace_bytes(int n, long long length, int vocab, int dim) {
    if (!valid_sizes(n, length, vocab, dim) || length > PARLE_TOKEN_MAX_ROWS / n) return 0;
    return plan_grad(n, length, vocab, dim).bytes;
}

extern "C" int parle_embedding_grad(const void *dout, int dout_dtype, long long dout_gs, long long ld_dout, const int32_t *tokens,
                                    int n, long long length, int vocab, int dim, double scale, float *dtable, long long dtable_gs,
                                    long long ld_dtable, int accumulate, void *workspace, size_t workspace_bytes, int32_t *flags,
                                    void *cuda_stream) {
    if (!valid_sizes(n, length, vocab, dim) || !valid_dtype(dout_dtype) || !isfinite((float)scale)) return PARLE_EINVAL;
    if (length > PARLE_TOKEN_MAX_ROWS / n) return PARLE_ETOOBIG;
    if (ld_dout < 0 || (n > 1 && dout_gs < 0) || !separate_rows(n, vocab, dim, dtable_gs, ld_dtable) || !dtable) return PARLE_EINVAL;
    if (length > 0 && (!dout || !tokens || !workspace)) return PARLE_EINVAL;
    if (!element_aligned(dout, dout_dtype) || !element_aligned(dtable, PARLE_F32) || !element_aligned(tokens, PARLE_F32) ||
        !element_aligned(flags, PARLE_F32) || reinterpret_cast<uintptr_t>(workspace) % 128) return PARLE_EALIGN;
    const GradPlan plan = plan_grad(n, length, vocab, dim);
    if (workspace_bytes < plan.bytes) return PARLE_EWORKSPACE;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    char *ws = static_cast<char *>(workspace);
    int *keys[2], *places[2];
    for (int i = 0; i < 2; ++i) {
        keys[i] = reinterpret_cast<int *>(ws + plan.keys[i]);
        places[i] = reinterpret_cast<int *>(ws + plan.places[i]);
    }
    int sorted = 0, rc = PARLE_OK;
    const int T = (int)length;
    if (plan.passes) {
        int *counts = reinterpret_cast<int *>(ws + plan.counts);
        const dim3 grid(plan.tiles, n);
        for (int pass = 0; pass < plan.passes; ++pass) {
            const int32_t *in = pass ? keys[sorted] : tokens;
            const int to = pass ? 1 - sorted : 0;
            radix_count_kernel<<<grid, kThreads, 0, stream>>>(in, T, vocab, 8 * pass, pass == 0, counts, flags);
            if ((rc = launch_status()) != PARLE_OK) return rc;
            radix_move_kernel<<<grid, kThreads, 0, stream>>>(in, places[sorted], T, vocab, 8 * pass, pass == 0, counts, keys[to], places[to]);
            if ((rc = launch_status()) != PARLE_OK) return rc;
            sorted = to;
        }
    } else if (T > 0) {
        const int per_block = kThreads / kSplit;
        rank_tokens_kernel<<<dim3((T + per_block - 1) / per_block, n), kThreads, 0, stream>>>(tokens, T, vocab, keys[0], places[0], flags);
        if ((rc = launch_status()) != PARLE_OK) return rc;
    }
    GradArgs a = {};
    a.dout = dout; a.dtable = dtable; a.keys = keys[sorted]; a.places = places[sorted];
    a.partial = reinterpret_cast<float *>(ws + plan.partial);
    a.dout_gs = dout_gs; a.ld_dout = ld_dout; a.dtable_gs = dtable_gs; a.ld_dtable = ld_dtable;
    a.length = T; a.vocab = vocab; a.dim = dim; a.chunks = plan.chunks;
    a.scale = (float)scale; a.accumulate = accumulate != 0;
    const bool wide_table = dim % 4 == 0 && rows_aligned16(dtable, ld_dtable, PARLE_F32) && (n == 1 || dtable_gs % 4 == 0);
    if (!accumulate) {
        const dim3 grid((unsigned)(((long long)vocab + kZeroRows - 1) / kZeroRows), n);
        if (wide_table)
            embedding_grad_zero_kernel<4><<<grid, kThreads, 0, stream>>>(a);
        else embedding_grad_zero_kernel<1><<<grid, kThreads, 0, stream>>>(a);
        if ((rc = launch_status()) != PARLE_OK) return rc;
    }
    if (T == 0) return PARLE_OK;
    const bool wide = wide_table && dim % 8 == 0 && rows_aligned16(dout, ld_dout, dout_dtype) && (n == 1 || rows_aligned16(dout, dout_gs, dout_dtype));
    const int columns = wide ? kThreads * 8 : kThreads;
    const dim3 grid(plan.chunks, (dim + columns - 1) / columns, n);
    rc = with_dtype(dout_dtype, [&](auto *tag) {
        using TD = std::remove_pointer_t<decltype(tag)>;
        if (wide) embedding_grad_kernel<TD, 8><<<grid, kThreads, 0, stream>>>(a);
        else embedding_grad_kernel<TD, 1><<<grid, kThreads, 0, stream>>>(a);
        return launch_status();
    });
    if (rc != PARLE_OK || plan.chunks < 2) return rc;
    embedding_grad_join_kernel<<<dim3(plan.chunks - 1, (dim + 511) / 512, n), kThreads, 0, stream>>>(a);
    return launch_status();
}
