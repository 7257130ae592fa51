// parle_embedding, parle_embedding_grad: rows of n tables by token, scaled, and the gradient of the tables.
//
//   out[g, t, :] = scale * table[g, token[g, t], :]
//   dtable[g, v, :] = scale * sum over t with token[g, t] = v of dout[g, t, :]      (fp32)
//
// No floating-point atomics: the same inputs give the same bits.  The positions of a token are cut into runs by the tokens alone (not by
// dim, pitches or types); a run's rows are added in ascending order, then the runs' sums in theirs.  Two ways to the gradient:
//
// Up to kDirectMost positions ("direct", one launch, no workspace): a block takes a set of table rows, looks through all the
// tokens, notes for each of its rows the positions that hold its token, puts them in order and sums.
//
// More positions ("sorted"): the positions are sorted by (token, position), up to kRankedMost by counting, up to kSortMost in the shared
// memory of a cluster, beyond by launches of their own.  The sorted sequence is then cut into chunks of kChunk positions; a block sums the runs of equal tokens in its chunk and writes the rows of
// those that begin and end there, while other blocks write zeros to the rows of tokens that do not occur.  A run that crosses a
// chunk's border leaves one partial row per chunk, which a last kernel joins.  Work is shared out by position, so it does not
// matter how often which token occurs.
#include <limits.h>
#include <math.h>

#include <algorithm>
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
    long long length;
    int vocab, dim;
    float scale;
    int32_t *flags;
};

// E elements per access (8: everything on 16-byte boundaries; 1: any pitch and alignment).  1 << log_per_row threads of a block share a
// row; a thread has R rows and U accesses of each in flight, R U = 4: long rows U = 4, short ones R = 4.  grid (rows, n).
template <typename TI, typename TO, int E, int R>
__global__ void __launch_bounds__(kThreads) embedding_kernel(const LookupArgs p, int log_per_row) {
    constexpr int U = 4 / R;
    const int per_row = 1 << log_per_row, lane = threadIdx.x & (per_row - 1), slots = kThreads >> log_per_row;
    const long long row0 = (long long)blockIdx.x * (slots * R) + (threadIdx.x >> log_per_row);
    const int32_t *tokens = p.tokens + blockIdx.y * p.length;
    const TI *table = static_cast<const TI *>(p.table) + blockIdx.y * p.table_gs;
    TO *out = static_cast<TO *>(p.out) + blockIdx.y * p.out_gs;
    int token[R];
    bool real[R];
#pragma unroll
    for (int r = 0; r < R; ++r) token[r] = row0 + r * slots < p.length ? tokens[row0 + r * slots] : PARLE_NO_TOKEN;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        real[r] = (unsigned)token[r] < (unsigned)p.vocab;
        if (!real[r] && token[r] != PARLE_NO_TOKEN && lane == 0 && p.flags) atomicOr(p.flags, PARLE_FLAG_BAD_LABEL);
    }
    const int steps = p.dim / E;
    for (int c0 = lane; c0 < steps; c0 += per_row * U) {
        std::conditional_t<E == 8, Pack8<TI>, TI> v[R][U];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const TI *from = table + (real[r] ? token[r] * p.ld_table : 0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * per_row;
                if (!real[r] || c >= steps) continue;
                if constexpr (E == 8) v[r][u].load(from + (long long)c * 8); else v[r][u] = from[c];
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (row0 + r * slots >= p.length) break;
            TO *to = out + (row0 + r * slots) * p.ld_out;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * per_row;
                if (c >= steps) break;
                float f[E];
                if constexpr (E == 8) v[r][u].get(f); else f[0] = to_float(v[r][u]);
#pragma unroll
                for (int i = 0; i < E; ++i) f[i] = real[r] ? f[i] * p.scale : 0.f;
                if constexpr (E == 8) {
                    Pack8<TO> o;
                    o.set(f);
                    o.store(to + (long long)c * 8);
                } else {
                    to[c] = from_float<TO>(f[0]);
                }
            }
        }
    }
}

// Threads for a row: up to 64, so that a thread has several accesses of a long row in flight; more where there are few rows.
// (16384 rows of 4096 bf16: 64 threads 35 us, 256 threads 39 us; 65536 rows of 512: four rows a thread 27 us, one 31 us.)
template <typename TI, typename TO, int E> int launch_lookup(const LookupArgs &a, int n, int sms, cudaStream_t stream) {
    const int steps = a.dim / E;
    int log_per_row = 0;
    while (log_per_row < 6 && (1 << log_per_row) < steps) ++log_per_row;
    int rows_each = steps <= (1 << log_per_row) ? 4 : steps <= (2 << log_per_row) ? 2 : 1;
    const auto blocks = [&] { return (a.length + (kThreads >> log_per_row) * rows_each - 1) / ((kThreads >> log_per_row) * rows_each); };
    if (blocks() * n < 2 * sms) {
        rows_each = 1;
        while (log_per_row < 8 && (1 << log_per_row) < steps && blocks() * n < 2 * sms) ++log_per_row;
    }
    const dim3 grid((unsigned)blocks(), n);
    if (rows_each == 4) embedding_kernel<TI, TO, E, 4><<<grid, kThreads, 0, stream>>>(a, log_per_row);
    else if (rows_each == 2) embedding_kernel<TI, TO, E, 2><<<grid, kThreads, 0, stream>>>(a, log_per_row);
    else embedding_kernel<TI, TO, E, 1><<<grid, kThreads, 0, stream>>>(a, log_per_row);
    return launch_status();
}

// ---- gradient --------------------------------------------------------------------------------------------------------------------

struct GradArgs {
    const void *dout;
    float *dtable;
    const int32_t *tokens;
    int32_t *flags;
    const int *keys, *places;                             // sorted
    float *partial;                                       // [n][chunks][2][dim]: a chunk's first run (if it began before), last run (if it goes on)
    uint32_t *occurs;                                     // [n][words]: bit v of a table: token v occurs
    int words;
    int *crossings;                                       // how many runs cross a border, then (table, chunk in which it begins, token, -) of each
    long long dout_gs, ld_dout, dtable_gs, ld_dtable;
    int length, vocab, dim, chunks;
    float scale;
    int accumulate;
};

__device__ __forceinline__ void note_bad_token(int token, int vocab, int32_t *flags) {
    if (flags && token != PARLE_NO_TOKEN && (token < 0 || token >= vocab)) atomicOr(flags, PARLE_FLAG_BAD_LABEL);
}

// ---- direct gradient -------------------------------------------------------------------------------------------------------------

constexpr int kDirectMost = 1024;       // longest sequence
constexpr int kNoted = 16;              // positions of a row that are noted
constexpr int kRowsMost = 64;           // table rows of a block
constexpr int kColumns = 512;           // columns of a block
constexpr int kWarps = kThreads / 32;
constexpr int kSegments = 8;            // of the positions, for a frequent token: its sum is the sum of theirs, in order, at any width

// Eight columns of a lane out of 256 from `first` on: eight neighbours by wide loads (E = 8), or every 32nd (E = 1).
template <typename T, int E> struct Lane8 {
    Pack8<T> raw;
    T one[E == 1 ? 8 : 1];
    __device__ __forceinline__ static int column(int first, int k) { return E == 8 ? first + ((int)threadIdx.x % 32) * 8 + k : first + k * 32 + (int)threadIdx.x % 32; }
    __device__ __forceinline__ void load(const T *row, int first, int dim) {
        if constexpr (E == 8) {
            if (column(first, 0) < dim) raw.load(row + column(first, 0));
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (column(first, k) < dim) one[k] = row[column(first, k)];
        }
    }
    __device__ __forceinline__ void add_to(float (&acc)[8]) const {
        float v[8];
        if constexpr (E == 8) {
            raw.get(v);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = to_float(one[k]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] += v[k];
    }
};

template <int E> __device__ __forceinline__ void store_row(const GradArgs &p, float *row, int first, float (&acc)[8]) {
    if constexpr (E == 8) {
        const int c = Lane8<float, 8>::column(first, 0);
        if (c >= p.dim) return;
        if (p.accumulate) {
            Pack8<float> old;
            float v[8];
            old.load(row + c);
            old.get(v);
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[k] = fmaf(p.scale, acc[k], v[k]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[k] *= p.scale;
        }
        Pack8<float> out;
        out.set(acc);
        out.store(row + c);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = Lane8<float, 1>::column(first, k);
            if (c < p.dim) row[c] = p.accumulate ? fmaf(p.scale, acc[k], row[c]) : p.scale * acc[k];
        }
    }
}

// grid (G, column parts, n); block b has the table rows v with v mod G = b, so that neighbouring tokens, which are often frequent
// together, fall to different blocks.
template <typename T, int E>
__global__ void __launch_bounds__(kThreads, 4) embedding_grad_direct_kernel(const GradArgs p, int log_groups) {
    __shared__ int count[kRowsMost], frequent[kRowsMost], frequents;
    __shared__ int noted[kRowsMost][kNoted];
    __shared__ float parts[kSegments * kColumns];         // of a frequent token's row
    const int g = blockIdx.z, b = blockIdx.x, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int col0 = blockIdx.y * kColumns, groups = 1 << log_groups;
    const int rows = (p.vocab - b + groups - 1) >> log_groups;
    const int32_t *tokens = p.tokens + (long long)g * p.length;
    const T *dout = static_cast<const T *>(p.dout) + (long long)g * p.dout_gs;
    float *dtable = p.dtable + (long long)g * p.dtable_gs;
    if (threadIdx.x < kRowsMost) count[threadIdx.x] = 0;
    if (threadIdx.x == 0) frequents = 0;
    int token[kDirectMost / kThreads];
#pragma unroll
    for (int u = 0; u < kDirectMost / kThreads; ++u) {
        const int t = threadIdx.x + u * kThreads;
        token[u] = t < p.length ? tokens[t] : PARLE_NO_TOKEN;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kDirectMost / kThreads; ++u) {
        if (b == 0 && blockIdx.y == 0) note_bad_token(token[u], p.vocab, p.flags);
        if ((token[u] & (groups - 1)) != b || (unsigned)token[u] >= (unsigned)p.vocab) continue;
        const int row = token[u] >> log_groups, at = atomicAdd(&count[row], 1);
        if (at < kNoted) noted[row][at] = threadIdx.x + u * kThreads;
    }
    __syncthreads();
    // a warp per row and 256 columns
    const int halves = p.dim - col0 > 256 ? 2 : 1;
    for (int item = warp; item < rows * halves; item += kWarps) {
        const int i = halves == 2 ? item / 2 : item, first = col0 + (halves == 2 ? item % 2 * 256 : 0);
        const int m = count[i];
        float *row = dtable + (long long)((i << log_groups) + b) * p.ld_dtable;
        if (m == 0) {
            if (p.accumulate) continue;
            const int end = min(p.dim, first + 256);
            if constexpr (E == 8) {
                for (int c = first + lane * 4; c < end; c += 128) *reinterpret_cast<float4 *>(row + c) = make_float4(0.f, 0.f, 0.f, 0.f);
            } else {
                for (int c = first + lane; c < end; c += 32) row[c] = 0.f;
            }
            continue;
        }
        if (m > kNoted) {
            if (lane == 0 && first == col0) frequent[atomicAdd(&frequents, 1)] = i;
            continue;
        }
        // the noted positions in ascending order: one per lane, fetched from the lane with that many smaller ones
        int place = lane < m ? noted[i][lane] : INT_MAX;
        if (m > 1) {
            int smaller = lane < m ? 0 : lane, from = 0;
            for (int j = 0; j < m; ++j) {                 // (every lane takes part in the exchanges)
                const int other = __shfl_sync(0xffffffffu, place, j);
                if (lane < m && other < place) ++smaller;
            }
            for (int j = 0; j < 32; ++j) {
                const int s = __shfl_sync(0xffffffffu, smaller, j);
                if (s == lane) from = j;
            }
            place = __shfl_sync(0xffffffffu, place, from);
        }
        float acc[8] = {};
        for (int j = 0; j < m; j += 4) {
            Lane8<T, E> v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int at = __shfl_sync(0xffffffffu, place, min(j + u, m - 1));
                if (j + u < m) v[u].load(dout + (long long)at * p.ld_dout, first, p.dim);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j + u < m) v[u].add_to(acc);
        }
        store_row<E>(p, row, first, acc);
    }
    // rows of frequent tokens: all warps, side by side if there are columns for two, along the positions.  Then a warp has
    // two neighbouring segments, in one walk (1024 positions of four tokens, 512 columns: 44 us; in two loops 68).  The segments' parts
    // are added in order
    __syncthreads();
    const int first = warp % halves * 256, per_segment = (p.length + kSegments - 1) / kSegments, segment = warp / halves * halves;
    const int from = min(p.length, segment * per_segment), to = min(p.length, from + halves * per_segment);
    const int border = halves == 2 ? min(to, from + per_segment) : -1;      // of a warp's two segments
    for (int f = 0; f < frequents; ++f) {
        const int v = (frequent[f] << log_groups) + b;
        float acc[8] = {};
        const auto put = [&](int segment) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                parts[segment * kColumns + Lane8<T, E>::column(first, k)] = acc[k];
                acc[k] = 0.f;
            }
        };
        for (int t0 = from, next; t0 < to; t0 = next) {
            next = min(t0 + 32, t0 < border ? border : to);
            unsigned found = __ballot_sync(0xffffffffu, t0 + lane < next && tokens[t0 + lane] == v);
            while (found) {
                Lane8<T, E> x[4];
                int many = 0;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (!found) break;
                    x[u].load(dout + (long long)(t0 + __ffs(found) - 1) * p.ld_dout, col0 + first, p.dim);
                    found &= found - 1;
                    ++many;
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (u < many) x[u].add_to(acc);
            }
            if (next == border) put(segment);
        }
        if (halves == 2 && from == to) put(segment);
        put(segment + halves - 1);
        __syncthreads();
        float *row = dtable + (long long)v * p.ld_dtable;
        for (int c = threadIdx.x; c < halves * 256 && col0 + c < p.dim; c += kThreads) {
            float sum = parts[c];
            for (int s = 1; s < kSegments; ++s) sum += parts[s * kColumns + c];
            row[col0 + c] = p.accumulate ? fmaf(p.scale, sum, row[col0 + c]) : p.scale * sum;
        }
        __syncthreads();
    }
}

// ---- sorted gradient: the sort ---------------------------------------------------------------------------------------------------------

constexpr int kChunk = 32;              // sorted positions a block of the reduction sums
constexpr int kDigits = 256;            // of a radix pass (8 bits)
constexpr int kTile = 4096;             // positions a block of a radix pass moves

// Notes which tokens occur, by one lane for all lanes of the warp with the same key.  By whole warps; a lane without a position
// brings the key INT_MAX.
__device__ __forceinline__ void note_occurs(const GradArgs &p, int g, int key) {
    const unsigned same = __match_any_sync(0xffffffffu, key);
    if (key < p.vocab && __ffs(same) - 1 == (int)threadIdx.x % 32) atomicOr(p.occurs + (long long)g * p.words + key / 32, 1u << (key % 32));
}

// A position without a token sorts behind all others: key = vocab.
__device__ __forceinline__ int sort_key(int token, int vocab) { return token >= 0 && token < vocab ? token : vocab; }

// The kernels of one call are chained: the next one's blocks may be set up while one runs, and wait here for all of its results.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void await_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

constexpr int kRankedMost = 4096;       // longest sequence ranked by counting
constexpr int kSplit = 8;               // threads that share the counting for one position
constexpr int kWordsMost = 1024;        // words of the bits of tokens that occur, for a block

// Shorter sequences: the place of position t in the sorted order is the number of positions s with key(s) < key(t), or equal and
// s < t: length^2 comparisons, but no passes (5.6 us at 2048 positions where the cluster's sort takes 9.6; 17 against 11 at 8192).  As every block
// sees all tokens, each writes a part of the bits of the tokens that occur.
__global__ void __launch_bounds__(kThreads) rank_tokens_kernel(const GradArgs p, int words_each, int *keys, int *places) {
    constexpr int kTileKeys = kThreads * 4;
    __shared__ int4 tile[kThreads];
    __shared__ uint32_t occurs[kWordsMost];
    const int g = blockIdx.y, word0 = blockIdx.x * words_each;
    const int32_t *tokens = p.tokens + (long long)g * p.length;
    const int first = blockIdx.x * (kThreads / kSplit), t = first + threadIdx.x / kSplit, part = threadIdx.x % kSplit;
    let_next_start();
    if (blockIdx.x == 0 && g == 0 && threadIdx.x == 0) *p.crossings = 0;
    for (int w = threadIdx.x; w < words_each; w += kThreads) occurs[w] = 0;
    const int token = t < p.length ? tokens[t] : PARLE_NO_TOKEN, key = sort_key(token, p.vocab);
    int before = 0;
    for (int s0 = 0; s0 < p.length; s0 += kTileKeys) {
        int4 k;
        int *e = &k.x;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int s = s0 + (int)threadIdx.x * 4 + u;
            e[u] = s < p.length ? sort_key(tokens[s], p.vocab) : INT_MAX;
        }
        __syncthreads();
        tile[threadIdx.x] = k;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const unsigned w = (unsigned)(e[u] / 32 - word0);
            if (e[u] < p.vocab && w < (unsigned)words_each) atomicOr(&occurs[w], 1u << (e[u] % 32));
        }
        __syncthreads();
        if (s0 + kTileKeys <= first || s0 >= first + kThreads / kSplit) {         // altogether before, or behind, the block's positions
            const int limit = key + (s0 < first ? 1 : 0);
#pragma unroll 8
            for (int i = part; i < kThreads; i += kSplit) {
                const int4 v = tile[i];
                before += (v.x < limit) + (v.y < limit) + (v.z < limit) + (v.w < limit);
            }
        } else {
            for (int i = part; i < kThreads; i += kSplit) {
                const int4 v = tile[i];
                const int s = s0 + 4 * i;
                before += (v.x < key + (s < t)) + (v.y < key + (s + 1 < t)) + (v.z < key + (s + 2 < t)) + (v.w < key + (s + 3 < t));
            }
        }
    }
#pragma unroll
    for (int o = kSplit / 2; o > 0; o >>= 1) before += __shfl_down_sync(0xffffffffu, before, o, kSplit);
    if (t < p.length && part == 0) {
        keys[(long long)g * p.length + before] = key;
        places[(long long)g * p.length + before] = t;
        note_bad_token(token, p.vocab, p.flags);
    }
    for (int w = threadIdx.x; w < words_each && word0 + w < p.words; w += kThreads) p.occurs[(long long)g * p.words + word0 + w] = occurs[w];
}

constexpr int kSortThreads = 512, kSorters = 8;          // a cluster sorts up to
constexpr int kSortEach = 4096, kSortMost = kSorters * kSortEach;
constexpr int kSortBits = 9;            // of a pass at most: a thread per digit

// A cluster sorts a sequence: a stable radix sort, least significant digit first, every block with an eighth of the sequence in
// shared memory.  A position goes to (positions with a lower digit) + (same digit, in an earlier block, warp, or place of the warp).
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const GradArgs p, int passes, int bits, int *keys_out, int *places_out) {
    constexpr int W = kSortThreads / 32, D = 1 << kSortBits;
    static_assert(D == kSortThreads, "a thread per digit");
    extern __shared__ int2 items[];                       // [2][kSortEach]: (key, position)
    __shared__ int warp_count[W][D], block_count[D], scan[W];
    const int cluster = blockIdx.x / kSorters, rank = cluster_rank(), lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    let_next_start();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.crossings = 0;
    const int32_t *tokens = p.tokens + (long long)cluster * p.length;
    const int each = (p.length + kSorters - 1) / kSorters, each_warp = (each + W - 1) / W;
    const int mine = max(0, min(each, p.length - rank * each));
    for (int i0 = threadIdx.x; i0 < mine; i0 += kSortThreads * 4) {
        int token[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) token[u] = i0 + u * kSortThreads < mine ? tokens[rank * each + i0 + u * kSortThreads] : 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + u * kSortThreads;
            if (i >= mine) break;
            note_bad_token(token[u], p.vocab, p.flags);
            items[i] = make_int2(sort_key(token[u], p.vocab), rank * each + i);
        }
    }
    uint32_t *const occurs = p.occurs + (long long)cluster * p.words;
    for (int w = rank * kSortThreads + threadIdx.x; w < p.words; w += kSorters * kSortThreads) occurs[w] = 0;
    const int mask = (1 << bits) - 1;
    for (int pass = 0; pass < passes; ++pass) {
        const int2 *in = items + (pass & 1) * kSortEach;
        int2 *out = items + (1 - (pass & 1)) * kSortEach;
#pragma unroll
        for (int w = 0; w < W; ++w) warp_count[w][threadIdx.x] = 0;
        __syncthreads();
        const int from = min(mine, warp * each_warp), to = min(mine, from + each_warp);
        for (int i = from + lane; i < to; i += 32) atomicAdd(&warp_count[warp][(in[i].x >> (bits * pass)) & mask], 1);
        __syncthreads();
        int count[W], own = 0;                            // thread = digit
#pragma unroll
        for (int w = 0; w < W; ++w) { count[w] = warp_count[w][threadIdx.x]; own += count[w]; }
        block_count[threadIdx.x] = own;
        cluster_arrive();
        cluster_wait();
        int total = 0, earlier = 0;
#pragma unroll
        for (int r = 0; r < kSorters; ++r) {
            const int c = *at_rank(&block_count[threadIdx.x], r);
            total += c;
            if (r < rank) earlier += c;
        }
        int sum = total;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) scan[warp] = sum;
        __syncthreads();
        int lower = lane < warp ? scan[lane] : 0;         // (W <= 32)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) lower += __shfl_xor_sync(0xffffffffu, lower, o);
        int start = lower + sum - total + earlier;
#pragma unroll
        for (int w = 0; w < W; ++w) { warp_count[w][threadIdx.x] = start; start += count[w]; }
        __syncthreads();
        for (int i0 = from; i0 < to; i0 += 32) {
            const bool have = i0 + lane < to;
            const int2 item = have ? in[i0 + lane] : make_int2(0, 0);
            const int digit = have ? (item.x >> (bits * pass)) & mask : D;
            const unsigned same = __match_any_sync(0xffffffffu, digit);
            const int before = __popc(same & ((1u << lane) - 1u));
            const int place = have ? warp_count[warp][digit] + before : 0;
            __syncwarp();
            if (have && before == 0) warp_count[warp][digit] += __popc(same);
            __syncwarp();
            if (!have) continue;
            if (pass + 1 < passes) {
                *at_rank(out + place % each, place / each) = item;
            } else {
                keys_out[(long long)cluster * p.length + place] = item.x;
                places_out[(long long)cluster * p.length + place] = item.y;
            }
        }
        if (pass + 1 < passes) {
            cluster_arrive();                             // what the others put here has arrived; their reads here are done
        } else {
            // (nobody waits for the results here.)  Which tokens occur: the words were zero before the pass's first barrier
            cluster_done();
            for (int i0 = 0; i0 < mine; i0 += kSortThreads) note_occurs(p, cluster, i0 + (int)threadIdx.x < mine ? in[i0 + threadIdx.x].x : INT_MAX);
        }
        cluster_wait();
    }
}

// Longer sequences: the same sort by launches of its own, two a pass, or three.  First: how often each digit occurs in a tile.
__global__ void __launch_bounds__(kThreads)
radix_count_kernel(const GradArgs p, const int32_t *keys, int shift, int first_pass, int *counts) {
    __shared__ int hist[kDigits];
    const int g = blockIdx.y;
    keys += (long long)g * p.length;
    hist[threadIdx.x] = 0;
    if (first_pass && g == 0 && blockIdx.x == 0 && threadIdx.x == 0) *p.crossings = 0;
    __syncthreads();
    const long long t0 = (long long)blockIdx.x * kTile;
    for (int i = threadIdx.x; i < kTile; i += kThreads) {
        const bool have = t0 + i < p.length;
        int key = have ? keys[t0 + i] : PARLE_NO_TOKEN;
        if (first_pass) {
            note_bad_token(key, p.vocab, p.flags);
            key = sort_key(key, p.vocab);
            note_occurs(p, g, have ? key : INT_MAX);
        }
        if (!have) continue;
        atomicAdd(&hist[(key >> shift) & (kDigits - 1)], 1);
    }
    __syncthreads();
    counts[((long long)g * (gridDim.x + 1) + blockIdx.x) * kDigits + threadIdx.x] = hist[threadIdx.x];
}

constexpr int kSummedTiles = 64;        // most tiles whose counts every block of a move adds up by itself
constexpr int kScanDigits = 32, kScanThreads = 1024;

// Of many tiles, the counts become the counts of the tiles before, and the row behind them the totals: a move then reads two rows, where
// adding up all tiles' counts in every block takes reads that grow with the square of the length.  A block takes 32 digits of a
// table, a lane each; its warps take a part of the tiles each.  grid (digits / 32, n).
// Measured, added up by every block / scanned, 64 columns of bf16: 32769 positions 65 / 74 us, 65536 into 4000 rows 86 / 95, 131072 into
// 50021 rows 119 / 128, 262144 (64 tiles) 187 / 186.
__global__ void __launch_bounds__(kScanThreads) radix_scan_kernel(int *counts, int tiles) {
    constexpr int W = kScanThreads / 32;
    __shared__ int sums[W][kScanDigits];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int *const c = counts + (long long)blockIdx.y * (tiles + 1) * kDigits + blockIdx.x * kScanDigits + lane;
    const int each = (tiles + W - 1) / W, from = min(tiles, warp * each), to = min(tiles, from + each);
    int sum = 0;
#pragma unroll 8
    for (int t = from; t < to; ++t) sum += c[(long long)t * kDigits];
    sums[warp][lane] = sum;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < warp; ++w) before += sums[w][lane];
    if (warp == W - 1) c[(long long)tiles * kDigits] = before + sum;
#pragma unroll 8
    for (int t = from; t < to; ++t) {
        const int own = c[(long long)t * kDigits];
        c[(long long)t * kDigits] = before;
        before += own;
    }
}

// Then: every position moves to (positions with a lower digit) + (same digit, earlier tile) + (same digit, earlier in the tile).
// A warp owns kTile / 8 consecutive positions and ranks 32 at a time by matching digits.
__global__ void __launch_bounds__(kThreads)
radix_move_kernel(const int32_t *keys, const int *places, int length, int vocab, int shift, int first_pass, const int *counts, int scanned,
                  int *keys_out, int *places_out) {
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
    const int *c = counts + (long long)g * (gridDim.x + 1) * kDigits + threadIdx.x;
    if (scanned) {
        total = c[(long long)gridDim.x * kDigits];
        earlier = c[(long long)blockIdx.x * kDigits];
    } else {
        for (int b = 0; b < (int)gridDim.x; ++b) {
            const int v = c[(long long)b * kDigits];
            total += v;
            if (b < (int)blockIdx.x) earlier += v;
        }
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

// ---- sorted gradient: the sums ------------------------------------------------------------------------------------------------------------

// A thread's columns of a row: eight consecutive ones on a 16-byte boundary (WIDE), or C that lie kThreads apart.
template <typename T, bool WIDE, int C> struct Columns {
    static constexpr int N = WIDE ? 8 : C;
    std::conditional_t<WIDE, Pack8<T>, T> raw[WIDE ? 1 : C];
    __device__ __forceinline__ void load(const T *from, int left) {
        if constexpr (WIDE) {
            raw[0].load(from);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c * kThreads < left) raw[c] = from[c * kThreads];
        }
    }
    __device__ __forceinline__ void add_to(float (&acc)[N], int left) const {
        if constexpr (WIDE) {
            float v[8];
            raw[0].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += v[e];
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c * kThreads < left) acc[c] += to_float(raw[c]);
        }
    }
    __device__ __forceinline__ static void store(float *to, const float (&v)[N], int left) {
        if constexpr (WIDE) {
            Pack8<float> p;
            p.set(v);
            p.store(to);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c * kThreads < left) to[c * kThreads] = v[c];
        }
    }
    __device__ __forceinline__ static void scale(const GradArgs &p, const float *to, float (&v)[N], int left) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            if (!p.accumulate) v[c] *= p.scale;
            else if (WIDE || c * kThreads < left) v[c] = fmaf(p.scale, v[c], to[WIDE ? c : c * kThreads]);
        }
    }
};

// Behind a position: its run goes on; the run began before the chunk; it goes on behind it; else the sum goes to a table row.
constexpr int kOn = -1, kFirst = -2, kLast = -3;

// A chunk's runs: their sums inside the chunk and where those go.  A block takes kThreads * N columns, U rows in flight.
template <typename T, bool WIDE, int C, int U> __device__ __forceinline__ void sum_chunk(const GradArgs &p, int g, int chunk) {
    using Part = Columns<T, WIDE, C>;
    constexpr int N = Part::N;
    __shared__ int place[kChunk], goes[kChunk], live_rows;      // per position: its row of dout, where its run's sum goes behind it
    const int first = chunk * kChunk, count = min(kChunk, p.length - first);
    static_assert(kChunk == 32, "a lane per position");
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        const int *keys = p.keys + (long long)g * p.length + first;
        const int key = lane < count ? keys[lane] : -1, border = lane == 0 ? (first ? keys[-1] : -1) : lane == 1 && first + count < p.length ? keys[count] : -1;
        if (lane < count) place[lane] = p.places[(long long)g * p.length + first + lane];
        const int previous = __shfl_sync(0xffffffffu, border, 0), following = __shfl_sync(0xffffffffu, border, 1);      // next to the chunk
        const int down = __shfl_down_sync(0xffffffffu, key, 1), next = lane + 1 < count ? down : following;
        const bool before = previous == key, after = lane + 1 == count && next == key;
        // (a run that fills the chunk and goes on both ways counts as "began before")
        goes[lane] = next == key && !after ? kOn : before ? kFirst : after ? kLast : key;
        const unsigned live = __ballot_sync(0xffffffffu, lane < count && key < p.vocab);      // those without a token come last
        if (lane == 0) live_rows = __popc(live);
        if (lane + 1 == kChunk && after && !before && key < p.vocab && blockIdx.y == 0) {
            const int at = atomicAdd(p.crossings, 1);     // (the order of the list does not matter)
            reinterpret_cast<int4 *>(p.crossings)[1 + at] = make_int4(g, chunk, key, 0);
        }
    }
    __syncthreads();
    const int col = blockIdx.y * kThreads * N + threadIdx.x * (WIDE ? 8 : 1), left = p.dim - col, live = live_rows;
    if (left <= 0) return;
    const T *dout = static_cast<const T *>(p.dout) + (long long)g * p.dout_gs + col;
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    for (int i0 = 0; i0 < live; i0 += U) {
        Part raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u < live) raw[u].load(dout + (long long)place[i0 + u] * p.ld_dout, left);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u >= live) break;
            raw[u].add_to(acc, left);
            const int to_row = goes[i0 + u];
            if (to_row == kOn) continue;
            if (to_row < 0) {
                Part::store(p.partial + (((long long)g * p.chunks + chunk) * 2 + (to_row == kFirst ? 0 : 1)) * p.dim + col, acc, left);
            } else {
                float *to = p.dtable + (long long)g * p.dtable_gs + (long long)to_row * p.ld_dtable + col;
                Part::scale(p, to, acc, left);
                Part::store(to, acc, left);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] = 0.f;
        }
    }
}

// Zeros in those of `rows` table rows from v0 on whose tokens do not occur.
__device__ __forceinline__ void zero_absent(const GradArgs &p, int g, int v0, int rows, bool wide) {
    const uint32_t *occurs = p.occurs + (long long)g * p.words;
    const int limit = min(v0 + rows, p.vocab);
    const int lane = threadIdx.x % 32;
    for (int v = v0 + (int)threadIdx.x / 32; v < limit; v += kWarps) {     // a warp per row
        if ((occurs[v / 32] >> (v % 32)) & 1u) continue;
        float *row = p.dtable + (long long)g * p.dtable_gs + (long long)v * p.ld_dtable;
        if (wide) {
#pragma unroll 4
            for (int c = lane * 4; c < p.dim; c += 128) *reinterpret_cast<float4 *>(row + c) = make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
            for (int c = lane; c < p.dim; c += 32) row[c] = 0.f;
        }
    }
}

// Bound by memory: 16384 rows of 2048 bf16 into 50021 rows, 477 MB in 66-70 us, the copy rate.
// Blocks x < chunks sum a chunk each, the others clear `zero_rows` table rows each (y == 0 only); grid (.., column parts, n).
template <typename T, bool WIDE, int C, int U>
__global__ void __launch_bounds__(kThreads, 4) embedding_grad_kernel(const GradArgs p, int zero_rows, bool wide) {
    let_next_start();
    await_previous();
    if ((int)blockIdx.x < p.chunks) sum_chunk<T, WIDE, C, U>(p, blockIdx.z, blockIdx.x);
    else if (blockIdx.y == 0) zero_absent(p, blockIdx.z, (blockIdx.x - p.chunks) * zero_rows, zero_rows, wide);
}

// Runs that cross a border, in tiles of 256 columns.  Most have a few partial rows: a warp adds them up, eight columns a lane.  The
// longer ones a block adds up afterwards: its warps take a part of the partial rows each, in order, and their sums are added in order.
constexpr int kJoinThreads = 512;
constexpr int kPartsOfWarp = 16;

struct Crossing {
    const float *partial;                                 // of the chunk in which the run begins
    float *to;
    int parts;                                            // that chunk's last run, then the first runs of the following chunks
    int col;                                              // this lane's first column; the others lie 32 apart
};

// By a warp.  Chunks are probed 32 at a time for the first that begins with another token.
__device__ __forceinline__ Crossing find_crossing(const GradArgs &p, long long item, int tiles) {
    const int lane = threadIdx.x % 32;
    const int4 c = reinterpret_cast<const int4 *>(p.crossings)[1 + item / tiles];
    const int *keys = p.keys + (long long)c.x * p.length;
    int end = c.y + 2;
    for (;; end += 32) {
        const int at = end + lane;
        const unsigned other = __ballot_sync(0xffffffffu, at >= p.chunks || keys[(long long)at * kChunk] != c.z);
        if (other) { end += __ffs(other) - 1; break; }
    }
    Crossing r;
    r.col = (int)(item % tiles) * 256 + lane;
    r.parts = end - c.y;
    r.partial = p.partial + ((long long)c.x * p.chunks + c.y) * 2 * p.dim;
    r.to = p.dtable + (long long)c.x * p.dtable_gs + (long long)c.z * p.ld_dtable;
    return r;
}
__device__ __forceinline__ void add_parts(const GradArgs &p, const Crossing &r, int from, int to, float (&acc)[8]) {
#pragma unroll 4
    for (int i = from; i < to; ++i) {
        const float *row = r.partial + ((long long)i * 2 + (i == 0 ? 1 : 0)) * p.dim;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (r.col + j * 32 < p.dim) acc[j] += row[r.col + j * 32];
    }
}

__global__ void __launch_bounds__(kJoinThreads, 2) embedding_grad_join_kernel(const GradArgs p) {
    constexpr int W = kJoinThreads / 32;
    __shared__ float sums[W][256];
    __shared__ int longer[W], longers;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, tiles = (p.dim + 255) / 256;
    await_previous();
    const long long items = (long long)*p.crossings * tiles;
    // neighbouring items go to different blocks: the tiles of a long run are neighbours
    for (long long item0 = blockIdx.x; item0 < items; item0 += (long long)gridDim.x * W) {
        if (threadIdx.x == 0) longers = 0;
        __syncthreads();
        if (item0 + (long long)warp * gridDim.x < items) {
            const Crossing r = find_crossing(p, item0 + (long long)warp * gridDim.x, tiles);
            if (r.parts > kPartsOfWarp) {
                if (lane == 0) longer[atomicAdd(&longers, 1)] = warp;
            } else {
                float acc[8] = {};
                add_parts(p, r, 0, r.parts, acc);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float *to = r.to + r.col + j * 32;
                    if (r.col + j * 32 < p.dim) *to = p.accumulate ? fmaf(p.scale, acc[j], *to) : p.scale * acc[j];
                }
            }
        }
        __syncthreads();
        for (int l = 0; l < longers; ++l) {
            const Crossing r = find_crossing(p, item0 + (long long)longer[l] * gridDim.x, tiles);
            const int per_warp = (r.parts + W - 1) / W, from = min(r.parts, warp * per_warp);
            float acc[8] = {};
            add_parts(p, r, from, min(r.parts, from + per_warp), acc);
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[warp][j * 32 + lane] = acc[j];
            __syncthreads();
            const int c = threadIdx.x, col = r.col - lane + c;
            if (c < 256 && col < p.dim) {
                float s = sums[0][c];
                const int used = (r.parts + per_warp - 1) / per_warp;
                for (int w = 1; w < used; ++w) s += sums[w][c];
                r.to[col] = p.accumulate ? fmaf(p.scale, s, r.to[col]) : p.scale * s;
            }
            __syncthreads();
        }
    }
}

// ---- workspace -----------------------------------------------------------------------------------------------------------------

struct GradPlan {
    int chunks, tiles, passes, sort_passes, sort_bits, words;
    size_t keys[2], places[2], counts, occurs, crossings, partial, bytes;
};

GradPlan plan_grad(int n, long long length, int vocab, int dim) {
    GradPlan p = {};
    if (length <= kDirectMost) return p;
    p.chunks = (int)((length + kChunk - 1) / kChunk);
    const size_t ints = round_up((size_t)n * length * sizeof(int), 128);
    int bits = 1;
    while (bits < 31 && (vocab >> bits)) ++bits;          // keys 0 .. vocab
    p.passes = (bits + 7) / 8;
    p.sort_passes = (bits + kSortBits - 1) / kSortBits;
    p.sort_bits = (bits + p.sort_passes - 1) / p.sort_passes;
    p.words = (vocab + 31) / 32;
    size_t at = 0;
    if (length > kSortMost) p.tiles = (int)((length + kTile - 1) / kTile);
    for (int i = 0; i < (p.tiles ? 2 : 1); ++i) { p.keys[i] = at; at += ints; p.places[i] = at; at += ints; }
    p.counts = at;
    if (p.tiles) at += round_up((size_t)n * (p.tiles + 1) * kDigits * sizeof(int), 128);      // (a row of totals behind the tiles')
    p.occurs = at;
    at += round_up((size_t)n * p.words * sizeof(uint32_t), 128);
    p.crossings = at;
    at += round_up((1 + (size_t)n * p.chunks) * sizeof(int4), 128);
    p.partial = at;
    at += round_up((size_t)n * p.chunks * 2 * dim * sizeof(float), 128);
    p.bytes = at;
    return p;
}

template <typename T, int E> int launch_direct(const GradArgs &a, int n, int sms, cudaStream_t stream) {
    const int parts = (a.dim + kColumns - 1) / kColumns;
    int log_groups = 0;                                   // blocks of at most kRowsMost rows, and enough of them for the SMs
    while (((a.vocab - 1) >> log_groups) >= kRowsMost) ++log_groups;
    while ((a.vocab >> log_groups) > 8 && ((long long)parts * n << log_groups) < 4LL * sms) ++log_groups;
    embedding_grad_direct_kernel<T, E><<<dim3(1u << log_groups, parts, n), kThreads, 0, stream>>>(a, log_groups);
    return launch_status();
}

template <typename T>
int launch_sorted(GradArgs a, int n, const GradPlan &plan, bool wide, bool wide_table, char *ws, int sms, cudaStream_t stream) {
    int *keys[2], *places[2];
    for (int i = 0; i < 2; ++i) {
        keys[i] = reinterpret_cast<int *>(ws + plan.keys[i]);
        places[i] = reinterpret_cast<int *>(ws + plan.places[i]);
    }
    a.occurs = reinterpret_cast<uint32_t *>(ws + plan.occurs);
    a.words = plan.words;
    a.crossings = reinterpret_cast<int *>(ws + plan.crossings);
    a.partial = reinterpret_cast<float *>(ws + plan.partial);
    int sorted = 0, rc;
    const int rank_blocks = (a.length + kThreads / kSplit - 1) / (kThreads / kSplit), words_each = (plan.words + rank_blocks - 1) / rank_blocks;
    if (a.length <= kRankedMost && words_each <= kWordsMost) {
        rank_tokens_kernel<<<dim3(rank_blocks, n), kThreads, 0, stream>>>(a, words_each, keys[0], places[0]);
    } else if (!plan.tiles) {
        constexpr int bytes = 2 * kSortEach * (int)sizeof(int2);
        if (cudaFuncSetAttribute(sort_tokens_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return PARLE_ECUDA;
        cudaLaunchAttribute attr = {};
        const cudaLaunchConfig_t cfg = cluster_config(dim3((unsigned)n * kSorters), kSortThreads, bytes, kSorters, &attr, stream);
        if (cudaLaunchKernelEx(&cfg, sort_tokens_kernel, a, plan.sort_passes, plan.sort_bits,
                               keys[0], places[0]) != cudaSuccess) return PARLE_ECUDA;
    } else {
        int *counts = reinterpret_cast<int *>(ws + plan.counts);
        if (cudaMemsetAsync(a.occurs, 0, (size_t)n * a.words * sizeof(uint32_t), stream) != cudaSuccess) return PARLE_ECUDA;
        for (int pass = 0; pass < plan.passes; ++pass) {
            const dim3 grid(plan.tiles, n);
            const int32_t *in = pass ? keys[sorted] : a.tokens;
            const int to = pass ? 1 - sorted : 0;
            radix_count_kernel<<<grid, kThreads, 0, stream>>>(a, in, 8 * pass, pass == 0, counts);
            if ((rc = launch_status()) != PARLE_OK) return rc;
            const bool scanned = plan.tiles > kSummedTiles;
            if (scanned) {
                radix_scan_kernel<<<dim3(kDigits / kScanDigits, n), kScanThreads, 0, stream>>>(counts, plan.tiles);
                if ((rc = launch_status()) != PARLE_OK) return rc;
            }
            radix_move_kernel<<<grid, kThreads, 0, stream>>>(in, places[sorted], a.length, a.vocab, 8 * pass, pass == 0, counts, scanned, keys[to], places[to]);
            if ((rc = launch_status()) != PARLE_OK) return rc;
            sorted = to;
        }
    }
    if ((rc = launch_status()) != PARLE_OK) return rc;
    a.keys = keys[sorted];
    a.places = places[sorted];
    // Columns of a thread: eight, on 16-byte boundaries, or up to four single ones.  Measured, against one single column at a time: 16234
    // rows of 1310 bf16 into 4643 rows 40 / 64 us, 6563 of 780 fp32 into 2606 24 / 42, 6563 of 501 bf16 23 / 31.
    const int narrow = a.dim > 2 * kThreads ? 4 : a.dim > kThreads ? 2 : 1, columns = kThreads * (wide ? 8 : narrow);
    const long long row_bytes = (long long)a.dim * 4;
    const int zero_rows = (int)std::max(1LL, std::min(256LL, 65536 / row_bytes));
    const long long zero_blocks = a.accumulate ? 0 : ((long long)a.vocab + zero_rows - 1) / zero_rows;
    const dim3 grid((unsigned)(plan.chunks + zero_blocks), (a.dim + columns - 1) / columns, n);      // (at most 2^14 column parts)
    cudaLaunchAttribute chained = {};
    chained.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    chained.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = stream;
    cfg.attrs = &chained;
    cfg.numAttrs = 1;
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    const auto kernel = wide ? embedding_grad_kernel<T, true, 1, 8> : narrow == 4 ? embedding_grad_kernel<T, false, 4, 8>
                        : narrow == 2 ? embedding_grad_kernel<T, false, 2, 8> : embedding_grad_kernel<T, false, 1, 8>;
    if (cudaLaunchKernelEx(&cfg, kernel, a, zero_rows, wide_table) != cudaSuccess) return PARLE_ECUDA;
    cfg.gridDim = dim3(2 * sms);
    cfg.blockDim = dim3(kJoinThreads);
    if (cudaLaunchKernelEx(&cfg, embedding_grad_join_kernel, a) != cudaSuccess) return PARLE_ECUDA;
    return launch_status();
}

bool valid_sizes(int n, long long length, int vocab, int dim) {
    return n >= 1 && n <= PARLE_MAX_REPLICAS && length >= 0 && vocab >= 1 && dim >= 1;
}

bool too_big(int n, long long length, int vocab, int dim) {
    return length > PARLE_TOKEN_MAX_ROWS / n || vocab > PARLE_TOKEN_MAX_ROWS || dim > PARLE_EMBEDDING_MAX_DIM;
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
    if (too_big(n, length, vocab, dim)) return PARLE_ETOOBIG;
    if (ld_table < 0 || (n > 1 && table_gs < 0) || !separate_rows(n, length, dim, out_gs, ld_out)) return PARLE_EINVAL;
    if (length == 0) return PARLE_OK;
    if (!table || !tokens || !out) return PARLE_EINVAL;
    if (!element_aligned(table, table_dtype) || !element_aligned(out, out_dtype) || !element_aligned(tokens, PARLE_F32) ||
        !element_aligned(flags, PARLE_F32)) return PARLE_EALIGN;
    LookupArgs a = {};
    a.table = table; a.out = out; a.tokens = tokens; a.flags = flags;
    a.table_gs = table_gs; a.ld_table = ld_table; a.out_gs = out_gs; a.ld_out = ld_out;
    a.length = length;
    a.vocab = vocab; a.dim = dim; a.scale = (float)scale;
    const bool wide = dim % 8 == 0 && rows_aligned16(table, ld_table, table_dtype) && rows_aligned16(out, ld_out, out_dtype) &&
                      (n == 1 || (rows_aligned16(table, table_gs, table_dtype) && rows_aligned16(out, out_gs, out_dtype)));
    const int sms = current_sms();
    if (sms < 0) return PARLE_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return with_dtype(table_dtype, [&](auto *ti) {
        return with_dtype(out_dtype, [&](auto *to) {
            using TI = std::remove_pointer_t<decltype(ti)>;
            using TO = std::remove_pointer_t<decltype(to)>;
            return wide ? launch_lookup<TI, TO, 8>(a, n, sms, stream) : launch_lookup<TI, TO, 1>(a, n, sms, stream);
        });
    });
}

extern "C" size_t parle_embedding_grad_workspace_bytes(int n, long long length, int vocab, int dim) {
    if (!valid_sizes(n, length, vocab, dim) || too_big(n, length, vocab, dim)) return 0;
    return plan_grad(n, length, vocab, dim).bytes;
}

extern "C" int parle_embedding_grad(const void *dout, int dout_dtype, long long dout_gs, long long ld_dout, const int32_t *tokens,
                                    int n, long long length, int vocab, int dim, double scale, float *dtable, long long dtable_gs,
                                    long long ld_dtable, int accumulate, void *workspace, size_t workspace_bytes, int32_t *flags,
                                    void *cuda_stream) {
    if (!valid_sizes(n, length, vocab, dim) || !valid_dtype(dout_dtype) || !isfinite((float)scale)) return PARLE_EINVAL;
    if (too_big(n, length, vocab, dim)) return PARLE_ETOOBIG;
    if (ld_dout < 0 || (n > 1 && dout_gs < 0) || !separate_rows(n, vocab, dim, dtable_gs, ld_dtable) || !dtable) return PARLE_EINVAL;
    const GradPlan plan = plan_grad(n, length, vocab, dim);
    if (length > 0 && (!dout || !tokens || (!workspace && plan.bytes))) return PARLE_EINVAL;
    if (!element_aligned(dout, dout_dtype) || !element_aligned(dtable, PARLE_F32) || !element_aligned(tokens, PARLE_F32) ||
        !element_aligned(flags, PARLE_F32) || reinterpret_cast<uintptr_t>(workspace) % 128) return PARLE_EALIGN;
    if (workspace_bytes < plan.bytes) return PARLE_EWORKSPACE;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    GradArgs a = {};
    a.dout = dout; a.dtable = dtable; a.tokens = tokens; a.flags = flags;
    a.dout_gs = dout_gs; a.ld_dout = ld_dout; a.dtable_gs = dtable_gs; a.ld_dtable = ld_dtable;
    a.length = (int)length; a.vocab = vocab; a.dim = dim; a.chunks = plan.chunks;
    a.scale = (float)scale; a.accumulate = accumulate != 0;
    const bool wide_table = dim % 4 == 0 && rows_aligned16(dtable, ld_dtable, PARLE_F32) && (n == 1 || dtable_gs % 4 == 0);
    const bool wide = wide_table && dim % 8 == 0 && rows_aligned16(dout, ld_dout, dout_dtype) && (n == 1 || rows_aligned16(dout, dout_gs, dout_dtype));
    const int sms = current_sms();
    if (sms < 0) return PARLE_ECUDA;
    return with_dtype(dout_dtype, [&](auto *tag) {
        using TD = std::remove_pointer_t<decltype(tag)>;
        if (plan.passes) return launch_sorted<TD>(a, n, plan, wide, wide_table, static_cast<char *>(workspace), sms, stream);
        return wide ? launch_direct<TD, 8>(a, n, sms, stream) : launch_direct<TD, 1>(a, n, sms, stream);
    });
}
