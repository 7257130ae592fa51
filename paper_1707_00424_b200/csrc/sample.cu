// parle_sample_tokens: a token of each row of logits, with temperature, top-k, top-p and min-p, from one given random number a row.
//
// With m the row's largest logit, weights w_j = exp(scale (x_j - m)) and ranks by (logit descending, token ascending): the tokens kept are a
// prefix of the ranking, {x > T} and the first of the tokens with x = T by number; the one sampled is the first kept token, by number,
// at which the sum of kept weights exceeds u times their total.
//
// A token is right or wrong, and with 10^5 tokens u lies within 10^-6 of one of the sums' steps in every tenth row: sums of fp32
// exponentials would give another token there than the definition.  So weights are formed in fp64 (nine operations) and kept as whole
// numbers of 2^-44: their sums are exact and the same in any order, whichever threads and atomics form them.  u times the total is formed exactly,
// too (128 bits).  fp32 sums serve where their error, which is bounded, does not matter.
//
// A row is read by one block of 512 threads, or by a cluster of up to eight where there are few rows (of 128 threads up to 4096 tokens), two
// blocks an SM (one, with twice the registers, took 1.2 to 1.3 times as long).  By what is asked for:
//   top_k up to 256, min_p, top_p that is reached by as many: one pass over the row finds its largest logit and lists the logits from a
//     bound on, which the largest logits of the threads' first granules give; the list is sorted and decides everything.  512 rows of 131072 bf16
//     logits with all three 73 us: DRAM, then sorting while DRAM rests (the floor is 21 us).  One row 14 us: latency of a
//     cluster's joins.  Where the first granules hold more large logits than the rest, as where frequent tokens come first, a list is too short and a second
//     pass looks at all logits for the bound: 256 rows with top_k = 50 37 us (26 without), 512 rows with top_k = 200 and the others 93 (91).
//   nothing: one pass that forms all weights, relative to the guess that the first granules give, and their sums by segments of 256 or 1024 logits; the
//     segment and the token by sums of sums.  256 rows of 131072 bf16 logits 66 us: latency at 25 warps an SM, beside fp64 (20 us of its pipe) and
//     issue slots (62 %).
//   top_p of an undecided model, larger top_k: logits are counted by steps of scale (m - x), 1/128 wide, which tells nearly where the border lies;
//     one more pass forms the weights, their exact total and segments' sums, and lists the logits around the border.  256 rows with top_p = 0.95,
//     25000 tokens kept, 174 us: a fifth the counts, two fifths the weights.
//   what escapes these (thousands of equal logits at the border, a wrong guess): exact histograms of 64-bit sums, of which two 32-bit words lie
//     in shared memory and the adding thread passes on the carry, of steps of scale (m - x) and then of the logits' bits, 11 at a time.
#include <math.h>

#include <type_traits>

#include "token_types.cuh"

using namespace parle;

namespace {

// Entries of the list, bins of a histogram and segments of a block's part, for blocks of long and of short rows (of which fewer logits fall into
// a coarser bin, and 128 threads sort a long list slowly).
template <int THREADS> struct Sizes {
    static constexpr int kList = THREADS == 512 ? 1024 : 256;
    static constexpr int kLogBins = THREADS == 512 ? 11 : 9, kBins = 1 << kLogBins, kSegments = THREADS == 512 ? 1024 : 128;
};
constexpr uint32_t kNegInf = 0x007fffffu;                // key of -inf

struct SampleArgs {
    const void *logits;
    long long rows, ld;
    int vocab;
    float scale, top_p, min_p;
    int top_k;
    const float *u, *scales, *top_ps, *min_ps;
    const int32_t *top_ks;
    int32_t *token, *kept, *flags;
    float *logprob;
    int granules;                                        // of a block's part of a row
    int seg_steps;                                       // a segment is 32 x seg_steps granules
    int frac_bits;                                       // weights are whole numbers of 2^-frac_bits
};

typedef unsigned long long u64;

// Logits as unsigned numbers of the same order; -0 counts as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
// The number that logits of keys above `key` are above, and no others.  (The key below 0's is that of -0, which no logit has, and 0 > -0 is false.)
__device__ __forceinline__ float below(uint32_t key) { return value_of(key - (key == 0x7fffffffu ? 1 : 0)); }

// f total, f in [0, 1), exactly: rounded down or up to a whole number.
__device__ __forceinline__ u64 part_of(u64 total, float f, bool up) {
    if (!(f > 0.f)) return 0;
    const uint32_t b = __float_as_uint(f), e = b >> 23;
    const u64 mantissa = (b & 0x7fffffu) | (e ? 0x800000u : 0u);
    const int s = 150 - (e ? (int)e : 1);                // f = mantissa 2^-s, s >= 24
    const u64 low = total * mantissa, high = __umul64hi(total, mantissa);
    u64 whole, rest;
    if (s >= 128) { whole = 0; rest = low | high; }
    else if (s >= 64) { whole = high >> (s - 64); rest = low | (s == 64 ? 0 : high << (128 - s)); }
    else { whole = high << (64 - s) | low >> s; rest = low << (64 - s); }
    return whole + (up && rest ? 1 : 0);
}

struct Weigher {                                         // w(x) = exp(scale (x - best)) as a whole number of 2^-frac_bits
    double best, c, one;                                 // c: 32 scale log2 e; one: whose last bit is 2^-frac_bits
    float least;                                         // it and all logits below weigh nothing
    float most;                                          // logits above `best` that raw() may be used for (where best is a guess): w < e^4.8 < 2^7
    const double *table;                                 // 2^(i / 32), in shared memory; less i 2^15 in the upper word, which n 2^15 adds
    __device__ __forceinline__ void set(float best_, float scale, int frac_bits, const double *table_) {
        best = best_;
        table = table_;
        one = __hiloint2double((1023 + 52 - frac_bits) << 20, 0);
        // e^-45 < 2^-64.  Where best - 45 / scale is best again, the next number below weighs nothing, and is taken for as little as fits.
        least = fminf(best_ - 45.f / scale, value_of(key_of(best_) - 1));
        c = fmin(32.0 * 1.44269504088896340736 * scale, 4096.0 / (best - (double)least));
        most = __fadd_rd(best_, 4.8f / scale);           // (rounded down: the next logit above `best` may lie farther away)
    }
    // 2^(n / 32) from the table and its exponent, e^y of the rest, |y| <= ln 2 / 64 = h, by Taylor's polynomial of degree 5 whose last term is spread over y and y^3
    // (Chebyshev's economisation: 16 z^5 - 20 z^3 + 5 z is at most 1): off by h^5 / 1920 = 8 10^-14.  Nine operations in fp64.
    // raw(): of least <= x <= most, with the bits of `one` still on it
    __device__ __forceinline__ u64 raw(float x) const { return (u64)__double_as_longlong(formed(x, one)); }
    __device__ __forceinline__ u64 operator()(float x) const {
        if (x > most) return __double2ull_rn(formed(x, 0.0) * __hiloint2double(2 * 1023 + 52 - (__double2hiint(one) >> 20) << 20, 0));
        return raw(fmaxf(x, least)) - (u64)__double_as_longlong(one);
    }

  private:
    __device__ __forceinline__ double formed(float x, double more) const {
        constexpr double y = 0.69314718055994530942 / 32, h = y / 2;
        const double d = (double)x - best;
        const double shifted = fma(d, c, 6755399441055744.0);      // 1.5 2^52: rounds to a whole number
        const int n8 = __double2loint(shifted) << 3;
        const double r = fma(d, c, 6755399441055744.0 - shifted);
        double p = fma(r, y * y * y * y / 24, y * y * y * (1.0 / 6 + h * h / 96));
        p = fma(p, r, y * y / 2);
        p = fma(p, r, y * (1.0 - h * h * h * h / 384));
        p = fma(p, r, 1.0);
        const double power = *reinterpret_cast<const double *>(reinterpret_cast<const char *>(table) + (n8 & 0xf8));
        return fma(p, __hiloint2double(__double2hiint(power) + (n8 << 12), __double2loint(power)), more);
    }
};

// A row in granules of eight logits, cut at memory's 16-byte boundaries.  `flat`: all logits are -inf or the lowest number (a row that is masked
// altogether); the latter are then taken for 0, so that there is a number below the largest logit, always.
template <typename T> struct Row {
    const T *x;
    int vocab, skew;                                     // logits of the first granule before the row
    bool flat;
    int whole_from, whole_to;                            // granules that lie in the row altogether
    __device__ __forceinline__ long long first(int granule) const { return (long long)granule * 8 - skew; }
    __device__ __forceinline__ bool whole(int granule) const { return granule >= whole_from && granule < whole_to; }
    __device__ __forceinline__ float at(long long token) const {
        const float v = token >= 0 && token < vocab ? to_float(x[token]) : -INFINITY;
        return flat && v > -INFINITY ? 0.f : v;
    }
    __device__ __forceinline__ Pack8<T> fetch(int granule, int end) const {      // early; nothing where it is not whole
        Pack8<T> p = {};
        if (granule < end && whole(granule)) p.load(x + first(granule));
        return p;
    }
    __device__ __forceinline__ void get(const Pack8<T> &p, int granule, float (&v)[8]) const {
        if (whole(granule)) {
            p.get(v);
            if (flat) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = v[i] > -INFINITY ? 0.f : v[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = at(first(granule) + i);
        }
    }
    // The largest of a granule as fetched; NaN if one is.  (Not of flat rows.)
    __device__ __forceinline__ float most(const Pack8<T> &p, int granule) const;
    __device__ __forceinline__ void load(int granule, float (&v)[8]) const { get(fetch(granule, granule + 1), granule, v); }
};

__device__ __forceinline__ float largest(float v, float w) {      // NaN if either is
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(v), "f"(w));
    return m;
}
__device__ __forceinline__ __nv_bfloat162 largest(__nv_bfloat162 v, __nv_bfloat162 w) { return __hmax2_nan(v, w); }
__device__ __forceinline__ __half2 largest(__half2 v, __half2 w) { return __hmax2_nan(v, w); }
// The largest of granules of 16-bit logits in pairs (half the instructions), of fp32 ones one by one.
template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> { typedef __nv_bfloat162 type; };
template <> struct Pair<__half> { typedef __half2 type; };
template <typename T> struct Largest {
    typename Pair<T>::type pair;
    __device__ __forceinline__ Largest() { pair.x = pair.y = from_float<T>(-INFINITY); }
    __device__ __forceinline__ void take(const Pack8<T> &p) {
        typedef typename Pair<T>::type P2;
        const P2 *h = reinterpret_cast<const P2 *>(&p);
        pair = largest(pair, largest(largest(h[0], h[1]), largest(h[2], h[3])));
    }
    __device__ __forceinline__ float get() const { return largest(to_float(pair.x), to_float(pair.y)); }
};
template <> struct Largest<float> {
    float most = -INFINITY;
    __device__ __forceinline__ void take(const Pack8<float> &p) {
        most = largest(most, largest(largest(largest(p.a.x, p.a.y), largest(p.a.z, p.a.w)), largest(largest(p.b.x, p.b.y), largest(p.b.z, p.b.w))));
    }
    __device__ __forceinline__ float get() const { return most; }
};

template <typename T> __device__ __forceinline__ float Row<T>::most(const Pack8<T> &p, int granule) const {
    if (whole(granule)) {
        Largest<T> m;
        m.take(p);
        return m.get();
    }
    float m = -INFINITY;
#pragma unroll 1
    for (int k = 0; k < 8; ++k) m = largest(m, at(first(granule) + k));
    return m;
}

struct Cut {                                             // kept: logits of keys above `key`, and the first `ties` of those with it;
    uint32_t key;                                        // by_last: of those, the ones up to token `last`
    u64 ties;
    bool by_last;
    uint32_t last;
};

struct Part {                                            // what a block found out about its part of the row
    float best;
    uint32_t bound;                                      // key that as many logits of the part reach as were asked for
    double sum;                                          // of weights, in fp32's precision
    u64 mass, above;
    uint32_t count, ties;
};

enum Outcome { kDone, kNeedTotal, kNeedAll };            // of a list of the largest logits: sampled from; the weights' total is needed exactly; too short

enum Settled { kNot, kSums, kCutOnly };                  // a border was not found; with the segments' sums; without them

template <int THREADS> struct Shared {
    static constexpr int kBins = Sizes<THREADS>::kBins, kSegments = Sizes<THREADS>::kSegments, kList = Sizes<THREADS>::kList;
    double table[32];
    union alignas(16) {
        uint32_t hist[2][kBins];
        struct {
            u64 mass[kSegments];
            uint32_t ties[kList];                        // (of segments; or the keys of list entries)
        } seg;
    };
    alignas(16) u64 list[kList];                                     // ~key << 32 | token
    u64 weight[kList];
    u64 sums[kList];
    u64 scan[THREADS / 32];
    double scan_f[THREADS / 32];
    float maxima[THREADS / 32];
    float minima[THREADS / 32];
    uint32_t listed;
    Outcome outcome;
    Part part;
    struct {
        u64 above, total;
        int bin;
        uint32_t low, high;
    } found;
    struct {
        u64 before, upto;                                // logits in the steps before the bracket, and up to its end
        int from, to;
    } bracket;
    struct {                                             // by rank 0: what is kept, with its last token
        Settled settled;
        uint32_t key, last;
        u64 kept, ties;
    } choice;
    struct {
        u64 target;
        uint32_t ties_before;
        int segment;
    } hit;
};

// Every thread of the row's blocks has come here, and sees what the others wrote.
__device__ __forceinline__ void all_meet(int blocks) {
    if (blocks == 1) __syncthreads();
    else {
        cluster_arrive();
        cluster_wait();
    }
}

__device__ __forceinline__ u64 of_warp(u64 v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ u64 shfl_up64(u64 v, int by) { return __shfl_up_sync(0xffffffffu, v, by); }

// Exclusive sum over the block's threads; *total: of all.
template <int THREADS> __device__ __forceinline__ u64 block_scan(u64 v, u64 (&scratch)[THREADS / 32], u64 *total) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    u64 sum = v;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const u64 below = shfl_up64(sum, o);
        if (lane >= o) sum += below;
    }
    __syncthreads();                                     // (scratch may still be read from the last call)
    if (lane == 31) scratch[warp] = sum;
    __syncthreads();
    u64 before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        const u64 s = scratch[w];
        if (w < warp) before += s;
        all += s;
    }
    *total = all;
    return before + sum - v;
}

template <typename T, int THREADS> struct Sampler {
    static constexpr int kList = Sizes<THREADS>::kList, kLogBins = Sizes<THREADS>::kLogBins, kBins = Sizes<THREADS>::kBins, kPer = kBins / THREADS;
    Shared<THREADS> &sh;
    Row<T> row;
    int blocks, rank, begin, end;                        // the row's blocks; this one's granules
    float scale, best;
    Weigher weigh;

    __device__ __forceinline__ int step_of(float x) const { return min(kBins - 1, (int)((best - x) * scale * (kBins / 64.f))); }

    __device__ __forceinline__ Shared<THREADS> *block(int o) const { return blocks == 1 ? &sh : at_rank(&sh, o); }
    // f(o, value(block o)) for the row's blocks: a word of another block's shared memory takes some 200 ns, so all are fetched first.
    template <class V, class F> __device__ __forceinline__ void of_blocks(V value, F f) const {
        typedef decltype(value(sh)) W;
        if (blocks == 1) {
            f(0, value(sh));
            return;
        }
        W w[8];
#pragma unroll
        for (int o = 0; o < 8; ++o)
            if (o < blocks) w[o] = value(*at_rank(&sh, o));
#pragma unroll
        for (int o = 0; o < 8; ++o)
            if (o < blocks) f(o, w[o]);
    }
    // f(o, i, words) for four words after another of an array in the blocks' shared memory, the thread's N x 4 ones.
    template <int N, class A, class F> __device__ __forceinline__ void of_arrays(A array, F f) const {
#pragma unroll 2
        for (int o = 0; o < blocks; ++o) {
            const uint4 *const from = reinterpret_cast<const uint4 *>(array(*block(o))) + threadIdx.x * N;
            uint4 w[N];
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = from[i];
#pragma unroll
            for (int i = 0; i < N; ++i) f(i, w[i]);
        }
    }

    // f(granule, its raw form) for each granule of the block's part, some in flight.
    template <class F> __device__ __forceinline__ void each_granule(F f, int first = 0) const {
        constexpr int kFlight = 2;
        for (int g = begin + first + (int)threadIdx.x; g < end; g += THREADS * kFlight) {
            Pack8<T> p[kFlight];
#pragma unroll
            for (int i = 0; i < kFlight; ++i) p[i] = row.fetch(g + i * THREADS, end);
#pragma unroll
            for (int i = 0; i < kFlight; ++i) {
                if (g + i * THREADS >= end) break;
                f(g + i * THREADS, p[i]);
            }
        }
    }
    template <class F> __device__ __forceinline__ void each(F f) const {
        each_granule([&](int g, const Pack8<T> &p) {
            float v[8];
            row.get(p, g, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) f(v[i]);
        });
    }
    // The first granules of a thread stay in registers.
    static constexpr int kHeld = sizeof(T) == 2 ? 4 : 2;
    __device__ __forceinline__ void fetch_first(Pack8<T> (&held)[kHeld]) const {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) held[i] = row.fetch(begin + (int)threadIdx.x + i * THREADS, end);
    }
    template <class F> __device__ __forceinline__ void each_held(const Pack8<T> (&held)[kHeld], F f) const {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int g = begin + (int)threadIdx.x + i * THREADS;
            if (g >= end) break;
            f(g, held[i]);
        }
    }
    __device__ __forceinline__ float largest_of(const Pack8<T> (&p)[kHeld], int g) const {
        float mine = -INFINITY;
        Largest<T> most;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            if (g + i * THREADS >= end) break;
            if (row.whole(g + i * THREADS)) most.take(p[i]);
            else {
#pragma unroll 1
                for (int k = 0; k < 8; ++k) mine = largest(mine, row.at(row.first(g + i * THREADS) + k));
            }
        }
        return largest(mine, most.get());
    }
    __device__ __forceinline__ float largest_of_rest() const {
        float mine = -INFINITY;
        for (int g = begin + kHeld * THREADS + (int)threadIdx.x; g < end; g += THREADS * kHeld) {
            Pack8<T> p[kHeld];
#pragma unroll
            for (int i = 0; i < kHeld; ++i) p[i] = row.fetch(g + i * THREADS, end);
            mine = largest(mine, largest_of(p, g));
        }
        return mine;
    }
    // The row's largest logit, from the threads'.
    __device__ __forceinline__ float all_largest(float mine) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mine = largest(mine, __shfl_xor_sync(0xffffffffu, mine, o));
        __syncthreads();
        if (threadIdx.x % 32 == 0) sh.maxima[threadIdx.x / 32] = mine;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) mine = largest(mine, sh.maxima[w]);
        if (blocks > 1) {
            if (threadIdx.x == 0) sh.part.best = mine;
            all_meet(blocks);
            of_blocks([](const Shared<THREADS> &b) { return b.part.best; }, [&](int, float v) { mine = largest(mine, v); });
            all_meet(blocks);                            // (nobody leaves while its word is read)
        }
        return mine;
    }
    // The least key that min_p leaves, if `top` is the largest logit.
    __device__ __forceinline__ uint32_t least_of(float top, float min_p) const {
        if (!(min_p > 0.f)) return 0;
        const double low = (double)top + log((double)fminf(min_p, 1.f)) / scale;
        float f = (float)low;
        if ((double)f < low) f = value_of(key_of(f) + 1);
        return max(key_of(f), kNegInf + 1);
    }
    // Of a granule: its logits from `low` on are listed; returns the sum of the weights, relative to `top`, in fp32's precision.  mine: the thread's
    // largest logit.
    __device__ __forceinline__ float list_and_sum(int g, const Pack8<T> &p, float low, bool sum, float top, float c, float &mine) {
        const float most = row.flat ? top : row.most(p, g);
        mine = largest(mine, most);
        float part = 0.f;
        if (sum || most >= low) {
            float v[8];
            row.get(p, g, v);
            if (sum) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float e;
                    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"((v[i] - top) * c));
                    part += e;
                }
            }
            if (most >= low) note(g, v, low, INFINITY);
        }
        return part;
    }

    // f(granule, raw form, logits, sum) for the granules of each segment, a warp's granules side by side and the whole warp in each call (behind the
    // part's end with logits of -inf); then done(segment, the lane's sum).
    template <class F, class G> __device__ __forceinline__ void each_segment(int seg_steps, F f, G done) const {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, segments = (end - begin + 32 * seg_steps - 1) / (32 * seg_steps);
        int at = begin + warp * seg_steps * 32 + lane;
        Pack8<T> next = row.fetch(at, end);
        for (int g = warp; g < segments; g += THREADS / 32) {
            u64 m = 0;
            for (int i = 0; i < seg_steps; ++i) {
                const Pack8<T> p = next;
                const int now = at;
                at += i + 1 < seg_steps ? 32 : 32 + (THREADS / 32 - 1) * seg_steps * 32;
                next = row.fetch(at, end);
                float v[8];
                if (now < end) row.get(p, now, v);
                else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = -INFINITY;
                }
                f(now, p, v, m);
            }
            done(g, m);
        }
    }
    // Lists the granule's logits in [low, high].
    __device__ __forceinline__ void note(int granule, const float (&v)[8], float low, float high) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (v[k] >= low && v[k] <= high && v[k] > -INFINITY) {
                const uint32_t place = atomicAdd(&sh.listed, 1u);
                if (place < kList) sh.list[place] = (u64)~key_of(v[k]) << 32 | (uint32_t)(row.first(granule) + k);
            }
    }

    // Adds w to bin b: a count, or a 64-bit number in two words.
    template <bool MASS> __device__ __forceinline__ void add(int b, u64 w) {
        if (!MASS) {
            atomicAdd(&sh.hist[0][b], 1u);
        } else {
            const uint32_t low = (uint32_t)w, before = atomicAdd(&sh.hist[0][b], low), high = (uint32_t)(w >> 32) + (before + low < low ? 1u : 0u);
            if (high) atomicAdd(&sh.hist[1][b], high);
        }
    }
    __device__ __forceinline__ void clear() {
        for (int i = threadIdx.x; i < 2 * kBins; i += THREADS) (&sh.hist[0][0])[i] = 0;
        __syncthreads();
    }
    // The first bin at which `above` and the bins up to it, of all blocks, reach the target; target(total) may depend on the total.  -1 if none does.
    template <bool MASS, class F> __device__ __forceinline__ void find(u64 above, F target) {
        all_meet(blocks);
        u64 bin[kPer] = {}, sum = 0;
        const auto put = [&](int i, const uint4 &w, int shift) {
            bin[4 * i] += (u64)w.x << shift;
            bin[4 * i + 1] += (u64)w.y << shift;
            bin[4 * i + 2] += (u64)w.z << shift;
            bin[4 * i + 3] += (u64)w.w << shift;
        };
        of_arrays<kPer / 4>([](const Shared<THREADS> &b) { return b.hist[0]; }, [&](int i, const uint4 &w) { put(i, w, 0); });
        if (MASS) of_arrays<kPer / 4>([](const Shared<THREADS> &b) { return b.hist[1]; }, [&](int i, const uint4 &w) { put(i, w, 32); });
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum += bin[i];
        if (threadIdx.x == 0) sh.found.bin = -1;
        u64 total;
        u64 before = above + block_scan<THREADS>(sum, sh.scan, &total);
        const u64 goal = target(total);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (before < goal && before + bin[i] >= goal) {
                sh.found.bin = threadIdx.x * kPer + i;
                sh.found.above = before;
            }
            before += bin[i];
        }
        if (threadIdx.x == 0) sh.found.total = total;
        all_meet(blocks);                                // (the histograms are read, found is written)
    }

    // The cut at which counts (or weights) of logits with keys above `floor` reach a goal, goal(total).  False if all together do not.
    template <bool MASS, class F> __device__ __forceinline__ bool narrow(uint32_t floor, F goal_of, Cut *cut, u64 *goal) {
        clear();
        each([&](float x) {
            if (key_of(x) > floor) add<MASS>(step_of(x), MASS ? weigh(x) : 1);
        });
        u64 want = 0;
        find<MASS>(0, [&](u64 total) { return want = goal_of(total); });
        *goal = want;
        int bin = sh.found.bin;
        if (bin < 0) return false;
        u64 above = sh.found.above;
        if (threadIdx.x < 2) {                           // the bin's keys: the smallest one of a step up to `bin`, and of a step before it
            const int step = bin - (int)threadIdx.x;
            uint32_t low = floor + 1, high = key_of(best) + 1;
            while (low < high) {
                const uint32_t mid = low + (high - low) / 2;
                if (step_of(value_of(mid)) <= step) high = mid; else low = mid + 1;
            }
            if (threadIdx.x == 0) sh.found.low = low; else sh.found.high = low - 1;
        }
        __syncthreads();
        uint32_t low = sh.found.low, high = sh.found.high;
        for (;;) {
            const uint32_t range = high - low;
            const int shift = max(0, 32 - __clz(range) - kLogBins);      // (range >> shift) < kBins
            clear();
            each([&](float x) {
                const uint32_t key = key_of(x);
                if (key >= low && key <= high) add<MASS>((int)((high - key) >> shift), MASS ? weigh(x) : 1);
            });
            find<MASS>(above, [&](u64) { return want; });
            bin = sh.found.bin;                          // (there is one: the interval holds the border)
            above = sh.found.above;
            const uint32_t top = high - ((uint32_t)bin << shift);
            if (shift == 0) {
                cut->key = top;
                cut->ties = MASS ? (want - above + weigh(value_of(top)) - 1) / max(weigh(value_of(top)), (u64)1) : want - above;
                return true;
            }
            const uint32_t width = (1u << shift) - 1;
            low = top - low > width ? top - width : low;
            high = top;
        }
    }

    // A key that at least `wanted` of the block's logits reach, and not many more: found among the threads' largest ones (as many threads reach
    // it).  The least key of a number where there are fewer such threads.
    __device__ __forceinline__ uint32_t bound(float mine, float least, float most, int wanted) const {
        const uint32_t key = key_of(mine);
        uint32_t low = key_of(least), high = key_of(most) + 1;
        if (low <= kNegInf) low = kNegInf + 1;
        if (__syncthreads_count(key >= low) < wanted) return kNegInf + 1;
        while (high - low > 1) {
            const uint32_t mid = low + (high - low) / 2;
            const int reach = __syncthreads_count(key >= mid);
            if (reach >= wanted) {
                low = mid;
                if (reach <= wanted + wanted / 8) break;
            } else high = mid;
        }
        return low;
    }

    // The blocks' lists, one behind the other, in the first one's; their length.
    __device__ __forceinline__ int merge() {
        int n = 0, first[8] = {}, there[8] = {};
        of_blocks([](const Shared<THREADS> &b) { return b.listed; }, [&](int o, uint32_t count) {
            first[o] = n;
            there[o] = (int)count;
            n += (int)count;
        });
        if (blocks > 1) {
            // an entry a thread, so that all are fetched at once
            for (int i = threadIdx.x; i < n; i += THREADS) {
                int o = 0, at = i;
#pragma unroll
                for (int k = 1; k < 8; ++k)
                    if (k < blocks && i >= first[k]) {
                        o = k;
                        at = i - first[k];
                    }
                if (o) sh.list[i] = at_rank(&sh, o)->list[at];
            }
        }
        __syncthreads();
        return n;
    }

    // Sorts list[0 .. n), all different: runs of 32 by a warp each (Batcher's bitonic sort, between lanes), then each entry's place is the sum of its
    // places in all runs, found by halving.  (Barriers between all the steps of one bitonic sort took five times as long: 11000 cycles for 100 entries.)
    __device__ __forceinline__ void sort(int n) {
        constexpr int kEach = kList / THREADS;
        const int lane = threadIdx.x % 32, runs = (n + 31) / 32;
        __syncthreads();
        for (int run = threadIdx.x / 32; run < runs; run += THREADS / 32) {
            const int i = run * 32 + lane;
            u64 x = i < n ? sh.list[i] : ~0ull;
#pragma unroll
            for (int size = 2; size <= 32; size *= 2)
#pragma unroll
                for (int apart = size / 2; apart > 0; apart /= 2) {
                    const u64 y = __shfl_xor_sync(0xffffffffu, x, apart);
                    const bool lower = (lane & apart) == 0, rising = (lane & size) == 0;
                    x = (x < y) == (lower == rising) ? x : y;
                }
            sh.list[i] = x;
        }
        __syncthreads();
        if (runs > 1) {
            u64 mine[kEach];
            int place[kEach];
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                const int i = k * THREADS + (int)threadIdx.x;
                if (i >= n) break;
                mine[k] = sh.list[i];
                place[k] = i % 32;
#pragma unroll 4
                for (int run = 0; run < runs; ++run) {
                    if (run == i / 32) continue;
                    const u64 *const other = sh.list + run * 32;
                    int below = 0;
#pragma unroll
                    for (int step = 16; step > 0; step /= 2) below += other[below + step - 1] < mine[k] ? step : 0;
                    place[k] += below + (other[below] < mine[k] ? 1 : 0);
                }
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kEach; ++k)
                if (k * THREADS + (int)threadIdx.x < n) sh.list[place[k]] = mine[k];
            __syncthreads();
        }
    }

    // sums[i] = value(0) + .. + value(i), i < n.
    template <class F> __device__ __forceinline__ void running(int n, F value) {
        const int per = (n + THREADS - 1) / THREADS, first = min(n, (int)threadIdx.x * per), last = min(n, first + per);
        u64 sum = 0, all;
        __syncthreads();                                 // (what value() reads is written)
        for (int i = first; i < last; ++i) sum += value(i);
        u64 before = block_scan<THREADS>(sum, sh.scan, &all);
        for (int i = first; i < last; ++i) sh.sums[i] = before += value(i);
        __syncthreads();
    }

    __device__ __forceinline__ int how_many(int n, u64 limit) const {      // of sums[0 .. n) are below limit
        int count = 0;
        for (int i = 0; i < n; i += THREADS) count += __syncthreads_count(i + (int)threadIdx.x < n && sh.sums[i + threadIdx.x] < limit);
        return count;
    }

    // Samples from the n largest logits, in list[], if these hold all that is kept.  complete: whatever is not in the list is below min_p (-inf where
    // both top_k and top_p limit).  top_k (0: none) is at most n, or the list complete.  total_low, total_high: bounds of the weights' total where no top_k gives it, equal where it
    // is known.
    __device__ __forceinline__ Outcome from_list(const SampleArgs &a, long long r, int n, bool complete, int top_k, float top_p, u64 total_low, u64 total_high, uint32_t least_key, float u) {
        if (top_p < 1.f && top_k == 0 && !complete) {    // far from enough, as of an undecided model: no need to sort
            u64 sum = 0, all;
            for (int i = threadIdx.x; i < n; i += THREADS) sum += weigh(value_of(~(uint32_t)(sh.list[i] >> 32)));
            block_scan<THREADS>(sum, sh.scan, &all);
            if (part_of(total_low, top_p, true) > all) {
                if (threadIdx.x == 0) sh.sums[n - 1] = all;
                return kNeedAll;
            }
        }
        sort(n);
        for (int i = threadIdx.x; i < n; i += THREADS) sh.weight[i] = weigh(value_of(~(uint32_t)(sh.list[i] >> 32)));
        running(n, [&](int i) { return sh.weight[i]; });
        int kept = top_k > 0 ? min(top_k, n) : n;
        if (top_p < 1.f) {
            if (top_k > 0) total_low = total_high = sh.sums[kept - 1];
            const u64 low = max((u64)1, part_of(total_low, top_p, true)), high = max((u64)1, part_of(total_high, top_p, true)), all = sh.sums[kept - 1];
            if (high > all) {                            // (for a top_k, what is asked for is there)
                if (low <= all) return kNeedTotal;
                if (!complete) return kNeedAll;
            } else {
                const int some = how_many(kept, low) + 1;
                if (low != high && how_many(kept, high) + 1 != some) return kNeedTotal;
                kept = some;
            }
        } else if (top_k == 0 && !complete) return kNeedAll;
        if (least_key) {
            int reach = 0;
            for (int i = 0; i < kept; i += THREADS) reach += __syncthreads_count(i + (int)threadIdx.x < kept && ~(uint32_t)(sh.list[i + threadIdx.x] >> 32) >= least_key);
            kept = reach;
        }
        const u64 total = sh.sums[kept - 1], target = min(part_of(total, u, false), total - 1);
        const auto answer = [&](uint32_t key, uint32_t token) {
            a.token[r] = (int32_t)token;
            if (a.logprob) a.logprob[r] = (float)(((double)value_of(key) - best) * scale - log((double)total * exp2(-(double)a.frac_bits)));
            if (a.kept) a.kept[r] = kept;
        };
        if (kept <= 128) {                               // each kept token adds up those before it
            if ((int)threadIdx.x < kept) {
                const uint32_t token = (uint32_t)sh.list[threadIdx.x];
                const u64 own = sh.weight[threadIdx.x];
                u64 before = 0;
                for (int i = 0; i < kept; ++i) before += (uint32_t)sh.list[i] < token ? sh.weight[i] : 0;
                if (target >= before && target - before < own) answer(~(uint32_t)(sh.list[threadIdx.x] >> 32), token);
            }
            return kDone;
        }
        __syncthreads();
        u64 mine[kList / THREADS];                       // by number: (token, place in weight[])
#pragma unroll
        for (int k = 0; k < kList / THREADS; ++k) {
            const int i = k * THREADS + threadIdx.x;
            if (i < kept) mine[k] = sh.list[i];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kList / THREADS; ++k) {
            const int i = k * THREADS + threadIdx.x;
            if (i < kept) {
                sh.list[i] = (u64)(uint32_t)mine[k] << 32 | (uint32_t)i;
                sh.seg.ties[i] = ~(uint32_t)(mine[k] >> 32);      // the key
            }
        }
        __syncthreads();
        sort(kept);
        running(kept, [&](int i) { return sh.weight[(uint32_t)sh.list[i]]; });
        for (int i = threadIdx.x; i < kept; i += THREADS) {
            const int place = (int)(uint32_t)sh.list[i];
            if (target < sh.sums[i] && target >= sh.sums[i] - sh.weight[place]) answer(sh.seg.ties[place], (uint32_t)(sh.list[i] >> 32));
        }
        return kDone;
    }

    // Steps for counts: of 1/128, or 1/32 for short rows.
    static constexpr int kCounts = 2 * kBins;
    static constexpr float kPerNat = kCounts / 32.f;
    __device__ __forceinline__ float count_place_of(float x) const { return fminf((best - x) * scale * kPerNat, kCounts - 1); }
    __device__ __forceinline__ int count_step_of(float x) const { return (int)count_place_of(x); }
    // The smallest key above `floor` of a step up to `step`.
    __device__ __forceinline__ uint32_t first_key(uint32_t floor, int step) const {
        uint32_t low = floor + 1, high = key_of(best) + 1;
        while (low < high) {
            const uint32_t mid = low + (high - low) / 2;
            if (count_step_of(value_of(mid)) <= step) high = mid; else low = mid + 1;
        }
        return low;
    }

    // What is kept of the logits above `floor` (and the first `ties` of it): by top_p, else by top_k (then floor is -inf's).  Counts by steps say near
    // which one the border lies; for top_p every eighth logit's place within its step is added up, too: sums by counts and mean places are
    // off by some 10^-5.  What is known already saves counting: `known` logits from `known_key` on, of the sum known_sum, and the sum of all
    // (0: not known; in units of 2^-30).  One more pass adds up the weights, exactly, of all logits and of those above the steps around the border,
    // these by segments, and lists the logits between, whose ranking gives the border (and shows whether the guess was right).
    __device__ __forceinline__ Settled general(int seg_steps, uint32_t floor, u64 ties, int top_k, float top_p, uint32_t least_key, int known, uint32_t known_key,
                                               u64 known_sum, u64 known_total) {
        constexpr int kPer = kBins / THREADS;            // bins of a thread: kPer, and as many of the second half
        uint32_t *const counts = &sh.hist[0][0];
        uint32_t *const places = reinterpret_cast<uint32_t *>(sh.weight);      // (unused meanwhile, as long as counts)
        static_assert(sizeof(sh.weight) + sizeof(sh.sums) >= kCounts * sizeof(uint32_t), "");
        for (int i = threadIdx.x; i < kCounts; i += THREADS) counts[i] = places[i] = 0;
        __syncthreads();
        const float floor_value = value_of(floor), ceiling = known ? value_of(known_key) : INFINITY;
        float low_value = floor_value;
        // Logits that weigh less than (1 - top_p) total / vocab are all together less than what top_p leaves out.
        if (known_total) low_value = fmaxf(low_value, best + (logf((1.f - top_p) * 0.999f * ((float)known_total * 0x1p-30f) / row.vocab)) / scale);
        each_granule([&](int g, const Pack8<T> &p) {
            float v[8];
            row.get(p, g, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (v[i] > low_value && v[i] < ceiling) {
                    const float t = count_place_of(v[i]);
                    const int b = (int)t;
                    atomicAdd(&counts[b], 1u);
                    if (i == 0 && top_p < 1.f) atomicAdd(&places[b], 1u << 20 | (uint32_t)((t - b) * 256.f));
                }
            }
        });
        if (threadIdx.x == 0) {
            sh.listed = 0;
            sh.found.bin = -1;
        }
        all_meet(blocks);
        uint32_t n[2 * kPer] = {}, samples[2 * kPer] = {};
        float place[2 * kPer] = {};
        u64 sum = 0, count;
        of_arrays<kPer / 2>([](const Shared<THREADS> &b) { return b.hist[0]; }, [&](int i, const uint4 &w) {
            n[4 * i] += w.x; n[4 * i + 1] += w.y; n[4 * i + 2] += w.z; n[4 * i + 3] += w.w;
        });
        if (top_p < 1.f) {
            of_arrays<kPer / 2>([](const Shared<THREADS> &b) { return b.weight; }, [&](int i, const uint4 &w) {
                const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    place[4 * i + k] += q[k] & 0xfffffu;
                    samples[4 * i + k] += q[k] >> 20;
                }
            });
        }
#pragma unroll
        for (int i = 0; i < 2 * kPer; ++i) {
            place[i] = samples[i] ? fminf(place[i] / (256.f * samples[i]), 1.f) : 0.5f;
            sum += n[i];
        }
        const u64 before = known + block_scan<THREADS>(sum, sh.scan, &count);
        if (top_p < 1.f) {
            const auto weight = [&](float step) { return exp2f(step * (-1.44269504f / kPerNat)) * 0x1p30f; };
            u64 part[2 * kPer], sum = 0, all;
#pragma unroll
            for (int i = 0; i < 2 * kPer; ++i) sum += part[i] = (u64)(n[i] * weight(threadIdx.x * 2 * kPer + i + place[i]));
            u64 at = known_sum + block_scan<THREADS>(sum, sh.scan, &all);
            all += known_sum;
            const u64 tied = ties * (u64)weight((best - floor_value) * scale * kPerNat);
            const u64 goal = part_of(known_total ? known_total : all + tied, top_p, true), low = max((u64)1, goal - (goal >> 13)), high = max((u64)1, min(goal + (goal >> 13), all));
#pragma unroll
            for (int i = 0; i < 2 * kPer; ++i) {
                if (at < low && at + part[i] >= low) sh.found.bin = threadIdx.x * 2 * kPer + i;
                if (at < high && at + part[i] >= high) sh.found.low = threadIdx.x * 2 * kPer + i;
                at += part[i];
            }
        } else {
            u64 at = before;
            if (count <= (u64)top_k && threadIdx.x == 0) sh.found.bin = -2;
#pragma unroll
            for (int i = 0; i < 2 * kPer; ++i) {
                if (count > (u64)top_k && at < (u64)top_k && at + n[i] >= (u64)top_k) sh.found.bin = sh.found.low = threadIdx.x * 2 * kPer + i;
                at += n[i];
            }
        }
        __syncthreads();
        int from = sh.found.bin, to = (int)sh.found.low;
        if (from == -2) {                                // top_k does not bind
            if (threadIdx.x == 0) {
                sh.choice.key = floor;
                sh.choice.ties = ties;
            }
            all_meet(blocks);
            return kCutOnly;
        }
        const auto bounds = [&](u64 first, u64 last) {   // steps and numbers of the logits first + 1 .. last of the ranking
            u64 at = before;
#pragma unroll
            for (int i = 0; i < 2 * kPer; ++i) {
                const u64 next = at + n[i];
                if (at <= first && next > first) {
                    sh.bracket.from = threadIdx.x * 2 * kPer + i;
                    sh.bracket.before = at;
                }
                if (at < last && next >= last) {
                    sh.bracket.to = threadIdx.x * 2 * kPer + i;
                    sh.bracket.upto = next;
                }
                at = next;
            }
        };
        u64 at = before;
#pragma unroll
        for (int i = 0; i < 2 * kPer; ++i) {
            if ((int)threadIdx.x * 2 * kPer + i == from) {
                sh.bracket.from = from;
                sh.bracket.before = at;
            }
            at += n[i];
            if ((int)threadIdx.x * 2 * kPer + i == to) {
                sh.bracket.to = to;
                sh.bracket.upto = at;
            }
        }
        __syncthreads();
        u64 above_count = sh.bracket.before, upto = sh.bracket.upto;
        if (from >= 0 && upto - above_count < kList && top_p < 1.f) {      // some more, as sums of few logits are less exact
            const u64 more = (kList - (upto - above_count)) / 8;
            __syncthreads();
            bounds(above_count - min(above_count - known, more), min(upto + more, known + count));
            __syncthreads();
            if (sh.bracket.upto - sh.bracket.before <= kList) {
                from = sh.bracket.from;
                to = sh.bracket.to;
                above_count = sh.bracket.before;
                upto = sh.bracket.upto;
            }
        }
        all_meet(blocks);                                // (the histograms are read)
        if (from < 0 || upto - above_count > kList) return kNot;
        if (threadIdx.x < 2) {
            const uint32_t key = first_key(floor, threadIdx.x == 0 ? to : from - 1);
            if (threadIdx.x == 0) sh.found.low = key; else sh.found.high = known ? min(key, known_key) - 1 : key - 1;
        }
        __syncthreads();
        const float low = value_of(sh.found.low), high = below(sh.found.high);
        const int lane = threadIdx.x % 32;
        const u64 one = (u64)__double_as_longlong(weigh.one);
        const float weightless = fmaxf(top_p < 1.f ? floor_value : high, weigh.least);
        u64 total = 0, above = 0;
        const auto summed = [&](int g, u64 m) {
            m = of_warp(m);
            if (lane == 0) {
                sh.seg.mass[g] = m;
                above += m;
            }
        };
        if (top_p < 1.f) {
            each_segment(seg_steps, [&](int at, const Pack8<T> &, const float (&v)[8], u64 &m) {
                bool some = false;
                u64 all = 0, most = 0;
                uint32_t many = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const u64 w = weigh.raw(v[k] > weightless ? v[k] : weigh.least);
                    all += w;
                    if (v[k] > high) {
                        most += w;
                        ++many;
                    } else some |= v[k] >= low;
                }
                total += all - 8 * one;
                m += most - many * one;
                if (some) note(at, v, low, high);
            }, summed);
        } else {
            each_segment(seg_steps, [&](int at, const Pack8<T> &, const float (&v)[8], u64 &m) {
                bool some = false, any = false;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (v[k] > high) any = true; else some |= v[k] >= low;
                }
                if (__any_sync(0xffffffffu, any)) {
                    u64 most = 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k) most += weigh.raw(v[k] > weightless ? v[k] : weigh.least);
                    m += most - 8 * one;
                }
                if (some) note(at, v, low, high);
            }, summed);
        }
        u64 all_total, all_above;
        block_scan<THREADS>(total, sh.scan, &all_total);
        block_scan<THREADS>(above, sh.scan, &all_above);
        if (threadIdx.x == 0) {
            sh.part.mass = all_total;
            sh.part.above = all_above;
        }
        all_meet(blocks);
        int n_list = (int)sh.listed;
        const int own_list = n_list;
        if (rank == 0) {
            total = above = 0;
            int listed = 0;
            of_blocks([](const Shared<THREADS> &b) { return b.part.mass; }, [&](int, u64 m) { total += m; });
            of_blocks([](const Shared<THREADS> &b) { return b.part.above; }, [&](int, u64 m) { above += m; });
            of_blocks([](const Shared<THREADS> &b) { return b.listed; }, [&](int o, uint32_t n) { listed += (int)min(n, (uint32_t)kList + 1); });
            const bool fits = listed <= kList;
            n_list = fits ? merge() : 0;
            sort(n_list);
            for (int i = threadIdx.x; i < n_list; i += THREADS) sh.weight[i] = weigh(value_of(~(uint32_t)(sh.list[i] >> 32)));
            running(n_list, [&](int i) { return sh.weight[i]; });
            Settled settled = fits && n_list ? kSums : kNot;
            int kept = top_k - (int)above_count;         // of the list
            uint32_t key = floor;
            u64 taken = 0;
            if (settled == kSums && top_p < 1.f) {
                const u64 tied = ties ? weigh(value_of(floor)) : 0, goal = max((u64)1, part_of(total + ties * tied, top_p, true));
                if (goal <= above) settled = kNot;
                else {
                    kept = how_many(n_list, goal - above) + 1;
                    if (kept > n_list) {                 // beyond the list: among the ties of floor, or the guess was wrong
                        settled = upto == count + known && tied ? kCutOnly : kNot;
                        if (settled == kCutOnly) taken = (goal - total + tied - 1) / tied;
                    }
                }
            }
            if (settled == kSums) {
                if (least_key) {
                    int reach = 0;
                    for (int i = 0; i < kept; i += THREADS) reach += __syncthreads_count(i + (int)threadIdx.x < kept && ~(uint32_t)(sh.list[i + threadIdx.x] >> 32) >= least_key);
                    kept = reach;
                }
                if (kept == 0) {                         // min_p cuts above the list
                    settled = kCutOnly;
                    key = least_key - 1;
                } else key = ~(uint32_t)(sh.list[kept - 1] >> 32);
            }
            if (threadIdx.x == 0) {
                sh.choice.settled = settled;
                sh.choice.key = key;
                sh.choice.ties = taken;
                sh.choice.last = settled == kSums ? (uint32_t)sh.list[kept - 1] : 0;
                sh.choice.kept = above_count + kept;
            }
        }
        all_meet(blocks);
        if (blocks > 1 && rank > 0) {
            if (threadIdx.x == 0) sh.choice = at_rank(&sh, 0)->choice;
            __syncthreads();
        }
        if (blocks > 1) all_meet(blocks);
        if (sh.choice.settled == kSums) {                // the kept ones of the list, to their segments
            const int mine = rank == 0 ? n_list : own_list;
            for (int i = threadIdx.x; i < mine; i += THREADS) {
                const uint32_t key = ~(uint32_t)(sh.list[i] >> 32), token = (uint32_t)sh.list[i];
                const int granule = (int)((token + row.skew) / 8);
                if (granule >= begin && granule < end && (key > sh.choice.key || (key == sh.choice.key && token <= sh.choice.last)))
                    atomicAdd(&sh.seg.mass[(granule - begin) / (32 * seg_steps)], weigh(value_of(key)));
            }
            __syncthreads();
        }
        return sh.choice.settled;
    }
};

template <typename T, int THREADS> __global__ void __launch_bounds__(THREADS, THREADS == 512 ? 2 : 6) sample_kernel(const __grid_constant__ SampleArgs a, int blocks) {
    __shared__ Shared<THREADS> sh;
    constexpr int kList = Sizes<THREADS>::kList;
    const int rank = blocks == 1 ? 0 : cluster_rank();
    const long long r = blockIdx.x / blocks;
    const T *const x = static_cast<const T *>(a.logits) + r * a.ld;
    const int skew = (int)(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T));
    Row<T> row{x, a.vocab, skew, false, skew > 0, (a.vocab + skew) / 8};
    const int all = (a.vocab + row.skew + 7) / 8, begin = min(all, rank * a.granules), end = min(all, begin + a.granules);
    const float scale = a.scales ? a.scales[r] : a.scale, top_p = a.top_ps ? a.top_ps[r] : a.top_p, min_p = a.min_ps ? a.min_ps[r] : a.min_p, u = a.u[r];
    int top_k = a.top_ks ? a.top_ks[r] : a.top_k;
    if (top_k >= a.vocab) top_k = 0;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    if (threadIdx.x < 32) {
        const double power = exp2((double)threadIdx.x / 32);
        sh.table[threadIdx.x] = __hiloint2double(__double2hiint(power) - ((int)threadIdx.x << 15), __double2loint(power));
    }

    Sampler<T, THREADS> s{sh, row, blocks, rank, begin, end, scale, -INFINITY, {}};
    // The first granules of each thread: the largest of their logits serves as a first guess.  The largest logits are listed where they may be all
    // that is kept: as many as top_k, or some for top_p to be reached by; how large they have to be, the threads' largest ones of the first granules
    // tell (each block its share of them), so that one pass over the row finds them; three standard deviations more of them, where the first
    // granules are not all.
    Pack8<T> held[s.kHeld];
    s.fetch_first(held);
    if (threadIdx.x == 0) sh.listed = 0;
    float mine = s.largest_of(held, begin + (int)threadIdx.x);
    const bool rest = a.granules > s.kHeld * THREADS, limited = top_k > 0;
    const bool by_k = top_k > 0 && top_k <= THREADS / 2, some = by_k || (top_k <= 0 && top_p < 1.f), unlimited = !limited && top_p >= 1.f && !(min_p > 0.f);
    const int share = ((by_k ? top_k : THREADS / 2) + blocks - 1) / blocks;
    float guess;
    uint32_t bound = kNegInf + 1;
    {
        float most = mine, least = mine;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            most = largest(most, __shfl_xor_sync(0xffffffffu, most, o));
            least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
        }
        if (lane == 0) {
            sh.maxima[warp] = most;
            sh.minima[warp] = least;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) {
            most = largest(most, sh.maxima[w]);
            least = fminf(least, sh.minima[w]);
        }
        if (some && fabsf(most) < INFINITY) {
            const float expected = share * min(1.f, (float)(s.kHeld * THREADS) / a.granules);
            bound = s.bound(mine, least, most, rest ? min(share, (int)(expected + 3.f * sqrtf(expected)) + 2) : share);
        }
        guess = most;
    }
    if (blocks > 1) {
        if (threadIdx.x == 0) {
            sh.part.best = guess;
            sh.part.bound = bound;
        }
        all_meet(blocks);
        s.of_blocks([](const Shared<THREADS> &b) { return make_uint2(__float_as_uint(b.part.best), b.part.bound); }, [&](int, uint2 w) {
            guess = largest(guess, __uint_as_float(w.x));
            bound = min(bound, w.y);
        });
        all_meet(blocks);                                // (nobody leaves while its words are read)
    }
    const float lowest = -3.402823466e38f;
    const bool lists = some || (min_p > 0.f && top_p >= 1.f), summing = top_k <= 0 && top_p < 1.f, blind = !(guess > lowest && guess < INFINITY);
    const bool lower = by_k && top_p < 1.f;              // top_k's weights are all needed for top_p
    uint32_t from = 0;
    const auto list_from = [&](uint32_t least_key) { from = some ? (lower ? bound : max(bound, least_key)) : least_key; };
    const float log2_scale = scale * 1.44269504f;
    double sum = 0.0;
    if (lists && !blind) {
        list_from(s.least_of(guess, min_p));
        const float floor = value_of(from);
        const auto take = [&](int g, const Pack8<T> &p) { sum += s.list_and_sum(g, p, floor, summing, guess, log2_scale, mine); };
        s.each_held(held, take);
        s.each_granule(take, s.kHeld * THREADS);
    } else if (rest && (!unlimited || blind)) mine = largest(mine, s.largest_of_rest());
    // (An unlimited row's other logits are read once, for their weights relative to the guess, see below.)
    float best = rest && (!unlimited || blind) ? s.all_largest(mine) : guess;
    const bool valid = scale >= 1e-6f && scale <= 1e6f && top_p == top_p && min_p == min_p && u >= 0.f && u < 1.f;
    const auto no_answer = [&] {
        if (rank == 0 && threadIdx.x == 0) {
            a.token[r] = PARLE_NO_TOKEN;
            if (a.logprob) a.logprob[r] = valid && best == -INFINITY ? -INFINITY : NAN;
            if (a.kept) a.kept[r] = 0;
            if (!valid && a.flags) atomicOr(a.flags, PARLE_FLAG_BAD_SAMPLING);
        }
    };
    if (!valid || !(fabsf(best) < INFINITY)) return no_answer();
    if (best == lowest) {
        s.row.flat = row.flat = true;
        best = 0.f;
    }
    s.best = best;
    s.weigh.set(best, scale, a.frac_bits, sh.table);
    const uint32_t least_key = s.least_of(best, min_p);

    int known = 0;                                       // logits from known_key on, listed
    uint32_t known_key = 0;
    u64 known_sum = 0, known_total = 0;                  // of weights, in units of 2^-30; 0: not known
    for (int attempt = blind ? 1 : 0; lists && attempt < 2; ++attempt) {
        float top = guess;                               // the weights summed are relative to it
        if (attempt == 1) {                              // all logits are looked at for the bound
            bound = kNegInf + 1;
            if (some) {
                if (row.flat) mine = mine > -INFINITY ? 0.f : mine;
                bound = s.bound(mine, lowest, best, share);
                if (blocks > 1) {                        // each block its share, or one of them all, where another has not that many logits
                    const uint32_t all = s.bound(mine, lowest, best, share * blocks);
                    if (threadIdx.x == 0) {
                        sh.part.bound = bound;
                        sh.part.count = all;
                    }
                    all_meet(blocks);
                    uint32_t one = 0;
                    s.of_blocks([](const Shared<THREADS> &b) { return make_uint2(b.part.bound, b.part.count); }, [&](int, uint2 w) {
                        bound = min(bound, w.x);
                        one = max(one, w.y);
                    });
                    bound = max(bound, one);
                }
            }
            list_from(least_key);
            __syncthreads();
            if (threadIdx.x == 0) sh.listed = 0;
            all_meet(blocks);
            top = best;
            sum = 0.0;
            const float floor = value_of(from);
            s.each_granule([&](int g, const Pack8<T> &p) { sum += s.list_and_sum(g, p, floor, summing, best, log2_scale, mine); });
        }
        if (summing) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            __syncthreads();
            if (lane == 0) sh.scan_f[warp] = sum;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            sum = 0.0;
            if (summing)
                for (int w = 0; w < THREADS / 32; ++w) sum += sh.scan_f[w];
            sh.part.sum = sum;
        }
        all_meet(blocks);
        // (`lower`: what min_p leaves may be listed, but top_k's other weights are missing in top_p's total)
        const bool complete = from <= (lower ? kNegInf + 1 : max(least_key, kNegInf + 1));
        int n = 0;
        s.of_blocks([](const Shared<THREADS> &b) { return b.listed; }, [&](int, uint32_t k) { n += (int)min(2u * kList + 1, k); });
        u64 low = 0, high = 0;
        bool fits = n <= kList && !(by_k && n < top_k && !complete);
        if (summing) {
            sum = 0.0;
            s.of_blocks([](const Shared<THREADS> &b) { return b.part.sum; }, [&](int, double p) { sum += p; });
            const double off_by = ((double)best - top) * log2_scale;
            if (!(sum < 1e30) || off_by > 60.0) fits = false;
            else {
                // An exponential is off by 2^-22, its argument t by 3 roundings, eight of them added by 7: (2^-22 + 2^-24 (2.1 |t| + 8)) w; and
                // sum w |t|, t relative to the largest logit, is at most sum w log2(vocab / sum w), as no distribution's entropy is above log2 vocab.
                sum *= exp2(-off_by);
                const double off = sum * 0x1p-24 * (14.0 + 2.1 * (max(0.0, log2((double)a.vocab / sum)) + off_by)), unit = exp2((double)a.frac_bits);
                low = (u64)fmax((sum - off) * unit - a.vocab, 0.0);      // (whole numbers: each may be half of one less, or more)
                high = (u64)((sum + off) * unit) + (u64)a.vocab;
                known_total = (u64)(sum * 0x1p30);
            }
        }
        if (!fits) {
            all_meet(blocks);                            // (the blocks' numbers are read)
            if (!rest || (!some && n > 2 * kList)) break;      // (the bound was that of all logits; min_p leaves far too many)
            continue;
        }
        Outcome outcome = kNeedAll;
        if (rank == 0) {
            s.merge();
            outcome = s.from_list(a, r, n, complete, max(top_k, 0), top_p, low, high, least_key, u);
        }
        const auto agree = [&] {                         // on rank 0's outcome
            if (threadIdx.x == 0) {
                sh.outcome = outcome;
                sh.part.above = sh.sums[n - 1];
            }
            all_meet(blocks);
            outcome = s.block(0)->outcome;
            known_sum = s.block(0)->part.above >> (a.frac_bits - 30);
            all_meet(blocks);
        };
        agree();
        if (outcome == kDone) return;
        if (outcome == kNeedTotal) {                     // (the list stays as it is: sorted, at rank 0)
            u64 mass = 0;
            s.each([&](float v) { mass += s.weigh(v); });
            u64 all;
            block_scan<THREADS>(mass, sh.scan, &all);
            if (threadIdx.x == 0) sh.part.mass = all;
            all_meet(blocks);
            if (rank == 0) {
                all = 0;
                s.of_blocks([](const Shared<THREADS> &b) { return b.part.mass; }, [&](int, u64 m) { all += m; });
                outcome = s.from_list(a, r, n, complete, 0, top_p, all, all, least_key, u);
            }
            agree();
            if (outcome == kDone) return;
        }
        if (summing) {
            known = n;
            known_key = from;
        }
        break;
    }

    Cut cut{kNegInf, 0, false, 0};
    u64 goal;
    bool summed = false;                                 // the segments' sums are there
    if (limited && top_p < 1.f) {
        Cut c;
        if (s.template narrow<false>(kNegInf, [&](u64) { return (u64)top_k; }, &c, &goal)) cut = Cut{c.key, c.ties, false, 0};
    }
    if (limited || top_p < 1.f) {
        const Settled settled = s.general(a.seg_steps, cut.key, cut.ties, limited ? top_k : 0, top_p, least_key, known, known_key, known ? known_sum : 0, known_total);
        if (settled == kSums) {
            cut = Cut{sh.choice.key, 0, true, sh.choice.last};
            summed = true;
        } else if (settled == kCutOnly) {
            cut = Cut{sh.choice.key, sh.choice.ties, false, 0};
        } else if (top_p < 1.f) {
            const u64 tied = cut.ties ? s.weigh(value_of(cut.key)) : 0;
            Cut c;
            const bool inside = s.template narrow<true>(cut.key, [&](u64 total) { return max((u64)1, part_of(total + cut.ties * tied, top_p, true)); }, &c, &goal);
            if (inside) cut = Cut{c.key, c.ties, false, 0};
            else if (tied) cut.ties = (goal - sh.found.total + tied - 1) / tied;
        } else {
            Cut c;
            if (s.template narrow<false>(kNegInf, [&](u64) { return (u64)top_k; }, &c, &goal)) cut = Cut{c.key, c.ties, false, 0};
        }
    }
    if (least_key > cut.key) cut = Cut{least_key - 1, 0, false, 0};

    // Sums of the kept weights by segments of the row, in its order.
    const int segments = (end - begin + 32 * a.seg_steps - 1) / (32 * a.seg_steps);
    u64 mass = 0;
    uint32_t count = 0, ties = 0;
    if (summed) {
        for (int g = threadIdx.x; g < segments; g += THREADS) {
            mass += sh.seg.mass[g];
            sh.seg.ties[g] = 0;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, o);
    } else {
        __syncthreads();
        const u64 one = (u64)__double_as_longlong(s.weigh.one);
        if (unlimited) {
            // All logits are kept.  Where the largest one is not known yet, weights are relative to the guess, and the largest logit is found beside
            // them.  The sums stand if a thread's of a segment fit into 64 bits (w < e^10, at most
            // vocab / 2^15 or 32 of them) and so do all (their fp64 sum is below 2^62), else they are formed again.
            for (;;) {
                sum = 0.0;
                s.each_segment(a.seg_steps, [&](int g, const Pack8<T> &, const float (&v)[8], u64 &m) {
                    const float most = largest(largest(largest(v[0], v[1]), largest(v[2], v[3])), largest(largest(v[4], v[5]), largest(v[6], v[7])));
                    mine = largest(mine, most);
                    u64 part = 0;
                    if (most > s.weigh.most) {
#pragma unroll 1
                        for (int k = 0; k < 8; ++k) part += s.weigh(row.at(row.first(g) + k));
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) part += s.weigh.raw(fmaxf(v[k], s.weigh.least));
                        part -= 8 * one;
                    }
                    m += part;
                    if (fminf(fminf(fminf(v[0], v[1]), fminf(v[2], v[3])), fminf(fminf(v[4], v[5]), fminf(v[6], v[7]))) > -INFINITY) count += 8;
                    else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) count += v[k] > -INFINITY;
                    }
                }, [&](int g, u64 m) {
                    sum += (double)m;
                    m = of_warp(m);
                    if (lane == 0) {
                        sh.seg.mass[g] = m;
                        sh.seg.ties[g] = 0;
                        mass += m;
                    }
                });
                if (!rest || blind) break;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (lane == 0) sh.scan_f[warp] = sum;
                const float top = s.all_largest(mine);   // (a barrier between)
                if (!(fabsf(top) < INFINITY)) {
                    best = top;
                    return no_answer();
                }
                if (top == best) break;
                if (threadIdx.x == 0) {
                    sum = 0.0;
                    for (int w = 0; w < THREADS / 32; ++w) sum += sh.scan_f[w];
                    sh.part.sum = sum;
                }
                all_meet(blocks);
                sum = 0.0;
                s.of_blocks([](const Shared<THREADS> &b) { return b.part.sum; }, [&](int, double p) { sum += p; });
                all_meet(blocks);
                if (((double)top - best) * scale < 10.0 && sum < 0x1p62) break;
                s.best = best = top;
                s.weigh.set(best, scale, a.frac_bits, sh.table);
                mass = 0;
                count = 0;
            }
        } else {
            const float border = below(cut.key), weightless = fmaxf(border, s.weigh.least);      // (the key of ties is a logit's)
            uint32_t t = 0;
            s.each_segment(a.seg_steps, [&](int, const Pack8<T> &, const float (&v)[8], u64 &m) {
                bool some = false;
                if (cut.ties) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) t += v[k] == border;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    some |= v[k] > border;
                    count += v[k] > border;
                }
                if (!__any_sync(0xffffffffu, some)) return;
                u64 part = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) part += s.weigh.raw(v[k] > weightless ? v[k] : s.weigh.least);
                m += part - 8 * one;
            }, [&](int g, u64 m) {
                m = of_warp(m);
                const uint32_t equal = cut.ties ? __reduce_add_sync(0xffffffffu, t) : 0;
                t = 0;
                if (lane == 0) {
                    sh.seg.mass[g] = m;
                    sh.seg.ties[g] = equal;
                    mass += m;
                    ties += equal;
                }
            });
        }
        count = __reduce_add_sync(0xffffffffu, count);
    }
    // the block's own sums
    if (threadIdx.x == 0) sh.part = Part{best, 0, 0.0, 0, 0, 0, 0};
    __syncthreads();
    if (lane == 0) {
        atomicAdd(&sh.part.mass, mass);
        atomicAdd(&sh.part.count, count);
        atomicAdd(&sh.part.ties, ties);
    }
    all_meet(blocks);
    const u64 tied = cut.ties || cut.by_last ? s.weigh(value_of(cut.key)) : 0;
    const auto of_ties = [&](u64 before, uint32_t there) { return before >= cut.ties ? (u64)0 : min(cut.ties - before, (u64)there); };
    u64 total = 0, mass_before = 0, ties_before = 0, all_ties = 0, kept = 0, own = 0;
    s.of_blocks([](const Shared<THREADS> &b) { return b.part; }, [&](int o, const Part &p) {
        const u64 taken = of_ties(all_ties, p.ties), there = p.mass + taken * tied;
        if (o == rank) { mass_before = total; ties_before = all_ties; own = there; }
        total += there;
        all_ties += p.ties;
        kept += p.count + taken;
    });
    if (summed) kept = sh.choice.kept;
    const u64 target = min(part_of(total, u, false), total - 1);
    if (target >= mass_before && target - mass_before < own) {      // the token lies in this block's part
        constexpr int kPer = Sizes<THREADS>::kSegments / THREADS;
        u64 t[kPer], m[kPer], sum = 0, any;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int g = threadIdx.x * kPer + i;
            sum += t[i] = g < segments ? sh.seg.ties[g] : 0;
        }
        u64 before = ties_before + block_scan<THREADS>(sum, sh.scan, &any);
        sum = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int g = threadIdx.x * kPer + i;
            sum += m[i] = (g < segments ? sh.seg.mass[g] : 0) + of_ties(before, (uint32_t)t[i]) * tied;
            before += t[i];
        }
        for (int i = 0; i < kPer; ++i) before -= t[i];
        u64 below = mass_before + block_scan<THREADS>(sum, sh.scan, &any);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (target >= below && target - below < m[i]) {
                sh.hit.segment = threadIdx.x * kPer + i;
                sh.hit.target = target - below;
                sh.hit.ties_before = (uint32_t)min(before, (u64)0xffffffffu);
            }
            below += m[i];
            before += t[i];
        }
        __syncthreads();
        if (warp == 0) {
            u64 rest = sh.hit.target, tb = sh.hit.ties_before;
            for (int i = 0; i < a.seg_steps; ++i) {
                const int at = begin + (sh.hit.segment * a.seg_steps + i) * 32 + lane;
                float v[8];
                uint32_t mine = 0;
                u64 w[8], sum = 0;
                if (at < end) row.load(at, v);
                else
                    for (int k = 0; k < 8; ++k) v[k] = -INFINITY;
#pragma unroll
                for (int k = 0; k < 8; ++k) mine += key_of(v[k]) == cut.key;
                uint32_t upto = mine;
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const uint32_t b = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += b;
                }
                u64 at_tie = tb + upto - mine;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t key = key_of(v[k]);
                    w[k] = key > cut.key ? s.weigh(v[k]) : key == cut.key && (cut.by_last ? (uint32_t)(row.first(at) + k) <= cut.last : at_tie++ < cut.ties) ? tied : 0;
                    sum += w[k];
                }
                u64 sums = sum;
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const u64 b = shfl_up64(sums, o);
                    if (lane >= o) sums += b;
                }
                u64 before_lane = sums - sum;
                if (rest >= before_lane && rest < sums) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (rest >= before_lane && rest - before_lane < w[k]) {
                            a.token[r] = (int32_t)(row.first(at) + k);
                            if (a.logprob) a.logprob[r] = (float)(((double)v[k] - best) * scale - log((double)total * exp2(-(double)a.frac_bits)));
                        }
                        before_lane += w[k];
                    }
                }
                const u64 whole = __shfl_sync(0xffffffffu, sums, 31);
                if (rest < whole) break;
                rest -= whole;
                tb += __shfl_sync(0xffffffffu, upto, 31);
            }
        }
    }
    if (rank == 0 && threadIdx.x == 0 && a.kept) a.kept[r] = (int32_t)kept;
    if (blocks > 1) all_meet(blocks);                    // (nobody leaves while its sums are read)
}

template <typename T, int THREADS> int launch_sample(SampleArgs a, int blocks, cudaStream_t stream) {
    const int granules = a.vocab / 8 + 2;                // wherever a row begins
    a.seg_steps = blocks == 1 && granules >= 128 * (THREADS / 32) ? 4 : 1;      // (adding up a segment over a warp takes as long as half a step)
    for (;;) {
        const int each = 32 * a.seg_steps;
        a.granules = ((granules + blocks - 1) / blocks + each - 1) / each * each;
        if (a.granules / each <= Sizes<THREADS>::kSegments) break;
        a.seg_steps *= 2;
    }
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = cluster_config(dim3((unsigned)(a.rows * blocks)), THREADS, 0, blocks, &attr, stream);
    if (cudaLaunchKernelEx(&cfg, sample_kernel<T, THREADS>, a, blocks) != cudaSuccess) {
        cudaGetLastError();
        return PARLE_ECUDA;
    }
    return PARLE_OK;
}

bool aligned4(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

}  // namespace

extern "C" int parle_sample_tokens(const void *logits, int dtype, long long rows, int vocab, long long ld, const float *u,
                                   const parle_sampling *sampling, int32_t *token, float *logprob, int32_t *kept, int32_t *flags, void *cuda_stream) {
    if (!valid_dtype(dtype) || rows < 0 || vocab < 1 || (rows > 1 && ld < 0) || !sampling) return PARLE_EINVAL;
    const parle_sampling &h = *sampling;
    const float scale = (float)h.scale, top_p = (float)h.top_p, min_p = (float)h.min_p;
    if (!h.scales && !(h.scale >= 1e-6 && h.scale <= 1e6)) return PARLE_EINVAL;
    if (!h.top_ks && h.top_k < 0) return PARLE_EINVAL;
    if ((!h.top_ps && !(h.top_p >= 0.0 && h.top_p <= 1.0)) || (!h.min_ps && !(h.min_p >= 0.0 && h.min_p <= 1.0))) return PARLE_EINVAL;
    if (rows == 0) return PARLE_OK;
    if (!logits || !u || !token) return PARLE_EINVAL;
    if (rows > PARLE_TOKEN_MAX_ROWS / 8 || vocab > 1 << 30) return PARLE_ETOOBIG;
    if (!element_aligned(logits, dtype) || !aligned4(u) || !aligned4(h.scales) || !aligned4(h.top_ks) || !aligned4(h.top_ps) || !aligned4(h.min_ps) ||
        !aligned4(token) || !aligned4(logprob) || !aligned4(kept) || !aligned4(flags)) return PARLE_EALIGN;
    SampleArgs a = {};
    a.logits = logits; a.rows = rows; a.ld = ld; a.vocab = vocab;
    a.scale = fminf(fmaxf(scale, 1e-6f), 1e6f); a.top_p = top_p; a.min_p = min_p; a.top_k = h.top_k;
    a.u = u; a.scales = h.scales; a.top_ks = h.top_ks; a.top_ps = h.top_ps; a.min_ps = h.min_ps;
    a.token = token; a.logprob = logprob; a.kept = kept; a.flags = flags;
    a.frac_bits = 44;
    while (a.frac_bits > 8 && ((unsigned long long)vocab >> (63 - a.frac_bits))) --a.frac_bits;      // sums stay below 2^63
    const int sms = current_sms();
    if (sms < 0) return PARLE_ECUDA;
    int blocks = 1;
    while (blocks < 8 && rows * blocks * 2 <= 2 * sms && vocab / blocks >= 16384) blocks *= 2;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return with_dtype(dtype, [&](auto *tag) {
        using T = std::remove_pointer_t<decltype(tag)>;
        return vocab <= 4096 ? launch_sample<T, 128>(a, blocks, stream) : launch_sample<T, 512>(a, blocks, stream);
    });
}
