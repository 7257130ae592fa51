// parle_token_logprobs, parle_token_logprobs_grad: per row of logits x[0 .. V),
//
//   log p_j = s (x_j - m) - log S,   m = max x,  S = sum_j exp(s (x_j - m))
//   log p of a given token t, entropy H = -sum_j p_j log p_j = log S - (1/S) sum_j e_j d_j   (d_j = s (x_j - m), e_j = exp d_j),
//   the k most probable tokens (ties: lower token first), and
//   d/dx_j (g log p_t + h H) = s ( g (1[j = t] - p_j) - h p_j (log p_j + H) ).
//
// A row is read once by one block (or, when there are few rows, by the blocks of one cluster), in 16-byte granules cut at
// 16-byte boundaries of memory, so rows of any pitch are read with wide loads; only a row's first and last granule may be
// partial and are read by element.  Maximum, sum and sum of e d are carried together ("online": when a thread meets a larger
// maximum it rescales its two sums), all in fp32.  Exponentials are base 2: e_j = 2^(x_j c - R) with c = s log2(e), one fused
// multiply-add per argument, where the reference R is the rounded product of c and the largest logit so far.  R's rounding is
// common to every term of the row and to log S, so it cancels.
#include <math.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "token_types.cuh"

using namespace parle;

namespace {

constexpr int kTopMost = PARLE_TOP_MAX;
constexpr int kCandidates = 512;        // logits at least as large as the bound that are ranked at once
constexpr int kClusterMost = 8;

struct RowsArgs {
    const void *logits;
    const int32_t *tokens;
    long long ld, rows;
    int vocab, k;
    float scale, scale_log2e;                              // s, s log2(e)
    float *logprob, *entropy, *top_logprob;
    int32_t *top_token, *flags;
    const float *d_logprob, *d_entropy;
    void *dlogits;
    long long ld_d;
};

__device__ __forceinline__ float exp2_approx(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// Two fp32 numbers in one register pair: one instruction for two products, sums or multiply-adds.
typedef unsigned long long float_pair;
__device__ __forceinline__ float_pair pair(float lo, float hi) {
    float_pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split(float_pair v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ float_pair fma2(float_pair a, float_pair b, float_pair c) {
    float_pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float_pair add2(float_pair a, float_pair b) {
    float_pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float_pair mul2(float_pair a, float_pair b) {
    float_pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Scaled logits x c below -kFar count as -kFar (their probability is 0 either way, and 0 * -inf does not arise in the sum of
// e d); references below -kNear as -kNear.  Rows whose largest scaled logit is not between -kNear and kNear -- all masked with
// -inf or large negative numbers, or with very large logits -- are summed again with (x - max) c ("far"): there the reference's
// rounding, 2^-24 of it, would shift the exponents by more than 2^-4.
constexpr float kFar = 2097152.f, kNear = 1048576.f;      // 2^21, 2^20

template <typename T> struct Granule;
template <typename T, int U> __device__ __forceinline__ float largest_of(const Granule<T> (&g)[U]);

// 16 bytes of logits.
template <typename T> struct Granule {
    static constexpr int N = 16 / sizeof(T);
    uint4 raw;
    __device__ __forceinline__ void fill_none() {        // -inf everywhere
        const uint32_t w = sizeof(T) == 4 ? 0xff800000u : (std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u);
        raw = make_uint4(w, w, w, w);
    }
    __device__ __forceinline__ void get(float (&v)[N]) const {
        if constexpr (sizeof(T) == 4) {
            v[0] = __uint_as_float(raw.x); v[1] = __uint_as_float(raw.y); v[2] = __uint_as_float(raw.z); v[3] = __uint_as_float(raw.w);
        } else {
            Pack8<T> p;
            p.a = raw;
            p.get(v);
        }
    }
    // As pairs, not below `low` (low_bound()); NaN stays.
    __device__ __forceinline__ void pairs(uint32_t low, float_pair (&v)[N / 2]) const {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        if constexpr (sizeof(T) == 4) {
            v[0] = pair(clamped(__uint_as_float(w[0]), low), clamped(__uint_as_float(w[1]), low));
            v[1] = pair(clamped(__uint_as_float(w[2]), low), clamped(__uint_as_float(w[3]), low));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (std::is_same<T, __half>::value) {      // fp16 has no number below the references: clamped as fp32
                    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                    v[i] = pair(clamped(f.x, low), clamped(f.y, low));
                } else {
                    uint32_t u;
                    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(u) : "r"(w[i]), "r"(low));
                    v[i] = pair(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
                }
            }
        }
    }
    __device__ __forceinline__ static float clamped(float v, uint32_t low) {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(__uint_as_float(low)));
        return r;
    }
    __device__ __forceinline__ float largest() const { return largest_of<T, 1>({*this}); }
    // of the elements of even and of odd number
    __device__ __forceinline__ void largest_two(float &even, float &odd) const {
        if constexpr (sizeof(T) == 4) {
            even = fmaxf(__uint_as_float(raw.x), __uint_as_float(raw.z));
            odd = fmaxf(__uint_as_float(raw.y), __uint_as_float(raw.w));
        } else {
            using T2 = std::conditional_t<std::is_same<T, __half>::value, __half2, __nv_bfloat162>;
            const T2 *h = reinterpret_cast<const T2 *>(&raw), m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
            even = to_float(m.x);
            odd = to_float(m.y);
        }
    }
};

// Largest element of some granules; NaN is passed over (the sums carry it).
template <typename T, int U> __device__ __forceinline__ float largest_of(const Granule<T> (&g)[U]) {
    if constexpr (sizeof(T) == 4) {
        float m = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
            m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(g[u].raw.x), __uint_as_float(g[u].raw.y)),
                               fmaxf(__uint_as_float(g[u].raw.z), __uint_as_float(g[u].raw.w))));
        return m;
    } else {
        using T2 = std::conditional_t<std::is_same<T, __half>::value, __half2, __nv_bfloat162>;
        T2 m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const T2 *h = reinterpret_cast<const T2 *>(&g[u].raw);
            const T2 v = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
            m = u ? __hmax2(m, v) : v;
        }
        return fmaxf(to_float(m.x), to_float(m.y));
    }
}

// The bound -kFar / c, as Granule::pairs() takes it: an fp32 number, or two bf16 ones.
template <typename T> __device__ __forceinline__ uint32_t low_bound(float c) {
    const uint32_t w = __float_as_uint(-kFar / c);
    if constexpr (!std::is_same<T, __nv_bfloat16>::value) return w;
    return (w >> 16) | (w & 0xffff0000u);                 // towards zero
}

// A row as granules: granule q is base[q] and holds elements q N - head .. q N - head + N - 1.
template <typename T> struct Row {
    static constexpr int N = Granule<T>::N;
    const uint4 *base;
    int vocab, head, granules;
    int first_whole, wholes;                              // granules that lie in the row altogether: consecutive
    __device__ __forceinline__ Row(const void *logits, long long ld, long long row, int vocab_) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(static_cast<const T *>(logits) + row * ld);
        base = reinterpret_cast<const uint4 *>(at & ~(uintptr_t)15);
        vocab = vocab_;
        head = (int)((at & 15) / sizeof(T));
        granules = (head + vocab + N - 1) / N;
        first_whole = head ? 1 : 0;
        wholes = (head + vocab) / N - first_whole;        // (-1 for a row inside one granule)
    }
    __device__ __forceinline__ const T *x() const { return reinterpret_cast<const T *>(base) + head; }
    __device__ __forceinline__ int first_element(int q) const { return q * N - head; }
    __device__ __forceinline__ bool whole(int q) const { return q >= first_whole && q - first_whole < wholes; }
    __device__ __forceinline__ bool all_whole(int first, int last, int end) const {
        return first >= first_whole && last - first_whole < wholes && last < end;
    }
    // The granule that holds an element.
    __device__ __forceinline__ int granule_of(int element) const { return (element + head) / N; }
    __device__ __forceinline__ Granule<T> load(int q, int end) const {
        Granule<T> g;
        if (q >= end) { g.fill_none(); return g; }
        if (whole(q)) {
            g.raw = base[q];
        } else {
            g.fill_none();
            T *v = reinterpret_cast<T *>(&g.raw);
            const int e0 = first_element(q);
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (e0 + i >= 0 && e0 + i < vocab) v[i] = x()[e0 + i];
        }
        return g;
    }
    // U granules, `step` apart, that belong to one thread; granules from `end` on are -inf.
    template <int U> __device__ __forceinline__ void load_all(int q0, int step, int end, Granule<T> (&raw)[U]) const {
        if (all_whole(q0, q0 + (U - 1) * step, end)) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u].raw = base[q0 + u * step];
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = load(q0 + u * step, end);
        }
    }
};

// Reference R, sum of e = 2^(x c - R) and sum of e (x c - R) over some logits.
struct Sums {
    float r, s, a;
    __device__ __forceinline__ void clear() { r = -kNear; s = 0.f; a = 0.f; }
    // The same sums relative to a reference `to` >= r.
    __device__ __forceinline__ void rebase(float to) {
        const float shift = r - to, f = exp2_approx(shift);
        a = f == 0.f ? 0.f : f * fmaf(shift, s, a);
        s *= f;                                           // (a NaN stays)
        r = to;
    }
};

// Orders (logit, token) pairs: larger logit first, then the lower position.
__device__ __forceinline__ unsigned long long order_key(float v, uint32_t position) {
    const uint32_t u = __float_as_uint(v + 0.f);         // -0 counts as 0
    const uint32_t o = (u >> 31) ? ~u : (u | 0x80000000u);
    return ((unsigned long long)o << 32) | (uint32_t)~position;
}
__device__ __forceinline__ float key_value(unsigned long long key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float((o >> 31) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ int key_token(unsigned long long key) { return (int)~(uint32_t)key; }

__device__ __forceinline__ void cluster_sync_all() {
    cluster_arrive();
    cluster_wait();
}

template <int BLOCK> struct SharedSums {
    Sums warp[BLOCK / 32];
    Sums block;                                           // read by the other blocks of its cluster
};

template <int BLOCK> struct Shared : SharedSums<BLOCK> {
    // groups of logits whose maxima bound the k-th largest from below (a warp's: 32, or two a thread)
    static constexpr int kGroups = BLOCK < 64 ? BLOCK : 64;
    alignas(16) unsigned long long group[BLOCK < 64 ? 64 : BLOCK];      // the threads' best (logit, granule)
    unsigned long long bound;
    int found, owners;
    int owner[BLOCK];
    unsigned long long candidate[kCandidates];
    unsigned long long top[kTopMost];
};

// The sums of all 32 lanes, in every lane: one rescaling to the largest reference, then plain sums.
__device__ __forceinline__ Sums warp_sums(Sums t) {
    float to = t.r;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, o));
    t.rebase(to);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        t.s += __shfl_xor_sync(0xffffffffu, t.s, o);
        t.a += __shfl_xor_sync(0xffffffffu, t.a, o);
    }
    return t;
}

// Sums over a block, the same in every thread.  (What a thread wrote to shared memory before is visible to all after.)
template <int BLOCK> __device__ __forceinline__ Sums block_sums(Sums t, SharedSums<BLOCK> &sh) {
    t = warp_sums(t);
    if constexpr (BLOCK == 32) {
        __syncwarp();
        return t;
    }
    if (threadIdx.x % 32 == 0) sh.warp[threadIdx.x / 32] = t;
    __syncthreads();
    t.clear();
    if (threadIdx.x % 32 < BLOCK / 32) t = sh.warp[threadIdx.x % 32];
    return warp_sums(t);
}

// The k largest of a block's logits.
//
// The k-th largest of 64 thread groups' maxima is a lower bound of the k-th largest logit, and only threads whose own maximum
// reaches it can hold one of the k: they hand their logits above the bound on (typically k to 2 k of them), which are ranked by
// counting.  Equal maxima are ordered by granule, so a row of equal logits hands on k granules, not all.

// Before block_sums(): every thread's largest (logit, granule), 0 if it has none above -inf.
template <int BLOCK> __device__ __forceinline__ void offer_best(unsigned long long best, Shared<BLOCK> &sh) {
    sh.group[threadIdx.x] = best;
    if (threadIdx.x < kTopMost) sh.top[threadIdx.x] = 0;
    if (threadIdx.x == 0) { sh.found = 0; sh.owners = 0; sh.bound = 0; }
}

// The same with two groups a thread, for rows of one warp: its logits of even and of odd number, as (logit, 2 granule + 0 or 1).
__device__ __forceinline__ void offer_two(unsigned long long even, unsigned long long odd, Shared<32> &sh) {
    offer_best<32>(even, sh);
    sh.group[threadIdx.x + 32] = odd;
}

// After it: the bound, as (logit, granule); 0 where fewer than G groups' k have a logit.  No two groups' keys are the same, but for 0.
template <int G, int BLOCK> __device__ __forceinline__ unsigned long long top_bound(int k, Shared<BLOCK> &sh) {
    if constexpr (BLOCK < G) {                            // two groups a thread
        const ulonglong2 g = *reinterpret_cast<const ulonglong2 *>(&sh.group[2 * threadIdx.x]);
        int above0 = 0, above1 = 0;
#pragma unroll
        for (int t = 0; t < G; t += 2) {
            const ulonglong2 o = *reinterpret_cast<const ulonglong2 *>(&sh.group[t]);
            above0 += (o.x > g.x) + (o.y > g.x);
            above1 += (o.x > g.y) + (o.y > g.y);
        }
        if (above0 == k - 1) sh.bound = g.x;
        if (above1 == k - 1) sh.bound = g.y;
    } else {
        constexpr int PARTS = BLOCK / G;
        if constexpr (PARTS > 1) {
            if (threadIdx.x < G) {
                unsigned long long g = sh.group[threadIdx.x];
#pragma unroll
                for (int t = threadIdx.x + G; t < BLOCK; t += G) g = max(g, sh.group[t]);
                sh.group[threadIdx.x] = g;
            }
            __syncthreads();
        }
        const int i = threadIdx.x / PARTS, part = threadIdx.x % PARTS;
        const unsigned long long g = sh.group[i];
        int above = 0;
#pragma unroll
        for (int t = part; t < G; t += PARTS) above += sh.group[t] > g;
#pragma unroll
        for (int o = PARTS / 2; o > 0; o >>= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
        if (above == k - 1 && part == 0) sh.bound = g;
    }
    __syncthreads();
    return sh.bound;
}

// Hands on a granule's logits that reach the bound.  TWO: all of them at the even group's place, whatever their own group, since the
// bound orders equal logits of one granule by group and the alternatives are ordered by token.  What is left behind is then smaller
// than the bound's logit, or equal to it in a later granule: k larger or earlier ones exist.  (The thread that holds what is handed on
// reaches the bound: if only the odd group's place does not, the bound is the thread's own even group.)
template <bool TWO = false, typename T, int BLOCK>
__device__ __forceinline__ void hand_on(const Row<T> &row, const Granule<T> &raw, int q, unsigned long long bound, Shared<BLOCK> &sh) {
    constexpr int N = Granule<T>::N;
    const uint32_t place = TWO ? 2 * q : q;
    if (order_key(raw.largest(), place) < bound) return;  // (a granule of NaN alone compares either way)
    float v[N];
    raw.get(v);
    const int e0 = row.first_element(q);
    uint32_t reach = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (v[i] > -INFINITY && order_key(v[i], place) >= bound) reach |= 1u << i;      // (beside the row lies -inf)
    if (!reach) return;
    int at = atomicAdd(&sh.found, __popc(reach));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (!((reach >> i) & 1u)) continue;
        if (at < kCandidates) sh.candidate[at] = order_key(v[i], (uint32_t)(e0 + i));
        ++at;
    }
}

// Ranks what was handed on (after a barrier): the k largest, best first, into sh.top; 0 where there are fewer.
template <typename T, int BLOCK>
__device__ __forceinline__ void rank_candidates(const Row<T> &row, int begin, int end, int k, Shared<BLOCK> &sh) {
    constexpr int PARTS = 4;
    const int found = sh.found;
    if (found <= kCandidates) {
        for (int i0 = 0; i0 < found; i0 += BLOCK / PARTS) {
            const int i = i0 + (int)threadIdx.x / PARTS;
            const unsigned long long key = i < found ? sh.candidate[i] : 0;
            int above = 0;
#pragma unroll 8
            for (int j = threadIdx.x % PARTS; j < found; j += PARTS) above += sh.candidate[j] > key;
#pragma unroll
            for (int o = PARTS / 2; o > 0; o >>= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
            if (i < found && above < k) sh.top[above] = key;
        }
    } else {
        // too many logits above the bound (large ones gathered in few groups): one pass over the block's logits per rank.  200 rows of
        // 65536 bf16 logits whose large ones lie in three of every 64 granules, 32 alternatives: 543 us, ordinary ones 12.5
        constexpr int N = Granule<T>::N;
        unsigned long long last = ~0ull;
        for (int r = 0; r < k; ++r) {
            unsigned long long mine = 0;
            for (int q = begin + threadIdx.x; q < end; q += BLOCK) {
                float v[N];
                row.load(q, end).get(v);
                const int e0 = row.first_element(q);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const unsigned long long key = order_key(v[i], (uint32_t)(e0 + i));
                    if (v[i] > -INFINITY && key < last && key > mine) mine = key;
                }
            }
            for (int o = 16; o > 0; o >>= 1) mine = max(mine, __shfl_xor_sync(0xffffffffu, mine, o));
            __syncthreads();
            if (threadIdx.x % 32 == 0) sh.group[threadIdx.x / 32] = mine;
            __syncthreads();
            for (int w = 0; w < BLOCK / 32; ++w) mine = max(mine, sh.group[w]);
            if (threadIdx.x == 0) sh.top[r] = mine;
            last = mine;
        }
    }
    __syncthreads();
}

// A thread's sums while it goes over granules, U at a time.
template <typename T> struct Online {
    static constexpr int P = Granule<T>::N / 2;
    Sums t;
    float top;                                            // largest logit so far, and the first granule that holds it
    int best;
    float c;
    uint32_t low;
    float_pair s2, a2;
    __device__ __forceinline__ explicit Online(float c_) : top(-INFINITY), best(-1), c(c_), low(low_bound<T>(c_)) {
        t.clear();
        s2 = a2 = pair(0.f, 0.f);
    }
    template <int U> __device__ __forceinline__ void add(const Granule<T> (&raw)[U], int q0, int step) {
        const float most = largest_of(raw);
        if (most > top) {                                 // rare after the first granules
#pragma unroll
            for (int u = U - 1; u >= 0; --u)
                if (raw[u].largest() == most) best = q0 + u * step;
            top = most;
            const float to = fmaxf(top * c, -kNear);
            if (to > t.r) {
                collect();
                t.rebase(to);
                s2 = pair(t.s, 0.f);
                a2 = pair(t.a, 0.f);
            }
        }
        const float_pair c2 = pair(c, c), r2 = pair(-t.r, -t.r);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float_pair x[P];
            raw[u].pairs(low, x);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float_pair d = fma2(x[i], c2, r2);
                float lo, hi;
                split(d, lo, hi);
                const float_pair e = pair(exp2_approx(lo), exp2_approx(hi));
                s2 = add2(s2, e);
                a2 = fma2(e, d, a2);
            }
        }
    }
    __device__ __forceinline__ const Sums &collect() {
        float lo, hi;
        split(s2, lo, hi); t.s = lo + hi;
        split(a2, lo, hi); t.a = lo + hi;
        return t;
    }
};

// First pass over a row: the next U granules are on their way while U are summed.
template <typename T, int BLOCK, int U> __device__ __forceinline__ void pass_sums(const Row<T> &row, Online<T> &sums) {
    const int end = row.granules;
    Granule<T> next[U];
    row.load_all((int)threadIdx.x, BLOCK, end, next);
    for (int q0 = threadIdx.x; q0 < end; q0 += BLOCK * U) {
        Granule<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = next[u];
        if (q0 + BLOCK * U < end) row.load_all(q0 + BLOCK * U, BLOCK, end, next);
        sums.add(raw, q0, BLOCK);
    }
}

template <int BLOCK> __device__ __forceinline__ float block_max(float v, SharedSums<BLOCK> &sh) {
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();                                      // (others may still read sh.warp)
    if (threadIdx.x % 32 == 0) sh.warp[threadIdx.x / 32].r = v;
    __syncthreads();
    for (int w = 0; w < BLOCK / 32; ++w) v = fmaxf(v, sh.warp[w].r);
    __syncthreads();
    return v;
}

// The sums of a far row, relative to its largest logit (in Sums::r, unscaled): every block of a cluster goes over the whole row (such rows are few).
template <typename T, int BLOCK> __device__ __noinline__ Sums far_sums(const Row<T> row, float c, SharedSums<BLOCK> &sh) {
    constexpr int N = Granule<T>::N;
    float most = -INFINITY;
    for (int q = threadIdx.x; q < row.granules; q += BLOCK) most = fmaxf(most, row.load(q, row.granules).largest());
    const float m = block_max(most, sh);
    Sums t;
    t.r = 0.f; t.s = 0.f; t.a = 0.f;
    for (int q = threadIdx.x; q < row.granules; q += BLOCK) {
        float v[N];
        row.load(q, row.granules).get(v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (v[i] == -INFINITY) continue;              // (also what lies beside the row)
            const float d = (v[i] - m) * c, e = exp2_approx(d);
            t.s += e;
            if (e != 0.f) t.a = fmaf(e, d, t.a);
        }
    }
    t = block_sums<BLOCK>(t, sh);
    t.r = m;
    return t;
}

// Sums of the whole row from the blocks' sums; also what a block has put into its shared memory before is visible to the others after.
template <int BLOCK> __device__ __forceinline__ Sums cluster_sums(Sums t, SharedSums<BLOCK> &sh, int blocks) {
    if (blocks == 1) return t;
    if (threadIdx.x == 0) sh.block = t;
    cluster_sync_all();
    t.clear();
    if ((int)threadIdx.x % 32 < blocks) t = *at_rank(&sh.block, threadIdx.x % 32);
    return warp_sums(t);                                  // the same in every block
}

// What a row's outputs are made of.  A row without a logit above -inf ("empty") has S = 0; NaN or +inf among the logits make S NaN.
struct RowResult {
    float scale, c, r, log2_s, entropy, inv_s;             // far: r is the largest logit itself
    bool empty, far;
    __device__ __forceinline__ RowResult() : scale(0.f), c(0.f), r(0.f), log2_s(0.f), entropy(0.f), inv_s(0.f), empty(true), far(false) {}
    __device__ __forceinline__ void set(const Sums &t) {
        empty = t.s == 0.f;
        r = t.r;
        log2_s = empty ? 0.f : log2f(t.s);
        inv_s = empty ? 0.f : 1.f / t.s;
        entropy = empty ? 0.f : kLn2 * (log2_s - t.a * inv_s);
    }
    __device__ __forceinline__ float logprob(float x) const {
        if (empty) return -INFINITY;
        if (far) return (x - r) * scale - kLn2 * log2_s;
        const float d = fmaf(x, c, -r);
        if (d == -INFINITY) return x * scale + 0.f * inv_s;       // x c overflows and x s may not; the rest is less than its rounding
        return kLn2 * (d - log2_s);
    }
    static constexpr float kLn2 = 0.6931471805599453f;
};

// The row's result from its sums, with the far rows' second way.
template <typename T, int BLOCK>
__device__ __forceinline__ RowResult row_result(const Row<T> &row, const Sums &t, float scale, float c, SharedSums<BLOCK> &sh) {
    RowResult r;
    r.scale = scale;
    r.c = c;
    if (fabsf(t.r) < kNear) {
        r.set(t);
    } else {                                              // the same decision in every block of the cluster
        r.far = true;
        r.set(far_sums<T, BLOCK>(row, c, sh));
    }
    return r;
}

// A row's given token.  Its logit is read before the row's sums are joined: after that an in-place gradient may overwrite it.
struct Given {
    int token;
    bool real;
    float x;
    template <typename T> __device__ __forceinline__ Given(const RowsArgs &p, const Row<T> &row, long long at) {
        token = p.tokens ? p.tokens[at] : PARLE_NO_TOKEN;
        real = token >= 0 && token < p.vocab;
        x = p.logprob && real && threadIdx.x == 0 ? to_float(row.x()[token]) : 0.f;
    }
    // by one thread
    __device__ __forceinline__ void write(const RowsArgs &p, long long at, const RowResult &r) const {
        if (p.logprob) p.logprob[at] = real ? r.logprob(x) : 0.f;
        if (p.entropy) p.entropy[at] = r.entropy;
    }
    __device__ __forceinline__ void note_bad(const RowsArgs &p) const {
        if (!real && token != PARLE_NO_TOKEN && p.flags) atomicOr(p.flags, PARLE_FLAG_BAD_LABEL);
    }
};

// The k largest of a cluster's sh.top lists, in its first block (after a cluster barrier), into sh.top.  No key below the largest of
// the lists' k-th keys can be among them, which leaves little more than k to rank.
template <int BLOCK> __device__ __forceinline__ void merge_top(int k, int blocks, Shared<BLOCK> &sh) {
    __syncthreads();                                      // (sh.group, sh.candidate and sh.found were in use)
    if (threadIdx.x == 0) sh.found = 0;
    unsigned long long key = 0;                           // one each: blocks * k <= BLOCK
    static_assert(kClusterMost * kTopMost <= 256, "a thread per key");
    if ((int)threadIdx.x < blocks * k) {
        key = at_rank(sh.top, threadIdx.x / k)[threadIdx.x % k];
        if ((int)threadIdx.x % k == k - 1) sh.group[threadIdx.x / k] = key;
    }
    __syncthreads();
    unsigned long long bound = 0;
#pragma unroll
    for (int b = 0; b < kClusterMost; ++b)
        if (b < blocks) bound = max(bound, sh.group[b]);
    if (key && key >= bound) sh.candidate[atomicAdd(&sh.found, 1)] = key;
    __syncthreads();
    const int found = sh.found;
    if (threadIdx.x < kTopMost) sh.top[threadIdx.x] = 0;  // (every block but this one is done with its own list)
    __syncthreads();
    for (int i = threadIdx.x; i < found; i += BLOCK) {
        const unsigned long long key = sh.candidate[i];
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < found; ++j) above += sh.candidate[j] > key;
        if (above < k) sh.top[above] = key;
    }
    __syncthreads();
}

// The alternatives of a row.
template <int BLOCK>
__device__ __forceinline__ void write_top(const RowsArgs &p, long long at, const RowResult &r, Shared<BLOCK> &sh) {
    if (threadIdx.x >= p.k) return;
    const unsigned long long key = sh.top[threadIdx.x];
    const bool undefined = !(r.inv_s == r.inv_s), real = !undefined && key;
    if (p.top_token) p.top_token[at * p.k + threadIdx.x] = real ? key_token(key) : PARLE_NO_TOKEN;
    if (p.top_logprob) p.top_logprob[at * p.k + threadIdx.x] = undefined ? r.inv_s : real ? r.logprob(key_value(key)) : -INFINITY;
}

// Rows of any length, streamed: one block per row.  2048 x 131072 bf16 logits in a graph: 85 us without alternatives, 92 (0.89 of the copy
// rate) where every call has other logits and so none in L2; 105 with eight alternatives, 138 with 32; called, some 3-5 us more.  Exponentials (a warp instruction takes 7.8 cycles of their pipe) and issue slots are both in use at 62-65 %.
template <typename T, int BLOCK, int U>
__global__ void __launch_bounds__(BLOCK, 1024 / BLOCK) token_logprobs_kernel(const RowsArgs p) {
    __shared__ Shared<BLOCK> sh;
    const long long at = blockIdx.x;
    const Row<T> row(p.logits, p.ld, at, p.vocab);
    const Given given(p, row, at);
    Online<T> sums(p.scale_log2e);
    pass_sums<T, BLOCK, U>(row, sums);
    const unsigned long long best = sums.best >= 0 ? order_key(sums.top, (uint32_t)sums.best) : 0;
    if (p.k > 0) offer_best(best, sh);
    const RowResult r = row_result<T, BLOCK>(row, block_sums<BLOCK>(sums.collect(), sh), p.scale, p.scale_log2e, sh);
    if (threadIdx.x == 0) {
        given.write(p, at, r);
        given.note_bad(p);
    }
    if (p.k == 0) return;
    const unsigned long long bound = top_bound<Shared<BLOCK>::kGroups>(p.k, sh);
    if (best && best >= bound) sh.owner[atomicAdd(&sh.owners, 1)] = threadIdx.x;
    __syncthreads();
    // the granules of the threads that reach the bound, two in flight per thread
    const int each = (row.granules + BLOCK - 1) / BLOCK, all = sh.owners * each;
    const auto granule = [&](int i) { return i < all ? sh.owner[i / each] + i % each * BLOCK : row.granules; };
    for (int i = threadIdx.x; i < all; i += 2 * BLOCK) {
        const int q0 = granule(i), q1 = granule(i + BLOCK);
        const Granule<T> first = row.load(q0, row.granules), second = row.load(q1, row.granules);
        if (q0 < row.granules) hand_on(row, first, q0, bound, sh);
        if (q1 < row.granules) hand_on(row, second, q1, bound, sh);
    }
    __syncthreads();
    rank_candidates(row, 0, row.granules, p.k, sh);
    write_top(p, at, r, sh);
}

// dlogits but for the given token's 1: e ( a + b d ), with a and b over S.
template <typename T, bool ENT> struct Slope {
    static constexpr int N = Granule<T>::N, P = N / 2;
    float_pair c2, r2, a2, b2;
    uint32_t low;
    __device__ __forceinline__ Slope(const RowResult &t, float a, float b)
        : c2(pair(t.c, t.c)), r2(pair(-t.r, -t.r)), a2(pair(a, a)), b2(pair(b, b)), low(low_bound<T>(t.c)) {}
    __device__ __forceinline__ float_pair value(float_pair x) const {
        const float_pair d = fma2(x, c2, r2);
        float lo, hi;
        split(d, lo, hi);
        return mul2(pair(exp2_approx(lo), exp2_approx(hi)), ENT ? fma2(b2, d, a2) : a2);
    }
    __device__ __forceinline__ void values(const Granule<T> &raw, float (&v)[N]) const {
        float_pair x[P];
        raw.pairs(low, x);
#pragma unroll
        for (int i = 0; i < P; ++i) split(value(x[i]), v[2 * i], v[2 * i + 1]);
    }
    // of one logit, by the same steps
    __device__ __forceinline__ float value(T x) const {
        Granule<T> g;
        g.fill_none();
        *reinterpret_cast<T *>(&g.raw) = x;
        float_pair f[P];
        g.pairs(low, f);
        float lo, hi;
        split(value(f[0]), lo, hi);
        return lo;
    }
};

template <typename T> __device__ __forceinline__ uint4 packed(const float (&v)[Granule<T>::N]) {
    if constexpr (sizeof(T) == 4) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    } else {
        Pack8<T> o;
        o.set(v);
        return o.a;
    }
}

// Where a row of dlogits goes: by granule where it begins at the same place of 16 bytes as the logits, else in joined pieces.
template <typename T> struct OutRow {
    static constexpr int N = Granule<T>::N;
    T *out;
    uint4 *base;                                          // NULL: begins at another place
    int skew;                                             // bytes of a granule's first element behind a 16-byte boundary
    __device__ __forceinline__ OutRow(const RowsArgs &p, const Row<T> &row, long long at) {
        out = static_cast<T *>(p.dlogits) + at * p.ld_d;
        const uintptr_t a = reinterpret_cast<uintptr_t>(out);
        skew = (int)((a - reinterpret_cast<uintptr_t>(row.x())) & 15);
        base = skew == 0 ? reinterpret_cast<uint4 *>(a & ~(uintptr_t)15) : nullptr;
    }
    // elements from .. until - 1 of a granule, those that lie in the row
    __device__ __noinline__ static void store_elements(T *out, int e0, int vocab, uint4 packed, int from, int until) {
        const T *v = reinterpret_cast<const T *>(&packed);
        for (int j = max(from, -e0); j < until && e0 + j < vocab; ++j) out[e0 + j] = v[j];
    }
    __device__ __forceinline__ void store(const Row<T> &row, int q, bool whole, const float (&v)[N]) const {
        if (whole) base[q] = packed<T>(v);                // (then base is not NULL)
        else store_elements(out, row.first_element(q), row.vocab, packed<T>(v), 0, N);
    }
    // By a whole warp, whose lanes bring consecutive granules (from `end` on none), with base == NULL: a lane stores the 16 bytes that
    // end its left neighbour's granule and begin its own; what is at the ends goes by element.
    __device__ __forceinline__ void store_joined(const Row<T> &row, int q, int end, const float (&v)[N]) const {
        const uint4 own = packed<T>(v);
        const int lane = threadIdx.x % 32, cut = (16 - skew) / (int)sizeof(T), e0 = row.first_element(q);
        const unsigned wholes = __ballot_sync(0xffffffffu, q < end && row.whole(q)), both = wholes & (wholes << 1);
        uint32_t w[8] = {__shfl_up_sync(0xffffffffu, own.x, 1), __shfl_up_sync(0xffffffffu, own.y, 1),
                         __shfl_up_sync(0xffffffffu, own.z, 1), __shfl_up_sync(0xffffffffu, own.w, 1), own.x, own.y, own.z, own.w};
        skip_bytes<4, sizeof(T) == 2>(w, 16 - skew);
        const bool joined = (both >> lane) & 1u, next = lane < 31 && ((both >> (lane + 1)) & 1u);
        if (joined) *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(out + e0) - skew) = make_uint4(w[0], w[1], w[2], w[3]);
        const int from = joined ? cut : 0, until = next ? cut : N;
        if (q < end && from < until) store_elements(out, e0, row.vocab, own, from, until);
    }
};

// The given token's share g of a row of dlogits, added after the rest by the thread that wrote its granule.
template <typename T> struct TokenShare {
    bool mine;
    T x;                                                  // the token's logit (read before an in-place gradient may overwrite it)
    __device__ __forceinline__ TokenShare(const Row<T> &row, const Given &given, int first, int step, int end) {
        const int q = given.real ? row.granule_of(given.token) : -1;
        mine = given.real && q >= first && q < end && (q - first) % step == 0;
        if (mine) x = row.x()[given.token];
    }
};

// The gradient of granules first, first + step, .. < end of a far row.
template <typename T>
__device__ __noinline__ void far_gradient(const Row<T> row, int first, int step, int end, const RowResult r, float a, float b, float g, int token, const OutRow<T> out) {
    constexpr int N = Granule<T>::N;
    for (int q = first; q < end; q += step) {
        float v[N];
        row.load(q, end).get(v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = (v[i] - r.r) * r.c, e = exp2_approx(d);
            v[i] = e == 0.f ? 0.f * a : e * fmaf(b, d, a);          // (an undefined row's a is NaN)
            if (row.first_element(q) + i == token) v[i] += g;
        }
        out.store(row, q, false, v);
    }
}

// The gradient of a row that may begin at another place of 16 bytes than the logits (and is not the logits themselves), by dlogits' 16-byte pieces: their logits lie in two
// granules, the second of them the next lane's first.
template <typename T, int BLOCK, bool ENT>
__device__ __noinline__ void shifted_gradient(const Row<T> row, const RowResult r, float a, float b, float g, int token, T *out) {
    constexpr int N = Granule<T>::N, S = sizeof(T), U = 2;
    const Slope<T, ENT> slope(r, a, b);
    const int skew = (int)((reinterpret_cast<uintptr_t>(row.x()) - reinterpret_cast<uintptr_t>(out)) & 15);      // of a piece's first logit
    const int head = (int)((reinterpret_cast<uintptr_t>(out) & 15) / S), pieces = (head + row.vocab + N - 1) / N;
    // pieces whose logits' granules lie in the row
    const int low = head + (skew + S - 1) / S, high = head + row.vocab - N - (16 - skew) / S;
    for (int j0 = (int)threadIdx.x + (pieces - 1) / (BLOCK * U) * (BLOCK * U); j0 >= 0; j0 -= BLOCK * U) {
        uint4 first[U], second[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = (j0 + u * BLOCK) * N;
            if (at < low || at > high) continue;
            const uint4 *from = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(row.x() + (at - head)) - skew);
            first[u] = from[0];
            second[u] = from[1];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = (j0 + u * BLOCK) * N, e0 = at - head;
            if (at >= low && at <= high) {
                uint32_t w[8] = {first[u].x, first[u].y, first[u].z, first[u].w, second[u].x, second[u].y, second[u].z, second[u].w};
                skip_bytes<4, S == 2>(w, skew);
                Granule<T> raw;
                raw.raw = make_uint4(w[0], w[1], w[2], w[3]);
                float v[N];
                slope.values(raw, v);
                __stcs(reinterpret_cast<uint4 *>(out + e0), packed<T>(v));
            } else {
                for (int e = max(0, e0); e < min(row.vocab, e0 + N); ++e) out[e] = from_float<T>(slope.value(row.x()[e]));
            }
        }
    }
    if (token >= 0 && (token + head) / N % BLOCK == (int)threadIdx.x)      // by the thread that wrote its piece
        out[token] = from_float<T>(slope.value(row.x()[token]) + g);
}

// What a row of the gradient needs besides its sums.
struct Incoming {
    float g, h;
    bool none;                                            // no incoming gradient: zeros, whatever the logits
    __device__ __forceinline__ Incoming(const RowsArgs &p, const Given &given, long long at) {
        g = given.real && p.d_logprob ? p.d_logprob[at] * p.scale : 0.f;
        h = p.d_entropy ? p.d_entropy[at] * p.scale : 0.f;
        none = g == 0.f && h == 0.f;
    }
    // e ( a + b d ) / S + g 1[j = t]: a = -(g + h (H - log S)), b = -h log 2
    __device__ __forceinline__ float a(const RowResult &r) const { return -fmaf(h, r.entropy - RowResult::kLn2 * r.log2_s, g) * r.inv_s; }
    __device__ __forceinline__ float b(const RowResult &r) const { return -h * RowResult::kLn2 * r.inv_s; }
};

// Zeros in the block's share of a row of dlogits.
template <typename T, int BLOCK> __device__ __forceinline__ void zero_row(const RowsArgs &p, long long at, int rank, int blocks) {
    constexpr int N = Granule<T>::N;
    const Row<T> to(p.dlogits, p.ld_d, at, p.vocab);
    T *out = static_cast<T *>(p.dlogits) + at * p.ld_d;
    const int share = (to.granules + blocks - 1) / blocks, from = rank * share;
    for (int q = from + threadIdx.x; q < min(to.granules, from + share); q += BLOCK) {
        const int e0 = to.first_element(q);
        if (to.whole(q)) const_cast<uint4 *>(to.base)[q] = make_uint4(0, 0, 0, 0);
        else
            for (int i = max(0, -e0); i < N && e0 + i < p.vocab; ++i) out[e0 + i] = from_float<T>(0.f);
    }
}

// The gradient of long rows, by a block each: a second pass reads the row again, from L2.  Its reads and the stores are marked as the
// last use of their lines, so that rows between their two passes stay (a fifth of them does not).  2048 x 131072 bf16 logits: 204-211 us;
// two exponentials per logit take 116 us of their pipe, the bytes 164 us at the copy rate.  SHIFTED: rows of
// dlogits may begin at other places of 16 bytes than the logits; 2048 x 131071 of pitch 131072 to 131071: 243 us, element by element 802.
template <typename T, int BLOCK, int U, bool ENT, bool SHIFTED>
__global__ void __launch_bounds__(BLOCK, 1024 / BLOCK) token_logprobs_grad_kernel(const RowsArgs p) {
    __shared__ SharedSums<BLOCK> sh;
    const long long at = blockIdx.x;
    const Row<T> row(p.logits, p.ld, at, p.vocab);
    const int end = row.granules;
    const Given given(p, row, at);
    const Incoming in(p, given, at);
    const OutRow<T> out(p, row, at);
    const TokenShare<T> share(row, given, threadIdx.x, BLOCK, end);
    if (threadIdx.x == 0) given.note_bad(p);
    if (in.none && !p.logprob && !p.entropy) return zero_row<T, BLOCK>(p, at, 0, 1);
    Online<T> sums(p.scale_log2e);
    pass_sums<T, BLOCK, U>(row, sums);
    const RowResult r = row_result<T, BLOCK>(row, block_sums<BLOCK>(sums.collect(), sh), p.scale, p.scale_log2e, sh);
    if (threadIdx.x == 0) given.write(p, at, r);
    if (in.none || r.empty) {
        zero_row<T, BLOCK>(p, at, 0, 1);
    } else if (r.far) {
        far_gradient<T>(row, threadIdx.x, BLOCK, end, r, in.a(r), in.b(r), in.g, given.token, out);
    } else if constexpr (SHIFTED) {
        shifted_gradient<T, BLOCK, ENT>(row, r, in.a(r), in.b(r), in.g, given.real ? given.token : -1, out.out);
    } else {
        const Slope<T, ENT> slope(r, in.a(r), in.b(r));
        // from the end: what was read last is the likeliest to be in L1 and L2 still
        const int stride = BLOCK * U;
        const auto fast = [&](int q0) { return row.all_whole(q0, q0 + (U - 1) * BLOCK, end); };
        const auto fetch = [&](int q0, Granule<T> (&raw)[U]) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u].raw = __ldcs(row.base + q0 + u * BLOCK);
        };
        int q0 = (int)threadIdx.x + (end - 1) / stride * stride;
        Granule<T> next[U];
        if (fast(q0)) fetch(q0, next);
        for (; q0 >= 0; q0 -= stride) {
            if (fast(q0)) {
                Granule<T> raw[U];
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = next[u];
                if (q0 >= stride && fast(q0 - stride)) fetch(q0 - stride, next);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float v[Granule<T>::N];
                    slope.values(raw[u], v);
                    __stcs(out.base + q0 + u * BLOCK, packed<T>(v));
                }
            } else {
                if (q0 >= stride && fast(q0 - stride)) fetch(q0 - stride, next);
                for (int u = 0; u < U; ++u) {
                    const int q = q0 + u * BLOCK;
                    if (q >= end) break;
                    float v[Granule<T>::N];
                    slope.values(row.load(q, end), v);
                    out.store(row, q, row.whole(q), v);
                }
            }
        }
        if (share.mine) out.out[given.token] = from_float<T>(slope.value(share.x) + in.g);
    }
}

// Rows held in registers, U granules a thread, by a block or a cluster of blocks: everything is in flight at once and read once,
// and the gradient is formed from what is held.  GRAD: the gradient (ENT: with an entropy's; TWO: rows of
// dlogits may begin at other places of 16 bytes than the logits); else log probabilities, entropy, top (TWO: from two groups a thread).
template <typename T, int BLOCK, int U, bool GRAD, bool ENT, bool TWO>
__global__ void __launch_bounds__(BLOCK, 1024 / BLOCK) token_logprobs_held_kernel(const RowsArgs p, int blocks) {
    __shared__ Shared<BLOCK> sh;
    constexpr int P = Granule<T>::N / 2;
    const long long at = blockIdx.x / blocks;
    const int rank = blocks > 1 ? cluster_rank() : 0;
    const Row<T> row(p.logits, p.ld, at, p.vocab);
    const int per_block = (row.granules + blocks - 1) / blocks;      // at most BLOCK * U
    const int begin = min(row.granules, rank * per_block), end = min(row.granules, begin + per_block);
    const int q0 = begin + (int)threadIdx.x;
    const Given given(p, row, at);
    const Incoming in(p, given, at);
    if (threadIdx.x == 0 && rank == 0) given.note_bad(p);
    if (GRAD && in.none && !p.logprob && !p.entropy) return zero_row<T, BLOCK>(p, at, rank, blocks);      // (every block of the cluster)
    const TokenShare<T> share(row, given, q0, BLOCK, GRAD ? end : 0);
    Granule<T> raw[U];
    row.load_all(q0, BLOCK, end, raw);
    float top = -INFINITY, top_odd = -INFINITY;
    int best_granule = -1, best_odd = -1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float v, odd;
        if constexpr (TWO && !GRAD) {
            raw[u].largest_two(v, odd);
            if (odd > top_odd) { top_odd = odd; best_odd = q0 + u * BLOCK; }
        } else {
            v = raw[u].largest();
        }
        if (v > top) { top = v; best_granule = q0 + u * BLOCK; }
    }
    const float c = p.scale_log2e;
    Sums t;
    t.r = fmaxf((TWO && !GRAD ? fmaxf(top, top_odd) : top) * c, -kNear);
    {
        const uint32_t low = low_bound<T>(c);
        const float_pair c2 = pair(c, c), r2 = pair(-t.r, -t.r);
        float_pair s2 = pair(0.f, 0.f), a2 = pair(0.f, 0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (q0 + u * BLOCK >= end) break;
            float_pair x[P];
            raw[u].pairs(low, x);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float_pair d = fma2(x[i], c2, r2);
                float lo, hi;
                split(d, lo, hi);
                const float_pair e = pair(exp2_approx(lo), exp2_approx(hi));
                s2 = add2(s2, e);
                if (ENT || !GRAD) a2 = fma2(e, d, a2);
            }
        }
        float lo, hi;
        split(s2, lo, hi); t.s = lo + hi;
        split(a2, lo, hi); t.a = lo + hi;
    }
    unsigned long long best = best_granule >= 0 ? order_key(top, (uint32_t)(TWO ? 2 * best_granule : best_granule)) : 0;
    if constexpr (TWO && !GRAD) {
        const unsigned long long odd = best_odd >= 0 ? order_key(top_odd, (uint32_t)(2 * best_odd + 1)) : 0;
        offer_two(best, odd, sh);
        best = max(best, odd);
    } else if constexpr (!GRAD) {
        if (p.k > 0) offer_best(best, sh);
    }
    t = block_sums<BLOCK>(t, sh);
    if constexpr (!GRAD) if (p.k > 0) {
        const unsigned long long bound = top_bound<TWO ? 64 : Shared<BLOCK>::kGroups>(p.k, sh);
        if (best && best >= bound) {                      // few threads, and mostly one granule of each: it is read again
            unsigned reach = 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (order_key(raw[u].largest(), (uint32_t)((TWO ? 2 : 1) * (q0 + u * BLOCK))) >= bound) reach |= 1u << u;
            while (reach) {
                const int q = q0 + (__ffs(reach) - 1) * BLOCK;
                reach &= reach - 1;
                if (q < end) hand_on<TWO>(row, row.load(q, end), q, bound, sh);
            }
        }
        __syncthreads();
        rank_candidates(row, begin, end, p.k, sh);
    }
    const RowResult r = row_result<T, BLOCK>(row, cluster_sums<BLOCK>(t, sh, blocks), p.scale, c, sh);
    if (threadIdx.x == 0 && rank == 0) given.write(p, at, r);
    if constexpr (GRAD) {
        const OutRow<T> out(p, row, at);
        if (r.far && blocks > 1) cluster_sync_all();      // each block has read the whole row before any writes an in-place gradient
        if (blocks > 1) cluster_done();
        if (in.none || r.empty) {
            zero_row<T, BLOCK>(p, at, rank, blocks);
        } else if (r.far) {
            far_gradient<T>(row, q0, BLOCK, end, r, in.a(r), in.b(r), in.g, given.token, out);
        } else {
            const Slope<T, ENT> slope(r, in.a(r), in.b(r));
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int q = q0 + u * BLOCK;
                if (!TWO || out.base ? q >= end : q - (int)threadIdx.x % 32 >= end) break;
                float v[Granule<T>::N];
                slope.values(raw[u], v);
                if (!TWO || out.base) out.store(row, q, row.whole(q), v);
                else out.store_joined(row, q, end, v);
            }
            if (TWO) __syncwarp();                        // (a neighbour may have written the token's place)
            if (share.mine) out.out[given.token] = from_float<T>(slope.value(share.x) + in.g);
        }
    } else if (p.k > 0 && rank == 0) {
        if (blocks > 1) merge_top(p.k, blocks, sh);
        write_top(p, at, r, sh);
    }
    if (!GRAD && blocks > 1) cluster_done();
    if (blocks > 1) cluster_wait();                       // no block leaves while another may read its shared memory
}

// Whether rows of dlogits begin at other places of 16 bytes than the logits (never where they are the logits).
template <typename T> bool begins_elsewhere(const RowsArgs &p) {
    return (reinterpret_cast<uintptr_t>(p.logits) - reinterpret_cast<uintptr_t>(p.dlogits)) % 16 || (p.rows > 1 && (p.ld - p.ld_d) * (long long)sizeof(T) % 16);
}

template <typename T, int BLOCK, int U, bool GRAD, bool ENT, bool TWO = false> int launch_held(const RowsArgs &p, int blocks, cudaStream_t stream) {
    if constexpr (GRAD && !TWO)
        if (begins_elsewhere<T>(p)) return launch_held<T, BLOCK, U, GRAD, ENT, true>(p, blocks, stream);
    cudaLaunchAttribute attr = {};
    const cudaLaunchConfig_t cfg = cluster_config(dim3((unsigned)(p.rows * blocks)), BLOCK, 0, blocks, &attr, stream);
    if (cudaLaunchKernelEx(&cfg, token_logprobs_held_kernel<T, BLOCK, U, GRAD, ENT, TWO>, p, blocks) != cudaSuccess) return PARLE_ECUDA;
    return launch_status();
}

template <typename T, bool GRAD, bool ENT> int launch_rows(const RowsArgs &p, int sms, cudaStream_t stream) {
    // granules of a row, one more where rows do not all begin on 16-byte boundaries
    const long long granules = ((long long)p.vocab * sizeof(T) + 15) / 16 + (reinterpret_cast<uintptr_t>(p.logits) % 16 || p.ld * sizeof(T) % 16 ? 1 : 0);
    constexpr int U = 8;
    // Alternatives of few short rows: four warps each.  Measured, four warps / one, 5 alternatives of 500 bf16 logits: 64 rows 4.3 / 4.8 us,
    // 600 rows 5.0 / 5.5, 1200 rows 6.8 / 5.8; 20 of 1900: 4.2 / 7.8 (one row), 5.6 / 10.4 (300 rows), 8.7 / 10.9, 2400 rows 14.2 / 12.8.
    if constexpr (!GRAD)
        if (p.k > 0 && granules > 32 && granules <= 128 * 2 && p.rows <= (p.k > 12 ? 8 : 4) * sms) return launch_held<T, 128, 2, GRAD, ENT>(p, 1, stream);
    // Short rows: a warp each; with two groups a thread where so many alternatives are wanted that 32 groups, or a very short row's
    // fewer, set their bound too low.  Measured, with / without: 8192 x 500 bf16 logits, 20 alternatives 19.3 us without, 25: 22.3 / 23.8,
    // 32: 23.6 / 88; 6827 x 150, 20: 15.9 / 46.
    if constexpr (!GRAD)
        if (4LL * p.k > 3 * std::min(32LL, granules) && granules <= 32 * U)
            return granules <= 32 * 4 ? launch_held<T, 32, 4, GRAD, ENT, true>(p, 1, stream) : launch_held<T, 32, U, GRAD, ENT, true>(p, 1, stream);
    if (granules <= 32 * 4) return launch_held<T, 32, 4, GRAD, ENT>(p, 1, stream);
    if (granules <= 32 * U) return launch_held<T, 32, U, GRAD, ENT>(p, 1, stream);
    if (granules <= 128 * U) return launch_held<T, 128, U, GRAD, ENT>(p, 1, stream);
    // Few rows, held by larger blocks.  Measured, held / streamed: 148 rows of 12000 bf16 logits 6.2 / 6.3 us (gradient 4.9 / 5.3, one row
    // 4.8 / 5.0); gradient of 26549 bf16 logits, 1 row 6.5 / 7.9, 148 rows 6.8 / 8.8, 296 rows 9.4 / 10.2, 592 rows 16.7 / 14.5 (log
    // probabilities of 148 rows: 6.9 / 6.2).
    if (granules <= 256 * U) {
        if (p.rows <= sms) return launch_held<T, 256, U, GRAD, ENT>(p, 1, stream);
    } else if (GRAD && granules <= 512 * U && p.rows <= 2 * sms) {
        return launch_held<T, 512, U, GRAD, ENT>(p, 1, stream);
    }
    // Few long rows: a cluster of up to 8 blocks each (a cluster costs some microseconds of its own).  Measured, 131072 bf16 logits,
    // cluster against one block: 1 row 6.5 / 10.8 us (gradient 8.4 / 16.7), 32 rows 8.6 / 11.8 (10.5 / 16.7), 64 rows 10.6 / 12.4
    // (12.6 / 16.7), 128 rows 16.9 / 12.6 (20.9 / 16.6); 20000 bf16 logits, 1 row: 6.5 / 5.9 (8.0 / 7.5).  131072 fp32 logits, blocks of
    // 512 threads, 1 row: 7.7 / 10.8 (6.1 / 18.7); 96788 fp32 logits, 13 rows: 7.9 / 9.3 (6.5 / 15.7), 37 rows: - / 9.4 (8.9 / 15.7).
    const long long blocks = (granules + 256 * U - 1) / (256 * U), large = (granules + 512 * U - 1) / (512 * U);
    if (granules > 4096 && blocks <= kClusterMost) {
        if (p.rows * blocks <= (GRAD ? 4 : 2) * sms) return launch_held<T, 256, U, GRAD, ENT>(p, (int)blocks, stream);
    } else if (blocks > kClusterMost && large <= kClusterMost) {
        if (p.rows * large <= (GRAD ? 2 : 1) * sms) return launch_held<T, 512, U, GRAD, ENT>(p, (int)large, stream);
    }
    // One block a row.  More threads where fewer rows between the gradient's two passes keep them in L2, fewer where what a block does
    // per row (joining sums, ranking) counts.  Measured: gradient of 2048 x 131072 bf16 logits with 512 / 256 threads 204 / 231 us, 1024 x
    // 65536 59 / 60, 1024 x 32760 with 256 / 128 threads 33 / 30.5, 4096 x 10000 51 / 41; log probabilities with alternatives of 1024 x
    // 32760 with 256 / 128 threads 23 / 27, 4096 x 20000 66 / 68, 4096 x 10000 49 / 35, 128 x 131072 with 512 / 256 threads 12.6 / 16.7.
    const unsigned rows = (unsigned)p.rows;
    if constexpr (GRAD) {
        const bool shifted = begins_elsewhere<T>(p);
        const auto launch = [&](auto *kernel, auto *kernel_shifted, int threads) { (shifted ? kernel_shifted : kernel)<<<rows, threads, 0, stream>>>(p); };
        if (granules > 8192) launch(token_logprobs_grad_kernel<T, 512, 4, ENT, false>, token_logprobs_grad_kernel<T, 512, 4, ENT, true>, 512);
        else if (granules > 4096) launch(token_logprobs_grad_kernel<T, 256, 4, ENT, false>, token_logprobs_grad_kernel<T, 256, 4, ENT, true>, 256);
        else launch(token_logprobs_grad_kernel<T, 128, 4, ENT, false>, token_logprobs_grad_kernel<T, 128, 4, ENT, true>, 128);
    } else {
        if (granules > 2048 && p.rows <= 2 * sms) token_logprobs_kernel<T, 512, 4><<<rows, 512, 0, stream>>>(p);
        else if (granules > 2048) token_logprobs_kernel<T, 256, 4><<<rows, 256, 0, stream>>>(p);
        else token_logprobs_kernel<T, 128, 4><<<rows, 128, 0, stream>>>(p);
    }
    return launch_status();
}

template <typename T> int launch_logprobs(const RowsArgs &p, bool grad, cudaStream_t stream) {
    const int sms = current_sms();
    if (sms < 0) return PARLE_ECUDA;
    if (!grad) return launch_rows<T, false, true>(p, sms, stream);
    return p.entropy || p.d_entropy ? launch_rows<T, true, true>(p, sms, stream) : launch_rows<T, true, false>(p, sms, stream);
}

int check_rows(const void *logits, int dtype, long long rows, int vocab, long long ld, const int32_t *tokens, double scale) {
    if (!valid_dtype(dtype) || rows < 0 || vocab < 1 || ld < 0) return PARLE_EINVAL;
    if (!(scale >= 1e-6 && scale <= 1e6)) return PARLE_EINVAL;      // (keeps scaled logits and bounds on them in fp32's range)
    if (rows > 0 && !logits) return PARLE_EINVAL;
    if (rows > PARLE_TOKEN_MAX_ROWS / kClusterMost || vocab > PARLE_TOKEN_MAX_ROWS) return PARLE_ETOOBIG;
    if (!element_aligned(logits, dtype) || !element_aligned(tokens, PARLE_F32)) return PARLE_EALIGN;
    return PARLE_OK;
}

bool words_aligned(std::initializer_list<const void *> pointers) {
    for (const void *p : pointers)
        if (!element_aligned(p, PARLE_F32)) return false;
    return true;
}

}  // namespace

extern "C" int parle_token_logprobs(const void *logits, int dtype, long long rows, int vocab, long long ld, const int32_t *tokens,
                                    double scale, int k, float *logprob, float *entropy, int32_t *top_token, float *top_logprob,
                                    int32_t *flags, void *cuda_stream) {
    const int rc = check_rows(logits, dtype, rows, vocab, ld, tokens, scale);
    if (rc != PARLE_OK) return rc;
    if (k < 0 || k > kTopMost || (logprob && !tokens) || (k == 0 && (top_token || top_logprob))) return PARLE_EINVAL;
    if (rows == 0) return PARLE_OK;
    if (!logprob && !entropy && !top_token && !top_logprob) return PARLE_EINVAL;
    if (!words_aligned({logprob, entropy, top_token, top_logprob, flags})) return PARLE_EALIGN;
    RowsArgs a = {};
    a.logits = logits; a.tokens = tokens; a.ld = ld; a.rows = rows; a.vocab = vocab;
    a.k = top_token || top_logprob ? k : 0;
    a.scale = (float)scale; a.scale_log2e = (float)(scale * 1.4426950408889634);
    a.logprob = logprob; a.entropy = entropy; a.top_token = top_token; a.top_logprob = top_logprob; a.flags = flags;
    return with_dtype(dtype, [&](auto *tag) {
        return launch_logprobs<std::remove_pointer_t<decltype(tag)>>(a, false, static_cast<cudaStream_t>(cuda_stream));
    });
}

extern "C" int parle_token_logprobs_grad(const void *logits, int dtype, long long rows, int vocab, long long ld, const int32_t *tokens,
                                         double scale, const float *d_logprob, const float *d_entropy, float *logprob, float *entropy,
                                         void *dlogits, long long ld_d, int32_t *flags, void *cuda_stream) {
    const int rc = check_rows(logits, dtype, rows, vocab, ld, tokens, scale);
    if (rc != PARLE_OK) return rc;
    if ((!d_logprob && !d_entropy) || ((d_logprob || logprob) && !tokens) || ld_d < vocab) return PARLE_EINVAL;
    if (rows == 0) return PARLE_OK;
    if (!dlogits || (dlogits == logits && rows > 1 && ld_d != ld)) return PARLE_EINVAL;
    if (!element_aligned(dlogits, dtype) || !words_aligned({d_logprob, d_entropy, logprob, entropy, flags})) return PARLE_EALIGN;
    RowsArgs a = {};
    a.logits = logits; a.tokens = tokens; a.ld = ld; a.rows = rows; a.vocab = vocab;
    a.scale = (float)scale; a.scale_log2e = (float)(scale * 1.4426950408889634);
    a.logprob = logprob; a.entropy = entropy; a.flags = flags;
    a.d_logprob = d_logprob; a.d_entropy = d_entropy; a.dlogits = dlogits; a.ld_d = ld_d;
    return with_dtype(dtype, [&](auto *tag) {
        return launch_logprobs<std::remove_pointer_t<decltype(tag)>>(a, true, static_cast<cudaStream_t>(cuda_stream));
    });
}
