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
// maximum it rescales its two sums), all in fp32; exponentials are base 2 on s log2(e) (x - m).
#include <math.h>

#include <initializer_list>
#include <type_traits>

#include "token_types.cuh"

using namespace parle;

namespace {

constexpr int kGroups = 64;             // thread groups whose maxima bound the k-th largest logit from below
constexpr int kTopMost = PARLE_TOP_MAX;
constexpr int kCandidates = 768;        // logits at least as large as the bound that are ranked at once
constexpr int kClusterMost = 8;

struct RowsArgs {
    const void *logits;
    const int32_t *tokens;
    long long ld, rows;
    int vocab, k;
    float scale, scale_log2e;
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
// max that hands a NaN on
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// 2^-200 is zero in fp32: below it e d counts as 0 (and 0 * -inf does not arise)
constexpr float kFar = -200.f;

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
};

// A row as granules: granule q holds elements q N - head .. q N - head + N - 1.
template <typename T> struct Row {
    static constexpr int N = Granule<T>::N;
    const T *x;
    int vocab, head, granules;
    __device__ __forceinline__ Row(const void *logits, long long ld, long long row, int vocab_) {
        x = static_cast<const T *>(logits) + row * ld;
        vocab = vocab_;
        head = (int)((reinterpret_cast<uintptr_t>(x) / sizeof(T)) % N);
        granules = (head + vocab + N - 1) / N;
    }
    __device__ __forceinline__ int first_element(int q) const { return q * N - head; }
    __device__ __forceinline__ bool whole(int q) const { return q * N >= head && (q + 1) * N - head <= vocab; }
    __device__ __forceinline__ Granule<T> load(int q, int end) const {
        Granule<T> g;
        if (q >= end) { g.fill_none(); return g; }
        const int e0 = first_element(q);
        if (whole(q)) {
            g.raw = *reinterpret_cast<const uint4 *>(x + e0);
        } else {
            g.fill_none();
            T *v = reinterpret_cast<T *>(&g.raw);
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (e0 + i >= 0 && e0 + i < vocab) v[i] = x[e0 + i];
        }
        return g;
    }
};

// Maximum, sum of 2^((x - m) c) and sum of 2^((x - m) c) (x - m) c over some logits.
struct Sums {
    float m, s, a;
    __device__ __forceinline__ void clear() { m = -INFINITY; s = 0.f; a = 0.f; }
    // The same sums relative to a maximum `to` >= m.
    __device__ __forceinline__ void rebase(float to, float c) {
        const float shift = m == to ? 0.f : (m - to) * c, f = m == to ? 1.f : exp2_approx(shift);
        a = f == 0.f ? 0.f : f * (a + shift * s);        // f > 0: shift is finite
        s *= f;                                           // (a NaN stays)
        m = to;
    }
    __device__ __forceinline__ void add(Sums o, float c) {
        const float to = fmaxf(m, o.m);
        rebase(to, c);
        o.rebase(to, c);
        s += o.s;
        a += o.a;
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

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
// Address of another block's copy of a shared variable.
template <typename V> __device__ __forceinline__ const V *at_rank(const V *p, uint32_t rank) {
    uint64_t r;
    asm volatile("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
    return reinterpret_cast<const V *>(r);
}

template <int BLOCK> struct Shared {
    float m[BLOCK / 32], s[BLOCK / 32], a[BLOCK / 32];
    float bm, bs, ba;                                     // the block's sums, read by the other blocks of its cluster
    unsigned long long group[BLOCK];                      // the threads' best (logit, granule)
    unsigned long long bound;
    int found;
    unsigned long long candidate[kCandidates];
    unsigned long long top[kTopMost];
};

// Sums over a block, the same in every thread.
template <int BLOCK> __device__ __forceinline__ Sums block_sums(Sums t, Shared<BLOCK> &sh, float c) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Sums u;
        u.m = __shfl_xor_sync(0xffffffffu, t.m, o);
        u.s = __shfl_xor_sync(0xffffffffu, t.s, o);
        u.a = __shfl_xor_sync(0xffffffffu, t.a, o);
        t.add(u, c);
    }
    if (threadIdx.x % 32 == 0) { sh.m[threadIdx.x / 32] = t.m; sh.s[threadIdx.x / 32] = t.s; sh.a[threadIdx.x / 32] = t.a; }
    __syncthreads();
    Sums r;
    r.m = sh.m[0]; r.s = sh.s[0]; r.a = sh.a[0];
#pragma unroll
    for (int w = 1; w < BLOCK / 32; ++w) {
        Sums u;
        u.m = sh.m[w]; u.s = sh.s[w]; u.a = sh.a[w];
        r.add(u, c);
    }
    return r;
}

// The k largest of the block's logits (granules begin .. end), best first, into sh.top; fewer than k finite or -inf logits leave
// keys of 0.  `best` is this thread's largest (logit, granule).
//
// The k-th largest of 64 groups' maxima is a lower bound of the k-th largest logit, and only threads whose own maximum reaches
// it can hold one of the k: they hand their logits above the bound on (typically k to 2 k of them), which are ranked by
// counting.  Equal maxima are ordered by granule, so a row of equal logits hands on 8 k, not V, of them.
template <typename T, int BLOCK>
__device__ void block_top(const Row<T> &row, int begin, int end, int k, unsigned long long best, Shared<BLOCK> &sh) {
    constexpr int N = Granule<T>::N;
    const int lane = threadIdx.x % 32;
    sh.group[threadIdx.x] = best;
    if (threadIdx.x < k) sh.top[threadIdx.x] = 0;
    if (threadIdx.x == 0) { sh.found = 0; sh.bound = 0; }
    __syncthreads();
    if (threadIdx.x < kGroups) {
        unsigned long long g = sh.group[threadIdx.x];
#pragma unroll
        for (int t = threadIdx.x + kGroups; t < BLOCK; t += kGroups) g = max(g, sh.group[t]);
        sh.group[threadIdx.x] = g;
    }
    __syncthreads();
    if (threadIdx.x < kGroups) {
        const unsigned long long g = sh.group[threadIdx.x];
        int above = 0;
#pragma unroll 8
        for (int t = 0; t < kGroups; ++t) above += sh.group[t] > g || (sh.group[t] == g && t < (int)threadIdx.x);
        if (above == k - 1) sh.bound = g;
    }
    __syncthreads();
    const unsigned long long bound = sh.bound;            // (logit, granule) of the k-th group; 0 if fewer groups have any logits
    // threads that reach the bound, one after the other; the warp reads such a thread's granules together
    unsigned reach = __ballot_sync(0xffffffffu, best >= bound && best != 0);
    while (reach) {
        const int owner = __ffs(reach) - 1;
        reach &= reach - 1;
        const int own0 = begin + (int)(threadIdx.x - lane) + owner;
        for (int q0 = own0; q0 < end; q0 += BLOCK * 32) {
            const int q = q0 + lane * BLOCK;
            if (q >= end) continue;
            float v[N];
            row.load(q, end).get(v);
            const int e0 = row.first_element(q);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (e0 + i < 0 || e0 + i >= row.vocab || !(v[i] == v[i]) || order_key(v[i], q) < bound) continue;
                const int at = atomicAdd(&sh.found, 1);
                if (at < kCandidates) sh.candidate[at] = order_key(v[i], (uint32_t)(e0 + i));
            }
        }
        __syncwarp();
    }
    __syncthreads();
    const int found = sh.found;
    if (found <= kCandidates) {
        for (int i = threadIdx.x; i < found; i += BLOCK) {
            const unsigned long long key = sh.candidate[i];
            int above = 0;
            for (int j = 0; j < found; ++j) above += sh.candidate[j] > key;
            if (above < k) sh.top[above] = key;
        }
    } else {
        // too many logits above the bound (large ones gathered in few groups): one pass over the block's logits per rank
        unsigned long long last = ~0ull;
        for (int r = 0; r < k; ++r) {
            unsigned long long mine = 0;
            for (int q = begin + threadIdx.x; q < end; q += BLOCK) {
                float v[N];
                row.load(q, end).get(v);
                const int e0 = row.first_element(q);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (e0 + i < 0 || e0 + i >= row.vocab || !(v[i] == v[i])) continue;
                    const unsigned long long key = order_key(v[i], (uint32_t)(e0 + i));
                    if (key < last && key > mine) mine = key;
                }
            }
            for (int o = 16; o > 0; o >>= 1) mine = max(mine, __shfl_xor_sync(0xffffffffu, mine, o));
            __syncthreads();
            if (lane == 0) sh.group[threadIdx.x / 32] = mine;
            __syncthreads();
            for (int w = 0; w < BLOCK / 32; ++w) mine = max(mine, sh.group[w]);
            if (threadIdx.x == 0) sh.top[r] = mine;
            last = mine;
        }
    }
    __syncthreads();
}

// Maximum of a granule's logits (NaN is passed over; the sums carry it).
template <typename T> __device__ __forceinline__ float granule_max(const float (&v)[Granule<T>::N]) {
    float g = v[0];
#pragma unroll
    for (int i = 1; i < Granule<T>::N; ++i) g = fmaxf(g, v[i]);
    return g;
}

// First pass over a block's share of a row.  best: largest (logit, granule) of this thread.
template <typename T, int BLOCK, bool ENT>
__device__ __forceinline__ Sums pass_sums(const Row<T> &row, int begin, int end, float c, int &best_granule) {
    constexpr int N = Granule<T>::N, U = 4;
    Sums t;
    t.clear();
    best_granule = -1;
    for (int q0 = begin + threadIdx.x; q0 < end; q0 += BLOCK * U) {
        Granule<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = row.load(q0 + u * BLOCK, end);
        float top = t.m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[N];
            raw[u].get(v);
            const float g = granule_max<T>(v);
            if (g > top) { top = g; best_granule = q0 + u * BLOCK; }
        }
        if (top > t.m) t.rebase(top, c);
        const float m = t.m == -INFINITY ? 0.f : t.m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[N];
            raw[u].get(v);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = (v[i] - m) * c, e = exp2_approx(d);
                t.s += e;
                if (ENT) t.a = fmaf(e, max_nan(d, kFar), t.a);
            }
        }
    }
    return t;
}

// Sums of the whole row: the block's, joined with those of the other blocks of its cluster.
template <int BLOCK> __device__ __forceinline__ Sums row_sums(Sums t, Shared<BLOCK> &sh, float c, int blocks) {
    Sums r = block_sums<BLOCK>(t, sh, c);
    if (blocks > 1) {
        if (threadIdx.x == 0) { sh.bm = r.m; sh.bs = r.s; sh.ba = r.a; }
        cluster_sync_all();
        r.clear();
        for (int b = 0; b < blocks; ++b) {                // the same order in every block
            Sums u;
            u.m = *at_rank(&sh.bm, b); u.s = *at_rank(&sh.bs, b); u.a = *at_rank(&sh.ba, b);
            r.add(u, c);
        }
    }
    return r;
}

// What a row's outputs are made of.  A row without a logit above -inf ("empty") has S = 0; NaN or +inf among the logits make S NaN.
struct RowResult {
    float m, log_s, entropy, inv_s;
    bool empty;
    __device__ __forceinline__ RowResult(const Sums &r) {
        empty = r.s == 0.f;
        m = empty ? 0.f : r.m;
        log_s = empty ? 0.f : logf(r.s);
        inv_s = empty ? 0.f : 1.f / r.s;
        entropy = empty ? 0.f : log_s - 0.6931471805599453f * r.a * inv_s;
    }
    __device__ __forceinline__ float logprob(float x, float scale) const {
        if (empty) return -INFINITY;
        return (x - m) * scale - log_s;
    }
};

// A row's given token.  Its logit is read before the row's sums are joined: after that an in-place gradient may overwrite it.
struct Given {
    int token;
    bool real;
    float x;
    template <typename T> __device__ __forceinline__ Given(const RowsArgs &p, const Row<T> &row, long long at) {
        token = p.tokens ? p.tokens[at] : PARLE_NO_TOKEN;
        real = token >= 0 && token < p.vocab;
        x = p.logprob && real && threadIdx.x == 0 ? to_float(row.x[token]) : 0.f;
    }
    // by one thread
    __device__ __forceinline__ void write(const RowsArgs &p, long long at, const RowResult &r) const {
        if (p.logprob) p.logprob[at] = real ? r.logprob(x, p.scale) : 0.f;
        if (p.entropy) p.entropy[at] = r.entropy;
    }
    __device__ __forceinline__ void note_bad(const RowsArgs &p) const {
        if (!real && token != PARLE_NO_TOKEN && p.flags) atomicOr(p.flags, PARLE_FLAG_BAD_LABEL);
    }
};

// One row per block, or per cluster of `blocks` blocks that take a slice of its granules each.
template <typename T, int BLOCK, bool ENT>
__global__ void __launch_bounds__(BLOCK) token_logprobs_kernel(const RowsArgs p, int blocks) {
    __shared__ Shared<BLOCK> sh;
    const long long at = blockIdx.x / blocks;
    const int rank = blocks > 1 ? (int)cluster_rank() : 0;
    const Row<T> row(p.logits, p.ld, at, p.vocab);
    const int per_block = (row.granules + blocks - 1) / blocks;
    const int begin = min(row.granules, rank * per_block), end = min(row.granules, begin + per_block);
    const Given given(p, row, at);
    int best_granule;
    const Sums t = pass_sums<T, BLOCK, ENT>(row, begin, end, p.scale_log2e, best_granule);
    const unsigned long long best = best_granule >= 0 ? order_key(t.m, (uint32_t)best_granule) : 0;
    const RowResult r(row_sums<BLOCK>(t, sh, p.scale_log2e, blocks));
    if (threadIdx.x == 0 && rank == 0) {
        given.write(p, at, r);
        given.note_bad(p);
    }
    if (p.k > 0) {
        block_top<T, BLOCK>(row, begin, end, p.k, best, sh);
        if (blocks > 1) {                                 // rank the cluster's k-lists in its first block
            cluster_sync_all();
            if (rank == 0) {
                const int all = blocks * p.k;
                for (int i = threadIdx.x; i < all; i += BLOCK) sh.candidate[i] = at_rank(sh.top, i / p.k)[i % p.k];
                __syncthreads();
                if (threadIdx.x < p.k) sh.group[threadIdx.x] = 0;
                __syncthreads();
                for (int i = threadIdx.x; i < all; i += BLOCK) {
                    const unsigned long long key = sh.candidate[i];
                    int above = 0;
                    for (int j = 0; j < all; ++j) above += sh.candidate[j] > key;
                    if (key && above < p.k) sh.group[above] = key;
                }
                __syncthreads();
            }
        }
        if (rank == 0 && threadIdx.x < p.k) {
            const unsigned long long key = blocks > 1 ? sh.group[threadIdx.x] : sh.top[threadIdx.x];
            const float x = key ? key_value(key) : -INFINITY;
            const bool undefined = !(r.inv_s == r.inv_s), real = !undefined && x > -INFINITY;
            if (p.top_token) p.top_token[at * p.k + threadIdx.x] = real ? key_token(key) : PARLE_NO_TOKEN;
            if (p.top_logprob) p.top_logprob[at * p.k + threadIdx.x] = undefined ? r.inv_s : real ? r.logprob(x, p.scale) : -INFINITY;
        }
    }
    if (blocks > 1) cluster_sync_all();                   // no block leaves while another may read its shared memory
}

// The gradient, in a second pass over the row (which is then in L2).
template <typename T, int BLOCK, bool ENT>
__global__ void __launch_bounds__(BLOCK) token_logprobs_grad_kernel(const RowsArgs p, int blocks) {
    __shared__ Shared<BLOCK> sh;
    constexpr int N = Granule<T>::N, U = 4;
    const long long at = blockIdx.x / blocks;
    const int rank = blocks > 1 ? (int)cluster_rank() : 0;
    const Row<T> row(p.logits, p.ld, at, p.vocab);
    const int per_block = (row.granules + blocks - 1) / blocks;
    const int begin = min(row.granules, rank * per_block), end = min(row.granules, begin + per_block);
    const Given given(p, row, at);
    float g = given.real && p.d_logprob ? p.d_logprob[at] * p.scale : 0.f;
    const float h = p.d_entropy ? p.d_entropy[at] * p.scale : 0.f;
    const bool none = g == 0.f && h == 0.f;               // a row without an incoming gradient: zeros, whatever its logits
    const float c = p.scale_log2e;
    RowResult r{Sums{-INFINITY, 0.f, 0.f}};
    if (!none || p.logprob || p.entropy) {
        int best_granule;
        r = RowResult(row_sums<BLOCK>(pass_sums<T, BLOCK, ENT>(row, begin, end, c, best_granule), sh, c, blocks));
        if (threadIdx.x == 0 && rank == 0) given.write(p, at, r);
    }
    if (threadIdx.x == 0 && rank == 0) given.note_bad(p);
    if (r.empty) g = 0.f;
    // p_j ( a + b d_j ) + g 1[j = t], d in units of log 2
    const float a = none ? 0.f : -(g + h * (r.entropy - r.log_s)), b = -h * 0.6931471805599453f;
    const float inv_s = none ? 0.f : r.inv_s, m = none ? 0.f : r.m;
    T *out = static_cast<T *>(p.dlogits) + at * p.ld_d;
    const bool same_phase = (reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(row.x)) % 16 == 0;
    for (int q0 = begin + threadIdx.x; q0 < end; q0 += BLOCK * U) {
        Granule<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (none) raw[u].fill_none();
            else raw[u] = row.load(q0 + u * BLOCK, end);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int q = q0 + u * BLOCK;
            if (q >= end) break;
            float v[N];
            raw[u].get(v);
            const int e0 = row.first_element(q);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = (v[i] - m) * c, e = exp2_approx(d) * inv_s;
                v[i] = e * (ENT ? fmaf(b, max_nan(d, kFar), a) : a);
                if (e0 + i == given.token) v[i] += g;
            }
            if (same_phase && row.whole(q)) {
                T w[N];
#pragma unroll
                for (int i = 0; i < N; ++i) w[i] = from_float<T>(v[i]);
                *reinterpret_cast<uint4 *>(out + e0) = *reinterpret_cast<const uint4 *>(w);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (e0 + i >= 0 && e0 + i < p.vocab) out[e0 + i] = from_float<T>(v[i]);
            }
        }
    }
    if (blocks > 1) cluster_sync_all();
}

// How many blocks share a row: few rows of many granules are split so that the SMs have work.
int blocks_per_row(long long rows, long long granules, int block, int sms) {
    int blocks = 1;
    while (blocks < kClusterMost && rows * blocks * 2 <= 2 * sms && granules >= (long long)block * blocks * 8) blocks *= 2;
    return blocks;
}

template <typename T, int BLOCK> int launch_rows(const RowsArgs &p, bool grad, int blocks, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * blocks));
    cfg.blockDim = dim3(BLOCK);
    cfg.stream = stream;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = blocks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = blocks > 1 ? 1 : 0;
    const bool ent = p.entropy || p.d_entropy;
    cudaError_t e;
    if (grad) e = ent ? cudaLaunchKernelEx(&cfg, token_logprobs_grad_kernel<T, BLOCK, true>, p, blocks)
                      : cudaLaunchKernelEx(&cfg, token_logprobs_grad_kernel<T, BLOCK, false>, p, blocks);
    else e = ent ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, BLOCK, true>, p, blocks)
                 : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, BLOCK, false>, p, blocks);
    if (e != cudaSuccess) return PARLE_ECUDA;
    return launch_status();
}

template <typename T> int launch_logprobs(const RowsArgs &p, bool grad, cudaStream_t stream) {
    const long long granules = ((long long)p.vocab * sizeof(T) + 15) / 16;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return PARLE_ECUDA;
    if (granules <= 256) return launch_rows<T, 64>(p, grad, 1, stream);
    if (granules <= 1024) return launch_rows<T, 128>(p, grad, 1, stream);
    if (granules <= 4096) return launch_rows<T, 256>(p, grad, blocks_per_row(p.rows, granules, 256, sms), stream);
    return launch_rows<T, 512>(p, grad, blocks_per_row(p.rows, granules, 512, sms), stream);
}

int check_rows(const void *logits, int dtype, long long rows, int vocab, long long ld, const int32_t *tokens, double scale) {
    if (!valid_dtype(dtype) || rows < 0 || vocab < 1 || ld < 0) return PARLE_EINVAL;
    if (!(scale > 0.0) || !isfinite((float)(scale * 1.4426950408889634)) || (float)scale == 0.f) return PARLE_EINVAL;
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
