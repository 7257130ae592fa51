// parle_adamw: one AdamW step (Loshchilov, Hutter, "Decoupled weight decay regularization", 2019) of a list of tensors, moments in 32 or
// in 8 bits.
//
//   g = c grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = (1 - lr wd) p - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// Every element is read once and written once: bound by DRAM, 28 bytes an fp32 element with 32-bit moments, 10 to 16 with 8-bit ones.
// All arithmetic is fp32; in the step of p the root (of 32-bit moments) and the reciprocal are the hardware's (2^-22 of the step, which moves p by
// far less than p's own rounding).
//
// 8-bit moments.  256 elements, a warp's eight a lane, share an fp32 scale; codes are e4m3 (range 2^-9 .. 448) of m and of r = sqrt(v),
// whose range is half of v's in powers of two.  A code's neighbours are 6 to 12 % away, but b2 = 0.999 moves v by 0.1 % a step: rounded to
// nearest, r would stay on its code for good.  So the value between two codes goes to the upper one when the rest reaches a threshold that
// runs evenly through [0, 1) from step to step and from element to element, u = frac(i a + t b) with a, b powers of the plastic
// number's inverse (Weyl's equidistribution; Roberts' choice of a, b): a drift of f codes a step moves the code in a share f of the
// steps.  24 bits of u: with 8, as in the hardware's stochastic conversion, f itself (0.008 a step) would be rounded to 0.4 % of a code.
// The threshold is a function of (i, t): no random state, the same call gives the same bits.
#include <math.h>
#include <stdlib.h>

#include <type_traits>

#include "tensor_list.cuh"

using namespace parle;

namespace {

constexpr int kThreads32 = 256, kThreads8 = 128;
constexpr int kBlock = 256;                              // elements that share a scale
constexpr float kLargest = 448.f;                        // of e4m3
constexpr float kNothing = 0x1p-100f;                    // a block whose values all lie below this holds zeros
constexpr uint32_t kWeylI = 12664745, kWeylT = 9560335;  // 2^24 / p and 2^24 / p^2, p the plastic number; odd: all 2^24 thresholds occur
constexpr int kSteps32 = 2, kSteps8 = 4;                 // groups of a thread in a chunk
constexpr int kChunk32 = kThreads32 * 8 * kSteps32, kChunk8 = kThreads8 * 8 * kSteps8;
constexpr int kStages = 2;                               // of them in shared memory, 8-bit moments

struct Entry {
    void *param, *exp_avg, *exp_avg_sq, *copy;
    const void *grad;
    float *exp_avg_scale, *exp_avg_sq_scale;
    long long size_shift;                                // size << 4 | shift << 1 | whether whole groups lie on 16-byte boundaries
};
template <int CAP> struct List {
    int count;
    uint32_t first[CAP];                                 // first chunk of each entry
    Entry entry[CAP];
};
constexpr int kFew = 24, kMany = 440;                    // a launch takes 32764 bytes of arguments at most

struct StepArgs {
    float b1, one_minus_b1, b2, one_minus_b2, eps, minus_zero;
    float rate, root_scale, decay;                       // lr / (1 - b1^t), 1 / sqrt(1 - b2^t), 1 - lr wd, where neither step_dev nor lr_dev is given
    float grad_scale, max_norm;
    double lr, weight_decay, log_b1, log_b2;
    long long step;
    const float *norm, *lr_dev;
    const long long *step_dev;
    int32_t *flags;
};

struct NoCopy {};
template <typename T> struct Limit;                      // magnitudes below it are finite once rounded to the type
template <> struct Limit<float> { static constexpr float value = INFINITY; };
template <> struct Limit<NoCopy> { static constexpr float value = INFINITY; };
template <> struct Limit<__nv_bfloat16> { static constexpr float value = 0x1.ffp127f; };
template <> struct Limit<__half> { static constexpr float value = 65520.f; };

struct Scalars {                                         // what a block needs beside its elements
    float c, rate, root_scale, decay;
    uint32_t weyl;                                       // t's part of the threshold
    bool skip;
    bool tiny_eps;                                       // it does not hide small errors of small roots
};

__device__ __forceinline__ float root(float v) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float inverse_root(float v) {
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float larger(float v, float w) {      // NaN if either is
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(v), "f"(w));
    return m;
}
__device__ __forceinline__ float reciprocal(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ Scalars scalars(const StepArgs &a) {
    __shared__ Scalars shared;
    Scalars s{a.grad_scale, a.rate, a.root_scale, a.decay, (uint32_t)a.step * kWeylT, false, false};
    if (a.step_dev || a.lr_dev) {                        // (the same for all blocks)
        if (threadIdx.x == 0) {
            const long long t = a.step + (a.step_dev ? *a.step_dev : 0);
            const double lr = a.lr * (a.lr_dev ? (double)*a.lr_dev : 1.0);
            s.rate = (float)(lr / -expm1((double)t * a.log_b1));
            s.root_scale = (float)(1.0 / sqrt(-expm1((double)t * a.log_b2)));
            s.decay = (float)(1.0 - lr * a.weight_decay);
            s.weyl = (uint32_t)t * kWeylT;
            shared = s;
        }
        __syncthreads();
        s = shared;
    }
    s.tiny_eps = a.eps < s.root_scale * 0x1p-39f;
    if (a.norm) {
        const float norm = *a.norm;
        s.skip = !(fabsf(norm) < INFINITY);
        const float scaled = norm * a.grad_scale;        // (may be beyond fp32 where what is left of it after clipping is not)
        s.c = scaled < INFINITY ? s.c * fminf(1.f, __fmul_rn(__frcp_rn(scaled), a.max_norm)) : fminf(s.c, __fmul_rn(__frcp_rn(norm), a.max_norm));
        if (s.skip && a.flags && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.flags, PARLE_FLAG_NONFINITE);
    }
    return s;
}

// Two e4m3 codes as fp32.
__device__ __forceinline__ float2 decode2(uint32_t codes) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)codes));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
// A code in the top byte.  y in [0, 448] 2^-120: its exponent is fp32's, subnormal where the code is: 20 bits lie below the code, 24 with the shift,
// where the threshold is added.  (A subnormal y is a multiple of 2^-149, which 2^-120 away is the definition's multiple of 2^-29: one rounding, of the product.)
__device__ __forceinline__ uint32_t code_above(float y, uint32_t threshold) { return (__float_as_uint(y) << 4) + threshold; }
__device__ __forceinline__ uint32_t top_bytes(const uint32_t *t) {
    return __byte_perm(__byte_perm(t[0], t[1], 0x0073), __byte_perm(t[2], t[3], 0x0073), 0x5410);
}

// The largest of a warp's magnitudes, NaN if one is.  (As bits, what is no number is largest.)
__device__ __forceinline__ float warp_largest(float v) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v))); }

// The scale of a block from its largest magnitude (NaN if that is); factor: 448 (1 / largest) 2^-120, by which values come to
// lie in [0, 448] 2^-120 or a rounding above.  Blocks with values from 2^14 on are scaled by a part of 2^-120 first, so that the factor is no subnormal number;
// what becomes one so is 0 as a code all the same (but not 0 itself: a root above 0 stays above it).
__device__ __forceinline__ float block_scale(float top, float (&x)[8], float *factor) {
    const bool none = top < kNothing, finite = top < INFINITY;
    const float scale = none ? 0.f : finite ? __fmul_rn(top, 1.f / kLargest) : NAN;
    float rest = 0x1p-120f;
    if (top >= 0x1p14f) {
        const float part = top < 0x1p74f ? 0x1p-60f : 0x1p-120f;
        rest = top < 0x1p74f ? 0x1p-60f : 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] > 0.f ? fmaxf(__fmul_rn(x[i], part), 0x1p-149f) : __fmul_rn(x[i], part);
    }
    *factor = none || !finite ? 0.f : __fmul_rn(__fmul_rn(__frcp_rn(top), kLargest), rest);
    return scale;
}

// Pairs of fp32 numbers: their instructions run at the rate of single ones, but take half of the issue slots, which bound this kernel.
typedef unsigned long long Two;
__device__ __forceinline__ Two two(float x, float y) {
    Two t;
    asm("mov.b64 %0, {%1, %2};" : "=l"(t) : "f"(x), "f"(y));
    return t;
}
__device__ __forceinline__ void split(Two t, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(t)); }
__device__ __forceinline__ Two mul(Two a, Two b) {
    Two t;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(t) : "l"(a), "l"(b));
    return t;
}
__device__ __forceinline__ Two add(Two a, Two b) {
    Two t;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(t) : "l"(a), "l"(b));
    return t;
}
__device__ __forceinline__ Two mul_add(Two a, Two b, Two c) {
    Two t;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(t) : "l"(a), "l"(b), "l"(c));
    return t;
}

// The root of a number from 2^-102 on or of 0, to nearest: one of Newton's steps with the exact remainder (Markstein, "Computation of elementary functions on
// the IBM RISC System/6000 processor", 1990).  (All numbers were compared with the library's root: that of some below 2^-102 is wrong, where the remainder is
// subnormal, and that of infinity is NaN.)
__device__ __forceinline__ float root_of(float v) {
    const float inverse = inverse_root(fmaxf(v, 0x1p-126f)), guess = __fmul_rn(v, inverse);
    return fmaf(fmaf(-guess, guess, v), __fmul_rn(inverse, 0.5f), guess);
}

// One step of eight elements with moments in 8 bits, a whole warp's block: mc and rc come as the old codes and go as the new ones.  (param: the elements'
// old values, for those whose roots are formed in another way.)
// The moments, their root and what the codes are taken from are rounded after every operation, to nearest: a value next to the border
// between two codes falls to one side in any implementation of these operations, so that codes can be compared.  (102 M bf16 parameters 183 us; fused and with
// the hardware's root 174.)
template <typename P>
__device__ __forceinline__ void step8(const StepArgs &a, const Scalars &s, float limit, const P *param, long long e0, float m_scale, float r_scale, float (&p)[8], const float (&g)[8], uint2 &mc, uint2 &rc,
                                      long long n, bool whole, float *new_m_scale, float *new_r_scale, bool &ok) {
    float m[8], r[8], m_top = 0.f, v_top = 0.f;          // r: first of v, then of its root
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 cm = decode2((i < 2 ? mc.x : mc.y) >> (i % 2 * 16)), cr = decode2((i < 2 ? rc.x : rc.y) >> (i % 2 * 16));
        Two old_m = mul(two(cm.x, cm.y), two(m_scale, m_scale)), old_r = mul(two(cr.x, cr.y), two(r_scale, r_scale));
        float x, y;
        if (!whole) {                                    // (a scale may be NaN: behind the end there are zeros all the same)
            const bool first = e0 + 2 * i < n, second = e0 + 2 * i + 1 < n;
            split(old_m, x, y);
            old_m = two(first ? x : 0.f, second ? y : 0.f);
            split(old_r, x, y);
            old_r = two(first ? x : 0.f, second ? y : 0.f);
        }
        const Two gg = mul(two(g[2 * i], g[2 * i + 1]), two(s.c, s.c));
        const Two zero = two(a.minus_zero, a.minus_zero);      // (products to be added: the assembler makes one operation of mul.rn.f32x2 and add.rn.f32x2)
        split(add(mul_add(old_m, two(a.b1, a.b1), zero), mul_add(gg, two(a.one_minus_b1, a.one_minus_b1), zero)), m[2 * i], m[2 * i + 1]);
        split(add(mul_add(mul(old_r, old_r), two(a.b2, a.b2), zero), mul_add(mul(gg, gg), two(a.one_minus_b2, a.one_minus_b2), zero)), r[2 * i], r[2 * i + 1]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        m_top = larger(m_top, fabsf(m[i]));
        v_top = larger(v_top, r[i]);
    }
    m_top = warp_largest(m_top);
    v_top = warp_largest(v_top);
    // root_of() is not for v below 2^-102.  In a block of small ones the roots are formed of 2^64 v.  Beside a largest v of 2^-66 or more, such a root's code is
    // the smallest one in any case, and beside eps >= 2^-39 root_scale it moves the step of p by less than 2^-24; beside a smaller eps it is formed so, too.
    const bool small = v_top < 0x1p-66f && v_top > 0.f;
    float root_scale = s.root_scale;
    uint32_t apart = 0;                                  // elements whose root is formed in another way than the block's
    bool mixed = !(v_top < INFINITY);
    if (s.tiny_eps && !small) {
        bool low = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) low |= r[i] > 0.f && r[i] < 0x1p-102f;
        mixed |= __any_sync(0xffffffffu, low);
    }
    if (small) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = __fmul_rn(r[i], 0x1p64f);
        v_top = __fmul_rn(v_top, 0x1p64f);
        root_scale = __fmul_rn(root_scale, 0x1p-32f);
    }
    if (mixed) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool low = r[i] > 0.f && r[i] < 0x1p-102f;
            if (low) r[i] = __fmul_rn(r[i], 0x1p64f);
            apart |= low || r[i] == INFINITY ? 1u << i : 0u;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // (as root_of)
        float x = r[2 * i], y = r[2 * i + 1];
        const Two v = two(x, y), inverse = two(inverse_root(fmaxf(x, 0x1p-126f)), inverse_root(fmaxf(y, 0x1p-126f))), guess = mul(v, inverse);
        const Two rest = mul_add(mul(guess, two(-1.f, -1.f)), guess, v), root = mul_add(rest, mul(inverse, two(0.5f, 0.5f)), guess);
        split(root, r[2 * i], r[2 * i + 1]);
        split(mul_add(root, two(root_scale, root_scale), two(a.eps, a.eps)), x, y);
        const Two ratio = mul(two(m[2 * i], m[2 * i + 1]), two(reciprocal(x), reciprocal(y)));
        split(mul_add(two(p[2 * i], p[2 * i + 1]), two(s.decay, s.decay), mul(ratio, two(-s.rate, -s.rate))), p[2 * i], p[2 * i + 1]);
    }
    if (mixed) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (apart >> i & 1) {
                r[i] = r[i] < INFINITY ? __fmul_rn(r[i], 0x1p-32f) : INFINITY;
                p[i] = fmaf(to_float(param[i]), s.decay, -s.rate * (m[i] * reciprocal(fmaf(r[i], s.root_scale, a.eps))));
            }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) ok &= fabsf(p[i]) < limit;
    float r_top = root_of(v_top);
    if (small) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = __fmul_rn(r[i], 0x1p-32f);
        r_top = __fmul_rn(r_top, 0x1p-32f);
    }
    float m_factor, r_factor;
    *new_m_scale = block_scale(m_top, m, &m_factor);
    *new_r_scale = block_scale(r_top, r, &r_factor);
    uint32_t mt[8], rt[8];
    const uint32_t first = (uint32_t)e0 * kWeylI + s.weyl;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = (first + i * kWeylI) & 0xffffffu;
        // (__fmul_rn: a product that ends in a subnormal number, by itself, whatever stands beside it)
        mt[i] = code_above(fminf(__fmul_rn(fabsf(m[i]), m_factor), kLargest * 0x1p-120f), u) | (__float_as_uint(m[i]) & 0x80000000u);
        rt[i] = code_above(fminf(__fmul_rn(r[i], r_factor), kLargest * 0x1p-120f), u ^ 0xffffffu);
        if (r[i] > 0.f) rt[i] = max(rt[i], 1u << 24);    // else m would be divided by eps alone one day
    }
    mc = make_uint2(top_bytes(mt), top_bytes(mt + 4));
    rc = make_uint2(top_bytes(rt), top_bytes(rt + 4));
}

template <int BYTES> __device__ __forceinline__ void copy_async(void *to, const void *from) {
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

// Eight elements of each thread on their way, in shared memory.  Of 32-bit types a warp's 1024 bytes are fetched in two runs of 512: fetched as each
// thread's own 32 bytes, every sector comes from L2 twice, as these copies pass L1 by (60 M fp32 parameters 191 us, so 144).  Threads of a warp read what
// others fetched.
template <typename P, typename G> struct Stage {
    static constexpr int kWarps = kThreads8 / 32;
    uint4 p[kWarps][sizeof(P) / 2 * 32], g[kWarps][sizeof(G) / 2 * 32];
    uint2 mc[kThreads8], rc[kThreads8];
    template <typename T> __device__ __forceinline__ static void fetch(uint4 *to, const T *from) {      // from: the thread's elements
        const int lane = threadIdx.x % 32;
        const uint4 *const first = reinterpret_cast<const uint4 *>(from - lane * 8);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) copy_async<16>(to + i * 32 + lane, first + i * 32 + lane);
    }
    __device__ __forceinline__ void fetch(const Entry &t, long long e0) {
        fetch(p[threadIdx.x / 32], static_cast<const P *>(t.param) + e0);
        fetch(g[threadIdx.x / 32], static_cast<const G *>(t.grad) + e0);
        copy_async<8>(&mc[threadIdx.x], static_cast<const char *>(t.exp_avg) + e0);
        copy_async<8>(&rc[threadIdx.x], static_cast<const char *>(t.exp_avg_sq) + e0);
    }
    template <typename T> __device__ __forceinline__ static void take(const uint4 *from, float (&v)[8]) {
        Pack8<T> pack;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(&pack)[i] = from[threadIdx.x % 32 * (sizeof(T) / 2) + i];
        pack.get(v);
    }
};

// A chunk on 16-byte boundaries is fetched a step ahead through shared memory (one step ahead in registers, 62 to 72 of them a thread, it waited for DRAM:
// 102 M bf16 parameters 282 us; without 347).  Measured in us when the step had 3 instructions an element less, with 2 / 3 / 4 stages and chunks of four steps:
// 102 M bf16 176, 179, 187 (floor 159; 183 with 2 now); 60 M fp32 144, 144, 148 (149); 15 M fp32 40, 40, 45 (37); chunks of eight steps 15 M 55, of
// sixteen 67, as few blocks fill the SMs unevenly.
template <typename P, typename G, typename C, class L>
__global__ void __launch_bounds__(kThreads8) adamw8_kernel(const __grid_constant__ L list, const __grid_constant__ StepArgs a) {
    __shared__ Stage<P, G> stage[kStages];
    const Scalars s = scalars(a);
    if (s.skip) return;
    const int index = entry_of(list, blockIdx.x), lane = threadIdx.x % 32;
    const Entry &t = list.entry[index];
    const long long n = t.size_shift >> 4, first = (long long)(blockIdx.x - list.first[index]) * kChunk8;
    P *const param = static_cast<P *>(t.param);
    char *const m_codes = static_cast<char *>(t.exp_avg), *const r_codes = static_cast<char *>(t.exp_avg_sq);
    const float limit = fminf(Limit<P>::value, Limit<C>::value);
    bool ok = true;
    float m_scale, r_scale;
    long long e0 = first + threadIdx.x * 8;
    if ((t.size_shift & 1) && first + kChunk8 <= n) {
#pragma unroll
        for (int step = 0; step < kStages - 1; ++step) {
            stage[step].fetch(t, e0 + step * kThreads8 * 8);
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        static_assert(kSteps8 <= 16, "");
        // the steps' scales: a lane each, m's in the lower half of the warp
        const float *const scale_of = lane < 16 ? t.exp_avg_scale : t.exp_avg_sq_scale;
        const long long block = e0 / kBlock;
        const float scales = lane % 16 < kSteps8 ? scale_of[block + lane % 16 * (kThreads8 * 8 / kBlock)] : 0.f;
#pragma unroll 1
        for (int step = 0; step < kSteps8; ++step, e0 += kThreads8 * 8) {
            if (step + kStages - 1 < kSteps8) stage[(step + kStages - 1) % kStages].fetch(t, e0 + (kStages - 1) * kThreads8 * 8);
            asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            __syncwarp();                                // (what the others fetched is there)
            Stage<P, G> &now = stage[step % kStages];
            float p[8], g[8];
            now.template take<P>(now.p[threadIdx.x / 32], p);
            now.template take<G>(now.g[threadIdx.x / 32], g);
            uint2 mc = now.mc[threadIdx.x], rc = now.rc[threadIdx.x];
            __syncwarp();                                // (it is read, before the next step fetches into this place)
            step8(a, s, limit, param + e0, e0, __shfl_sync(0xffffffffu, scales, step), __shfl_sync(0xffffffffu, scales, 16 + step), p, g, mc, rc, n, true, &m_scale, &r_scale, ok);
            Pack8<P> pack;
            pack.set(p);
            pack.store(param + e0);
            *reinterpret_cast<uint2 *>(m_codes + e0) = mc;
            *reinterpret_cast<uint2 *>(r_codes + e0) = rc;
            if (lane == 0) {
                t.exp_avg_scale[e0 / kBlock] = m_scale;
                t.exp_avg_sq_scale[e0 / kBlock] = r_scale;
            }
            if constexpr (!std::is_same<C, NoCopy>::value) {
                Pack8<C> c;
                c.set(p);
                c.store(static_cast<C *>(t.copy) + e0);
            }
        }
    } else {
#pragma unroll 1
        for (int step = 0; step < kSteps8; ++step, e0 += kThreads8 * 8) {
            if (e0 - lane * 8 >= n) break;               // (whole warps: a block's lanes meet)
            const bool whole = (t.size_shift & 1) && e0 + 8 <= n;
            float p[8], g[8];
            uint2 mc, rc;
            if (whole) {
                Pack8<P> pack;
                Pack8<G> grads;
                pack.load(param + e0);
                grads.load(static_cast<const G *>(t.grad) + e0);
                mc = *reinterpret_cast<const uint2 *>(m_codes + e0);
                rc = *reinterpret_cast<const uint2 *>(r_codes + e0);
                pack.get(p);
                grads.get(g);
            } else {
                load_some(param, e0, n, p);
                load_some(static_cast<const G *>(t.grad), e0, n, g);
                uint32_t c[4] = {};
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (e0 + i < n) {
                        c[i / 4] |= (uint32_t)(unsigned char)m_codes[e0 + i] << (i % 4 * 8);
                        c[2 + i / 4] |= (uint32_t)(unsigned char)r_codes[e0 + i] << (i % 4 * 8);
                    }
                mc = make_uint2(c[0], c[1]);
                rc = make_uint2(c[2], c[3]);
            }
            const long long block = min(e0, n - 1) / kBlock;
            step8(a, s, limit, param + e0, e0, t.exp_avg_scale[block], t.exp_avg_sq_scale[block], p, g, mc, rc, n, whole, &m_scale, &r_scale, ok);
            if (lane == 0) {
                t.exp_avg_scale[block] = m_scale;
                t.exp_avg_sq_scale[block] = r_scale;
            }
            if (whole) {
                Pack8<P> pack;
                pack.set(p);
                pack.store(param + e0);
                *reinterpret_cast<uint2 *>(m_codes + e0) = mc;
                *reinterpret_cast<uint2 *>(r_codes + e0) = rc;
            } else {
                store_some(param, e0, n, p);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (e0 + i < n) {
                        m_codes[e0 + i] = (char)((i < 4 ? mc.x : mc.y) >> (i % 4 * 8));
                        r_codes[e0 + i] = (char)((i < 4 ? rc.x : rc.y) >> (i % 4 * 8));
                    }
            }
            if constexpr (!std::is_same<C, NoCopy>::value) store_some(static_cast<C *>(t.copy), e0, n, p);
        }
    }
    if (a.flags && !ok) atomicOr(a.flags, PARLE_FLAG_NONFINITE);
}

// Bound by DRAM: 243 M fp32 parameters 991 us, 1.06 of the copy rate; 15 M 66 us (floor 65); 300 tensors of 5000 10 us (6), 1 M in one 6 us (4.3).
template <typename P, typename G, typename C, class L>
__global__ void __launch_bounds__(kThreads32) adamw32_kernel(const __grid_constant__ L list, const __grid_constant__ StepArgs a) {
    const Scalars s = scalars(a);
    if (s.skip) return;
    const int index = entry_of(list, blockIdx.x);
    const Entry &t = list.entry[index];
    const long long n = t.size_shift >> 4;
    const int shift = (int)(t.size_shift >> 1) & 7;
    const bool aligned = t.size_shift & 1;
    P *const param = static_cast<P *>(t.param);
    const G *const grad = static_cast<const G *>(t.grad);
    float *const exp_avg = static_cast<float *>(t.exp_avg), *const exp_avg_sq = static_cast<float *>(t.exp_avg_sq);
    const float limit = fminf(Limit<P>::value, Limit<C>::value);
    bool ok = true;
    long long e0 = (long long)(blockIdx.x - list.first[index]) * kChunk32 + threadIdx.x * 8 - shift;
    for (int step = 0; step < kSteps32; ++step, e0 += kThreads32 * 8) {
        if (e0 >= n) break;
        const bool whole = aligned && e0 >= 0 && e0 + 8 <= n;
        float p[8], g[8], m[8], v[8];
        if (whole) {
            Pack8<P> pp;
            Pack8<G> gg;
            Pack8<float> mm, vv;
            pp.load(param + e0);
            gg.load(grad + e0);
            mm.load(exp_avg + e0);
            vv.load(exp_avg_sq + e0);
            pp.get(p);
            gg.get(g);
            mm.get(m);
            vv.get(v);
        } else {
            load_some(param, e0, n, p);
            load_some(grad, e0, n, g);
            load_some(exp_avg, e0, n, m);
            load_some(exp_avg_sq, e0, n, v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            g[i] *= s.c;
            m[i] = fmaf(a.b1, m[i], a.one_minus_b1 * g[i]);
            v[i] = fmaf(a.b2, v[i], a.one_minus_b2 * (g[i] * g[i]));
            p[i] = fmaf(p[i], s.decay, -s.rate * (m[i] * reciprocal(fmaf(root(v[i]), s.root_scale, a.eps))));
            ok &= fabsf(p[i]) < limit;
        }
        if (whole) {
            Pack8<P> pp;
            Pack8<float> mm, vv;
            pp.set(p);
            mm.set(m);
            vv.set(v);
            pp.store(param + e0);
            mm.store(exp_avg + e0);
            vv.store(exp_avg_sq + e0);
            if constexpr (!std::is_same<C, NoCopy>::value) {
                Pack8<C> cc;
                cc.set(p);
                cc.store(static_cast<C *>(t.copy) + e0);
            }
        } else {
            store_some(param, e0, n, p);
            store_some(exp_avg, e0, n, m);
            store_some(exp_avg_sq, e0, n, v);
            if constexpr (!std::is_same<C, NoCopy>::value) store_some(static_cast<C *>(t.copy), e0, n, p);
        }
    }
    if (a.flags && !ok) atomicOr(a.flags, PARLE_FLAG_NONFINITE);
}

// Whether an address occurs twice among those given to see(), or is one of them.  Room for the addresses is on the stack for a list of one launch's size.
class Addresses {
    static constexpr int kSmall = 4096;                  // (of which a short list uses less)
    uintptr_t small_[kSmall];
    uintptr_t *slot_ = small_;
    size_t mask_ = kSmall - 1;

  public:
    ~Addresses() {
        if (slot_ != small_) free(slot_);
    }
    bool prepare(size_t addresses) {
        size_t slots = 64;
        while (slots < 2 * addresses) slots *= 2;
        if (slots > kSmall && !(slot_ = static_cast<uintptr_t *>(malloc(slots * sizeof(uintptr_t))))) {
            slot_ = small_;
            return false;
        }
        mask_ = slots - 1;
        for (size_t i = 0; i < slots; ++i) slot_[i] = 0;
        return true;
    }
    bool see(const void *p) {
        uintptr_t &slot = place(p);
        if (slot) return true;
        slot = reinterpret_cast<uintptr_t>(p);
        return false;
    }
    bool seen(const void *p) { return p && place(p) != 0; }

  private:
    uintptr_t &place(const void *p) {                    // where it is, or the empty one where it would be
        const uintptr_t key = reinterpret_cast<uintptr_t>(p);
        size_t i = (size_t)((key * 0x9E3779B97F4A7C15ull) >> 20) & mask_;
        while (slot_[i] != key && slot_[i] != 0) i = (i + 1) & mask_;
        return slot_[i];
    }
};

template <typename P, typename G, typename C, int BITS, class L> int launch_list(const L &list, const StepArgs &a, unsigned chunks, cudaStream_t stream) {
    if constexpr (BITS == 8) adamw8_kernel<P, G, C, L><<<chunks, kThreads8, 0, stream>>>(list, a);
    else adamw32_kernel<P, G, C, L><<<chunks, kThreads32, 0, stream>>>(list, a);
    return launch_status();
}

template <int CAP, typename P, typename G, typename C, int BITS>
int launch_all(const parle_adamw_tensor *tensors, int count, const StepArgs &a, cudaStream_t stream) {
    constexpr int kChunk = BITS == 8 ? kChunk8 : kChunk32;
    List<CAP> list;
    list.count = 0;
    unsigned chunks = 0;
    for (int i = 0;; ++i) {
        const bool end = i == count;
        const long long n = end ? 0 : tensors[i].size;
        const long long more = (n + 7 + kChunk - 1) / kChunk;
        if (list.count && (end || list.count == CAP || chunks + more >= 1LL << 31)) {
            const int rc = launch_list<P, G, C, BITS>(list, a, chunks, stream);
            if (rc != PARLE_OK) return rc;
            list.count = 0;
            chunks = 0;
        }
        if (end) return PARLE_OK;
        if (n == 0) continue;
        const parle_adamw_tensor &t = tensors[i];
        // 32-bit moments: groups are cut where all arrays' are, if they agree on that; 8-bit ones: at every eighth element
        const int shift = BITS == 8 ? 0 : group_shift(t.param, sizeof(P));
        bool aligned = group_shift(t.param, sizeof(P)) == shift && group_shift(t.grad, sizeof(G)) == shift;
        if (BITS == 32) aligned = aligned && group_shift(t.exp_avg, 4) == shift && group_shift(t.exp_avg_sq, 4) == shift;
        else aligned = aligned && group_shift(t.exp_avg, 1) == 0 && group_shift(t.exp_avg_sq, 1) == 0;
        if constexpr (!std::is_same<C, NoCopy>::value) aligned = aligned && group_shift(t.copy, sizeof(C)) == shift;
        list.first[list.count] = chunks;
        list.entry[list.count++] = {t.param, t.exp_avg, t.exp_avg_sq, t.copy, t.grad, t.exp_avg_scale, t.exp_avg_sq_scale,
                                    n << 4 | (aligned ? shift : 0) << 1 | (aligned ? 1 : 0)};
        chunks += (unsigned)((n + (aligned ? shift : 0) + kChunk - 1) / kChunk);
    }
}

template <typename P, typename G, typename C>
int launch_bits(const parle_adamw_tensor *tensors, int count, int bits, const StepArgs &a, cudaStream_t stream) {
    if (bits == 8) return count <= kFew ? launch_all<kFew, P, G, C, 8>(tensors, count, a, stream) : launch_all<kMany, P, G, C, 8>(tensors, count, a, stream);
    return count <= kFew ? launch_all<kFew, P, G, C, 32>(tensors, count, a, stream) : launch_all<kMany, P, G, C, 32>(tensors, count, a, stream);
}

}  // namespace

extern "C" int parle_adamw(const parle_adamw_tensor *tensors, int count, int param_dtype, int grad_dtype, int copy_dtype, int state_bits,
                           const parle_adamw_step *step, int32_t *flags, void *cuda_stream) {
    if (count < 0 || (count && !tensors) || !step || !valid_dtype(param_dtype) || !valid_dtype(grad_dtype)) return PARLE_EINVAL;
    if (state_bits != 8 && state_bits != 32) return PARLE_EINVAL;
    if (copy_dtype != PARLE_NO_COPY && (param_dtype != PARLE_F32 || (copy_dtype != PARLE_BF16 && copy_dtype != PARLE_F16))) return PARLE_EINVAL;
    const parle_adamw_step &h = *step;
    const float lr = (float)h.lr, decay = (float)(1.0 - h.lr * h.weight_decay), grad_scale = (float)h.grad_scale;
    if (!(h.lr >= 0.0 && isfinite(lr)) || !(h.beta1 >= 0.0 && h.beta1 < 1.0) || !(h.beta2 >= 0.0 && h.beta2 < 1.0)) return PARLE_EINVAL;
    if (!(h.eps >= 0x1p-60 && h.eps <= 1.0) || !(h.weight_decay >= 0.0 && isfinite(decay))) return PARLE_EINVAL;
    if (!(grad_scale > 0.f && isfinite(grad_scale)) || !(h.max_norm > 0.0) || (float)h.max_norm == 0.f) return PARLE_EINVAL;
    if (!(h.norm || h.max_norm == INFINITY)) return PARLE_EINVAL;
    if (h.step_dev ? h.step < 0 : h.step < 1) return PARLE_EINVAL;
    if (reinterpret_cast<uintptr_t>(h.norm) % 4 || reinterpret_cast<uintptr_t>(h.lr_dev) % 4 || reinterpret_cast<uintptr_t>(h.step_dev) % 8 ||
        reinterpret_cast<uintptr_t>(flags) % 4) return PARLE_EALIGN;
    const bool copies = copy_dtype != PARLE_NO_COPY;
    // The same array twice would be stepped by two blocks at once.
    Addresses seen;
    if (count > (1 << 26) || !seen.prepare((size_t)count * (3 + copies + (state_bits == 8 ? 2 : 0)))) return PARLE_ETOOBIG;
    const uintptr_t param_mask = dtype_bytes(param_dtype) - 1, grad_mask = dtype_bytes(grad_dtype) - 1;
    for (int i = 0; i < count; ++i) {
        const parle_adamw_tensor &t = tensors[i];
        if (t.size <= 0) {
            if (t.size < 0) return PARLE_EINVAL;
            continue;
        }
        if (t.size > PARLE_TOKEN_MAX_ELEMENTS) return PARLE_ETOOBIG;
        if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq || (copies && !t.copy)) return PARLE_EINVAL;
        if (state_bits == 8 && (!t.exp_avg_scale || !t.exp_avg_sq_scale)) return PARLE_EINVAL;
        uintptr_t off = (reinterpret_cast<uintptr_t>(t.param) & param_mask) | (reinterpret_cast<uintptr_t>(t.grad) & grad_mask);
        if (copies) off |= reinterpret_cast<uintptr_t>(t.copy) & 1;
        if (state_bits == 32) off |= (reinterpret_cast<uintptr_t>(t.exp_avg) | reinterpret_cast<uintptr_t>(t.exp_avg_sq)) & 3;
        else off |= (reinterpret_cast<uintptr_t>(t.exp_avg_scale) | reinterpret_cast<uintptr_t>(t.exp_avg_sq_scale)) & 3;
        if (off) return PARLE_EALIGN;
        if (seen.see(t.param) || seen.see(t.exp_avg) || seen.see(t.exp_avg_sq) || (copies && seen.see(t.copy))) return PARLE_EINVAL;
        if (state_bits == 8 && (seen.see(t.exp_avg_scale) || seen.see(t.exp_avg_sq_scale))) return PARLE_EINVAL;
    }
    // What is read may be shared, but not be written by another block meanwhile.
    for (int i = 0; i < count; ++i)
        if (tensors[i].size && seen.seen(tensors[i].grad)) return PARLE_EINVAL;
    if (seen.seen(h.norm) || seen.seen(h.lr_dev) || seen.seen(h.step_dev) || seen.seen(flags)) return PARLE_EINVAL;
    StepArgs a = {};
    a.b1 = (float)h.beta1; a.one_minus_b1 = (float)(1.0 - h.beta1);
    a.b2 = (float)h.beta2; a.one_minus_b2 = (float)(1.0 - h.beta2);
    a.eps = (float)h.eps;
    a.minus_zero = -0.f;
    a.log_b1 = log(h.beta1); a.log_b2 = log(h.beta2);    // (-inf for 0: b^t = 0)
    a.lr = h.lr; a.weight_decay = h.weight_decay; a.step = h.step;
    if (!h.step_dev) {
        a.rate = (float)(h.lr / -expm1((double)h.step * a.log_b1));
        a.root_scale = (float)(1.0 / sqrt(-expm1((double)h.step * a.log_b2)));
    }
    a.decay = decay;
    a.grad_scale = grad_scale; a.max_norm = (float)h.max_norm;
    a.norm = h.norm; a.lr_dev = h.lr_dev; a.step_dev = reinterpret_cast<const long long *>(h.step_dev); a.flags = flags;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return with_dtype(param_dtype, [&](auto *p) {
        return with_dtype(grad_dtype, [&](auto *g) {
            using P = std::remove_pointer_t<decltype(p)>;
            using G = std::remove_pointer_t<decltype(g)>;
            if constexpr (std::is_same<P, float>::value) {
                if (copy_dtype == PARLE_BF16) return launch_bits<P, G, __nv_bfloat16>(tensors, count, state_bits, a, stream);
                if (copy_dtype == PARLE_F16) return launch_bits<P, G, __half>(tensors, count, state_bits, a, stream);
            }
            return launch_bits<P, G, NoCopy>(tensors, count, state_bits, a, stream);
        });
    });
}
