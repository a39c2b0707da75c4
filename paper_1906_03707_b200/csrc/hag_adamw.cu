// One AdamW step over a list of tensors, in place.  With g' = c g, c = min(1, max_norm / (N + 1e-6)) or 1:
//   m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = p (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// The states of all tensors lie in one array of blocks of 256 elements, a tensor's first block behind the previous
// tensor's last, so a launch needs few addresses and the states' alignment does not depend on the parameters'.
// In 8 bits a block holds m and sqrt(v) as e4m3 with an fp32 scale each: the largest of the block becomes 448.  The root
// rather than v: it spans half the binades, and it is what the step divides by.  A positive root is never stored as
// zero, since m of the same element, which has a scale of its own, might not be: m / eps would be a step of any size.
// Neighbouring codes are 6 to 12 % apart, but without a gradient a root shrinks by (1 - b2) / 2 a step: rounded to nearest
// it stays where it is until its block's scale moves, and is wrong for good once the gradients of a block change unequally.  Rounded
// by chance, with the probability of its nearness, it is right on average at every step.  That takes a hash and two roundings in
// integers per element: 200 million bf16 parameters 555 us instead of 319, 150 million fp32 ones 435 instead of 374.
//
// A warp takes a block, eight elements per lane; the largest of a block is a maximum over the warp.  Coefficients are folded
// so that a pair of elements takes few instructions (m: one product and one fused product of what is read; v: the square of
// one product plus that of another), two elements per instruction where there is one for that; the root, the reciprocal
// and the codes are the hardware's.
//
// Bound by memory: 10 bytes per bf16 parameter with 8-bit states, 28 per fp32 one with fp32 states.  Measured on B200,
// 24 to 40 tensors of 200 million parameters together: bf16 with 8-bit states 319 us (6.3 TB/s), fp32 with bf16 gradients and
// copies and fp32 states 825 us (6.8 TB/s); 12 tensors of 50 000 values together 3.5 and 3.0 us.  A warp that copied its
// blocks into a ring in shared memory first took 415 us and 998, one that read the next block into registers 458 and 911.
// Tensors that do not begin on four of their elements are read one element at a time: 7 million fp32 parameters with
// 8-bit states, bf16 gradients and copies 35 us, aligned 23.
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "hag.h"
#include "hag_kernels.cuh"
#include "hag_launch.h"
#include "hag_rows.cuh"

namespace {

constexpr int kAdamThreads = 256, kAdamWarps = kAdamThreads / 32;
constexpr int kAdamList = 64;                   // tensors per launch: the list must fit in 4 KB of parameters
constexpr int kAdamBlock = HAG_ADAMW_BLOCK;
constexpr int kPerLane = kAdamBlock / 32;
static_assert(kAdamBlock == 256, "two groups of four elements per lane");
constexpr int kSms = 148;
constexpr float kTop = 448.0f;                  // the largest value of e4m3
constexpr float kLeastScale = FLT_MIN;          // its reciprocal is finite too
constexpr float kLowest = 0.001953125f;         // 2^-9, the smallest positive value of e4m3

struct AdamArgs {
    int32_t tensors;
    void *mean, *square;                        // of all tensors
    float2 *scales;
    float lr, b1, rest1, b2, eps;               // rest = 1 - b
    float root2, root_rest2;                    // sqrt(b2), sqrt(1 - b2)
    float rate, root;                           // lr / (1 - b1^t), 1 / sqrt(1 - b2^t): where the step is the host's
    double beta1, beta2;
    uint64_t seed;                              // of the roundings by chance
    int64_t step;                               // where it is the host's
    const float *lr_at, *norm;
    const int64_t *step_at;
    float max_norm;
    void *p[kAdamList];
    const void *g[kAdamList];
    void *copy[kAdamList];
    int64_t len[kAdamList], state[kAdamList];   // elements; first block of the states
    float decay[kAdamList];
    uint32_t units;                             // of this launch's tensors
    uint32_t first[kAdamList];                  // units before those of each
    uint32_t blocks[kAdamList], whole[kAdamList];      // how many, and how many of them are read by vectors
    uint8_t p_bf16[kAdamList], g_bf16[kAdamList];
};
static_assert(sizeof(AdamArgs) <= 4096, "the list must fit in the parameters of a launch");

struct Coefficients {
    float lr, rate, root;
    float norm;                                 // as it was read: it arrives while the first blocks do
};
// What the gradient is multiplied with for m, and, before its square, for v.
__device__ __forceinline__ float2 of_gradient(const AdamArgs &p, float norm) {
    if (!p.norm) return make_float2(p.rest1, p.root_rest2);
    const float ratio = p.max_norm / (norm + 1e-6f);
    const float factor = ratio >= 1.0f ? 1.0f : ratio;         // a norm that is no number gives a factor that is none
    return make_float2(p.rest1 * factor, p.root_rest2 * factor);
}

__device__ double power(double base, int64_t n) {          // base^n by squaring
    double r = 1.0;
    for (; n > 0; n >>= 1, base *= base)
        if (n & 1) r *= base;
    return r;
}

// Random bits from a counter, so that a call's results depend on its arguments alone: products with odd numbers (the
// fractions of the roots of 2 and 3 and of the golden ratio) carry low bits upwards, shifts bring high bits down again.
__device__ __forceinline__ uint64_t mix64(uint64_t x) {
    x = (x ^ (x >> 32)) * 0x6a09e667f3bcc909ull;
    x = (x ^ (x >> 29)) * 0xbb67ae8584caa73bull;
    return x ^ (x >> 32);
}
__device__ __forceinline__ uint64_t step_key(uint64_t seed, int64_t step) { return mix64(mix64(seed + 0x9e3779b97f4a7c15ull) + uint64_t(step)); }
// Of element `place` of a block with key `block`: 16 bits for the mean, 16 for the root.
__device__ __forceinline__ uint32_t random_bits(uint64_t block, uint32_t place) {
    uint32_t x = uint32_t(block) + place * 0x9e3779b9u;
    x = (x ^ (x >> 16)) * 0x6a09e667u;
    x = (x ^ (x >> 15)) * 0xbb67ae85u;
    return (x ^ (x >> 16)) + uint32_t(block >> 32);
}

// What the step and the rate on the device make of the coefficients; one thread's work.
__device__ __forceinline__ Coefficients coefficients(const AdamArgs &p) {
    Coefficients c{p.lr, p.rate, p.root, 0.0f};
    if (p.lr_at) c.lr = __ldcg(p.lr_at);
    if (p.step_at) {
        const int64_t t = max(int64_t(1), int64_t(__ldcg(reinterpret_cast<const long long *>(p.step_at))));
        c.rate = float(1.0 / (1.0 - power(p.beta1, t)));
        c.root = float(1.0 / sqrt(1.0 - power(p.beta2, t)));
    }
    c.rate = float(double(c.lr) * double(c.rate));
    return c;
}
__device__ __forceinline__ uint64_t key_of(const AdamArgs &p) {
    return step_key(p.seed, p.step_at ? max(int64_t(1), int64_t(__ldcg(reinterpret_cast<const long long *>(p.step_at)))) : p.step);
}

// The elements of a block that a lane holds, as pairs: two groups of four, 128 apart, so that a warp's accesses are
// contiguous; or, where the addresses do not allow that, eight single ones, 32 apart.
constexpr int kPairs = kPerLane / 2;
// Eight elements of a lane as they are in memory.
template <typename T, bool VEC>
struct Eight {
    hagr::Vec<T, VEC ? 4 : 1> v[VEC ? 2 : kPerLane];
    __device__ __forceinline__ void load(const T *at, int lane, int count) {
        if constexpr (VEC) {
#pragma unroll
            for (int h = 0; h < 2; ++h) v[h].template load<hagr::kKeep>(at + h * 128, lane);
        } else {
#pragma unroll
            for (int j = 0; j < kPerLane; ++j) {
                v[j].zero();
                if (j * 32 + lane < count) v[j].template load<hagr::kKeep>(at, j * 32 + lane);
            }
        }
    }
    __device__ __forceinline__ float2 pair(int j) const {
        if constexpr (VEC) return make_float2(v[j / 2].get(j % 2 * 2), v[j / 2].get(j % 2 * 2 + 1));
        else return make_float2(v[2 * j].get(0), v[2 * j + 1].get(0));
    }
};

template <typename T, bool VEC>
__device__ __forceinline__ void store8(const float2 (&v)[kPairs], T *at, int lane, int count) {
    if constexpr (VEC) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float four[4] = {v[2 * h].x, v[2 * h].y, v[2 * h + 1].x, v[2 * h + 1].y};
            hagr::Vec<T, 4> q;
            q.set(four);
            q.store(at + h * 128, lane);
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            hagr::Vec<T, 1> a, b;
            a.set(&v[j].x);
            b.set(&v[j].y);
            if (j * 64 + lane < count) a.store(at, j * 64 + lane);
            if (j * 64 + 32 + lane < count) b.store(at, j * 64 + 32 + lane);
        }
    }
}

__device__ __forceinline__ float2 from_e4m3(uint32_t two) {    // of the lower 16 bits
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(uint16_t(two)));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
__device__ __forceinline__ uint32_t to_e4m3(float2 v) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(v.y), "f"(v.x));
    return r;
}

template <bool VEC>
struct EightCodes {
    uint32_t w[VEC ? 2 : kPairs];                              // four codes, or two
    __device__ __forceinline__ void load(const uint8_t *block, int lane, int count) {
        if constexpr (VEC) {
#pragma unroll
            for (int h = 0; h < 2; ++h) w[h] = __ldcg(reinterpret_cast<const uint32_t *>(block + h * 128) + lane);
        } else {
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                const uint32_t a = j * 64 + lane < count ? __ldcg(block + j * 64 + lane) : 0;
                w[j] = a | (j * 64 + 32 + lane < count ? __ldcg(block + j * 64 + 32 + lane) : 0) << 8;
            }
        }
    }
    __device__ __forceinline__ float2 pair(int j) const { return from_e4m3(VEC ? w[j / 2] >> (j % 2 * 16) : w[j]); }
};

template <bool VEC>
__device__ __forceinline__ void store_codes(const float2 (&v)[kPairs], uint8_t *block, int lane, int count) {
    if constexpr (VEC) {
#pragma unroll
        for (int h = 0; h < 2; ++h) reinterpret_cast<uint32_t *>(block + h * 128)[lane] = to_e4m3(v[2 * h]) | to_e4m3(v[2 * h + 1]) << 16;
    } else {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            const uint32_t a = to_e4m3(v[j]);
            if (j * 64 + lane < count) block[j * 64 + lane] = uint8_t(a);
            if (j * 64 + 32 + lane < count) block[j * 64 + 32 + lane] = uint8_t(a >> 8);
        }
    }
}

// Root and reciprocal to an error of 2^-22 or less; what is below 2^-126 counts as zero.
__device__ __forceinline__ float root_of(float v) {
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float one_over(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float at_least_lowest(float v) {    // NaN stays NaN
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(kLowest));
    return r;
}
__device__ __forceinline__ float2 both(float f) { return make_float2(f, f); }

// The largest magnitude of a block; NaN does not count.
__device__ __forceinline__ float block_largest(const float2 (&v)[kPairs]) {
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) top = fmaxf(top, fmaxf(fabsf(v[j].x), fabsf(v[j].y)));
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
}
__device__ __forceinline__ float scale_of(float largest) { return fmaxf(largest * (1.0f / kTop), kLeastScale); }

// For the rare block with an infinity: NaN takes its place, which e4m3 has; infinity it has not.
__device__ __forceinline__ void drop_infinities(float2 (&v)[kPairs]) {
    const float none = __uint_as_float(0x7fffffffu);
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        if (!(fabsf(v[j].x) <= FLT_MAX)) v[j].x = none;
        if (!(fabsf(v[j].y) <= FLT_MAX)) v[j].y = none;
    }
}

// The value of e4m3 below or above a quotient of magnitude 448 at most, each with the probability of its nearness: 20 bits of
// the mantissa lie behind the type's three, and a random number of 20 bits (16, and half a unit of those) carries into them or does
// not.  Below 2^-6 the type's values are multiples of 2^-9, as are those of the binade above: the quotient is rounded there.
__device__ __forceinline__ float by_chance(float q, uint32_t random16) {
    const float a = fabsf(q), up = a < 0.015625f ? 0.015625f : 0.0f;
    const uint32_t r = (__float_as_uint(a + up) + (random16 << 4 | 8u)) & 0xfff00000u;
    const float v = __uint_as_float(r) - up;
    return a <= FLT_MAX ? copysignf(v, q) : q;
}

// m and the root of v in 8 bits.  A block seldom has an infinity or a root of zero: a test for the whole warp decides
// whether its elements are looked at one by one.
template <bool VEC, bool CHANCE>
__device__ __forceinline__ void store_8_bits(float2 (&m)[kPairs], float2 (&r)[kPairs], uint8_t *to_m, uint8_t *to_r, float2 *scale, int lane, int count,
                                             uint64_t key) {
    float top_m = block_largest(m), top_r = block_largest(r);
    if (fmaxf(top_m, top_r) > FLT_MAX) {
        drop_infinities(m);
        drop_infinities(r);
        top_m = block_largest(m);
        top_r = block_largest(r);
    }
    const float sm = scale_of(top_m), sr = scale_of(top_r);
    const float2 im = both(one_over(sm)), ir = both(one_over(sr));
    float least = r[0].x;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        least = fminf(least, fminf(r[j].x, r[j].y));
        m[j] = __fmul2_rn(m[j], im);
        r[j] = __fmul2_rn(r[j], ir);
    }
    if constexpr (CHANCE) {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            const uint32_t at = VEC ? j / 2 * 128 + lane * 4 + j % 2 * 2 : j * 64 + lane;
            const uint32_t x = random_bits(key, at), y = random_bits(key, at + (VEC ? 1 : 32));
            m[j] = make_float2(by_chance(m[j].x, x & 0xffffu), by_chance(m[j].y, y & 0xffffu));
            const float rx = by_chance(r[j].x, x >> 16), ry = by_chance(r[j].y, y >> 16);
            r[j] = make_float2(r[j].x > 0.0f ? at_least_lowest(rx) : rx, r[j].y > 0.0f ? at_least_lowest(ry) : ry);
        }
    } else if (__any_sync(0xffffffffu, least == 0.0f)) {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            if (r[j].x > 0.0f && r[j].x < kLowest) r[j].x = kLowest;
            if (r[j].y > 0.0f && r[j].y < kLowest) r[j].y = kLowest;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) r[j] = make_float2(at_least_lowest(r[j].x), at_least_lowest(r[j].y));
    }
    store_codes<VEC>(m, to_m, lane, count);
    store_codes<VEC>(r, to_r, lane, count);
    if (lane == 0) *scale = make_float2(sm, sr);
}

// Where the arrays of a tensor's blocks lie, from one of them on.
template <typename P, typename G, bool BITS8>
struct Arrays {
    using State = std::conditional_t<BITS8, uint8_t, float>;
    P *p;
    const G *g;
    __nv_bfloat16 *copy;
    State *m, *v;
    float2 *scales;
    __device__ __forceinline__ Arrays(const AdamArgs &a, int t, int64_t within) {
        const int64_t first = within * kAdamBlock, block = a.state[t] + within;
        p = static_cast<P *>(a.p[t]) + first;
        g = static_cast<const G *>(a.g[t]) + first;
        copy = a.copy[t] ? static_cast<__nv_bfloat16 *>(a.copy[t]) + first : nullptr;
        m = static_cast<State *>(a.mean) + block * kAdamBlock;
        v = static_cast<State *>(a.square) + block * kAdamBlock;
        scales = a.scales + block;
    }
};

// What a lane reads of one block.
template <typename P, typename G, bool BITS8, bool VEC>
struct Piece {
    Eight<P, VEC> p;
    Eight<G, VEC> g;
    std::conditional_t<BITS8, EightCodes<VEC>, Eight<float, VEC>> m, v;
    float2 scale;
    __device__ __forceinline__ void load(const Arrays<P, G, BITS8> &at, int block, int lane, int count) {
        p.load(at.p + block * kAdamBlock, lane, count);
        g.load(at.g + block * kAdamBlock, lane, count);
        m.load(at.m + block * kAdamBlock, lane, count);
        v.load(at.v + block * kAdamBlock, lane, count);
        if (BITS8) scale = __ldcg(at.scales + block);
    }
};

template <typename P, typename G, bool BITS8, bool CHANCE, bool VEC>
__device__ __forceinline__ void step_block(const AdamArgs &a, const Coefficients &c, uint64_t of_step, float keep_, float2 of_g,
                                           const Piece<P, G, BITS8, VEC> &in, const Arrays<P, G, BITS8> &to, int block, int lane, int count) {
    const float2 keep = both(keep_), of_m = both(of_g.x), of_v = both(of_g.y);
    const float2 of_old_m = both(BITS8 ? in.scale.x * a.b1 : a.b1), of_old_v = both(BITS8 ? in.scale.y * a.root2 : a.b2);
    float2 p[kPairs], m[kPairs], v[kPairs], r[kPairs];
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        const float2 g = in.g.pair(j);
        m[j] = __ffma2_rn(g, of_m, __fmul2_rn(in.m.pair(j), of_old_m));
        const float2 e = __fmul2_rn(g, of_v);
        v[j] = __fmul2_rn(in.v.pair(j), of_old_v);
        if (BITS8) v[j] = __fmul2_rn(v[j], v[j]);
        v[j] = __ffma2_rn(e, e, v[j]);
        r[j] = make_float2(root_of(v[j].x), root_of(v[j].y));
        const float2 d = __ffma2_rn(r[j], both(c.root), both(a.eps));
        const float2 x = __fmul2_rn(m[j], make_float2(one_over(d.x), one_over(d.y)));
        p[j] = __ffma2_rn(x, both(-c.rate), __fmul2_rn(in.p.pair(j), keep));
    }
    store8<P, VEC>(p, to.p + block * kAdamBlock, lane, count);
    if (to.copy) store8<__nv_bfloat16, VEC>(p, to.copy + block * kAdamBlock, lane, count);
    if constexpr (BITS8) {
        const uint64_t key = CHANCE ? mix64(of_step + uint64_t(to.scales + block - a.scales)) : 0;
        store_8_bits<VEC, CHANCE>(m, r, to.m + block * kAdamBlock, to.v + block * kAdamBlock, to.scales + block, lane, count, key);
    } else {
        store8<float, VEC>(m, to.m + block * kAdamBlock, lane, count);
        store8<float, VEC>(v, to.v + block * kAdamBlock, lane, count);
    }
}

// T blocks of a tensor from block `within` on; of the whole ones as many as the registers hold are read at once.
template <typename P, typename G, bool BITS8, bool CHANCE, int T>
__device__ __forceinline__ void step_unit(const AdamArgs &a, const Coefficients &c, uint64_t key, int t, uint32_t within) {
    constexpr int kWords = 2 * int(sizeof(P) + sizeof(G)) + (BITS8 ? 4 : 16);          // per lane and block
    constexpr int B = kWords * T <= 48 ? T : kWords * 2 <= 64 && T > 1 ? 2 : 1;
    const int lane = threadIdx.x & 31;
    const float keep = fmaf(-c.lr, a.decay[t], 1.0f);
    const Arrays<P, G, BITS8> at(a, t, within);
    if (within + T <= a.whole[t]) {
#pragma unroll 1
        for (int i = 0; i < T; i += B) {
            Piece<P, G, BITS8, true> in[B];
#pragma unroll
            for (int k = 0; k < B; ++k) in[k].load(at, i + k, lane, kAdamBlock);
            const float2 of_g = of_gradient(a, c.norm);
#pragma unroll
            for (int k = 0; k < B; ++k) step_block<P, G, BITS8, CHANCE, true>(a, c, key, keep, of_g, in[k], at, i + k, lane, kAdamBlock);
        }
    } else {
        const int n = int(min(uint32_t(T), a.blocks[t] - within));
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            if (T > 1 && within + i < a.whole[t]) {
                Piece<P, G, BITS8, true> in;
                in.load(at, i, lane, kAdamBlock);
                step_block<P, G, BITS8, CHANCE, true>(a, c, key, keep, of_gradient(a, c.norm), in, at, i, lane, kAdamBlock);
            } else {
                const int count = int(min(int64_t(kAdamBlock), a.len[t] - int64_t(within + i) * kAdamBlock));
                Piece<P, G, BITS8, false> in;
                in.load(at, i, lane, count);
                step_block<P, G, BITS8, CHANCE, false>(a, c, key, keep, of_gradient(a, c.norm), in, at, i, lane, count);
            }
        }
    }
}

// T: blocks that a warp takes at a time.  CHANCE: states are rounded by chance.
template <bool BITS8, bool CHANCE, int T>
__global__ void __launch_bounds__(kAdamThreads, T > 1 ? 2 : 4) adamw_kernel(const __grid_constant__ AdamArgs a) {
    hagk::pdl_launch_dependents();
    __shared__ Coefficients shared;
    __shared__ uint32_t first[kAdamList];                              // units before each tensor's
    if (threadIdx.x < kAdamList) first[threadIdx.x] = int(threadIdx.x) < a.tensors ? a.first[threadIdx.x] : 0xffffffffu;
    hagk::pdl_wait();
    Coefficients c{a.lr, a.rate, a.root};
    uint64_t key = 0;
    if constexpr (CHANCE) {
        __shared__ uint64_t shared_key;
        if (threadIdx.x == 0) shared_key = key_of(a);
        __syncthreads();
        key = shared_key;
    }
    if (a.step_at || a.lr_at) {
        if (threadIdx.x == 0) shared = coefficients(a);
        __syncthreads();
        c = shared;
    } else {
        __syncthreads();
    }
    c.norm = a.norm ? __ldcg(a.norm) : 0.0f;
    const int lane = threadIdx.x & 31;
    const uint32_t step = gridDim.x * kAdamWarps;
    for (uint32_t k = blockIdx.x * kAdamWarps + (threadIdx.x >> 5); k < a.units; k += step) {
        static_assert(kAdamList == 64, "two per lane");
        const int t = __popc(__ballot_sync(0xffffffffu, first[lane] <= k)) + __popc(__ballot_sync(0xffffffffu, first[lane + 32] <= k)) - 1;
        const uint32_t within = (k - first[t]) * T;
        if (a.p_bf16[t]) {
            if (a.g_bf16[t]) step_unit<__nv_bfloat16, __nv_bfloat16, BITS8, CHANCE, T>(a, c, key, t, within);
            else step_unit<__nv_bfloat16, float, BITS8, CHANCE, T>(a, c, key, t, within);
        } else {
            if (a.g_bf16[t]) step_unit<float, __nv_bfloat16, BITS8, CHANCE, T>(a, c, key, t, within);
            else step_unit<float, float, BITS8, CHANCE, T>(a, c, key, t, within);
        }
    }
}

int64_t blocks_of(int64_t len) { return len / kAdamBlock + (len % kAdamBlock != 0); }
bool dtype_ok(hag_dtype d) { return d == HAG_F32 || d == HAG_BF16; }
int size_of(hag_dtype d) { return d == HAG_F32 ? 4 : 2; }
bool on(const void *p, int bytes) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(bytes) == 0; }

// Blocks that a warp takes at a time where a launch has more than kFewBlocks: four, all of whose data is read before the
// first is worked on, so that what surrounds a block (its tensor, its addresses) is shared.  200 million bf16 parameters
// with 8-bit states: four 319 us, two 364, eight 363; one, as a launch of few blocks takes them, 391.  Of few blocks one at
// a time, for more warps.  Both sides, us, one and four at a time, at 5, 8, 12 and 24 million parameters: fp32 with 8-bit states
// 16.3 and 19.9, 25.0 and 26.8, 35.4 and 35.2, 67.4 and 65.1; fp32 with fp32 states 23.5 and 25.1, 35.7 and 36.4, 52.7 and 52.7,
// 103.9 and 100.9; rounded by chance 19.5 and 21.9, 28.3 and 32.4, 41.9 and 41.1, 77.2 and 75.9; other types meet there too.
// Where all is bf16 and 8 bits, a block has 2.5 KB and more of them have to be on their way: 12.8 and 13.1, 20.4 and 19.1,
// 28.7 and 23.9, 53.2 and 43.6 (6 million 16.1 and 15.5).
// The grid: with 8-bit states as many thread blocks as run at once (150 million fp32 parameters 377 us, a hundred per SM
// 423); with fp32 states up to a hundred per SM, which take their units as others end (150 million fp32 parameters 611 us,
// as many as run 690; of few blocks up to sixteen: 5 million 23.8 us, four 26.2).
constexpr int kUnit = 4;
constexpr int64_t kFewBlocks = kSms * 304;             // 11.5 million elements
constexpr int64_t kFewNarrowBlocks = kSms * 140;       // 5.3 million
constexpr int64_t kMostBlocks = 0x7fffffffLL;   // of a tensor and of a launch
}  // namespace

extern "C" int64_t hag_adamw_state_blocks(int32_t count, const int64_t *lengths) {
    if (count < 0 || (count > 0 && !lengths)) return -1;
    int64_t n = 0;
    for (int32_t t = 0; t < count; ++t) {
        if (lengths[t] < 0) return -1;
        const int64_t here = blocks_of(lengths[t]);
        if (here > kMostBlocks || n > (int64_t(1) << 50)) return -1;
        n += here;
    }
    return n;
}

extern "C" hag_status hag_adamw_step(int32_t count, void *const *params, const hag_dtype *param_dtypes, const void *const *grads,
                                     const hag_dtype *grad_dtypes, void *const *copies, const int64_t *lengths, const double *decays,
                                     hag_state_type state, void *mean, void *square, float *scales, const hag_adamw_options *options,
                                     void *cuda_stream) {
    if (!options) return HAG_ERR_NULL;
    const hag_adamw_options &o = *options;
    if (state != HAG_STATE32 && state != HAG_STATE8) return HAG_ERR_DTYPE;
    if (count < 0 || !(o.beta1 >= 0.0 && o.beta1 < 1.0) || !(o.beta2 >= 0.0 && o.beta2 < 1.0) || !(o.eps >= 0.0)) return HAG_ERR_ARG;
    if ((!o.step_device && o.step < 1) || (!o.lr_device && !(o.lr >= 0.0))) return HAG_ERR_ARG;
    if (o.total_norm && !(o.max_norm >= 0.0)) return HAG_ERR_ARG;
    if (o.rounding != HAG_NEAREST && o.rounding != HAG_CHANCE) return HAG_ERR_ARG;
    if (count > 0 && (!params || !param_dtypes || !grads || !grad_dtypes || !lengths || !decays)) return HAG_ERR_NULL;
    if (!on(o.lr_device, 4) || !on(o.total_norm, 4) || !on(o.step_device, 8)) return HAG_ERR_ALIGN;
    int64_t total = 0;
    for (int32_t t = 0; t < count; ++t) {
        if (!dtype_ok(param_dtypes[t]) || !dtype_ok(grad_dtypes[t])) return HAG_ERR_DTYPE;
        if (lengths[t] < 0 || !(decays[t] >= 0.0)) return HAG_ERR_ARG;
        if (blocks_of(lengths[t]) > kMostBlocks) return HAG_ERR_TOO_LARGE;
        total += blocks_of(lengths[t]);
        if (lengths[t] == 0 || !grads[t]) continue;
        if (!params[t]) return HAG_ERR_NULL;
        if (!on(params[t], size_of(param_dtypes[t])) || !on(grads[t], size_of(grad_dtypes[t])) || (copies && !on(copies[t], 2))) return HAG_ERR_ALIGN;
    }
    if (total == 0) return HAG_OK;
    if (!mean || !square || (state == HAG_STATE8 && !scales)) return HAG_ERR_NULL;
    if (!hagl::aligned16(mean) || !hagl::aligned16(square) || !hagl::aligned16(scales)) return HAG_ERR_ALIGN;
    AdamArgs a{};
    a.mean = mean;
    a.square = square;
    a.scales = reinterpret_cast<float2 *>(scales);
    a.lr = float(o.lr);
    a.b1 = float(o.beta1);
    a.rest1 = float(1.0 - o.beta1);
    a.b2 = float(o.beta2);
    a.root2 = float(std::sqrt(o.beta2));
    a.root_rest2 = float(std::sqrt(1.0 - o.beta2));
    a.eps = float(o.eps);
    a.beta1 = o.beta1;
    a.beta2 = o.beta2;
    a.seed = o.seed;
    a.step = o.step;
    a.lr_at = o.lr_device;
    a.step_at = o.step_device;
    a.norm = o.total_norm;
    a.max_norm = float(o.max_norm);
    if (!o.step_device) {
        const double rest = 1.0 / (1.0 - std::pow(o.beta1, double(o.step)));
        a.rate = float(o.lr_device ? rest : o.lr * rest);
        a.root = float(1.0 / std::sqrt(1.0 - std::pow(o.beta2, double(o.step))));
    }
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool bits8 = state == HAG_STATE8, chance = bits8 && o.rounding == HAG_CHANCE;
    cudaError_t err = cudaSuccess;
    int64_t at = 0, blocks = 0;
    auto launch = [&]() {
        if (a.tensors > 0) {
            bool narrow = bits8 && !chance;
            for (int i = 0; i < a.tensors; ++i) narrow = narrow && a.p_bf16[i] && a.g_bf16[i];
            const bool many = blocks > (narrow ? kFewNarrowBlocks : kFewBlocks);
            a.units = 0;
            for (int i = 0; i < a.tensors; ++i) {
                a.first[i] = a.units;
                a.units += many ? (a.blocks[i] + kUnit - 1) / kUnit : a.blocks[i];
            }
            const unsigned grid = unsigned(std::min<int64_t>((int64_t(a.units) + kAdamWarps - 1) / kAdamWarps, kSms * (bits8 ? (many ? 2 : 4) : (many ? 100 : 16))));
            void (*const kernel)(AdamArgs) = chance ? many ? adamw_kernel<true, true, kUnit> : adamw_kernel<true, true, 1>
                                             : bits8 ? many ? adamw_kernel<true, false, kUnit> : adamw_kernel<true, false, 1>
                                                     : many ? adamw_kernel<false, false, kUnit> : adamw_kernel<false, false, 1>;
            err = hagl::launch_pdl<AdamArgs>(kernel, grid, unsigned(kAdamThreads), a, s);
        }
        a.tensors = 0;
        blocks = 0;
    };
    for (int32_t t = 0; t < count && err == cudaSuccess; ++t) {
        const int64_t here = blocks_of(lengths[t]);
        if (here == 0) continue;
        if (grads[t]) {
            if (a.tensors == kAdamList || blocks + here > kMostBlocks) launch();
            if (err != cudaSuccess) break;
            const int i = a.tensors++, ps = size_of(param_dtypes[t]), gs = size_of(grad_dtypes[t]);
            a.p[i] = params[t];
            a.g[i] = grads[t];
            a.copy[i] = copies ? copies[t] : nullptr;
            a.len[i] = lengths[t];
            a.state[i] = at;
            a.decay[i] = float(decays[t]);
            a.p_bf16[i] = ps == 2;
            a.g_bf16[i] = gs == 2;
            a.blocks[i] = uint32_t(here);
            a.whole[i] = on(params[t], 4 * ps) && on(grads[t], 4 * gs) && on(a.copy[i], 8) ? uint32_t(lengths[t] / kAdamBlock) : 0;
            blocks += here;
        }
        at += here;
    }
    if (err == cudaSuccess) launch();
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
