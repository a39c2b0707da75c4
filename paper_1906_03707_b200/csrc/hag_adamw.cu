// One AdamW step over a list of tensors, in place.  With g' = c g, c = min(1, max_norm / (N + 1e-6)) or 1:
//   m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = p (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// The states of all tensors lie in one array of blocks of 256 elements, a tensor's first block behind the previous
// tensor's last, so a launch needs few addresses and the states' alignment does not depend on the parameters'.
// In 8 bits a block holds m and sqrt(v) as e4m3 with an fp32 scale each: the largest of the block becomes 448.  The root
// rather than v: it spans half the binades, and it is what the step divides by.  A positive root is never stored as
// zero, since m of the same element, which has a scale of its own, might not be: m / eps would be a step of any size.
//
// A warp takes a block, eight elements per lane; the largest of a block is two warp-wide maxima.
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>

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
    uint32_t blocks;                            // of this launch's tensors
    void *mean, *square;                        // of all tensors
    float2 *scales;
    float lr, b1, rest1, b2, rest2, eps;        // rest = 1 - b
    float rate, root;                           // lr / (1 - b1^t), 1 / sqrt(1 - b2^t): where the step is the host's
    double beta1, beta2;
    const float *lr_at, *norm;
    const int64_t *step_at;
    float max_norm;
    void *p[kAdamList];
    const void *g[kAdamList];
    void *copy[kAdamList];
    int64_t len[kAdamList], state[kAdamList];   // elements; first block of the states
    float decay[kAdamList];
    uint32_t first[kAdamList];                  // first block among this launch's
    uint8_t p_bf16[kAdamList], g_bf16[kAdamList];
    uint8_t vec[kAdamList];                     // whether four elements can be read at once
};
static_assert(sizeof(AdamArgs) <= 4096, "the list must fit in the parameters of a launch");

struct Coefficients {
    float lr, rate, root, factor;
};

__device__ double power(double base, int64_t n) {          // base^n by squaring
    double r = 1.0;
    for (; n > 0; n >>= 1, base *= base)
        if (n & 1) r *= base;
    return r;
}

// What the step, the rate and the norm on the device make of the coefficients; one thread's work.
__device__ __forceinline__ Coefficients coefficients(const AdamArgs &p) {
    Coefficients c{p.lr, p.rate, p.root, 1.0f};
    if (p.lr_at) c.lr = __ldcg(p.lr_at);
    if (p.step_at) {
        const int64_t t = max(int64_t(1), int64_t(__ldcg(reinterpret_cast<const long long *>(p.step_at))));
        c.rate = float(1.0 / (1.0 - power(p.beta1, t)));
        c.root = float(1.0 / sqrt(1.0 - power(p.beta2, t)));
    }
    if (p.lr_at || p.step_at) c.rate = float(double(c.lr) * double(c.rate));
    if (p.norm) {
        const float ratio = p.max_norm / (__ldcg(p.norm) + 1e-6f);
        c.factor = ratio >= 1.0f ? 1.0f : ratio;               // a norm that is no number gives a factor that is none
    }
    return c;
}

// The elements of a block that a lane holds: two groups of four, 128 apart, so that a warp's accesses are contiguous;
// or, where the addresses do not allow that, eight single ones, 32 apart.
template <bool VEC>
__device__ __forceinline__ int place(int lane, int j) {
    return VEC ? (j / 4) * 128 + lane * 4 + j % 4 : j * 32 + lane;
}

template <typename T, bool VEC>
__device__ __forceinline__ void load8(float (&v)[kPerLane], const void *at, int64_t first, int lane, int count) {
    if constexpr (VEC) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            hagr::Vec<T, 4> q;
            q.template load<hagr::kKeep>(static_cast<const T *>(at) + first + h * 128, lane);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[h * 4 + j] = q.get(j);
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPerLane; ++j) {
            hagr::Vec<T, 1> q;
            q.zero();
            if (j * 32 + lane < count) q.template load<hagr::kKeep>(at, first + j * 32 + lane);
            v[j] = q.get(0);
        }
    }
}

template <typename T, bool VEC>
__device__ __forceinline__ void store8(const float (&v)[kPerLane], void *at, int64_t first, int lane, int count) {
    if constexpr (VEC) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            hagr::Vec<T, 4> q;
            q.set(v + h * 4);
            q.store(static_cast<T *>(at) + first + h * 128, lane);
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPerLane; ++j) {
            hagr::Vec<T, 1> q;
            q.set(v + j);
            if (j * 32 + lane < count) q.store(at, first + j * 32 + lane);
        }
    }
}

__device__ __forceinline__ float2 from_e4m3(uint16_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
__device__ __forceinline__ uint16_t to_e4m3(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

template <bool VEC>
__device__ __forceinline__ void load_codes(float (&v)[kPerLane], const uint8_t *block, int lane, int count) {
#pragma unroll
    for (int j = 0; j < kPerLane; j += VEC ? 4 : 2) {
        if constexpr (VEC) {
            const uint32_t w = __ldcg(reinterpret_cast<const uint32_t *>(block + place<true>(lane, j)));
            const float2 a = from_e4m3(uint16_t(w)), b = from_e4m3(uint16_t(w >> 16));
            v[j] = a.x; v[j + 1] = a.y; v[j + 2] = b.x; v[j + 3] = b.y;
        } else {
            const uint32_t a = place<false>(lane, j) < count ? __ldcg(block + place<false>(lane, j)) : 0;
            const uint32_t b = place<false>(lane, j + 1) < count ? __ldcg(block + place<false>(lane, j + 1)) : 0;
            const float2 t = from_e4m3(uint16_t(a | b << 8));
            v[j] = t.x; v[j + 1] = t.y;
        }
    }
}
template <bool VEC>
__device__ __forceinline__ void store_codes(const float (&v)[kPerLane], uint8_t *block, int lane, int count) {
#pragma unroll
    for (int j = 0; j < kPerLane; j += VEC ? 4 : 2) {
        const uint32_t a = to_e4m3(v[j], v[j + 1]);
        if constexpr (VEC) {
            *reinterpret_cast<uint32_t *>(block + place<true>(lane, j)) = a | uint32_t(to_e4m3(v[j + 2], v[j + 3])) << 16;
        } else {
            if (place<false>(lane, j) < count) block[place<false>(lane, j)] = uint8_t(a);
            if (place<false>(lane, j + 1) < count) block[place<false>(lane, j + 1)] = uint8_t(a >> 8);
        }
    }
}

__device__ __forceinline__ float root_of(float v) {            // to two units in the last place
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// The largest finite magnitude of the block (the bits of positive floats are ordered as the floats are).
__device__ __forceinline__ float block_largest(const float (&v)[kPerLane]) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
        const uint32_t b = __float_as_uint(fabsf(v[j]));
        top = max(top, b < 0x7f800000u ? b : 0u);
    }
    return __uint_as_float(__reduce_max_sync(0xffffffffu, top));
}
__device__ __forceinline__ float scale_of(float largest) { return fmaxf(largest * (1.0f / kTop), kLeastScale); }

// One block of one tensor.  A value that is not finite is stored as NaN, which e4m3 has; infinity it has not.
template <typename P, typename G, bool BITS8, bool VEC>
__device__ __forceinline__ void step_block(const AdamArgs &a, const Coefficients &c, int t, int64_t first, int64_t block, int count) {
    const int lane = threadIdx.x & 31;
    float p[kPerLane], g[kPerLane], m[kPerLane], v[kPerLane];
    load8<P, VEC>(p, a.p[t], first, lane, count);
    load8<G, VEC>(g, a.g[t], first, lane, count);
    uint8_t *const codes_m = static_cast<uint8_t *>(a.mean) + block * kAdamBlock, *const codes_r = static_cast<uint8_t *>(a.square) + block * kAdamBlock;
    if constexpr (BITS8) {
        load_codes<VEC>(m, codes_m, lane, count);
        load_codes<VEC>(v, codes_r, lane, count);
        const float2 s = __ldcg(a.scales + block);
#pragma unroll
        for (int j = 0; j < kPerLane; ++j) {
            m[j] *= s.x;
            v[j] *= s.y;
            v[j] *= v[j];
        }
    } else {
        load8<float, VEC>(m, a.mean, block * kAdamBlock, lane, count);
        load8<float, VEC>(v, a.square, block * kAdamBlock, lane, count);
    }
    const float keep = fmaf(-c.lr, a.decay[t], 1.0f);
    float r[kPerLane];
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
        const float d = g[j] * c.factor;
        m[j] = fmaf(a.b1, m[j], a.rest1 * d);
        v[j] = fmaf(a.b2, v[j], a.rest2 * (d * d));
        r[j] = root_of(v[j]);
        p[j] = fmaf(p[j], keep, -c.rate * __fdividef(m[j], fmaf(r[j], c.root, a.eps)));
    }
    store8<P, VEC>(p, a.p[t], first, lane, count);
    if (a.copy[t]) store8<__nv_bfloat16, VEC>(p, a.copy[t], first, lane, count);
    if constexpr (BITS8) {
        const float sm = scale_of(block_largest(m)), sr = scale_of(block_largest(r));
        const float im = __fdividef(1.0f, sm), ir = __fdividef(1.0f, sr);
        const float none = __uint_as_float(0x7fffffffu);
#pragma unroll
        for (int j = 0; j < kPerLane; ++j) {
            m[j] = fabsf(m[j]) <= FLT_MAX ? m[j] * im : none;
            r[j] = r[j] <= FLT_MAX ? (r[j] > 0.0f ? fmaxf(r[j] * ir, kLowest) : 0.0f) : none;
        }
        store_codes<VEC>(m, codes_m, lane, count);
        store_codes<VEC>(r, codes_r, lane, count);
        if (lane == 0) a.scales[block] = make_float2(sm, sr);
    } else {
        store8<float, VEC>(m, a.mean, block * kAdamBlock, lane, count);
        store8<float, VEC>(v, a.square, block * kAdamBlock, lane, count);
    }
}

template <bool BITS8>
__global__ void __launch_bounds__(kAdamThreads, 4) adamw_kernel(const __grid_constant__ AdamArgs a) {
    hagk::pdl_launch_dependents();
    __shared__ Coefficients shared;
    hagk::pdl_wait();
    if (threadIdx.x == 0) shared = coefficients(a);
    __syncthreads();
    const Coefficients c = shared;
    int t = 0;
    const uint32_t step = gridDim.x * kAdamWarps;
    for (uint64_t k = blockIdx.x * kAdamWarps + (threadIdx.x >> 5); k < a.blocks; k += step) {
        while (t + 1 < a.tensors && a.first[t + 1] <= k) ++t;
        const int64_t within = int64_t(k - a.first[t]), first = within * kAdamBlock, block = a.state[t] + within;
        const int count = int(min(int64_t(kAdamBlock), a.len[t] - first));
        const bool vec = a.vec[t] && count == kAdamBlock;
        auto run = [&](auto p, auto g) {
            using P = decltype(p);
            using G = decltype(g);
            if (vec) step_block<P, G, BITS8, true>(a, c, t, first, block, count);
            else step_block<P, G, BITS8, false>(a, c, t, first, block, count);
        };
        if (a.p_bf16[t]) {
            if (a.g_bf16[t]) run(__nv_bfloat16(), __nv_bfloat16());
            else run(__nv_bfloat16(), float());
        } else {
            if (a.g_bf16[t]) run(float(), __nv_bfloat16());
            else run(float(), float());
        }
    }
}

int64_t blocks_of(int64_t len) { return len / kAdamBlock + (len % kAdamBlock != 0); }
bool dtype_ok(hag_dtype d) { return d == HAG_F32 || d == HAG_BF16; }
int size_of(hag_dtype d) { return d == HAG_F32 ? 4 : 2; }
bool on(const void *p, int bytes) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(bytes) == 0; }

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
    if (!hagl::aligned16(mean) || !hagl::aligned16(square) || !on(scales, 8)) return HAG_ERR_ALIGN;
    AdamArgs a{};
    a.mean = mean;
    a.square = square;
    a.scales = reinterpret_cast<float2 *>(scales);
    a.lr = float(o.lr);
    a.b1 = float(o.beta1);
    a.rest1 = float(1.0 - o.beta1);
    a.b2 = float(o.beta2);
    a.rest2 = float(1.0 - o.beta2);
    a.eps = float(o.eps);
    a.beta1 = o.beta1;
    a.beta2 = o.beta2;
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
    void (*const kernel)(AdamArgs) = state == HAG_STATE8 ? adamw_kernel<true> : adamw_kernel<false>;
    cudaError_t err = cudaSuccess;
    int64_t at = 0, blocks = 0;
    auto launch = [&]() {
        a.blocks = uint32_t(blocks);
        const unsigned grid = unsigned(std::min<int64_t>((blocks + kAdamWarps - 1) / kAdamWarps, kSms * 4));
        if (a.tensors > 0) err = hagl::launch_pdl<AdamArgs>(kernel, grid, unsigned(kAdamThreads), a, s);
        a.tensors = 0;
        blocks = 0;
    };
    for (int32_t t = 0; t < count && err == cudaSuccess; ++t) {
        const int64_t here = blocks_of(lengths[t]);
        if (here == 0) continue;
        if (grads[t]) {
            if (a.tensors == kAdamList || blocks + here > kMostBlocks) launch();
            if (err != cudaSuccess) break;
            const int i = a.tensors++;
            a.p[i] = params[t];
            a.g[i] = grads[t];
            a.copy[i] = copies ? copies[t] : nullptr;
            a.len[i] = lengths[t];
            a.state[i] = at;
            a.decay[i] = float(decays[t]);
            a.first[i] = uint32_t(blocks);
            a.p_bf16[i] = param_dtypes[t] == HAG_BF16;
            a.g_bf16[i] = grad_dtypes[t] == HAG_BF16;
            a.vec[i] = on(params[t], 4 * size_of(param_dtypes[t])) && on(grads[t], 4 * size_of(grad_dtypes[t])) && on(a.copy[i], 8);
            blocks += here;
        }
        at += here;
    }
    if (err == cudaSuccess) launch();
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
