// Layer norm over the columns of a matrix, forward and backward.
//   forward   mu = mean(x_r), rstd = 1 / sqrt(mean((x_r - mu)^2) + eps), y = (x - mu) * rstd * w + b
//   backward  xh = (x - mu) * rstd, q = g * w:  gx = rstd * (q - mean(q) - xh * mean(q * xh))
//             gw = sum over rows of g * xh,  gb = sum over rows of g
// The variance is the mean of squared differences from the mean (two steps over the row, never
// E[x^2] - mu^2, which cancels when the mean is large against the spread).
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "hag.h"
#include "hag_kernels.cuh"
#include "hag_launch.h"
#include "hag_rows.cuh"

namespace {

struct NormArgs {
    int64_t n;
    int32_t D;
    int32_t w_bf16;             // type of w, b, gw, gb
    const void *x, *w, *b;
    const void *g;              // backward: gradient of y
    int64_t ld_x, ld_g, ld_y;
    void *y;                    // forward: y; backward: gx
    float *mean, *rstd;
    const float *mean_in, *rstd_in;
    float eps;
    float *partial;             // backward: [parts][2][D]
    void *gw, *gb;
    int32_t parts;
};

constexpr int kRowThreads = 256;

template <typename T>
__device__ __forceinline__ float load1(const void *p, int64_t i) {
    hagr::Vec<T, 1> v;
    v.template load<hagr::kKeep>(p, i);
    return v.get(0);
}
template <typename T>
__device__ __forceinline__ void store1(void *p, int64_t i, float f) {
    hagr::Vec<T, 1> v;
    v.set(&f);
    v.store(p, i);
}
__device__ __forceinline__ float load_param(const void *p, int bf16, int64_t i) {
    return bf16 ? load1<__nv_bfloat16>(p, i) : load1<float>(p, i);
}
__device__ __forceinline__ void store_param(void *p, int bf16, int64_t i, float v) {
    if (bf16) store1<__nv_bfloat16>(p, i, v); else store1<float>(p, i, v);
}

// Sum over the block, returned to every thread; `slot` alternates so that one barrier per sum is enough.
template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float *slot) {
    v = hagr::warp_sum(v);
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) s += slot[w];
    return s;
}

// Rows of any width: one block per row, which it reads three times (the second and third time out of the caches).
template <typename T>
__global__ void __launch_bounds__(kRowThreads) norm_fwd_any_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float slot[2][kRowThreads / 32];
    const float cols = float(p.D);
    hagk::pdl_wait();
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x) {
        const T *x = static_cast<const T *>(p.x) + r * p.ld_x;
        T *y = static_cast<T *>(p.y) + r * p.ld_y;
        float s = 0.0f;
        for (int32_t c = threadIdx.x; c < p.D; c += kRowThreads) s += load1<T>(x, c);
        const float mean = block_sum<kRowThreads>(s, slot[0]) / cols;
        s = 0.0f;
        for (int32_t c = threadIdx.x; c < p.D; c += kRowThreads) {
            const float d = load1<T>(x, c) - mean;
            s += d * d;
        }
        const float rstd = rsqrtf(block_sum<kRowThreads>(s, slot[1]) / cols + p.eps);
        for (int32_t c = threadIdx.x; c < p.D; c += kRowThreads) {
            float v = (load1<T>(x, c) - mean) * rstd;
            if (p.w) v *= load_param(p.w, p.w_bf16, c);
            if (p.b) v += load_param(p.b, p.w_bf16, c);
            store1<T>(y, c, v);
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) norm_bwd_any_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float slot[2][2][kRowThreads / 32];
    const float cols = float(p.D);
    hagk::pdl_wait();
    int turn = 0;
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x, turn ^= 1) {
        const T *x = static_cast<const T *>(p.x) + r * p.ld_x;
        const T *g = static_cast<const T *>(p.g) + r * p.ld_g;
        T *gx = static_cast<T *>(p.y) + r * p.ld_y;
        const float mean = __ldcg(p.mean_in + r), rstd = __ldcg(p.rstd_in + r);
        float s1 = 0.0f, s2 = 0.0f;
        for (int32_t c = threadIdx.x; c < p.D; c += kRowThreads) {
            const float q = load1<T>(g, c) * (p.w ? load_param(p.w, p.w_bf16, c) : 1.0f);
            s1 += q;
            s2 += q * ((load1<T>(x, c) - mean) * rstd);
        }
        s1 = block_sum<kRowThreads>(s1, slot[turn][0]) / cols;
        s2 = block_sum<kRowThreads>(s2, slot[turn][1]) / cols;
        for (int32_t c = threadIdx.x; c < p.D; c += kRowThreads) {
            const float q = load1<T>(g, c) * (p.w ? load_param(p.w, p.w_bf16, c) : 1.0f);
            const float xh = (load1<T>(x, c) - mean) * rstd;
            store1<T>(gx, c, rstd * (q - s1 - xh * s2));
        }
    }
}

// gw and gb of one strip of 32 columns and one part of the rows.
constexpr int kStripRows = 8;
template <typename T>
__global__ void __launch_bounds__(32 * kStripRows) norm_params_any_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float sum[2][kStripRows][32];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane;
    const int64_t step = int64_t(p.parts) * kStripRows;
    float aw = 0.0f, ab = 0.0f;
    hagk::pdl_wait();
    if (c < p.D)
        for (int64_t r = int64_t(blockIdx.y) * kStripRows + part; r < p.n; r += step) {
            const float g = load1<T>(p.g, r * p.ld_g + c);
            aw += g * ((load1<T>(p.x, r * p.ld_x + c) - __ldcg(p.mean_in + r)) * __ldcg(p.rstd_in + r));
            ab += g;
        }
    sum[0][part][lane] = aw;
    sum[1][part][lane] = ab;
    __syncthreads();
    if (part < 2 && c < p.D) {
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < kStripRows; ++k) s += sum[part][k][lane];
        p.partial[(int64_t(blockIdx.y) * 2 + part) * p.D + c] = s;
    }
}

__global__ void __launch_bounds__(kRowThreads) norm_params_join_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    const int64_t k = int64_t(blockIdx.x) * kRowThreads + threadIdx.x;       // column of [gw | gb]
    hagk::pdl_wait();
    if (k >= 2 * int64_t(p.D)) return;
    float s = 0.0f;
    for (int q = 0; q < p.parts; ++q) s += __ldcg(p.partial + int64_t(q) * 2 * p.D + k);
    void *to = k < p.D ? p.gw : p.gb;
    if (to) store_param(to, p.w_bf16, k < p.D ? k : k - p.D, s);
}

constexpr int kParts = 64;

cudaError_t launch2d(void (*kernel)(NormArgs), dim3 grid, unsigned threads, const NormArgs &p, cudaStream_t s) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

bool dtype_ok(hag_dtype d) { return d == HAG_F32 || d == HAG_BF16; }
int elem_size(hag_dtype d) { return d == HAG_F32 ? 4 : 2; }

struct Need {
    const void *p;
    int64_t ld;
    bool rows;      // an n x D matrix of `dtype` (else a vector of the parameters' type)
    bool out;
};

template <int N>
hag_status norm_check(int64_t n, int32_t D, hag_dtype dtype, hag_dtype w_dtype, const Need (&a)[N]) {
    if (!dtype_ok(dtype) || !dtype_ok(w_dtype)) return HAG_ERR_DTYPE;
    if (n < 0 || D <= 0) return HAG_ERR_ARG;
    if (D > (1 << 30)) return HAG_ERR_TOO_LARGE;
    for (const Need &x : a) {
        if (!x.rows) continue;
        if (x.ld < 0 || (x.out && n > 1 && x.ld < D)) return HAG_ERR_ARG;
        if (!x.p && n > 0) return HAG_ERR_NULL;
    }
    for (const Need &x : a)
        if (!hagr::element_aligned(x.p, x.rows ? elem_size(dtype) : elem_size(w_dtype))) return HAG_ERR_ALIGN;
    for (const Need &x : a)              // in place row by row is fine; the same start with other rows is not
        for (const Need &y : a)
            if (n > 1 && x.rows && y.rows && y.out && x.p == y.p && x.ld != y.ld) return HAG_ERR_ARG;
    return HAG_OK;
}

}  // namespace

extern "C" hag_status hag_layer_norm_fwd(int64_t n, int32_t D, hag_dtype dtype, const void *x, int64_t ld_x, const void *weight,
                                         const void *bias, hag_dtype weight_dtype, float eps, void *y, int64_t ld_y, float *mean,
                                         float *rstd, void *cuda_stream) {
    const Need need[] = {{x, ld_x, true, false}, {y, ld_y, true, true}, {weight, 0, false, false}, {bias, 0, false, false}};
    const hag_status st = norm_check(n, D, dtype, weight_dtype, need);
    if (st != HAG_OK) return st;
    if (!(eps >= 0.0f)) return HAG_ERR_ARG;
    if (!hagr::element_aligned(mean, 4) || !hagr::element_aligned(rstd, 4)) return HAG_ERR_ALIGN;
    if (n == 0) return HAG_OK;
    NormArgs p{};
    p.n = n; p.D = D; p.w_bf16 = weight_dtype == HAG_BF16;
    p.x = x; p.ld_x = ld_x; p.w = weight; p.b = bias; p.y = y; p.ld_y = ld_y; p.mean = mean; p.rstd = rstd; p.eps = eps;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const unsigned grid = unsigned(std::min<int64_t>(n, 148 * 8));
    const cudaError_t err = hagl::launch_pdl(dtype == HAG_F32 ? norm_fwd_any_kernel<float> : norm_fwd_any_kernel<__nv_bfloat16>, grid,
                                             unsigned(kRowThreads), p, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}

extern "C" size_t hag_layer_norm_bwd_workspace_bytes(int64_t n, int32_t D) {
    if (n < 0 || D <= 0) return 0;
    return size_t(kParts) * 2 * size_t(D) * 4;
}

extern "C" hag_status hag_layer_norm_bwd(int64_t n, int32_t D, hag_dtype dtype, const void *grad_y, int64_t ld_grad_y, const void *x,
                                         int64_t ld_x, const float *mean, const float *rstd, const void *weight,
                                         hag_dtype weight_dtype, void *grad_x, int64_t ld_grad_x, void *grad_weight, void *grad_bias,
                                         void *workspace, void *cuda_stream) {
    const Need need[] = {{grad_y, ld_grad_y, true, false}, {x, ld_x, true, false}, {grad_x, ld_grad_x, true, true},
                         {weight, 0, false, false}, {grad_weight, 0, false, true}, {grad_bias, 0, false, true}};
    const hag_status st = norm_check(n, D, dtype, weight_dtype, need);
    if (st != HAG_OK) return st;
    if (n > 0 && (!mean || !rstd)) return HAG_ERR_NULL;
    if (!hagr::element_aligned(mean, 4) || !hagr::element_aligned(rstd, 4)) return HAG_ERR_ALIGN;
    const bool params = grad_weight || grad_bias;
    if (params && !workspace) return HAG_ERR_WORKSPACE;
    if (!hagl::aligned16(workspace)) return HAG_ERR_ALIGN;
    NormArgs p{};
    p.n = n; p.D = D; p.w_bf16 = weight_dtype == HAG_BF16;
    p.x = x; p.ld_x = ld_x; p.g = grad_y; p.ld_g = ld_grad_y; p.w = weight; p.y = grad_x; p.ld_y = ld_grad_x;
    p.mean_in = mean; p.rstd_in = rstd; p.partial = static_cast<float *>(workspace); p.gw = grad_weight; p.gb = grad_bias;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err = cudaSuccess;
    const bool f32 = dtype == HAG_F32;
    if (params) {      // first: grad_x may take the place of grad_y or x
        p.parts = int(std::min<int64_t>(std::max<int64_t>((n + kStripRows - 1) / kStripRows, 1), kParts));
        err = launch2d(f32 ? norm_params_any_kernel<float> : norm_params_any_kernel<__nv_bfloat16>,
                       dim3(unsigned((D + 31) / 32), unsigned(p.parts)), 32 * kStripRows, p, s);
        if (err == cudaSuccess)
            err = hagl::launch_pdl(norm_params_join_kernel, unsigned((2 * int64_t(D) + kRowThreads - 1) / kRowThreads), unsigned(kRowThreads), p, s);
    }
    if (err == cudaSuccess && n > 0)
        err = hagl::launch_pdl(f32 ? norm_bwd_any_kernel<float> : norm_bwd_any_kernel<__nv_bfloat16>,
                               unsigned(std::min<int64_t>(n, 148 * 8)), unsigned(kRowThreads), p, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
