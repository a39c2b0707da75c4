// Layer norm over the columns of a matrix, forward and backward.
//   forward   mu = mean(x_r), rstd = 1 / sqrt(mean((x_r - mu)^2) + eps), y = (x - mu) * rstd * w + b
//   backward  xh = (x - mu) * rstd, q = g * w:  gx = rstd * (q - mean(q) - xh * mean(q * xh))
//             gw = sum over rows of g * xh,  gb = sum over rows of g
// The variance is the mean of squared differences from the mean (two steps over the row, never
// E[x^2] - mu^2, which cancels when the mean is large against the spread).
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
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

// ---------------------------------------------------------------------------------------------------------------
// Rows held in registers.  A group of lanes owns a row, K vectors of V elements per lane, so a row is read once; the
// weights stay in registers over all rows of the group.
//   warp kernels : L = 8, 16 or 32 lanes of a warp per row, R rows per group at a time (loads in flight)
//   block kernels: a whole block per row, sums over the block through shared memory
constexpr int kPerLane = 16;              // elements of a row per lane, at most
constexpr int kWarpThreads = 256;
constexpr int kWarpRows = kWarpThreads / 32;

template <int V, int K>
__device__ __forceinline__ void load_params(const void *p, int bf16, int32_t D, int first, int step, float fill, float *v) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int32_t c = (first + k * step) * V + j;
            v[k * V + j] = p && c < D ? load_param(p, bf16, c) : fill;
        }
}

// Sums of R values per lane over the L lanes of a group: lanes trade halves of the list while it has more than one
// value, so the R sums take about L + R shuffles' worth less than R butterflies, and each lane ends with ONE of the
// sums: number (gl * R / L).  What follows a sum (a division, a root) is then done once, not once per value.
template <int L, int R>
__device__ __forceinline__ float spread_sums(const float (&in)[R], int gl) {
    float v[R];
#pragma unroll
    for (int i = 0; i < R; ++i) v[i] = in[i];
    int o = L / 2;
#pragma unroll
    for (int h = R / 2; h >= 1; h /= 2, o /= 2) {
        const bool upper = gl & o;
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const float keep = upper ? v[i + h] : v[i], give = upper ? v[i] : v[i + h];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
#pragma unroll
    for (; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    return v[0];
}
// Value number i of a list spread that way, in every lane of the group.
template <int L, int R>
__device__ __forceinline__ float spread_get(float v, int i, int lane) {
    return __shfl_sync(0xffffffffu, v, (lane & ~(L - 1)) + i * (L / R));
}

// Two fp32 operations per instruction; N is even or 1.
template <int N>
struct Pairs {
    float v[N];
    template <typename F2, typename F1>
    static __device__ __forceinline__ void each(F2 f2, F1 f1) {
#pragma unroll
        for (int j = 0; j + 1 < N; j += 2) f2(j);
        if constexpr (N % 2) f1(N - 1);
    }
    __device__ __forceinline__ float2 two(int j) const { return make_float2(v[j], v[j + 1]); }
    __device__ __forceinline__ void put(int j, float2 t) { v[j] = t.x; v[j + 1] = t.y; }
    __device__ __forceinline__ void fill(float f) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = f;
    }
    __device__ __forceinline__ void add(const Pairs &a) {                                     // v += a
        each([&](int j) { put(j, __fadd2_rn(two(j), a.two(j))); }, [&](int j) { v[j] += a.v[j]; });
    }
    __device__ __forceinline__ void fma(const Pairs &a, const Pairs &b) {                     // v += a * b
        each([&](int j) { put(j, __ffma2_rn(a.two(j), b.two(j), two(j))); }, [&](int j) { v[j] = fmaf(a.v[j], b.v[j], v[j]); });
    }
    __device__ __forceinline__ void mul(const Pairs &a) {
        each([&](int j) { put(j, __fmul2_rn(two(j), a.two(j))); }, [&](int j) { v[j] *= a.v[j]; });
    }
    __device__ __forceinline__ void shift_scale(float s, float m) {                           // v = (v + s) * m
        each([&](int j) { put(j, __fmul2_rn(__fadd2_rn(two(j), make_float2(s, s)), make_float2(m, m))); },
             [&](int j) { v[j] = (v[j] + s) * m; });
    }
    __device__ __forceinline__ void mul_all(float m) {
        each([&](int j) { put(j, __fmul2_rn(two(j), make_float2(m, m))); }, [&](int j) { v[j] *= m; });
    }
    __device__ __forceinline__ void shift(float s) {                                          // v += s
        each([&](int j) { put(j, __fadd2_rn(two(j), make_float2(s, s))); }, [&](int j) { v[j] += s; });
    }
    __device__ __forceinline__ void affine(float m, float s) {                                // v = v * m + s
        each([&](int j) { put(j, __ffma2_rn(two(j), make_float2(m, m), make_float2(s, s))); }, [&](int j) { v[j] = fmaf(v[j], m, s); });
    }
    __device__ __forceinline__ float sum() const {
        float2 s = make_float2(v[0], N > 1 ? v[N > 1] : 0.0f);
#pragma unroll
        for (int j = 2; j + 1 < N; j += 2) s = __fadd2_rn(s, two(j));
        return s.x + s.y;
    }
    __device__ __forceinline__ float dot(const Pairs &a) const {
        if constexpr (N == 1) return v[0] * a.v[0];
        float2 s = __fmul2_rn(two(0), a.two(0));
#pragma unroll
        for (int j = 2; j + 1 < N; j += 2) s = __ffma2_rn(two(j), a.two(j), s);
        return s.x + s.y;
    }
};

// A lane's share of a row: K vectors of V elements, `step` vectors apart.
template <typename T, int V, int K>
struct RowPart {
    hagr::Vec<T, V> raw[K];
    __device__ __forceinline__ void load(const void *base, int64_t ld, int64_t r, bool live, int first, int step, int32_t n_vec) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw[k].zero();
            if (live && first + k * step < n_vec) raw[k].template load<hagr::kOnce>(static_cast<const T *>(base) + r * ld, first + k * step);
        }
    }
    __device__ __forceinline__ Pairs<K * V> wide() const {
        Pairs<K * V> f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) f.v[k * V + j] = raw[k].get(j);
        return f;
    }
    static __device__ __forceinline__ void store(void *base, int64_t ld, int64_t r, bool live, int first, int step, int32_t n_vec,
                                                 const Pairs<K * V> &f) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!live || first + k * step >= n_vec) continue;
            hagr::Vec<T, V> o;
            o.set(&f.v[k * V]);
            o.store(static_cast<T *>(base) + r * ld, first + k * step);
        }
    }
    // differences from the mean; lanes beyond the row hold zeros
    __device__ __forceinline__ Pairs<K * V> centred(float mean, int first, int step, int32_t n_vec) const {
        Pairs<K * V> f = wide();
        f.shift(-mean);
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (first + k * step >= n_vec)
#pragma unroll
                for (int j = 0; j < V; ++j) f.v[k * V + j] = 0.0f;
        return f;
    }
};

template <typename T, int V, int L, int K, int R>
__global__ void __launch_bounds__(kWarpThreads) norm_fwd_warp_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int G = 32 / L;                                  // rows side by side in a warp
    const int lane = threadIdx.x & 31, gl = lane % L;
    const int32_t n_vec = p.D / V;
    const float cols = float(p.D);
    const int64_t group = (int64_t(blockIdx.x) * kWarpRows + (threadIdx.x >> 5)) * G + lane / L;
    const int64_t groups = int64_t(gridDim.x) * kWarpRows * G;
    Pairs<K * V> w, b;
    hagk::pdl_wait();
    load_params<V, K>(p.w, p.w_bf16, p.D, gl, L, 1.0f, w.v);
    load_params<V, K>(p.b, p.w_bf16, p.D, gl, L, 0.0f, b.v);
    RowPart<T, V, K> x[R], next[R];
    auto load = [&](RowPart<T, V, K> (&to)[R], int64_t r0) {
#pragma unroll
        for (int i = 0; i < R; ++i) to[i].load(p.x, p.ld_x, r0 + i, r0 + i < p.n, gl, L, n_vec);
    };
    // a warp's groups leave together: the row of its first group decides
    int64_t r0 = group * R;
    load(x, r0);
    for (; r0 - (lane / L) * R < p.n; r0 += groups * R) {
        load(next, r0 + groups * R);                           // in flight while these rows are worked on
        float s[R], mean[R];
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = x[i].wide().sum();
        const float my_mean = spread_sums<L, R>(s, gl) / cols;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            mean[i] = spread_get<L, R>(my_mean, i, lane);
            const Pairs<K * V> d = x[i].centred(mean[i], gl, L, n_vec);
            s[i] = d.dot(d);
        }
        const float my_rstd = rsqrtf(spread_sums<L, R>(s, gl) / cols + p.eps);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float rstd = spread_get<L, R>(my_rstd, i, lane);
            Pairs<K * V> v = x[i].wide(), y = b;
            v.shift_scale(-mean[i], rstd);
            y.fma(v, w);
            RowPart<T, V, K>::store(p.y, p.ld_y, r0 + i, r0 + i < p.n, gl, L, n_vec, y);
        }
        const int64_t r = r0 + gl * R / L;                     // the row whose statistics this lane holds
        if (gl % (L / R) == 0 && r < p.n) {
            if (p.mean) p.mean[r] = my_mean;
            if (p.rstd) p.rstd[r] = my_rstd;
        }
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = next[i];
    }
}

// Sum of two values over the block; `slot` alternates between calls, so one barrier is enough.
__device__ __forceinline__ float2 block_sum2(float a, float b, float2 *slot) {
    a = hagr::warp_sum(a);
    b = hagr::warp_sum(b);
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    float2 s = make_float2(0.0f, 0.0f);
    for (int w = 0; w < int(blockDim.x >> 5); ++w) {
        s.x += slot[w].x;
        s.y += slot[w].y;
    }
    return s;
}

template <typename T, int V, int MAX_THREADS>
__global__ void __launch_bounds__(MAX_THREADS) norm_fwd_block_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int K = kPerLane / V;
    __shared__ float2 slot[2][32];
    const int32_t n_vec = p.D / V, step = blockDim.x;
    const float cols = float(p.D);
    const int first = threadIdx.x;
    Pairs<K * V> w, b;
    hagk::pdl_wait();
    load_params<V, K>(p.w, p.w_bf16, p.D, first, step, 1.0f, w.v);
    load_params<V, K>(p.b, p.w_bf16, p.D, first, step, 0.0f, b.v);
    RowPart<T, V, K> x, next;
    x.load(p.x, p.ld_x, blockIdx.x, blockIdx.x < p.n, first, step, n_vec);
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x) {
        next.load(p.x, p.ld_x, r + gridDim.x, r + gridDim.x < p.n, first, step, n_vec);
        const float mean = block_sum2(x.wide().sum(), 0.0f, slot[0]).x / cols;
        const Pairs<K * V> d = x.centred(mean, first, step, n_vec);
        const float rstd = rsqrtf(block_sum2(d.dot(d), 0.0f, slot[1]).x / cols + p.eps);
        Pairs<K * V> v = x.wide(), y = b;
        v.shift_scale(-mean, rstd);
        y.fma(v, w);
        RowPart<T, V, K>::store(p.y, p.ld_y, r, true, first, step, n_vec, y);
        if (first == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
        x = next;
    }
}

// One row of the backward pass: its sums, what it adds to the parameters' gradients, and its gradient.
template <typename T, int V, int K>
struct BwdRow {
    RowPart<T, V, K> x, g;
    float mean, rstd;

    __device__ __forceinline__ void load(const NormArgs &p, int64_t r, int first, int step, int32_t n_vec) {
        const bool live = r < p.n;
        mean = live ? __ldcg(p.mean_in + r) : 0.0f;
        rstd = live ? __ldcg(p.rstd_in + r) : 0.0f;
        x.load(p.x, p.ld_x, r, live, first, step, n_vec);
        g.load(p.g, p.ld_g, r, live, first, step, n_vec);
    }
    // sum q and sum q * xh over this lane; where the lane is beyond the row g is zero and its terms vanish
    __device__ __forceinline__ void sums(const Pairs<K * V> &w, Pairs<K * V> &aw, Pairs<K * V> &ab, float &s1, float &s2) const {
        Pairs<K * V> xh = x.wide(), q = g.wide();
        xh.shift_scale(-mean, rstd);
        ab.add(q);
        aw.fma(q, xh);
        q.mul(w);
        s1 = q.sum();
        s2 = q.dot(xh);
    }
    __device__ __forceinline__ void store(const NormArgs &p, int64_t r, int first, int step, int32_t n_vec, const Pairs<K * V> &w,
                                          float s1, float s2) const {
        Pairs<K * V> xh = x.wide(), q = g.wide();
        xh.shift_scale(-mean, rstd);
        xh.affine(-s2, -s1);
        xh.fma(q, w);
        xh.mul_all(rstd);
        RowPart<T, V, K>::store(p.y, p.ld_y, r, r < p.n, first, step, n_vec, xh);
    }
};

template <typename T, int V, int L, int K, int R>
__global__ void __launch_bounds__(kWarpThreads) norm_bwd_warp_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int G = 32 / L;
    extern __shared__ float joined[];                          // [warps][2][L * K * V], only if gw or gb is wanted
    const int lane = threadIdx.x & 31, gl = lane % L, warp = threadIdx.x >> 5;
    const int32_t n_vec = p.D / V;
    const float cols = float(p.D);
    const int64_t group = (int64_t(blockIdx.x) * kWarpRows + warp) * G + lane / L;
    const int64_t groups = int64_t(gridDim.x) * kWarpRows * G;
    Pairs<K * V> w, aw, ab;
    aw.fill(0.0f);
    ab.fill(0.0f);
    hagk::pdl_wait();
    load_params<V, K>(p.w, p.w_bf16, p.D, gl, L, 1.0f, w.v);
    BwdRow<T, V, K> row[R], next[R];
    int64_t r0 = group * R;
#pragma unroll
    for (int i = 0; i < R; ++i) row[i].load(p, r0 + i, gl, L, n_vec);
    for (; r0 - (lane / L) * R < p.n; r0 += groups * R) {
        float s[2 * R];
#pragma unroll
        for (int i = 0; i < R; ++i) next[i].load(p, r0 + groups * R + i, gl, L, n_vec);
#pragma unroll
        for (int i = 0; i < R; ++i) row[i].sums(w, aw, ab, s[2 * i], s[2 * i + 1]);
        const float mine = spread_sums<L, 2 * R>(s, gl) / cols;
#pragma unroll
        for (int i = 0; i < R; ++i)
            row[i].store(p, r0 + i, gl, L, n_vec, w, spread_get<L, 2 * R>(mine, 2 * i, lane), spread_get<L, 2 * R>(mine, 2 * i + 1, lane));
#pragma unroll
        for (int i = 0; i < R; ++i) row[i] = next[i];
    }
    if (!p.partial) return;
    // groups of the warp, then warps of the block, in a fixed order
#pragma unroll
    for (int o = L; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < K * V; ++i) {
            aw.v[i] += __shfl_xor_sync(0xffffffffu, aw.v[i], o);
            ab.v[i] += __shfl_xor_sync(0xffffffffu, ab.v[i], o);
        }
    constexpr int C = L * K * V;
    if (lane < L)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                joined[(warp * 2 + 0) * C + (gl + k * L) * V + j] = aw.v[k * V + j];
                joined[(warp * 2 + 1) * C + (gl + k * L) * V + j] = ab.v[k * V + j];
            }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * C; c += kWarpThreads) {
        const int which = c / C, col = c - which * C;
        if (col >= p.D) continue;
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < kWarpRows; ++q) s += joined[q * 2 * C + c];
        p.partial[(int64_t(blockIdx.x) * 2 + which) * p.D + col] = s;
    }
}

template <typename T, int V, int MAX_THREADS>
__global__ void __launch_bounds__(MAX_THREADS) norm_bwd_block_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int K = kPerLane / V;
    __shared__ float2 slot[2][32];
    const int32_t n_vec = p.D / V, step = blockDim.x;
    const float cols = float(p.D);
    Pairs<K * V> w, aw, ab;
    aw.fill(0.0f);
    ab.fill(0.0f);
    hagk::pdl_wait();
    load_params<V, K>(p.w, p.w_bf16, p.D, threadIdx.x, step, 1.0f, w.v);
    int turn = 0;
    BwdRow<T, V, K> row, next;
    row.load(p, blockIdx.x, threadIdx.x, step, n_vec);
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x, turn ^= 1) {
        next.load(p, r + gridDim.x, threadIdx.x, step, n_vec);
        float s1, s2;
        row.sums(w, aw, ab, s1, s2);
        const float2 s = block_sum2(s1, s2, slot[turn]);
        row.store(p, r, threadIdx.x, step, n_vec, w, s.x / cols, s.y / cols);
        row = next;
    }
    if (!p.partial) return;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int32_t c = (int32_t(threadIdx.x) + k * step) * V + j;
            if (c >= p.D) continue;
            p.partial[int64_t(blockIdx.x) * 2 * p.D + c] = aw.v[k * V + j];
            p.partial[(int64_t(blockIdx.x) * 2 + 1) * p.D + c] = ab.v[k * V + j];
        }
}

// gw and gb from the parts: a block takes 32 columns of [gw | gb], its 32 warps every 32nd part each.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(32 * kJoinWarps) norm_params_join_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float sum[kJoinWarps][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane;
    hagk::pdl_wait();
    float s = 0.0f;
    if (c < 2 * int64_t(p.D)) {
#pragma unroll 8
        for (int q = warp; q < p.parts; q += kJoinWarps) s += __ldcg(p.partial + int64_t(q) * 2 * p.D + c);
    }
    sum[warp][lane] = s;
    __syncthreads();
    s = hagr::warp_sum(sum[lane][warp]);                       // column `warp` of this block
    const int64_t k = int64_t(blockIdx.x) * 32 + warp;
    if (lane == 0 && k < 2 * int64_t(p.D)) {
        void *to = k < p.D ? p.gw : p.gb;
        if (to) store_param(to, p.w_bf16, k < p.D ? k : k - p.D, s);
    }
}

constexpr int kParts = 64;                // of the kernels for rows of any width
constexpr int kSms = 148;
constexpr int kMaxParts = kSms * 8;       // of the register kernels: their blocks

cudaError_t launch(void (*kernel)(NormArgs), dim3 grid, unsigned threads, size_t shared, const NormArgs &p, cudaStream_t s) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

// How many blocks of the kernel the device runs at once (asked once per kernel and block size).
int resident_blocks(void (*kernel)(NormArgs), unsigned threads, size_t shared) {
    int per_sm = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, int(threads), shared) != cudaSuccess || per_sm < 1) {
        cudaGetLastError();
        per_sm = 1;
    }
    return std::min(per_sm * kSms, kMaxParts);
}

template <typename T, int V, int L, int K>
cudaError_t launch_warp(NormArgs &p, bool bwd, cudaStream_t s) {
    constexpr int RF = kPerLane / (K * V) < 4 ? kPerLane / (K * V) : 4, RB = K * V <= 8 ? 2 : 1;
    void (*const kernel)(NormArgs) = bwd ? norm_bwd_warp_kernel<T, V, L, K, RB> : norm_fwd_warp_kernel<T, V, L, K, RF>;
    const size_t shared = bwd && p.partial ? size_t(kWarpRows) * 2 * L * K * V * 4 : 0;
    static const int resident[2] = {resident_blocks(norm_fwd_warp_kernel<T, V, L, K, RF>, kWarpThreads, 0),
                                    resident_blocks(norm_bwd_warp_kernel<T, V, L, K, RB>, kWarpThreads, size_t(kWarpRows) * 2 * L * K * V * 4)};
    const int64_t rows_per_block = int64_t(kWarpRows) * (32 / L) * (bwd ? RB : RF);
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>((p.n + rows_per_block - 1) / rows_per_block, resident[bwd]));
    p.parts = int32_t(blocks);
    return launch(kernel, dim3(unsigned(blocks)), kWarpThreads, shared, p, s);
}

// MAX_THREADS 512 leaves a thread the 128 registers that the three per-column sets of the backward pass need; only
// rows that need more threads pay with spills.
template <typename T, int V, int MAX_THREADS>
cudaError_t launch_block(NormArgs &p, bool bwd, cudaStream_t s) {
    constexpr int K = kPerLane / V;
    void (*const kernel)(NormArgs) = bwd ? norm_bwd_block_kernel<T, V, MAX_THREADS> : norm_fwd_block_kernel<T, V, MAX_THREADS>;
    const unsigned threads = unsigned(((p.D / V + K - 1) / K + 31) / 32 * 32);
    static std::atomic<int> resident[2][MAX_THREADS / 32 + 1];
    int most = resident[bwd][threads / 32].load(std::memory_order_relaxed);
    if (most == 0) resident[bwd][threads / 32].store(most = resident_blocks(kernel, threads, 0), std::memory_order_relaxed);
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(p.n, most));
    p.parts = int32_t(blocks);
    return launch(kernel, dim3(unsigned(blocks)), threads, 0, p, s);
}

// Rows of up to 32 * kPerLane elements go to a warp or a part of one, rows of up to 1024 * kPerLane to a block.
template <typename T, int V>
cudaError_t launch_rows(NormArgs &p, bool bwd, cudaStream_t s) {
    const int32_t n_vec = p.D / V;
    if constexpr (V * int(sizeof(T)) == 16) {
        if (n_vec <= 8) return launch_warp<T, V, 8, 1>(p, bwd, s);
        if (n_vec <= 16) return launch_warp<T, V, 16, 1>(p, bwd, s);
    }
    if (n_vec <= 32) return launch_warp<T, V, 32, 1>(p, bwd, s);
    if (n_vec <= 64) return launch_warp<T, V, 32, 2>(p, bwd, s);
    if constexpr (V <= 4)
        if (n_vec <= 128) return launch_warp<T, V, 32, 4>(p, bwd, s);
    if constexpr (V <= 2)
        if (n_vec <= 256) return launch_warp<T, V, 32, 8>(p, bwd, s);
    if constexpr (V == 1)
        if (n_vec <= 512) return launch_warp<T, V, 32, 16>(p, bwd, s);
    if (p.D <= 512 * kPerLane) return launch_block<T, V, 512>(p, bwd, s);
    return launch_block<T, V, 1024>(p, bwd, s);
}

constexpr int32_t kMostInRegisters = 1024 * kPerLane;

template <typename T>
cudaError_t launch_typed(NormArgs &p, bool bwd, cudaStream_t s) {
    const int e = int(sizeof(T));
    const hagr::Operand ops[] = {{p.x, p.ld_x, e}, {p.y, p.ld_y, e}, {p.g, p.ld_g, e}};
    const int v = hagr::vector_elems(16 / e, p.D, ops);
    if (v == 16 / e) return launch_rows<T, 16 / e>(p, bwd, s);
    if constexpr (sizeof(T) == 2)
        if (v > 1) return launch_rows<T, 2>(p, bwd, s);
    return launch_rows<T, 1>(p, bwd, s);
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
    cudaError_t err;
    if (D <= kMostInRegisters)
        err = dtype == HAG_F32 ? launch_typed<float>(p, false, s) : launch_typed<__nv_bfloat16>(p, false, s);
    else
        err = launch(dtype == HAG_F32 ? norm_fwd_any_kernel<float> : norm_fwd_any_kernel<__nv_bfloat16>,
                     dim3(unsigned(std::min<int64_t>(n, kSms * 8))), kRowThreads, 0, p, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}

extern "C" size_t hag_layer_norm_bwd_workspace_bytes(int64_t n, int32_t D) {
    if (n < 0 || D <= 0) return 0;
    return size_t(D <= kMostInRegisters ? kMaxParts : kParts) * 2 * size_t(D) * 4;
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
    const dim3 join_grid(unsigned((2 * int64_t(D) + 31) / 32));
    if (!params) p.partial = nullptr;
    if (D <= kMostInRegisters) {
        if (n > 0 || params) err = f32 ? launch_typed<float>(p, true, s) : launch_typed<__nv_bfloat16>(p, true, s);
        if (params && err == cudaSuccess) err = launch(norm_params_join_kernel, join_grid, 32 * kJoinWarps, 0, p, s);
    } else {
        if (params) {      // first: grad_x may take the place of grad_y or x
            p.parts = int(std::min<int64_t>(std::max<int64_t>((n + kStripRows - 1) / kStripRows, 1), kParts));
            err = launch(f32 ? norm_params_any_kernel<float> : norm_params_any_kernel<__nv_bfloat16>,
                         dim3(unsigned((D + 31) / 32), unsigned(p.parts)), 32 * kStripRows, 0, p, s);
            if (err == cudaSuccess) err = launch(norm_params_join_kernel, join_grid, 32 * kJoinWarps, 0, p, s);
        }
        if (err == cudaSuccess && n > 0)
            err = launch(f32 ? norm_bwd_any_kernel<float> : norm_bwd_any_kernel<__nv_bfloat16>,
                         dim3(unsigned(std::min<int64_t>(n, kSms * 8))), kRowThreads, 0, p, s);
    }
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
