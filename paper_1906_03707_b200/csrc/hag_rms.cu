// Root-mean-square norm with the residual's addition, forward.
//   h = x + residual, rstd = 1 / sqrt(mean(h^2) + eps), y = h * rstd * w
// or, in 8 bits, q = round(y / scale) with scale = max|y| / top over a row or a block of its columns.
// h is added in fp32 and stays in registers between the sum of its squares and y, so a row is read once and y comes from
// the sum before it is rounded to the stream's type.  Rows of more columns than a block's registers hold are read two or
// three times, from the second time on out of the caches.
#include "hag_rms.cuh"

#include <cfloat>

namespace {

using namespace hagn;

struct RmsArgs {
    int64_t n;
    int32_t D;
    int32_t w_bf16, w_vectors;
    const void *x, *res, *w;
    int64_t ld_x, ld_res, ld_y, ld_total;
    void *y, *total;                    // y: or q
    float *rstd;
    float eps;
    float *scales;
    int32_t block, n_scales;            // columns per scale (0: all), scales per row
    int32_t int8;
    float top;
};

// 8-bit codes of V quotients.
template <int V>
__device__ __forceinline__ hagr::Words<V> pack(const float (&v)[V], bool int8) {
    hagr::Words<V> r;
    static_assert(V % 4 == 0, "");
#pragma unroll
    for (int j = 0; j < V; j += 4) {
        if (int8) {
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) w |= uint32_t(uint8_t(int8_t(__float2int_rn(v[j + i])))) << (8 * i);
            r.w[j / 4] = w;
        } else {
            uint16_t a, b;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(a) : "f"(v[j + 1]), "f"(v[j]));
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(v[j + 3]), "f"(v[j + 2]));
            r.w[j / 4] = uint32_t(a) | uint32_t(b) << 16;
        }
    }
    return r;
}
__device__ __forceinline__ uint8_t pack_one(float v, bool int8) {
    if (int8) return uint8_t(int8_t(__float2int_rn(v)));
    uint16_t a;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(a) : "f"(0.0f), "f"(v));
    return uint8_t(a);
}
template <int V>
__device__ __forceinline__ void store_codes(const float (&v)[V], void *row, int64_t i, bool int8) {
    if constexpr (V == 1) static_cast<uint8_t *>(row)[i] = pack_one(v[0], int8);
    else hagr::store_words<hagr::kKeep, V>(static_cast<char *>(row) + i * V, pack<V>(v, int8));
}

// The largest of magnitudes; NaN is larger than anything (the bits of positive floats are ordered as the floats are).
template <int L>
__device__ __forceinline__ float lanes_largest(float v) {
    uint32_t b = __float_as_uint(v);
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, o));
    return __uint_as_float(b);
}
__device__ __forceinline__ float larger(float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }
template <int L>
__device__ __forceinline__ float group_largest(float v, float *slot) {
    v = lanes_largest<L ? L : 32>(v);
    if constexpr (L == 0) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = lanes_largest<32>((threadIdx.x & 31) < (blockDim.x >> 5) ? slot[threadIdx.x & 31] : 0.0f);
    }
    return v;
}
// the same over the first `lanes` (a power of two) only
__device__ __forceinline__ float some_largest(float v, int lanes) {
    uint32_t b = __float_as_uint(v);
    for (int o = lanes / 2; o > 0; o >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, o));
    return __uint_as_float(b);
}
// top is 448 or 127; a largest value that is not finite gives a scale that is none
__device__ __forceinline__ float scale_of(float largest, const RmsArgs &p) {
    const float s = largest * (1.0f / p.top);
    return s < FLT_MIN ? FLT_MIN : s;
}

template <typename X, typename S, int V>
__device__ __forceinline__ void add_rows(float (&h)[V], const Wide<X, V> &x, const Wide<S, V> &r, bool res) {
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = res ? x.v.get(j) + r.v.get(j) : x.v.get(j);
}

// Scales and codes of K vectors of a thread, which lie kStep = 32 apart (or are a row's all, of fewer lanes): `y` are the
// values, first their number in the row.  A scale's columns lie within a warp: they are block / V lanes of one vector, or,
// for V = 1, block / 32 vectors of all lanes.
template <int V, int K, int STEP>
__device__ __forceinline__ void quant_blocks(float (&y)[K][V], const RmsArgs &p, int64_t r, int first, int n_vec, bool live) {
    char *q = static_cast<char *>(p.y) + r * p.ld_y;
    const int lanes = V == 1 ? 32 : p.block / V, together = V == 1 ? p.block / 32 : 1;
    float top[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        top[k] = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) top[k] = larger(top[k], fabsf(y[k][j]));
        top[k] = some_largest(top[k], lanes);
    }
    if constexpr (V == 1 && K > 1) {
#pragma unroll
        for (int k = 0; k < K; k += 2)
            if (together > 1) top[k] = top[k + 1] = larger(top[k], top[k + 1]);
        if constexpr (K % 4 == 0) {
#pragma unroll
            for (int k = 0; k < K; k += 4)
                if (together > 2) top[k] = top[k + 1] = top[k + 2] = top[k + 3] = larger(top[k], top[k + 2]);
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int vec = first + k * STEP;
        const float scale = scale_of(top[k], p), inverse = __fdividef(1.0f, scale);
        float t[V];
#pragma unroll
        for (int j = 0; j < V; ++j) t[j] = y[k][j] * inverse;
        if (!live || vec >= n_vec) continue;
        store_codes<V>(t, q, vec, p.int8);
        const int c = vec * V;
        if (c % p.block == 0) p.scales[r * p.n_scales + c / p.block] = scale;
    }
}

template <int PER_LANE> constexpr int kTurnRows = PER_LANE >= 32 ? 1 : 32 / PER_LANE < 4 ? 32 / PER_LANE : 4;

template <typename X, typename S, typename Y, int V, int L, int K, bool QUANT>
__global__ void __launch_bounds__(L ? kWarpRowThreads : kRowThreads, L ? 2 : 1) rms_fwd_kernel(const __grid_constant__ RmsArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int R = L ? kTurnRows<V * K> : 1;
    using P = Place<L, K>;
    __shared__ float slots[4][32];
    const P at;
    const int n_vec = p.D / V;
    const float inverse = 1.0f / float(p.D);
    const bool res = p.res != nullptr;
    bool mine[K];
    float w[K][V];
    hagk::pdl_wait();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        mine[k] = at.first + k * P::kStep < n_vec;
        if (mine[k]) load_weights<V>(w[k], p.w, p.w_bf16, p.w_vectors, int64_t(at.first + k * P::kStep) * V);
    }
    int turn = 0;
    for (int64_t lead = at.leader() * R, r0 = at.group * R; lead < p.n; lead += at.groups * R, r0 += at.groups * R, turn ^= 1) {
        float h[R][K][V], s[R];
        {
            Wide<X, V> x[R][K];
            Wide<S, V> q[R][K];
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    x[i][k].v.zero();
                    q[i][k].v.zero();
                    if (mine[k] && r0 + i < p.n) {
                        x[i][k].load(static_cast<const X *>(p.x) + (r0 + i) * p.ld_x, at.first + k * P::kStep);
                        if (res) q[i][k].load(static_cast<const S *>(p.res) + (r0 + i) * p.ld_res, at.first + k * P::kStep);
                    }
                }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                s[i] = 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    add_rows<X, S, V>(h[i][k], x[i][k], q[i][k], res);
                    float t = 0.0f;
#pragma unroll
                    for (int j = 0; j < V; ++j) t = fmaf(h[i][k][j], h[i][k][j], t);
                    s[i] += t;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t r = r0 + i;
            const bool live = r < p.n;
            const float rstd = rsqrtf(group_sum<L>(s[i], slots[turn]) * inverse + p.eps);
            if (p.rstd && live && at.first == 0) p.rstd[r] = rstd;
            if (p.total && live) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    Wide<S, V> o;
                    o.v.set(h[i][k]);
                    if (mine[k]) o.store(static_cast<S *>(p.total) + r * p.ld_total, at.first + k * P::kStep);
                }
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) h[i][k][j] = mine[k] ? h[i][k][j] * rstd * w[k][j] : 0.0f;
            if constexpr (!QUANT) {
                if (live) {
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        Wide<Y, V> o;
                        o.v.set(h[i][k]);
                        if (mine[k]) o.store(static_cast<Y *>(p.y) + r * p.ld_y, at.first + k * P::kStep);
                    }
                }
            } else if (p.block) {
                quant_blocks<V, K, P::kStep>(h[i], p, r, at.first, n_vec, live);
            } else {
                float top = 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int j = 0; j < V; ++j) top = larger(top, fabsf(h[i][k][j]));
                const float scale = scale_of(group_largest<L>(top, slots[2 + turn]), p), inv = __fdividef(1.0f, scale);
                if (!live) continue;
                if (at.first == 0) p.scales[r] = scale;
#pragma unroll
                for (int k = 0; k < K; ++k) {
#pragma unroll
                    for (int j = 0; j < V; ++j) h[i][k][j] *= inv;
                    if (mine[k]) store_codes<V>(h[i][k], static_cast<char *>(p.y) + r * p.ld_y, at.first + k * P::kStep, p.int8);
                }
            }
        }
    }
}

// Rows of more columns: a block walks its row, a warp 32 K vectors at a time, once for the squares, once more for the
// largest value where a row has one scale, and once for the results.
template <typename X, typename S, typename Y, int V, bool QUANT>
__global__ void __launch_bounds__(kRowThreads, 1) rms_fwd_long_kernel(const __grid_constant__ RmsArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int K = 4;
    __shared__ float slots[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n_vec = p.D / V, stride = (kRowThreads / 32) * 32 * K;
    const bool res = p.res != nullptr;
    hagk::pdl_wait();
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x) {
        const X *xr = static_cast<const X *>(p.x) + r * p.ld_x;
        const S *qr = static_cast<const S *>(p.res) + (res ? r * p.ld_res : 0);
        auto rows = [&](int base, float (&h)[K][V]) {                  // the sums of 32 K vectors from `base` on
            Wide<X, V> x[K];
            Wide<S, V> q[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                x[k].v.zero();
                q[k].v.zero();
                if (base + k * 32 + lane < n_vec) {
                    x[k].load(xr, base + k * 32 + lane);
                    if (res) q[k].load(qr, base + k * 32 + lane);
                }
            }
#pragma unroll
            for (int k = 0; k < K; ++k) add_rows<X, S, V>(h[k], x[k], q[k], res);
        };
        auto scaled = [&](int base, float rstd, float (&h)[K][V]) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float w[V];
                const int vec = base + k * 32 + lane;
                if (vec < n_vec) load_weights<V>(w, p.w, p.w_bf16, p.w_vectors, int64_t(vec) * V);
#pragma unroll
                for (int j = 0; j < V; ++j) h[k][j] = vec < n_vec ? h[k][j] * rstd * w[j] : 0.0f;
            }
        };
        float s = 0.0f, h[K][V];
        for (int base = warp * 32 * K; base < n_vec; base += stride) {
            rows(base, h);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float t = 0.0f;
#pragma unroll
                for (int j = 0; j < V; ++j) t = fmaf(h[k][j], h[k][j], t);
                s += t;
            }
        }
        const float rstd = rsqrtf(group_sum<0>(s, slots[0]) / float(p.D) + p.eps);
        if (p.rstd && threadIdx.x == 0) p.rstd[r] = rstd;
        float inv = 0.0f;
        if constexpr (QUANT) {
            if (!p.block) {
                float top = 0.0f;
                for (int base = warp * 32 * K; base < n_vec; base += stride) {
                    rows(base, h);
                    scaled(base, rstd, h);
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int j = 0; j < V; ++j) top = larger(top, fabsf(h[k][j]));
                }
                const float scale = scale_of(group_largest<0>(top, slots[1]), p);
                if (threadIdx.x == 0) p.scales[r] = scale;
                inv = __fdividef(1.0f, scale);
            }
        }
        for (int base = warp * 32 * K; base < n_vec; base += stride) {
            rows(base, h);
            if (p.total) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    Wide<S, V> o;
                    o.v.set(h[k]);
                    if (base + k * 32 + lane < n_vec) o.store(static_cast<S *>(p.total) + r * p.ld_total, base + k * 32 + lane);
                }
            }
            scaled(base, rstd, h);
            if constexpr (!QUANT) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    Wide<Y, V> o;
                    o.v.set(h[k]);
                    if (base + k * 32 + lane < n_vec) o.store(static_cast<Y *>(p.y) + r * p.ld_y, base + k * 32 + lane);
                }
            } else if (p.block) {
                quant_blocks<V, K, 32>(h, p, r, base + lane, n_vec, true);
            } else {
#pragma unroll
                for (int k = 0; k < K; ++k) {
#pragma unroll
                    for (int j = 0; j < V; ++j) h[k][j] *= inv;
                    if (base + k * 32 + lane < n_vec) store_codes<V>(h[k], static_cast<char *>(p.y) + r * p.ld_y, base + k * 32 + lane, p.int8);
                }
            }
        }
        __syncthreads();                                               // the slots are written again
    }
}

template <typename X, typename S, typename Y, int V, int L, int K, bool QUANT>
cudaError_t launch_rows(const RmsArgs &p, cudaStream_t s) {
    constexpr auto kernel = rms_fwd_kernel<X, S, Y, V, L, K, QUANT>;
    constexpr int R = L ? kTurnRows<V * K> : 1;
    const unsigned threads = L ? kWarpRowThreads : unsigned((p.D / V + 32 * K - 1) / (32 * K)) * 32;
    const int64_t rows = L ? int64_t(kWarpRowThreads / 32) * (32 / (L ? L : 32)) * R : 1;
    const int64_t grid = std::min<int64_t>((p.n + rows - 1) / rows, int64_t(kSms) * blocks_per_sm<kernel>(threads, 0));
    return launch(kernel, dim3(unsigned(grid)), threads, 0, p, s);
}

// Rows of up to 32 columns per lane go to a warp or a part of one, wider ones to a block.
template <typename X, typename S, typename Y, int V, bool QUANT>
cudaError_t launch_width(const RmsArgs &p, cudaStream_t s) {
    const int32_t n_vec = p.D / V;
    if (p.D > kMostInRegisters) {
        constexpr auto kernel = rms_fwd_long_kernel<X, S, Y, V, QUANT>;
        return launch(kernel, dim3(unsigned(std::min<int64_t>(p.n, int64_t(kSms) * blocks_per_sm<kernel>(kRowThreads, 0)))), kRowThreads, 0, p, s);
    }
    if (n_vec <= 4) return launch_rows<X, S, Y, V, 4, 1, QUANT>(p, s);
    if (n_vec <= 8) return launch_rows<X, S, Y, V, 8, 1, QUANT>(p, s);
    if (n_vec <= 16) return launch_rows<X, S, Y, V, 16, 1, QUANT>(p, s);
    if (n_vec <= 32) return launch_rows<X, S, Y, V, 32, 1, QUANT>(p, s);
    if (n_vec <= 64) return launch_rows<X, S, Y, V, 32, 2, QUANT>(p, s);
    if (n_vec <= 128) return launch_rows<X, S, Y, V, 32, 4, QUANT>(p, s);
    if constexpr (V == 1) {
        if (n_vec <= 256) return launch_rows<X, S, Y, V, 32, 8, QUANT>(p, s);
        if (n_vec <= 512) return launch_rows<X, S, Y, V, 32, 16, QUANT>(p, s);
    }
    return launch_rows<X, S, Y, V, 0, kPerThread / V, QUANT>(p, s);
}

template <typename X, typename S, typename Y, bool QUANT, int N>
cudaError_t launch_typed(RmsArgs &p, const Matrix (&m)[N], cudaStream_t s) {
    constexpr int kMost = sizeof(X) == 2 || sizeof(Y) == 2 ? 8 : 4;       // the narrowest type fills 16 bytes
    const int we = p.w_bf16 ? 2 : 4;
    if (vectors_fit(kMost, p.D, m)) {
        p.w_vectors = on(p.w, std::min(16, kMost * we));
        return launch_width<X, S, Y, kMost, QUANT>(p, s);
    }
    if constexpr (kMost == 8)
        if (vectors_fit(4, p.D, m)) {
            p.w_vectors = on(p.w, 4 * we);
            return launch_width<X, S, Y, 4, QUANT>(p, s);
        }
    p.w_vectors = 0;
    return launch_width<X, S, Y, 1, QUANT>(p, s);
}

bool types_ok(hag_dtype x, hag_dtype stream, hag_dtype y, bool res) {
    if (!dtype_ok(x) || !dtype_ok(stream) || !dtype_ok(y)) return false;
    if (x != stream) return res && x == HAG_BF16 && y == HAG_BF16;       // bf16 around an fp32 stream
    return y == stream || stream == HAG_F32;
}

}  // namespace

extern "C" hag_status hag_rms_norm_fwd(int64_t n, int32_t D, const void *x, hag_dtype x_dtype, int64_t ld_x, const void *residual,
                                       hag_dtype stream_dtype, int64_t ld_residual, const void *weight, hag_dtype weight_dtype,
                                       float eps, void *y, hag_dtype y_dtype, int64_t ld_y, void *total, int64_t ld_total,
                                       float *rstd, void *cuda_stream) {
    if (!types_ok(x_dtype, stream_dtype, y_dtype, residual != nullptr) || !dtype_ok(weight_dtype)) return HAG_ERR_DTYPE;
    const Matrix m[] = {{x, ld_x, size_of(x_dtype), false, true}, {residual, ld_residual, size_of(stream_dtype), false, false},
                        {y, ld_y, size_of(y_dtype), true, true}, {total, ld_total, size_of(stream_dtype), true, false}};
    const hag_status st = check(n, D, weight, weight_dtype, rstd, m);
    if (st != HAG_OK) return st;
    if (!(eps >= 0.0f)) return HAG_ERR_ARG;
    if (n == 0) return HAG_OK;
    RmsArgs p{};
    p.n = n; p.D = D; p.w_bf16 = weight_dtype == HAG_BF16; p.w = weight; p.eps = eps;
    p.x = x; p.ld_x = ld_x; p.res = residual; p.ld_res = ld_residual; p.y = y; p.ld_y = ld_y; p.total = total; p.ld_total = ld_total;
    p.rstd = rstd;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err;
    if (x_dtype != stream_dtype) err = launch_typed<__nv_bfloat16, float, __nv_bfloat16, false>(p, m, s);
    else if (x_dtype == HAG_BF16) err = launch_typed<__nv_bfloat16, __nv_bfloat16, __nv_bfloat16, false>(p, m, s);
    else if (y_dtype == HAG_BF16) err = launch_typed<float, float, __nv_bfloat16, false>(p, m, s);
    else err = launch_typed<float, float, float, false>(p, m, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}

extern "C" hag_status hag_rms_norm_quant_fwd(int64_t n, int32_t D, const void *x, hag_dtype x_dtype, int64_t ld_x,
                                             const void *residual, hag_dtype stream_dtype, int64_t ld_residual, const void *weight,
                                             hag_dtype weight_dtype, float eps, hag_quant kind, int32_t block, void *q, int64_t ld_q,
                                             float *scales, void *total, int64_t ld_total, float *rstd, void *cuda_stream) {
    if (!types_ok(x_dtype, stream_dtype, x_dtype, residual != nullptr) || !dtype_ok(weight_dtype)) return HAG_ERR_DTYPE;
    if (kind != HAG_E4M3 && kind != HAG_I8) return HAG_ERR_DTYPE;
    if (block != 0 && block != 32 && block != 64 && block != 128) return HAG_ERR_ARG;
    const Matrix m[] = {{x, ld_x, size_of(x_dtype), false, true}, {residual, ld_residual, size_of(stream_dtype), false, false},
                        {q, ld_q, 1, true, true}, {total, ld_total, size_of(stream_dtype), true, false}};
    const hag_status st = check(n, D, weight, weight_dtype, rstd, m);
    if (st != HAG_OK) return st;
    if (!(eps >= 0.0f)) return HAG_ERR_ARG;
    if (n == 0) return HAG_OK;
    if (!scales) return HAG_ERR_NULL;
    if (!on(scales, 4)) return HAG_ERR_ALIGN;
    RmsArgs p{};
    p.n = n; p.D = D; p.w_bf16 = weight_dtype == HAG_BF16; p.w = weight; p.eps = eps;
    p.x = x; p.ld_x = ld_x; p.res = residual; p.ld_res = ld_residual; p.y = q; p.ld_y = ld_q; p.total = total; p.ld_total = ld_total;
    p.rstd = rstd;
    p.scales = scales;
    p.block = block >= D ? 0 : block;
    p.n_scales = p.block ? (D + block - 1) / block : 1;
    p.int8 = kind == HAG_I8;
    p.top = kind == HAG_I8 ? 127.0f : 448.0f;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err;
    if (x_dtype != stream_dtype) err = launch_typed<__nv_bfloat16, float, uint8_t, true>(p, m, s);
    else if (x_dtype == HAG_BF16) err = launch_typed<__nv_bfloat16, __nv_bfloat16, uint8_t, true>(p, m, s);
    else err = launch_typed<float, float, uint8_t, true>(p, m, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
