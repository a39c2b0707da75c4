// Root-mean-square norm with the residual's addition, forward.
//   h = x + residual, rstd = 1 / sqrt(mean(h^2) + eps), y = h * rstd * w
// or, in 8 bits, q = round(y / scale) with scale = max|y| / top over a row or a block of its columns.  The quotient is that of an
// fp32 division: the product with a reciprocal alone is off by a place or two, and moves one code in 10^5 to its neighbour.
// h is added in fp32 and stays in registers between the sum of its squares and y, so a row is read once and y comes from
// the sum before it is rounded to the stream's type.  Rows of more than 16 384 columns are read two or three times, from the
// second time on out of the caches.
//
// Bound by memory.  Measured on B200 against a copy at 6.53 TB/s: 10^6 x 256 bf16 319 us (6.4 TB/s), around an fp32 stream 472
// (6.5), into e4m3 with a scale per row 285 (6.3); 233 000 x 128 fp32 75.5 us (6.3); 30 000 x 4096 bf16 149 us (6.6); 10 000 x
// 12 000 bf16 150 us (6.4).  Into 8 bits the instructions come near, 59 % of the issue slots (30 000 x 4096 bf16 with a scale
// per 128 columns 149 us, 5.8 TB/s; into int8, whose codes are converted one by one, 162).  Rows that do not begin on 16
// bytes are read and written one element at a time: 300 000 x 333 fp32 275 us (5.8 TB/s), bf16 171 (4.7), 50 000 x 1433 bf16
// into e4m3 173 (2.9: a byte per store).
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
    int32_t stages;                     // of the ring
    float inverse_top;                  // 1 / the type's largest value
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

// The larger magnitude; NaN is larger than anything.
__device__ __forceinline__ float larger(float top, float v) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(top), "f"(fabsf(v)));
    return r;
}
// The largest over the first `lanes` (a power of two) lanes of each such group: the bits of positive floats are ordered as
// the floats are, and NaN is above them.
__device__ __forceinline__ float lanes_largest(float v, int lanes) {
    uint32_t b = __float_as_uint(v);
    if (lanes == 32) return __uint_as_float(__reduce_max_sync(0xffffffffu, b));
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
        if (lanes > o) b = max(b, __shfl_xor_sync(0xffffffffu, b, o));
    return __uint_as_float(b);
}
template <int L>
__device__ __forceinline__ float group_largest(float v, float *slot) {
    v = lanes_largest(v, L > 0 ? L : 32);
    if constexpr (L <= 0) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = lanes_largest((threadIdx.x & 31) < (blockDim.x >> 5) ? slot[threadIdx.x & 31] : 0.0f, 32);
    }
    return v;
}
// the largest value's product with 1 / 448 or 1 / 127; one that is not finite gives a scale that is none
__device__ __forceinline__ float scale_of(float largest, const RmsArgs &p) {
    const float s = largest * p.inverse_top;
    return s < FLT_MIN ? FLT_MIN : s;
}

// Scales and codes of K vectors of a thread: `y` are the values.  A scale's columns lie within a warp: they are block / V
// lanes of one vector, or, for V = 1, T = block / 32 vectors of all lanes.
template <int T, int V, int K, typename At>
__device__ __forceinline__ void quant_groups(hagr::Pairs<V> (&y)[K], const RmsArgs &p, int64_t r, const At &at, int n_vec, bool live, int lanes) {
    char *q = static_cast<char *>(p.y) + r * p.ld_y;
#pragma unroll
    for (int k0 = 0; k0 < K; k0 += T) {
        float top = 0.0f;
#pragma unroll
        for (int k = k0; k < k0 + T && k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) top = larger(top, y[k].v[j]);
        const float scale = scale_of(lanes_largest(top, lanes), p), inverse = __fdividef(1.0f, scale);
        if (!live) continue;
#pragma unroll
        for (int k = k0; k < k0 + T && k < K; ++k) {
            y[k].divide(scale, inverse);
            if (at.mine(k, n_vec)) store_codes<V>(y[k].v, q, at.vec(k), p.int8);
        }
        const int c = at.vec(k0) * V;
        if (c % p.block == 0 && at.mine(k0, n_vec)) p.scales[r * p.n_scales + c / p.block] = scale;
    }
}
template <int V, int K, typename At>
__device__ __forceinline__ void quant_blocks(hagr::Pairs<V> (&y)[K], const RmsArgs &p, int64_t r, const At &at, int n_vec, bool live) {
    if constexpr (V > 1) {
        quant_groups<1, V, K>(y, p, r, at, n_vec, live, p.block / V);
    } else {
        if (p.block == 128) quant_groups<4, V, K>(y, p, r, at, n_vec, live, 32);
        else if (p.block == 64) quant_groups<2, V, K>(y, p, r, at, n_vec, live, 32);
        else quant_groups<1, V, K>(y, p, r, at, n_vec, live, 32);
    }
}

// Rows whose vectors fill 16 bytes are copied into a ring in shared memory some turns ahead, so that what is in flight does
// not take registers; others are read when their turn comes, all of them before the first is used.
template <typename X, typename S, int V> constexpr bool kRing = V * int(sizeof(X) < sizeof(S) ? sizeof(X) : sizeof(S)) >= 16;
// Rows per turn: 32 bytes per lane of the ring, or 16 columns.
constexpr int kTurnBytes = 32;
template <typename X, typename S, int V, int K, bool RES> constexpr int kRowBytes = K * V * int(sizeof(X) + (RES ? sizeof(S) : 0));     // per lane
template <typename X, typename S, int V, int L, int K, bool RES> constexpr int kTurnRows =
    L <= 0 ? 1 : kRing<X, S, V> ? (kRowBytes<X, S, V, K, RES> >= kTurnBytes ? 1 : kTurnBytes / kRowBytes<X, S, V, K, RES>)
                                : V * K >= 16 ? 1 : 16 / (V * K) < 4 ? 16 / (V * K) : 4;

template <typename X, typename S, typename Y, int V, int L, int K, bool QUANT, bool RES>
__global__ void __launch_bounds__(kThreadsOf<L>, L > 0 ? 2 : 1) rms_fwd_kernel(const __grid_constant__ RmsArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int R = kTurnRows<X, S, V, L, K, RES>;
    constexpr bool RING = kRing<X, S, V>;
    using P = Place<L, K, QUANT && V == 1>;
    using CX = ChunkCopy<X, V, P, K>;
    using CS = ChunkCopy<S, V, P, K>;
    extern __shared__ __align__(16) char raw[];
    __shared__ float slots[4][32];
    const P at;
    const int n_vec = p.D / V;
    const float inverse = 1.0f / float(p.D);
    const int64_t ld_x = p.ld_x * int64_t(sizeof(X)), ld_res = p.ld_res * int64_t(sizeof(S));
    const int row_bytes = CX::bytes() + (RES ? CS::bytes() : 0), stage = R * row_bytes, end = p.stages * stage;
    int64_t next = at.group * R;
    int write = 0, read = 0;
    auto issue = [&]() {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t r = next + i;
            char *const to = raw + write + i * row_bytes;
            CX::issue(to, static_cast<const char *>(p.x) + r * ld_x, at, n_vec, r < p.n);
            if (RES) CS::issue(to + CX::bytes(), static_cast<const char *>(p.res) + r * ld_res, at, n_vec, r < p.n);
        }
        hagr::commit_copies();
        next += at.groups * R;
        write = write + stage == end ? 0 : write + stage;
    };
    hagk::pdl_wait();
    if constexpr (RING) {
        for (int s = 0; s < p.stages; ++s) issue();
    }
    hagr::Pairs<V> w[kKeepWeights<L> ? K : 1];
    if constexpr (kKeepWeights<L>) load_all_weights<V, K>(w, p.w, p.w_bf16, p.w_vectors, at, n_vec);
    int turn = 0;
    for (int64_t lead = at.leader() * R, r0 = at.group * R; lead < p.n; lead += at.groups * R, r0 += at.groups * R, turn ^= 1) {
        hagr::Pairs<V> h[R][K];
        float s[R];
        if constexpr (RING) {
            hagr::wait_oldest(p.stages);
            if (CX::kCrosses || (RES && CS::kCrosses)) __syncwarp();
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const char *from = raw + read + i * row_bytes;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    h[i][k] = CX::get(from, at, k);
                    if (RES) h[i][k].add(CS::get(from + CX::bytes(), at, k));
                }
            }
            if (CX::kCrosses || (RES && CS::kCrosses)) __syncwarp();
            issue();
            read = read + stage == end ? 0 : read + stage;
        } else {
            hagr::Vec<X, V> x[R][K];
            hagr::Vec<S, V> q[R][K];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const bool live = r0 + i < p.n;
                const char *xr = static_cast<const char *>(p.x) + (r0 + i) * ld_x, *qr = static_cast<const char *>(p.res) + (r0 + i) * ld_res;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    x[i][k].zero();
                    if (live && at.mine(k, n_vec)) x[i][k].template load<hagr::kKeep>(xr, at.vec(k));
                }
                if (RES) {
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        q[i][k].zero();
                        if (live && at.mine(k, n_vec)) q[i][k].template load<hagr::kKeep>(qr, at.vec(k));
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    h[i][k] = hagr::widen(x[i][k]);
                    if (RES) h[i][k].add(hagr::widen(q[i][k]));
                }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[i] = 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) s[i] += h[i][k].dot(h[i][k]);
        }
        const Sums<L, R> rstds(s, slots[turn], [&](float q) { return rsqrtf(q * inverse + p.eps); });
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t r = r0 + i;
            const bool live = r < p.n;
            const float rstd = rstds.get(i);
            if (p.rstd && live && at.first()) p.rstd[r] = rstd;
            if (p.total && live) {
                char *const to = static_cast<char *>(p.total) + r * p.ld_total * int64_t(sizeof(S));
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    Wide<S, V> o;
                    o.v.set(h[i][k].v);
                    if (at.mine(k, n_vec)) o.store(to, at.vec(k));
                }
            }
#pragma unroll
            for (int k = 0; k < K; ++k) h[i][k].mul_all(rstd);
            if constexpr (kKeepWeights<L>) {
#pragma unroll
                for (int k = 0; k < K; ++k) h[i][k].mul(w[k]);
            } else {
                constexpr int U = V > 1 ? 1 : K % 4 == 0 ? 4 : 2;
                static_assert(K % U == 0, "");
#pragma unroll
                for (int k = 0; k < K; k += U) {
                    hagr::Pairs<V> some[U];
                    load_all_weights<V, U>(some, p.w, p.w_bf16, p.w_vectors, From<P>{at, k}, n_vec);
#pragma unroll
                    for (int u = 0; u < U; ++u) h[i][k + u].mul(some[u]);
                }
            }
            char *const to = static_cast<char *>(p.y) + r * p.ld_y * int64_t(sizeof(Y));
            if constexpr (!QUANT) {
                if (live) {
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        Wide<Y, V> o;
                        o.v.set(h[i][k].v);
                        if (at.mine(k, n_vec)) o.store(to, at.vec(k));
                    }
                }
            } else if (p.block) {
                quant_blocks<V, K>(h[i], p, r, at, n_vec, live);
            } else {
                float top = 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int j = 0; j < V; ++j) top = larger(top, h[i][k].v[j]);
                const float scale = scale_of(group_largest<L>(top, slots[2 + turn]), p), inv = __fdividef(1.0f, scale);
                if (!live) continue;
                if (at.first()) p.scales[r] = scale;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    h[i][k].divide(scale, inv);
                    if (at.mine(k, n_vec)) store_codes<V>(h[i][k].v, to, at.vec(k), p.int8);
                }
            }
        }
    }
    if constexpr (RING) hagr::wait_copies<0>();
}

// Rows of more columns: a block walks its row, a warp 32 K vectors at a time, once for the squares, once more for the
// largest value where a row has one scale, and once for the results.
template <typename X, typename S, typename Y, int V, bool QUANT>
__global__ void __launch_bounds__(kRowThreads, 1) rms_fwd_long_kernel(const __grid_constant__ RmsArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int K = V == 8 ? 2 : 4;
    __shared__ float slots[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n_vec = p.D / V, stride = (kRowThreads / 32) * 32 * K;
    const bool res = p.res != nullptr;
    struct Walk {                                                      // K chunks side by side
        int base;
        __device__ __forceinline__ int vec(int k) const { return base + k * 32; }
        __device__ __forceinline__ bool mine(int k, int n) const { return base + k * 32 < n; }
    };
    hagk::pdl_wait();
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x) {
        const X *xr = static_cast<const X *>(p.x) + r * p.ld_x;
        const S *qr = static_cast<const S *>(p.res) + (res ? r * p.ld_res : 0);
        auto rows = [&](const Walk &at, hagr::Pairs<V> (&h)[K]) {      // the sums of K vectors
            Wide<X, V> x[K];
            Wide<S, V> q[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                x[k].v.zero();
                q[k].v.zero();
                if (at.mine(k, n_vec)) {
                    x[k].load(xr, at.vec(k));
                    if (res) q[k].load(qr, at.vec(k));
                }
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                h[k] = hagr::widen(x[k].v);
                if (res) h[k].add(hagr::widen(q[k].v));
            }
        };
        auto scaled = [&](const Walk &at, float rstd, hagr::Pairs<V> (&h)[K]) {
            hagr::Pairs<V> w[K];
            load_all_weights<V, K>(w, p.w, p.w_bf16, p.w_vectors, at, n_vec);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                h[k].mul_all(rstd);
                h[k].mul(w[k]);
            }
        };
        float s = 0.0f;
        hagr::Pairs<V> h[K];
        for (Walk at{warp * 32 * K + lane}; at.base - lane < n_vec; at.base += stride) {
            rows(at, h);
#pragma unroll
            for (int k = 0; k < K; ++k) s += h[k].dot(h[k]);
        }
        const float rstd = rsqrtf(group_sum<0>(s, slots[0]) / float(p.D) + p.eps);
        if (p.rstd && threadIdx.x == 0) p.rstd[r] = rstd;
        float scale = 0.0f, inv = 0.0f;
        if constexpr (QUANT) {
            if (!p.block) {
                float top = 0.0f;
                for (Walk at{warp * 32 * K + lane}; at.base - lane < n_vec; at.base += stride) {
                    rows(at, h);
                    scaled(at, rstd, h);
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int j = 0; j < V; ++j) top = larger(top, h[k].v[j]);
                }
                scale = scale_of(group_largest<0>(top, slots[1]), p);
                if (threadIdx.x == 0) p.scales[r] = scale;
                inv = __fdividef(1.0f, scale);
            }
        }
        for (Walk at{warp * 32 * K + lane}; at.base - lane < n_vec; at.base += stride) {
            rows(at, h);
            if (p.total) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    Wide<S, V> o;
                    o.v.set(h[k].v);
                    if (at.mine(k, n_vec)) o.store(static_cast<S *>(p.total) + r * p.ld_total, at.vec(k));
                }
            }
            scaled(at, rstd, h);
            if constexpr (!QUANT) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    Wide<Y, V> o;
                    o.v.set(h[k].v);
                    if (at.mine(k, n_vec)) o.store(static_cast<Y *>(p.y) + r * p.ld_y, at.vec(k));
                }
            } else if (p.block) {
                quant_blocks<V, K>(h, p, r, at, n_vec, true);
            } else {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    h[k].divide(scale, inv);
                    if (at.mine(k, n_vec)) store_codes<V>(h[k].v, static_cast<char *>(p.y) + r * p.ld_y, at.vec(k), p.int8);
                }
            }
        }
        __syncthreads();                                               // the slots are written again
    }
}

// Threads per SM of the kernels with a ring: what is on its way at a time, and how rows are handed out, decide how near they
// come to the memory's rate.  Rows of up to 32 bytes per lane and turn: two stages of 512 threads, as many blocks as run at
// once (10^6 x 256 bf16 319 us, with three stages 365, with twice the threads 333, with one stage of them 419).  More bytes
// per lane: one stage, and more blocks than run at once, which take their rows as others end: 6144 threads (200 000 x 512
// fp32 243 us, 500 000 x 256 fp32 307, 10^6 x 256 bf16 around an fp32 stream 472; 1536 threads 253, 327 and 479; two stages
// of 512 threads 269, 354 and 542).
constexpr int kShortThreads = 512, kLongThreads = 6144;

template <typename X, typename S, typename Y, int V, int L, int K, bool QUANT, bool RES>
cudaError_t launch_rows(RmsArgs &p, int warps, cudaStream_t s) {
    constexpr auto kernel = rms_fwd_kernel<X, S, Y, V, L, K, QUANT, RES>;
    constexpr int R = kTurnRows<X, S, V, L, K, RES>, kGroup = L > 0 ? L : 32;
    const unsigned threads = L > 0 ? kWarpRowThreads : unsigned(warps) * 32;
    if (!columns_fit<Place<L, K, QUANT && V == 1>, K>(p.D / V, warps)) return cudaErrorInvalidConfiguration;
    const cudaError_t err = allow_shared<kernel>();
    if (err != cudaSuccess) return err;
    const int64_t rows = L > 0 ? int64_t(kWarpRowThreads / kGroup) * R : 1;
    size_t shared = 0;
    int most;
    if constexpr (kRing<X, S, V>) {
        constexpr int kLane = R * kRowBytes<X, S, V, K, RES>;
        constexpr bool kShort = kLane <= kTurnBytes || (L <= 0 && QUANT);
        p.stages = kShort && size_t(kLane) * threads * 2 <= size_t(kMostShared) ? 2 : 1;
        shared = size_t(kLane) * threads * p.stages;
        most = std::max(L < 0 ? 1 : 2, (kShort ? kShortThreads : kLongThreads) / int(threads));
        if (kShort || L < 0) most = std::min(most, blocks_per_sm<kernel>(threads, shared));      // 10 000 x 12 000 bf16 150 us, else 163
    } else {
        most = blocks_per_sm<kernel>(threads, shared);
    }
    const int64_t grid = std::min<int64_t>((p.n + rows - 1) / rows, int64_t(kSms) * most);
    return launch(kernel, dim3(unsigned(grid)), threads, shared, p, s);
}

// Rows of up to 1024 columns (narrow vectors: 512) go to a warp or a part of one, wider ones to a block: the fewest warps
// with 16 columns per thread, and then as few chunks per warp as they need.
template <typename X, typename S, typename Y, int V, bool QUANT, bool RES>
cudaError_t launch_width(RmsArgs &p, cudaStream_t s) {
    const int32_t n_vec = p.D / V, chunks = (n_vec + 31) / 32;
    if (p.D > kMostInRegisters) {
        constexpr auto kernel = rms_fwd_long_kernel<X, S, Y, V, QUANT>;
        return launch(kernel, dim3(unsigned(std::min<int64_t>(p.n, int64_t(kSms) * blocks_per_sm<kernel>(kRowThreads, 0)))), kRowThreads, 0, p, s);
    }
    if constexpr (V > 1) {
        if (n_vec == 1) return launch_rows<X, S, Y, V, 1, 1, QUANT, RES>(p, 1, s);
        if (n_vec == 2) return launch_rows<X, S, Y, V, 2, 1, QUANT, RES>(p, 1, s);
    }
    if (n_vec <= 4) return launch_rows<X, S, Y, V, 4, 1, QUANT, RES>(p, 1, s);
    if constexpr (V > 1) {
        if (n_vec <= 8) return launch_rows<X, S, Y, V, 8, 1, QUANT, RES>(p, 1, s);
        if (n_vec <= 16) return launch_rows<X, S, Y, V, 16, 1, QUANT, RES>(p, 1, s);
        if (chunks == 1) return launch_rows<X, S, Y, V, 32, 1, QUANT, RES>(p, 1, s);
    } else {
        if (n_vec <= 8) return launch_rows<X, S, Y, V, 4, 2, QUANT, RES>(p, 1, s);
        if (n_vec <= 16) return launch_rows<X, S, Y, V, 8, 2, QUANT, RES>(p, 1, s);
        if (n_vec <= 32) return launch_rows<X, S, Y, V, 8, 4, QUANT, RES>(p, 1, s);
        if constexpr (!QUANT)              // 32 columns of a scale lie in one vector of a warp
            if (n_vec <= 64) return launch_rows<X, S, Y, V, 16, 4, QUANT, RES>(p, 1, s);
    }
    if constexpr (V > 1 || QUANT)
        if (chunks == 2) return launch_rows<X, S, Y, V, 32, 2, QUANT, RES>(p, 1, s);
    if (chunks <= 4) return launch_rows<X, S, Y, V, 32, 4, QUANT, RES>(p, 1, s);
    const bool wide = p.D > kRowThreads * kPerThread;
    if constexpr (V > 1) {
        const int warps = (chunks * V + kPerThread - 1) / kPerThread;
        if (wide) return launch_rows<X, S, Y, V, -1, kPerThread / V, QUANT, RES>(p, warps, s);
        return launch_rows<X, S, Y, V, 0, kPerThread / V, QUANT, RES>(p, warps, s);
    } else {
        if (chunks <= 6) return launch_rows<X, S, Y, V, 32, 6, QUANT, RES>(p, 1, s);
        if (chunks <= 8) return launch_rows<X, S, Y, V, 32, 8, QUANT, RES>(p, 1, s);
        if (chunks <= 10) return launch_rows<X, S, Y, V, 32, 10, QUANT, RES>(p, 1, s);
        if (chunks <= 12) return launch_rows<X, S, Y, V, 32, 12, QUANT, RES>(p, 1, s);
        if (chunks <= 14) return launch_rows<X, S, Y, V, 32, 14, QUANT, RES>(p, 1, s);
        if (chunks <= 16) return launch_rows<X, S, Y, V, 32, 16, QUANT, RES>(p, 1, s);
        const int each = QUANT ? 4 : 2, units = (chunks + each - 1) / each;             // chunks that stay together
        const int warps = (units * each + kPerThread - 1) / kPerThread, k = (units + warps - 1) / warps * each;
        if (wide) {                        // as many warps as a block may have: their columns' loads are all that hides latency
            const int most = kWideThreads / 32, few = (units + most - 1) / most, many = (units + few - 1) / few;
            if constexpr (!QUANT) {
                if (few * each <= 10) return launch_rows<X, S, Y, V, -1, 10, QUANT, RES>(p, many, s);
                if (few * each == 14) return launch_rows<X, S, Y, V, -1, 14, QUANT, RES>(p, many, s);
            }
            if (few * each <= 12) return launch_rows<X, S, Y, V, -1, 12, QUANT, RES>(p, many, s);
            return launch_rows<X, S, Y, V, -1, 16, QUANT, RES>(p, many, s);
        }
        if constexpr (!QUANT) {
            if (k <= 10) return launch_rows<X, S, Y, V, 0, 10, QUANT, RES>(p, warps, s);
            if (k == 14) return launch_rows<X, S, Y, V, 0, 14, QUANT, RES>(p, warps, s);
        }
        if (k <= 12) return launch_rows<X, S, Y, V, 0, 12, QUANT, RES>(p, warps, s);
        return launch_rows<X, S, Y, V, 0, 16, QUANT, RES>(p, warps, s);
    }
}

template <typename X, typename S, typename Y, bool QUANT, bool RES, int N>
cudaError_t launch_vectors(RmsArgs &p, const Matrix (&m)[N], cudaStream_t s) {
    constexpr int kMost = sizeof(X) == 2 || sizeof(Y) == 2 ? 8 : 4;       // the narrowest type fills 16 bytes
    const int we = p.w_bf16 ? 2 : 4;
    if (vectors_fit(kMost, p.D, m)) {
        p.w_vectors = on(p.w, std::min(16, kMost * we));
        return launch_width<X, S, Y, kMost, QUANT, RES>(p, s);
    }
    if constexpr (kMost == 8)
        if (vectors_fit(4, p.D, m)) {
            p.w_vectors = on(p.w, 4 * we);
            return launch_width<X, S, Y, 4, QUANT, RES>(p, s);
        }
    p.w_vectors = 0;
    return launch_width<X, S, Y, 1, QUANT, RES>(p, s);
}
template <typename X, typename S, typename Y, bool QUANT, int N>
cudaError_t launch_typed(RmsArgs &p, const Matrix (&m)[N], cudaStream_t s) {
    if constexpr (std::is_same<X, S>::value)                              // an fp32 stream around bf16 is there
        if (!p.res) return launch_vectors<X, S, Y, QUANT, false>(p, m, s);
    return launch_vectors<X, S, Y, QUANT, true>(p, m, s);
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
    p.inverse_top = 1.0f / (kind == HAG_I8 ? 127.0f : 448.0f);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err;
    if (x_dtype != stream_dtype) err = launch_typed<__nv_bfloat16, float, uint8_t, true>(p, m, s);
    else if (x_dtype == HAG_BF16) err = launch_typed<__nv_bfloat16, __nv_bfloat16, uint8_t, true>(p, m, s);
    else err = launch_typed<float, float, uint8_t, true>(p, m, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
