// The gradient of the root-mean-square norm with the residual's addition.  With hh = h * rstd and q = g * w:
//   grad = rstd * (q - hh * mean(q * hh)) + what arrives along the residual stream,  gw = sum over rows of g * hh
// A row is read once and its gradient written once; gw stays with the threads over all their rows, is joined per block
// and then over the blocks, in a fixed order.
//
// Bound by memory.  Measured on B200, where a copy runs at 6.53 TB/s: with a gradient along the stream 10^6 x 256 bf16 294 us
// (7.0 TB/s: three reads for a write), around an fp32 stream 624 (6.6), 30 000 x 4096 bf16 147 (6.7); without one 10^6 x 256
// bf16 235 us (6.5).  Blocks of more than 512 threads have 64 registers each and no room for what they read: they read it twice,
// convert it twice and wait for it, one block per SM: 10 000 x 12 000 bf16 277 us (3.5), at 54 % of the issue slots.  The 384 to
// 464 bytes that a thread of these kernels spills are not it: reads and writes of them are 0.4 % of the
// instructions.  Rows that do not begin on 16 bytes are read one element at a time: 300 000 x 333 fp32 244 us (6.6), bf16 183
// (4.4), 5001 x 1433 fp32 without a gradient along the stream 21.6 (4.0; 3 of them the join).
#include "hag_rms.cuh"

namespace {

using namespace hagn;

struct RmsBwdArgs {
    int64_t n;
    int32_t D;
    int32_t w_bf16, w_vectors;
    const void *g, *total, *w, *along;      // along: gradient that arrives along the residual stream
    const float *rstd;
    int64_t ld_g, ld_total, ld_along, ld_out, ld_x;
    void *out, *x;                          // x: the gradient in bf16 besides
    float *partial;                         // [parts][D]; NULL: gw is not wanted
    void *gw;
    int32_t stages;                         // of the ring
    int32_t parts;                          // blocks that leave a sum of their own
    bool joined;                            // the only block leaves gw itself
};

// A block's sum for column c of gw: a part of it, or, from the only block, the result.
__device__ __forceinline__ void leave(const RmsBwdArgs &p, int64_t c, float v) {
    if (p.parts > 1) p.partial[int64_t(blockIdx.x) * p.D + c] = v;
    else store_weight(p.gw, p.w_bf16, c, v);
}

template <typename S, int V>
__device__ __forceinline__ void store_gradient(const RmsBwdArgs &p, int64_t r, int64_t vec, const hagr::Pairs<V> &o) {
    Wide<S, V> a;
    a.v.set(o.v);
    a.store(static_cast<S *>(p.out) + r * p.ld_out, vec);
    if constexpr (sizeof(S) == 4) {
        if (p.x) {
            Wide<__nv_bfloat16, V> b;
            b.v.set(o.v);
            b.store(static_cast<__nv_bfloat16 *>(p.x) + r * p.ld_x, vec);
        }
    }
}

// Rows whose vectors fill 16 bytes are copied into a ring in shared memory some turns ahead; others are read when their turn
// comes, all of them before the first is used.
template <typename Y, int V> constexpr bool kRing = V * int(sizeof(Y)) >= 16;
// Rows per turn: two where they are 96 bytes per lane of the ring (10^6 x 256 bf16 295 us, with one 323; of one or two
// lanes one: 2 000 000 x 8 bf16 27 us, with two 36), or 8 columns.  Two stages of as much, one of more or where lanes read
// what others copied (100 000 x 1024 fp32 237 us, with two 256; 10^6 x 256 bf16 around an fp32 stream 623 and 665;
// 500 000 x 512 bf16 304, with two 293).
constexpr int kTurnBytes = 96;
template <typename S, typename Y, int V, int K, bool ALONG> constexpr int kRowBytes = K * V * int(sizeof(Y) + (ALONG ? 2 : 1) * sizeof(S));    // per lane
template <typename S, typename Y, int V, int L, int K, bool ALONG> constexpr int kTurnRows =
    L <= 0 ? 1 : kRing<Y, V> ? (kRowBytes<S, Y, V, K, ALONG> * 2 <= kTurnBytes && L > 2 ? 2 : 1) : V * K <= 8 ? 2 : 1;

template <typename S, typename Y, int V, int L, int K, bool ALONG>
__global__ void __launch_bounds__(kThreadsOf<L>, L > 0 ? 2 : 1) rms_bwd_kernel(const __grid_constant__ RmsBwdArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int R = kTurnRows<S, Y, V, L, K, ALONG>;
    constexpr bool RING = kRing<Y, V>;
    using P = Place<L, K, false>;
    using CY = ChunkCopy<Y, V, P, K>;
    using CS = ChunkCopy<S, V, P, K>;
    using Values = hagr::Pairs<V>;
    extern __shared__ __align__(16) char raw[];
    __shared__ float slots[2][32];
    const P at;
    const int n_vec = p.D / V;
    const float inverse = 1.0f / float(p.D);
    const int64_t ld_g = p.ld_g * int64_t(sizeof(Y)), ld_total = p.ld_total * int64_t(sizeof(S)), ld_along = p.ld_along * int64_t(sizeof(S));
    const int row_bytes = CY::bytes() + (ALONG ? 2 : 1) * CS::bytes(), stage = R * row_bytes, end = p.stages * stage;
    int64_t next = at.group * R;
    int write = 0, read = 0;
    float rstd_next[R];
    auto statistics = [&](int64_t r) {                         // of a turn ahead
#pragma unroll
        for (int i = 0; i < R; ++i) rstd_next[i] = r + i < p.n ? __ldcg(p.rstd + r + i) : 0.0f;
    };
    auto issue = [&]() {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t r = next + i;
            char *const to = raw + write + i * row_bytes;
            CY::issue(to, static_cast<const char *>(p.g) + r * ld_g, at, n_vec, r < p.n);
            CS::issue(to + CY::bytes(), static_cast<const char *>(p.total) + r * ld_total, at, n_vec, r < p.n);
            if (ALONG) CS::issue(to + CY::bytes() + CS::bytes(), static_cast<const char *>(p.along) + r * ld_along, at, n_vec, r < p.n);
        }
        hagr::commit_copies();
        next += at.groups * R;
        write = write + stage == end ? 0 : write + stage;
    };
    hagk::pdl_wait();
    if constexpr (RING) {
        for (int s = 0; s < p.stages; ++s) issue();
    }
    statistics(at.group * R);
    // Blocks of many threads keep the sums of gw in registers and read everything else twice, out of the ring (or the
    // caches); the ring's stage is given back at the end of the row.
    constexpr bool kHold = kKeepWeights<L>;
    Values w[kHold ? K : 1], sum[K];
#pragma unroll
    for (int k = 0; k < K; ++k) sum[k].fill(0.0f);
    if constexpr (kHold) load_all_weights<V, K>(w, p.w, p.w_bf16, p.w_vectors, at, n_vec);
    // narrow vectors: rows as they are in memory, the next ones on their way while a row of a block is worked on
    constexpr bool kAhead = !RING && L == 0 && K <= 8;
    struct Raw {
        hagr::Vec<Y, V> g[R][K];
        hagr::Vec<S, V> t[R][K], a[ALONG ? R : 1][ALONG ? K : 1];
    };
    auto fetch = [&](Raw &x, int64_t r0) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const bool live = r0 + i < p.n;
            const char *gr = static_cast<const char *>(p.g) + (r0 + i) * ld_g, *tr = static_cast<const char *>(p.total) + (r0 + i) * ld_total;
            const char *ar = static_cast<const char *>(p.along) + (r0 + i) * ld_along;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                x.g[i][k].zero();
                x.t[i][k].zero();
                if (live && at.mine(k, n_vec)) {
                    x.g[i][k].template load<hagr::kKeep>(gr, at.vec(k));
                    x.t[i][k].template load<hagr::kKeep>(tr, at.vec(k));
                }
            }
            if constexpr (ALONG) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    x.a[i][k].zero();
                    if (live && at.mine(k, n_vec)) x.a[i][k].template load<hagr::kKeep>(ar, at.vec(k));
                }
            }
        }
    };
    Raw next_rows;
    if constexpr (kAhead) fetch(next_rows, at.group * R);
    auto give_back = [&]() {
        if (CY::kCrosses || CS::kCrosses) __syncwarp();
        issue();
        read = read + stage == end ? 0 : read + stage;
    };
    int turn = 0;
    for (int64_t lead = at.leader() * R, r0 = at.group * R; lead < p.n; lead += at.groups * R, r0 += at.groups * R, turn ^= 1) {
        float rstd[R], s[R];
#pragma unroll
        for (int i = 0; i < R; ++i) rstd[i] = rstd_next[i];
        statistics(r0 + at.groups * R);
        if constexpr (RING) {
            hagr::wait_oldest(p.stages);
            if (CY::kCrosses || CS::kCrosses) __syncwarp();
        }
        if constexpr (kHold) {
            Values hh[R][K], q[R][K], a[R][K];
            if constexpr (RING) {
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const char *from = raw + read + i * row_bytes;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        q[i][k] = CY::get(from, at, k);
                        hh[i][k] = CS::get(from + CY::bytes(), at, k);
                        if (ALONG) a[i][k] = CS::get(from + CY::bytes() + CS::bytes(), at, k);
                        else a[i][k].fill(0.0f);
                    }
                }
                give_back();
            } else {
                Raw now;
                if constexpr (kAhead) {
                    now = next_rows;
                    fetch(next_rows, r0 + at.groups * R);
                } else {
                    fetch(now, r0);
                }
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        q[i][k] = hagr::widen(now.g[i][k]);
                        hh[i][k] = hagr::widen(now.t[i][k]);
                        if constexpr (ALONG) a[i][k] = hagr::widen(now.a[i][k]);
                        else a[i][k].fill(0.0f);
                    }
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                s[i] = 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    hh[i][k].mul_all(rstd[i]);
                    sum[k].fma(q[i][k], hh[i][k]);
                    q[i][k].mul(w[k]);
                    s[i] += q[i][k].dot(hh[i][k]);
                }
            }
            const Sums<L, R> means(s, slots[turn], [&](float v) { return -v * inverse; });
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float m = means.get(i);
                if (r0 + i >= p.n) continue;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    hh[i][k].affine(m, q[i][k]);
                    a[i][k].add_scaled(hh[i][k], rstd[i]);
                    if (at.mine(k, n_vec)) store_gradient<S, V>(p, r0 + i, at.vec(k), a[i][k]);
                }
            }
        } else {
            static_assert(kHold || R == 1, "");
            const char *gr = static_cast<const char *>(p.g) + r0 * ld_g, *tr = static_cast<const char *>(p.total) + r0 * ld_total;
            const char *br = static_cast<const char *>(p.along) + r0 * ld_along, *from = raw + read;
            constexpr int U = V >= 4 ? 1 : K % 4 == 0 ? 4 : 2; // vectors at a time
            static_assert(K % U == 0, "");
            auto pass = [&](auto f) {
#pragma unroll
                for (int k0 = 0; k0 < K; k0 += U) {
                    Values g[U], hh[U], w1[U];
                    if constexpr (RING) {
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            g[u] = CY::get(from, at, k0 + u);
                            hh[u] = CS::get(from + CY::bytes(), at, k0 + u);
                        }
                    } else {
                        hagr::Vec<Y, V> x[U];
                        hagr::Vec<S, V> y[U];
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            x[u].zero();
                            y[u].zero();
                            if (at.mine(k0 + u, n_vec)) {
                                x[u].template load<hagr::kKeep>(gr, at.vec(k0 + u));
                                y[u].template load<hagr::kKeep>(tr, at.vec(k0 + u));
                            }
                        }
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            g[u] = hagr::widen(x[u]);
                            hh[u] = hagr::widen(y[u]);
                        }
                    }
                    load_all_weights<V, U>(w1, p.w, p.w_bf16, p.w_vectors, From<P>{at, k0}, n_vec);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        hh[u].mul_all(rstd[0]);
                        f(k0 + u, g[u], hh[u], w1[u]);
                    }
                }
            };
            s[0] = 0.0f;
            pass([&](int k, Values &g, const Values &hh, const Values &w1) {
                sum[k].fma(g, hh);
                g.mul(w1);
                s[0] += g.dot(hh);
            });
            const float m = -group_sum<L>(s[0], slots[turn]) * inverse;
            pass([&](int k, Values &g, Values &hh, const Values &w1) {
                Values o;
                o.fill(0.0f);
                if (ALONG) {
                    if constexpr (RING) {
                        o = CS::get(from + CY::bytes() + CS::bytes(), at, k);
                    } else {
                        hagr::Vec<S, V> b;
                        b.zero();
                        if (at.mine(k, n_vec)) b.template load<hagr::kKeep>(br, at.vec(k));
                        o = hagr::widen(b);
                    }
                }
                g.mul(w1);
                hh.affine(m, g);
                o.add_scaled(hh, rstd[0]);
                if (at.mine(k, n_vec)) store_gradient<S, V>(p, r0, at.vec(k), o);
            });
            if constexpr (RING) give_back();
        }
    }
    if constexpr (RING) hagr::wait_copies<0>();
    if (!p.partial) return;
    if constexpr (L <= 0) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (at.mine(k, n_vec)) leave(p, int64_t(at.vec(k)) * V + j, sum[k].v[j]);
    } else {
        // groups of the warp, then warps of the block, in a fixed order
        constexpr int C = L * K * V, kWarps = kWarpRowThreads / 32;
        float *const joined = reinterpret_cast<float *>(raw);              // [warps][C], over the ring
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float v = sum[k].v[j];
#pragma unroll
                for (int o = L; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                if ((threadIdx.x & 31) < L) joined[(threadIdx.x >> 5) * C + at.vec(k) * V + j] = v;
            }
        __syncthreads();
        for (int c = threadIdx.x; c < p.D; c += kWarpRowThreads) {
            float v = 0.0f;
#pragma unroll
            for (int o = 0; o < kWarps; ++o) v += joined[o * C + c];
            leave(p, c, v);
        }
    }
}

// Rows of more columns: a block walks its row twice, the second time out of the caches; gw has a kernel of its own.
template <typename S, typename Y, int V>
__global__ void __launch_bounds__(kRowThreads, 1) rms_bwd_long_kernel(const __grid_constant__ RmsBwdArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int K = V == 8 ? 1 : V == 4 ? 2 : 4;
    using Values = hagr::Pairs<V>;
    __shared__ float slots[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n_vec = p.D / V, stride = (kRowThreads / 32) * 32 * K;
    struct Walk {                                             // K chunks side by side
        int base;
        __device__ __forceinline__ int vec(int k) const { return base + k * 32; }
        __device__ __forceinline__ bool mine(int k, int n) const { return base + k * 32 < n; }
    };
    auto walk = [&](auto f) {
        for (Walk at{warp * 32 * K + lane}; at.base - lane < n_vec; at.base += stride) f(at);
    };
    hagk::pdl_wait();
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x) {
        const Y *gr = static_cast<const Y *>(p.g) + r * p.ld_g;
        const S *tr = static_cast<const S *>(p.total) + r * p.ld_total;
        const S *ar = static_cast<const S *>(p.along) + (p.along ? r * p.ld_along : 0);
        const float rstd = __ldcg(p.rstd + r);
        // hh and g of the vectors, and the weights
        auto rows = [&](const Walk &at, Values (&hh)[K], Values (&g)[K], Values (&w)[K]) {
            Wide<Y, V> x[K];
            Wide<S, V> t[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                x[k].v.zero();
                t[k].v.zero();
                if (at.mine(k, n_vec)) {
                    x[k].load(gr, at.vec(k));
                    t[k].load(tr, at.vec(k));
                }
            }
            load_all_weights<V, K>(w, p.w, p.w_bf16, p.w_vectors, at, n_vec);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                g[k] = hagr::widen(x[k].v);
                hh[k] = hagr::widen(t[k].v);
                hh[k].mul_all(rstd);
            }
        };
        float s = 0.0f;
        walk([&](const Walk &at) {
            Values hh[K], g[K], w[K];
            rows(at, hh, g, w);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                g[k].mul(hh[k]);
                s += g[k].dot(w[k]);
            }
        });
        const float m = -group_sum<0>(s, slots) / float(p.D);
        walk([&](const Walk &at) {
            Values hh[K], g[K], w[K];
            Wide<S, V> a[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                a[k].v.zero();
                if (p.along && at.mine(k, n_vec)) a[k].load(ar, at.vec(k));
            }
            rows(at, hh, g, w);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                g[k].mul(w[k]);
                hh[k].affine(m, g[k]);
                Values o = hagr::widen(a[k].v);
                o.add_scaled(hh[k], rstd);
                if (at.mine(k, n_vec)) store_gradient<S, V>(p, r, at.vec(k), o);
            }
        });
        __syncthreads();                                      // the slots are written again
    }
}

// gw of one strip of 32 columns and one part of the rows.
constexpr int kStripRows = 8;
template <typename S, typename Y>
__global__ void __launch_bounds__(32 * kStripRows) rms_weight_strips_kernel(const __grid_constant__ RmsBwdArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float sum[kStripRows][32];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane, step = int64_t(gridDim.y) * kStripRows;
    float a = 0.0f;
    hagk::pdl_wait();
    if (c < p.D)
        for (int64_t r = int64_t(blockIdx.y) * kStripRows + part; r < p.n; r += step)
            a += load_one<Y>(p.g, r * p.ld_g + c) * (load_one<S>(p.total, r * p.ld_total + c) * __ldcg(p.rstd + r));
    sum[part][lane] = a;
    __syncthreads();
    if (part == 0 && c < p.D) {
        a = 0.0f;
#pragma unroll
        for (int k = 0; k < kStripRows; ++k) a += sum[k][lane];
        p.partial[int64_t(blockIdx.y) * p.D + c] = a;
    }
}

// gw from the parts: a block takes 32 columns, its 32 warps every 32nd part each.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(32 * kJoinWarps) rms_weight_join_kernel(const __grid_constant__ RmsBwdArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float sum[kJoinWarps][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane;
    hagk::pdl_wait();
    float s = 0.0f;
    if (c < p.D) {
#pragma unroll 8
        for (int q = warp; q < p.parts; q += kJoinWarps) s += __ldcg(p.partial + int64_t(q) * p.D + c);
    }
    sum[warp][lane] = s;
    __syncthreads();
    s = hagr::warp_sum(sum[lane][warp]);                      // column `warp` of this block
    const int64_t k = int64_t(blockIdx.x) * 32 + warp;
    if (lane == 0 && k < p.D) store_weight(p.gw, p.w_bf16, k, s);
}

constexpr int kParts = 64;                                    // of the strips
// Parts of gw, i.e. blocks of the other kernels, at most: the wider the rows, the fewer blocks fit an SM.
int most_parts(int32_t D) { return kSms * std::max(1, std::min(8, 16384 / D)); }
// Values of a gradient that one block takes alone, without a second launch.
constexpr int64_t kFewValues = 16384;

template <typename S, typename Y, int V, int L, int K, bool ALONG>
cudaError_t launch_rows(RmsBwdArgs &p, int warps, cudaStream_t s) {
    constexpr auto kernel = rms_bwd_kernel<S, Y, V, L, K, ALONG>;
    constexpr int R = kTurnRows<S, Y, V, L, K, ALONG>, kGroup = L > 0 ? L : 32;
    const unsigned threads = L > 0 ? kWarpRowThreads : unsigned(warps) * 32;
    if (!columns_fit<Place<L, K, false>, K>(p.D / V, warps)) return cudaErrorInvalidConfiguration;
    const cudaError_t err = allow_shared<kernel>();
    if (err != cudaSuccess) return err;
    size_t shared = L > 0 ? size_t(threads / 32) * L * K * V * 4 : 0;
    if constexpr (kRing<Y, V>) {
        constexpr int kLane = R * kRowBytes<S, Y, V, K, ALONG>;
        p.stages = (kLane <= kTurnBytes && V * sizeof(S) == 16) || L < 0 ? 2 : 1;
        if (size_t(kLane) * threads * p.stages > size_t(kMostShared)) p.stages = 1;
        shared = std::max(shared, size_t(kLane) * threads * p.stages);
    }
    // Two operands: four times as many blocks as run at once, but no more than there are parts (eight per SM at most), which take
    // their rows as others end (10^6 x 256 bf16 235 us, as many as run 247); three operands, or rows of blocks: as many as run
    // (10^6 x 256 bf16 295 us, four times as many 300).  Without gw the number of parts binds nothing, and costs nothing: 2 000 000
    // x 8 bf16 20.1 us, without that limit 20.7, 10^6 x 64 60.8 and 60.9.
    const int most = blocks_per_sm<kernel>(threads, shared) * (kRing<Y, V> && L > 0 && !ALONG ? 4 : 1);
    const int64_t rows = L > 0 ? int64_t(kWarpRowThreads / kGroup) * R : 1;
    int64_t grid = std::min<int64_t>((p.n + rows - 1) / rows, std::min(kSms * most, most_parts(p.D)));
    if (L > 0 && p.partial && p.n * p.D <= kFewValues) grid = 1;
    p.parts = int32_t(grid);
    p.joined = grid == 1;
    return launch(kernel, dim3(unsigned(grid)), threads, shared, p, s);
}

template <typename S, typename Y, int V, bool ALONG>
cudaError_t launch_width(RmsBwdArgs &p, cudaStream_t s) {
    const int32_t n_vec = p.D / V, chunks = (n_vec + 31) / 32;
    if (p.D > kMostInRegisters) {
        if (p.partial) {       // first: the gradient may take the place of what they read
            p.parts = int32_t(std::min<int64_t>((p.n + kStripRows - 1) / kStripRows, kParts));
            const cudaError_t err = launch(rms_weight_strips_kernel<S, Y>, dim3(unsigned((p.D + 31) / 32), unsigned(p.parts)), 32 * kStripRows, 0, p, s);
            if (err != cudaSuccess) return err;
        }
        return launch(rms_bwd_long_kernel<S, Y, V>, dim3(unsigned(std::min<int64_t>(p.n, kSms * 2))), kRowThreads, 0, p, s);
    }
    if constexpr (V > 1) {
        if (n_vec == 1) return launch_rows<S, Y, V, 1, 1, ALONG>(p, 1, s);
        if (n_vec == 2) return launch_rows<S, Y, V, 2, 1, ALONG>(p, 1, s);
    }
    if (n_vec <= 4) return launch_rows<S, Y, V, 4, 1, ALONG>(p, 1, s);
    if constexpr (V > 1) {
        if (n_vec <= 8) return launch_rows<S, Y, V, 8, 1, ALONG>(p, 1, s);
        if (n_vec <= 16) return launch_rows<S, Y, V, 16, 1, ALONG>(p, 1, s);
        if (chunks == 1) return launch_rows<S, Y, V, 32, 1, ALONG>(p, 1, s);
        if (chunks == 2) return launch_rows<S, Y, V, 32, 2, ALONG>(p, 1, s);
    } else {
        if (n_vec <= 8) return launch_rows<S, Y, V, 4, 2, ALONG>(p, 1, s);
        if (n_vec <= 16) return launch_rows<S, Y, V, 8, 2, ALONG>(p, 1, s);
        if (n_vec <= 32) return launch_rows<S, Y, V, 8, 4, ALONG>(p, 1, s);
        if (n_vec <= 64) return launch_rows<S, Y, V, 16, 4, ALONG>(p, 1, s);
    }
    if constexpr (V < 8)
        if (chunks <= 4) return launch_rows<S, Y, V, 32, 4, ALONG>(p, 1, s);
    const bool wide = p.D > kRowThreads * kPerThread;
    if constexpr (V > 1) {
        const int warps = (chunks * V + kPerThread - 1) / kPerThread;
        if (wide) return launch_rows<S, Y, V, -1, kPerThread / V, ALONG>(p, warps, s);
        return launch_rows<S, Y, V, 0, kPerThread / V, ALONG>(p, warps, s);
    } else {
        if (chunks <= 6) return launch_rows<S, Y, V, 32, 6, ALONG>(p, 1, s);
        if (chunks <= 8) return launch_rows<S, Y, V, 32, 8, ALONG>(p, 1, s);
        if (chunks <= 10) return launch_rows<S, Y, V, 32, 10, ALONG>(p, 1, s);
        if (chunks <= 12) return launch_rows<S, Y, V, 32, 12, ALONG>(p, 1, s);
        if (chunks <= 14) return launch_rows<S, Y, V, 32, 14, ALONG>(p, 1, s);
        if (chunks <= 16) return launch_rows<S, Y, V, 32, 16, ALONG>(p, 1, s);
        // eight chunks per warp leave registers for the next row: 39 960 x 1001 bf16 76 us, with up to sixteen 87; 5000 x 1001
        // fp32 17.6 and 22.4 (of 17 and 18 chunks more than the last two of a warp would lie beyond the row)
        if (chunks > 18 && chunks <= kRowThreads / 32 * 8) return launch_rows<S, Y, V, 0, 8, ALONG>(p, (chunks + 7) / 8, s);
        const int pairs = (chunks + 1) / 2, warps = (2 * pairs + kPerThread - 1) / kPerThread, k = (pairs + warps - 1) / warps * 2;
        if (wide) {            // as many warps as a block may have: their columns' loads are all that hides latency
            const int most = kWideThreads / 32, few = (pairs + most - 1) / most, many = (pairs + few - 1) / few;
            if (few <= 5) return launch_rows<S, Y, V, -1, 10, ALONG>(p, many, s);
            if (few == 6) return launch_rows<S, Y, V, -1, 12, ALONG>(p, many, s);
            if (few == 7) return launch_rows<S, Y, V, -1, 14, ALONG>(p, many, s);
            return launch_rows<S, Y, V, -1, 16, ALONG>(p, many, s);
        }
        if (k <= 10) return launch_rows<S, Y, V, 0, 10, ALONG>(p, warps, s);
        if (k <= 12) return launch_rows<S, Y, V, 0, 12, ALONG>(p, warps, s);
        if (k <= 14) return launch_rows<S, Y, V, 0, 14, ALONG>(p, warps, s);
        return launch_rows<S, Y, V, 0, 16, ALONG>(p, warps, s);
    }
}

template <typename S, typename Y, bool ALONG, int N>
cudaError_t launch_vectors(RmsBwdArgs &p, const Matrix (&m)[N], cudaStream_t s) {
    constexpr int kMost = sizeof(Y) == 2 ? 8 : 4;             // the narrowest type fills 16 bytes
    const int we = p.w_bf16 ? 2 : 4;
    if (vectors_fit(kMost, p.D, m)) {
        p.w_vectors = on(p.w, std::min(16, kMost * we));
        return launch_width<S, Y, kMost, ALONG>(p, s);
    }
    if constexpr (kMost == 8)
        if (vectors_fit(4, p.D, m)) {
            p.w_vectors = on(p.w, 4 * we);
            return launch_width<S, Y, 4, ALONG>(p, s);
        }
    p.w_vectors = 0;
    return launch_width<S, Y, 1, ALONG>(p, s);
}
template <typename S, typename Y, int N>
cudaError_t launch_typed(RmsBwdArgs &p, const Matrix (&m)[N], cudaStream_t s) {
    return p.along ? launch_vectors<S, Y, true>(p, m, s) : launch_vectors<S, Y, false>(p, m, s);
}

}  // namespace

extern "C" size_t hag_rms_norm_bwd_workspace_bytes(int64_t n, int32_t D) {
    if (n < 0 || D <= 0) return 0;
    return size_t(std::max<int64_t>(std::min<int64_t>(most_parts(D), n), 1)) * size_t(D) * 4;
}

extern "C" hag_status hag_rms_norm_bwd(int64_t n, int32_t D, const void *grad_y, hag_dtype y_dtype, int64_t ld_grad_y,
                                       const void *total, hag_dtype stream_dtype, int64_t ld_total, const float *rstd,
                                       const void *weight, hag_dtype weight_dtype, const void *grad_total, int64_t ld_grad_total,
                                       void *grad_residual, int64_t ld_grad_residual, void *grad_x, int64_t ld_grad_x,
                                       void *grad_weight, void *workspace, void *cuda_stream) {
    if (!dtype_ok(y_dtype) || !dtype_ok(stream_dtype) || !dtype_ok(weight_dtype)) return HAG_ERR_DTYPE;
    if (y_dtype != stream_dtype && stream_dtype != HAG_F32) return HAG_ERR_DTYPE;
    if (grad_x && stream_dtype != HAG_F32) return HAG_ERR_DTYPE;
    const int se = size_of(stream_dtype);
    const Matrix m[] = {{grad_y, ld_grad_y, size_of(y_dtype), false, true}, {total, ld_total, se, false, true},
                        {grad_total, ld_grad_total, se, false, false}, {grad_residual, ld_grad_residual, se, true, true},
                        {grad_x, ld_grad_x, 2, true, false}};
    const hag_status st = check(n, D, weight, weight_dtype, rstd, m);
    if (st != HAG_OK) return st;
    if (n > 0 && !rstd) return HAG_ERR_NULL;
    if (!on(grad_weight, size_of(weight_dtype))) return HAG_ERR_ALIGN;
    if (grad_weight && !workspace) return HAG_ERR_WORKSPACE;
    if (!hagl::aligned16(workspace)) return HAG_ERR_ALIGN;
    RmsBwdArgs p{};
    p.n = n; p.D = D; p.w_bf16 = weight_dtype == HAG_BF16; p.w = weight; p.rstd = rstd;
    p.g = grad_y; p.ld_g = ld_grad_y; p.total = total; p.ld_total = ld_total; p.along = grad_total; p.ld_along = ld_grad_total;
    p.out = grad_residual; p.ld_out = ld_grad_residual; p.x = grad_x; p.ld_x = ld_grad_x;
    p.partial = grad_weight ? static_cast<float *>(workspace) : nullptr;
    p.gw = grad_weight;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err = cudaSuccess;
    if (n > 0) {
        if (y_dtype != stream_dtype) err = launch_typed<float, __nv_bfloat16>(p, m, s);
        else if (y_dtype == HAG_BF16) err = launch_typed<__nv_bfloat16, __nv_bfloat16>(p, m, s);
        else err = launch_typed<float, float>(p, m, s);
    }
    if (err == cudaSuccess && grad_weight && !p.joined)            // no rows: the sum of no parts
        err = launch(rms_weight_join_kernel, dim3(unsigned((int64_t(D) + 31) / 32)), 32 * kJoinWarps, 0, p, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
