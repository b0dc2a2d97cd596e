// Group normalisation with the channels last: pixels of c neighbouring
// channels, of which a block takes `tile`.
#pragma once
#include "group_norm.h"

namespace psc {
namespace gn {
namespace {

// What a thread of a block has: V channels (from channel `c` on, `rel` of the
// block's `width`; none if `rel` is past them) of every rows-th pixel.
struct Place {
    int n, chunk, c0, width;
    int rel, row, rows;
    int first, last;        // pixels of the block
    bool on;
};
// Blocks that are eight apart run on the same compute die, whose cache holds a
// line of memory once: the `near` tiles that share lines are eight apart.
template <int V>
__device__ __forceinline__ bool place(const Cols& q, int images, Place& p) {
    const unsigned per = 8u * unsigned(q.near);
    const unsigned slab = blockIdx.x / per * 8 + (blockIdx.x & 7);      // of an image, a chunk and `near` tiles
    const unsigned wide = unsigned(q.tiles + q.near - 1) / unsigned(q.near);
    const unsigned unit = slab / wide;
    const int tile = int((slab - unit * wide) * unsigned(q.near) + (blockIdx.x % per >> 3));
    p.n = int(unit / unsigned(q.chunks));
    if (p.n >= images || tile >= q.tiles) return false;
    p.chunk = int(unit % unsigned(q.chunks));
    p.c0 = tile * q.tile;
    p.width = q.c - p.c0 < q.tile ? q.c - p.c0 : q.tile;
    const int cols = 1 << q.cols_log2;
    p.rel = int(threadIdx.x & unsigned(cols - 1)) * V;
    p.row = int(threadIdx.x >> q.cols_log2);
    p.rows = int(blockDim.x >> q.cols_log2);
    p.first = p.chunk * q.pixels;
    p.last = q.hw - p.first < q.pixels ? q.hw : p.first + q.pixels;
    p.on = p.rel < p.width;
    return true;
}
// The element that the block's offsets count from.
__device__ __forceinline__ int64_t base_of(const Cols& q, const Place& p) {
    return (int64_t(p.n) * q.hw + p.first) * q.c + p.c0;
}
// Calls f(i, byte) for the vectors of this thread: slot i, which begins `byte` bytes behind the base.
template <int DT, int K, class F>
__device__ __forceinline__ void each(const Cols& q, const Place& p, F f) {
    if (!p.on) return;
    constexpr uint32_t elt = sizeof(typename Elt<DT>::T);
    uint32_t byte = (uint32_t(p.row) * uint32_t(q.c) + uint32_t(p.rel)) * elt;
    const uint32_t step = uint32_t(p.rows) * uint32_t(q.c) * elt;
    int left = p.last - p.first - p.row;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        if (left > 0) f(i, byte);
        left -= p.rows, byte += step;
    }
}
// V values of the thread's channels; they lie at multiples of four bytes.
typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
template <int V> __device__ __forceinline__ void values(const float* p, bool on, float fill, float (&f)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = fill;
    if (!p || !on) return;
    if constexpr (V == 1) {
        f[0] = *p;
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const f4u t = *reinterpret_cast<const f4u*>(p + j);
            f[j] = t.x, f[j + 1] = t.y, f[j + 2] = t.z, f[j + 3] = t.w;
        }
    }
}

// Calls f(g, sum) once for each of the block's groups, the sums weighted: a
// thread adds a group of few channels, a wave one of many.
template <class F>
__device__ __forceinline__ void each_group(const Cols& q, int count, const float* ch, const float* weight, F f) {
    if (q.cg <= 16) {
        for (int g = threadIdx.x; g < count; g += blockDim.x) {
            float s = 0.f;
            for (int k = 0; k < q.cg; ++k) s = fmaf(or_one(weight, g * q.cg + k), ch[g * q.cg + k], s);
            f(g, s);
        }
    } else {
        for (int g = int(threadIdx.x >> 6); g < count; g += int(blockDim.x >> 6)) {
            float s = 0.f;
            for (int k = int(threadIdx.x & 63); k < q.cg; k += 64) s = fmaf(or_one(weight, g * q.cg + k), ch[g * q.cg + k], s);
            s = wave_sum(s);
            if ((threadIdx.x & 63) == 0) f(g, s);
        }
    }
}

template <int DT, int V, int K, int ACT, int PAST>
__global__ __launch_bounds__(threads_of(DT, V, K)) void k_gn_cols_fwd(const typename Elt<DT>::T* __restrict__ x, Cols q,
                                                                  int images, Params w, float eps,
                                                                  typename Elt<DT>::T* __restrict__ y,
                                                                  float* __restrict__ mean, float* __restrict__ rstd) {
    using P = Pack<DT, V>;
    extern __shared__ float lds[];              // the waves' sums, the channels', the groups'
    Place p;
    if (!place<V>(q, images, p)) return;
    float* ch = lds + sum_rows(q) * q.tile;
    float* gr = ch + q.tile;
    const int count = p.width / q.cg;
    const float m = float(q.cg) * float(q.hw);
    const int64_t g0 = int64_t(p.n) * q.groups + p.c0 / q.cg;
    const int64_t at = base_of(q, p);
    const typename Elt<DT>::T* xb = x + at;
    typename P::R d[K];
    each<DT, K>(q, p, [&](int i, uint32_t byte) { d[i] = get<typename P::R, false>(xb, byte); });
    float ga[V], be[V];
    values<V>(w.gamma ? w.gamma + p.c0 + p.rel : nullptr, p.on, 1.f, ga);
    values<V>(w.beta ? w.beta + p.c0 + p.rel : nullptr, p.on, 0.f, be);
    float s[V], mu[V], r[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
    each<DT, K>(q, p, [&](int i, uint32_t) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] += f[j];
    });
    wave_channels<V>(s, q, p.width, lds);
    __syncthreads();
    for (int k = threadIdx.x; k < p.width; k += blockDim.x) ch[k] = sum_of_channel(lds, q, k);
    __syncthreads();
    each_group(q, count, ch, nullptr, [&](int g, float sum) { gr[g] = sum / m; });
    __syncthreads();
    int g[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        g[j] = p.on ? group_of(q, p.rel + j) : 0;
        mu[j] = gr[g[j]];
        s[j] = 0.f;
    }
    each<DT, K>(q, p, [&](int i, uint32_t) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float e = f[j] - mu[j];
            s[j] = fmaf(e, e, s[j]);
        }
    });
    wave_channels<V>(s, q, p.width, lds);
    __syncthreads();
    for (int k = threadIdx.x; k < p.width; k += blockDim.x) ch[k] = sum_of_channel(lds, q, k);
    __syncthreads();
    each_group(q, count, ch, nullptr, [&](int g, float sum) {
        const float2 ms = stats_of(gr[g], sum / m, eps);
        gr[g] = ms.y;
        if (mean) mean[g0 + g] = ms.x, rstd[g0 + g] = ms.y;
    });
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] = gr[g[j]];
    each<DT, K>(q, p, [&](int i, uint32_t byte) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = forward<ACT>(Coeff{mu[j], r[j], ga[j], be[j]}, f[j]);
        put<PAST == 2>(y + at, byte, P::close(f));
    });
}

// The mean and rstd that lie in memory, of the thread's channel j.
__device__ __forceinline__ auto kept(const Cols& q, const Place& p, const float* mean, const float* rstd) {
    return [&q, &p, mean, rstd](int j) {
        const int64_t g = int64_t(p.n) * q.groups + (p.on ? group_of(q, p.c0 + p.rel + j) : 0);
        return make_float2(mean[g], rstd[g]);
    };
}
template <int V, class F>
__device__ __forceinline__ void coefficients(const Cols& q, const Place& p, const Params& w, F stats, Coeff (&k)[V]) {
    float ga[V], be[V];
    const int c = p.c0 + p.rel;
    values<V>(w.gamma ? w.gamma + c : nullptr, p.on, 1.f, ga);
    values<V>(w.beta ? w.beta + c : nullptr, p.on, 0.f, be);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float2 ms = stats(j);
        k[j] = Coeff{ms.x, ms.y, ga[j], be[j]};
    }
}

template <int DT, int V, int K, int ACT>
__device__ __forceinline__ void sums_back(const typename Pack<DT, V>::R (&d)[K], const typename Pack<DT, V>::R (&e)[K],
                                          const Cols& q, const Place& p, const Coeff (&k)[V], float (&a)[V], float (&b)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] = 0.f, b[j] = 0.f;
    each<DT, K>(q, p, [&](int i, uint32_t) {
        float f[V], g[V];
        Pack<DT, V>::open(d[i], f);
        Pack<DT, V>::open(e[i], g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = normal(k[j], f[j]);
            const float du = slope<ACT>(k[j], xh, g[j]);
            a[j] += du;
            b[j] = fmaf(du, xh, b[j]);
        }
    });
}
template <int DT, int V, int K, int ACT, int PAST>
__device__ __forceinline__ void write_back(const typename Pack<DT, V>::R (&d)[K], const typename Pack<DT, V>::R (&e)[K],
                                           const Cols& q, const Place& p, const Coeff (&k)[V], const Back (&s)[V],
                                           typename Elt<DT>::T* dxb) {
    each<DT, K>(q, p, [&](int i, uint32_t byte) {
        float f[V], g[V];
        Pack<DT, V>::open(d[i], f);
        Pack<DT, V>::open(e[i], g);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = backward<ACT>(k[j], s[j], f[j], g[j]);
        put<PAST == 2>(dxb, byte, Pack<DT, V>::close(f));
    });
}

template <int DT, int V, int K, int ACT, int PAST>
__global__ __launch_bounds__(threads_of(DT, V, K), 4) void k_gn_cols_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                                     const typename Elt<DT>::T* __restrict__ dy, Cols q,
                                                                     int images, Params w,
                                                                     const float* __restrict__ mean,
                                                                     const float* __restrict__ rstd,
                                                                     typename Elt<DT>::T* __restrict__ dx, Sums sums) {
    using P = Pack<DT, V>;
    extern __shared__ float lds[];              // two each: the waves' sums, the channels', the groups'
    Place p;
    if (!place<V>(q, images, p)) return;
    const int all = sum_rows(q) * q.tile;
    float *ch = lds + 2 * all, *ch2 = ch + q.tile, *gr = ch2 + q.tile, *gr2 = gr + q.tile;
    const int count = p.width / q.cg;
    const float m = float(q.cg) * float(q.hw);
    const int64_t at = base_of(q, p);
    const typename Elt<DT>::T *xb = x + at, *gb = dy + at;
    typename P::R d[K], e[K];
    each<DT, K>(q, p, [&](int i, uint32_t byte) {
        d[i] = get<typename P::R, (PAST > 0)>(xb, byte);
        e[i] = get<typename P::R, (PAST > 0)>(gb, byte);
    });
    Coeff k[V];
    coefficients<V>(q, p, w, kept(q, p, mean, rstd), k);
    float a[V], b[V];
    sums_back<DT, V, K, ACT>(d, e, q, p, k, a, b);
    wave_channels<V>(a, q, p.width, lds);
    wave_channels<V>(b, q, p.width, lds + all);
    __syncthreads();
    for (int c = threadIdx.x; c < p.width; c += blockDim.x) {
        const float2 ab = make_float2(sum_of_channel(lds, q, c), sum_of_channel(lds + all, q, c));
        ch[c] = ab.x, ch2[c] = ab.y;
        if (sums.ab) sums.ab[int64_t(p.n) * q.c + p.c0 + c] = ab;
        if (sums.dgamma) sums.dgamma[p.c0 + c] = ab.y;
        if (sums.dbeta) sums.dbeta[p.c0 + c] = ab.x;
    }
    __syncthreads();
    const float* gamma = w.gamma ? w.gamma + p.c0 : nullptr;
    each_group(q, count, ch, gamma, [&](int g, float sum) { gr[g] = sum / m; });
    each_group(q, count, ch2, gamma, [&](int g, float sum) { gr2[g] = sum / m; });
    __syncthreads();
    Back s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int g = p.on ? group_of(q, p.rel + j) : 0;
        s[j] = back_of(k[j], gr[g], gr2[g]);
    }
    write_back<DT, V, K, ACT, PAST>(d, e, q, p, k, s, dx + at);
}

// ---- pieces: some pixels of some channels.

template <int DT, int V, int K>
__global__ __launch_bounds__(256, 4) void k_gn_colparts_fwd(const typename Elt<DT>::T* __restrict__ x, Cols q, int images,
                                                         float4* __restrict__ parts) {
    using P = Pack<DT, V>;
    extern __shared__ float lds[];              // the waves' sums, three, and the channels' means
    Place p;
    if (!place<V>(q, images, p)) return;
    const int all = sum_rows(q) * q.tile;
    float* ch = lds + 3 * all;
    const int64_t at = base_of(q, p);
    const typename Elt<DT>::T* xb = x + at;
    typename P::R d[K];
    each<DT, K>(q, p, [&](int i, uint32_t byte) { d[i] = get<typename P::R, false>(xb, byte); });
    float s[V], mu[V], both[2 * V];             // squares about the mean, and what it lacks
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
    each<DT, K>(q, p, [&](int i, uint32_t) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] += f[j];
    });
    const float num = float(p.last - p.first);
    wave_channels<V>(s, q, p.width, lds);
    __syncthreads();
    for (int c = threadIdx.x; c < p.width; c += blockDim.x) ch[c] = sum_of_channel(lds, q, c) / num;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) {
        mu[j] = p.on ? ch[p.rel + j] : 0.f;
        both[j] = both[V + j] = 0.f;
    }
    each<DT, K>(q, p, [&](int i, uint32_t) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float e = f[j] - mu[j];
            both[j] = fmaf(e, e, both[j]);
            both[V + j] += e;
        }
    });
    wave_channels<V>(both, q, p.width, lds + all);
    __syncthreads();
    for (int c = threadIdx.x; c < p.width; c += blockDim.x)
        parts[(int64_t(p.n) * q.c + p.c0 + c) * q.chunks + p.chunk] =
            make_float4(ch[c], sum_of_channel(lds + all, q, c), num, sum_of_channel(lds + 2 * all, q, c) * __builtin_amdgcn_rcpf(num));
}

// Calls f(group, lane) with a run of q.join_lanes lanes for each of the block's groups.
template <class F> __device__ __forceinline__ void each_joined(const Cols& q, int count, F f) {
    const int lane = int(threadIdx.x) & (q.join_lanes - 1);
    for (int g = int(threadIdx.x) / q.join_lanes; g < count; g += int(blockDim.x) / q.join_lanes) f(g, lane);
}

template <int DT, int V, int K, int ACT, int PAST>
__global__ __launch_bounds__(256, 4) void k_gn_colwrite_fwd(const typename Elt<DT>::T* __restrict__ x, Cols q, int images,
                                                            Params w, float* __restrict__ mean,
                                                            float* __restrict__ rstd,
                                                            const float4* __restrict__ parts, float eps,
                                                            typename Elt<DT>::T* __restrict__ y) {
    using P = Pack<DT, V>;
    extern __shared__ float2 joined[];          // the groups' statistics
    Place p;
    if (!place<V>(q, images, p)) return;
    const int64_t at = base_of(q, p);
    const typename Elt<DT>::T* xb = x + at;
    typename P::R d[K];
    each<DT, K>(q, p, [&](int i, uint32_t byte) { d[i] = get<typename P::R, false>(xb, byte); });
    Coeff k[V];
    if (parts) {
        const int64_t first = int64_t(p.n) * q.c + p.c0, g0 = int64_t(p.n) * q.groups + group_of(q, p.c0);
        each_joined(q, group_of(q, p.width), [&](int g, int lane) {
            const int per = q.cg * q.chunks;
            const float2 ms = joined_stats(parts + (first * q.chunks + int64_t(g) * per), per, lane, q.join_lanes, eps);
            if (lane == 0) {
                joined[g] = ms;
                if (mean && p.chunk == 0) mean[g0 + g] = ms.x, rstd[g0 + g] = ms.y;
            }
        });
        __syncthreads();
        coefficients<V>(q, p, w, [&](int j) { return joined[p.on ? group_of(q, p.rel + j) : 0]; }, k);
    } else {
        coefficients<V>(q, p, w, kept(q, p, mean, rstd), k);
    }
    each<DT, K>(q, p, [&](int i, uint32_t byte) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = forward<ACT>(k[j], f[j]);
        put<PAST == 2>(y + at, byte, P::close(f));
    });
}

template <int DT, int V, int K, int ACT>
__global__ __launch_bounds__(256, 4) void k_gn_colparts_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                         const typename Elt<DT>::T* __restrict__ dy, Cols q, int images,
                                                         Params w, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, float2* __restrict__ parts) {
    using P = Pack<DT, V>;
    extern __shared__ float lds[];              // the waves' sums, two
    Place p;
    if (!place<V>(q, images, p)) return;
    const int all = sum_rows(q) * q.tile;
    const int64_t at = base_of(q, p);
    const typename Elt<DT>::T *xb = x + at, *gb = dy + at;
    typename P::R d[K], e[K];
    each<DT, K>(q, p, [&](int i, uint32_t byte) {
        d[i] = get<typename P::R, false>(xb, byte);
        e[i] = get<typename P::R, false>(gb, byte);
    });
    Coeff k[V];
    coefficients<V>(q, p, w, kept(q, p, mean, rstd), k);
    float a[V], b[V];
    sums_back<DT, V, K, ACT>(d, e, q, p, k, a, b);
    wave_channels<V>(a, q, p.width, lds);
    wave_channels<V>(b, q, p.width, lds + all);
    __syncthreads();
    for (int c = threadIdx.x; c < p.width; c += blockDim.x)
        parts[(int64_t(p.n) * q.c + p.c0 + c) * q.chunks + p.chunk] =
            make_float2(sum_of_channel(lds, q, c), sum_of_channel(lds + all, q, c));
}

template <int DT, int V, int K, int ACT, int PAST>
__global__ __launch_bounds__(256, 4) void k_gn_colwrite_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                         const typename Elt<DT>::T* __restrict__ dy, Cols q, int images,
                                                         Params w, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, const float2* __restrict__ s12,
                                                         const float2* __restrict__ parts, Tail tail,
                                                         typename Elt<DT>::T* __restrict__ dx) {
    using P = Pack<DT, V>;
    extern __shared__ float2 joined[];          // the groups' sums
    if (blockIdx.x >= tail.first) return param_block(tail);
    Place p;
    if (!place<V>(q, images, p)) return;
    const int64_t at = base_of(q, p);
    const typename Elt<DT>::T *xb = x + at, *gb = dy + at;
    typename P::R d[K], e[K];
    each<DT, K>(q, p, [&](int i, uint32_t byte) {
        d[i] = get<typename P::R, false>(xb, byte);
        e[i] = get<typename P::R, false>(gb, byte);
    });
    Coeff k[V];
    coefficients<V>(q, p, w, kept(q, p, mean, rstd), k);
    if (parts) {
        const int64_t first = int64_t(p.n) * q.c + p.c0;
        each_joined(q, group_of(q, p.width), [&](int g, int lane) {
            const int per = q.cg * q.chunks;
            const float2 s = joined_back(parts + (first * q.chunks + int64_t(g) * per), per, q.chunks,
                                         w.gamma ? w.gamma + p.c0 + g * q.cg : nullptr, float(q.cg) * float(q.hw), lane,
                                         q.join_lanes);
            if (lane == 0) joined[g] = s;
        });
        __syncthreads();
    }
    Back s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c = p.on ? p.rel + j : 0;
        const float2 t = parts ? joined[group_of(q, c)] : s12[int64_t(p.n) * q.groups + group_of(q, p.c0 + c)];
        s[j] = back_of(k[j], t.x, t.y);
    }
    write_back<DT, V, K, ACT, PAST>(d, e, q, p, k, s, dx + at);
}

// LDS of a block that joins its groups' pieces.
unsigned joined_lds(const Plan& p) { return p.joined ? unsigned(sizeof(float2)) * unsigned(p.cols.tile / p.cols.cg) : 0u; }

// Calls go with what goes past the caches: 2, stores and what is read once,
// where they fill 64 bytes; in the backward, whose lanes write half as much, the
// stores where they fill 128 (64 x 512 x 28 x 28 fp16 in tiles of 64 bytes:
// nothing 50 us, loads 46, both 49, stores 52).
template <int DT, int V, bool BACK, class F> void with_past(const Cols& q, F go) {
    if constexpr (V > 1) {
        const int bytes = q.tile * int(sizeof(typename Elt<DT>::T));
        if (bytes >= (BACK ? 128 : 64)) return go(IntC<2>{});
        if constexpr (BACK)
            if (bytes >= 64) return go(IntC<1>{});
    }
    go(IntC<0>{});
}

template <int DT, int V>
void fwd(const Plan& p, int n, const void* x, const Params& q, float eps, void* y, float* mean, float* rstd, float4* parts,
         hipStream_t st) {
    using T = typename Elt<DT>::T;
    const T* xt = static_cast<const T*>(x);
    T* yt = static_cast<T*>(y);
    const dim3 grid(static_cast<unsigned>(p.grid)), block(static_cast<unsigned>(p.threads));
    if (!p.held)
        hipLaunchKernelGGL((k_gn_colparts_fwd<DT, V, piece_of(DT, V)>), grid, block, cols_lds(p.cols, p.threads, 3, 1), st, xt,
                           p.cols, n, parts);
    if (!p.held && !p.joined) combine_fwd(parts, int64_t(n) * p.cols.groups, p.cols.cg * p.pieces, eps, mean, rstd, st);
    with_act(q.act, [&](auto act) {
        with_past<DT, V, false>(p.cols, [&](auto past) {
            constexpr int A = decltype(act)::value;
            constexpr int P = decltype(past)::value;
            if (p.held)
                with_count<DT, V, false>(p.k, [&](auto k) {
                    hipLaunchKernelGGL((k_gn_cols_fwd<DT, V, decltype(k)::value, A, P>), grid, block,
                                       cols_lds(p.cols, p.threads, 1, 2), st, xt, p.cols, n, q, eps, yt, mean, rstd);
                });
            else
                hipLaunchKernelGGL((k_gn_colwrite_fwd<DT, V, piece_of(DT, V), A, P>), grid, block, joined_lds(p), st, xt,
                                   p.cols, n, q, mean, rstd, p.joined ? parts : nullptr, eps, yt);
        });
    });
}

template <int DT, int V>
void bwd(const Plan& p, int n, const void* x, const void* dy, const Params& q, const float* mean, const float* rstd,
         void* dx, const Sums& sums, float2* s12, Tail tail, hipStream_t st) {
    using T = typename Elt<DT>::T;
    const T *xt = static_cast<const T*>(x), *gt = static_cast<const T*>(dy);
    T* dt = static_cast<T*>(dx);
    const dim3 grid(static_cast<unsigned>(p.grid)), block(static_cast<unsigned>(p.threads));
    tail.first = grid.x;
    with_act(q.act, [&](auto act) {
        constexpr int A = decltype(act)::value;
        constexpr int K = piece_of(DT, V);
        if (!p.held)
            hipLaunchKernelGGL((k_gn_colparts_bwd<DT, V, K, A>), grid, block, cols_lds(p.cols, p.threads, 2, 0), st, xt, gt,
                               p.cols, n, q, mean, rstd, sums.ab);
        if (!p.held && !p.joined)
            combine_bwd(sums.ab, int64_t(n) * p.cols.groups, p.cols.cg * p.pieces, p.pieces, p.cols.groups, p.cols.cg,
                        float(p.cols.cg) * float(p.cols.hw), q.gamma, s12, st);
        with_past<DT, V, true>(p.cols, [&](auto past) {
            constexpr int P = decltype(past)::value;
            if (p.held)
                with_count<DT, V, true>(p.k, [&](auto k) {
                    hipLaunchKernelGGL((k_gn_cols_bwd<DT, V, decltype(k)::value, A, P>), grid, block,
                                       cols_lds(p.cols, p.threads, 2, 4), st, xt, gt, p.cols, n, q, mean, rstd, dt, sums);
                });
            else
                hipLaunchKernelGGL((k_gn_colwrite_bwd<DT, V, K, A, P>), dim3(grid.x + tail_blocks(tail)), block,
                                   joined_lds(p), st, xt, gt, p.cols, n, q, mean, rstd, s12, p.joined ? sums.ab : nullptr,
                                   tail, dt);
        });
    });
}

}  // namespace

template <int DT>
void cols_fwd(const Plan& p, int n, const void* x, const Params& q, float eps, void* y, float* mean, float* rstd,
              float4* parts, hipStream_t st) {
    constexpr int V = vector_of(DT, false);
    if (p.vec == 0) fwd<DT, 1>(p, n, x, q, eps, y, mean, rstd, parts, st);
    else fwd<DT, V>(p, n, x, q, eps, y, mean, rstd, parts, st);
}
template <int DT>
void cols_bwd(const Plan& p, int n, const void* x, const void* dy, const Params& q, const float* mean, const float* rstd,
              void* dx, const Sums& sums, float2* s12, Tail tail, hipStream_t st) {
    constexpr int V = vector_of(DT, true);
    if (p.vec == 0) bwd<DT, 1>(p, n, x, dy, q, mean, rstd, dx, sums, s12, tail, st);
    else bwd<DT, V>(p, n, x, dy, q, mean, rstd, dx, sums, s12, tail, st);
}

}  // namespace gn
}  // namespace psc
