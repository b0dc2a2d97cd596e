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
// Blocks that are eight apart run on the same compute die, whose cache their
// neighbouring channels share: the tiles of an image are eight apart.
template <int V>
__device__ __forceinline__ bool place(const Cols& q, int images, Place& p) {
    const int per = 8 * q.tiles * q.chunks;
    const int b = int(blockIdx.x);
    const int in = b % per;
    p.n = b / per * 8 + (in & 7);
    if (p.n >= images) return false;
    const int rest = in >> 3;
    p.chunk = rest / q.tiles;
    p.c0 = rest % q.tiles * q.tile;
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
// Calls f(i, at) for the vectors of this thread: slot i, which begins at element `at`.
template <int K, class F>
__device__ __forceinline__ void each(const Cols& q, const Place& p, F f) {
    if (!p.on) return;
    const int64_t at = int64_t(p.n) * q.hw * q.c + p.c0 + p.rel;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const int px = p.first + i * p.rows + p.row;
        if (px < p.last) f(i, at + int64_t(px) * q.c);
    }
}
template <int DT, int V>
__device__ __forceinline__ typename Pack<DT, V>::R get(const typename Elt<DT>::T* p, int64_t at) {
    return *reinterpret_cast<const typename Pack<DT, V>::R*>(p + at);
}
template <int DT, int V>
__device__ __forceinline__ void put(typename Elt<DT>::T* p, int64_t at, const float (&f)[V]) {
    *reinterpret_cast<typename Pack<DT, V>::R*>(p + at) = Pack<DT, V>::close(f);
}

// LDS of a block: the threads' sums, the channels', the groups' (two of each).
__device__ __forceinline__ float* lds_of_channels(float* lds, const Cols& q) {
    const int span_log2 = q.cols_log2 > 6 ? q.cols_log2 : 6;
    return lds + (blockDim.x >> span_log2) * q.tile;
}

template <int DT, int V, int K>
__global__ __launch_bounds__(K <= 4 ? 1024 : 512) void k_gn_cols_fwd(const typename Elt<DT>::T* __restrict__ x, Cols q,
                                                                     int images, Params w, float eps,
                                                                     typename Elt<DT>::T* __restrict__ y,
                                                                     float* __restrict__ mean, float* __restrict__ rstd) {
    using P = Pack<DT, V>;
    extern __shared__ float lds[];
    Place p;
    if (!place<V>(q, images, p)) return;
    float* ch = lds_of_channels(lds, q);
    float* gr = ch + q.tile;
    const int count = p.width / q.cg;
    const float m = float(q.cg) * float(q.hw);
    typename P::R d[K];
    each<K>(q, p, [&](int i, int64_t at) { d[i] = get<DT, V>(x, at); });
    float s[V], mu[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
    each<K>(q, p, [&](int i, int64_t) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] += f[j];
    });
    channel_sums<V>(s, q, p.width, lds, ch);
    group_sums(ch, nullptr, q.cg, count, gr);
    int g[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        g[j] = p.on ? (p.rel + j) / q.cg : 0;
        mu[j] = gr[g[j]] / m;
        s[j] = 0.f;
    }
    const int64_t g0 = int64_t(p.n) * q.groups + p.c0 / q.cg;
    if (mean)
        for (int k = threadIdx.x; k < count; k += blockDim.x) mean[g0 + k] = gr[k] / m;
    each<K>(q, p, [&](int i, int64_t) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float e = f[j] - mu[j];
            s[j] = fmaf(e, e, s[j]);
        }
    });
    channel_sums<V>(s, q, p.width, lds, ch);
    group_sums(ch, nullptr, q.cg, count, gr);
    float r[V], ga[V], be[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        r[j] = 1.f / sqrtf(gr[g[j]] / m + eps);
        ga[j] = p.on ? or_one(w.gamma, p.c0 + p.rel + j) : 1.f;
        be[j] = p.on ? or_zero(w.beta, p.c0 + p.rel + j) : 0.f;
    }
    if (rstd)
        for (int k = threadIdx.x; k < count; k += blockDim.x) rstd[g0 + k] = 1.f / sqrtf(gr[k] / m + eps);
    each<K>(q, p, [&](int i, int64_t at) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = act_of(affine((f[j] - mu[j]) * r[j], ga[j], be[j]), w.act);
        put<DT, V>(y, at, f);
    });
}

template <int V>
struct Coeff {
    float mu[V], r[V], ga[V], be[V];
};
template <int V>
__device__ __forceinline__ void coefficients(const Cols& q, const Place& p, const Params& w, const float* mean,
                                             const float* rstd, Coeff<V>& k) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c = p.on ? p.c0 + p.rel + j : 0;
        const int64_t g = int64_t(p.n) * q.groups + c / q.cg;
        k.mu[j] = mean[g];
        k.r[j] = rstd[g];
        k.ga[j] = or_one(w.gamma, c);
        k.be[j] = or_zero(w.beta, c);
    }
}

template <int DT, int V, int K>
__device__ __forceinline__ void sums_back(const typename Pack<DT, V>::R (&d)[K], const typename Pack<DT, V>::R (&e)[K],
                                          const Cols& q, const Place& p, const Coeff<V>& k, int act, float (&a)[V],
                                          float (&b)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] = 0.f, b[j] = 0.f;
    each<K>(q, p, [&](int i, int64_t) {
        float f[V], g[V];
        Pack<DT, V>::open(d[i], f);
        Pack<DT, V>::open(e[i], g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = (f[j] - k.mu[j]) * k.r[j];
            const float du = act_back(affine(xh, k.ga[j], k.be[j]), g[j], act);
            a[j] += du;
            b[j] = fmaf(du, xh, b[j]);
        }
    });
}
template <int DT, int V, int K>
__device__ __forceinline__ void write_back(const typename Pack<DT, V>::R (&d)[K], const typename Pack<DT, V>::R (&e)[K],
                                           const Cols& q, const Place& p, const Coeff<V>& k, int act,
                                           const float (&s1)[V], const float (&s2)[V], typename Elt<DT>::T* dx) {
    each<K>(q, p, [&](int i, int64_t at) {
        float f[V], g[V];
        Pack<DT, V>::open(d[i], f);
        Pack<DT, V>::open(e[i], g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = (f[j] - k.mu[j]) * k.r[j];
            const float du = act_back(affine(xh, k.ga[j], k.be[j]), g[j], act);
            f[j] = k.r[j] * (fmaf(k.ga[j], du, -s1[j]) - xh * s2[j]);
        }
        put<DT, V>(dx, at, f);
    });
}

template <int DT, int V, int K>
__global__ __launch_bounds__(K <= 4 ? 1024 : 512) void k_gn_cols_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                                     const typename Elt<DT>::T* __restrict__ dy, Cols q,
                                                                     int images, Params w,
                                                                     const float* __restrict__ mean,
                                                                     const float* __restrict__ rstd,
                                                                     typename Elt<DT>::T* __restrict__ dx,
                                                                     float2* __restrict__ sums) {
    using P = Pack<DT, V>;
    extern __shared__ float lds[];
    Place p;
    if (!place<V>(q, images, p)) return;
    float* ch = lds_of_channels(lds, q);
    float* ch2 = ch + q.tile;
    float* gr = ch2 + q.tile;
    float* gr2 = gr + q.tile;
    const int count = p.width / q.cg;
    const float m = float(q.cg) * float(q.hw);
    typename P::R d[K], e[K];
    each<K>(q, p, [&](int i, int64_t at) {
        d[i] = get<DT, V>(x, at);
        e[i] = get<DT, V>(dy, at);
    });
    Coeff<V> k;
    coefficients<V>(q, p, w, mean, rstd, k);
    float a[V], b[V];
    sums_back<DT, V, K>(d, e, q, p, k, w.act, a, b);
    channel_sums<V>(a, q, p.width, lds, ch);
    channel_sums<V>(b, q, p.width, lds, ch2);
    if (sums)
        for (int c = threadIdx.x; c < p.width; c += blockDim.x)
            sums[int64_t(p.n) * q.c + p.c0 + c] = make_float2(ch[c], ch2[c]);
    const float* gamma = w.gamma ? w.gamma + p.c0 : nullptr;
    group_sums(ch, gamma, q.cg, count, gr);
    group_sums(ch2, gamma, q.cg, count, gr2);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int g = p.on ? (p.rel + j) / q.cg : 0;
        a[j] = gr[g] / m;
        b[j] = gr2[g] / m;
    }
    write_back<DT, V, K>(d, e, q, p, k, w.act, a, b, dx);
}

// ---- pieces: some pixels of some channels.

template <int DT, int V, int K>
__global__ __launch_bounds__(256) void k_gn_colparts_fwd(const typename Elt<DT>::T* __restrict__ x, Cols q, int images,
                                                         float4* __restrict__ parts) {
    using P = Pack<DT, V>;
    extern __shared__ float lds[];
    Place p;
    if (!place<V>(q, images, p)) return;
    float* ch = lds_of_channels(lds, q);
    float* ch2 = ch + q.tile;
    typename P::R d[K];
    each<K>(q, p, [&](int i, int64_t at) { d[i] = get<DT, V>(x, at); });
    float s[V], mu[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
    each<K>(q, p, [&](int i, int64_t) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] += f[j];
    });
    const float num = float(p.last - p.first);
    channel_sums<V>(s, q, p.width, lds, ch);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        mu[j] = p.on ? ch[p.rel + j] / num : 0.f;
        s[j] = 0.f;
    }
    each<K>(q, p, [&](int i, int64_t) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float e = f[j] - mu[j];
            s[j] = fmaf(e, e, s[j]);
        }
    });
    channel_sums<V>(s, q, p.width, lds, ch2);
    for (int c = threadIdx.x; c < p.width; c += blockDim.x)
        parts[(int64_t(p.n) * q.c + p.c0 + c) * q.chunks + p.chunk] = make_float4(ch[c] / num, ch2[c], num, 0.f);
}

template <int DT, int V, int K>
__global__ __launch_bounds__(256) void k_gn_colwrite_fwd(const typename Elt<DT>::T* __restrict__ x, Cols q, int images,
                                                         Params w, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd,
                                                         typename Elt<DT>::T* __restrict__ y) {
    using P = Pack<DT, V>;
    Place p;
    if (!place<V>(q, images, p)) return;
    typename P::R d[K];
    each<K>(q, p, [&](int i, int64_t at) { d[i] = get<DT, V>(x, at); });
    Coeff<V> k;
    coefficients<V>(q, p, w, mean, rstd, k);
    each<K>(q, p, [&](int i, int64_t at) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = act_of(affine((f[j] - k.mu[j]) * k.r[j], k.ga[j], k.be[j]), w.act);
        put<DT, V>(y, at, f);
    });
}

template <int DT, int V, int K>
__global__ __launch_bounds__(256) void k_gn_colparts_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                         const typename Elt<DT>::T* __restrict__ dy, Cols q, int images,
                                                         Params w, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, float2* __restrict__ parts) {
    using P = Pack<DT, V>;
    extern __shared__ float lds[];
    Place p;
    if (!place<V>(q, images, p)) return;
    float* ch = lds_of_channels(lds, q);
    float* ch2 = ch + q.tile;
    typename P::R d[K], e[K];
    each<K>(q, p, [&](int i, int64_t at) {
        d[i] = get<DT, V>(x, at);
        e[i] = get<DT, V>(dy, at);
    });
    Coeff<V> k;
    coefficients<V>(q, p, w, mean, rstd, k);
    float a[V], b[V];
    sums_back<DT, V, K>(d, e, q, p, k, w.act, a, b);
    channel_sums<V>(a, q, p.width, lds, ch);
    channel_sums<V>(b, q, p.width, lds, ch2);
    for (int c = threadIdx.x; c < p.width; c += blockDim.x)
        parts[(int64_t(p.n) * q.c + p.c0 + c) * q.chunks + p.chunk] = make_float2(ch[c], ch2[c]);
}

template <int DT, int V, int K>
__global__ __launch_bounds__(256) void k_gn_colwrite_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                         const typename Elt<DT>::T* __restrict__ dy, Cols q, int images,
                                                         Params w, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, const float2* __restrict__ s12,
                                                         typename Elt<DT>::T* __restrict__ dx) {
    using P = Pack<DT, V>;
    Place p;
    if (!place<V>(q, images, p)) return;
    typename P::R d[K], e[K];
    each<K>(q, p, [&](int i, int64_t at) {
        d[i] = get<DT, V>(x, at);
        e[i] = get<DT, V>(dy, at);
    });
    Coeff<V> k;
    coefficients<V>(q, p, w, mean, rstd, k);
    float s1[V], s2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c = p.on ? p.c0 + p.rel + j : 0;
        const float2 t = s12[int64_t(p.n) * q.groups + c / q.cg];
        s1[j] = t.x, s2[j] = t.y;
    }
    write_back<DT, V, K>(d, e, q, p, k, w.act, s1, s2, dx);
}

// Bytes of LDS: `more` arrays of the tile's width behind the threads' sums.
unsigned lds_bytes(const Plan& p, int more) {
    const int span_log2 = p.cols.cols_log2 > 6 ? p.cols.cols_log2 : 6;
    return unsigned(sizeof(float)) * unsigned(p.cols.tile) * unsigned((p.threads >> span_log2) + more);
}

template <int DT, int V>
void fwd(const Plan& p, int n, const void* x, const Params& q, float eps, void* y, float* mean, float* rstd, float4* parts,
         hipStream_t st) {
    using T = typename Elt<DT>::T;
    const T* xt = static_cast<const T*>(x);
    T* yt = static_cast<T*>(y);
    const dim3 grid(static_cast<unsigned>(p.grid)), block(static_cast<unsigned>(p.threads));
    if (p.held) {
        const auto go = [&](auto k) {
            hipLaunchKernelGGL((k_gn_cols_fwd<DT, V, decltype(k)::value>), grid, block, lds_bytes(p, 2), st, xt, p.cols, n,
                               q, eps, yt, mean, rstd);
        };
        if (p.k <= 2) go(IntC<2>{});
        else if (p.k <= 4) go(IntC<4>{});
        else if (p.k <= 8) go(IntC<8>{});
        else go(IntC<16>{});
        return;
    }
    constexpr int K = V == 1 ? kPieceSingle : kPiece;
    hipLaunchKernelGGL((k_gn_colparts_fwd<DT, V, K>), grid, block, lds_bytes(p, 2), st, xt, p.cols, n, parts);
    combine_fwd(parts, int64_t(n) * p.cols.groups, p.cols.cg * p.pieces, eps, mean, rstd, st);
    hipLaunchKernelGGL((k_gn_colwrite_fwd<DT, V, K>), grid, block, 0, st, xt, p.cols, n, q, mean, rstd, yt);
}

template <int DT, int V>
void bwd(const Plan& p, int n, const void* x, const void* dy, const Params& q, const float* mean, const float* rstd,
         void* dx, float2* parts, float2* s12, hipStream_t st) {
    using T = typename Elt<DT>::T;
    const T *xt = static_cast<const T*>(x), *gt = static_cast<const T*>(dy);
    T* dt = static_cast<T*>(dx);
    const dim3 grid(static_cast<unsigned>(p.grid)), block(static_cast<unsigned>(p.threads));
    if (p.held) {
        const auto go = [&](auto k) {
            hipLaunchKernelGGL((k_gn_cols_bwd<DT, V, decltype(k)::value>), grid, block, lds_bytes(p, 4), st, xt, gt, p.cols,
                               n, q, mean, rstd, dt, parts);
        };
        if (p.k <= 2) go(IntC<2>{});
        else if (p.k <= 4) go(IntC<4>{});
        else go(IntC<8>{});
        return;
    }
    constexpr int K = V == 1 ? kPieceSingle : kPiece;
    hipLaunchKernelGGL((k_gn_colparts_bwd<DT, V, K>), grid, block, lds_bytes(p, 2), st, xt, gt, p.cols, n, q, mean, rstd,
                       parts);
    combine_bwd(parts, int64_t(n) * p.cols.groups, p.cols.cg * p.pieces, p.pieces, p.cols.groups, p.cols.cg,
                float(p.cols.cg) * float(p.cols.hw), q.gamma, s12, st);
    hipLaunchKernelGGL((k_gn_colwrite_bwd<DT, V, K>), grid, block, 0, st, xt, gt, p.cols, n, q, mean, rstd, s12, dt);
}

}  // namespace

template <int DT>
void cols_fwd(const Plan& p, int n, const void* x, const Params& q, float eps, void* y, float* mean, float* rstd,
              float4* parts, hipStream_t st) {
    constexpr int V = DT == DT_F16 ? 8 : 4;
    if (p.vec == 0) fwd<DT, 1>(p, n, x, q, eps, y, mean, rstd, parts, st);
    else fwd<DT, V>(p, n, x, q, eps, y, mean, rstd, parts, st);
}
template <int DT>
void cols_bwd(const Plan& p, int n, const void* x, const void* dy, const Params& q, const float* mean, const float* rstd,
              void* dx, float2* parts, float2* s12, hipStream_t st) {
    constexpr int V = DT == DT_F16 ? 8 : 4;
    if (p.vec == 0) bwd<DT, 1>(p, n, x, dy, q, mean, rstd, dx, parts, s12, st);
    else bwd<DT, V>(p, n, x, dy, q, mean, rstd, dx, parts, s12, st);
}

}  // namespace gn
}  // namespace psc
