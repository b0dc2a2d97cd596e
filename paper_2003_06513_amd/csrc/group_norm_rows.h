// Group normalisation in NCHW: a group of an image is cg rows of hw elements
// in one piece.
#pragma once
#include "group_norm.h"

namespace psc {
namespace gn {
namespace {

// Calls f(i, row, window) for the vectors of this thread: slot i, row of the
// group.  base: the group's first element.
template <int V, bool MASK, int K, class F>
__device__ __forceinline__ void each(const Rows& s, int64_t base, F f) {
    const int lanes = 1 << s.lanes_log2;
    const int lane = threadIdx.x & (lanes - 1), rows = int(blockDim.x >> s.lanes_log2);
    int row = int(threadIdx.x >> s.lanes_log2), v = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        if (i < s.slots) {
            if (row < s.cg) {
                const Window w = window<V, MASK>(s, base + int64_t(row) * s.hw, v * lanes + lane);
                if (w.hi > w.lo) f(i, row, w);
            }
            if (++v == s.vi) v = 0, row += rows;
        }
    }
}

template <int DT, int V, bool MASK, int K>
__global__ __launch_bounds__(K <= 4 ? 1024 : 512) void k_gn_rows_fwd(const typename Elt<DT>::T* __restrict__ x, Rows s,
                                                                     Params q, float eps,
                                                                     typename Elt<DT>::T* __restrict__ y,
                                                                     float* __restrict__ mean, float* __restrict__ rstd) {
    using P = Pack<DT, V>;
    __shared__ float part[16];
    const int64_t ng = blockIdx.x, base = ng * s.cg * s.hw;
    const int c0 = int(ng % s.groups) * s.cg;
    typename P::R d[K];
    each<V, MASK, K>(s, base, [&](int i, int, const Window& w) { d[i] = load<DT, V, MASK>(x, w, s.total); });
    float sum = 0.f;
    each<V, MASK, K>(s, base, [&](int i, int, const Window& w) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) sum += in<MASK>(w, j) ? f[j] : 0.f;
    });
    const float m = float(s.cg) * float(s.hw);
    const float mu = block_sum(sum, part) / m;
    float sq = 0.f;
    each<V, MASK, K>(s, base, [&](int i, int, const Window& w) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float e = in<MASK>(w, j) ? f[j] - mu : 0.f;
            sq = fmaf(e, e, sq);
        }
    });
    const float r = 1.f / sqrtf(block_sum(sq, part) / m + eps);
    if (threadIdx.x == 0 && mean) {
        mean[ng] = mu;
        rstd[ng] = r;
    }
    each<V, MASK, K>(s, base, [&](int i, int row, const Window& w) {
        const float ga = or_one(q.gamma, c0 + row), be = or_zero(q.beta, c0 + row);
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = act_of(affine((f[j] - mu) * r, ga, be), q.act);
        store<DT, V, MASK>(y, w, f);
    });
}

// sums [n][c]: A and B of each row, for the parameters' gradients; may be NULL.
template <int DT, int V, bool MASK, int K>
__global__ __launch_bounds__(K <= 4 ? 1024 : 512) void k_gn_rows_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                                     const typename Elt<DT>::T* __restrict__ dy, Rows s,
                                                                     Params q, const float* __restrict__ mean,
                                                                     const float* __restrict__ rstd,
                                                                     typename Elt<DT>::T* __restrict__ dx,
                                                                     float2* __restrict__ sums) {
    using P = Pack<DT, V>;
    extern __shared__ float2 row_parts[];       // [cg][waves that share a row]
    __shared__ float part[16];
    const int64_t ng = blockIdx.x, base = ng * s.cg * s.hw;
    const int c0 = int(ng % s.groups) * s.cg;
    const float mu = mean[ng], r = rstd[ng];
    typename P::R d[K], e[K];
    each<V, MASK, K>(s, base, [&](int i, int, const Window& w) {
        d[i] = load<DT, V, MASK>(x, w, s.total);
        e[i] = load<DT, V, MASK>(dy, w, s.total);
    });
    const int lanes = 1 << s.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int share = lanes > 64 ? lanes >> 6 : 1;
    {
        const int rows = int(blockDim.x >> s.lanes_log2);
        int row = int(threadIdx.x >> s.lanes_log2), v = 0;
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            if (i < s.slots) {
                if (row < s.cg) {
                    const Window w = window<V, MASK>(s, base + int64_t(row) * s.hw, v * lanes + lane);
                    if (w.hi > w.lo) {
                        const float ga = or_one(q.gamma, c0 + row), be = or_zero(q.beta, c0 + row);
                        float f[V], g[V];
                        P::open(d[i], f);
                        P::open(e[i], g);
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            const float xh = (f[j] - mu) * r;
                            const float du = in<MASK>(w, j) ? act_back(affine(xh, ga, be), g[j], q.act) : 0.f;
                            a += du;
                            b = in<MASK>(w, j) ? fmaf(du, xh, b) : b;
                        }
                    }
                }
                if (++v == s.vi) {
                    for (int off = 1; off < lanes && off < 64; off <<= 1) {
                        a += __shfl_xor(a, off);
                        b += __shfl_xor(b, off);
                    }
                    if (row < s.cg && (lane & 63) == 0) row_parts[row * share + (lane >> 6)] = make_float2(a, b);
                    a = 0.f, b = 0.f;
                    v = 0, row += rows;
                }
            }
        }
    }
    __syncthreads();
    float s1 = 0.f, s2 = 0.f;
    for (int row = threadIdx.x; row < s.cg; row += blockDim.x) {
        float a = 0.f, b = 0.f;
        for (int i = 0; i < share; ++i) {
            const float2 ab = row_parts[row * share + i];
            a += ab.x;
            b += ab.y;
        }
        if (sums) sums[ng * s.cg + row] = make_float2(a, b);
        const float ga = or_one(q.gamma, c0 + row);
        s1 = fmaf(ga, a, s1);
        s2 = fmaf(ga, b, s2);
    }
    const float m = float(s.cg) * float(s.hw);
    s1 = block_sum(s1, part) / m;
    s2 = block_sum(s2, part) / m;
    each<V, MASK, K>(s, base, [&](int i, int row, const Window& w) {
        const float ga = or_one(q.gamma, c0 + row), be = or_zero(q.beta, c0 + row);
        float f[V], g[V];
        P::open(d[i], f);
        P::open(e[i], g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = (f[j] - mu) * r;
            const float du = act_back(affine(xh, ga, be), g[j], q.act);
            f[j] = r * (fmaf(ga, du, -s1) - xh * s2);
        }
        store<DT, V, MASK>(dx, w, f);
    });
}

// ---- pieces: a wave takes K x 64 vectors of a row.

template <int V, bool MASK, int K, class F>
__device__ __forceinline__ void each_of_piece(const Rows& s, int64_t at, int piece, F f) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const Window w = window<V, MASK>(s, at, (piece * K + i) * 64 + lane);
        if (w.hi > w.lo) f(i, w);
    }
}

// The number of elements, their mean and their squares about it.
template <int DT, int V, bool MASK, int K>
__global__ __launch_bounds__(256) void k_gn_rowparts_fwd(const typename Elt<DT>::T* __restrict__ x, Rows s, int pieces,
                                                         int64_t count, float4* __restrict__ parts) {
    using P = Pack<DT, V>;
    const int64_t id = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (id >= count) return;
    const int64_t at = id / pieces * s.hw;
    const int piece = int(id % pieces);
    typename P::R d[K];
    each_of_piece<V, MASK, K>(s, at, piece, [&](int i, const Window& w) { d[i] = load<DT, V, MASK>(x, w, s.total); });
    float sum = 0.f, num = 0.f;
    each_of_piece<V, MASK, K>(s, at, piece, [&](int i, const Window& w) {
        float f[V];
        P::open(d[i], f);
        num += float(w.hi - w.lo);
#pragma unroll
        for (int j = 0; j < V; ++j) sum += in<MASK>(w, j) ? f[j] : 0.f;
    });
    num = wave_sum(num);
    const float mu = num > 0.f ? wave_sum(sum) / num : 0.f;
    float sq = 0.f;
    each_of_piece<V, MASK, K>(s, at, piece, [&](int i, const Window& w) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float e = in<MASK>(w, j) ? f[j] - mu : 0.f;
            sq = fmaf(e, e, sq);
        }
    });
    sq = wave_sum(sq);
    if ((threadIdx.x & 63) == 0) parts[id] = make_float4(mu, sq, num, 0.f);
}

template <int DT, int V, bool MASK, int K>
__global__ __launch_bounds__(256) void k_gn_rowwrite_fwd(const typename Elt<DT>::T* __restrict__ x, Rows s, Params q,
                                                         int pieces, int64_t count, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd,
                                                         typename Elt<DT>::T* __restrict__ y) {
    using P = Pack<DT, V>;
    const int64_t id = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (id >= count) return;
    const int64_t row = id / pieces, at = row * s.hw;
    const int piece = int(id % pieces);
    const int64_t ng = row / s.cg;
    const int c = int(row % (int64_t(s.cg) * s.groups));
    typename P::R d[K];
    each_of_piece<V, MASK, K>(s, at, piece, [&](int i, const Window& w) { d[i] = load<DT, V, MASK>(x, w, s.total); });
    const float mu = mean[ng], r = rstd[ng], ga = or_one(q.gamma, c), be = or_zero(q.beta, c);
    each_of_piece<V, MASK, K>(s, at, piece, [&](int i, const Window& w) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = act_of(affine((f[j] - mu) * r, ga, be), q.act);
        store<DT, V, MASK>(y, w, f);
    });
}

template <int DT, int V, bool MASK, int K>
__global__ __launch_bounds__(256) void k_gn_rowparts_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                         const typename Elt<DT>::T* __restrict__ dy, Rows s, Params q,
                                                         int pieces, int64_t count, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, float2* __restrict__ parts) {
    using P = Pack<DT, V>;
    const int64_t id = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (id >= count) return;
    const int64_t row = id / pieces, at = row * s.hw;
    const int piece = int(id % pieces);
    const int64_t ng = row / s.cg;
    const int c = int(row % (int64_t(s.cg) * s.groups));
    typename P::R d[K], e[K];
    each_of_piece<V, MASK, K>(s, at, piece, [&](int i, const Window& w) {
        d[i] = load<DT, V, MASK>(x, w, s.total);
        e[i] = load<DT, V, MASK>(dy, w, s.total);
    });
    const float mu = mean[ng], r = rstd[ng], ga = or_one(q.gamma, c), be = or_zero(q.beta, c);
    float a = 0.f, b = 0.f;
    each_of_piece<V, MASK, K>(s, at, piece, [&](int i, const Window& w) {
        float f[V], g[V];
        P::open(d[i], f);
        P::open(e[i], g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = (f[j] - mu) * r;
            const float du = in<MASK>(w, j) ? act_back(affine(xh, ga, be), g[j], q.act) : 0.f;
            a += du;
            b = in<MASK>(w, j) ? fmaf(du, xh, b) : b;
        }
    });
    a = wave_sum(a);
    b = wave_sum(b);
    if ((threadIdx.x & 63) == 0) parts[id] = make_float2(a, b);
}

template <int DT, int V, bool MASK, int K>
__global__ __launch_bounds__(256) void k_gn_rowwrite_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                         const typename Elt<DT>::T* __restrict__ dy, Rows s, Params q,
                                                         int pieces, int64_t count, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, const float2* __restrict__ s12,
                                                         typename Elt<DT>::T* __restrict__ dx) {
    using P = Pack<DT, V>;
    const int64_t id = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (id >= count) return;
    const int64_t row = id / pieces, at = row * s.hw;
    const int piece = int(id % pieces);
    const int64_t ng = row / s.cg;
    const int c = int(row % (int64_t(s.cg) * s.groups));
    typename P::R d[K], e[K];
    each_of_piece<V, MASK, K>(s, at, piece, [&](int i, const Window& w) {
        d[i] = load<DT, V, MASK>(x, w, s.total);
        e[i] = load<DT, V, MASK>(dy, w, s.total);
    });
    const float mu = mean[ng], r = rstd[ng], ga = or_one(q.gamma, c), be = or_zero(q.beta, c);
    const float2 sum = s12[ng];
    each_of_piece<V, MASK, K>(s, at, piece, [&](int i, const Window& w) {
        float f[V], g[V];
        P::open(d[i], f);
        P::open(e[i], g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = (f[j] - mu) * r;
            const float du = act_back(affine(xh, ga, be), g[j], q.act);
            f[j] = r * (fmaf(ga, du, -sum.x) - xh * sum.y);
        }
        store<DT, V, MASK>(dx, w, f);
    });
}

template <int DT, int V, bool MASK>
void fwd(const Plan& p, int64_t count, const void* x, const Params& q, float eps, void* y, float* mean, float* rstd,
         float4* parts, hipStream_t st) {
    using T = typename Elt<DT>::T;
    const T* xt = static_cast<const T*>(x);
    T* yt = static_cast<T*>(y);
    if (p.held) {
        const dim3 grid(static_cast<unsigned>(p.grid)), block(static_cast<unsigned>(p.threads));
        const auto go = [&](auto k) {
            hipLaunchKernelGGL((k_gn_rows_fwd<DT, V, MASK, decltype(k)::value>), grid, block, 0, st, xt, p.rows, q, eps, yt,
                               mean, rstd);
        };
        if (p.k <= 2) go(IntC<2>{});
        else if (p.k <= 4) go(IntC<4>{});
        else if (p.k <= 8) go(IntC<8>{});
        else go(IntC<16>{});
        return;
    }
    constexpr int K = V == 1 ? kPieceSingle : kPiece;
    const dim3 grid(static_cast<unsigned>((count + 3) / 4));
    hipLaunchKernelGGL((k_gn_rowparts_fwd<DT, V, MASK, K>), grid, dim3(256), 0, st, xt, p.rows, p.pieces, count, parts);
    combine_fwd(parts, count / (int64_t(p.rows.cg) * p.pieces), p.rows.cg * p.pieces, eps, mean, rstd, st);
    hipLaunchKernelGGL((k_gn_rowwrite_fwd<DT, V, MASK, K>), grid, dim3(256), 0, st, xt, p.rows, q, p.pieces, count, mean,
                       rstd, yt);
}

template <int DT, int V, bool MASK>
void bwd(const Plan& p, int64_t count, const void* x, const void* dy, const Params& q, const float* mean,
         const float* rstd, void* dx, float2* parts, float2* s12, hipStream_t st) {
    using T = typename Elt<DT>::T;
    const T *xt = static_cast<const T*>(x), *gt = static_cast<const T*>(dy);
    T* dt = static_cast<T*>(dx);
    if (p.held) {
        const dim3 grid(static_cast<unsigned>(p.grid)), block(static_cast<unsigned>(p.threads));
        const int lanes = 1 << p.rows.lanes_log2;
        const unsigned lds = unsigned(sizeof(float2)) * unsigned(p.rows.cg) * unsigned(lanes > 64 ? lanes / 64 : 1);
        const auto go = [&](auto k) {
            hipLaunchKernelGGL((k_gn_rows_bwd<DT, V, MASK, decltype(k)::value>), grid, block, lds, st, xt, gt, p.rows, q,
                               mean, rstd, dt, parts);
        };
        if (p.k <= 2) go(IntC<2>{});
        else if (p.k <= 4) go(IntC<4>{});
        else go(IntC<8>{});
        return;
    }
    constexpr int K = V == 1 ? kPieceSingle : kPiece;
    const dim3 grid(static_cast<unsigned>((count + 3) / 4));
    hipLaunchKernelGGL((k_gn_rowparts_bwd<DT, V, MASK, K>), grid, dim3(256), 0, st, xt, gt, p.rows, q, p.pieces, count,
                       mean, rstd, parts);
    const float m = float(p.rows.cg) * float(p.rows.hw);
    combine_bwd(parts, count / (int64_t(p.rows.cg) * p.pieces), p.rows.cg * p.pieces, p.pieces, p.rows.groups, p.rows.cg,
                m, q.gamma, s12, st);
    hipLaunchKernelGGL((k_gn_rowwrite_bwd<DT, V, MASK, K>), grid, dim3(256), 0, st, xt, gt, p.rows, q, p.pieces, count,
                       mean, rstd, s12, dt);
}

}  // namespace

template <int DT>
void rows_fwd(const Plan& p, int64_t count, const void* x, const Params& q, float eps, void* y, float* mean, float* rstd,
              float4* parts, hipStream_t st) {
    constexpr int V = DT == DT_F16 ? 8 : 4;
    if (p.vec == 0) fwd<DT, 1, false>(p, count, x, q, eps, y, mean, rstd, parts, st);
    else if (p.vec == 1) fwd<DT, V, false>(p, count, x, q, eps, y, mean, rstd, parts, st);
    else fwd<DT, V, true>(p, count, x, q, eps, y, mean, rstd, parts, st);
}
template <int DT>
void rows_bwd(const Plan& p, int64_t count, const void* x, const void* dy, const Params& q, const float* mean,
              const float* rstd, void* dx, float2* parts, float2* s12, hipStream_t st) {
    constexpr int V = DT == DT_F16 ? 8 : 4;
    if (p.vec == 0) bwd<DT, 1, false>(p, count, x, dy, q, mean, rstd, dx, parts, s12, st);
    else if (p.vec == 1) bwd<DT, V, false>(p, count, x, dy, q, mean, rstd, dx, parts, s12, st);
    else bwd<DT, V, true>(p, count, x, dy, q, mean, rstd, dx, parts, s12, st);
}

}  // namespace gn
}  // namespace psc
