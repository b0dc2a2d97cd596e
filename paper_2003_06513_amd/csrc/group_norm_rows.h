// Group normalisation in NCHW: a group of an image is cg rows of hw elements
// in one piece.
#pragma once
#include "group_norm.h"

namespace psc {
namespace gn {
namespace {

// Calls f(i, row, window, on) for the vectors of this thread: slot i, row of
// the group, and after(row) where the thread has done with a row.  Where a
// slot has nothing (not on) it is given the group's first vector: branches
// around every slot cost more than a load that all such lanes share (compiled
// with them, the kernels of pieces took 400 registers).
template <int V, bool MASK, int K, class F, class G>
__device__ __forceinline__ void each(const Rows& s, const Base<V, MASK>& b, F f, G after) {
    const int lanes = 1 << s.lanes_log2;
    const int lane = int(threadIdx.x) & (lanes - 1), rows = int(blockDim.x >> s.lanes_log2);
    int row = int(threadIdx.x >> s.lanes_log2), v = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        if (i < s.slots) {
            const int k = v * lanes + lane;
            const bool on = row < s.cg && has<V, MASK>(b, row * s.hw, s.hw, k);
            const int r = on ? row : 0;
            f(i, r, window<V, MASK>(b, r * s.hw, s.hw, on ? k : 0), on);
            if (++v == s.vi) {
                after(row);
                v = 0, row += rows;
            }
        }
    }
}
struct Nothing {
    __device__ __forceinline__ void operator()(int) const {}
};

template <int DT, int V, bool MASK, int K, int ACT>
__global__ __launch_bounds__(threads_of(DT, V, K)) void k_gn_rows_fwd(const typename Elt<DT>::T* __restrict__ x, Rows s,
                                                                  Params q, float eps,
                                                                  typename Elt<DT>::T* __restrict__ y,
                                                                  float* __restrict__ mean, float* __restrict__ rstd) {
    using P = Pack<DT, V>;
    __shared__ float part[32];
    extern __shared__ float2 row_params[];      // gamma and beta of the rows
    const Base<V, MASK> b(s, int64_t(blockIdx.x) * s.cg * s.hw);
    const int c0 = int(blockIdx.x % unsigned(s.groups)) * s.cg;
    typename P::R d[K];
    each<V, MASK, K>(s, b, [&](int i, int, const Window& w, bool) { d[i] = load<DT, V, MASK, true>(x, b, w); }, Nothing());
    for (int row = threadIdx.x; row < s.cg; row += blockDim.x)
        row_params[row] = make_float2(or_one(q.gamma, c0 + row), or_zero(q.beta, c0 + row));
    float sum = 0.f;
    each<V, MASK, K>(s, b, [&](int i, int, const Window& w, bool on) {
        float f[V], t = 0.f;
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) t += in<MASK>(w, j) ? f[j] : 0.f;
        sum += on ? t : 0.f;
    }, Nothing());
    const float m = float(s.cg) * float(s.hw);
    Coeff k;
    k.mu = block_sum(sum, part) / m;
    float sq = 0.f;
    each<V, MASK, K>(s, b, [&](int i, int, const Window& w, bool on) {
        float f[V], t = 0.f;
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float e = in<MASK>(w, j) ? f[j] - k.mu : 0.f;
            t = fmaf(e, e, t);
        }
        sq += on ? t : 0.f;
    }, Nothing());
    const float2 ms = stats_of(k.mu, block_sum(sq, part + 16) / m, eps);
    k.r = ms.y;
    if (threadIdx.x == 0 && mean) mean[blockIdx.x] = ms.x, rstd[blockIdx.x] = ms.y;
    if (blockDim.x == 64) __syncthreads();      // the sums of larger blocks had one
    each<V, MASK, K>(s, b, [&](int i, int row, const Window& w, bool on) {
        const float2 gb = row_params[row];
        k.ga = gb.x, k.be = gb.y;
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = forward<ACT>(k, f[j]);
        if (on) store<DT, V, MASK>(y, b, w, f);
    }, Nothing());
}

template <int DT, int V, bool MASK, int K, int ACT>
__global__ __launch_bounds__(threads_of(DT, V, K)) void k_gn_rows_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                                  const typename Elt<DT>::T* __restrict__ dy, Rows s,
                                                                  Params q, const float* __restrict__ mean,
                                                                  const float* __restrict__ rstd,
                                                                  typename Elt<DT>::T* __restrict__ dx,
                                                                  Sums sums) {
    using P = Pack<DT, V>;
    extern __shared__ float2 row_params[];      // gamma and beta of the rows
    float2* row_parts = row_params + s.cg;      // [cg][waves that share a row]
    __shared__ float part[32];
    const Base<V, MASK> b(s, int64_t(blockIdx.x) * s.cg * s.hw);
    const int c0 = int(blockIdx.x % unsigned(s.groups)) * s.cg;
    Coeff k;
    k.mu = mean[blockIdx.x], k.r = rstd[blockIdx.x];
    typename P::R d[K], e[K];
    each<V, MASK, K>(s, b, [&](int i, int, const Window& w, bool) {
        d[i] = load<DT, V, MASK, true>(x, b, w);
        e[i] = load<DT, V, MASK, true>(dy, b, w);
    }, Nothing());
    for (int row = threadIdx.x; row < s.cg; row += blockDim.x)
        row_params[row] = make_float2(or_one(q.gamma, c0 + row), or_zero(q.beta, c0 + row));
    __syncthreads();
    const int lanes = 1 << s.lanes_log2, lane = int(threadIdx.x) & (lanes - 1);
    const int share = lanes > 64 ? lanes >> 6 : 1;
    float sa = 0.f, sb = 0.f;
    each<V, MASK, K>(s, b, [&](int i, int row, const Window& w, bool on) {
        const float2 gb = row_params[row];
        k.ga = gb.x, k.be = gb.y;
        float f[V], g[V], ta = 0.f, tb = 0.f;
        P::open(d[i], f);
        P::open(e[i], g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = normal(k, f[j]);
            const float du = in<MASK>(w, j) ? slope<ACT>(k, xh, g[j]) : 0.f;
            ta += du;
            tb = in<MASK>(w, j) ? fmaf(du, xh, tb) : tb;
        }
        sa += on ? ta : 0.f;
        sb += on ? tb : 0.f;
    }, [&](int row) {
        sa = run_sum(sa, lanes);
        sb = run_sum(sb, lanes);
        if (row < s.cg && (lane & 63) == 0) row_parts[row * share + (lane >> 6)] = make_float2(sa, sb);
        sa = 0.f, sb = 0.f;
    });
    __syncthreads();
    float s1 = 0.f, s2 = 0.f;
    for (int row = threadIdx.x; row < s.cg; row += blockDim.x) {
        float a = 0.f, c = 0.f;
        for (int i = 0; i < share; ++i) {
            const float2 t = row_parts[row * share + i];
            a += t.x;
            c += t.y;
        }
        if (sums.ab) sums.ab[int64_t(blockIdx.x) * s.cg + row] = make_float2(a, c);
        if (sums.dgamma) sums.dgamma[c0 + row] = c;
        if (sums.dbeta) sums.dbeta[c0 + row] = a;
        const float ga = row_params[row].x;
        s1 = fmaf(ga, a, s1);
        s2 = fmaf(ga, c, s2);
    }
    const float m = float(s.cg) * float(s.hw);
    const float2 both = block_sum2(s1, s2, part);
    s1 = both.x / m, s2 = both.y / m;
    each<V, MASK, K>(s, b, [&](int i, int row, const Window& w, bool on) {
        const float2 gb = row_params[row];
        k.ga = gb.x, k.be = gb.y;
        float f[V], g[V];
        P::open(d[i], f);
        P::open(e[i], g);
        const Back s = back_of(k, s1, s2);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = backward<ACT>(k, s, f[j], g[j]);
        if (on) store<DT, V, MASK>(dx, b, w, f);
    }, Nothing());
}

// ---- pieces: a wave takes K x 64 vectors of a row.

struct Piece {
    unsigned id, row, ng;
    int c, piece;
};
__device__ __forceinline__ Piece this_piece(const Rows& s, int pieces) {
    Piece p;
    p.id = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    p.row = p.id / unsigned(pieces);
    p.piece = int(p.id - p.row * unsigned(pieces));
    p.ng = p.row / unsigned(s.cg);
    p.c = int(p.row % unsigned(s.cg * s.groups));
    return p;
}
// The base of a piece: its first vector, `skip` vectors behind the row's.  (From
// there, a row of 2^30 elements has no offset of more than 32 bits.)
template <int V, bool MASK> struct PieceBase : Base<V, MASK> {
    bool first;         // the row begins in this piece
    int left;           // elements from the base to the end of the row
    __device__ __forceinline__ PieceBase(const Rows& s, int64_t row, int skip)
        : Base<V, MASK>(s, row), first(skip == 0), left(this->phase + s.hw - skip * V) {
        this->shift(s, int64_t(skip) * V);
    }
};
// Calls f(i, window, on) for the vectors of a piece, as above.
template <int V, bool MASK, int K, class F>
__device__ __forceinline__ void each_of_piece(const PieceBase<V, MASK>& b, F f) {
    const int lane = int(threadIdx.x & 63);
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const int from = (i * 64 + lane) * V;
        const bool on = from < b.left;
        Window w;
        w.from = on ? from : 0;
        const int left = b.left - w.from;
        w.lo = MASK && b.first && w.from == 0 ? b.phase : 0;
        w.hi = !MASK || left >= V ? V : left;
        f(i, w, on);
    }
}

// Calls go with the vectors per lane of a piece: fewer where a row is one piece
// and has no more (33 x 778 x 11 x 11, two groups: fp32 forward 31 -> 19 us, fp16
// backward 59 -> 27; 16 x 512 x 14 x 14, one group, fp16 22 -> 12, 25 -> 13).
template <int DT, int V, class F> void with_piece(int vpr, F go) {
    constexpr int n = piece_of(DT, V);
    if (vpr <= 64 * (n / 8)) go(IntC<n / 8>{});
    else if (vpr <= 64 * (n / 4)) go(IntC<n / 4>{});
    else if (vpr <= 64 * (n / 2)) go(IntC<n / 2>{});
    else go(IntC<n>{});
}

// The mean of the elements, their squares about it, their number, and what the mean lacks.
template <int DT, int V, bool MASK, int K>
__global__ __launch_bounds__(256, 4) void k_gn_rowparts_fwd(const typename Elt<DT>::T* __restrict__ x, Rows s, int pieces,
                                                         unsigned count, float4* __restrict__ parts) {
    using P = Pack<DT, V>;
    const Piece p = this_piece(s, pieces);
    if (p.id >= count) return;
    const PieceBase<V, MASK> b(s, int64_t(p.row) * s.hw, p.piece * K * 64);
    typename P::R d[K];
    each_of_piece<V, MASK, K>(b, [&](int i, const Window& w, bool) { d[i] = load<DT, V, MASK, false>(x, b, w); });
    const int most = K * 64 * V, have = (b.left < most ? b.left : most) - (MASK && b.first ? b.phase : 0);
    const float num = have > 0 ? float(have) : 0.f;
    float sum = 0.f;
    each_of_piece<V, MASK, K>(b, [&](int i, const Window& w, bool on) {
        float f[V], t = 0.f;
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) t += in<MASK>(w, j) ? f[j] : 0.f;
        sum += on ? t : 0.f;
    });
    const float mu = num > 0.f ? wave_sum(sum) / num : 0.f;
    float sq = 0.f, rest = 0.f;
    each_of_piece<V, MASK, K>(b, [&](int i, const Window& w, bool on) {
        float f[V], t = 0.f, u = 0.f;
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float e = in<MASK>(w, j) ? f[j] - mu : 0.f;
            t = fmaf(e, e, t);
            u += e;
        }
        sq += on ? t : 0.f;
        rest += on ? u : 0.f;
    });
    sq = wave_sum(sq), rest = wave_sum(rest);
    if ((threadIdx.x & 63) == 0) parts[p.id] = make_float4(mu, sq, num, num > 0.f ? rest * __builtin_amdgcn_rcpf(num) : 0.f);
}

__device__ __forceinline__ Coeff coeff_of(const Piece& p, const Params& q, const float* mean, const float* rstd) {
    return Coeff{mean[p.ng], rstd[p.ng], or_one(q.gamma, p.c), or_zero(q.beta, p.c)};
}

template <int DT, int V, bool MASK, int K, int ACT>
__global__ __launch_bounds__(256, 4) void k_gn_rowwrite_fwd(const typename Elt<DT>::T* __restrict__ x, Rows s, Params q,
                                                            int pieces, unsigned count, float* __restrict__ mean,
                                                            float* __restrict__ rstd,
                                                            const float4* __restrict__ parts, float eps,
                                                            typename Elt<DT>::T* __restrict__ y) {
    using P = Pack<DT, V>;
    const Piece p = this_piece(s, pieces);
    if (p.id >= count) return;
    const PieceBase<V, MASK> b(s, int64_t(p.row) * s.hw, p.piece * K * 64);
    typename P::R d[K];
    each_of_piece<V, MASK, K>(b, [&](int i, const Window& w, bool) { d[i] = load<DT, V, MASK, false>(x, b, w); });
    Coeff k{0.f, 0.f, or_one(q.gamma, p.c), or_zero(q.beta, p.c)};
    if (parts) {
        const int per = s.cg * pieces;
        const float2 ms = joined_stats(parts + int64_t(p.ng) * per, per, int(threadIdx.x & 63), 64, eps);
        k.mu = ms.x, k.r = ms.y;
        if (mean && p.id == p.ng * unsigned(per) && (threadIdx.x & 63) == 0) mean[p.ng] = k.mu, rstd[p.ng] = k.r;
    } else {
        k.mu = mean[p.ng], k.r = rstd[p.ng];
    }
    each_of_piece<V, MASK, K>(b, [&](int i, const Window& w, bool on) {
        float f[V];
        P::open(d[i], f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = forward<ACT>(k, f[j]);
        if (on) store<DT, V, MASK>(y, b, w, f);
    });
}

template <int DT, int V, bool MASK, int K, int ACT>
__global__ __launch_bounds__(256, MASK ? 3 : 4) void k_gn_rowparts_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                         const typename Elt<DT>::T* __restrict__ dy, Rows s, Params q,
                                                         int pieces, unsigned count, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, float2* __restrict__ parts) {
    using P = Pack<DT, V>;
    const Piece p = this_piece(s, pieces);
    if (p.id >= count) return;
    const PieceBase<V, MASK> b(s, int64_t(p.row) * s.hw, p.piece * K * 64);
    typename P::R d[K], e[K];
    each_of_piece<V, MASK, K>(b, [&](int i, const Window& w, bool) {
        d[i] = load<DT, V, MASK, false>(x, b, w);
        e[i] = load<DT, V, MASK, false>(dy, b, w);
    });
    const Coeff k = coeff_of(p, q, mean, rstd);
    float sa = 0.f, sb = 0.f;
    each_of_piece<V, MASK, K>(b, [&](int i, const Window& w, bool on) {
        float f[V], g[V], ta = 0.f, tb = 0.f;
        P::open(d[i], f);
        P::open(e[i], g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = normal(k, f[j]);
            const float du = in<MASK>(w, j) ? slope<ACT>(k, xh, g[j]) : 0.f;
            ta += du;
            tb = in<MASK>(w, j) ? fmaf(du, xh, tb) : tb;
        }
        sa += on ? ta : 0.f;
        sb += on ? tb : 0.f;
    });
    sa = wave_sum(sa);
    sb = wave_sum(sb);
    if ((threadIdx.x & 63) == 0) parts[p.id] = make_float2(sa, sb);
}

template <int DT, int V, bool MASK, int K, int ACT>
__global__ __launch_bounds__(256, 4) void k_gn_rowwrite_bwd(const typename Elt<DT>::T* __restrict__ x,
                                                         const typename Elt<DT>::T* __restrict__ dy, Rows s, Params q,
                                                         int pieces, unsigned count, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, const float2* __restrict__ s12,
                                                         const float2* __restrict__ parts, Tail tail,
                                                         typename Elt<DT>::T* __restrict__ dx) {
    using P = Pack<DT, V>;
    if (blockIdx.x >= tail.first) return param_block(tail);
    const Piece p = this_piece(s, pieces);
    if (p.id >= count) return;
    const PieceBase<V, MASK> b(s, int64_t(p.row) * s.hw, p.piece * K * 64);
    typename P::R d[K], e[K];
    each_of_piece<V, MASK, K>(b, [&](int i, const Window& w, bool) {
        d[i] = load<DT, V, MASK, false>(x, b, w);
        e[i] = load<DT, V, MASK, false>(dy, b, w);
    });
    const Coeff k = coeff_of(p, q, mean, rstd);
    const int per = s.cg * pieces;
    const float2 sum = parts ? joined_back(parts + int64_t(p.ng) * per, per, pieces, q.gamma ? q.gamma + p.c / s.cg * s.cg : nullptr,
                                           float(s.cg) * float(s.hw), int(threadIdx.x & 63), 64)
                             : s12[p.ng];
    const Back back = back_of(k, sum.x, sum.y);
    each_of_piece<V, MASK, K>(b, [&](int i, const Window& w, bool on) {
        float f[V], g[V];
        P::open(d[i], f);
        P::open(e[i], g);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = backward<ACT>(k, back, f[j], g[j]);
        if (on) store<DT, V, MASK>(dx, b, w, f);
    });
}

template <int DT, int V, bool MASK>
void fwd(const Plan& p, int64_t count, const void* x, const Params& q, float eps, void* y, float* mean, float* rstd,
         float4* parts, hipStream_t st) {
    using T = typename Elt<DT>::T;
    const T* xt = static_cast<const T*>(x);
    T* yt = static_cast<T*>(y);
    if constexpr (V > 1)
        if (p.held) {
            const dim3 grid(static_cast<unsigned>(p.grid)), block(static_cast<unsigned>(p.threads));
            const unsigned lds = unsigned(sizeof(float2)) * unsigned(p.rows.cg);
            with_act(q.act, [&](auto act) {
                with_count<DT, V, false>(p.k, [&](auto k) {
                    hipLaunchKernelGGL((k_gn_rows_fwd<DT, V, MASK, decltype(k)::value, decltype(act)::value>), grid, block,
                                       lds, st, xt, p.rows, q, eps, yt, mean, rstd);
                });
            });
            return;
        }
    const dim3 grid(static_cast<unsigned>((count + 3) / 4));
    with_piece<DT, V>(p.rows.vpr, [&](auto k) {
        constexpr int K = decltype(k)::value;
        hipLaunchKernelGGL((k_gn_rowparts_fwd<DT, V, MASK, K>), grid, dim3(256), 0, st, xt, p.rows, p.pieces,
                           unsigned(count), parts);
        if (!p.joined) combine_fwd(parts, count / (int64_t(p.rows.cg) * p.pieces), p.rows.cg * p.pieces, eps, mean, rstd, st);
        with_act(q.act, [&](auto act) {
            hipLaunchKernelGGL((k_gn_rowwrite_fwd<DT, V, MASK, K, decltype(act)::value>), grid, dim3(256), 0, st, xt, p.rows,
                               q, p.pieces, unsigned(count), mean, rstd, p.joined ? parts : nullptr, eps, yt);
        });
    });
}

template <int DT, int V, bool MASK>
void bwd(const Plan& p, int64_t count, const void* x, const void* dy, const Params& q, const float* mean,
         const float* rstd, void* dx, const Sums& sums, float2* s12, Tail tail, hipStream_t st) {
    using T = typename Elt<DT>::T;
    const T *xt = static_cast<const T*>(x), *gt = static_cast<const T*>(dy);
    T* dt = static_cast<T*>(dx);
    if constexpr (V > 1)
        if (p.held) {
            const dim3 grid(static_cast<unsigned>(p.grid)), block(static_cast<unsigned>(p.threads));
            const int lanes = 1 << p.rows.lanes_log2;
            const unsigned lds = unsigned(sizeof(float2)) * unsigned(p.rows.cg) * unsigned(1 + (lanes > 64 ? lanes / 64 : 1));
            with_act(q.act, [&](auto act) {
                with_count<DT, V, true>(p.k, [&](auto k) {
                    hipLaunchKernelGGL((k_gn_rows_bwd<DT, V, MASK, decltype(k)::value, decltype(act)::value>), grid, block,
                                       lds, st, xt, gt, p.rows, q, mean, rstd, dt, sums);
                });
            });
            return;
        }
    const dim3 grid(static_cast<unsigned>((count + 3) / 4));
    tail.first = grid.x;
    with_piece<DT, V>(p.rows.vpr, [&](auto k) {
        constexpr int K = decltype(k)::value;
        with_act(q.act, [&](auto act) {
            hipLaunchKernelGGL((k_gn_rowparts_bwd<DT, V, MASK, K, decltype(act)::value>), grid, dim3(256), 0, st, xt, gt,
                               p.rows, q, p.pieces, unsigned(count), mean, rstd, sums.ab);
            const float m = float(p.rows.cg) * float(p.rows.hw);
            if (!p.joined)
                combine_bwd(sums.ab, count / (int64_t(p.rows.cg) * p.pieces), p.rows.cg * p.pieces, p.pieces,
                            p.rows.groups, p.rows.cg, m, q.gamma, s12, st);
            hipLaunchKernelGGL((k_gn_rowwrite_bwd<DT, V, MASK, K, decltype(act)::value>), dim3(grid.x + tail_blocks(tail)),
                               dim3(256), 0, st, xt, gt, p.rows, q, p.pieces, unsigned(count), mean, rstd, s12,
                               p.joined ? sums.ab : nullptr, tail, dt);
        });
    });
}

}  // namespace

template <int DT>
void rows_fwd(const Plan& p, int64_t count, const void* x, const Params& q, float eps, void* y, float* mean, float* rstd,
              float4* parts, hipStream_t st) {
    constexpr int V = vector_of(DT, false);
    if (p.vec == 0) fwd<DT, 1, false>(p, count, x, q, eps, y, mean, rstd, parts, st);
    else if (p.vec == 1) fwd<DT, V, false>(p, count, x, q, eps, y, mean, rstd, parts, st);
    else fwd<DT, V, true>(p, count, x, q, eps, y, mean, rstd, parts, st);
}
template <int DT>
void rows_bwd(const Plan& p, int64_t count, const void* x, const void* dy, const Params& q, const float* mean,
              const float* rstd, void* dx, const Sums& sums, float2* s12, Tail tail, hipStream_t st) {
    constexpr int V = vector_of(DT, false);
    if (p.vec == 0) bwd<DT, 1, false>(p, count, x, dy, q, mean, rstd, dx, sums, s12, tail, st);
    else if (p.vec == 1) bwd<DT, V, false>(p, count, x, dy, q, mean, rstd, dx, sums, s12, tail, st);
    else bwd<DT, V, true>(p, count, x, dy, q, mean, rstd, dx, sums, s12, tail, st);
}

}  // namespace gn
}  // namespace psc
