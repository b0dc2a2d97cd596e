// Device code of the group normalisation that its translation units share:
// vectors of 16 bytes (or single elements), activations, sums.
//
// For image n and group g of Cg = C / G channels, over its M = Cg H W values:
//   mu = mean x,  r = 1 / sqrt(var x + eps),  xh = (x - mu) r
//   y  = act(u),  u = gamma[c] xh + beta[c]
// and for the gradient dy of y, with du = dy act'(u):
//   A[n,c] = sum du,  B[n,c] = sum du xh        (over H W)
//   dbeta = sum_n A,  dgamma = sum_n B
//   dx = r (gamma du - (S1 + xh S2) / M),  S1 = sum_c gamma A,  S2 = sum_c gamma B
// Everything is summed in fp32, the variance about the mean.
//
// A call is bound by memory: x read and y written once (backward: x and dy
// read, dx written).  A block that holds the whole of its groups in registers
// does that (k_gn_rows_* in NCHW, where a group lies in one piece, k_gn_cols_*
// with the channels last, where a block takes all pixels of some whole
// groups).  Groups too large or too few for that are read twice: partial sums
// over pieces (k_gn_rowparts_*, k_gn_colparts_*), their combination
// (k_gn_combine_*), and the same pieces again to write the result.
#pragma once
#include "common.h"
#include "launch.h"

namespace psc {
namespace gn {

enum : int { ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2 };

__device__ __forceinline__ float sigmoid(float u) { return __builtin_amdgcn_rcpf(1.f + __expf(-u)); }
template <int ACT> __device__ __forceinline__ float act_of(float u) {
    if (ACT == ACT_RELU) return u < 0.f ? 0.f : u;
    if (ACT == ACT_SILU) return u * sigmoid(u);
    return u;
}
// u rounds after the product and after the sum, in the forward and in the
// backward: the ReLU passes the gradient of exactly the outputs above zero.
__device__ __forceinline__ float affine(float xh, float ga, float be) {
#pragma clang fp contract(off)
    return xh * ga + be;
}
// The gradient at u of a gradient dy at act(u).
template <int ACT> __device__ __forceinline__ float act_back(float u, float dy) {
    if (ACT == ACT_RELU) return u > 0.f ? dy : 0.f;
    if (ACT == ACT_SILU) {
        const float s = sigmoid(u);
        return dy * (s * fmaf(u, 1.f - s, 1.f));
    }
    return dy;
}
// What a value x of a group and channel becomes, and its normalised value.
struct Coeff {
    float mu, r, ga, be;
};
__device__ __forceinline__ float normal(const Coeff& k, float x) { return (x - k.mu) * k.r; }
template <int ACT> __device__ __forceinline__ float forward(const Coeff& k, float x) {
    return act_of<ACT>(affine(normal(k, x), k.ga, k.be));
}
template <int ACT> __device__ __forceinline__ float slope(const Coeff& k, float xh, float dy) {
    return act_back<ACT>(affine(xh, k.ga, k.be), dy);
}
// s: r gamma, r S1 / M and r S2 / M.
struct Back {
    float ga, s1, s2;
};
__device__ __forceinline__ Back back_of(const Coeff& k, float s1, float s2) { return Back{k.r * k.ga, k.r * s1, k.r * s2}; }
template <int ACT> __device__ __forceinline__ float backward(const Coeff& k, const Back& s, float x, float dy) {
    const float xh = normal(k, x);
    return fmaf(-s.s2, xh, fmaf(s.ga, slope<ACT>(k, xh, dy), -s.s1));
}

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

// V elements as they lie in memory: 16 bytes, 8, or one element.
template <int DT, int V> struct Pack;
template <> struct Pack<DT_F32, 4> {
    using R = u4;
    __device__ __forceinline__ static void open(const R& r, float (&f)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t b = r[j];
            f[j] = __builtin_bit_cast(float, b);
        }
    }
    __device__ __forceinline__ static R close(const float (&f)[4]) {
        R r;
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = __builtin_bit_cast(uint32_t, f[j]);
        return r;
    }
};
template <> struct Pack<DT_F16, 8> {
    using R = u4;
    __device__ __forceinline__ static void open(const R& r, float (&f)[8]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t b = r[j];
            f[2 * j] = float(__builtin_bit_cast(_Float16, uint16_t(b)));
            f[2 * j + 1] = float(__builtin_bit_cast(_Float16, uint16_t(b >> 16)));
        }
    }
    __device__ __forceinline__ static R close(const float (&f)[8]) {
        R r;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            r[j] = uint32_t(Elt<DT_F16>::from_f(f[2 * j])) | uint32_t(Elt<DT_F16>::from_f(f[2 * j + 1])) << 16;
        return r;
    }
};
template <> struct Pack<DT_F16, 4> {
    using R = u2;
    __device__ __forceinline__ static void open(const R& r, float (&f)[4]) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t b = r[j];
            f[2 * j] = float(__builtin_bit_cast(_Float16, uint16_t(b)));
            f[2 * j + 1] = float(__builtin_bit_cast(_Float16, uint16_t(b >> 16)));
        }
    }
    __device__ __forceinline__ static R close(const float (&f)[4]) {
        R r;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            r[j] = uint32_t(Elt<DT_F16>::from_f(f[2 * j])) | uint32_t(Elt<DT_F16>::from_f(f[2 * j + 1])) << 16;
        return r;
    }
};
template <int DT> struct Pack<DT, 1> {
    using R = typename Elt<DT>::T;
    __device__ __forceinline__ static void open(const R& r, float (&f)[1]) { f[0] = Elt<DT>::load(&r, 0); }
    __device__ __forceinline__ static R close(const float (&f)[1]) { return Elt<DT>::from_f(f[0]); }
};

// Sums over lanes, in every one of them, by moves within the register file
// (a permutation through the LDS takes several times as long, and these sums
// are most of what a small call waits for).  Step OFF adds the lanes whose
// numbers differ in bit OFF; the mirrors do as much once the smaller steps
// are done.
template <int OFF> __device__ __forceinline__ float lane_step(float x) {
    const int b = __builtin_bit_cast(int, x);
    if constexpr (OFF == 16 || OFF == 32) {
        const auto r = OFF == 16 ? __builtin_amdgcn_permlane16_swap(b, b, false, false)
                                 : __builtin_amdgcn_permlane32_swap(b, b, false, false);
        const unsigned lo = r[0], hi = r[1];
        return __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
    } else {
        // quad_perm [1,0,3,2] and [2,3,0,1], row_half_mirror, row_mirror
        constexpr int ctrl = OFF == 1 ? 0xB1 : OFF == 2 ? 0x4E : OFF == 4 ? 0x141 : 0x140;
        return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, b, ctrl, 0xf, 0xf, true));
    }
}
// x plus the x of the lane BY further on in its row of 16.
template <int BY> __device__ __forceinline__ float turned_sum(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x120 + BY, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float x) {
    x = lane_step<1>(x), x = lane_step<2>(x), x = lane_step<4>(x), x = lane_step<8>(x);
    return lane_step<32>(lane_step<16>(x));
}
// Over runs of `lanes` lanes, a power of two up to 64.
__device__ __forceinline__ float run_sum(float x, int lanes) {
    if (lanes > 1) x = lane_step<1>(x);
    if (lanes > 2) x = lane_step<2>(x);
    if (lanes > 4) x = lane_step<4>(x);
    if (lanes > 8) x = lane_step<8>(x);
    if (lanes > 16) x = lane_step<16>(x);
    if (lanes > 32) x = lane_step<32>(x);
    return x;
}
// Sum over the block, in every thread.  part: 16 floats of LDS; the caller
// has no other use of them before the next barrier but one.
__device__ __forceinline__ float block_sum(float x, float* part) {
    x = wave_sum(x);
    const int waves = int(blockDim.x >> 6);
    if (waves == 1) return x;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    const int l = threadIdx.x & 15;
    return run_sum(l < waves ? part[l] : 0.f, 16);
}
// Two sums at once; part: 32 floats.
__device__ __forceinline__ float2 block_sum2(float x, float y, float* part) {
    x = wave_sum(x), y = wave_sum(y);
    const int waves = int(blockDim.x >> 6);
    if (waves == 1) return make_float2(x, y);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x, part[16 + (threadIdx.x >> 6)] = y;
    __syncthreads();
    const int l = threadIdx.x & 15;
    return make_float2(run_sum(l < waves ? part[l] : 0.f, 16), run_sum(l < waves ? part[16 + l] : 0.f, 16));
}

__device__ __forceinline__ float or_one(const float* p, int64_t i) { return p ? p[i] : 1.f; }
__device__ __forceinline__ float or_zero(const float* p, int64_t i) { return p ? p[i] : 0.f; }

// Accesses at a byte offset of 32 bits from an address that the block (or the
// wave) has in common: one register a lane instead of two, and no sums.  PAST:
// past the caches.  What a die's cache keeps of the output has to leave it at
// the end of the launch, before other dies may read it, so that it had better
// go at once, and what is read once need not be kept: 64 x 512 x 28 x 28 fp16
// forward 31 -> 22 us with the channels last, 28 -> 26 in NCHW; 256 x 128 x 16
// x 16 fp32 13.2 -> 11.6, backward 25 -> 21 us.  Not for less than half a line
// of memory: lines come together in the cache (tiles of 16 bytes, 32 x 64 x 56
// x 56 fp16: 16 us, 28 us past it).
template <class R, bool PAST, class T> __device__ __forceinline__ R get(const T* base, uint32_t byte) {
    const R* p = reinterpret_cast<const R*>(reinterpret_cast<const char*>(base) + byte);
    if constexpr (PAST) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool PAST, class R, class T> __device__ __forceinline__ void put(T* base, uint32_t byte, const R& r) {
    R* p = reinterpret_cast<R*>(reinterpret_cast<char*>(base) + byte);
    if constexpr (PAST) __builtin_nontemporal_store(r, p);
    else *p = r;
}

// Where the sums of channels go: [n][c][pieces], and, where an image is the
// whole batch, the parameters' gradients at once.
struct Sums {
    float2* ab;
    float* dgamma;
    float* dbeta;
};
// dbeta and dgamma from the sums: the blocks from `first` on of a launch add 8
// channels each, over the images and pieces, blockDim / 8 of them at a time,
// in a fixed order.
struct Tail {
    const float2* sums;
    int n, c, pieces;
    float* dgamma;
    float* dbeta;
    unsigned first;
};
__device__ __forceinline__ void param_block(const Tail& t) {
    __shared__ float2 part[16][8];
    const int k = int(blockIdx.x - t.first) * 8 + int(threadIdx.x & 7);
    float a = 0.f, b = 0.f;
    if (k < t.c) {
        const unsigned count = unsigned(t.n) * unsigned(t.pieces);
        for (unsigned i = threadIdx.x >> 3; i < count; i += blockDim.x >> 3) {
            const unsigned img = i / unsigned(t.pieces), piece = i - img * unsigned(t.pieces);
            const float2 ab = t.sums[(int64_t(img) * t.c + k) * t.pieces + piece];
            a += ab.x;
            b += ab.y;
        }
    }
    a = turned_sum<8>(a), b = turned_sum<8>(b);
    a = lane_step<32>(lane_step<16>(a)), b = lane_step<32>(lane_step<16>(b));
    if ((threadIdx.x & 63) < 8) part[threadIdx.x >> 6][threadIdx.x & 7] = make_float2(a, b);
    __syncthreads();
    if (threadIdx.x < 8 && k < t.c) {
        a = 0.f, b = 0.f;
        for (unsigned i = 0; i < blockDim.x >> 6; ++i) a += part[i][threadIdx.x].x, b += part[i][threadIdx.x].y;
        if (t.dgamma) t.dgamma[k] = b;
        if (t.dbeta) t.dbeta[k] = a;
    }
}

// mean and rstd as they are kept: both NaN where a value of the group is not
// finite, or a sum passed fp32 (then the variance is not finite, whatever the
// mean is).  That of joined pieces without a spread, all of it roundings of
// their means, may round below zero, by more than a tiny eps.
__device__ __forceinline__ float2 stats_of(float mu, float var, float eps) {
    const bool fine = __builtin_isfinite(var);
    const float nan = __builtin_nanf("");
    return make_float2(fine ? mu : nan, fine ? 1.f / sqrtf((var < 0.f ? 0.f : var) + eps) : nan);
}

// A piece in the sums of its group: mean x (rounded, and w what that lacks of
// the true one), squares y about x, count z.  Its part of the sum, and of the
// squares about mu.  Without w the rounding of x, which is of the size of the
// values, not of their spread, would count once for every piece's distance
// from the others: 10^4 spreads from zero rstd was 6e-5 off.
__device__ __forceinline__ float sum_with(const float4& p, float sum) { return fmaf(p.z, p.x, fmaf(p.z, p.w, sum)); }
__device__ __forceinline__ float squares_about(const float4& p, float mu) {
    const float d = p.x - mu;
    return fmaf(p.z * d, fmaf(2.f, p.w, d), p.y);
}

// The statistics of a group from its pieces, by a run of `lanes` lanes.
__device__ __forceinline__ float2 joined_stats(const float4* p, int count, int lane, int lanes, float eps) {
    float sum = 0.f, num = 0.f;
    for (int i = lane; i < count; i += lanes) {
        const float4 t = p[i];
        sum = sum_with(t, sum);
        num += t.z;
    }
    num = run_sum(num, lanes);
    const float mu = run_sum(sum, lanes) / num;
    float sq = 0.f;
    for (int i = lane; i < count; i += lanes) sq += squares_about(p[i], mu);
    return stats_of(mu, run_sum(sq, lanes) / num, eps);
}
// S1 / M and S2 / M of the group whose channels begin with gamma[0].
__device__ __forceinline__ float2 joined_back(const float2* p, int count, int pieces, const float* gamma, float m, int lane,
                                              int lanes) {
    float s1 = 0.f, s2 = 0.f;
    for (int i = lane; i < count; i += lanes) {
        const float ga = or_one(gamma, i / pieces);
        s1 = fmaf(ga, p[i].x, s1);
        s2 = fmaf(ga, p[i].y, s2);
    }
    return make_float2(run_sum(s1, lanes) / m, run_sum(s2, lanes) / m);
}

// ---- NCHW.  A channel of an image is a row of hw elements; rows lie one
// after the other.  With MASK a row need not begin or end at a multiple of 16
// bytes: its vectors lie at multiples of 16 bytes in memory, and of the first
// and the last only some elements are the row's.  All tensors of the call lie
// alike to 16 bytes.
struct Rows {
    int cg, groups, hw;
    int lead;           // elements between a multiple of 16 bytes and the tensor's first
    int64_t total;      // elements of the tensor
    int vpr;            // vectors of a row, at most
    int lanes_log2;     // lanes (a power of two) that share a row
    int vi;             // vectors of a row per lane
    int slots;          // vectors per thread: vi times the rows per lane
};

// The element that offsets of a block or wave count from: `first`, or up to V -
// 1 elements before it, at a multiple of 16 bytes.  [lo, hi): where the
// offsets lie in the tensor.
template <int V, bool MASK> struct Base {
    int64_t at;
    int phase, lo, hi;
    __device__ __forceinline__ Base(const Rows& s, int64_t first) {
        phase = MASK ? int((first + s.lead) & (V - 1)) : 0;
        at = first - phase;
        shift(s, 0);
    }
    __device__ __forceinline__ void shift(const Rows& s, int64_t by) {
        at += by;
        lo = at < 0 ? int(-at) : 0;
        const int64_t left = s.total - at;
        hi = left < (1 << 30) ? int(left) : 1 << 30;
    }
};
// A vector: its first element from the base; elements lo .. hi of it are the row's.
struct Window {
    int from, lo, hi;
};
// Whether vector k of the row of `len` elements that begins `row` elements behind the base's `first` has any of it.
template <int V, bool MASK>
__device__ __forceinline__ bool has(const Base<V, MASK>& b, int row, int len, int k) {
    return k * V < len + (MASK ? (b.phase + row) & (V - 1) : 0);
}
template <int V, bool MASK>
__device__ __forceinline__ Window window(const Base<V, MASK>& b, int row, int len, int k) {
    Window w;
    if (!MASK) {
        w.from = row + k * V;
        w.lo = 0;
        w.hi = V;
    } else {
        const int at = b.phase + row, phase = at & (V - 1);
        w.from = at - phase + k * V;
        const int left = at + len - w.from;
        w.lo = k == 0 ? phase : 0;
        w.hi = left < V ? left : V;
    }
    return w;
}
// Sixteen bytes moved by an element: to higher places, `e` in the lowest; to lower ones.
template <int BITS> __device__ __forceinline__ u4 shifted_up(const u4& r, uint32_t e) {
    if constexpr (BITS == 32) return u4{e, r.x, r.y, r.z};
    else return u4{r.x << 16 | e, r.y << 16 | r.x >> 16, r.z << 16 | r.y >> 16, r.w << 16 | r.z >> 16};
}
template <int BITS> __device__ __forceinline__ u4 shifted_down(const u4& r) {
    if constexpr (BITS == 32) return u4{r.y, r.z, r.w, 0};
    else return u4{r.x >> 16 | r.y << 16, r.y >> 16 | r.z << 16, r.z >> 16 | r.w << 16, r.w >> 16};
}
template <int DT, int V, bool MASK, bool PAST>
__device__ __forceinline__ typename Pack<DT, V>::R load(const typename Elt<DT>::T* p, const Base<V, MASK>& b, const Window& w) {
    using T = typename Elt<DT>::T;
    // the elements beside the row's are other rows', or there are none: nothing outside the tensor is read
    if (!MASK || (w.from >= b.lo && w.from + V <= b.hi))
        return get<typename Pack<DT, V>::R, PAST && !MASK>(p + b.at, uint32_t(w.from) * uint32_t(sizeof(T)));
    if constexpr (MASK) {
        // rare and small: element by element, each moved up as the next comes
        u4 r = {0, 0, 0, 0};
#pragma unroll 1
        for (int j = V - 1; j >= 0; --j) {
            const uint32_t e = j >= w.lo && j < w.hi ? uint32_t(reinterpret_cast<const typename Elt<DT>::Bits*>(p + b.at)[w.from + j]) : 0u;
            r = shifted_up<8 * sizeof(T)>(r, e);
        }
        return r;
    }
}
template <int DT, int V, bool MASK>
__device__ __forceinline__ void store(typename Elt<DT>::T* p, const Base<V, MASK>& b, const Window& w, const float (&f)[V]) {
    using T = typename Elt<DT>::T;
    const auto r = Pack<DT, V>::close(f);
    const uint32_t byte = uint32_t(w.from) * uint32_t(sizeof(T));
    if (!MASK || (w.lo == 0 && w.hi == V)) {
        put<!MASK && (V > 1)>(p + b.at, byte, r);
        return;
    }
    if constexpr (MASK) {
        u4 e = r;
#pragma unroll 1
        for (int j = 0; j < w.hi; ++j) {
            if (j >= w.lo) put<false>(p + b.at, byte + j * uint32_t(sizeof(T)), typename Elt<DT>::Bits(e.x));
            e = shifted_down<8 * sizeof(T)>(e);
        }
    }
}
template <bool MASK> __device__ __forceinline__ bool in(const Window& w, int j) { return !MASK || (j >= w.lo && j < w.hi); }

// ---- channels last.  A block takes `tile` channels (its threads `cols`
// vectors, a power of two, side by side) and some of the pixels.
struct Cols {
    int c, cg, groups;
    int hw;
    int tile;           // channels of a block
    int tiles;
    int near;           // tiles that share lines of memory
    int cols_log2;
    int pixels;         // pixels of a block
    int chunks;         // blocks that share the pixels of an image
    uint32_t cg_m;      // 2^32 / cg, rounded up
    int join_lanes;     // lanes that join a group's pieces
};
// k / cg for k, cg < 2^16 (cg_m is at most cg - 1 too large: less than 2^32 / cg in the product); cg == 1: 0.
__device__ __forceinline__ int group_of(const Cols& q, int k) { return q.cg_m ? int(__umulhi(uint32_t(k), q.cg_m)) : k; }

// Adds s[N] of each thread over the threads of the wave that have the same
// channels: the lanes of a row of 16 by turning it, which keeps the columns
// below the turn apart.  Several sums go together, step by step: each step of
// one waits for the one before (a third sum of eight channels apart cost 1.2
// us of 12).
template <int N> __device__ __forceinline__ void add_columns(float (&s)[N], int cols) {
    const auto step = [&](auto f) {
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] = f(s[j]);
    };
    if (cols <= 8) step([](float x) { return turned_sum<8>(x); });
    if (cols <= 4) step([](float x) { return turned_sum<4>(x); });
    if (cols <= 2) step([](float x) { return turned_sum<2>(x); });
    if (cols <= 1) step([](float x) { return turned_sum<1>(x); });
    if (cols <= 16) step([](float x) { return lane_step<16>(x); });
    if (cols <= 32) step([](float x) { return lane_step<32>(x); });
}
// Those sums of N / V values of each of the V channels, left in `buf`: for
// each value sum_rows(q) rows of `tile`.
__device__ __forceinline__ int span_log2(const Cols& q) { return q.cols_log2 > 6 ? q.cols_log2 : 6; }
__device__ __forceinline__ int sum_rows(const Cols& q) { return int(blockDim.x >> span_log2(q)); }
template <int V, int N>
__device__ __forceinline__ void wave_channels(float (&s)[N], const Cols& q, int width, float* buf) {
    const int cols = 1 << q.cols_log2, col = int(threadIdx.x) & (cols - 1);
    add_columns(s, cols);
    if (int(threadIdx.x & 63u) < cols && col * V < width) {
        float* to = buf + int(threadIdx.x >> span_log2(q)) * q.tile + col * V;
#pragma unroll
        for (int j = 0; j < N; ++j) to[(j / V) * sum_rows(q) * q.tile + j % V] = s[j];
    }
}
__device__ __forceinline__ float sum_of_channel(const float* buf, const Cols& q, int k) {
    float s = 0.f;
    const int rows = sum_rows(q);
    for (int i = 0; i < rows; ++i) s += buf[i * q.tile + k];
    return s;
}

struct Params {
    const float* gamma;
    const float* beta;
    int act;
};

// How a call runs (host).  pieces: partial sums of each channel, [n][c][pieces].
struct Plan {
    bool held;          // a block holds its whole groups
    bool joined;        // else: who writes a piece adds up its group's pieces itself
    int vec;            // 0: single elements, 1: 16 bytes, 2: 16 bytes with windows
    int k;              // vectors per thread, rounded up to a compiled count
    int threads;
    int64_t grid;
    int pieces;
    Rows rows;
    Cols cols;
};
// Elements of a vector.  The backward with the channels last holds six values
// for each channel of a thread besides x and dy: with eight channels of fp16
// it took more than 128 registers and one block filled a CU (512 @ 28x28 b64:
// 62 us), so it takes four.
constexpr int vector_of(int dtype, bool columns_back) { return dtype == DT_F16 && !columns_back ? 8 : 4; }
// Vectors per lane of the kernels that work piece by piece: 128 bytes, or as
// many single elements.
constexpr int kPieceSingle = 16;
constexpr int piece_of(int dtype, int v) { return v == 1 ? kPieceSingle : 128 / (v * (dtype == DT_F16 ? 2 : 4)); }
// The most vectors per thread of the kernels that hold their groups, and the
// threads that leave registers for so many.
constexpr int most_of(int dtype, int v, bool back) { return v == 1 ? 32 : (back ? 1 : 2) * piece_of(dtype, v); }
constexpr int threads_of(int dtype, int v, int k) { return 2 * k <= piece_of(dtype, v) ? 1024 : 512; }

// Calls go with the compiled activation and count of vectors per thread.
template <class F> void with_act(int act, F go) {
    if (act == ACT_NONE) go(IntC<ACT_NONE>{});
    else if (act == ACT_RELU) go(IntC<ACT_RELU>{});
    else go(IntC<ACT_SILU>{});
}
template <int DT, int V, bool BACK, class F> void with_count(int k, F go) {
    if constexpr (V == 1) {
        if (k <= 8) go(IntC<8>{});
        else go(IntC<32>{});
    } else {
        constexpr int n = piece_of(DT, V);
        if (k <= n / 4) go(IntC<n / 4>{});
        else if (k <= n / 2) go(IntC<n / 2>{});
        else if (k <= n) go(IntC<n>{});
        else if constexpr (!BACK) go(IntC<2 * n>{});
    }
}

// LDS of a block of columns: `sums` arrays of the waves' sums, `more` of one value per channel.
inline unsigned cols_lds(const Cols& q, int threads, int sums, int more) {
    return unsigned(sizeof(float)) * unsigned(q.tile) * unsigned(sums * (threads >> (q.cols_log2 > 6 ? q.cols_log2 : 6)) + more);
}

template <int DT> void rows_fwd(const Plan& p, int64_t count, const void* x, const Params& q, float eps, void* y,
                                float* mean, float* rstd, float4* parts, hipStream_t st);
template <int DT> void rows_bwd(const Plan& p, int64_t count, const void* x, const void* dy, const Params& q,
                                const float* mean, const float* rstd, void* dx, const Sums& sums, float2* s12,
                                Tail tail, hipStream_t st);
template <int DT> void cols_fwd(const Plan& p, int n, const void* x, const Params& q, float eps, void* y, float* mean,
                                float* rstd, float4* parts, hipStream_t st);
template <int DT> void cols_bwd(const Plan& p, int n, const void* x, const void* dy, const Params& q, const float* mean,
                                const float* rstd, void* dx, const Sums& sums, float2* s12, Tail tail, hipStream_t st);
// The blocks that a tail adds to a launch.
inline unsigned tail_blocks(const Tail& t) { return t.dgamma || t.dbeta ? unsigned(t.c + 7) / 8u : 0u; }
// Between the two passes over pieces (group_norm.hip): the statistics of each
// of `groups` groups, or S1 / M and S2 / M, from its parts.
void combine_fwd(const float4* parts, int64_t groups, int per_group, float eps, float* mean, float* rstd, hipStream_t st);
void combine_bwd(const float2* parts, int64_t groups, int per_group, int pieces, int groups_per_image, int cg, float m,
                 const float* gamma, float2* s12, hipStream_t st);

}  // namespace gn
}  // namespace psc
