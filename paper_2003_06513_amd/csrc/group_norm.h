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
__device__ __forceinline__ float act_of(float u, int act) {
    return act == ACT_RELU ? (u < 0.f ? 0.f : u) : act == ACT_SILU ? u * sigmoid(u) : u;
}
// u rounds after the product and after the sum, in the forward and in the
// backward: the ReLU passes the gradient of exactly the outputs above zero.
__device__ __forceinline__ float affine(float xh, float ga, float be) {
#pragma clang fp contract(off)
    return xh * ga + be;
}
// The gradient at u of a gradient dy at act(u).
__device__ __forceinline__ float act_back(float u, float dy, int act) {
    if (act == ACT_RELU) return u > 0.f ? dy : 0.f;
    if (act == ACT_SILU) {
        const float s = sigmoid(u);
        return dy * (s * fmaf(u, 1.f - s, 1.f));
    }
    return dy;
}

typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// V elements as they lie in memory: 16 bytes, or one element.
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
template <int DT> struct Pack<DT, 1> {
    using R = typename Elt<DT>::T;
    __device__ __forceinline__ static void open(const R& r, float (&f)[1]) { f[0] = Elt<DT>::load(&r, 0); }
    __device__ __forceinline__ static R close(const float (&f)[1]) { return Elt<DT>::from_f(f[0]); }
};

// Sum over the block, in every thread.  part: 16 floats of LDS; the caller
// has no other use of them before the next barrier.
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    return x;
}
__device__ __forceinline__ float block_sum(float x, float* part) {
    x = wave_sum(x);
    const int waves = int(blockDim.x >> 6);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    const int l = threadIdx.x & 15;
    float s = l < waves ? part[l] : 0.f;
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) s += __shfl_xor(s, off);
    __syncthreads();
    return s;
}

__device__ __forceinline__ float or_one(const float* p, int64_t i) { return p ? p[i] : 1.f; }
__device__ __forceinline__ float or_zero(const float* p, int64_t i) { return p ? p[i] : 0.f; }

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

// Vector k of the row that begins at element `at` of the tensor: elements lo
// .. hi of it are the row's, and it begins at element `from`.
struct Window {
    int64_t from;
    int lo, hi;
};
template <int V, bool MASK>
__device__ __forceinline__ Window window(const Rows& s, int64_t at, int k) {
    Window w;
    if (!MASK) {
        w.from = at + int64_t(k) * V;
        w.lo = 0;
        w.hi = k < s.vpr ? V : 0;
    } else {
        const int phase = int((at + s.lead) & (V - 1));
        w.from = at - phase + int64_t(k) * V;
        const int64_t left = at + s.hw - w.from;
        w.lo = k == 0 ? phase : 0;
        w.hi = left >= V ? V : left > 0 ? int(left) : 0;
    }
    return w;
}
template <int DT, int V, bool MASK>
__device__ __forceinline__ typename Pack<DT, V>::R load(const typename Elt<DT>::T* p, const Window& w, int64_t total) {
    using R = typename Pack<DT, V>::R;
    // the elements beside the row's are other rows', or there are none: nothing outside the tensor is read
    if (!MASK || (w.from >= 0 && w.from + V <= total)) return *reinterpret_cast<const R*>(p + w.from);
    float f[V];
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = j >= w.lo && j < w.hi ? Elt<DT>::load(p, w.from + j) : 0.f;
    return Pack<DT, V>::close(f);
}
template <int DT, int V, bool MASK>
__device__ __forceinline__ void store(typename Elt<DT>::T* p, const Window& w, const float (&f)[V]) {
    using R = typename Pack<DT, V>::R;
    if (!MASK || (w.lo == 0 && w.hi == V)) {
        *reinterpret_cast<R*>(p + w.from) = Pack<DT, V>::close(f);
        return;
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j >= w.lo && j < w.hi) p[w.from + j] = Elt<DT>::from_f(f[j]);
}
template <bool MASK> __device__ __forceinline__ bool in(const Window& w, int j) { return !MASK || (j >= w.lo && j < w.hi); }

// ---- channels last.  A block takes `tile` channels (its threads `cols`
// vectors, a power of two, side by side) and some of the pixels.
struct Cols {
    int c, cg, groups;
    int hw;
    int tile;           // channels of a block
    int tiles;
    int cols_log2;
    int pixels;         // pixels of a block
    int chunks;         // blocks that share the pixels of an image
};

// The sums of the block's channels: s[V] of each thread, over the threads
// that have the same channels; in `ch` [tile] of LDS, `buf` [threads / max(cols,
// 64)][tile].
template <int V>
__device__ __forceinline__ void channel_sums(const float (&s)[V], const Cols& q, int width, float* buf, float* ch) {
    const int cols = 1 << q.cols_log2;
    const int col = threadIdx.x & (cols - 1);
    float t[V];
#pragma unroll
    for (int j = 0; j < V; ++j) t[j] = s[j];
    for (int off = cols; off < 64; off <<= 1)
#pragma unroll
        for (int j = 0; j < V; ++j) t[j] += __shfl_xor(t[j], off);
    const int span_log2 = q.cols_log2 > 6 ? q.cols_log2 : 6;
    const int row = int(threadIdx.x >> span_log2), rows = int(blockDim.x >> span_log2);
    if ((threadIdx.x & 63) < unsigned(cols) && col * V < width)
#pragma unroll
        for (int j = 0; j < V; ++j) buf[row * q.tile + col * V + j] = t[j];
    __syncthreads();
    for (int k = threadIdx.x; k < width; k += blockDim.x) {
        float sum = 0.f;
        for (int i = 0; i < rows; ++i) sum += buf[i * q.tile + k];
        ch[k] = sum;
    }
    __syncthreads();
}

// Sums of the groups of the block's channels, weighted: out[g] for width / cg
// groups, from ch.  A thread per group of few channels, a wave otherwise.
__device__ __forceinline__ void group_sums(const float* ch, const float* weight, int cg, int count, float* out) {
    if (cg <= 16) {
        for (int g = threadIdx.x; g < count; g += blockDim.x) {
            float s = 0.f;
            for (int k = 0; k < cg; ++k) s = fmaf(or_one(weight, g * cg + k), ch[g * cg + k], s);
            out[g] = s;
        }
    } else {
        for (int g = threadIdx.x >> 6; g < count; g += blockDim.x >> 6) {
            float s = 0.f;
            for (int k = threadIdx.x & 63; k < cg; k += 64) s = fmaf(or_one(weight, g * cg + k), ch[g * cg + k], s);
            s = wave_sum(s);
            if ((threadIdx.x & 63) == 0) out[g] = s;
        }
    }
    __syncthreads();
}

struct Params {
    const float* gamma;
    const float* beta;
    int act;
};

// How a call runs (host).  pieces: partial sums of each channel, [n][c][pieces].
struct Plan {
    bool held;          // a block holds its whole groups
    int vec;            // 0: single elements, 1: 16 bytes, 2: 16 bytes with windows
    int k;              // vectors per thread, rounded up to a compiled count
    int threads;
    int64_t grid;
    int pieces;
    Rows rows;
    Cols cols;
};
// Vectors per lane of the kernels that work piece by piece: 16 bytes, single elements.
constexpr int kPiece = 8, kPieceSingle = 32;

template <int DT> void rows_fwd(const Plan& p, int64_t count, const void* x, const Params& q, float eps, void* y,
                                float* mean, float* rstd, float4* parts, hipStream_t st);
template <int DT> void rows_bwd(const Plan& p, int64_t count, const void* x, const void* dy, const Params& q,
                                const float* mean, const float* rstd, void* dx, float2* parts, float2* s12, hipStream_t st);
template <int DT> void cols_fwd(const Plan& p, int n, const void* x, const Params& q, float eps, void* y, float* mean,
                                float* rstd, float4* parts, hipStream_t st);
template <int DT> void cols_bwd(const Plan& p, int n, const void* x, const void* dy, const Params& q, const float* mean,
                                const float* rstd, void* dx, float2* parts, float2* s12, hipStream_t st);
// Between the two passes over pieces (group_norm.hip): the statistics of each
// of `groups` groups, or S1 / M and S2 / M, from its parts.
void combine_fwd(const float4* parts, int64_t groups, int per_group, float eps, float* mean, float* rstd, hipStream_t st);
void combine_bwd(const float2* parts, int64_t groups, int per_group, int pieces, int groups_per_image, int cg, float m,
                 const float* gamma, float2* s12, hipStream_t st);

}  // namespace gn
}  // namespace psc
