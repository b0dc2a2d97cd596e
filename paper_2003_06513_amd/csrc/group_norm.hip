// Group normalisation with an activation, forward and backward, for
// activations in NCHW or with the channels last.
//
// For image n and group g of Cg = C / G channels, over its M = Cg H W values:
//   mu = mean x,  r = 1 / sqrt(var x + eps),  xh = (x - mu) r
//   y  = act(u),  u = gamma[c] xh + beta[c]
// and for the gradient dy of y, with du = dy act'(u):
//   A[n,c] = sum du,  B[n,c] = sum du xh        (over H W)
//   dbeta = sum_n A,  dgamma = sum_n B
//   dx = r (gamma du - (S1 + xh S2) / M),  S1 = sum_c gamma A,  S2 = sum_c gamma B
// Everything is summed in fp32, the variance about the mean.
#include "common.h"
#include "launch.h"

namespace psc {
namespace {

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

__device__ __forceinline__ float block_sum(float x, float* part) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// Where element j of group (n, g), or pixel s of channel c, lies.
struct Shape {
    int c, cg, groups;
    int64_t hw;
    int64_t sc, ss;      // strides of a channel and of a pixel
};

template <int DT>
__global__ __launch_bounds__(256) void k_gn_stats(const typename Elt<DT>::T* __restrict__ x, Shape s, float eps,
                                                  float* __restrict__ mean, float* __restrict__ rstd) {
    __shared__ float part[4];
    const int64_t n = blockIdx.x / s.groups;
    const int g = int(blockIdx.x % s.groups);
    const typename Elt<DT>::T* p = x + n * s.c * s.hw + int64_t(g) * s.cg * s.sc;
    float sum = 0.f;
    for (int c = 0; c < s.cg; ++c)
        for (int64_t i = threadIdx.x; i < s.hw; i += 256) sum += Elt<DT>::load(p, c * s.sc + i * s.ss);
    const float m = float(s.cg) * float(s.hw);
    const float mu = block_sum(sum, part) / m;
    float sq = 0.f;
    for (int c = 0; c < s.cg; ++c)
        for (int64_t i = threadIdx.x; i < s.hw; i += 256) {
            const float d = Elt<DT>::load(p, c * s.sc + i * s.ss) - mu;
            sq = fmaf(d, d, sq);
        }
    sq = block_sum(sq, part);
    if (threadIdx.x == 0) {
        mean[blockIdx.x] = mu;
        rstd[blockIdx.x] = 1.f / sqrtf(sq / m + eps);
    }
}

// One channel of one image per block.
template <int DT>
__global__ __launch_bounds__(256) void k_gn_apply(const typename Elt<DT>::T* __restrict__ x, Shape s,
                                                  const float* __restrict__ gamma, const float* __restrict__ beta,
                                                  const float* __restrict__ mean, const float* __restrict__ rstd,
                                                  int act, typename Elt<DT>::T* __restrict__ y) {
    const int64_t n = blockIdx.x / s.c;
    const int c = int(blockIdx.x % s.c);
    const int64_t at = n * s.c * s.hw + c * s.sc, g = n * s.groups + c / s.cg;
    const float mu = mean[g], r = rstd[g], ga = gamma ? gamma[c] : 1.f, be = beta ? beta[c] : 0.f;
    for (int64_t i = threadIdx.x; i < s.hw; i += 256)
        y[at + i * s.ss] = Elt<DT>::from_f(act_of(affine((Elt<DT>::load(x, at + i * s.ss) - mu) * r, ga, be), act));
}

template <int DT>
__global__ __launch_bounds__(256) void k_gn_sums(const typename Elt<DT>::T* __restrict__ x,
                                                 const typename Elt<DT>::T* __restrict__ dy, Shape s,
                                                 const float* __restrict__ gamma, const float* __restrict__ beta,
                                                 const float* __restrict__ mean, const float* __restrict__ rstd,
                                                 int act, float2* __restrict__ sums) {
    __shared__ float part[4];
    const int64_t n = blockIdx.x / s.c;
    const int c = int(blockIdx.x % s.c);
    const int64_t at = n * s.c * s.hw + c * s.sc, g = n * s.groups + c / s.cg;
    const float mu = mean[g], r = rstd[g], ga = gamma ? gamma[c] : 1.f, be = beta ? beta[c] : 0.f;
    float a = 0.f, b = 0.f;
    for (int64_t i = threadIdx.x; i < s.hw; i += 256) {
        const float xh = (Elt<DT>::load(x, at + i * s.ss) - mu) * r;
        const float du = act_back(affine(xh, ga, be), Elt<DT>::load(dy, at + i * s.ss), act);
        a += du;
        b = fmaf(du, xh, b);
    }
    a = block_sum(a, part);
    b = block_sum(b, part);
    if (threadIdx.x == 0) sums[blockIdx.x] = make_float2(a, b);
}

template <int DT>
__global__ __launch_bounds__(256) void k_gn_dx(const typename Elt<DT>::T* __restrict__ x,
                                               const typename Elt<DT>::T* __restrict__ dy, Shape s,
                                               const float* __restrict__ gamma, const float* __restrict__ beta,
                                               const float* __restrict__ mean, const float* __restrict__ rstd, int act,
                                               const float2* __restrict__ sums, typename Elt<DT>::T* __restrict__ dx) {
    __shared__ float part[4];
    const int64_t n = blockIdx.x / s.c;
    const int c = int(blockIdx.x % s.c), g0 = c / s.cg * s.cg;
    const int64_t at = n * s.c * s.hw + c * s.sc, g = n * s.groups + c / s.cg;
    const float mu = mean[g], r = rstd[g], ga = gamma ? gamma[c] : 1.f, be = beta ? beta[c] : 0.f;
    float s1 = 0.f, s2 = 0.f;
    for (int k = threadIdx.x; k < s.cg; k += 256) {
        const float2 ab = sums[n * s.c + g0 + k];
        const float gk = gamma ? gamma[g0 + k] : 1.f;
        s1 = fmaf(gk, ab.x, s1);
        s2 = fmaf(gk, ab.y, s2);
    }
    const float m = float(s.cg) * float(s.hw);
    s1 = block_sum(s1, part) / m;
    s2 = block_sum(s2, part) / m;
    for (int64_t i = threadIdx.x; i < s.hw; i += 256) {
        const float xh = (Elt<DT>::load(x, at + i * s.ss) - mu) * r;
        const float du = act_back(affine(xh, ga, be), Elt<DT>::load(dy, at + i * s.ss), act);
        dx[at + i * s.ss] = Elt<DT>::from_f(r * (fmaf(ga, du, -s1) - xh * s2));
    }
}

// dbeta and dgamma: the sums of a channel over the images, in their order.
__global__ __launch_bounds__(256) void k_gn_param(const float2* __restrict__ sums, int n, int c,
                                                  float* __restrict__ dgamma, float* __restrict__ dbeta) {
    const int k = blockIdx.x * 256 + threadIdx.x;
    if (k >= c) return;
    float a = 0.f, b = 0.f;
    for (int i = 0; i < n; ++i) {
        const float2 ab = sums[int64_t(i) * c + k];
        a += ab.x;
        b += ab.y;
    }
    if (dgamma) dgamma[k] = b;
    if (dbeta) dbeta[k] = a;
}

Shape shape_of(const GroupNormArgs& a) {
    Shape s;
    s.c = a.c, s.groups = a.groups, s.cg = a.c / a.groups;
    s.hw = int64_t(a.h) * a.w;
    s.sc = a.channels_last ? 1 : s.hw;
    s.ss = a.channels_last ? a.c : 1;
    return s;
}

template <int DT>
hipError_t fwd(const GroupNormArgs& a, const void* x, const float* gamma, const float* beta, float eps, void* y,
               float* mean, float* rstd, void* ws, hipStream_t stream) {
    using T = typename Elt<DT>::T;
    const Shape s = shape_of(a);
    const int64_t ng = int64_t(a.n) * a.groups;
    if (!mean) mean = static_cast<float*>(ws), rstd = mean + ng;
    hipLaunchKernelGGL((k_gn_stats<DT>), dim3(unsigned(ng)), dim3(256), 0, stream, static_cast<const T*>(x), s, eps,
                       mean, rstd);
    hipLaunchKernelGGL((k_gn_apply<DT>), dim3(unsigned(int64_t(a.n) * a.c)), dim3(256), 0, stream,
                       static_cast<const T*>(x), s, gamma, beta, mean, rstd, a.act, static_cast<T*>(y));
    return hipGetLastError();
}

template <int DT>
hipError_t bwd(const GroupNormArgs& a, const void* x, const void* dy, const float* gamma, const float* beta,
               const float* mean, const float* rstd, void* dx, float* dgamma, float* dbeta, void* ws,
               hipStream_t stream) {
    using T = typename Elt<DT>::T;
    const Shape s = shape_of(a);
    float2* sums = static_cast<float2*>(ws);
    const dim3 grid(unsigned(int64_t(a.n) * a.c));
    if (a.n > 0) {
        hipLaunchKernelGGL((k_gn_sums<DT>), grid, dim3(256), 0, stream, static_cast<const T*>(x),
                           static_cast<const T*>(dy), s, gamma, beta, mean, rstd, a.act, sums);
        hipLaunchKernelGGL((k_gn_dx<DT>), grid, dim3(256), 0, stream, static_cast<const T*>(x),
                           static_cast<const T*>(dy), s, gamma, beta, mean, rstd, a.act, sums, static_cast<T*>(dx));
    }
    if (dgamma || dbeta)
        hipLaunchKernelGGL(k_gn_param, dim3(unsigned((a.c + 255) / 256)), dim3(256), 0, stream, sums, a.n, a.c, dgamma,
                           dbeta);
    return hipGetLastError();
}

}  // namespace

size_t group_norm_workspace_bytes(const GroupNormArgs& a, bool backward) {
    const int64_t k = int64_t(a.n) * (backward ? a.c : a.groups);
    return size_t(k) * 2 * sizeof(float);
}

hipError_t launch_group_norm_fwd(const GroupNormArgs& a, const void* x, const float* gamma, const float* beta, float eps,
                                 void* y, float* mean, float* rstd, void* ws, hipStream_t stream) {
    return a.dtype == DT_F16 ? fwd<DT_F16>(a, x, gamma, beta, eps, y, mean, rstd, ws, stream)
                             : fwd<DT_F32>(a, x, gamma, beta, eps, y, mean, rstd, ws, stream);
}

hipError_t launch_group_norm_bwd(const GroupNormArgs& a, const void* x, const void* dy, const float* gamma,
                                 const float* beta, const float* mean, const float* rstd, void* dx, float* dgamma,
                                 float* dbeta, void* ws, hipStream_t stream) {
    return a.dtype == DT_F16 ? bwd<DT_F16>(a, x, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, ws, stream)
                             : bwd<DT_F32>(a, x, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, ws, stream);
}

}  // namespace psc
