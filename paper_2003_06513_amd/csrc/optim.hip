// The optimiser of the retraining (Sec. 3.3): the norm of all gradients and
// the AdamW step, over many tensors in one launch.
//
//   norm   = s sqrt(sum g^2),  factor = s min(1, max_norm / norm)
//   g'     = factor g
//   m      = b1 m + (1 - b1) g',   v = b2 v + (1 - b2) g'^2
//   p      = p - lr wd p - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// The tensors' addresses travel in the kernel's arguments (a table of up to
// kMaxEntries), so nothing is kept between calls and a captured launch holds
// all it needs.
#include <cmath>
#include <cstring>

#include "common.h"
#include "launch.h"

namespace psc {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint16_t h4 __attribute__((ext_vector_type(4)));
typedef int8_t c4 __attribute__((ext_vector_type(4)));
typedef uint8_t b4 __attribute__((ext_vector_type(4)));

// A table of tensors as a kernel argument (the arguments of a launch stay
// under 4 KiB).
constexpr int kMaxEntries = 52;
constexpr int kGroup = 256;       // elements that share the scales of 8-bit moments: 4 per lane of a wave
constexpr int kNormBlocks = 1024; // partial sums of the norm (fixed: deterministic order)

enum : uint32_t { kWide = 1, kGradF16 = 2 };

struct Entry {
    float* p;
    const void* g;
    uint16_t* copy;
    void* m;
    void* v;
    float2* scale;
    int64_t numel;
    float wd;
    uint32_t flags;      // kWide: every pointer is aligned for four elements
};
struct Table {
    Entry e[kMaxEntries];
    int32_t first[kMaxEntries + 1];   // first chunk of each tensor; [n]: the number of chunks
    int32_t n;
};

struct GradEntry {
    const void* g;
    int64_t numel;
    uint32_t flags;
    int32_t first;
};
constexpr int kMaxGrads = 160;
struct GradTable {
    GradEntry e[kMaxGrads];
    int32_t chunks;
    int32_t n;
};

// What a step reads besides the tensors: worked out once on the device, in
// 64 bits, from the count of steps.  In the caller's state, behind the count.
struct Ctl {
    int64_t steps;
    float rate;       // lr / (1 - b1^t)
    float root;       // 1 / sqrt(1 - b2^t)
    float lr;
    float factor;
    int32_t go;       // 0: the factor is not finite, and nothing is changed
    int32_t pad;
};
static_assert(sizeof(Ctl) <= kAdamwStateBytes, "the caller's state holds it");

__global__ void k_adamw_begin(Ctl* __restrict__ ctl, const float* __restrict__ factor, const float* __restrict__ d_lr,
                              float lr, float b1, float b2) {
    const float f = factor ? *factor : 1.f;
    const bool go = __builtin_isfinite(f);
    const int64_t t = ctl->steps + 1;
    if (d_lr) lr = *d_lr;
    ctl->go = go;
    if (!go) return;
    ctl->steps = t;
    ctl->lr = lr;
    ctl->factor = f;
    ctl->rate = float(double(lr) / (1.0 - pow(double(b1), double(t))));
    ctl->root = float(1.0 / sqrt(1.0 - pow(double(b2), double(t))));
}

// The entry whose chunks hold chunk c.
__device__ __forceinline__ int find_entry(const int32_t* first, int n, int c) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= c) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ f4 load_f32(const float* p, int left, bool wide) {
    if (wide && left >= 4) return *reinterpret_cast<const f4*>(p);
    f4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) r[j] = p[j];
    return r;
}
__device__ __forceinline__ void store_f32(float* p, const f4& x, int left, bool wide) {
    if (wide && left >= 4) {
        *reinterpret_cast<f4*>(p) = x;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) p[j] = x[j];
}
template <class V, class T>
__device__ __forceinline__ V load4(const T* p, int left, bool wide) {
    if (wide && left >= 4) return *reinterpret_cast<const V*>(p);
    V r = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) r[j] = p[j];
    return r;
}
template <class V, class T>
__device__ __forceinline__ void store4(T* p, const V& x, int left, bool wide) {
    if (wide && left >= 4) {
        *reinterpret_cast<V*>(p) = x;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) p[j] = x[j];
}
__device__ __forceinline__ f4 load_grad(const void* g, int64_t i, int left, uint32_t flags) {
    const bool wide = flags & kWide;
    if (!(flags & kGradF16)) return load_f32(static_cast<const float*>(g) + i, left, wide);
    const h4 h = load4<h4>(static_cast<const uint16_t*>(g) + i, left, wide);
    f4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint16_t b = h[j];        // of its own: a cast of the element itself reads element 0
        r[j] = float(__builtin_bit_cast(_Float16, b));
    }
    return r;
}

struct Hyper {
    float b1, b2, c1, c2, eps;      // c = 1 - b
};

// p from the new moments.  The quotient by v_rcp_f32 and v_sqrt_f32, each
// within one unit in the last place: the step is at most a few 2^-23 of
// itself off, far below the rounding of p.
__device__ __forceinline__ float updated(float p, float m, float v, float decay, float rate, float root, float eps) {
    const float d = fmaf(__builtin_amdgcn_sqrtf(v), root, eps);
    const float q = fmaf(-decay, p, p);
    return fmaf(-rate * m, __builtin_amdgcn_rcpf(d), q);
}

// One chunk of 1024 elements per block, four in a row per lane.
__global__ __launch_bounds__(256) void k_adamw32(Table tab, Hyper hp, const Ctl* __restrict__ ctl) {
    if (!ctl->go) return;
    const int c = blockIdx.x;
    const int at = find_entry(tab.first, tab.n, c);
    const Entry& e = tab.e[at];
    const int64_t i = int64_t(c - tab.first[at]) * 1024 + threadIdx.x * 4;
    const int64_t rest = e.numel - i;
    if (rest <= 0) return;
    const int left = rest < 4 ? int(rest) : 4;
    const bool wide = e.flags & kWide;
    const float factor = ctl->factor, rate = ctl->rate, root = ctl->root, decay = ctl->lr * e.wd;
    float* mp = static_cast<float*>(e.m) + i;
    float* vp = static_cast<float*>(e.v) + i;
    const f4 g = load_grad(e.g, i, left, e.flags);
    f4 p = load_f32(e.p + i, left, wide), m = load_f32(mp, left, wide), v = load_f32(vp, left, wide);
    h4 h;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float gj = g[j] * factor;
        m[j] = fmaf(hp.b1, m[j], hp.c1 * gj);
        v[j] = fmaf(hp.b2, v[j], hp.c2 * (gj * gj));
        p[j] = updated(p[j], m[j], v[j], decay, rate, root, hp.eps);
        h[j] = Elt<DT_F16>::from_f(p[j]);
    }
    store_f32(e.p + i, p, left, wide);
    store_f32(mp, m, left, wide);
    store_f32(vp, v, left, wide);
    if (e.copy) store4<h4>(e.copy + i, h, left, wide);
}

// ---- moments in 8 bits
//
// A group of 256 elements of m is int8 codes q with one scale a: q stands for
// sign(q) (q / 127)^2 a, where a = max |m|; of v, uint8 codes c for
// (c / 255)^4 a, a = max v.  The powers spend the codes where the values are:
// sqrt(v), which the step divides by, moves by 2/c of itself from code to
// code, m likewise.  The code of x is the number of borders (k - 1/2)^2 (or
// ^4) at or below x 127^2 / a (x 255^4 / a), taken in 64 bits, which this
// machine multiplies as fast as 32: the borders are exact there, so that the
// codes are those of the formula.  A v above zero keeps a code above zero:
// with code 0 the next step would divide by eps alone.
constexpr double kTopM = 127.0 * 127.0, kTopV = 255.0 * 255.0 * 255.0 * 255.0;

__device__ __forceinline__ double decode_m(int q, double a) { return double(q * (q < 0 ? -q : q)) * (a * (1.0 / kTopM)); }
__device__ __forceinline__ double decode_v(uint32_t c, double a) {
    const uint32_t s = c * c;
    return double(s * s) * (a * (1.0 / kTopV));
}
// The root is raised by more than its error, so that the code is right or one
// too high; one look at the border below tells which.
__device__ __forceinline__ int encode_m(double t) {
    int c = int(fmaf(__builtin_amdgcn_sqrtf(float(t)), 1.f + 0x1p-20f, 0.5f));
    const double b = double(c) - 0.5;
    c -= c > 0 && b * b > t;
    return c > 127 ? 127 : c;
}
__device__ __forceinline__ int encode_v(double t) {
    int c = int(fmaf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(float(t))), 1.f + 0x1p-20f, 0.5f));
    const double b = double(c) - 0.5, bb = b * b;
    c -= c > 0 && bb * bb > t;
    return c > 255 ? 255 : c;
}

// The largest of the wave's magnitudes by their bits: a NaN is the largest of all.
__device__ __forceinline__ float wave_peak(uint32_t bits) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const uint32_t o = __shfl_xor(bits, off);
        bits = o > bits ? o : bits;
    }
    return __builtin_bit_cast(float, bits);
}
__device__ __forceinline__ uint32_t magnitude_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// One group per wave: lane l has the elements 4 l .. 4 l + 3 of it.
__global__ __launch_bounds__(256) void k_adamw8(Table tab, Hyper hp, const Ctl* __restrict__ ctl) {
    if (!ctl->go) return;
    const int c = blockIdx.x;
    const int at = find_entry(tab.first, tab.n, c);
    const Entry& e = tab.e[at];
    const int64_t group = int64_t(c - tab.first[at]) * 4 + (threadIdx.x >> 6);
    const int64_t i = group * kGroup + (threadIdx.x & 63) * 4;
    if (group * kGroup >= e.numel) return;      // the whole wave
    const int64_t rest = e.numel - i;
    const int left = rest < 0 ? 0 : rest < 4 ? int(rest) : 4;
    const bool wide = e.flags & kWide;
    const float rate = ctl->rate, root = ctl->root, decay = ctl->lr * e.wd;
    const double factor = ctl->factor, b1 = hp.b1, b2 = hp.b2;
    int8_t* mp = static_cast<int8_t*>(e.m) + i;
    uint8_t* vp = static_cast<uint8_t*>(e.v) + i;
    const float2 peak = e.scale[group];
    const f4 g = load_grad(e.g, i, left, e.flags);
    f4 p = load_f32(e.p + i, left, wide);
    c4 qm = load4<c4>(mp, left, wide);
    b4 qv = load4<b4>(vp, left, wide);
    double m[4], v[4];
    uint32_t top_m = 0, top_v = 0;
    h4 h;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const double gj = double(g[j]) * factor;
        m[j] = b1 * decode_m(qm[j], peak.x) + (1.0 - b1) * gj;
        v[j] = b2 * decode_v(qv[j], peak.y) + (1.0 - b2) * (gj * gj);
        p[j] = updated(p[j], float(m[j]), float(v[j]), decay, rate, root, hp.eps);
        h[j] = Elt<DT_F16>::from_f(p[j]);
        if (j < left) {
            const uint32_t bm = magnitude_bits(float(m[j])), bv = magnitude_bits(float(v[j]));
            top_m = bm > top_m ? bm : top_m;
            top_v = bv > top_v ? bv : top_v;
        }
    }
    store_f32(e.p + i, p, left, wide);
    if (e.copy) store4<h4>(e.copy + i, h, left, wide);
    const float am = wave_peak(top_m), av = wave_peak(top_v);
    const double inv_m = am > 0.f ? kTopM / double(am) : 0.0, inv_v = av > 0.f ? kTopV / double(av) : 0.0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int cm = encode_m(fabs(m[j]) * inv_m), cv = encode_v(v[j] * inv_v);
        qm[j] = int8_t(m[j] < 0 ? -cm : cm);
        qv[j] = uint8_t(cv == 0 && v[j] > 0 ? 1 : cv);
    }
    store4<c4>(mp, qm, left, wide);
    store4<b4>(vp, qv, left, wide);
    if ((threadIdx.x & 63) == 0) e.scale[group] = make_float2(am, av);
}

// The moments that codes stand for: whole groups, four elements per lane.
__global__ __launch_bounds__(256) void k_moments(const int8_t* __restrict__ qm, const uint8_t* __restrict__ qv,
                                                 const float2* __restrict__ scale, int64_t numel, bool wide,
                                                 float* __restrict__ m, float* __restrict__ v) {
    const int64_t i = int64_t(blockIdx.x) * 1024 + threadIdx.x * 4;
    const int64_t rest = numel - i;
    if (rest <= 0) return;
    const int left = rest < 4 ? int(rest) : 4;
    const c4 a = load4<c4>(qm + i, left, wide);
    const b4 b = load4<b4>(qv + i, left, wide);
    const float2 peak = scale[i / kGroup];
    f4 x, y;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[j] = float(decode_m(a[j], peak.x));
        y[j] = float(decode_v(b[j], peak.y));
    }
    store_f32(m + i, x, left, wide);
    store_f32(v + i, y, left, wide);
}

// ---- the norm: squares in 64 bits, so that no finite gradient overflows or
// vanishes; one partial sum per block, added in a fixed order.
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double part[4];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(256) void k_norm_parts(GradTable tab, bool add, double* __restrict__ part) {
    double acc = 0.0;
    for (int c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
        int lo = 0, hi = tab.n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (tab.e[mid].first <= c) lo = mid; else hi = mid;
        }
        const GradEntry& e = tab.e[lo];
        const int64_t i = int64_t(c - e.first) * 1024 + threadIdx.x * 4;
        const int64_t rest = e.numel - i;
        if (rest <= 0) continue;
        const f4 g = load_grad(e.g, i, rest < 4 ? int(rest) : 4, e.flags);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = fma(double(g[j]), double(g[j]), acc);
    }
    acc = block_sum(acc);
    if (threadIdx.x == 0) part[blockIdx.x] = add ? part[blockIdx.x] + acc : acc;
}

__global__ __launch_bounds__(256) void k_norm_end(const double* __restrict__ part, int n, float scale, float max_norm,
                                                  float* __restrict__ out) {
    double acc = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) acc += part[i];
    acc = block_sum(acc);
    if (threadIdx.x == 0) {
        const double norm = double(scale) * sqrt(acc);
        out[0] = float(norm);
        // a norm that is not finite has no factor: the step that reads it leaves everything as it was
        out[1] = !__builtin_isfinite(float(norm)) ? __builtin_nanf("")
                                                  : float(double(scale) * (norm > double(max_norm) ? double(max_norm) / norm : 1.0));
    }
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

uint32_t grad_flags(const ParamView& q) {
    const bool half = q.grad_dtype == DT_F16;
    return (half ? kGradF16 : 0u) | (aligned(q.grad, half ? 8 : 16) ? kWide : 0u);
}

}  // namespace

size_t grad_norm_workspace_bytes() { return size_t(kNormBlocks) * sizeof(double); }

hipError_t launch_grad_norm(const ParamView* q, int count, float scale, float max_norm, float* out, void* ws,
                            hipStream_t stream) {
    double* part = static_cast<double*>(ws);
    int64_t most = 1;       // chunks of the largest launch: every launch of the call has one grid
    int64_t sum = 0;
    int in = 0;
    for (int i = 0; i < count; ++i) {
        const int64_t ch = (q[i].numel + 1023) / 1024;
        if (ch == 0) continue;
        if (in == kMaxGrads || sum + ch > (int64_t(1) << 30)) sum = 0, in = 0;
        sum += ch, ++in;
        most = sum > most ? sum : most;
    }
    const int grid = int(most < kNormBlocks ? most : kNormBlocks);
    GradTable tab;
    tab.n = 0, tab.chunks = 0;
    bool add = false;
    const auto flush = [&] {
        hipLaunchKernelGGL(k_norm_parts, dim3(unsigned(grid)), dim3(256), 0, stream, tab, add, part);
        add = true;
        tab.n = 0, tab.chunks = 0;
    };
    for (int i = 0; i < count; ++i) {
        const int64_t ch = (q[i].numel + 1023) / 1024;
        if (ch == 0) continue;
        if (tab.n == kMaxGrads || tab.chunks + ch > (int64_t(1) << 30)) flush();
        tab.e[tab.n++] = GradEntry{q[i].grad, q[i].numel, grad_flags(q[i]), tab.chunks};
        tab.chunks += int32_t(ch);
    }
    if (tab.n || !add) flush();
    hipLaunchKernelGGL(k_norm_end, dim3(1), dim3(256), 0, stream, part, grid, scale, max_norm, out);
    return hipGetLastError();
}

hipError_t launch_adamw(const ParamView* q, int count, const AdamwArgs& a, const float* factor, void* state,
                        hipStream_t stream) {
    Ctl* ctl = static_cast<Ctl*>(state);
    hipLaunchKernelGGL(k_adamw_begin, dim3(1), dim3(1), 0, stream, ctl, factor, a.d_lr, a.lr, a.beta1, a.beta2);
    const Hyper hp{a.beta1, a.beta2, float(1.0 - double(a.beta1)), float(1.0 - double(a.beta2)), a.eps};
    for (int bits : {32, 8}) {
        Table tab;
        tab.n = 0, tab.first[0] = 0;
        const auto flush = [&] {
            if (tab.n == 0) return;
            const dim3 grid(unsigned(tab.first[tab.n]));
            if (bits == 32) hipLaunchKernelGGL(k_adamw32, grid, dim3(256), 0, stream, tab, hp, ctl);
            else hipLaunchKernelGGL(k_adamw8, grid, dim3(256), 0, stream, tab, hp, ctl);
            tab.n = 0;
        };
        for (int i = 0; i < count; ++i) {
            if (q[i].state_bits != bits || q[i].numel == 0) continue;
            const int64_t ch = (q[i].numel + 1023) / 1024;
            if (tab.n == kMaxEntries || (tab.n && tab.first[tab.n] + ch > (int64_t(1) << 30))) flush();
            uint32_t flags = grad_flags(q[i]);
            const size_t am = bits == 32 ? 16 : 4;
            if (!aligned(q[i].param, 16) || !aligned(q[i].m, am) || !aligned(q[i].v, am) || !aligned(q[i].copy, 8))
                flags &= ~uint32_t(kWide);
            tab.e[tab.n] = Entry{q[i].param, q[i].grad, static_cast<uint16_t*>(q[i].copy), q[i].m, q[i].v,
                                 static_cast<float2*>(static_cast<void*>(q[i].scale)), q[i].numel, q[i].weight_decay, flags};
            tab.first[tab.n + 1] = tab.first[tab.n] + int32_t(ch);
            ++tab.n;
        }
        flush();
    }
    return hipGetLastError();
}

hipError_t launch_moments(const int8_t* qm, const uint8_t* qv, const float* scale, int64_t numel, float* m, float* v,
                          hipStream_t stream) {
    const bool wide = aligned(qm, 4) && aligned(qv, 4) && aligned(m, 16) && aligned(v, 16);
    hipLaunchKernelGGL(k_moments, dim3(unsigned((numel + 1023) / 1024)), dim3(256), 0, stream, qm, qv,
                       static_cast<const float2*>(static_cast<const void*>(scale)), numel, wide, m, v);
    return hipGetLastError();
}

}  // namespace psc
