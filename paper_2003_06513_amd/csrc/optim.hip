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
//
// The times in these comments compare two forms in one sitting.  From sitting to
// sitting the largest differ by some percent (64 x 512 x 512 x 9 with 8 bits: 443
// to 480 us).
#include <cmath>
#include <cstring>

#include "common.h"
#include "launch.h"

namespace psc {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef uint16_t h4 __attribute__((ext_vector_type(4)));
typedef int8_t c4 __attribute__((ext_vector_type(4)));
typedef uint8_t b4 __attribute__((ext_vector_type(4)));

// A table of tensors as a kernel argument (the arguments of a launch stay
// under 4 KiB).  Chunks of 1024 elements are numbered through the table, and a
// block of a step takes one: blocks that go on to other chunks were slower (64
// x 512 x 512 x 9 with 32 bits 869 us, not 783), as were chunks of 2048 (802).
constexpr int kMaxEntries = 83;
constexpr int kGroup = 256;       // elements that share the scales of 8-bit moments: 4 per lane of a wave
constexpr int kNormBlocks = 1024; // partial sums of the norm (fixed: deterministic order)
// Chunks that one block takes by itself, in one launch: 8.9 -> 5.9 us a call, in
// a captured chain 4.2 -> 4.6; with 32 of them, of as many tensors, 4.2 -> 8.
constexpr int kNormAlone = 16;

enum : uint32_t { kWide = 1, kGradF16 = 2 };

// A tensor in 44 bytes, so that many fit: the addresses' low and high halves
// (they have 48 bits), the flags in bits that are free.  161 tensors, 10 M
// elements with 8 bits: 42 us, with 58 entries of 64 bytes 45 (64 x 512 x 512 x
// 9, where the bytes decide: 472 and 464).
enum : int { kParam, kGrad, kCopy, kM, kV, kScale, kAddresses };
struct Entry {
    uint32_t lo[kAddresses], hi[kAddresses / 2];
    uint32_t size;          // bit 31: kWide, every pointer is aligned for four elements
    float wd;
};
// The same as the kernels use it.
struct Tensor {
    float* p;
    const void* g;
    uint16_t* copy;
    void *m, *v;
    float2* scale;
    uint32_t numel, flags;
    float wd;
};
template <class T> __device__ __forceinline__ T* address(const Entry& e, int k, uint32_t clear = 0u) {
    const uint32_t high = e.hi[k / 2] >> (16 * (k & 1)) & 0xffffu;
    // as an address of global memory: loads and stores of any would go by the LDS too
    return (T*)(__attribute__((address_space(1))) T*)(uint64_t(high) << 32 | (e.lo[k] & ~clear));
}
__device__ __forceinline__ Tensor tensor(const Entry& e) {
    Tensor t;
    t.p = address<float>(e, kParam);
    t.g = address<const void>(e, kGrad, 1u);
    t.copy = address<uint16_t>(e, kCopy);
    t.m = address<void>(e, kM), t.v = address<void>(e, kV);
    t.scale = address<float2>(e, kScale);
    t.numel = e.size & 0x7fffffffu;
    t.flags = (e.size >> 31 ? kWide : 0u) | (e.lo[kGrad] & 1u ? kGradF16 : 0u);
    t.wd = e.wd;
    return t;
}
// first[i]: the first chunk of tensor i; where there is none, past all chunks.
struct Table {
    uint32_t first[kMaxEntries + 1];
    Entry e[kMaxEntries];
    int32_t n;
    uint32_t chunks;
};

struct GradEntry {
    const void* g;
    uint32_t numel;
    uint32_t flags;
};
constexpr int kMaxGrads = 192;
struct GradTable {
    uint32_t first[kMaxGrads];
    GradEntry e[kMaxGrads];
    int32_t n;
    uint32_t chunks;
};
static_assert(sizeof(Entry) == 44 && sizeof(Table) <= 4000 && sizeof(GradTable) <= 4000, "kernel arguments");

// The caller's state.  The last block of a step's last launch to read the
// count raises it.  The blocks are counted at kEnds words, each in a line of
// its own, and the last ones of those at one more (additions to one word take
// 9 ns each: 20 us for 2149 blocks).  All are zero between steps.
constexpr int kEnds = 32;
struct alignas(128) Line {
    uint32_t ended;
};
struct State {
    int64_t steps;
    Line all, some[kEnds];
};
static_assert(sizeof(State) <= kAdamwStateBytes, "the caller's state holds it");

struct Hyper {
    float b1, b2, c1, c2, eps, lr;      // c = 1 - b
    float ln1, ln2;                     // log b
    const float* d_lr;
    const float* factor;
};
__device__ __forceinline__ bool last_of(Line& line, uint32_t count) {
    if (atomicAdd(&line.ended, 1u) != count - 1) return false;
    atomicExch(&line.ended, 0u);
    return true;
}
// What a step takes from the count of steps and from device memory.  1 - b^t
// is -expm1(t log b): nothing cancels where b^t is near one.  One wave works
// it out for the block.
struct Now {
    float factor, rate, root, lr;
    bool go;             // the factor and the rate are finite; else nothing is changed
};
__device__ __forceinline__ Now now(const Hyper& hp, State* st, bool last) {
    __shared__ float both[2];
    Now n;
    n.factor = hp.factor ? *hp.factor : 1.f;
    n.lr = hp.d_lr ? *hp.d_lr : hp.lr;
    n.go = __builtin_isfinite(n.factor) && __builtin_isfinite(n.lr);
    int64_t steps = 0;
    if (threadIdx.x < 64) {
        steps = st->steps;
        const float t = float(steps + 1);
        const float rate = n.lr / -expm1f(t * hp.ln1), root = 1.f / sqrtf(-expm1f(t * hp.ln2));
        if (threadIdx.x == 0) both[0] = rate, both[1] = root;
    }
    __syncthreads();
    n.rate = both[0];
    n.root = both[1];
    // the block has read the count: behind the barrier, that waited for what came of it
    if (last && n.go && threadIdx.x == 0) {
        const uint32_t at = blockIdx.x % kEnds, blocks = gridDim.x;
        if (last_of(st->some[at], (blocks - at + kEnds - 1) / kEnds) && last_of(st->all, blocks < kEnds ? blocks : kEnds))
            st->steps = steps + 1;
    }
    return n;
}

// The tensor that chunk c belongs to: every lane looks at one tensor's first
// chunk (or a few), so that one load is waited for; a binary search waits for
// one after the other (161 tensors, 10 M elements with 8 bits: 57 us, not 53).
struct Found {
    int at;
    uint32_t first;
};
template <int N> __device__ __forceinline__ Found find_entry(const uint32_t (&first)[N], uint32_t c) {
    constexpr int R = (N + 63) / 64;
    const int lane = int(threadIdx.x & 63);
    uint32_t f[R];
#pragma unroll
    for (int i = 0; i < R; ++i) f[i] = first[i * 64 + lane < N ? i * 64 + lane : N - 1];
    int at = -1;
#pragma unroll
    for (int i = 0; i < R; ++i) at += __popcll(__ballot((i * 64 + lane < N) & (f[i] <= c)));
    at = __builtin_amdgcn_readfirstlane(at);
    uint32_t v = f[0];
#pragma unroll
    for (int i = 1; i < R; ++i) v = at >= i * 64 ? f[i] : v;
    return Found{at, uint32_t(__builtin_amdgcn_readlane(int(v), at & 63))};
}

// Four elements, as far as there are any.  What a step reads and writes goes
// past the caches: it is touched once (161 tensors of 10 M elements: 67 -> 57
// us with 32 bits, 54 -> 45 with 8; 64 x 512 x 512 x 9: 778 -> 747, 468 -> 455).
template <class V, bool PAST, class T>
__device__ __forceinline__ V load4(const T* p, int left, bool wide) {
    if (wide && left >= 4) {
        const V* q = reinterpret_cast<const V*>(p);
        if constexpr (PAST) return __builtin_nontemporal_load(q);
        else return *q;
    }
    V r = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) r[j] = p[j];
    return r;
}
template <class V, class T>
__device__ __forceinline__ void store4(T* p, const V& x, int left, bool wide) {
    if (wide && left >= 4) {
        __builtin_nontemporal_store(x, reinterpret_cast<V*>(p));
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) p[j] = x[j];
}
__device__ __forceinline__ f4 widened(const h4& h) {
    f4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint16_t b = h[j];        // of its own: a cast of the element itself reads element 0
        r[j] = float(__builtin_bit_cast(_Float16, b));
    }
    return r;
}
// Four gradients as they lie in memory; opened where they are needed, so that
// nothing is waited for between the loads of a block.
template <bool PAST>
__device__ __forceinline__ f4 load_grad(const void* g, int64_t i, int left, uint32_t flags) {
    const bool wide = flags & kWide;
    if (!(flags & kGradF16)) return load4<f4, PAST>(static_cast<const float*>(g) + i, left, wide);
    const f2 raw = __builtin_bit_cast(f2, load4<h4, PAST>(static_cast<const uint16_t*>(g) + i, left, wide));
    return f4{raw.x, raw.y, 0.f, 0.f};
}
__device__ __forceinline__ f4 opened(const f4& raw, uint32_t flags) {
    if (!(flags & kGradF16)) return raw;
    const f2 half = {raw.x, raw.y};
    return widened(__builtin_bit_cast(h4, half));
}

// sqrt(v) root + eps, by v_sqrt_f32, which is within one unit in the last place
// but takes a v below 2^-126 for zero: a small one is scaled by 2^192 first (8
// bits: in fp64, where codes far below their group's largest are less than
// fp32's least).  A zero needs no scaling, and is common; of the others a wave
// rarely has any.
template <class T>
__device__ __forceinline__ void denominators(const T (&v)[4], float root, float eps, float (&d)[4]) {
    constexpr int up = sizeof(T) == 8 ? 192 : 96;
    constexpr T least = T(0x1p-96);
    bool small = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        d[j] = fmaf(__builtin_amdgcn_sqrtf(float(v[j])), root, eps);
        small |= (v[j] < least) & (v[j] > T(0));
    }
    if (small) {
        const T scale = up == 192 ? T(0x1p192) : T(0x1p96f);
        const float less = root * (up == 192 ? 0x1p-96f : 0x1p-48f);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (v[j] < least) d[j] = fmaf(__builtin_amdgcn_sqrtf(float(v[j] * scale)), less, eps);
    }
}
// p from the new m and sqrt(v) / sqrt(1 - b2^t) + eps.  The quotient by
// v_rcp_f32, which is within one unit in the last place (d is at least
// FLT_MIN): the step is at most a few 2^-23 of itself off, far below the
// rounding of p.  m by the reciprocal first: the rate times m may be subnormal.
__device__ __forceinline__ float updated(float p, float m, float d, float decay, float rate) {
    const float q = fmaf(-decay, p, p);
    return fmaf(-rate, m * __builtin_amdgcn_rcpf(d), q);
}

// A step of nothing.
__global__ void k_adamw_none(Hyper hp, State* __restrict__ st) {
    if (hp.factor && !__builtin_isfinite(*hp.factor)) return;
    if (hp.d_lr && !__builtin_isfinite(*hp.d_lr)) return;
    st->steps = st->steps + 1;
}

// Four elements in a row per lane.
__global__ __launch_bounds__(256) void k_adamw32(Table tab, Hyper hp, State* __restrict__ st, bool last) {
    const Found found = find_entry(tab.first, blockIdx.x);
    const Tensor e = tensor(tab.e[found.at]);
    const uint32_t i = (blockIdx.x - found.first) * 1024 + threadIdx.x * 4;
    const int left = i >= e.numel ? 0 : e.numel - i < 4 ? int(e.numel - i) : 4;
    const bool wide = e.flags & kWide;
    float* mp = static_cast<float*>(e.m) + i;
    float* vp = static_cast<float*>(e.v) + i;
    const f4 raw = load_grad<true>(e.g, i, left, e.flags);
    f4 p = load4<f4, true>(e.p + i, left, wide), m = load4<f4, true>(mp, left, wide), v = load4<f4, true>(vp, left, wide);
    const Now n = now(hp, st, last);        // while those are on their way
    if (!n.go) return;
    const f4 g = opened(raw, e.flags);
    const float decay = n.lr * e.wd;
    float w[4], d[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float gj = g[j] * n.factor;
        m[j] = fmaf(hp.b1, m[j], hp.c1 * gj);
        w[j] = fmaf(hp.b2, v[j], hp.c2 * gj * gj);      // in this order: the square may pass fp32 where this does not
    }
    denominators(w, n.root, hp.eps, d);
    h4 h;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = w[j];
        p[j] = updated(p[j], m[j], d[j], decay, n.rate);
        h[j] = Elt<DT_F16>::from_f(p[j]);
    }
    store4<f4>(e.p + i, p, left, wide);
    store4<f4>(mp, m, left, wide);
    store4<f4>(vp, v, left, wide);
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
// machine multiplies as fast as 32.  The borders are exact there; the product
// has two roundings, and is raised by more than those (2^-50 of itself), so
// that an x on a border, as gradients of few bits and betas of 0 or 1/2 put
// one, has the code above it.  A v above zero keeps a code above zero: with
// code 0 the next step would divide by eps alone.
constexpr double kTopM = 127.0 * 127.0, kTopV = 255.0 * 255.0 * 255.0 * 255.0;
constexpr double kRaise = 1.0 + 0x1p-50;

// Whole numbers in 64 bits: laid behind the exponent of 2^52 and that taken
// away.  A conversion takes as long as four such operations; with them, the
// peaks by the LDS and a division each 64 x 512 x 512 x 9 took 456 us, not 443.
__device__ __forceinline__ double whole(uint32_t n) {
    return __builtin_bit_cast(double, uint64_t(0x43300000u) << 32 | n) - 0x1p52;
}
__device__ __forceinline__ double whole_signed(int n) {
    return __builtin_bit_cast(double, uint64_t(0x43300000u) << 32 | (uint32_t(n) ^ 0x80000000u)) - (0x1p52 + 0x1p31);
}
// q |q| and c^4, which times the scale and 1 / kTop are the values.
__device__ __forceinline__ double power_m(int q) { return whole_signed(q * (q < 0 ? -q : q)); }
__device__ __forceinline__ double power_v(uint32_t c) {
    const uint32_t s = c * c;
    return whole(s * s);
}
// Codes from 4 |m| 127^2 / a and 16 v 255^4 / a (raised), and these in 32 bits.  The
// root is raised by more than its error, so that the code is right or one too
// high; one look at the border below, (2 c - 1)^2 or ^4, tells which.
__device__ __forceinline__ int encode_m(double t4, float near) {
    int c = int(fmaf(__builtin_amdgcn_sqrtf(near), 0.5f + 0x1p-21f, 0.5f));
    const uint32_t b = uint32_t(2 * c - 1) & 0x3ffu;
    c -= c > 0 && whole(b * b) > t4;
    return c > 127 ? 127 : c;
}
__device__ __forceinline__ int encode_v(double t16, float near) {
    int c = int(fmaf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(near)), 0.5f + 0x1p-21f, 0.5f));
    const uint32_t b = uint32_t(2 * c - 1) & 0x3ffu;
    const double bb = whole(b * b);
    c -= c > 0 && bb * bb > t16;
    return c > 255 ? 255 : c;
}

// The largest of the wave's magnitudes by their bits, by moves within the
// register file: a NaN is the largest of all.
template <int OFF> __device__ __forceinline__ uint32_t lane_max(uint32_t x) {
    uint32_t a = x, b;
    if constexpr (OFF == 16 || OFF == 32) {
        const auto r = OFF == 16 ? __builtin_amdgcn_permlane16_swap(x, x, false, false)
                                 : __builtin_amdgcn_permlane32_swap(x, x, false, false);
        a = r[0], b = r[1];
    } else {
        // quad_perm [1,0,3,2] and [2,3,0,1], row_half_mirror, row_mirror
        constexpr int ctrl = OFF == 1 ? 0xB1 : OFF == 2 ? 0x4E : OFF == 4 ? 0x141 : 0x140;
        b = uint32_t(__builtin_amdgcn_update_dpp(0, int(x), ctrl, 0xf, 0xf, true));
    }
    return a > b ? a : b;
}
__device__ __forceinline__ float wave_peak(uint32_t x) {
    x = lane_max<1>(x), x = lane_max<2>(x), x = lane_max<4>(x), x = lane_max<8>(x);
    x = lane_max<32>(lane_max<16>(x));
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(int(x)));
}
__device__ __forceinline__ double of_lane(double x, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = uint32_t(__builtin_amdgcn_readlane(int(uint32_t(b)), lane)),
                   hi = uint32_t(__builtin_amdgcn_readlane(int(uint32_t(b >> 32)), lane));
    return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
__device__ __forceinline__ uint32_t magnitude_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// One group per wave: lane l has the elements 4 l .. 4 l + 3 of it.
__global__ __launch_bounds__(256) void k_adamw8(Table tab, Hyper hp, State* __restrict__ st, bool last) {
    const Found found = find_entry(tab.first, blockIdx.x);
    const Tensor e = tensor(tab.e[found.at]);
    const uint32_t group = (blockIdx.x - found.first) * 4 + (threadIdx.x >> 6), lane4 = (threadIdx.x & 63) * 4;
    const uint32_t i = group * kGroup + lane4;
    const int left = i >= e.numel ? 0 : e.numel - i < 4 ? int(e.numel - i) : 4;
    const bool wide = e.flags & kWide;
    int8_t* mp = static_cast<int8_t*>(e.m) + i;
    uint8_t* vp = static_cast<uint8_t*>(e.v) + i;
    const float2 peak = e.scale[group * kGroup < e.numel ? group : 0];
    const f4 raw = load_grad<true>(e.g, i, left, e.flags);
    f4 p = load4<f4, true>(e.p + i, left, wide);
    c4 qm = load4<c4, true>(mp, left, wide);
    b4 qv = load4<b4, true>(vp, left, wide);
    const Now n = now(hp, st, last);        // while those are on their way
    if (!n.go || group * kGroup >= e.numel) return;     // the whole wave
    const f4 g = opened(raw, e.flags);
    const float decay = n.lr * e.wd;
    const double factor = n.factor;
    const double km = hp.b1 * (1.0 / kTopM) * peak.x, kv = hp.b2 * (1.0 / kTopV) * peak.y,
                 kg = (1.0 - hp.b1) * factor, kgg = (1.0 - hp.b2) * factor * factor;
    double m[4], v[4];
    uint32_t top_m = 0, top_v = 0;
    h4 h;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const double gj = g[j];
        m[j] = fma(power_m(qm[j]), km, gj * kg);
        v[j] = fma(power_v(qv[j]), kv, gj * gj * kgg);
    }
    float d[4];
    denominators(v, n.root, hp.eps, d);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        p[j] = updated(p[j], float(m[j]), d[j], decay, n.rate);
        h[j] = Elt<DT_F16>::from_f(p[j]);
        if (j < left) {
            const uint32_t bm = magnitude_bits(float(m[j])), bv = magnitude_bits(float(v[j]));
            top_m = bm > top_m ? bm : top_m;
            top_v = bv > top_v ? bv : top_v;
        }
    }
    store4<f4>(e.p + i, p, left, wide);
    if (e.copy) store4<h4>(e.copy + i, h, left, wide);
    const float am = wave_peak(top_m), av = wave_peak(top_v);
    // one division for both: the even lanes' and the odd lanes'
    const bool odd = threadIdx.x & 1;
    const float a = odd ? av : am;
    const double inv = a > 0.f ? (odd ? 16.0 * kRaise * kTopV : 4.0 * kRaise * kTopM) / double(a) : 0.0;
    const double inv_m = of_lane(inv, 0), inv_v = of_lane(inv, 1);
    // in 32 bits from products of 32 where none of them overflows
    const bool plain = am > 0x1p-80f && av > 0x1p-80f && am < 0x1p80f && av < 0x1p80f;
    const float near_m = float(inv_m), near_v = float(inv_v);
    f4 nm, nv;
#pragma unroll
    for (int j = 0; j < 4; ++j) nm[j] = fabsf(float(m[j])) * near_m, nv[j] = float(v[j]) * near_v;
    if (!plain) {
        asm volatile("");       // a branch: as selections both ways would be worked out
#pragma unroll
        for (int j = 0; j < 4; ++j) nm[j] = float(fabs(m[j]) * inv_m), nv[j] = float(v[j] * inv_v);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int cm = encode_m(fabs(m[j]) * inv_m, nm[j]), cv = encode_v(v[j] * inv_v, nv[j]);
        qm[j] = int8_t(m[j] < 0 ? -cm : cm);
        qv[j] = uint8_t(cv == 0 && v[j] > 0 ? 1 : cv);
    }
    store4<c4>(mp, qm, left, wide);
    store4<b4>(vp, qv, left, wide);
    if (lane4 == 0) e.scale[group] = make_float2(am, av);
}

// The moments that codes stand for: whole groups, four elements per lane.
__global__ __launch_bounds__(256) void k_moments(const int8_t* __restrict__ qm, const uint8_t* __restrict__ qv,
                                                 const float2* __restrict__ scale, int64_t numel, bool wide,
                                                 float* __restrict__ m, float* __restrict__ v) {
    const int64_t i = int64_t(blockIdx.x) * 1024 + threadIdx.x * 4;
    const int64_t rest = numel - i;
    if (rest <= 0) return;
    const int left = rest < 4 ? int(rest) : 4;
    const c4 a = load4<c4, false>(qm + i, left, wide);
    const b4 b = load4<b4, false>(qv + i, left, wide);
    const float2 peak = scale[i / kGroup];
    f4 x, y;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[j] = float(power_m(a[j]) * (peak.x * (1.0 / kTopM)));
        y[j] = float(power_v(b[j]) * (peak.y * (1.0 / kTopV)));
    }
    store4<f4>(m + i, x, left, wide);
    store4<f4>(v + i, y, left, wide);
}

// ---- the norm.  Sums in 64 bits, one partial sum per block, added in a fixed
// order; no finite gradient's square overflows or vanishes.  An fp32 one is
// squared in 64 bits.  An fp16 one has an exact square in 32, whose bits, moved
// up by 29, are those of a double 2^896 times smaller: a conversion takes as
// long as four other operations, and with one for every element 64 x 512 x 512
// x 9 took 164 us, not 51.  (Four squares added in 32 bits first, as fast, were
// not exact enough: the clip factor's last bit decides codes of 8-bit moments.)
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double part[16];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
    for (unsigned i = 0; i < blockDim.x >> 6; i += 4) x += (part[i] + part[i + 1]) + (part[i + 2] + part[i + 3]);
    return x;
}

struct Squares {
    double sum = 0.0, tiny = 0.0;       // tiny: 2^-896 of the fp16 squares
    float rough = 0.f;                  // of those, whether any is not finite: no sum of finite ones overflows
    __device__ __forceinline__ void add(const f4& g, bool half) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (half) {
                const float q = g[j] * g[j];
                const uint32_t b = __builtin_bit_cast(uint32_t, q);
                tiny += __builtin_bit_cast(double, uint64_t(b) << 29);
                rough += q;
            } else {
                sum = fma(double(g[j]), double(g[j]), sum);
            }
        }
    }
    __device__ __forceinline__ double all() const {
        const double s = fma(tiny, 0x1p896, sum);
        return __builtin_isfinite(rough) ? s : s + double(rough);
    }
};

struct Clip {
    float scale, max_norm;
    float* out;
};
__device__ __forceinline__ void clip(const Clip& k, double squares) {
    const double norm = double(k.scale) * sqrt(squares);
    k.out[0] = float(norm);
    // a norm that is not finite has no factor: the step that reads it leaves everything as it was
    k.out[1] = !__builtin_isfinite(float(norm))
                   ? __builtin_nanf("")
                   : float(double(k.scale) * (norm > double(k.max_norm) ? double(k.max_norm) / norm : 1.0));
}

// 256 threads' chunks lie side by side, so that they go through the table once;
// inside a tensor they load kAhead of them before it adds the first (one by one
// too little is on its way: 64 x 512 x 512 x 9 fp16 115 us, not 51).
constexpr int kAhead = 8;
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm_parts(GradTable tab, bool add, double* __restrict__ part, Clip alone) {
    Squares acc;
    const uint32_t all = gridDim.x * (THREADS / 256), per = (tab.chunks + all - 1) / all;
    // the same for a whole wave, which the compiler has to know: 51 us, not 76, on 64 x 512 x 512 x 9 fp16
    uint32_t c = (blockIdx.x * (THREADS / 256) + uint32_t(__builtin_amdgcn_readfirstlane(int(threadIdx.x >> 8)))) * per;
    const uint32_t c1 = c + per < tab.chunks ? c + per : tab.chunks;
    Found found = find_entry(tab.first, c);
    while (c < c1) {
        if (found.at + 1 < tab.n && tab.first[found.at + 1] == c) ++found.at, found.first = c;      // every tensor of the table has a chunk
        const GradEntry& e = tab.e[found.at];
        const uint32_t chunk = c - found.first, i = chunk * 1024 + (threadIdx.x & 255) * 4;
        const bool half = e.flags & kGradF16;
        if ((e.flags & kWide) && c + kAhead <= c1 && (chunk + kAhead) * 1024 <= e.numel) {
            if (half) {
                h4 g[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) g[u] = *reinterpret_cast<const h4*>(static_cast<const uint16_t*>(e.g) + i + u * 1024);
#pragma unroll
                for (int u = 0; u < kAhead; ++u) acc.add(widened(g[u]), true);
            } else {
                f4 g[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) g[u] = *reinterpret_cast<const f4*>(static_cast<const float*>(e.g) + i + u * 1024);
#pragma unroll
                for (int u = 0; u < kAhead; ++u) acc.add(g[u], false);
            }
            c += kAhead;
        } else {
            if (i < e.numel)
                acc.add(opened(load_grad<false>(e.g, i, e.numel - i < 4 ? int(e.numel - i) : 4, e.flags), e.flags), half);
            ++c;
        }
    }
    const double sum = block_sum(acc.all());
    if (threadIdx.x != 0) return;
    if (alone.out) clip(alone, sum);
    else part[blockIdx.x] = add ? part[blockIdx.x] + sum : sum;
}

__global__ __launch_bounds__(256) void k_norm_end(const double* __restrict__ part, int n, Clip k) {
    double acc = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) acc += part[i];
    acc = block_sum(acc);
    if (threadIdx.x == 0) clip(k, acc);
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

uint32_t grad_flags(const ParamView& q) {
    const bool half = q.grad_dtype == DT_F16;
    return (half ? kGradF16 : 0u) | (aligned(q.grad, half ? 8 : 16) ? kWide : 0u);
}

}  // namespace

size_t grad_norm_workspace_bytes() { return size_t(kNormBlocks) * sizeof(double); }

namespace {
// Tables are filled up to their room and to 2^23 chunks (a launch has fewer than 2^32 threads).
template <class T> bool full(const T& tab, int room, int64_t more) { return tab.n == room || tab.chunks + more > (int64_t(1) << 23); }
template <class T> void clear(T& tab) {
    tab.n = 0, tab.chunks = 0;
    for (uint32_t& f : tab.first) f = ~0u;
}
template <class T, class E> void add_entry(T& tab, const E& e, int64_t chunks) {
    tab.first[tab.n] = tab.chunks;
    tab.e[tab.n++] = e;
    tab.chunks += uint32_t(chunks);
}
int64_t chunks_of(const ParamView& q) { return (q.numel + 1023) / 1024; }
}  // namespace

hipError_t launch_grad_norm(const ParamView* q, int count, float scale, float max_norm, float* out, void* ws,
                            hipStream_t stream) {
    double* part = static_cast<double*>(ws);
    GradTable tab;
    clear(tab);
    // Every launch of the call writes or adds the same partial sums: as many as
    // the chunks of all tensors, as far as there is room.
    int64_t all = 0;
    for (int i = 0; i < count; ++i) all += chunks_of(q[i]);
    const int grid = int(all < 1 ? 1 : all < kNormBlocks ? all : kNormBlocks);
    const Clip whole{scale, max_norm, out}, none{scale, max_norm, nullptr};
    bool add = false;
    const auto flush = [&] {
        if (all <= kNormAlone)
            hipLaunchKernelGGL(k_norm_parts<1024>, dim3(1), dim3(1024), 0, stream, tab, add, part, whole);
        else
            hipLaunchKernelGGL(k_norm_parts<256>, dim3(unsigned(grid)), dim3(256), 0, stream, tab, add, part, none);
        add = true;
        clear(tab);
    };
    for (int i = 0; i < count; ++i) {
        const int64_t ch = chunks_of(q[i]);
        if (ch == 0) continue;
        if (full(tab, kMaxGrads, ch)) flush();
        add_entry(tab, GradEntry{q[i].grad, uint32_t(q[i].numel), grad_flags(q[i])}, ch);
    }
    if (tab.n || !add) flush();
    if (all > kNormAlone) hipLaunchKernelGGL(k_norm_end, dim3(1), dim3(256), 0, stream, part, grid, whole);
    return hipGetLastError();
}

hipError_t launch_adamw(const ParamView* q, int count, const AdamwArgs& a, const float* factor, void* state,
                        hipStream_t stream) {
    State* st = static_cast<State*>(state);
    const Hyper hp{a.beta1, a.beta2, float(1.0 - double(a.beta1)), float(1.0 - double(a.beta2)), a.eps, a.lr,
                   float(std::log(double(a.beta1))), float(std::log(double(a.beta2))), a.d_lr, factor};
    int64_t left[2] = {0, 0};       // tensors that are not in a table yet: 32 bits, 8 bits
    for (int i = 0; i < count; ++i)
        if (q[i].numel) ++left[q[i].state_bits == 8];
    Table tab;
    clear(tab);
    const auto flush = [&](int bits) {
        const dim3 grid(unsigned(tab.chunks));
        const bool last = left[0] + left[1] == 0;
        if (bits == 32) hipLaunchKernelGGL(k_adamw32, grid, dim3(256), 0, stream, tab, hp, st, last);
        else hipLaunchKernelGGL(k_adamw8, grid, dim3(256), 0, stream, tab, hp, st, last);
        clear(tab);
    };
    if (left[0] + left[1] == 0) hipLaunchKernelGGL(k_adamw_none, dim3(1), dim3(1), 0, stream, hp, st);
    for (int bits : {32, 8}) {
        for (int i = 0; i < count; ++i) {
            if (q[i].state_bits != bits || q[i].numel == 0) continue;
            const int64_t ch = chunks_of(q[i]);
            if (tab.n && full(tab, kMaxEntries, ch)) flush(bits);
            uint32_t flags = grad_flags(q[i]);
            const size_t am = bits == 32 ? 16 : 4;
            if (!aligned(q[i].param, 16) || !aligned(q[i].m, am) || !aligned(q[i].v, am) || !aligned(q[i].copy, 8))
                flags &= ~uint32_t(kWide);
            const void* at[kAddresses] = {q[i].param, q[i].grad, q[i].copy, q[i].m, q[i].v, bits == 8 ? q[i].scale : nullptr};
            Entry e{};
            for (int k = 0; k < kAddresses; ++k) {
                const uint64_t a = reinterpret_cast<uintptr_t>(at[k]);
                e.lo[k] = uint32_t(a);
                e.hi[k / 2] |= uint32_t(a >> 32) << (16 * (k & 1));
            }
            if (flags & kGradF16) e.lo[kGrad] |= 1u;
            e.size = uint32_t(q[i].numel) | (flags & kWide ? 1u << 31 : 0u);
            e.wd = q[i].weight_decay;
            add_entry(tab, e, ch);
            --left[bits == 8];
        }
        if (tab.n) flush(bits);
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
