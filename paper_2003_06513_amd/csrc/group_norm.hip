// Group normalisation: how a call runs, and the sums between the passes over
// pieces.
#include <cstdlib>
#include "group_norm.h"

namespace psc {
namespace gn {
namespace {

// The statistics of a group from its pieces: the means weighted by their
// counts, the squares about the common mean.
__global__ __launch_bounds__(256) void k_gn_combine_fwd(const float4* __restrict__ parts, int per, float eps,
                                                        float* __restrict__ mean, float* __restrict__ rstd) {
    __shared__ float part[32];
    const float4* p = parts + int64_t(blockIdx.x) * per;
    float sum = 0.f, num = 0.f;
    for (int i = threadIdx.x; i < per; i += 256) {
        sum = fmaf(p[i].z, p[i].x, sum);
        num += p[i].z;
    }
    const float2 both = block_sum2(num, sum, part);
    num = both.x;
    const float mu = both.y / num;
    float sq = 0.f;
    for (int i = threadIdx.x; i < per; i += 256) {
        const float d = p[i].x - mu;
        sq += fmaf(p[i].z * d, d, p[i].y);
    }
    __syncthreads();
    sq = block_sum(sq, part);
    if (threadIdx.x == 0) {
        mean[blockIdx.x] = mu;
        rstd[blockIdx.x] = 1.f / sqrtf(sq / num + eps);
    }
}

__global__ __launch_bounds__(256) void k_gn_combine_bwd(const float2* __restrict__ parts, int per, int pieces,
                                                        int groups, int cg, float m, const float* __restrict__ gamma,
                                                        float2* __restrict__ s12) {
    __shared__ float part[32];
    const float2* p = parts + int64_t(blockIdx.x) * per;
    const int c0 = int(blockIdx.x % unsigned(groups)) * cg;
    float s1 = 0.f, s2 = 0.f;
    for (int i = threadIdx.x; i < per; i += 256) {
        const float ga = or_one(gamma, c0 + i / pieces);
        s1 = fmaf(ga, p[i].x, s1);
        s2 = fmaf(ga, p[i].y, s2);
    }
    const float2 sum = block_sum2(s1, s2, part);
    if (threadIdx.x == 0) s12[blockIdx.x] = make_float2(sum.x / m, sum.y / m);
}

// dbeta and dgamma: a block adds 32 channels, each over the images' and
// pieces' sums, 32 of them at a time, in a fixed order.
__global__ __launch_bounds__(1024) void k_gn_param(const float2* __restrict__ sums, int n, int c, int pieces,
                                                   float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ float2 part[32][33];
    const int k = int(blockIdx.x) * 32 + int(threadIdx.x & 31), row = int(threadIdx.x >> 5);
    float a = 0.f, b = 0.f;
    if (k < c) {
        const int64_t count = int64_t(n) * pieces;
        for (int64_t i = row; i < count; i += 32) {
            const int64_t img = i / pieces, piece = i - img * pieces;
            const float2 ab = sums[(img * c + k) * pieces + piece];
            a += ab.x;
            b += ab.y;
        }
    }
    part[row][threadIdx.x & 31] = make_float2(a, b);
    __syncthreads();
    if (row == 0 && k < c) {
        a = 0.f, b = 0.f;
        for (int i = 0; i < 32; ++i) a += part[i][threadIdx.x].x, b += part[i][threadIdx.x].y;
        if (dgamma) dgamma[k] = b;
        if (dbeta) dbeta[k] = a;
    }
}

int log2_ceil(int64_t x) {
    int l = 0;
    while ((int64_t(1) << l) < x) ++l;
    return l;
}
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int vector_of(int dtype) { return dtype == DT_F16 ? 8 : 4; }

struct Try {
    int threads, k;
};
// Blocks by size, for units of work that there are many of (a few vectors a
// thread, small blocks) or few of (every thread one or two).
constexpr Try kMany[] = {{64, 4}, {128, 4}, {256, 4}, {256, 8}, {512, 8}, {1024, 4}, {512, 32}};
constexpr Try kFew[] = {{64, 2}, {128, 2}, {256, 2}, {512, 2}, {1024, 2}, {1024, 4}, {512, 8}, {512, 32}};
int most_of(bool backward, int vec) { return vec == 0 ? kMostSingle : backward ? kMostBwd : kMostFwd; }

// The lanes that share a row so that a thread has the fewest vectors.
int64_t rows_slots(int cg, int vpr, int threads, int* lanes_log2, int* vi) {
    int64_t best = -1;
    for (int l = 0; (1 << l) <= threads; ++l) {
        const int64_t v = ceil_div(vpr, 1 << l), n = v * ceil_div(cg, threads >> l);
        if (best < 0 || n <= best) best = n, *lanes_log2 = l, *vi = int(v);
    }
    return best;
}

// The plan of a call whose tensors allow 16-byte accesses (vec 1: at the
// beginning of each row, 2: within rows) or not (0).
Plan plan_rows(const GroupNormArgs& a, bool backward, int vec) {
    Plan p{};
    const int v = vec ? vector_of(a.dtype) : 1;
    Rows& s = p.rows;
    s.cg = a.c / a.groups, s.groups = a.groups, s.hw = a.h * a.w;
    s.total = int64_t(a.n) * a.c * s.hw;
    s.vpr = vec == 2 ? int(ceil_div(s.hw + v - 1, v)) : int(ceil_div(s.hw, v));
    p.vec = vec;
    const int64_t units = int64_t(a.n) * a.groups;
    const auto fits = [&](const Try& t) {
        const int64_t n = rows_slots(s.cg, s.vpr, t.threads, &s.lanes_log2, &s.vi);
        if (n > t.k || n > most_of(backward, vec)) return false;
        p.held = true, p.threads = t.threads, p.k = s.slots = int(n), p.grid = units, p.pieces = 1;
        return true;
    };
    if (vec && s.cg <= 2048) {      // the rows' parameters and sums fit the LDS
        if (units >= 512) {
            for (const Try& t : kMany)
                if (fits(t)) return p;
        } else {
            for (const Try& t : kFew)
                if (fits(t)) return p;
        }
    }
    p.pieces = int(ceil_div(s.vpr, 64 * (vec ? kPiece : kPieceSingle)));
    return p;
}

Plan plan_cols(const GroupNormArgs& a, bool backward, int vec) {
    Plan p{};
    const int v = vec ? vector_of(a.dtype) : 1, elt = a.dtype == DT_F16 ? 2 : 4;
    Cols& s = p.cols;
    s.c = a.c, s.groups = a.groups, s.cg = a.c / a.groups, s.hw = a.h * a.w;
    p.vec = vec;
    s.cg_m = s.cg == 1 ? 0 : uint32_t(((uint64_t(1) << 32) + s.cg - 1) / s.cg);
    int unit = s.cg;        // the fewest channels that are whole groups and whole vectors
    while (unit % v) unit += s.cg;
    // Tiles as wide as a cache line, or half or a quarter of one, of whole groups.
    const int want = getenv("GN_UNITS") ? atoi(getenv("GN_UNITS")) : 512;
    const int least = getenv("GN_LEAST") ? atoi(getenv("GN_LEAST")) : 16;
    Plan best{};
    for (int bytes = 128; bytes >= least; bytes /= 2) {
        const int tile = int(ceil_div(bytes, int64_t(unit) * elt)) * unit;
        s.tile = tile < a.c ? tile : a.c;
        s.tiles = int(ceil_div(a.c, s.tile));
        s.cols_log2 = log2_ceil(ceil_div(s.tile, v));
        const int64_t units = int64_t(a.n) * s.tiles;
        const auto fits = [&](const Try& t) {
            if (t.threads < (1 << s.cols_log2) || int64_t(s.hw) * a.c * elt >> 32) return false;
            const int64_t n = ceil_div(s.hw, t.threads >> s.cols_log2);
            if (n > t.k || n > most_of(backward, vec)) return false;
            if (cols_lds(s, t.threads, backward ? 2 : 1, backward ? 4 : 2) > 60 * 1024) return false;
            p.held = true, p.threads = t.threads, p.k = int(n), p.pieces = 1;
            s.pixels = s.hw, s.chunks = 1;
            p.grid = ceil_div(a.n, 8) * 8 * s.tiles;
            return true;
        };
        bool found = false;
        if (units >= 512) {
            for (const Try& t : kMany)
                if (!found) found = fits(t);
        } else {
            for (const Try& t : kFew)
                if (!found) found = fits(t);
        }
        if (found) best = p;
        if (found && units >= want) break;
    }
    if (best.held && !getenv("GN_PIECES")) return best;
    p = best = Plan{};
    p.vec = vec;
    s.c = a.c, s.groups = a.groups, s.cg = a.c / a.groups, s.hw = a.h * a.w;
    s.cg_m = s.cg == 1 ? 0 : uint32_t(((uint64_t(1) << 32) + s.cg - 1) / s.cg);
    // pieces: 256 threads, up to 16 vectors (64 single channels) side by side
    s.cols_log2 = log2_ceil(ceil_div(a.c, v));
    const int most = vec ? 4 : 6;
    if (s.cols_log2 > most) s.cols_log2 = most;
    s.tile = v << s.cols_log2;
    s.tiles = int(ceil_div(a.c, s.tile));
    s.pixels = (256 >> s.cols_log2) * (vec ? kPiece : kPieceSingle);
    s.chunks = p.pieces = int(ceil_div(s.hw, s.pixels));
    p.threads = 256;
    p.grid = ceil_div(a.n, 8) * 8 * s.tiles * s.chunks;
    return p;
}

Plan plan_of(const GroupNormArgs& a, bool backward, int vec) {
    return a.channels_last ? plan_cols(a, backward, vec) : plan_rows(a, backward, vec);
}

// How the tensors lie: all alike to 16 bytes, and rows (pixels) of whole vectors.
int vec_of(const GroupNormArgs& a, const void* x, const void* y, const void* z) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(x) & 15u;
    for (const void* p : {y, z})
        if (p && (reinterpret_cast<uintptr_t>(p) & 15u) != at) return 0;
    const int64_t row = a.channels_last ? a.c : int64_t(a.h) * a.w;
    if (at == 0 && row % vector_of(a.dtype) == 0) return 1;
    return a.channels_last ? 0 : 2;
}

size_t bytes_of(const GroupNormArgs& a, bool backward, int vec) {
    const Plan p = plan_of(a, backward, vec);
    const size_t sums = size_t(a.n) * size_t(a.c) * size_t(p.pieces), groups = size_t(a.n) * size_t(a.groups);
    if (backward) return sums * sizeof(float2) + (p.held ? 0 : groups * sizeof(float2));
    return p.held ? 0 : sums * sizeof(float4) + groups * 2 * sizeof(float);
}

}  // namespace

void combine_fwd(const float4* parts, int64_t groups, int per_group, float eps, float* mean, float* rstd, hipStream_t st) {
    hipLaunchKernelGGL(k_gn_combine_fwd, dim3(unsigned(groups)), dim3(256), 0, st, parts, per_group, eps, mean, rstd);
}
void combine_bwd(const float2* parts, int64_t groups, int per_group, int pieces, int groups_per_image, int cg, float m,
                 const float* gamma, float2* s12, hipStream_t st) {
    hipLaunchKernelGGL(k_gn_combine_bwd, dim3(unsigned(groups)), dim3(256), 0, st, parts, per_group, pieces,
                       groups_per_image, cg, m, gamma, s12);
}

}  // namespace gn

// What the call may need however its tensors lie.
size_t group_norm_workspace_bytes(const GroupNormArgs& a, bool backward) {
    size_t most = 0;
    for (int vec : {0, 1, 2}) {
        const size_t b = gn::bytes_of(a, backward, vec);
        if (b > most) most = b;
    }
    return most;
}

hipError_t launch_group_norm_fwd(const GroupNormArgs& a, const void* x, const float* gamma, const float* beta, float eps,
                                 void* y, float* mean, float* rstd, void* ws, hipStream_t stream) {
    using namespace gn;
    Plan p = plan_of(a, false, vec_of(a, x, y, nullptr));
    const Params q{gamma, beta, a.act};
    float4* parts = static_cast<float4*>(ws);
    const int64_t rows = int64_t(a.n) * a.c * p.pieces, groups = int64_t(a.n) * a.groups;
    if (!p.held && !mean) {
        mean = static_cast<float*>(static_cast<void*>(parts + rows));
        rstd = mean + groups;
    }
    if (a.channels_last) {
        if (a.dtype == DT_F16) cols_fwd<DT_F16>(p, a.n, x, q, eps, y, mean, rstd, parts, stream);
        else cols_fwd<DT_F32>(p, a.n, x, q, eps, y, mean, rstd, parts, stream);
    } else {
        p.rows.lead = int((reinterpret_cast<uintptr_t>(x) & 15u) / (a.dtype == DT_F16 ? 2 : 4));
        if (a.dtype == DT_F16) rows_fwd<DT_F16>(p, rows, x, q, eps, y, mean, rstd, parts, stream);
        else rows_fwd<DT_F32>(p, rows, x, q, eps, y, mean, rstd, parts, stream);
    }
    return hipGetLastError();
}

hipError_t launch_group_norm_bwd(const GroupNormArgs& a, const void* x, const void* dy, const float* gamma,
                                 const float* beta, const float* mean, const float* rstd, void* dx, float* dgamma,
                                 float* dbeta, void* ws, hipStream_t stream) {
    using namespace gn;
    Plan p = plan_of(a, true, vec_of(a, x, dy, dx));
    const Params q{gamma, beta, a.act};
    float2* parts = static_cast<float2*>(ws);
    const int64_t rows = int64_t(a.n) * a.c * p.pieces;
    float2* s12 = parts + rows;
    const bool params = dgamma || dbeta;
    if (p.held && !params) parts = nullptr;
    if (a.n > 0) {
        if (a.channels_last) {
            if (a.dtype == DT_F16) cols_bwd<DT_F16>(p, a.n, x, dy, q, mean, rstd, dx, parts, s12, stream);
            else cols_bwd<DT_F32>(p, a.n, x, dy, q, mean, rstd, dx, parts, s12, stream);
        } else {
            p.rows.lead = int((reinterpret_cast<uintptr_t>(x) & 15u) / (a.dtype == DT_F16 ? 2 : 4));
            if (a.dtype == DT_F16) rows_bwd<DT_F16>(p, rows, x, dy, q, mean, rstd, dx, parts, s12, stream);
            else rows_bwd<DT_F32>(p, rows, x, dy, q, mean, rstd, dx, parts, s12, stream);
        }
    }
    if (params)
        hipLaunchKernelGGL(k_gn_param, dim3(unsigned((a.c + 31) / 32)), dim3(1024), 0, stream, parts, a.n, a.c, p.pieces,
                           dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace psc
