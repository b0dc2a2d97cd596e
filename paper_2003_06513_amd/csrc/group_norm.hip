// Group normalisation: how a call runs, and the sums between the passes over
// pieces.
#include "group_norm.h"

namespace psc {
namespace gn {
namespace {

// A block per group of many pieces, of 1024 threads where they are more than
// so many: 4 x 771 x 33 x 33 fp16, one group, channels last 40 -> 27 us.
int combine_threads(int per) { return per > 1024 ? 1024 : 256; }

__global__ __launch_bounds__(1024) void k_gn_combine_fwd(const float4* __restrict__ parts, int per, float eps,
                                                        float* __restrict__ mean, float* __restrict__ rstd) {
    __shared__ float part[32], again[16];
    const float4* p = parts + int64_t(blockIdx.x) * per;
    float sum = 0.f, num = 0.f;
#pragma unroll 4
    for (int i = threadIdx.x; i < per; i += blockDim.x) {
        const float4 t = p[i];
        sum = sum_with(t, sum);
        num += t.z;
    }
    const float2 both = block_sum2(num, sum, part);
    const float mu = both.y / both.x;
    float sq = 0.f;
#pragma unroll 4
    for (int i = threadIdx.x; i < per; i += blockDim.x) sq += squares_about(p[i], mu);
    sq = block_sum(sq, again);
    if (threadIdx.x == 0) {
        const float2 ms = stats_of(mu, sq / both.x, eps);
        mean[blockIdx.x] = ms.x, rstd[blockIdx.x] = ms.y;
    }
}

__global__ __launch_bounds__(1024) void k_gn_combine_bwd(const float2* __restrict__ parts, int per, int pieces,
                                                        int groups, int cg, float m, const float* __restrict__ gamma,
                                                        float2* __restrict__ s12) {
    __shared__ float part[32];
    const float2* p = parts + int64_t(blockIdx.x) * per;
    const int c0 = int(blockIdx.x % unsigned(groups)) * cg;
    float s1 = 0.f, s2 = 0.f;
#pragma unroll 4
    for (int i = threadIdx.x; i < per; i += blockDim.x) {
        const float ga = or_one(gamma, c0 + i / pieces);
        s1 = fmaf(ga, p[i].x, s1);
        s2 = fmaf(ga, p[i].y, s2);
    }
    const float2 sum = block_sum2(s1, s2, part);
    if (threadIdx.x == 0) s12[blockIdx.x] = make_float2(sum.x / m, sum.y / m);
}

__global__ __launch_bounds__(1024) void k_gn_param(Tail t) { param_block(t); }

int log2_ceil(int64_t x) {
    int l = 0;
    while ((int64_t(1) << l) < x) ++l;
    return l;
}
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Blocks by size, for units of work that there are many of (small blocks,
// a few vectors a thread) or few of (every thread one or two): threads, and
// the most sixteenths of the bytes that a thread can hold of one tensor.
struct Try {
    int threads, part;
};
constexpr Try kMany[] = {{64, 8}, {128, 8}, {256, 8}, {256, 16}, {512, 16}, {1024, 8}, {512, 32}};
constexpr Try kFew[] = {{64, 4}, {128, 4}, {256, 4}, {512, 4}, {1024, 4}, {1024, 8}, {512, 16}, {512, 32}};
// Columns that are more than the CUs but less than twice as many: of blocks of
// 512 threads a CU runs two, of 1024 one, and then those that are left (9 x 512
// x 28 x 28 fp32 backward, 288 blocks: 22.3 us, not 26.6; rows gain nothing).
constexpr Try kSome[] = {{64, 4}, {128, 4}, {256, 4}, {512, 4}, {512, 8}, {512, 16}, {1024, 8}, {512, 32}};
// The first of them that `count(threads)` vectors a thread fit, or none.
template <class F> bool choose(int64_t units, bool cols, int dtype, int v, bool backward, Plan& p, F count) {
    const Try* list = units >= 512 ? kMany : cols && units > 256 ? kSome : kFew;
    const int n = units >= 512 ? int(sizeof(kMany) / sizeof(Try)) : int(sizeof(kFew) / sizeof(Try));
    static_assert(sizeof(kSome) == sizeof(kFew), "one count");
    for (int i = 0; i < n; ++i) {
        const int64_t k = count(list[i].threads);
        if (k < 1 || k > most_of(dtype, v, backward) || 16 * k > int64_t(list[i].part) * piece_of(dtype, v)) continue;
        p.held = true, p.threads = list[i].threads, p.k = int(k), p.pieces = 1;
        return true;
    }
    return false;
}

// The lanes that share a row so that a thread has the fewest vectors.
int64_t rows_slots(int cg, int vpr, int threads, int* lanes_log2, int* vi) {
    int64_t best = -1;
    for (int l = 0; (1 << l) <= threads; ++l) {
        const int64_t v = ceil_div(vpr, 1 << l), n = v * ceil_div(cg, threads >> l);
        if (best < 0 || n <= best) best = n, *lanes_log2 = l, *vi = int(v);
    }
    return best;
}

// The most sums of pieces that every wave that writes one reads itself, and
// every block of columns.  More of them are joined by a launch of its own
// (about 2.5 us).
constexpr int kJoined = 256, kJoinedCols = 2048;

// The plan of a call whose tensors allow 16-byte accesses (vec 1: at the
// beginning of each row, 2: within rows) or not (0).
Plan plan_rows(const GroupNormArgs& a, bool backward, int vec) {
    Plan p{};
    const int v = vec ? vector_of(a.dtype, false) : 1;
    Rows& s = p.rows;
    s.cg = a.c / a.groups, s.groups = a.groups, s.hw = a.h * a.w;
    s.total = int64_t(a.n) * a.c * s.hw;
    s.vpr = vec == 2 ? int(ceil_div(s.hw + v - 1, v)) : int(ceil_div(s.hw, v));
    p.vec = vec;
    p.grid = int64_t(a.n) * a.groups;
    if (vec && s.cg <= 2048 &&      // the rows' parameters and sums fit the LDS
        choose(p.grid, false, a.dtype, v, backward, p, [&](int threads) {
            return rows_slots(s.cg, s.vpr, threads, &s.lanes_log2, &s.vi);
        })) {
        s.slots = p.k;
        return p;
    }
    p.pieces = int(ceil_div(s.vpr, 64 * piece_of(a.dtype, v)));
    p.joined = int64_t(s.cg) * p.pieces <= kJoined;
    return p;
}

// Blocks of the columns, in slabs of tiles that share lines of memory.
int64_t cols_grid(Cols& s, int n, int elt) {
    s.near = 128 / (s.tile * elt);
    if (s.near < 1) s.near = 1;
    // whole images, where every die gets as many of them, or many (48 x 512 x 28 x 28 fp32 backward 67 -> 56 us)
    const int64_t images = int64_t(n) * s.chunks;
    if (s.near > s.tiles || images >= 64 || (images >= 16 && images % 8 == 0)) s.near = s.tiles;
    // slabs alike: of 12 tiles 6 and 6, not 8 and 4 (20 x 96 x 40 x 40 fp16 14.5 -> 12 us)
    s.near = int(ceil_div(s.tiles, ceil_div(s.tiles, s.near)));
    return ceil_div(int64_t(n) * s.chunks * ceil_div(s.tiles, s.near), 8) * 8 * s.near;
}

// Whether tiles of less than half a line of memory lose.  Each of their lines
// goes from the die's cache to several CUs, which long columns (k of `piece`
// vectors a thread) pay for most: then wider tiles of fewer blocks, or pieces,
// are faster once there are more blocks than CUs (forward, 20 x 256 x 56 x 56
// fp32: 42 us in pieces, 57 held; 40 x 128 x 40 x 40 fp16: 14 in 160 blocks, 23
// in 640), in the backward in tiles of 16 bytes also before (64 x 64 x 56 x
// 56 fp16: 33 us in pieces, 41 held).  The limits lie between measured sides
// such as these; no model of the caches stands behind them.
bool narrow_loses(int64_t units, int threads, int64_t k, int bytes, bool wider, bool backward, int piece) {
    const bool many = units > 256;
    if (!backward) return many && (wider || 2 * k >= piece);
    return (many && threads == 1024) || (bytes <= 16 && 4 * k > piece - (many ? 4 : 0));
}

Plan plan_cols(const GroupNormArgs& a, bool backward, int vec) {
    const int v = vec ? vector_of(a.dtype, backward) : 1, elt = a.dtype == DT_F16 ? 2 : 4;
    Plan p{}, best{};
    Cols& s = p.cols;
    p.vec = vec;
    s.c = a.c, s.groups = a.groups, s.cg = a.c / a.groups, s.hw = a.h * a.w;
    s.cg_m = s.cg == 1 ? 0 : uint32_t(((uint64_t(1) << 32) + s.cg - 1) / s.cg);
    int unit = s.cg;        // the fewest channels that are whole groups and whole vectors
    while (unit % v) unit += s.cg;
    // Tiles of whole groups, a line of memory wide or a part of one: as wide as gives every CU a block.
    for (int bytes = 128; bytes >= 16; bytes /= 2) {
        const int tile = int(ceil_div(bytes, int64_t(unit) * elt)) * unit;
        s.tile = tile < a.c ? tile : a.c;
        s.tiles = int(ceil_div(a.c, s.tile));
        s.cols_log2 = log2_ceil(ceil_div(s.tile, v));
        if (int64_t(s.hw) * a.c * elt >> 32) break;     // offsets of 32 bits
        const int64_t units = int64_t(a.n) * s.tiles;
        p.held = false;
        if (choose(units, true, a.dtype, v, backward, p, [&](int threads) {
                if (threads < (1 << s.cols_log2) ||
                    cols_lds(s, threads, backward ? 2 : 1, backward ? 4 : 2) > 60 * 1024)
                    return int64_t(0);
                const int64_t k = ceil_div(s.hw, threads >> s.cols_log2);
                if (vec && s.tile * elt < 64 && narrow_loses(units, threads, k, s.tile * elt, best.held, backward,
                                                             piece_of(a.dtype, v)))
                    return int64_t(0);
                return k;
            })) {
            s.pixels = s.hw, s.chunks = 1;
            p.grid = cols_grid(s, a.n, elt);
            best = p;
            if (units >= 256) break;
        }
    }
    if (best.held) return best;
    // Pieces: 256 threads, whole groups if 16 vectors (64 single channels) side by side have room for one.
    p.held = false;
    const int room = vec ? 16 * v : 64;
    s.tile = unit <= room ? room / unit * unit : room;
    if (s.tile > a.c) s.tile = int(ceil_div(a.c, v)) * v;
    s.cols_log2 = log2_ceil(ceil_div(s.tile, v));
    s.tiles = int(ceil_div(a.c, s.tile));
    s.pixels = (256 >> s.cols_log2) * piece_of(a.dtype, v);
    s.chunks = p.pieces = int(ceil_div(s.hw, s.pixels));
    p.threads = 256;
    p.grid = cols_grid(s, a.n, elt);
    p.joined = unit <= room && int64_t(s.tile) * s.chunks <= kJoinedCols;
    s.join_lanes = 64;
    while (s.join_lanes > 4 && s.join_lanes * (s.tile / s.cg) > 256) s.join_lanes /= 2;
    return p;
}

Plan plan_of(const GroupNormArgs& a, bool backward, int vec) {
    return a.channels_last ? plan_cols(a, backward, vec) : plan_rows(a, backward, vec);
}

// How the tensors lie, by their offset from a multiple of 16 bytes (-1: not
// all alike): rows (pixels) of whole vectors, rows that begin anywhere, or
// single elements.
int vec_of(const GroupNormArgs& a, bool backward, int offset) {
    const int v = vector_of(a.dtype, a.channels_last && backward);
    if (offset < 0) return 0;
    if (offset % (v * (a.dtype == DT_F16 ? 2 : 4)) == 0 && (a.channels_last ? a.c : int64_t(a.h) * a.w) % v == 0) return 1;
    return a.channels_last ? 0 : 2;
}
int offset_of(const void* x, const void* y, const void* z) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(x) & 15u;
    for (const void* p : {y, z})
        if (p && (reinterpret_cast<uintptr_t>(p) & 15u) != at) return -1;
    return int(at);
}

size_t bytes_of(const GroupNormArgs& a, bool backward, int vec) {
    const Plan p = plan_of(a, backward, vec);
    const size_t sums = size_t(a.n) * size_t(a.c) * size_t(p.pieces), groups = size_t(a.n) * size_t(a.groups);
    if (backward) return sums * sizeof(float2) + (p.held ? 0 : groups * sizeof(float2));
    return p.held ? 0 : sums * sizeof(float4) + groups * 2 * sizeof(float);
}

}  // namespace

void combine_fwd(const float4* parts, int64_t groups, int per_group, float eps, float* mean, float* rstd, hipStream_t st) {
    hipLaunchKernelGGL(k_gn_combine_fwd, dim3(unsigned(groups)), dim3(unsigned(combine_threads(per_group))), 0, st, parts,
                       per_group, eps, mean, rstd);
}
void combine_bwd(const float2* parts, int64_t groups, int per_group, int pieces, int groups_per_image, int cg, float m,
                 const float* gamma, float2* s12, hipStream_t st) {
    hipLaunchKernelGGL(k_gn_combine_bwd, dim3(unsigned(groups)), dim3(unsigned(combine_threads(per_group))), 0, st, parts,
                       per_group, pieces, groups_per_image, cg, m, gamma, s12);
}

}  // namespace gn

// What the call may need however its tensors lie, or if they are aligned.
size_t group_norm_workspace_bytes(const GroupNormArgs& a, bool backward, bool aligned) {
    if (aligned) return gn::bytes_of(a, backward, gn::vec_of(a, backward, 0));
    size_t most = 0;
    for (int vec : {0, 1, 2}) {
        const size_t b = gn::bytes_of(a, backward, vec);
        if (b > most) most = b;
    }
    return most;
}

namespace {
using namespace gn;

// The images of a launch: a launch has fewer than 2^32 threads, which groups of
// one value pass before their tensor does its limit.  A multiple of 16, so
// that every launch's tensors lie as the first's.
int images_of(const GroupNormArgs& a, const Plan& p) {
    const int64_t blocks = !a.channels_last ? (p.held ? a.groups : ceil_div(int64_t(a.c) * p.pieces, 4) + 1)
                                            : int64_t(p.cols.tiles + p.cols.near) * p.cols.chunks;
    const int64_t threads = (blocks > a.groups ? blocks : a.groups) * (p.threads > 256 ? p.threads : 256);
    const int64_t most = (int64_t(1) << 31) / threads / 16 * 16;
    return a.n <= most ? a.n : int(most < 16 ? 16 : most);
}
// The plan of some of the images.
Plan part_of(const GroupNormArgs& a, Plan p, int n) {
    p.grid = a.channels_last ? cols_grid(p.cols, n, a.dtype == DT_F16 ? 2 : 4) : int64_t(n) * a.groups;
    p.rows.total = int64_t(n) * a.c * a.h * a.w;
    return p;
}
const void* at(const void* p, int64_t elements, int dtype) {
    return static_cast<const char*>(p) + elements * (dtype == DT_F16 ? 2 : 4);
}
void* at(void* p, int64_t elements, int dtype) { return static_cast<char*>(p) + elements * (dtype == DT_F16 ? 2 : 4); }

}  // namespace

hipError_t launch_group_norm_fwd(const GroupNormArgs& a, const void* x, const float* gamma, const float* beta, float eps,
                                 void* y, float* mean, float* rstd, void* ws, hipStream_t stream) {
    const int offset = offset_of(x, y, nullptr);
    Plan whole = plan_of(a, false, vec_of(a, false, offset));
    whole.rows.lead = offset < 0 ? 0 : offset / (a.dtype == DT_F16 ? 2 : 4);
    const Params q{gamma, beta, a.act};
    float4* all = static_cast<float4*>(ws);
    const int64_t image = int64_t(a.c) * a.h * a.w, rows = int64_t(a.c) * whole.pieces;
    if (!whole.held && !whole.joined && !mean) {
        mean = static_cast<float*>(static_cast<void*>(all + a.n * rows));
        rstd = mean + int64_t(a.n) * a.groups;
    }
    const int most = images_of(a, whole);
    for (int first = 0; first < a.n; first += most) {
        const int n = a.n - first < most ? a.n - first : most;
        const Plan p = part_of(a, whole, n);
        const void* xn = at(x, first * image, a.dtype);
        void* yn = at(y, first * image, a.dtype);
        float* mn = mean ? mean + int64_t(first) * a.groups : nullptr;
        float* rn = mean ? rstd + int64_t(first) * a.groups : nullptr;
        float4* parts = all + first * rows;
        if (a.channels_last) {
            if (a.dtype == DT_F16) cols_fwd<DT_F16>(p, n, xn, q, eps, yn, mn, rn, parts, stream);
            else cols_fwd<DT_F32>(p, n, xn, q, eps, yn, mn, rn, parts, stream);
        } else {
            if (a.dtype == DT_F16) rows_fwd<DT_F16>(p, n * rows, xn, q, eps, yn, mn, rn, parts, stream);
            else rows_fwd<DT_F32>(p, n * rows, xn, q, eps, yn, mn, rn, parts, stream);
        }
    }
    return hipGetLastError();
}

hipError_t launch_group_norm_bwd(const GroupNormArgs& a, const void* x, const void* dy, const float* gamma,
                                 const float* beta, const float* mean, const float* rstd, void* dx, float* dgamma,
                                 float* dbeta, void* ws, hipStream_t stream) {
    const int offset = offset_of(x, dy, dx);
    Plan whole = plan_of(a, true, vec_of(a, true, offset));
    whole.rows.lead = offset < 0 ? 0 : offset / (a.dtype == DT_F16 ? 2 : 4);
    const Params q{gamma, beta, a.act};
    const int64_t image = int64_t(a.c) * a.h * a.w, rows = int64_t(a.c) * whole.pieces;
    float2* all = static_cast<float2*>(ws);
    float2* s12 = all + a.n * rows;
    const Tail wanted{all, a.n, a.c, whole.pieces, dgamma, dbeta, 0};
    const unsigned last = tail_blocks(wanted);
    // a held batch of one image: the sums of its channels are the gradients
    const bool once = whole.held && a.n == 1;
    const int most = images_of(a, whole);
    for (int first = 0; first < a.n; first += most) {
        const int n = a.n - first < most ? a.n - first : most;
        const Plan p = part_of(a, whole, n);
        const void *xn = at(x, first * image, a.dtype), *gn = at(dy, first * image, a.dtype);
        void* dn = at(dx, first * image, a.dtype);
        const float *mn = mean + int64_t(first) * a.groups, *rn = rstd + int64_t(first) * a.groups;
        Sums sums{whole.held && (once || !last) ? nullptr : all + first * rows, once ? dgamma : nullptr,
                  once ? dbeta : nullptr};
        float2* sn = s12 + int64_t(first) * a.groups;
        Tail tail = wanted;         // behind the last images' pieces
        if (first + n < a.n) tail.dgamma = tail.dbeta = nullptr;
        if (a.channels_last) {
            if (a.dtype == DT_F16) cols_bwd<DT_F16>(p, n, xn, gn, q, mn, rn, dn, sums, sn, tail, stream);
            else cols_bwd<DT_F32>(p, n, xn, gn, q, mn, rn, dn, sums, sn, tail, stream);
        } else {
            if (a.dtype == DT_F16) rows_bwd<DT_F16>(p, n * rows, xn, gn, q, mn, rn, dn, sums, sn, tail, stream);
            else rows_bwd<DT_F32>(p, n * rows, xn, gn, q, mn, rn, dn, sums, sn, tail, stream);
        }
    }
    if (last && !once && (whole.held || a.n == 0))
        hipLaunchKernelGGL(k_gn_param, dim3(last), dim3(1024), 0, stream, wanted);
    return hipGetLastError();
}

}  // namespace psc
