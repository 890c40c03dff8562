// Gated feed-forward unit on gfx950, and its gradients.
//
//   G = X Wg', U = X Wu', H = act(G) U, Y = H Wd'
//   dH = dY Wd, dU = dH act(G), dG = dH U act'(G)
//   dX = dG Wg + dU Wu, dWg = dG' X, dWu = dU' X, dWd = dY' H
//
// Every product is a launch of one kernel, k_product, over tiles of its result:
//   G and U together: a tile's columns are halves of Wg and of Wu, so a lane has g
//     and u of the same places in its registers and stores h
//   dH: the epilogue reads g and u and stores dG and dU
//   dX: the contracted axis runs over Wg's rows, then Wu's
//   dWg, dWu, dWd: up to three products of one launch
// Operands whose contracted axis is in rows are read transposed from LDS, so no
// tensor is laid out anew.  bf16 rounds what is stored: H, dG and dU; sums are
// float32.
#include <algorithm>

#include <hip/hip_runtime.h>

#include "compute_units.hpp"
#include "products.hpp"
#include "token_ops.hpp"

namespace rtcc {
namespace kern {

namespace {

// ------------------------------------------------------------------ activation

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// activation(z) = z * gate; *slope = its derivative
__device__ inline float silu(float z, float *slope) {
    const float s = __builtin_amdgcn_rcpf(1.f + exp2_fast(-1.4426950408889634f * z));
    if (slope) *slope = s * fmaf(z, 1.f - s, 1.f);
    return z * s;
}
// Phi(-x) = erfc(x / sqrt 2) / 2 = t P(t) exp(-x^2 / 2) / 2 for x >= 0 with t = 1 /
// (1 + 0.4 x / sqrt 2): P is the least maximum relative error fit of degree 8 to
// exp(y^2) erfc(y) / t over y in [0, 122] (1.3e-7; 4.1e-7 evaluated in float32), so
// that the far negative side keeps its relative precision, which (1 + erf) / 2 loses.
__device__ inline float gelu(float z, float *slope) {
    const float x = fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(x, 0.28284271247461906f, 1.f));
    const float e = exp2_fast(-0.7213475204444817f * z * z);
    float p = 0.05027266591787338f;
    p = fmaf(p, t, -0.18294385075569153f);
    p = fmaf(p, t, 0.169155091047287f);
    p = fmaf(p, t, -0.0056677525863051414f);
    p = fmaf(p, t, 0.14146076142787933f);
    p = fmaf(p, t, 0.16853399574756622f);
    p = fmaf(p, t, 0.2078438252210617f);
    p = fmaf(p, t, 0.22566953301429749f);
    p = fmaf(p, t, 0.22567586600780487f);
    const float tail = 0.5f * p * t * e;
    const float phi = z < 0.f ? tail : 1.f - tail;
    if (slope) *slope = fmaf(z, 0.3989422804014327f * e, phi);
    return z * phi;
}
__device__ inline float activation(bool is_gelu, float z, float *slope) { return is_gelu ? gelu(z, slope) : silu(z, slope); }

// -------------------------------------------------------------------- products

// C [m][n] = sum over segments and k of A [m][k] B [n][k]; where K is in rows, A
// is [k][m] and B [k][n].
struct Product {
    const char *a[2], *b[2];  // of each segment; of a gated product b are the halves of a tile's columns
    uint32_t a_row, b_row[2];  // bytes between rows
    int32_t m, n, k;           // k: of a segment
    int32_t tiles_n, tiles;
    void *c;
    int64_t c_row;  // elements
    int64_t partial;  // floats before the product's part of a slice
};
constexpr int kMaxProducts = 3;
struct Work {
    Product p[kMaxProducts];
    int32_t products, segments;
    int32_t slices, per_slice;  // of the contracted axis, and steps of each
    float *partial;             // [slices][slice_size]
    int64_t slice_size;
    // gated products: [m][n] of one stride (elements)
    bool gelu;
    void *gate, *up, *act;
    int64_t hidden_s;
};

enum Epilogue { kPlain, kGated, kGatedGrad };

// The product, the slice and the tile of a block.  Blocks of one XCD (every eighth)
// take tiles that follow each other, in bands of kBand tiles of rows, so that their
// operands meet in its L2.
struct Spot {
    int which, slice, tile_m, tile_n;  // which < 0: none, of a folded launch's last blocks
};
constexpr int kBand = 4;
__device__ inline Spot spot(const Work &w) {
    uint32_t id = blockIdx.z * gridDim.x + blockIdx.x;
    int which = 0;
    uint32_t tiles = w.p[0].tiles, across = w.p[0].tiles_n;
#pragma unroll
    for (int i = 1; i < kMaxProducts; ++i)
        if (which == i - 1 && i < w.products && id >= tiles * w.slices) {
            id -= tiles * w.slices;
            which = i, tiles = w.p[i].tiles, across = w.p[i].tiles_n;
        }
    const uint32_t n = tiles * w.slices, x = id % 8;
    if (id >= n) return {-1, 0, 0, 0};
    id = x * (n / 8) + min(x, n % 8) + id / 8;
    const int slice = int(id / tiles);
    id %= tiles;
    const uint32_t down = tiles / across, top = id / (kBand * across) * kBand, rows = min(down - top, uint32_t(kBand));
    id -= top * across;
    // said to be uniform, so that all addresses stay in scalar registers
    return {__builtin_amdgcn_readfirstlane(which), __builtin_amdgcn_readfirstlane(slice),
            __builtin_amdgcn_readfirstlane(top + id % rows), __builtin_amdgcn_readfirstlane(id / rows)};
}
// A copy by constant indexes: an indexed one would go through memory.
__device__ inline Product pick(const Work &w, int which) { return which == 0 ? w.p[0] : which == 1 ? w.p[1] : w.p[2]; }

// Stores four neighbouring results c (a gated product's: of gate, with those of up
// in d) of row m from column n on.
template <typename T, int EPI>
__device__ inline void finish(const Work &w, const Product &p, int slice, int m, int n, f32x4_t c, f32x4_t d) {
    if constexpr (EPI == kGated) {
        const int64_t at = m * w.hidden_s + n;
        f32x4_t h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = activation(w.gelu, c[e], nullptr) * d[e];
        store4(static_cast<T *>(w.act) + at, h);
        if (w.gate) {
            store4(static_cast<T *>(w.gate) + at, c);
            store4(static_cast<T *>(w.up) + at, d);
        }
    } else if constexpr (EPI == kGatedGrad) {
        const int64_t at = m * w.hidden_s + n, to = int64_t(m) * p.n + n;
        const f32x4_t g = load4(static_cast<const T *>(w.gate) + at), u = load4(static_cast<const T *>(w.up) + at);
        f32x4_t dg, du;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float slope;
            du[e] = c[e] * activation(w.gelu, g[e], &slope);
            dg[e] = c[e] * u[e] * slope;
        }
        store4(static_cast<T *>(p.c) + to, dg);
        store4(static_cast<T *>(p.c) + int64_t(p.m) * p.n + to, du);
    } else if (w.slices > 1) {
        store4(w.partial + slice * w.slice_size + p.partial + int64_t(m) * p.n + n, c);
    } else {
        store4(static_cast<T *>(p.c) + m * p.c_row + n, c);
    }
}

// Columns of a tile lie in two halves of BN / 2 (of a gated product: of gate and
// up).  Four waves, two by two.
template <typename T, bool AK, bool BK, int EPI, int BM, int BN>
__global__ __launch_bounds__(256) void k_product(Work w) {
    constexpr int EL = sizeof(T), MT = BM / 32, NT = BN / 64;
    typedef Panel<T, AK, BM> PA;
    typedef Panel<T, BK, BN / 2> PB;
    constexpr uint32_t kStage = PA::kBytes + 2 * PB::kBytes;
    __shared__ __attribute__((aligned(1024))) char lds[2 * kStage];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const Spot at_tile = spot(w);
    if (at_tile.which < 0) return;
    const Product p = pick(w, at_tile.which);
    const int slice = at_tile.slice;
    const int m0 = at_tile.tile_m * BM, n0 = at_tile.tile_n * (EPI == kGated ? BN / 2 : BN);
    const int steps = (p.k + kStep<T> - 1) / kStep<T>;
    const int first = slice * w.per_slice, last = min(first + w.per_slice, steps * w.segments);

    const uint32_t base = lds_offset(lds), part = uint32_t(wave) * 1024u;
    typename PA::template Stager<256> sa;
    typename PB::template Stager<256> sb[2];
    int segment = first >= steps;
    auto aim = [&]() {
        sa.init(threadIdx.x, p.a_row, int64_t(p.m - m0) * EL);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            sb[h].init(threadIdx.x, (EPI == kGated ? h : segment) ? p.b_row[1] : p.b_row[0], int64_t(p.n - n0 - (EPI == kGated ? 0 : h * (BN / 2))) * EL);
    };
    auto load = [&](int step, uint32_t to) {
        if (w.segments == 2 && segment == 0 && step >= steps) {
            segment = 1;
            aim();
        }
        const int64_t k0 = int64_t(step - segment * steps) * kStep<T>;
        const int left = int(p.k - k0);
        sa.load((segment ? p.a[1] : p.a[0]) + (AK ? m0 * int64_t(p.a_row) + k0 * EL : k0 * p.a_row + int64_t(m0) * EL), p.a_row, p.m - m0,
                left, to, part);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t row = (EPI == kGated ? h : segment) ? p.b_row[1] : p.b_row[0];
            const int at = n0 + (EPI == kGated ? 0 : h * (BN / 2));
            const char *src = (EPI == kGated ? h : segment) ? p.b[1] : p.b[0];
            sb[h].load(src + (BK ? at * int64_t(row) + k0 * EL : k0 * row + int64_t(at) * EL), row, p.n - at, left,
                       to + PA::kBytes + h * PB::kBytes, part);
        }
    };

    typename PA::template Lanes<MT> la;
    typename PB::template Lanes<NT> lb;
    la.init(lane, base, wm * (BM / 2));
    lb.init(lane, base + PA::kBytes, wn * (BN / 4));
    f32x4_t acc[MT][2][NT] = {};
    aim();
    if (first < last) load(first, base);
    for (int step = first; step < last; ++step) {
        // this step's tiles are there, and the other buffer is free
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const uint32_t at = ((step - first) & 1) * kStage;
        if (step + 1 < last) load(step + 1, base + (kStage - at));
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            u32x4_t fa[MT], fb[2][NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) fa[i] = la.frag(i, s, at);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < NT; ++j) fb[h][j] = lb.frag(j, s, at + h * PB::kBytes);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][h][j] = mma(T(), fb[h][j], fa[i], acc[i][h][j]);
        }
    }

    const int fr = lane & 15, fk = lane >> 4;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = m0 + wm * (BM / 2) + 16 * i + fr;
        if (m >= p.m) continue;
#pragma unroll
        for (int h = 0; h < (EPI == kGated ? 1 : 2); ++h)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int n = n0 + h * (BN / 2) + wn * (BN / 4) + 16 * j + 4 * fk;
                if (n < p.n) finish<T, EPI>(w, p, slice, m, n, acc[i][h][j], acc[i][1][j]);
            }
    }
}

// bf16, tiles of 256 x 256, eight waves of 128 x 64: rows 64 wm .. of both halves of
// the tile's rows, columns 32 wn .. of both halves of its columns.  A step's four
// panels (two halves of A, two of B) have two buffers.  A wave goes through a step in
// four phases, each a quarter of its results:
//   1: reads A0             products of A0, B0     (B0 is in registers)
//   2: reads B1             products of A0, B1
//   3: reads A1             products of A1, B1
//   4: reads the next B0    products of A1, B0
// A phase reads, waits, meets the other waves at a barrier, multiplies, and meets
// them again.  Waves 4 .. 7 (the second wave of every SIMD) run one barrier behind,
// so that on each SIMD one wave multiplies while the other reads.  A panel that
// phase p has read is free in phase p + 1 and filled there with its values of two
// steps later; loads are waited for one phase before they are read, with those of
// the last six panels still under way.
template <bool AK, bool BK, int EPI>
__global__ __launch_bounds__(512) void k_product_large(Work w) {
    typedef uint16_t T;
    constexpr int EL = 2, BM = 256, BN = 256;
    typedef Panel<T, AK, 128> PA;
    typedef Panel<T, BK, 128> PB;
    constexpr uint32_t kPanel = 128 * 128, kStage = 4 * kPanel;
    constexpr uint32_t kA0 = 0, kA1 = kPanel, kB0 = 2 * kPanel, kB1 = 3 * kPanel;
    __shared__ __attribute__((aligned(1024))) char lds[2 * kStage];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 2, wn = wave & 3;
    const Spot at_tile = spot(w);
    if (at_tile.which < 0) return;
    const Product p = pick(w, at_tile.which);
    const int slice = at_tile.slice;
    const int m0 = at_tile.tile_m * BM, n0 = at_tile.tile_n * (EPI == kGated ? BN / 2 : BN);
    const int steps = (p.k + kStep<T> - 1) / kStep<T>;
    const int first = slice * w.per_slice, last = min(first + w.per_slice, steps * w.segments);

    const uint32_t base = lds_offset(lds), part = uint32_t(wave) * 1024u;
    typename PA::template Stager<512> sa[2];
    typename PB::template Stager<512> sb[2];
    static_assert(sa[0].kLoads == 2 && sb[0].kLoads == 2, "the waits count two loads a panel");
    auto aim_b = [&](int h, int segment) {
        sb[h].init(threadIdx.x, (EPI == kGated ? h : segment) ? p.b_row[1] : p.b_row[0], int64_t(p.n - n0 - (EPI == kGated ? 0 : h * 128)) * EL);
    };
    // The panels of half h in the buffer `to`; past the slice's end nothing is
    // fetched and zeros are stored, so that the number of loads stays the same.
    auto load_a = [&](int h, int step, uint32_t to) {
        const int segment = w.segments == 2 && step >= steps;
        const int64_t k0 = int64_t(step - segment * steps) * kStep<T>;
        const int left = step < last ? int(p.k - k0) : 0, at = m0 + h * 128;
        sa[h].load((segment ? p.a[1] : p.a[0]) + (AK ? at * int64_t(p.a_row) + k0 * EL : k0 * p.a_row + int64_t(at) * EL), p.a_row, p.m - at,
                   left, to + (h ? kA1 : kA0), part);
    };
    auto load_b = [&](int h, int step, uint32_t to) {
        const int segment = w.segments == 2 && step >= steps;
        if (w.segments == 2 && step == steps) aim_b(h, 1);
        const int64_t k0 = int64_t(step - segment * steps) * kStep<T>;
        const uint32_t row = (EPI == kGated ? h : segment) ? p.b_row[1] : p.b_row[0];
        const int left = step < last ? int(p.k - k0) : 0, at = n0 + (EPI == kGated ? 0 : h * 128);
        const char *src = (EPI == kGated ? h : segment) ? p.b[1] : p.b[0];
        sb[h].load(src + (BK ? at * int64_t(row) + k0 * EL : k0 * row + int64_t(at) * EL), row, p.n - at, left,
                   to + (h ? kB1 : kB0), part);
    };

    typename PA::template Lanes<4> la;
    typename PB::template Lanes<2> lb;
    la.init(lane, base, wm * 64);
    lb.init(lane, base, wn * 32);
    f32x4_t acc[2][4][2][2] = {};
    u32x4_t a[4][2], b0[2][2], b1[2][2], next[2][2];
    auto read_a = [&](uint32_t at) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int s = 0; s < 2; ++s) a[i][s] = la.frag(i, s, at);
    };
    auto read_b = [&](u32x4_t(&b)[2][2], uint32_t at) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int s = 0; s < 2; ++s) b[j][s] = lb.frag(j, s, at);
    };
    // the phase's reads have returned, and the next phase's panel has landed
    auto meet_read = [&]() {
        asm volatile("s_waitcnt vmcnt(12) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
    };
    auto meet = [&]() {
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](f32x4_t(&c)[4][2][2], int h, const u32x4_t(&b)[2][2]) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) c[i][h][j] = mma(T(), b[j][s], a[i][s], c[i][h][j]);
    };

    const int segment = first >= steps;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        sa[h].init(threadIdx.x, p.a_row, int64_t(p.m - m0 - h * 128) * EL);
        aim_b(h, segment);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        load_b(0, first + t, base + t * kStage);
        load_a(0, first + t, base + t * kStage);
        load_b(1, first + t, base + t * kStage);
        load_a(1, first + t, base + t * kStage);
    }
    asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read_b(b0, kB0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    if (wave >= 4) __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    for (int step = first; step < last; ++step) {
        const uint32_t at = ((step - first) & 1) * kStage, to = base + at;
        read_a(at + kA0);
        load_b(0, step + 2, to);
        meet_read();
        multiply(acc[0], 0, b0);
        meet();
        read_b(b1, at + kB1);
        load_a(0, step + 2, to);
        meet_read();
        multiply(acc[0], 1, b1);
        meet();
        read_a(at + kA1);
        load_b(1, step + 2, to);
        meet_read();
        multiply(acc[1], 1, b1);
        meet();
        read_b(next, (kStage - at) + kB0);
        load_a(1, step + 2, to);
        meet_read();
        multiply(acc[1], 0, b0);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int s = 0; s < 2; ++s) b0[j][s] = next[j][s];
        meet();
    }
    if (wave < 4) __builtin_amdgcn_s_barrier();
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load into LDS outlives the block

    const int fr = lane & 15, fk = lane >> 4;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = m0 + g * 128 + wm * 64 + 16 * i + fr;
            if (m >= p.m) continue;
#pragma unroll
            for (int h = 0; h < (EPI == kGated ? 1 : 2); ++h)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int n = n0 + h * 128 + wn * 32 + 16 * j + 4 * fk;
                    if (n < p.n) finish<T, EPI>(w, p, slice, m, n, acc[g][i][h][j], acc[g][i][1][j]);
                }
        }
}

// Adds up the slices in their order and rounds.
template <typename T>
__global__ __launch_bounds__(256) void k_join_slices(Work w) {
    for (int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4; i < w.slice_size; i += int64_t(gridDim.x) * 1024) {
        int which = 0;
        while (which + 1 < w.products && i >= w.p[which + 1].partial) ++which;
        const Product &p = w.p[which];
        f32x4_t sum = load4(w.partial + i);
        for (int s = 1; s < w.slices; ++s) sum += load4(w.partial + s * w.slice_size + i);
        const int64_t at = i - p.partial, m = at / p.n;
        store4(static_cast<T *>(p.c) + m * p.c_row + (at - m * p.n), sum);
    }
}

// ------------------------------------------------------------------------ plan

// Tile sizes and slices of a launch of products with one contracted length.
struct Plan {
    int bm, bn, slices, per_slice, steps;
    size_t partial;  // bytes
};

struct Size {
    int64_t m, n;
};

// cols: columns of a result that a tile of bn holds: bn, or half of a gated one.
int64_t tiles_of(const Size &s, int bm, int cols) { return ((s.m + bm - 1) / bm) * ((s.n + cols - 1) / cols); }

Plan plan(const Size *sizes, int count, bool bf16, int64_t k, int segments, Epilogue epi) {
    const int cus = compute_units(), step = bf16 ? 64 : 32;
    Plan p{128, 128, 1, 0, int((k + step - 1) / step) * segments, 0};
    auto tiles = [&](int b) {
        int64_t n = 0;
        for (int i = 0; i < count; ++i) n += tiles_of(sizes[i], b, epi == kGated ? b / 2 : b);
        return n;
    };
    if (bf16 && tiles(256) >= cus) p.bm = p.bn = 256;
    else if (tiles(128) < cus) p.bm = p.bn = 64;
    if (epi == kPlain) {
        const int64_t n = tiles(p.bm);
        // slices of four steps at least, until two blocks a CU
        if (n < cus) p.slices = int(std::max<int64_t>(1, std::min<int64_t>(p.steps / 4, 2 * cus / std::max<int64_t>(n, 1))));
    }
    p.per_slice = (p.steps + p.slices - 1) / p.slices;
    p.slices = p.per_slice ? (p.steps + p.per_slice - 1) / p.per_slice : 1;
    if (p.slices > 1) {
        int64_t values = 0;
        for (int i = 0; i < count; ++i) values += sizes[i].m * sizes[i].n;
        p.partial = size_t(values) * p.slices * sizeof(float);
    }
    return p;
}

template <typename T, bool AK, bool BK, int EPI>
hipError_t launch(Work &w, const Plan &plan, float *partial, hipStream_t s) {
    int64_t blocks = 0;
    w.slices = plan.slices;
    w.per_slice = plan.per_slice;
    w.partial = partial;
    w.slice_size = 0;
    for (int i = 0; i < w.products; ++i) {
        Product &p = w.p[i];
        const int cols = EPI == kGated ? plan.bn / 2 : plan.bn;
        p.tiles_n = (p.n + cols - 1) / cols;
        p.tiles = int(tiles_of({p.m, p.n}, plan.bm, cols));
        p.partial = w.slice_size;
        w.slice_size += int64_t(p.m) * p.n;
        blocks += int64_t(p.tiles) * plan.slices;
    }
    const Fold f = fold(blocks, 512);
    if (plan.bm == 256) {
        if constexpr (sizeof(T) == 2) k_product_large<AK, BK, EPI><<<dim3(f.x, 1, f.z), 512, 0, s>>>(w);
    } else if (plan.bm == 128) k_product<T, AK, BK, EPI, 128, 128><<<dim3(f.x, 1, f.z), 256, 0, s>>>(w);
    else k_product<T, AK, BK, EPI, 64, 64><<<dim3(f.x, 1, f.z), 256, 0, s>>>(w);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.slices == 1) return e;
    k_join_slices<T><<<int(std::min<int64_t>((w.slice_size + 1023) / 1024, 8 * compute_units())), 256, 0, s>>>(w);
    return hipGetLastError();
}

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

Plan plan_gated(const FfnArgs &a) {
    const Size s{a.rows, a.hidden};
    return plan(&s, 1, a.bf16, a.channels, 1, kGated);
}
Plan plan_down(const FfnArgs &a) {
    const Size s{a.rows, a.channels};
    return plan(&s, 1, a.bf16, a.hidden, 1, kPlain);
}
Plan plan_dhidden(const FfnArgs &a) {
    const Size s{a.rows, a.hidden};
    return plan(&s, 1, a.bf16, a.channels, 1, kGatedGrad);
}
Plan plan_dx(const FfnArgs &a) {
    const Size s{a.rows, a.channels};
    return plan(&s, 1, a.bf16, a.hidden, 2, kPlain);
}
Plan plan_weights(const FfnArgs &a) {
    Size s[kMaxProducts];
    int n = 0;
    if (a.dw_gate) s[n++] = {a.hidden, a.channels};
    if (a.dw_up) s[n++] = {a.hidden, a.channels};
    if (a.dw_down) s[n++] = {a.channels, a.hidden};
    return plan(s, n, a.bf16, a.rows, 1, kPlain);
}

bool wants_hidden(const FfnArgs &a) { return a.dx || a.dw_gate || a.dw_up; }
size_t hidden_bytes(const FfnArgs &a) { return size_t(a.rows) * a.hidden * (a.bf16 ? 2 : 4); }

template <typename T>
hipError_t forward(FfnArgs a, hipStream_t s) {
    char *space = static_cast<char *>(a.workspace);
    const bool saved = a.act;
    if (!saved) {
        a.act = space;
        a.hidden_s = a.hidden;
        space += round16(hidden_bytes(a));
    }
    Work w{};
    w.products = w.segments = 1;
    w.gelu = a.gelu;
    w.gate = a.gate, w.up = a.up, w.act = a.act, w.hidden_s = a.hidden_s;
    Product &p = w.p[0];
    p.a[0] = static_cast<const char *>(a.x);
    p.b[0] = static_cast<const char *>(a.w_gate), p.b[1] = static_cast<const char *>(a.w_up);
    p.a_row = uint32_t(a.x_s * sizeof(T));
    p.b_row[0] = uint32_t(a.w_gate_s * sizeof(T)), p.b_row[1] = uint32_t(a.w_up_s * sizeof(T));
    p.m = a.rows, p.n = a.hidden, p.k = a.channels;
    hipError_t e = launch<T, true, true, kGated>(w, plan_gated(a), nullptr, s);
    if (e != hipSuccess) return e;
    p = Product{};
    p.a[0] = static_cast<const char *>(a.act);
    p.b[0] = static_cast<const char *>(a.w_down);
    p.a_row = uint32_t(a.hidden_s * sizeof(T)), p.b_row[0] = uint32_t(a.w_down_s * sizeof(T));
    p.m = a.rows, p.n = a.channels, p.k = a.hidden;
    p.c = a.out, p.c_row = a.out_s;
    return launch<T, true, true, kPlain>(w, plan_down(a), reinterpret_cast<float *>(space), s);
}

template <typename T>
hipError_t gradient(const FfnArgs &a, hipStream_t s) {
    char *dgate = static_cast<char *>(a.workspace), *dup = dgate + hidden_bytes(a);
    float *partial = reinterpret_cast<float *>(dgate + (wants_hidden(a) ? round16(2 * hidden_bytes(a)) : 0));
    const uint32_t hidden_row = uint32_t(a.hidden * sizeof(T)), saved_row = uint32_t(a.hidden_s * sizeof(T));
    const uint32_t dout_row = uint32_t(a.dout_s * sizeof(T));
    hipError_t e;
    if (a.rows > 0 && wants_hidden(a)) {
        Work w{};
        w.products = w.segments = 1;
        w.gelu = a.gelu;
        w.gate = a.gate, w.up = a.up, w.hidden_s = a.hidden_s;
        Product &p = w.p[0];
        p.a[0] = static_cast<const char *>(a.dout), p.b[0] = static_cast<const char *>(a.w_down);
        p.a_row = dout_row, p.b_row[0] = uint32_t(a.w_down_s * sizeof(T));
        p.m = a.rows, p.n = a.hidden, p.k = a.channels;
        p.c = dgate;
        if ((e = launch<T, true, false, kGatedGrad>(w, plan_dhidden(a), nullptr, s)) != hipSuccess) return e;
    }
    if (a.rows > 0 && a.dx) {
        Work w{};
        w.products = 1, w.segments = 2;
        Product &p = w.p[0];
        p.a[0] = dgate, p.a[1] = dup;
        p.b[0] = static_cast<const char *>(a.w_gate), p.b[1] = static_cast<const char *>(a.w_up);
        p.a_row = hidden_row;
        p.b_row[0] = uint32_t(a.w_gate_s * sizeof(T)), p.b_row[1] = uint32_t(a.w_up_s * sizeof(T));
        p.m = a.rows, p.n = a.channels, p.k = a.hidden;
        p.c = a.dx, p.c_row = a.dx_s;
        if ((e = launch<T, true, false, kPlain>(w, plan_dx(a), partial, s)) != hipSuccess) return e;
    }
    Work w{};
    w.segments = 1;
    auto add = [&](void *c, int64_t c_row, const void *from, uint32_t from_row, const void *with, uint32_t with_row, int m, int n) {
        if (!c) return;
        Product &p = w.p[w.products++];
        p.a[0] = static_cast<const char *>(from), p.b[0] = static_cast<const char *>(with);
        p.a_row = from_row, p.b_row[0] = with_row;
        p.m = m, p.n = n, p.k = a.rows;
        p.c = c, p.c_row = c_row;
    };
    const uint32_t x_row = uint32_t(a.x_s * sizeof(T));
    add(a.dw_gate, a.dw_gate_s, dgate, hidden_row, a.x, x_row, a.hidden, a.channels);
    add(a.dw_up, a.dw_up_s, dup, hidden_row, a.x, x_row, a.hidden, a.channels);
    add(a.dw_down, a.dw_down_s, a.dout, dout_row, a.act, saved_row, a.channels, a.hidden);
    if (!w.products) return hipSuccess;
    return launch<T, false, false, kPlain>(w, plan_weights(a), partial, s);
}

}  // namespace

size_t gated_ffn_workspace(const FfnArgs &a) {
    if (a.rows == 0) return 0;
    return (a.act ? 0 : round16(hidden_bytes(a))) + plan_down(a).partial;
}

int gated_ffn(const FfnArgs &a, void *stream) {
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.bf16 ? forward<uint16_t>(a, s) : forward<float>(a, s);
}

size_t gated_ffn_grad_workspace(const FfnArgs &a) {
    const size_t hidden = wants_hidden(a) ? round16(2 * hidden_bytes(a)) : 0;
    const size_t dx = a.dx && a.rows ? plan_dx(a).partial : 0;
    const size_t weights = a.dw_gate || a.dw_up || a.dw_down ? plan_weights(a).partial : 0;
    return hidden + std::max(dx, weights);
}

int gated_ffn_grad(const FfnArgs &a, void *stream) {
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.bf16 ? gradient<uint16_t>(a, s) : gradient<float>(a, s);
}

}  // namespace kern
}  // namespace rtcc
