// Gated feed-forward unit on gfx950, and its gradients.
//
//   G = X Wg', U = X Wu', H = act(G) U, Y = H Wd'
//   dH = dY Wd, dU = dH act(G), dG = dH U act'(G)
//   dX = dG Wg + dU Wu, dWg = dG' X, dWu = dU' X, dWd = dY' H
//
// Products are tiles of one matrix kernel in three forms: k_product (tiles of 128 or
// 64, two to five blocks a CU), k_product_large (256, one block a CU that stays) and
// k_few (up to 16 rows, no tiles).  plan() chooses tiles and slices of the contracted
// axis by a model of their times.
//   G and U together: a tile's columns are halves of Wg and of Wu, so a lane has g
//     and u of the same places in its registers and stores h
//   dH: the results read g and u and become dG and dU before they are stored
//   dX: the contracted axis runs over Wg's rows, then Wu's
//   dWg, dWu, dWd: up to three products of one launch, which may hold dX's too
//     (k_products)
// Operands whose contracted axis is in rows are read transposed from LDS, so no
// tensor is laid out anew.
//
// bf16 rounds what is stored and then multiplied: h, dG and dU (matrix operands), and
// g and u where a gradient will read them.  Against 64-bit gradients dX, dWg and dWu
// are 0.30% off (root mean square; rounding the result alone: 0.17%).  Stored in
// float32, g and u would leave 0.24%, for 200 MB more traffic in the 275 us of a step
// over 16,384 rows of 384 channels, 1,536 hidden: some 40 us.  All sums are float32.
//
// What bounds them (kernel times of one MI355X): 16,384 rows, 2,048 channels, 8,192
// hidden: matrix units 53 to 66% busy at 2.0 GHz (the power limit's clock), 1,120 to
// 1,370 TFLOP/s (dG and dU 40%, 890: their tiles end in the most work); the LDS takes 2,560 cycles a step of 256 x 256 x 64 (64 KB written
// at 64 bytes a cycle, 192 KB read at 128) beside 2,048 of products.  16,384 rows of
// 384 channels, 1,536 hidden: 275 us a step with 1.0 GB of traffic (200 us at a copy's
// rate) and contracted axes of six steps, after which a tile's results cost as much.
#include <algorithm>
#include <initializer_list>
#include <string>

#include <hip/hip_runtime.h>

#include "compute_units.hpp"
#include "ffn_plan.hpp"
#include "matrix_overlap.hpp"
#include "products.hpp"
#include "token_ops.hpp"

namespace rtcc {
namespace kern {

namespace {

// ------------------------------------------------------------------ activation

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Activation of z; *slope, where asked for, its derivative.
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
template <bool GELU>
__device__ inline float activation(float z, float *slope) {
    return GELU ? gelu(z, slope) : silu(z, slope);
}

// -------------------------------------------------------------------- products

// C [m][n] = sum over segments and k of A [m][k] B [n][k]; where K is in rows, A
// is [k][m] and B [k][n].
struct Product {
    const char *a[2], *b[2];  // of each segment; of a gated product b are the halves of a tile's columns
    uint32_t a_row, b_row[2];  // bytes between rows
    int32_t m, n, k;           // k: of a segment
    int32_t tiles_m, tiles_n, tiles;
    void *c;
    int64_t c_row;  // elements
    int64_t partial;  // floats before the product's part of a slice
};
struct Work {
    Product p[kMaxProducts];
    int32_t products;
    int32_t slices, per_slice;  // of the contracted axis, and steps of each
    float *partial;             // [slices][slice_size]
    int64_t slice_size;
    // gated products: [m][n] of one stride (elements)
    bool gelu;
    void *gate, *up, *act;
    int64_t hidden_s;
};

// The product, the slice and the tile of a block.  Blocks of one XCD (every eighth)
// take tiles that follow each other, in bands of kBand tiles of rows, so that their
// operands meet in its L2.  A step over 16,384 rows of 2,048 channels, 8,192 hidden:
// 4.05 ms in bands of 4, 4.07 of 2, 4.15 of 8, 4.20 of 16.
struct Spot {
    int which, slice, tile_m, tile_n;  // which < 0: none, past the last one
};
constexpr int kBand = 4;
__device__ inline Spot spot(const Work &w, uint32_t id) {
    int which = 0, slice = 0;
    uint32_t tiles = w.p[0].tiles, across = w.p[0].tiles_n, down = w.p[0].tiles_m;
    if (w.products > 1) {
#pragma unroll
        for (int i = 1; i < kMaxProducts; ++i)
            if (which == i - 1 && i < w.products && id >= tiles * w.slices) {
                id -= tiles * w.slices;
                which = i, tiles = w.p[i].tiles, across = w.p[i].tiles_n, down = w.p[i].tiles_m;
            }
    }
    const uint32_t n = tiles * w.slices, x = id % 8;
    if (id >= n) return {-1, 0, 0, 0};
    id = x * (n / 8) + min(x, n % 8) + id / 8;
    if (w.slices > 1) {
        slice = int(id / tiles);
        id -= slice * tiles;
    }
    // one division where the band is whole: each costs some 40 instructions, and a
    // tile of the smallest step counts takes a few thousand cycles
    const uint32_t top = id / (kBand * across) * kBand, rows = min(down - top, uint32_t(kBand));
    id -= top * across;
    const uint32_t n_at = rows == kBand ? id / kBand : id / rows;
    // said to be uniform, so that all addresses stay in scalar registers
    return {__builtin_amdgcn_readfirstlane(which), __builtin_amdgcn_readfirstlane(slice),
            __builtin_amdgcn_readfirstlane(top + (id - n_at * rows)), __builtin_amdgcn_readfirstlane(n_at)};
}
// A copy by constant indexes: an indexed one would go through memory.
__device__ inline Product pick(const Work &w, int which) { return which == 0 ? w.p[0] : which == 1 ? w.p[1] : w.p[2]; }

// What a lane holds of a result: eight neighbouring columns of row m from column n on.
struct Place {
    int m, n;
};

// Stores a lane's UNITS results; at(u) is the place of the u-th, take(u, c, d) gives
// its values c (a gated product's: of gate, with those of up in d).
template <typename T, int EPI, int UNITS, bool GELU, class At, class Take>
__device__ inline void finish_with(const Work &w, const Product &p, int slice, At at, Take take) {
    if constexpr (EPI == kGatedGrad) {
        // g and u a batch ahead: the loads are waited for together, from places
        // that always exist
        constexpr int kBatch = UNITS == 8 ? 4 : 2, kBatches = UNITS / kBatch;  // as the registers allow
        static_assert(UNITS % kBatch == 0, "whole batches");
        Eight<T> g[2][kBatch], u[2][kBatch];
        auto fetch = [&](int b) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const Place o = at(b * kBatch + i);
                const int64_t from = min(o.m, p.m - 1) * w.hidden_s + min(o.n, p.n - 8);
                g[b & 1][i].load(static_cast<const T *>(w.gate) + from);
                u[b & 1][i].load(static_cast<const T *>(w.up) + from);
            }
        };
        fetch(0);
#pragma unroll
        for (int b = 0; b < kBatches; ++b) {
            if (b + 1 < kBatches) fetch(b + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const Place o = at(b * kBatch + i);
                float c[8], dg[8], du[8];
                take(b * kBatch + i, c, nullptr);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float slope;
                    du[e] = c[e] * activation<GELU>(g[b & 1][i][e], &slope);
                    dg[e] = c[e] * u[b & 1][i][e] * slope;
                }
                if (o.m >= p.m || o.n >= p.n) continue;
                const int64_t to = int64_t(o.m) * p.n + o.n;
                store8(static_cast<T *>(p.c) + to, dg);
                store8(static_cast<T *>(p.c) + int64_t(p.m) * p.n + to, du);
                __builtin_amdgcn_sched_barrier(0);  // more at once would not fit the registers
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const Place o = at(i);
            float c[8], d[8];
            take(i, c, d);
            if constexpr (EPI == kGated) {
                float h[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) h[e] = activation<GELU>(c[e], nullptr) * d[e];
                if (o.m >= p.m || o.n >= p.n) continue;
                const int64_t to = o.m * w.hidden_s + o.n;
                store8(static_cast<T *>(w.act) + to, h);
                if (w.gate) {
                    store8(static_cast<T *>(w.gate) + to, c);
                    store8(static_cast<T *>(w.up) + to, d);
                }
            } else {
                if (o.m >= p.m || o.n >= p.n) continue;
                if (w.slices > 1) store8(w.partial + slice * w.slice_size + p.partial + int64_t(o.m) * p.n + o.n, c);
                else store8(static_cast<T *>(p.c) + o.m * p.c_row + o.n, c);
            }
            if (EPI == kGated) __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// One branch for all of a lane's results: with one for each, no two of them overlap.
template <typename T, int EPI, int UNITS, class At, class Take>
__device__ inline void finish(const Work &w, const Product &p, int slice, At at, Take take) {
    if (EPI != kPlain && w.gelu) finish_with<T, EPI, UNITS, true>(w, p, slice, at, take);
    else finish_with<T, EPI, UNITS, false>(w, p, slice, at, take);
}

// Columns of a tile lie in two halves of BN / 2 (of a gated product: of gate and
// up).  Four waves, two by two.  STAGES buffers form a ring: the loads run STAGES - 1
// steps ahead.  A step has two halves, whose fragments have registers of their own:
// one half's are read while the other's are multiplied.  Reads and loads stand
// between the products, so that one wave on a SIMD keeps all units busy.  The LDS
// bounds it: 1,024 cycles a step of 128 x 128 x 64 bf16 (32 KB written, 64 KB read)
// beside 512 of products.  Four buffers for two where a CU has one or two small tiles
// (64 rows, 2,048 channels, 8,192 hidden: 17 us for 27, 10 for 15.5); elsewhere they
// change nothing.
template <typename T, int BM, int STAGES>
constexpr uint32_t kProductLds = STAGES * 2 * BM * 128;  // a step is 128 bytes, tiles are square

template <typename T, bool AK, bool BK, int EPI, int BM, int STAGES>
__device__ inline void product(const Work &w, uint32_t id, char *lds) {
    constexpr int BN = BM, MT = BM / 32, NT = BN / 64;
    constexpr bool kGate = EPI == kGated, kTwo = EPI == kPlain && AK && !BK;  // kTwo: two segments
    typedef Panel<T, AK, BM> PA;
    typedef Panel<T, BK, BN / 2> PB;
    typedef typename PA::template Feed<256> FA;
    typedef typename PB::template Feed<256> FB;
    constexpr uint32_t kStage = PA::kBytes + 2 * PB::kBytes;
    constexpr int kLoads = FA::kLoads + 2 * FB::kLoads, kStep = PA::kStep;
    static_assert(STAGES * kStage == kProductLds<T, BM, STAGES>, "LDS of a block");

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const Spot tile = spot(w, id);
    if (tile.which < 0) return;
    const Product p = pick(w, tile.which);
    const int m0 = tile.tile_m * BM, n0 = tile.tile_n * (kGate ? BN / 2 : BN);
    const int steps = (p.k + kStep - 1) / kStep;  // of a segment
    const int first = tile.slice * w.per_slice, last = min(first + w.per_slice, steps * (kTwo ? 2 : 1));

    FA fa;
    FB fb[2];
    Steps walk;
    int switch_in = 0;  // steps before the second segment
    auto aim = [&](int segment, int step) {
        fa.init(threadIdx.x, segment ? p.a[1] : p.a[0], p.a_row, m0, p.m - m0, step);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = n0 + (kGate ? 0 : h * (BN / 2)), from = kGate ? h : segment;
            fb[h].init(threadIdx.x, from ? p.b[1] : p.b[0], from ? p.b_row[1] : p.b_row[0], at, p.n - at, step);
        }
        walk.left = p.k - step * kStep;
    };
    const int segment = kTwo && first >= steps;
    aim(segment, first - segment * steps);
    walk.more = last - first;
    if (kTwo) switch_in = segment ? -1 : steps - first;

    // A step's loads, one at a time.
    const uint32_t base = lds_offset(lds), part = uint32_t(wave) * 1024u;
    u32x4_t ra, rb[2];
    int k = 0;
    auto prepare = [&]() {
        if (kTwo && switch_in-- == 0) aim(1, 0);
        k = walk.next<kStep>();
        ra = fa.next(k);
        rb[0] = fb[0].next(k);
        rb[1] = fb[1].next(k);
    };
    auto load = [&](int n, uint32_t to) {
        if (n < FA::kLoads) fa.load(n, ra, k, to + part);
        else if (n < FA::kLoads + FB::kLoads) fb[0].load(n - FA::kLoads, rb[0], k, to + PA::kBytes + part);
        else fb[1].load(n - FA::kLoads - FB::kLoads, rb[1], k, to + PA::kBytes + PB::kBytes + part);
    };

    typename PA::template Lanes<MT> la;
    typename PB::template Lanes<NT> lb;
    la.init(lane, base, wm * (BM / 2));
    lb.init(lane, base + PA::kBytes, wn * (BN / 4));
    f32x4_t acc[MT][2][NT] = {};
    u32x4_t a[2][MT], b[2][2][NT];
    constexpr int kReads = MT + 2 * NT;
    auto read = [&](int n, int s, uint32_t at) {
        if (n < MT) a[s][n] = la.frag(n, s, at);
        else b[s][(n - MT) / NT][(n - MT) % NT] = lb.frag((n - MT) % NT, s, at + (n - MT) / NT * PB::kBytes);
    };
    // The products of half s, with `items` calls of item spread between them.
    auto multiply = [&](int s, int items, auto item) {
        constexpr int kAll = MT * 2 * NT * kMmaSteps<T>;
        int done = 0;
#pragma unroll
        for (int e = 0; e < kMmaSteps<T>; ++e)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        const int q = ((e * MT + i) * 2 + h) * NT + j;
                        acc[i][h][j] = mma(T(), e, b[s][h][j], a[s][i], acc[i][h][j]);
#pragma unroll
                        for (; done < (q + 1) * items / kAll; ++done) item(done);
                        __builtin_amdgcn_sched_barrier(0);
                    }
    };
    // the next step's panels have landed and this wave's reads have returned: so
    // they have for all waves
    auto meet = [&]() {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES - 2) * kLoads) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int t = 0; t < STAGES; ++t) {
        if (t == STAGES - 1) meet();
        prepare();
#pragma unroll
        for (int n = 0; n < kLoads; ++n) load(n, base + t * kStage);
    }
#pragma unroll
    for (int n = 0; n < kReads; ++n) read(n, 0, 0);
    uint32_t at = 0;
    for (int step = first; step < last; ++step) {
        const uint32_t then = at + kStage == STAGES * kStage ? 0 : at + kStage;
        multiply(0, kReads + 1, [&](int n) {
            if (n < kReads) read(n, 1, at);
            else prepare();
        });
        meet();
        // bf16: loads first, each with a read: they have the longer way.  float32,
        // whose products take 16 times as long, has the reads first.
        multiply(1, kReads + kLoads, [&](int n) {
            constexpr int kBoth = sizeof(T) == 2 ? 2 * (kReads < kLoads ? kReads : kLoads) : 0;
            if (n < kBoth && n % 2 == 0) load(n / 2, base + at);
            else if (n < kBoth) read(n / 2, 0, then);
            else if (n < kReads + kBoth / 2) read(n - kBoth / 2, 0, then);
            else load(n - kReads, base + at);
        });
        at = then;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load into LDS outlives the block

    // pairs of tiles side by side, or below each other where there is one
    constexpr int kDown = NT == 1 ? 2 : 1;
    static_assert(NT * kDown == 2, "pairs");
    const int fr = lane & 15, second = (lane >> 4) & 1, col = (lane >> 5) * 8;
    // unit u: half h = u % kHalves, rows i = u / kHalves * kDown
    constexpr int kHalves = kGate ? 1 : 2, kUnits = MT / kDown * kHalves;
    auto place = [&](int u) -> Place {
        return {m0 + wm * (BM / 2) + 16 * (u / kHalves * kDown + (kDown - 1) * second) + fr,
                n0 + u % kHalves * (BN / 2) + wn * (BN / 4) + 16 * (NT - 1) * second + col};
    };
    finish<T, EPI, kUnits>(w, p, tile.slice, place, [&](int u, float *c, float *d) {
        const int i = u / kHalves * kDown, h = u % kHalves;
        pair_up(acc[i][h][0], acc[i + kDown - 1][h][NT - 1], c);
        if (kGate) pair_up(acc[i][1][0], acc[i + kDown - 1][1][NT - 1], d);
    });
}

template <typename T, bool AK, bool BK, int EPI, int BM, int STAGES>
__global__ __launch_bounds__(256, 2) void k_product(Work w) {
    __shared__ __attribute__((aligned(1024))) char lds[kProductLds<T, BM, STAGES>];
    product<T, AK, BK, EPI, BM, STAGES>(w, blockIdx.z * gridDim.x + blockIdx.x, lds);
}

// dX and the weights' gradients, neither of which needs the other's, in one launch;
// first: blocks of those with more steps, which start first (x_first: dX's).
template <typename T, int BM, int STAGES>
__global__ __launch_bounds__(256, 2) void k_products(Work x, Work w, uint32_t first, bool x_first) {
    __shared__ __attribute__((aligned(1024))) char lds[kProductLds<T, BM, STAGES>];
    uint32_t id = blockIdx.z * gridDim.x + blockIdx.x;
    const bool early = id < first;
    id = early ? id : id - first;
    if (early == x_first) product<T, true, false, kPlain, BM, STAGES>(x, id, lds);
    else product<T, false, false, kPlain, BM, STAGES>(w, id, lds);
}

// bf16, tiles of 256 x 256, eight waves of 128 x 64: rows 64 wm .. of both halves of
// the tile's rows, columns 32 wn .. of both halves of its columns.  A step's four
// panels (two halves of A, two of B) have two buffers.  A wave goes through a step in
// four phases, each a quarter of its results:
//   1: reads A0, B0    products of A0, B0
//   2: reads B1        products of A0, B1
//   3: reads A1        products of A1, B1
//   4:                 products of A1, B0
// A phase reads, waits, meets the other waves at a barrier, multiplies, and meets
// them again.  Waves 4 .. 7 (the second wave of every SIMD) run one barrier behind,
// so that on each SIMD one wave multiplies while the other reads.  A panel that
// phase p has read is free in phase p + 1; phases 2, 3, 4 and the next 1 fill B0, A0,
// B1 and A1 with their values of two steps later (in this order all along).  Loads are
// waited for one phase before they are read, with those of the last five panels
// still under way.  Blocks stay and take every gridDim.x-th tile; the next tile's
// first loads are under way while this one's results are stored.
//
// Four waves of 128 x 128 would read a third less from LDS; with the pipeline of
// k_product (512 registers a lane) they took 8% longer in a step over 16,384 rows of
// 2,048 channels, 8,192 hidden.  What is left is the end of a tile, which nothing
// covers: 7 us of plain results, 12 with g and u stored, 27 of dG and dU (512 KB a
// tile), beside 1.4 to 1.6 us a step.
template <bool AK, bool BK, int EPI>
__global__ __launch_bounds__(512) void k_product_large(Work w) {
    typedef uint16_t T;
    constexpr int BM = 256, BN = 256;
    constexpr bool kGate = EPI == kGated, kTwo = EPI == kPlain && AK && !BK;  // kTwo: two segments
    typedef Panel<T, AK, 128> PA;
    typedef Panel<T, BK, 128> PB;
    constexpr int kStep = PA::kStep;
    constexpr uint32_t kPanel = 128 * 128, kStage = 4 * kPanel;
    constexpr uint32_t kA0 = 0, kA1 = kPanel, kB0 = 2 * kPanel, kB1 = 3 * kPanel;
    __shared__ __attribute__((aligned(1024))) char lds[2 * kStage];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 2, wn = wave & 3;
    const uint32_t base = lds_offset(lds), part = uint32_t(wave) * 1024u;
    typename PA::template Feed<512> fa[2];
    typename PB::template Feed<512> fb[2];
    static_assert(fa[0].kLoads == 2 && fb[0].kLoads == 2, "the waits count two loads a panel");
    Steps walk;
    int switch_in = 0, k = 0;  // steps before the second segment; values of the step that is loaded
    Spot tile = {};
    Product p = w.p[0];
    int m0 = 0, n0 = 0, steps = 0, count = 0;  // of the tile; steps of a segment, and of the slice
    // The four loads of a step, in this order; past the slice's end nothing is
    // fetched and zeros are stored, so that the number of loads stays the same.
    auto load_a = [&](int h, uint32_t to) {
        const u32x4_t r = fa[h].next(k);
        fa[h].load(0, r, k, to + (h ? kA1 : kA0) + part);
        fa[h].load(1, r, k, to + (h ? kA1 : kA0) + part);
    };
    auto load_b = [&](int h, uint32_t to) {
        if (h == 0) {
            if (kTwo && switch_in-- == 0) {
                // the segments' rows are equally far apart: only the bases differ
                const uint64_t da = p.a[1] - p.a[0] - steps * int64_t(fa[0].ahead);
                const uint64_t db = p.b[1] - p.b[0] - steps * int64_t(fb[0].ahead);
                fa[0].at += da, fa[1].at += da, fb[0].at += db, fb[1].at += db;
                walk.left = p.k;
            }
            k = walk.next<kStep>();
        }
        const u32x4_t r = fb[h].next(k);
        fb[h].load(0, r, k, to + (h ? kB1 : kB0) + part);
        fb[h].load(1, r, k, to + (h ? kB1 : kB0) + part);
    };
    typename PA::template Lanes<4> la;
    typename PB::template Lanes<2> lb;
    la.init(lane, base, wm * 64);
    lb.init(lane, base, wn * 32);
    f32x4_t acc[2][4][2][2] = {};
    u32x4_t a[4][2], b0[2][2], b1[2][2];
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
    // All but the last five panels have landed; stores: after those of the stores
    // that a tile's end issued, at least kStores where they went ahead of none of
    // the panels waited for.  (Memory instructions are counted in their order: a wait
    // for ten would be one for the stores, which take as long as a step.)
    constexpr int kStores = kGate ? 8 : kPlain == EPI ? 16 : 32;
    auto landed = [&](bool stores) {
        if (!stores) asm volatile("s_waitcnt vmcnt(10)" ::: "memory");
        else if (kGate && w.gate) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(10 + 3 * 8) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(10 + kStores) : "memory");
    };
    // the phase's reads have returned, and the next phase's panel has landed
    auto meet_read = [&](bool stores = false) {
        landed(stores);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
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
                for (int j = 0; j < 2; ++j) c[i][h][j] = mma(T(), 0, b[j][s], a[i][s], c[i][h][j]);
    };

    for (uint32_t id = blockIdx.x;; id += gridDim.x) {
        // All waves are done with the buffers: the next tile's first loads go ahead
        // of the stores of the one before.
        const Product before = p;
        const bool whole = m0 + BM <= p.m && n0 + (kGate ? BN / 2 : BN) <= p.n;
        const int slice = tile.slice, row = m0 + wm * 64 + (lane & 15);
        const int col = n0 + wn * 32 + 16 * ((lane >> 4) & 1) + (lane >> 5) * 8;
        tile = spot(w, id);
        if (tile.which >= 0) {
            p = pick(w, tile.which);
            m0 = tile.tile_m * BM, n0 = tile.tile_n * (kGate ? BN / 2 : BN);
            steps = (p.k + kStep - 1) / kStep;
            const int first = tile.slice * w.per_slice;
            const int segment = kTwo && first >= steps, step = first - segment * steps;
            count = min(w.per_slice, steps * (kTwo ? 2 : 1) - first);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int am = m0 + h * 128, an = n0 + (kGate ? 0 : h * 128), from = kGate ? h : segment;
                fa[h].init(threadIdx.x, segment ? p.a[1] : p.a[0], p.a_row, am, p.m - am, step);
                fb[h].init(threadIdx.x, from ? p.b[1] : p.b[0], from ? p.b_row[1] : p.b_row[0], an, p.n - an, step);
            }
            walk = {p.k - step * kStep, count};
            if (kTwo) switch_in = segment ? -1 : steps - first;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                load_b(0, base + t * kStage);
                load_a(0, base + t * kStage);
                load_b(1, base + t * kStage);
                if (t == 0) load_a(1, base);
            }
        }
        if (id != blockIdx.x) {
            constexpr int kHalves = kGate ? 1 : 2;
            finish<T, EPI, 8 * kHalves>(
                w, before, slice,
                [&](int u) -> Place {
                    return {row + u / kHalves / 4 * 128 + 16 * (u / kHalves % 4), col + u % kHalves * 128};
                },
                [&](int u, float *c, float *d) {
                    const f32x4_t(&r)[2][2] = acc[u / kHalves / 4][u / kHalves % 4];
                    pair_up(r[u % kHalves][0], r[u % kHalves][1], c);
                    if (kGate) pair_up(r[1][0], r[1][1], d);
                });
        }
        if (tile.which < 0) break;
        const bool stores = id != blockIdx.x && whole;
        landed(stores);
        __builtin_amdgcn_s_barrier();
        if (wave >= 4) __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[i / 16][i / 4 % 4][i / 2 % 2][i % 2] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        uint32_t at = 0;
        for (int step = 0; step < count; ++step) {
            const uint32_t to = base + at;
            read_a(at + kA0);
            read_b(b0, at + kB0);
            load_a(1, base + (kStage - at));
            meet_read(stores && step == 0);
            multiply(acc[0], 0, b0);
            meet();
            read_b(b1, at + kB1);
            load_b(0, to);
            meet_read(stores && step == 0);
            multiply(acc[0], 1, b1);
            meet();
            read_a(at + kA1);
            load_a(0, to);
            meet_read(stores && step == 0);
            multiply(acc[1], 1, b1);
            meet();
            load_b(1, to);
            meet_read(stores && step == 0);
            multiply(acc[1], 0, b0);
            meet();
            at = kStage - at;
        }
        if (wave < 4) __builtin_amdgcn_s_barrier();
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's loads of zeros past the last step
    }
}

// Up to 16 rows: the weights are what is read, once, straight into registers.  A
// block has COLS (8 or 16) columns of the result; its eight waves share the
// contracted axis in turns of 128 bytes, kTurns of them under way at a time, and
// their sums are added up through LDS in the waves' order.  One row of 384 channels,
// 1,536 hidden: 4 + 4 us, most of it the launch; as tiles 5 + 8.  Of 4,096 channels,
// 12,288 hidden: 59 us, 5.2 TB/s; 16 rows, whose x and h every block reads, 85.
template <typename T, int EPI, int COLS>
__global__ __launch_bounds__(512) void k_few(Work w) {
    constexpr int kMats = EPI == kGated ? 2 : 1, kTurns = 4, kWaves = 8, kPer = 16 / int(sizeof(T)), kTurn = 128 / int(sizeof(T));
    __shared__ f32x4_t sums[kWaves][kMats][64];
    const Product &p = w.p[0];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, fk = lane >> 4;
    const int n0 = int(blockIdx.x) * COLS;
    // rows and columns past the end are read from the last one and not stored
    const T *x = reinterpret_cast<const T *>(p.a[0] + int64_t(min(fr, p.m - 1)) * p.a_row) + fk * kPer;
    const T *m[kMats];
#pragma unroll
    for (int i = 0; i < kMats; ++i)
        m[i] = reinterpret_cast<const T *>(p.b[i] + int64_t(min(n0 + fr % COLS, p.n - 1)) * p.b_row[i]) + fk * kPer;
    f32x4_t acc[kMats] = {};
    for (int k0 = wave * kTurn; k0 < p.k; k0 += kWaves * kTurns * kTurn) {
        u32x4_t a[kTurns][2] = {}, b[kTurns][2][kMats] = {};
#pragma unroll
        for (int t = 0; t < kTurns; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int k = k0 + t * kWaves * kTurn + s * (kTurn / 2);
                if (k + fk * kPer < p.k) {
                    a[t][s] = *reinterpret_cast<const u32x4_t *>(x + k);
#pragma unroll
                    for (int i = 0; i < kMats; ++i) b[t][s][i] = *reinterpret_cast<const u32x4_t *>(m[i] + k);
                }
            }
#pragma unroll
        for (int t = 0; t < kTurns; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < kMmaSteps<T>; ++e)
#pragma unroll
                    for (int i = 0; i < kMats; ++i) acc[i] = mma(T(), e, b[t][s][i], a[t][s], acc[i]);
    }
#pragma unroll
    for (int i = 0; i < kMats; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int i = 0; i < kMats; ++i)
#pragma unroll
        for (int v = 1; v < kWaves; ++v) acc[i] += sums[v][i][lane];
    // four neighbouring columns of row fr
    const int n = n0 + 4 * fk;
    if (fr >= p.m || 4 * fk >= COLS || n >= p.n) return;
    if constexpr (EPI == kGated) {
        f32x4_t h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = (w.gelu ? activation<true>(acc[0][e], nullptr) : activation<false>(acc[0][e], nullptr)) * acc[1][e];
        const int64_t to = fr * w.hidden_s + n;
        store4(static_cast<T *>(w.act) + to, h);
        if (w.gate) {
            store4(static_cast<T *>(w.gate) + to, acc[0]);
            store4(static_cast<T *>(w.up) + to, acc[1]);
        }
    } else {
        store4(static_cast<T *>(p.c) + fr * p.c_row + n, acc[0]);
    }
}

// Adds up the slices in their order and rounds.
template <typename T>
__global__ __launch_bounds__(256) void k_join_slices(Work w) {
    for (int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 8; i < w.slice_size; i += int64_t(gridDim.x) * 2048) {
        int which = 0;
        while (which + 1 < w.products && i >= w.p[which + 1].partial) ++which;
        const Product &p = w.p[which];
        float sum[8] = {};
        for (int s = 0; s < w.slices; ++s) {
            Eight<float> more;
            more.load(w.partial + s * w.slice_size + i);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += more[e];
        }
        const int64_t at = i - p.partial, m = at / p.n;
        store8(static_cast<T *>(p.c) + m * p.c_row + (at - m * p.n), sum);
    }
}

// -------------------------------------------------------------------- launches

// Fills in the tiles of w's products; the number of blocks.
int64_t cut(Work &w, const Plan &plan, Epilogue epi, float *partial) {
    int64_t tiles = 0;
    w.slices = plan.slices;
    w.per_slice = plan.per_slice;
    w.partial = partial;
    w.slice_size = 0;
    for (int i = 0; i < w.products; ++i) {
        Product &p = w.p[i];
        p.tiles_m = int(ceil_div(p.m, kSizeOf[plan.kind]));
        p.tiles_n = int(ceil_div(p.n, cols_of(plan.kind, epi)));
        p.tiles = p.tiles_m * p.tiles_n;
        p.partial = w.slice_size;
        w.slice_size += int64_t(p.m) * p.n;
        tiles += p.tiles;
    }
    return tiles * plan.slices;
}

template <typename T>
hipError_t join(const Work &w, hipStream_t s) {
    if (w.slices == 1) return hipSuccess;
    k_join_slices<T><<<int(std::min<int64_t>((w.slice_size + 2047) / 2048, 8 * compute_units())), 256, 0, s>>>(w);
    return hipGetLastError();
}

template <typename T, bool AK, bool BK, int EPI>
hipError_t launch(Work &w, const Plan &plan, float *partial, hipStream_t s) {
    const int64_t blocks = cut(w, plan, Epilogue(EPI), partial);
    const Fold f = fold(blocks, 256);
    const dim3 grid(f.x, 1, f.z);
    switch (plan.kind) {
        case kTiles256:
            if constexpr (sizeof(T) == 2)
                k_product_large<AK, BK, EPI><<<int(std::min<int64_t>(blocks, compute_units())), 512, 0, s>>>(w);
            break;
        case kTiles128: k_product<T, AK, BK, EPI, 128, 2><<<grid, 256, 0, s>>>(w); break;
        case kTiles64: k_product<T, AK, BK, EPI, 64, 2><<<grid, 256, 0, s>>>(w); break;
        case kTiles64Deep: k_product<T, AK, BK, EPI, 64, 4><<<grid, 256, 0, s>>>(w); break;
    }
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : join<T>(w, s);
}

// x and w in one launch, of one kind of tiles (not the largest).
template <typename T>
hipError_t launch_both(Work &x, const Plan &px, float *partial_x, Work &w, const Plan &pw, float *partial_w, hipStream_t s) {
    const int64_t blocks_x = cut(x, px, kPlain, partial_x), blocks_w = cut(w, pw, kPlain, partial_w);
    const bool x_first = px.per_slice >= pw.per_slice;
    const uint32_t first = uint32_t(x_first ? blocks_x : blocks_w);
    const Fold f = fold(blocks_x + blocks_w, 256);
    const dim3 grid(f.x, 1, f.z);
    switch (px.kind) {
        case kTiles128: k_products<T, 128, 2><<<grid, 256, 0, s>>>(x, w, first, x_first); break;
        case kTiles64: k_products<T, 64, 2><<<grid, 256, 0, s>>>(x, w, first, x_first); break;
        default: k_products<T, 64, 4><<<grid, 256, 0, s>>>(x, w, first, x_first); break;
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = join<T>(x, s);
    return e != hipSuccess ? e : join<T>(w, s);
}

// Eight columns a block where sixteen would leave CUs without one.
template <typename T, int EPI>
hipError_t launch_few(const Work &w, hipStream_t s) {
    const int n = w.p[0].n;
    if (ceil_div(n, 16) < compute_units()) k_few<T, EPI, 8><<<int(ceil_div(n, 8)), 512, 0, s>>>(w);
    else k_few<T, EPI, 16><<<int(ceil_div(n, 16)), 512, 0, s>>>(w);
    return hipGetLastError();
}

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

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
    w.products = 1;
    w.gelu = a.gelu;
    w.gate = a.gate, w.up = a.up, w.act = a.act, w.hidden_s = a.hidden_s;
    Product &p = w.p[0];
    p.a[0] = static_cast<const char *>(a.x);
    p.b[0] = static_cast<const char *>(a.w_gate), p.b[1] = static_cast<const char *>(a.w_up);
    p.a_row = uint32_t(a.x_s * sizeof(T));
    p.b_row[0] = uint32_t(a.w_gate_s * sizeof(T)), p.b_row[1] = uint32_t(a.w_up_s * sizeof(T));
    p.m = a.rows, p.n = a.hidden, p.k = a.channels;
    const bool few = a.rows <= kFewRows;
    hipError_t e = few ? launch_few<T, kGated>(w, s) : launch<T, true, true, kGated>(w, plan_gated(a, compute_units()), nullptr, s);
    if (e != hipSuccess) return e;
    p = Product{};
    p.a[0] = static_cast<const char *>(a.act);
    p.b[0] = static_cast<const char *>(a.w_down);
    p.a_row = uint32_t(a.hidden_s * sizeof(T)), p.b_row[0] = uint32_t(a.w_down_s * sizeof(T));
    p.m = a.rows, p.n = a.channels, p.k = a.hidden;
    p.c = a.out, p.c_row = a.out_s;
    return few ? launch_few<T, kPlain>(w, s)
               : launch<T, true, true, kPlain>(w, plan_down(a, compute_units()), reinterpret_cast<float *>(space), s);
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
        w.products = 1;
        w.gelu = a.gelu;
        w.gate = a.gate, w.up = a.up, w.hidden_s = a.hidden_s;
        Product &p = w.p[0];
        p.a[0] = static_cast<const char *>(a.dout), p.b[0] = static_cast<const char *>(a.w_down);
        p.a_row = dout_row, p.b_row[0] = uint32_t(a.w_down_s * sizeof(T));
        p.m = a.rows, p.n = a.hidden, p.k = a.channels;
        p.c = dgate;
        if ((e = launch<T, true, false, kGatedGrad>(w, plan_dhidden(a, compute_units()), nullptr, s)) != hipSuccess) return e;
    }
    const Backward plans = plan_backward(a, compute_units());
    Work x{}, w{};
    if (a.rows > 0 && a.dx) {
        x.products = 1;
        Product &p = x.p[0];
        p.a[0] = dgate, p.a[1] = dup;
        p.b[0] = static_cast<const char *>(a.w_gate), p.b[1] = static_cast<const char *>(a.w_up);
        p.a_row = hidden_row;
        p.b_row[0] = uint32_t(a.w_gate_s * sizeof(T)), p.b_row[1] = uint32_t(a.w_up_s * sizeof(T));
        p.m = a.rows, p.n = a.channels, p.k = a.hidden;
        p.c = a.dx, p.c_row = a.dx_s;
    }
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
    if (plans.both)
        return launch_both<T>(x, plans.x, partial, w, plans.w, partial + plans.x.partial / sizeof(float), s);
    if (x.products && (e = launch<T, true, false, kPlain>(x, plans.x, partial, s)) != hipSuccess) return e;
    return w.products ? launch<T, false, false, kPlain>(w, plans.w, partial, s) : hipSuccess;
}

// Tensors of a call that may not share memory.
struct Named {
    const char *name;
    Extent e;
};
// First of `some` and `others` that do.
std::string together(std::initializer_list<Named> some, std::initializer_list<Named> others) {
    for (const Named &s : some)
        for (const Named &o : others)
            if (overlap(s.e, o.e)) return std::string(s.name) + " overlaps " + o.name;
    return {};
}

}  // namespace

// The first product reads x, w_gate and w_up and writes gate, up and act; the second
// reads act and w_down and writes out.  So out may lie where x is.
std::string gated_ffn_overlap(const FfnArgs &a) {
    const int64_t n = a.rows, c = a.channels, f = a.hidden, el = a.bf16 ? 2 : 4;
    const Named x{"x", extent(a.x, n, a.x_s, c, el)}, out{"out", extent(a.out, n, a.out_s, c, el)};
    const Named wg{"w_gate", extent(a.w_gate, n ? f : 0, a.w_gate_s, c, el)}, wu{"w_up", extent(a.w_up, n ? f : 0, a.w_up_s, c, el)};
    const Named wd{"w_down", extent(a.w_down, n ? c : 0, a.w_down_s, f, el)};
    const Named g{"gate", extent(a.gate, n, a.hidden_s, f, el)}, u{"up", extent(a.up, n, a.hidden_s, f, el)};
    const Named h{"act", extent(a.act, n, a.hidden_s, f, el)};
    std::string why = together({g, u, h}, {x, wg, wu, wd, out});
    if (why.empty()) why = together({g}, {u, h});
    if (why.empty()) why = together({u}, {h});
    return why.empty() ? together({out}, {wd}) : why;
}

// dX reads w_gate and w_up, the weights' gradients x, dout and act, in one launch or
// in two in either order.
std::string gated_ffn_grad_overlap(const FfnArgs &a) {
    const int64_t n = a.rows, c = a.channels, f = a.hidden, el = a.bf16 ? 2 : 4;
    const bool of_x = a.dw_gate || a.dw_up, of_act = a.dw_down, of_weights = a.dx && n;
    const Named dx{"dx", extent(a.dx, n, a.dx_s, c, el)}, dg{"dw_gate", extent(a.dw_gate, f, a.dw_gate_s, c, el)};
    const Named du{"dw_up", extent(a.dw_up, f, a.dw_up_s, c, el)}, dd{"dw_down", extent(a.dw_down, c, a.dw_down_s, f, el)};
    const Named x{"x", extent(a.x, of_x ? n : 0, a.x_s, c, el)}, dout{"dout", extent(a.dout, of_act ? n : 0, a.dout_s, c, el)};
    const Named h{"act", extent(a.act, of_act ? n : 0, a.hidden_s, f, el)};
    const Named wg{"w_gate", extent(a.w_gate, of_weights ? f : 0, a.w_gate_s, c, el)};
    const Named wu{"w_up", extent(a.w_up, of_weights ? f : 0, a.w_up_s, c, el)};
    std::string why = together({dx, dg, du, dd}, {x, dout, h, wg, wu});
    if (why.empty()) why = together({dx}, {dg, du, dd});
    if (why.empty()) why = together({dg}, {du, dd});
    return why.empty() ? together({du}, {dd}) : why;
}

size_t gated_ffn_workspace(const FfnArgs &a) {
    if (a.rows == 0) return 0;
    return (a.act ? 0 : round16(hidden_bytes(a))) + (a.rows <= kFewRows ? 0 : plan_down(a, compute_units()).partial);
}

int gated_ffn(const FfnArgs &a, void *stream) {
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.bf16 ? forward<uint16_t>(a, s) : forward<float>(a, s);
}

size_t gated_ffn_grad_workspace(const FfnArgs &a) {
    const size_t hidden = wants_hidden(a) ? round16(2 * hidden_bytes(a)) : 0;
    return hidden + plan_backward(a, compute_units()).partial;
}

int gated_ffn_grad(const FfnArgs &a, void *stream) {
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.bf16 ? gradient<uint16_t>(a, s) : gradient<float>(a, s);
}

}  // namespace kern
}  // namespace rtcc
