// Gradients of attention on gfx950.
//
//   P = exp(x - lse) of the visible pairs, dV = P^T dO, dP = dO V^T,
//   delta = sum(dO o), dS = P (dP - delta) (1 - tanh^2 with a cap),
//   dQ = scale dS K,  dK = scale dS^T Q
//
// Two kernels that each own what they write, so nothing is added atomically
// and every sum has one order; both compute x and P again from lse.
//   dq:  the columns of the forward pass (attention.hip), 32 a wave; K and V
//     tiles in LDS, scores K Q^T and V dO^T, dQ accumulated as K^T dS^T, with
//     delta from the rows of dO and o it holds.  For a row that sees at most 32
//     keys lse and delta come from its weights themselves, as o's rounding to
//     bf16 (2^-8) would be large beside the few terms whose differences dS is (a
//     row of one key has dS = 0).  It also writes each row's lse and delta for
//     dkv, and by then the sum of P (dP - delta) has what delta was short of: dK
//     does not see o's rounding.  dQ does, where few keys have most of the
//     weight or the values have a large common part: 0.29% off 64-bit values,
//     dK 0.24%, four capped, biased histories.  Taking it out needs sum P K
//     beside dS K: 0.24%, forward and gradients 10% (heads of 64) and 15% (128)
//     slower.  dS as the sum of two bf16 operands: 0.23%, 6% and 37% slower.
//   dkv: 32 keys a wave, K and V rows in registers; the queries of the group's
//     heads pass through LDS, head by head, scores Q K^T and dO V^T, with the
//     keys as columns; dV and dK are accumulated as dO^T P and Q^T dS.  The
//     sum over the heads of a group is the order of the walk.
// Forward and gradients, bf16: four causal, capped, biased histories of up to
// 4,096 tokens, 6 heads of 64: 409 us, of these dq 129 us, dkv 170 us, with the
// matrix cores busy 18% of the time and vector work the rest.  dkv spills 21 to
// 45 registers at heads of 64.
#include <algorithm>
#include <type_traits>

#include "attention.hpp"
#include "compute_units.hpp"

namespace rtcc {
namespace kern {

namespace {

// S waves of a block (2 or 4) share their columns (dq) or keys (dkv) and take a
// 32-row part each of every tile along the long axis; the others are side by
// side.
template <int S>
constexpr int kRows = 32 * S;
constexpr int kSide = 128;  // columns or keys of a block if its waves shared none

// Two waves a SIMD, for dkv of wide heads and float32 one: they need up to all
// 512 registers.  dq of bf16 heads of 128 spills 60 to 90 registers at two and is
// faster all the same: forward and gradients of 2 x 8,192 causal tokens, 6 heads,
// 1,426 us, at one wave 1,525 us.
template <typename T, int D>
constexpr int kWavesDq = sizeof(T) == 2 ? 2 : 1;
template <typename T, int D>
constexpr int kWavesDkv = sizeof(T) == 2 && D <= 64 ? 2 : 1;

// lse in units of log 2; a row without visible keys gets weights of zero.
__device__ inline float base_of(float lse) { return lse == -kInf ? kInf : lse * kLog2e; }

// Adds up the S waves' sums in the first of them, through LDS.
template <int D, int S>
__device__ inline void gather(f32x16_t *acc, float *lds, int group, int turn, int lane) {
    if constexpr (S > 1) {
        constexpr int kStride = D + 4;
        float *mine = lds + (group * (S - 1) * 32 + (lane & 31)) * kStride + 4 * (lane >> 5);
        __syncthreads();
        if (turn > 0) {
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<float4 *>(mine + (turn - 1) * 32 * kStride + 32 * t + 8 * g) =
                        make_float4(acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]);
        }
        __syncthreads();
        if (turn == 0) {
#pragma unroll
            for (int w = 0; w < S - 1; ++w)
#pragma unroll
                for (int t = 0; t < D / 32; ++t)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float4 x = *reinterpret_cast<const float4 *>(mine + w * 32 * kStride + 32 * t + 8 * g);
                        acc[t][4 * g] += x.x;
                        acc[t][4 * g + 1] += x.y;
                        acc[t][4 * g + 2] += x.z;
                        acc[t][4 * g + 3] += x.w;
                    }
        }
    }
}

template <typename T, int D, Cap CAP, bool BIAS, int S>
__global__ __launch_bounds__(256, (kWavesDq<T, D>)) void k_dq(AttnArgs a, float *stats) {
    typedef Op<T> M;
    typedef Tile<T, D> L;
    constexpr int N = kRows<S>, kColumns = kSide / S;
    constexpr uint32_t kBytes = N * L::kRowBytes, kPart = 32 * L::kRowBytes;
    extern __shared__ __align__(1024) unsigned char lds[];
    Seq sq;
    if (!find_tile<false>(a, tile_of(a), kColumns, sq)) return;
    const int kvh = head_of(a), wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
    const int group = wave / S, turn = wave % S;
    const int64_t columns = int64_t(sq.nq) * a.group;
    const int mine = a.causal ? int((columns + kColumns - 1) / kColumns) - 1 - sq.tile : sq.tile;
    const int64_t c0 = int64_t(mine) * kColumns;
    Column at;
    at.init(a, sq, kvh, c0 + group * 32);
    const int limit = limit_of(a, sq, at.i);
    const int first_limit = __builtin_amdgcn_readlane(limit, 0), last_limit = __builtin_amdgcn_readlane(limit, 31);
    const int keys = limit_of(a, sq, int((min(c0 + kColumns, columns) - 1) / a.group));

    typename M::Frag q[D / 16], g[D / 16];
    load_row<T, D>(static_cast<const T *>(a.q) + at.row * a.q_s[0] + at.head * a.q_s[1], a.dim, h, q);
    load_row<T, D>(static_cast<const T *>(a.dout) + at.row * a.do_s[0] + at.head * a.do_s[1], a.dim, h, g);
    float delta = 0.f;
    {
        typename M::Frag o[D / 16];
        load_row<T, D>(static_cast<const T *>(a.out) + at.row * a.o_s[0] + at.head * a.o_s[1], a.dim, h, o);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf(M::widen(g[kk], e), M::widen(o[kk], e), delta);
    }
    delta = half_sum(delta);
    const int64_t stat = int64_t(at.head) * a.q_rows + at.row;
    float base = base_of(a.lse[stat]);
    const int place = sq.nk - sq.nq + at.i;
    const float slope = BIAS ? a.slopes[at.head] * kLog2e : 0.f;
    Score score;
    score.init(a);
    f32x16_t acc[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) acc[t] = f32x16_t{};
    float left_over = 0.f;  // sum P (dP - delta): what delta is short of
    wait_registers();

    const T *k = static_cast<const T *>(a.k) + sq.k0 * a.k_s[0] + kvh * a.k_s[1];
    const T *v = static_cast<const T *>(a.v) + sq.k0 * a.v_s[0] + kvh * a.v_s[1];
    Stager<T, D, N, 256> ks, vs;
    ks.init(threadIdx.x, a.k_s[0], a.dim);
    vs.init(threadIdx.x, a.v_s[0], a.dim);
    const uint32_t lds0 = lds_offset(lds), own = lds0 + turn * kPart;
    Lanes<T, D> from;
    from.init(lane, own);
    auto load = [&](int t, int buffer) __attribute__((always_inline)) {
        const uint32_t to = lds0 + buffer * 2 * kBytes;
        ks.load(k + int64_t(t) * N * a.k_s[0], keys - t * N, to, threadIdx.x);
        vs.load(v + int64_t(t) * N * a.v_s[0], keys - t * N, to + kBytes, threadIdx.x);
    };
    // P from a product, and the slope of the cap there
    auto weight_of = [&](float x, float away, int j, float &bend) __attribute__((always_inline)) {
        float y;
        if constexpr (CAP != kNone) {
            float th;
            y = score.capped<CAP>(x, th) - base;
            bend = fmaf(-th, th, 1.f);
        } else {
            y = fmaf(x, score.c1, -base);
        }
        if constexpr (BIAS) y = fmaf(-slope, fabsf(away - float(j)), y);
        return __builtin_amdgcn_exp2f(y);
    };
    // 32 keys from j0 on, some of them hidden from some columns; at: LDS address
    // of their part of the K tile
    auto part = [&](int j0, uint32_t at) __attribute__((always_inline)) {
        f32x16_t x = {}, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = 0.f;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) x = M::mma(from.row_frag(0, 0, kk), q[kk], x);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) dp = M::mma(from.row_frag(kBytes, 0, kk), g[kk], dp);
        const float away = float(place - j0 - 4 * h);
        const int left = limit - j0 - 4 * h;
        if (j0 == 0 && first_limit <= 32) {
            float p[16], top = -kInf, sum = 0.f, dot = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int j = 8 * (r >> 2) + (r & 3);
                float y = x[r] * score.c1, th;
                if constexpr (CAP != kNone) y = score.capped<CAP>(x[r], th);
                if constexpr (BIAS) y = fmaf(-slope, fabsf(away - float(j)), y);
                p[r] = j < left ? y : -kInf;
                top = fmaxf(top, p[r]);
            }
            top = half_max(top);
            const float low = top == -kInf ? 0.f : top;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += p[r] = __builtin_amdgcn_exp2f(p[r] - low);
            sum = half_sum(sum);
            const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + (r & 3) < left) dot = fmaf(p[r] * f, dp[r], dot);
            dot = half_sum(dot);
            if (limit <= 32) {
                base = sum == 0.f ? kInf : top + __builtin_amdgcn_logf(sum);
                delta = dot;
            }
        }
        float ds[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int j = 8 * (r >> 2) + (r & 3);
            float bend = 1.f;
            float d = weight_of(x[r], away, j, bend) * (dp[r] - delta);
            if (j >= left) d = 0.f;
            left_over += d;
            if constexpr (CAP != kNone) d *= bend;
            ds[r] = j >= left ? 0.f : d;
        }
        typename M::Frag w[2] = {M::pack(ds), M::pack(ds + 8)};
        Product<T, D, 2, true>::add(acc, w, at, lane, a.causal, [&](int j) { return j0 + j < limit; });
    };
    // 32 keys from j0 on that every column sees: the vector work beside the
    // products that do not wait for it, the reads ahead of both
    auto whole = [&](int j0) __attribute__((always_inline)) {
        constexpr int H = D / 16, W = D / 32, kAhead = sizeof(T) == 2 ? 4 : 1;
        typename M::Frag f[3 * H];
        auto read = [&](int i) __attribute__((always_inline)) {
            f[i] = i < 2 * H ? from.row_frag(i < H ? 0 : kBytes, 0, i % H) : from.col_frag(0, (i - 2 * H) / W, i % W);
        };
        f32x16_t x = {}, dp = {};
        float ds[16];
        typename M::Frag w0, w1;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read(i);
        const float away = float(place - j0 - 4 * h);
#pragma unroll
        for (int i = 0; i < 3 * H; ++i) {
            if (i < H) x = M::mma(f[i], q[i], x);
            else if (i < 2 * H) dp = M::mma(f[i], g[i - H], dp);
            else acc[i % W] = M::mma(f[i], i < 2 * H + W ? w0 : w1, acc[i % W]);
            if (i + kAhead < 3 * H) read(i + kAhead);
            if (i >= H && i < 2 * H) {
#pragma unroll
                for (int r = (i - H) * 16 / H; r < (i - H + 1) * 16 / H; ++r) {
                    float bend = 1.f;
                    ds[r] = weight_of(x[r], away, 8 * (r >> 2) + (r & 3), bend);
                    x[r] = bend;
                }
            }
            if (i == 2 * H - 1) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    ds[r] *= dp[r] - delta;
                    left_over += ds[r];
                    if constexpr (CAP != kNone) ds[r] *= x[r];
                }
                w0 = M::pack(ds);
                w1 = M::pack(ds + 8);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const int n = (keys + N - 1) / N;
    if (n > 0) load(0, 0);
    for (int t = 0; t < n; ++t) {
        wait_loads();
        barrier();
        if (t + 1 < n) load(t + 1, (t + 1) & 1);
        const int j0 = t * N + turn * 32;
        if (j0 + 32 <= first_limit && j0 > 0) whole(j0);
        else if (j0 < last_limit) part(j0, own + (t & 1) * 2 * kBytes);
        from.flip(2 * kBytes);
    }
    // the waves' parts of what delta is short of
    float *parts = reinterpret_cast<float *>(lds);
    left_over = half_sum(left_over);
    __syncthreads();
    if (h == 0) parts[wave * 32 + lane] = left_over;
    __syncthreads();
    if (turn == 0) {
#pragma unroll
        for (int w = 0; w < S; ++w) delta += parts[(wave + w) * 32 + (lane & 31)];
    }
    gather<D, S>(acc, reinterpret_cast<float *>(lds), group, turn, lane);
    if (!at.valid || turn > 0) return;
    if (h == 0) {
        stats[stat] = base;
        stats[int64_t(a.q_heads) * a.q_rows + stat] = delta;
    }
    store_column<T, D>(static_cast<T *>(a.dq) + at.row * a.dq_s[0] + at.head * a.dq_s[1], a.dim, h, acc, a.scale);
}

template <typename T, int D, Cap CAP, bool BIAS, int S>
__global__ __launch_bounds__(256, (kWavesDkv<T, D>)) void k_dkv(AttnArgs a, const float *row_stats) {
    typedef Op<T> M;
    typedef Tile<T, D> L;
    constexpr int N = kRows<S>, kKeys = kSide / S;
    constexpr uint32_t kBytes = N * L::kRowBytes, kPart = 32 * L::kRowBytes;
    extern __shared__ __align__(1024) unsigned char lds[];  // two of (Q tile, dO tile), then the rows' lse and delta
    Seq sq;
    if (!find_tile<true>(a, tile_of(a), kKeys, sq)) return;
    const int kvh = head_of(a), wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
    const int group = wave / S, turn = wave % S;
    const int j_block = sq.tile * kKeys, j_wave = j_block + group * 32, j = j_wave + (lane & 31);
    const int64_t key = sq.k0 + min(j, sq.nk - 1);  // the last key stands in for those past it
    typename M::Frag k[D / 16], v[D / 16];
    load_row<T, D>(static_cast<const T *>(a.k) + key * a.k_s[0] + kvh * a.k_s[1], a.dim, h, k);
    load_row<T, D>(static_cast<const T *>(a.v) + key * a.v_s[0] + kvh * a.v_s[1], a.dim, h, v);
    Score score;
    score.init(a);
    f32x16_t dk[D / 32], dv[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) dk[t] = dv[t] = f32x16_t{};
    wait_registers();

    // the queries that see the block's first key: from i0 on
    const int shift = sq.nk - sq.nq;
    int i0 = !a.causal || sq.prefix > j_block ? 0 : max(0, j_block - shift);
    i0 -= i0 % N;
    const int per_head = i0 < sq.nq ? (sq.nq - i0 + N - 1) / N : 0, n = per_head * a.group;
    Stager<T, D, N, 256> qs, gs;
    qs.init(threadIdx.x, a.q_s[0], a.dim);
    gs.init(threadIdx.x, a.do_s[0], a.dim);
    const uint32_t lds0 = lds_offset(lds), own = lds0 + turn * kPart;
    Lanes<T, D> from;
    from.init(lane, own);
    float *stats = reinterpret_cast<float *>(lds + 4 * kBytes);  // [2][lse, delta][N]
    float stat = 0.f;                                            // of the tile being loaded, threads 0 .. 2 N - 1
    int head = 0, qt = 0;                                        // of the tile being loaded
    auto load = [&](int buffer) __attribute__((always_inline)) {
        const int hq = kvh * a.group + head, i = i0 + qt * N;
        if (threadIdx.x < 2 * N) {
            const int row = i + int(threadIdx.x % N);
            const bool second = threadIdx.x >= N;
            stat = second ? 0.f : kInf;
            if (row < sq.nq) stat = row_stats[(int64_t(second ? a.q_heads : 0) + hq) * a.q_rows + sq.q0 + row];
        }
        const uint32_t to = lds0 + buffer * 2 * kBytes;
        const int64_t first = sq.q0 + i;
        qs.load(static_cast<const T *>(a.q) + first * a.q_s[0] + hq * a.q_s[1], sq.nq - i, to, threadIdx.x);
        gs.load(static_cast<const T *>(a.dout) + first * a.do_s[0] + hq * a.do_s[1], sq.nq - i, to + kBytes,
                threadIdx.x);
        if (++qt == per_head) qt = 0, ++head;
    };
    auto put = [&](int buffer) __attribute__((always_inline)) {
        if (threadIdx.x < 2 * N) stats[buffer * 2 * N + threadIdx.x] = stat;
    };
    if (n > 0) {
        load(0);
        put(0);
    }
    int now_head = 0, now_qt = 0;
    // lse and delta of the lane's 16 rows of a part
    auto stats_of = [&](const float *rows, float *base, float *delta) __attribute__((always_inline)) {
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
            const float *s = rows + 8 * g4 + 4 * h;
            const float4 s0 = *reinterpret_cast<const float4 *>(s), s1 = *reinterpret_cast<const float4 *>(s + N);
            base[4 * g4] = s0.x, base[4 * g4 + 1] = s0.y, base[4 * g4 + 2] = s0.z, base[4 * g4 + 3] = s0.w;
            delta[4 * g4] = s1.x, delta[4 * g4 + 1] = s1.y, delta[4 * g4 + 2] = s1.z, delta[4 * g4 + 3] = s1.w;
        }
    };
    // P from a product, and the slope of the cap there
    auto weight_of = [&](float x, float base, float away, int ir, float slope, float &bend)
        __attribute__((always_inline)) {
        float y;
        if constexpr (CAP != kNone) {
            float th;
            y = score.capped<CAP>(x, th) - base;
            bend = fmaf(-th, th, 1.f);
        } else {
            y = fmaf(x, score.c1, -base);
        }
        if constexpr (BIAS) y = fmaf(-slope, fabsf(away + float(ir)), y);
        return __builtin_amdgcn_exp2f(y);
    };
    // 32 queries from i on, some keys hidden from some of them; at: LDS address
    // of their part of the Q tile
    auto part = [&](int i, uint32_t at, const float *rows, float slope) __attribute__((always_inline)) {
        f32x16_t x = {}, dp = {};
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) x = M::mma(from.row_frag(0, 0, kk), k[kk], x);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) dp = M::mma(from.row_frag(kBytes, 0, kk), v[kk], dp);
        float base[16], delta[16];
        stats_of(rows, base, delta);
        const float away = float(shift + i - j + 4 * h);
        // key j is hidden from the tile's queries before `hidden`
        const int hidden = j < sq.prefix || !a.causal ? 0 : j - shift - i, seen_from = hidden - 4 * h;
        float p[16], ds[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int ir = 8 * (r >> 2) + (r & 3);
            float bend = 1.f;
            p[r] = weight_of(x[r], base[r], away, ir, slope, bend);
            float d = p[r] * (dp[r] - delta[r]);
            if constexpr (CAP != kNone) d *= bend;
            if (ir < seen_from) p[r] = d = 0.f;
            ds[r] = d;
        }
        auto seen = [&](int r) __attribute__((always_inline)) { return r >= hidden; };
        typename M::Frag w[2] = {M::pack(p), M::pack(p + 8)}, u[2] = {M::pack(ds), M::pack(ds + 8)};
        Product<T, D, 2, true>::add(dv, w, at + kBytes, lane, a.causal, seen);
        Product<T, D, 2, true>::add(dk, u, at, lane, a.causal, seen);
    };
    // 32 queries from i on that see all of the wave's keys: the vector work
    // beside the products that do not wait for it, the reads ahead of both
    auto whole = [&](int i0, const float *rows, float slope) __attribute__((always_inline)) {
        constexpr int H = D / 16, W = D / 32, kAhead = sizeof(T) == 2 ? 4 : 1;
        typename M::Frag f[4 * H], w[2];
        auto read = [&](int i) __attribute__((always_inline)) {
            const int c = i % H;
            f[i] = i < 2 * H ? from.row_frag(i < H ? 0 : kBytes, 0, c) : from.col_frag(i < 3 * H ? kBytes : 0, c / W, c % W);
        };
        f32x16_t x = {}, dp = {};
        float base[16], delta[16], p[16];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read(i);
        stats_of(rows, base, delta);
        const float away = float(shift + i0 - j + 4 * h);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4 * H; ++i) {
            const int c = i % H;
            if (i < H) x = M::mma(f[i], k[c], x);
            else if (i < 2 * H) dp = M::mma(f[i], v[c], dp);
            else if (i < 3 * H) dv[c % W] = M::mma(f[i], w[c / W], dv[c % W]);
            else dk[c % W] = M::mma(f[i], w[c / W], dk[c % W]);
            if (i + kAhead < 4 * H) read(i + kAhead);
#pragma unroll
            for (int r = c * 16 / H; r < (c + 1) * 16 / H; ++r) {
                if (i >= H && i < 2 * H) {
                    float bend = 1.f;
                    p[r] = weight_of(x[r], base[r], away, 8 * (r >> 2) + (r & 3), slope, bend);
                    if constexpr (CAP != kNone) x[r] = bend * p[r];
                    else x[r] = p[r];
                } else if (i >= 2 * H && i < 3 * H) {
                    x[r] *= dp[r] - delta[r];
                }
            }
            if (i == 2 * H - 1) {
                w[0] = M::pack(p);
                w[1] = M::pack(p + 8);
            } else if (i == 3 * H - 1) {
#pragma unroll
                for (int r = 0; r < 16; ++r) p[r] = x[r];
                w[0] = M::pack(p);
                w[1] = M::pack(p + 8);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int u = 0; u < n; ++u) {
        const int buffer = u & 1;
        wait_loads();
        barrier();
        if (u + 1 < n) load(buffer ^ 1);
        const float slope = BIAS ? a.slopes[kvh * a.group + now_head] * kLog2e : 0.f;
        const int row = turn * 32, i = i0 + now_qt * N + row;  // first query of the wave's part
        if (i < sq.nq) {
            const float *s = stats + buffer * 2 * N + row;
            if (j_wave + 32 <= limit_of(a, sq, i)) whole(i, s, slope);
            else if (j_wave < limit_of(a, sq, min(i + 31, sq.nq - 1))) part(i, own + buffer * 2 * kBytes, s, slope);
        }
        from.flip(2 * kBytes);
        if (++now_qt == per_head) now_qt = 0, ++now_head;
        if (u + 1 < n) put(buffer ^ 1);
    }
    gather<D, S>(dk, reinterpret_cast<float *>(lds), group, turn, lane);
    gather<D, S>(dv, reinterpret_cast<float *>(lds), group, turn, lane);
    if (j < sq.nk && turn == 0) {
        store_column<T, D>(static_cast<T *>(a.dk) + key * a.dk_s[0] + kvh * a.dk_s[1], a.dim, h, dk, a.scale);
        store_column<T, D>(static_cast<T *>(a.dv) + key * a.dv_s[0] + kvh * a.dv_s[1], a.dim, h, dv, 1.f);
    }
}

// Bytes of LDS: two of both tiles and their rows' two numbers, and what gather
// needs.
template <typename T, int D, int S>
constexpr int kLds = std::max(4 * kRows<S> * Tile<T, D>::kRowBytes + 4 * kRows<S> * 4,
                              (4 / S) * (S - 1) * 32 * (D + 4) * 4);

template <typename T, int D, Cap CAP, bool BIAS, int S>
hipError_t run_dq(const AttnArgs &a, hipStream_t s) {
    const Fold f = fold(column_blocks(a, kSide / S), 256);
    const hipError_t e = max_lds(k_dq<T, D, CAP, BIAS, S>, kLds<T, D, S>);
    if (e != hipSuccess) return e;
    k_dq<T, D, CAP, BIAS, S><<<dim3(f.x, 1, f.z), 256, kLds<T, D, S>, s>>>(a, static_cast<float *>(a.workspace));
    return hipGetLastError();
}
template <typename T, int D, Cap CAP, bool BIAS, int S>
hipError_t run_dkv(const AttnArgs &a, hipStream_t s) {
    const Fold f = fold(key_blocks(a, kSide / S), 256);
    const hipError_t e = max_lds(k_dkv<T, D, CAP, BIAS, S>, kLds<T, D, S>);
    if (e != hipSuccess) return e;
    k_dkv<T, D, CAP, BIAS, S><<<dim3(f.x, 1, f.z), 256, kLds<T, D, S>, s>>>(
        a, static_cast<const float *>(a.workspace));
    return hipGetLastError();
}

// workspace: lse in log 2 units and delta of every row, [2][q_heads][q_rows]
template <typename T, int D, Cap CAP, bool BIAS>
hipError_t run(const AttnArgs &a, hipStream_t s) {
    constexpr int kMost = sizeof(T) == 4 && D == 128 ? 2 : 4;  // as the LDS holds
    const int wanted = 4 * compute_units();
    auto two = [&](int64_t units) {
        return 2 * (units / kSide + a.n_seqs) * a.kv_heads >= wanted;
    };
    hipError_t e = hipSuccess;
    if (a.q_rows > 0)
        e = two(int64_t(a.q_rows) * a.group) ? run_dq<T, D, CAP, BIAS, 2>(a, s) : run_dq<T, D, CAP, BIAS, kMost>(a, s);
    if (e == hipSuccess && a.k_rows > 0)
        e = two(a.k_rows) ? run_dkv<T, D, CAP, BIAS, 2>(a, s) : run_dkv<T, D, CAP, BIAS, kMost>(a, s);
    return e;
}

template <typename T, int D>
hipError_t run(const AttnArgs &a, hipStream_t s) {
    return with_terms<T>(a, [&](auto cap, auto bias) { return run<T, D, cap.value, bias.value>(a, s); });
}

template <typename T>
hipError_t run(const AttnArgs &a, hipStream_t s) {
    switch (padded(a.dim)) {
        case 32: return run<T, 32>(a, s);
        case 64: return run<T, 64>(a, s);
        default: return run<T, 128>(a, s);
    }
}

}  // namespace

size_t attention_grad_workspace(const AttnArgs &a) {
    return a.n_seqs == 0 ? 0 : 2 * size_t(a.q_heads) * a.q_rows * sizeof(float);
}

int attention_grad(const AttnArgs &a, void *stream) {
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.bf16 ? run<uint16_t>(a, s) : run<float>(a, s);
}

}  // namespace kern
}  // namespace rtcc
