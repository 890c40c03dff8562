// Gradients of attention on gfx950.
//
//   P = exp(x - lse) of the visible pairs, dV = P^T dO, dP = dO V^T,
//   delta = sum(dO o), dS = P (dP - delta) (1 - tanh^2 with a cap),
//   dQ = scale dS K,  dK = scale dS^T Q
//
// Two kernels that each own what they write, so nothing is added atomically
// and every sum has one order; both compute x and P again from lse.
//   dq:  the columns of the forward pass (attention.hip), 32 a wave; K and V
//     tiles in LDS, scores K Q^T and V dO^T, dQ accumulated as K^T dS^T.  It
//     also writes each row's lse and delta for dkv: delta from the rows of dO
//     and o it holds; for a row that sees at most 32 keys both from its
//     weights themselves, as o's rounding to bf16 (2^-8) would be large beside
//     the few terms whose differences dS is (a row of one key has dS = 0).
//   dkv: 32 keys a wave, K and V rows in registers; the queries of the group's
//     heads pass through LDS, head by head, scores Q K^T and dO V^T, with the
//     keys as columns; dV and dK are accumulated as dO^T P and Q^T dS.  The
//     sum over the heads of a group is the order of the walk.
#include "attention.hpp"

namespace rtcc {
namespace kern {

namespace {

constexpr int kColumns = 128;  // of a block of dq
constexpr int kKeys = 128;     // of a block of dkv
constexpr int tile_rows(bool bf16) { return bf16 ? 64 : 32; }

// Two waves a SIMD where the registers of a wave allow it.
template <typename T, int D>
constexpr int kWavesDq = sizeof(T) == 2 ? 2 : 1;
template <typename T, int D>
constexpr int kWavesDkv = sizeof(T) == 2 && D <= 64 ? 2 : 1;

// lse in units of log 2; a row without visible keys gets weights of zero.
__device__ inline float base_of(float lse) { return lse == -kInf ? kInf : lse * kLog2e; }

template <typename T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, (kWavesDq<T, D>)) void k_dq(AttnArgs a, int tiles, float *stats) {
    typedef Op<T> M;
    typedef Tile<T, D> L;
    constexpr int N = tile_rows(sizeof(T) == 2);
    constexpr uint32_t kBytes = N * L::kRowBytes;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int id = spread(blockIdx.x, gridDim.x);
    Seq sq;
    if (!find_tile<false>(a, id % tiles, kColumns, sq)) return;
    const int kvh = id / tiles, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
    const int64_t columns = int64_t(sq.nq) * a.group;
    const int mine = a.causal ? int((columns + kColumns - 1) / kColumns) - 1 - sq.tile : sq.tile;
    const int64_t c0 = int64_t(mine) * kColumns;
    Column at;
    at.init(a, sq, kvh, c0 + wave * 32);
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
    const float place = float(sq.nk - sq.nq + at.i);
    const float slope = BIAS ? a.slopes[at.head] * kLog2e : 0.f;
    Score score;
    score.init(a);
    f32x16_t acc[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) acc[t] = f32x16_t{};

    const T *k = static_cast<const T *>(a.k) + sq.k0 * a.k_s[0] + kvh * a.k_s[1];
    const T *v = static_cast<const T *>(a.v) + sq.k0 * a.v_s[0] + kvh * a.v_s[1];
    Stager<T, D, N, 256> ks, vs;
    ks.init(threadIdx.x, a.k_s[0], a.dim);
    vs.init(threadIdx.x, a.v_s[0], a.dim);
    const uint32_t lds0 = lds_offset(lds);
    auto load = [&](int t, int buffer) {
        const uint32_t to = lds0 + buffer * 2 * kBytes;
        ks.load(k + int64_t(t) * N * a.k_s[0], keys - t * N, to, threadIdx.x);
        vs.load(v + int64_t(t) * N * a.v_s[0], keys - t * N, to + kBytes, threadIdx.x);
    };
    const int n = (keys + N - 1) / N;
    if (n > 0) load(0, 0);
    for (int t = 0; t < n; ++t) {
        wait_loads();
        barrier();
        if (t + 1 < n) load(t + 1, (t + 1) & 1);
        const uint32_t kt = lds0 + (t & 1) * 2 * kBytes, vt = kt + kBytes;
#pragma unroll
        for (int b = 0; b < N / 32; ++b) {
            const int j0 = t * N + b * 32;
            if (j0 >= last_limit) break;
            const uint32_t kb = kt + b * 32 * L::kRowBytes, vb = vt + b * 32 * L::kRowBytes;
            f32x16_t x = {}, dp = {};
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) x = M::mma(L::row_frag(kb, lane & 31, kk, h), q[kk], x);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) dp = M::mma(L::row_frag(vb, lane & 31, kk, h), g[kk], dp);
            const bool masked = j0 + 32 > first_limit;
            const float away = place - float(j0) - 4.f * h;
            const int left = limit - j0 - 4 * h;
            if (j0 == 0 && first_limit <= 32) {
                float p[16], top = -kInf, sum = 0.f, dot = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int j = 8 * (r >> 2) + (r & 3);
                    float y = CAP ? score.capl * score.tanh_of(x[r]) : x[r] * score.c1;
                    if constexpr (BIAS) y = fmaf(-slope, fabsf(away - float(j)), y);
                    p[r] = j < left ? y : -kInf;
                    top = fmaxf(top, p[r]);
                }
                top = half_max(top);
                const float from = top == -kInf ? 0.f : top;
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += p[r] = __builtin_amdgcn_exp2f(p[r] - from);
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
                float y, bend = 1.f;
                if constexpr (CAP) {
                    const float th = score.tanh_of(x[r]);
                    bend = fmaf(-th, th, 1.f);
                    y = fmaf(score.capl, th, -base);
                } else {
                    y = fmaf(x[r], score.c1, -base);
                }
                if constexpr (BIAS) y = fmaf(-slope, fabsf(away - float(j)), y);
                float d = __builtin_amdgcn_exp2f(y) * (dp[r] - delta);
                if constexpr (CAP) d *= bend;
                if (masked && j >= left) d = 0.f;
                ds[r] = d;
            }
            typename M::Frag w[2] = {M::pack(ds), M::pack(ds + 8)};
            Product<T, D, 2, true>::add(acc, w, kb, lane, masked && a.causal, [&](int j) { return j0 + j < limit; });
        }
    }
    if (!at.valid) return;
    if (h == 0) {
        stats[stat] = base;
        stats[int64_t(a.q_heads) * a.q_rows + stat] = delta;
    }
    store_column<T, D>(static_cast<T *>(a.dq) + at.row * a.dq_s[0] + at.head * a.dq_s[1], a.dim, h, acc, a.scale);
}

template <typename T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, (kWavesDkv<T, D>)) void k_dkv(AttnArgs a, int tiles, const float *row_stats) {
    typedef Op<T> M;
    typedef Tile<T, D> L;
    constexpr int N = tile_rows(sizeof(T) == 2);
    constexpr uint32_t kBytes = N * L::kRowBytes;
    extern __shared__ __align__(1024) unsigned char lds[];  // two of (Q tile, dO tile), then the rows' lse and delta
    const int id = spread(blockIdx.x, gridDim.x);
    Seq sq;
    if (!find_tile<true>(a, id % tiles, kKeys, sq)) return;
    const int kvh = id / tiles, wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
    const int j_block = sq.tile * kKeys, j_wave = j_block + wave * 32, j = j_wave + (lane & 31);
    const int64_t key = sq.k0 + min(j, sq.nk - 1);  // the last key stands in for those past it
    typename M::Frag k[D / 16], v[D / 16];
    load_row<T, D>(static_cast<const T *>(a.k) + key * a.k_s[0] + kvh * a.k_s[1], a.dim, h, k);
    load_row<T, D>(static_cast<const T *>(a.v) + key * a.v_s[0] + kvh * a.v_s[1], a.dim, h, v);
    Score score;
    score.init(a);
    f32x16_t dk[D / 32], dv[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) dk[t] = dv[t] = f32x16_t{};

    // the queries that see the block's first key: from i0 on
    const int shift = sq.nk - sq.nq;
    int i0 = !a.causal || sq.prefix > j_block ? 0 : max(0, j_block - shift);
    i0 -= i0 % N;
    const int per_head = i0 < sq.nq ? (sq.nq - i0 + N - 1) / N : 0, n = per_head * a.group;
    Stager<T, D, N, 256> qs, gs;
    qs.init(threadIdx.x, a.q_s[0], a.dim);
    gs.init(threadIdx.x, a.do_s[0], a.dim);
    const uint32_t lds0 = lds_offset(lds);
    float *stats = reinterpret_cast<float *>(lds + 4 * kBytes);  // [2][lse, delta][N]
    float stat = 0.f;                                            // of the tile being loaded, threads 0 .. 2 N - 1
    int head = 0, qt = 0;                                        // of the tile being loaded
    auto load = [&](int buffer) {
        const int hq = kvh * a.group + head, i = i0 + qt * N;
        if (threadIdx.x < 2 * N) {
            const int row = i + int(threadIdx.x % N);
            const bool second = threadIdx.x >= N;
            stat = second ? 0.f : kInf;
            if (row < sq.nq) {
                stat = row_stats[(int64_t(second ? a.q_heads : 0) + hq) * a.q_rows + sq.q0 + row];
            }
        }
        const uint32_t to = lds0 + buffer * 2 * kBytes;
        const int64_t first = sq.q0 + i;
        qs.load(static_cast<const T *>(a.q) + first * a.q_s[0] + hq * a.q_s[1], sq.nq - i, to, threadIdx.x);
        gs.load(static_cast<const T *>(a.dout) + first * a.do_s[0] + hq * a.do_s[1], sq.nq - i, to + kBytes,
                threadIdx.x);
        if (++qt == per_head) qt = 0, ++head;
    };
    auto put = [&](int buffer) {
        if (threadIdx.x < 2 * N) stats[buffer * 2 * N + threadIdx.x] = stat;
    };
    if (n > 0) {
        load(0);
        put(0);
    }
    int now_head = 0, now_qt = 0;
    for (int u = 0; u < n; ++u) {
        const int buffer = u & 1;
        wait_loads();
        barrier();
        if (u + 1 < n) load(buffer ^ 1);
        const uint32_t qtile = lds0 + buffer * 2 * kBytes, gtile = qtile + kBytes;
        const float slope = BIAS ? a.slopes[kvh * a.group + now_head] * kLog2e : 0.f;
#pragma unroll
        for (int b = 0; b < N / 32; ++b) {
            const int i = i0 + now_qt * N + b * 32;  // first query of the 32
            // visible to the wave: all of its keys by the first query, or
            // none by the last
            if (i >= sq.nq || j_wave >= limit_of(a, sq, min(i + 31, sq.nq - 1))) continue;
            const bool masked = j_wave + 32 > limit_of(a, sq, i);
            const uint32_t qb = qtile + b * 32 * L::kRowBytes, gb = gtile + b * 32 * L::kRowBytes;
            f32x16_t x = {}, dp = {};
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) x = M::mma(L::row_frag(qb, lane & 31, kk, h), k[kk], x);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) dp = M::mma(L::row_frag(gb, lane & 31, kk, h), v[kk], dp);
            float base[16], delta[16];
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
                const float *s = stats + buffer * 2 * N + b * 32 + 8 * g4 + 4 * h;
                const float4 s0 = *reinterpret_cast<const float4 *>(s), s1 = *reinterpret_cast<const float4 *>(s + N);
                base[4 * g4] = s0.x, base[4 * g4 + 1] = s0.y, base[4 * g4 + 2] = s0.z, base[4 * g4 + 3] = s0.w;
                delta[4 * g4] = s1.x, delta[4 * g4 + 1] = s1.y, delta[4 * g4 + 2] = s1.z, delta[4 * g4 + 3] = s1.w;
            }
            const float away = float(shift + i - j + 4 * h);
            // key j is hidden from the tile's queries before `hidden`
            const int hidden = j < sq.prefix || !a.causal ? 0 : j - shift - i, from = hidden - 4 * h;
            float p[16], ds[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int ir = 8 * (r >> 2) + (r & 3);
                float y, bend = 1.f;
                if constexpr (CAP) {
                    const float th = score.tanh_of(x[r]);
                    bend = fmaf(-th, th, 1.f);
                    y = fmaf(score.capl, th, -base[r]);
                } else {
                    y = fmaf(x[r], score.c1, -base[r]);
                }
                if constexpr (BIAS) y = fmaf(-slope, fabsf(away + float(ir)), y);
                p[r] = __builtin_amdgcn_exp2f(y);
                float d = p[r] * (dp[r] - delta[r]);
                if constexpr (CAP) d *= bend;
                if (masked && ir < from) p[r] = d = 0.f;
                ds[r] = d;
            }
            auto seen = [&](int r) { return r >= hidden; };
            const bool look = masked && a.causal;
            typename M::Frag w[2] = {M::pack(p), M::pack(p + 8)};
            Product<T, D, 2, true>::add(dv, w, gb, lane, look, seen);
            w[0] = M::pack(ds);
            w[1] = M::pack(ds + 8);
            Product<T, D, 2, true>::add(dk, w, qb, lane, look, seen);
        }
        if (++now_qt == per_head) now_qt = 0, ++now_head;
        if (u + 1 < n) put(buffer ^ 1);
    }
    if (j < sq.nk) {
        store_column<T, D>(static_cast<T *>(a.dk) + key * a.dk_s[0] + kvh * a.dk_s[1], a.dim, h, dk, a.scale);
        store_column<T, D>(static_cast<T *>(a.dv) + key * a.dv_s[0] + kvh * a.dv_s[1], a.dim, h, dv, 1.f);
    }
}

template <typename T, int D, bool CAP, bool BIAS>
hipError_t run(const AttnArgs &a, hipStream_t s) {
    constexpr int N = tile_rows(sizeof(T) == 2);
    constexpr int lds = 4 * N * Tile<T, D>::kRowBytes;
    float *stats = static_cast<float *>(a.workspace);  // lse in log 2 units and delta, [2][q_heads][q_rows]
    if (a.q_rows > 0) {
        const int tiles = int(int64_t(a.q_rows) * a.group / kColumns + a.n_seqs);
        const hipError_t e = max_lds(k_dq<T, D, CAP, BIAS>, lds);
        if (e != hipSuccess) return e;
        k_dq<T, D, CAP, BIAS><<<uint32_t(tiles) * a.kv_heads, 256, lds, s>>>(a, tiles, stats);
    }
    if (a.k_rows > 0) {
        constexpr int more = lds + 4 * N * int(sizeof(float));
        const int tiles = a.k_rows / kKeys + a.n_seqs;
        const hipError_t e = max_lds(k_dkv<T, D, CAP, BIAS>, more);
        if (e != hipSuccess) return e;
        k_dkv<T, D, CAP, BIAS><<<uint32_t(tiles) * a.kv_heads, 256, more, s>>>(a, tiles, stats);
    }
    return hipGetLastError();
}

template <typename T, int D>
hipError_t run(const AttnArgs &a, hipStream_t s) {
    if (a.softcap > 0.f) return a.slopes ? run<T, D, true, true>(a, s) : run<T, D, true, false>(a, s);
    return a.slopes ? run<T, D, false, true>(a, s) : run<T, D, false, false>(a, s);
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
