// Forward attention of packed sequences on gfx950.
//
//   o_i = sum_j softmax_j(x_ij) v_j over the keys j < limit(i), the maximum
//   and the sum of the softmax kept running over the keys (one pass).
//
// A column is one query of one query head; the columns of a key head are the
// queries of its group of heads, query by query (column i * group + g), so a
// group shares every load of its keys and values.  Scores are computed as
// K Q^T: a column's statistics and its rescaling are values of its lane
// (attention.hpp), and the output is accumulated transposed, V^T P^T.
//
//   tiles: four waves x 32 columns walk the keys together, K and V staged
//     straight into LDS, two buffers, one barrier a tile.
//   few:   for sequences of few columns (single tokens): the waves of a block
//     share 32 columns and walk tiles of 32 keys of their own, each through
//     its own LDS, without a barrier; their results are joined in LDS.
// Both take a share of a sequence's keys where whole sequences would leave
// compute units idle; `join` then adds the shares up in a fixed order.
#include <algorithm>

#include "attention.hpp"
#include "compute_units.hpp"

namespace rtcc {
namespace kern {

namespace {

// Shares of one output row: unnormalised sums over a share's keys, and the
// running maximum (log 2 units) and sum.
struct Shares {
    float *o;   // [splits][q_heads][q_rows][D]
    float2 *ml; // [splits][q_heads][q_rows]
    int splits;
};

// One wave's 32 columns.
template <typename T, int D, bool CAP, bool BIAS>
struct Columns {
    typedef Op<T> M;
    typedef Tile<T, D> L;
    typename M::Frag q[D / 16];
    f32x16_t acc[D / 32];
    float m, l;
    int lane, h, limit, first_limit, last_limit;
    float place, slope;
    Column at;
    Score score;

    // column: the wave's first
    __device__ void init(const AttnArgs &a, const Seq &sq, int kvh, int64_t column) {
        lane = threadIdx.x & 63;
        h = lane >> 5;
        at.init(a, sq, kvh, column);
        limit = limit_of(a, sq, at.i);
        first_limit = __builtin_amdgcn_readlane(limit, 0);
        last_limit = __builtin_amdgcn_readlane(limit, 31);
        place = float(sq.nk - sq.nq + at.i);
        slope = BIAS ? a.slopes[at.head] * kLog2e : 0.f;
        score.init(a);
        load_row<T, D>(static_cast<const T *>(a.q) + at.row * a.q_s[0] + at.head * a.q_s[1], a.dim, h, q);
#pragma unroll
        for (int t = 0; t < D / 32; ++t) acc[t] = f32x16_t{};
        m = -kInf;
        l = 0.f;
    }

    // Keys j0 .. j0 + 32 NB - 1 of the sequence, in LDS; without MASK every
    // column sees all of them.
    template <int NB, bool MASK>
    __device__ void step(const AttnArgs &a, uint32_t kt, uint32_t vt, int j0) {
        f32x16_t x[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            x[b] = f32x16_t{};
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
                x[b] = M::mma(L::row_frag(kt, b * 32 + (lane & 31), kk, h), q[kk], x[b]);
        }
        if constexpr (CAP || BIAS) {
            const float away = place - float(j0) - 4.f * h;  // the distance to the half's first key
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float y = x[b][r];
                    if constexpr (CAP) y = score.capl * score.tanh_of(y);
                    else y *= score.c1;
                    if constexpr (BIAS) y = fmaf(-slope, fabsf(away - float(b * 32 + 8 * (r >> 2) + (r & 3))), y);
                    x[b][r] = y;
                }
        }
        const float c1 = CAP || BIAS ? 1.f : score.c1;
        if constexpr (MASK) {
            const int left = limit - j0 - 4 * h;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (b * 32 + 8 * (r >> 2) + (r & 3) >= left) x[b][r] = -kInf;
        }
        float top = x[0][0];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, x[b][r]);
        top = half_max(top) * c1;
        // The running maximum follows only where it is left behind by more
        // than 2^8 (any value will do while the weights stay in range): the
        // output is rescaled a few times a row instead of once a tile.
        if (__any(top > m + 8.f)) {
            const float now = fmaxf(m, top);
            const float f = m == -kInf ? 0.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= f;
#pragma unroll
            for (int t = 0; t < D / 32; ++t) acc[t] *= f;
        }
        const float base = m == -kInf ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(x[b][r], c1, -base));
                x[b][r] = p;
                sum += p;
            }
        l += sum;
        typename M::Frag p[2 * NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = x[b][8 * s + e];
                p[2 * b + s] = M::pack(v);
            }
        const bool look = MASK && a.causal && j0 + 32 * NB > first_limit;
        Product<T, D, 2 * NB, MASK>::add(acc, p, vt, lane, look, [&](int j) { return j0 + j < limit; });
    }

    // Writes the columns: the result, or a share of it.
    __device__ void store(const AttnArgs &a, const Shares &sh, int split) {
        const float sum = half_sum(l);
        if (!at.valid) return;
        const int64_t place_of = int64_t(at.head) * a.q_rows + at.row;
        if (sh.splits > 1) {
            const int64_t to = int64_t(split) * a.q_heads * a.q_rows + place_of;
            if (h == 0) sh.ml[to] = make_float2(m, sum);
            if (m == -kInf && sum == 0.f) return;  // join does not read it
            store_column<float, D>(sh.o + to * D, D, h, acc, 1.f);
            return;
        }
        if (a.lse && h == 0) a.lse[place_of] = sum == 0.f ? -kInf : (m + log2f(sum)) * kLn2;
        store_column<T, D>(static_cast<T *>(a.out) + at.row * a.o_s[0] + at.head * a.o_s[1], a.dim, h, acc,
                           sum == 0.f ? 0.f : 1.f / sum);
    }
};

// The share [first, end) of n tiles that split `i` of `splits` takes: at least
// `least` tiles each while there are any.
__device__ inline void share(int n, int splits, int i, int least, int &first, int &end) {
    const int per = max((n + splits - 1) / splits, least);
    first = int(min(int64_t(n), int64_t(i) * per));
    end = min(n, first + per);
}

constexpr int kTileColumns = 128, kFewColumns = 32, kJoinColumns = 16;
constexpr int kTileKeys(bool bf16) { return bf16 ? 64 : 32; }
constexpr int kLeastShare = 4;  // tiles: 256 keys, or 128

template <typename T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void k_tiles(AttnArgs a, int tiles, Shares sh) {
    constexpr int N = kTileKeys(sizeof(T) == 2);
    constexpr uint32_t kBytes = N * Tile<T, D>::kRowBytes;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int id = spread(blockIdx.x, gridDim.x);
    Seq sq;
    if (!find_tile<false>(a, id % tiles, kTileColumns, sq)) return;
    const int kvh = id / tiles, wave = threadIdx.x >> 6;
    const int64_t columns = int64_t(sq.nq) * a.group;
    // the last tiles of a causal sequence have the most keys: first
    const int mine = a.causal ? int((columns + kTileColumns - 1) / kTileColumns) - 1 - sq.tile : sq.tile;
    const int64_t c0 = int64_t(mine) * kTileColumns;

    Columns<T, D, CAP, BIAS> col;
    col.init(a, sq, kvh, c0 + wave * 32);
    const int64_t c_last = min(c0 + kTileColumns, columns) - 1;
    const int keys = limit_of(a, sq, int(c_last / a.group));
    int t0, t1;
    share((keys + N - 1) / N, sh.splits, blockIdx.y, kLeastShare, t0, t1);

    const T *k = static_cast<const T *>(a.k) + sq.k0 * a.k_s[0] + kvh * a.k_s[1];
    const T *v = static_cast<const T *>(a.v) + sq.k0 * a.v_s[0] + kvh * a.v_s[1];
    Stager<T, D, N, 256> ks, vs;
    ks.init(threadIdx.x, a.k_s[0], a.dim);
    vs.init(threadIdx.x, a.v_s[0], a.dim);
    const uint32_t base = lds_offset(lds);
    auto load = [&](int t, int buffer) {
        const uint32_t at = base + buffer * 2 * kBytes;
        ks.load(k + int64_t(t) * N * a.k_s[0], keys - t * N, at, threadIdx.x);
        vs.load(v + int64_t(t) * N * a.v_s[0], keys - t * N, at + kBytes, threadIdx.x);
    };
    if (t0 < t1) load(t0, 0);
    int t = t0;
    // pairs of tiles that every column of the block sees whole, each with the
    // addresses of its buffer as constants
    const int whole = min(t1, limit_of(a, sq, int(c0 / a.group)) / N);
    for (; t + 2 <= whole; t += 2) {
        wait_loads();
        barrier();
        load(t + 1, 1);
        col.template step<N / 32, false>(a, base, base + kBytes, t * N);
        wait_loads();
        barrier();
        if (t + 2 < t1) load(t + 2, 0);
        col.template step<N / 32, false>(a, base + 2 * kBytes, base + 3 * kBytes, (t + 1) * N);
    }
    for (; t < t1; ++t) {
        const int buffer = (t - t0) & 1;
        wait_loads();
        barrier();
        if (t + 1 < t1) load(t + 1, buffer ^ 1);
        const uint32_t at = base + buffer * 2 * kBytes;
        if (t * N < col.last_limit) col.template step<N / 32, true>(a, at, at + kBytes, t * N);
    }
    col.store(a, sh, blockIdx.y);
}

// Waves of a block of `few`: as many as the LDS holds two buffers of.
template <typename T, int D>
constexpr int kFewWaves = sizeof(T) == 4 && D == 128 ? 2 : 4;

template <typename T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__((64 * kFewWaves<T, D>), 1) void k_few(AttnArgs a, int tiles, Shares sh) {
    constexpr int W = kFewWaves<T, D>, N = 32;
    constexpr uint32_t kBytes = N * Tile<T, D>::kRowBytes;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int id = spread(blockIdx.x, gridDim.x);
    Seq sq;
    if (!find_tile<false>(a, id % tiles, kFewColumns, sq)) return;
    const int kvh = id / tiles, wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t columns = int64_t(sq.nq) * a.group, c0 = int64_t(sq.tile) * kFewColumns;

    Columns<T, D, CAP, BIAS> col;
    col.init(a, sq, kvh, c0);
    const int keys = col.last_limit;
    int t0, t1;
    share((keys + N - 1) / N, sh.splits, blockIdx.y, kLeastShare * W, t0, t1);

    const T *k = static_cast<const T *>(a.k) + sq.k0 * a.k_s[0] + kvh * a.k_s[1];
    const T *v = static_cast<const T *>(a.v) + sq.k0 * a.v_s[0] + kvh * a.v_s[1];
    Stager<T, D, N, 64> ks, vs;
    ks.init(lane, a.k_s[0], a.dim);
    vs.init(lane, a.v_s[0], a.dim);
    const uint32_t base = lds_offset(lds) + wave * 4 * kBytes;
    auto load = [&](int t, int buffer) {
        const uint32_t at = base + buffer * 2 * kBytes;
        ks.load(k + int64_t(t) * N * a.k_s[0], keys - t * N, at, lane);
        vs.load(v + int64_t(t) * N * a.v_s[0], keys - t * N, at + kBytes, lane);
    };
    int buffer = 0;
    if (t0 + wave < t1) load(t0 + wave, 0);
    for (int t = t0 + wave; t < t1; t += W, buffer ^= 1) {
        if (t + W < t1) {
            wait_reads();
            load(t + W, buffer ^ 1);
            wait_loads_but<2 * Stager<T, D, N, 64>::kLoads>();
        } else {
            wait_loads();
        }
        const uint32_t at = base + buffer * 2 * kBytes;
        if ((t + 1) * N <= col.first_limit) col.template step<1, false>(a, at, at + kBytes, t * N);
        else col.template step<1, true>(a, at, at + kBytes, t * N);
    }

    // join the waves: [wave][column] maximum and sum, then the outputs
    barrier();
    col.l = half_sum(col.l);
    float2 *ml = reinterpret_cast<float2 *>(lds);
    float *o = reinterpret_cast<float *>(lds + W * 32 * sizeof(float2));
    constexpr int kStride = D + 4;  // neighbouring columns four banks apart
    if (lane < 32) ml[wave * 32 + lane] = make_float2(col.m, col.l);
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4 *>(o + (wave * 32 + (lane & 31)) * kStride + 32 * t + 8 * g + 4 * col.h) =
                make_float4(col.acc[t][4 * g], col.acc[t][4 * g + 1], col.acc[t][4 * g + 2], col.acc[t][4 * g + 3]);
    __syncthreads();
    const int n = int(min(columns - c0, int64_t(kFewColumns)));
    for (int e = threadIdx.x; e < n * (D / 4); e += 64 * W) {
        const int c = e / (D / 4), d = e % (D / 4) * 4;
        float m = -kInf;
#pragma unroll
        for (int w = 0; w < W; ++w) m = fmaxf(m, ml[w * 32 + c].x);
        const float top = m == -kInf ? 0.f : m;
        float sum = 0.f, r[4] = {};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float2 one = ml[w * 32 + c];
            const float f = __builtin_amdgcn_exp2f(one.x - top);
            const float4 x = *reinterpret_cast<const float4 *>(o + (w * 32 + c) * kStride + d);
            sum = fmaf(one.y, f, sum);
            r[0] = fmaf(x.x, f, r[0]);
            r[1] = fmaf(x.y, f, r[1]);
            r[2] = fmaf(x.z, f, r[2]);
            r[3] = fmaf(x.w, f, r[3]);
        }
        const uint32_t at_column = uint32_t(c0) + c, i = at_column / uint32_t(a.group);
        const int row = sq.q0 + int(i), head = kvh * a.group + int(at_column - i * a.group);
        if (sh.splits > 1) {
            const int64_t at = (int64_t(blockIdx.y) * a.q_heads + head) * a.q_rows + row;
            if (d == 0) sh.ml[at] = make_float2(m, sum);
            *reinterpret_cast<float4 *>(sh.o + at * D + d) = make_float4(r[0], r[1], r[2], r[3]);
        } else {
            if (d == 0 && a.lse) a.lse[int64_t(head) * a.q_rows + row] = sum == 0.f ? -kInf : (m + log2f(sum)) * kLn2;
            if (d < a.dim) {
                const float f = sum == 0.f ? 0.f : 1.f / sum;
                T *out = static_cast<T *>(a.out) + row * a.o_s[0] + head * a.o_s[1] + d;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if constexpr (sizeof(T) == 2) out[x] = __builtin_bit_cast(uint16_t, __bf16(r[x] * f));
                    else out[x] = r[x] * f;
                }
            }
        }
    }
}

// Adds the shares up, in order: 16 columns a block, a wave for every fourth.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_join(AttnArgs a, int tiles, Shares sh) {
    Seq sq;
    if (!find_tile<false>(a, blockIdx.x % tiles, kJoinColumns, sq)) return;
    const int kvh = blockIdx.x / tiles, lane = threadIdx.x & 63;
    const int64_t columns = int64_t(sq.nq) * a.group;
    for (int c = threadIdx.x >> 6; c < kJoinColumns; c += 4) {
        const int64_t column = int64_t(sq.tile) * kJoinColumns + c;
        if (column >= columns) return;
        const uint32_t i = uint32_t(column) / uint32_t(a.group);
        const int row = sq.q0 + int(i), head = kvh * a.group + int(uint32_t(column) - i * a.group);
        const int64_t at = int64_t(head) * a.q_rows + row, step = int64_t(a.q_heads) * a.q_rows;
        float m = -kInf;
        for (int s = 0; s < sh.splits; ++s) m = fmaxf(m, sh.ml[at + s * step].x);
        const float top = m == -kInf ? 0.f : m;
        constexpr int E = D <= 64 ? 1 : 2;  // channels of a lane
        float sum = 0.f, r[E] = {};
        for (int s = 0; s < sh.splits; ++s) {
            const float2 one = sh.ml[at + s * step];
            if (one.x == -kInf && one.y == 0.f) continue;  // nothing was written
            const float f = __builtin_amdgcn_exp2f(one.x - top);
            sum = fmaf(one.y, f, sum);
            if (lane * E < D) {
#pragma unroll
                for (int e = 0; e < E; ++e) r[e] = fmaf(sh.o[(at + s * step) * D + lane * E + e], f, r[e]);
            }
        }
        if (lane == 0 && a.lse) a.lse[at] = sum == 0.f ? -kInf : (m + log2f(sum)) * kLn2;
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        T *out = static_cast<T *>(a.out) + row * a.o_s[0] + head * a.o_s[1];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int d = lane * E + e;
            if (d < a.dim) {
                if constexpr (sizeof(T) == 2) out[d] = __builtin_bit_cast(uint16_t, __bf16(r[e] * f));
                else out[d] = r[e] * f;
            }
        }
    }
}

struct Plan {
    bool few;
    int tiles, splits;
};

Plan plan_of(const AttnArgs &a) {
    Plan p;
    const int64_t columns = int64_t(a.q_rows) * a.group;
    p.few = columns <= int64_t(kFewColumns) * a.n_seqs;
    const int per = p.few ? kFewColumns : kTileColumns;
    p.tiles = int(columns / per + a.n_seqs);  // at least the sum over sequences of their rounded tiles
    const int64_t blocks = int64_t(p.tiles) * a.kv_heads;
    const int64_t wanted = int64_t(compute_units()) * (p.few ? 4 : 2);
    const int64_t keys = (a.k_rows + a.n_seqs - 1) / std::max(a.n_seqs, 1);
    int64_t s = std::min<int64_t>((wanted + blocks - 1) / blocks, (keys + 255) / 256);
    p.splits = int(std::max<int64_t>(1, std::min<int64_t>(s, 64)));
    return p;
}

template <typename T, int D, bool CAP, bool BIAS>
hipError_t run(const AttnArgs &a, const Plan &p, hipStream_t s) {
    Shares sh{};
    sh.splits = p.splits;
    const int64_t rows = int64_t(p.splits) * a.q_heads * a.q_rows;
    if (p.splits > 1) {
        sh.o = static_cast<float *>(a.workspace);
        sh.ml = reinterpret_cast<float2 *>(sh.o + rows * D);
    }
    const dim3 grid(uint32_t(p.tiles) * a.kv_heads, p.splits);
    if (p.few) {
        constexpr int W = kFewWaves<T, D>;
        constexpr int stage = W * 4 * 32 * Tile<T, D>::kRowBytes, ends = W * 32 * (8 + (D + 4) * 4);
        constexpr int lds = stage > ends ? stage : ends;
        const hipError_t e = max_lds(k_few<T, D, CAP, BIAS>, lds);
        if (e != hipSuccess) return e;
        k_few<T, D, CAP, BIAS><<<grid, 64 * W, lds, s>>>(a, p.tiles, sh);
    } else {
        constexpr int lds = 4 * kTileKeys(sizeof(T) == 2) * Tile<T, D>::kRowBytes;
        const hipError_t e = max_lds(k_tiles<T, D, CAP, BIAS>, lds);
        if (e != hipSuccess) return e;
        k_tiles<T, D, CAP, BIAS><<<grid, 256, lds, s>>>(a, p.tiles, sh);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) {
        const int tiles = int(int64_t(a.q_rows) * a.group / kJoinColumns + a.n_seqs);
        k_join<T, D><<<uint32_t(tiles) * a.kv_heads, 256, 0, s>>>(a, tiles, sh);
        e = hipGetLastError();
    }
    return e;
}

template <typename T, int D>
hipError_t run(const AttnArgs &a, const Plan &p, hipStream_t s) {
    if (a.softcap > 0.f) return a.slopes ? run<T, D, true, true>(a, p, s) : run<T, D, true, false>(a, p, s);
    return a.slopes ? run<T, D, false, true>(a, p, s) : run<T, D, false, false>(a, p, s);
}

template <typename T>
hipError_t run(const AttnArgs &a, const Plan &p, hipStream_t s) {
    switch (padded(a.dim)) {
        case 32: return run<T, 32>(a, p, s);
        case 64: return run<T, 64>(a, p, s);
        default: return run<T, 128>(a, p, s);
    }
}

}  // namespace

size_t attention_workspace(const AttnArgs &a) {
    if (a.n_seqs == 0 || a.q_rows == 0) return 0;
    const Plan p = plan_of(a);
    if (p.splits == 1) return 0;
    return size_t(p.splits) * a.q_heads * a.q_rows * (padded(a.dim) + 2) * sizeof(float);
}

int attention(const AttnArgs &a, void *stream) {
    const Plan p = plan_of(a);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.bf16 ? run<uint16_t>(a, p, s) : run<float>(a, p, s);
}

}  // namespace kern
}  // namespace rtcc
