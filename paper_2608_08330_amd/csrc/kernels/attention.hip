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
//     straight into LDS, two buffers, one barrier a tile.  Tiles that all
//     columns see whole run in turns (bf16): the products of the next tile and
//     of the last beside the softmax of this one.
//   few:   for sequences of few columns (single tokens): the waves of a block
//     share 32 columns and walk tiles of 32 keys of their own, each through
//     its own LDS, without a barrier; their results are joined in LDS.
// Both take a share of a sequence's keys where whole sequences would leave
// compute units idle; `join` then adds the shares up in a fixed order.
//
// bf16: the weights are rounded for their product with V, whose matrix
// instruction takes bf16; outputs are 0.19 to 0.23% off 64-bit values, their own
// rounding 0.17%.  Weights as the sum of two operands would take half as many
// products again (few queries, 64 caches: 0.17%, 197 us instead of 181).
//
// Whole calls, bf16: 16,384 tokens, 6 heads of 64: 453 to 468 us (910 to 881
// TFLOP/s), matrix cores busy 44%, the exponentials beside the products; 8,192
// tokens, causal, capped, 6 heads of 128: 181 us; one token against 64 caches of
// up to 32,768 keys, 2 heads of 128: 185 us (3.3 TB/s).
#include <algorithm>
#include <type_traits>

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

// One wave's 32 columns.  BEHIND: by how much (in log 2) a weight may pass 1
// before the maximum follows.  At 0 a row's largest weight is 1 and not rounded
// in bf16: single tokens, 0.20% off instead of 0.27% (512 keys), for 2% more
// time (64 caches of up to 32,768 keys).  `tiles` rescales more columns in a
// pipeline that waits for it: 8,192 causal, capped tokens, 6 heads of 128, take
// 190 us at 0 and 180 us at 8, 0.19% and 0.22% off; it keeps 8.
template <typename T, int D, Cap CAP, bool BIAS, int BEHIND>
struct Columns {
    typedef Op<T> M;
    typedef Tile<T, D> L;
    typename M::Frag q[D / 16];
    f32x16_t acc[D / 32];
    float m, l;
    int lane, h, limit, first_limit, last_limit;
    int place;  // of the query; distances are taken in whole numbers
    float slope;
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
        place = sq.nk - sq.nq + at.i;
        slope = BIAS ? a.slopes[at.head] * kLog2e : 0.f;
        score.init(a);
        load_row<T, D>(static_cast<const T *>(a.q) + at.row * a.q_s[0] + at.head * a.q_s[1], a.dim, h, q);
#pragma unroll
        for (int t = 0; t < D / 32; ++t) acc[t] = f32x16_t{};
        m = -kInf;
        l = 0.f;
        wait_registers();
    }

    // Products <k, q> of the keys in a tile.
    template <int NB>
    __device__ void products(f32x16_t *x, uint32_t kt) const {
#pragma unroll
        for (int b = 0; b < NB; ++b) x[b] = f32x16_t{};
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
            for (int b = 0; b < NB; ++b) x[b] = M::mma(L::row_frag(kt, b * 32 + (lane & 31), kk, h), q[kk], x[b]);
    }

    // One score from its product; `key` is counted from the half's first key,
    // `away` the query's distance to that.
    __device__ float scored(float x, int key, float away) const {
        float th;
        if constexpr (CAP != kNone) x = score.capped<CAP>(x, th);
        else if constexpr (BIAS) x *= score.c1;
        if constexpr (BIAS) x = fmaf(-slope, fabsf(away - float(key)), x);
        return x;
    }
    // What is left to multiply scores by.
    __device__ float factor() const { return CAP != kNone || BIAS ? 1.f : score.c1; }

    // Advances the running maximum past `top`, a tile's own in this half.  It
    // follows only where it is left behind by more than 2^BEHIND (any value will
    // do while the weights stay in range), so that the output is rescaled a few
    // times a row instead of once a tile.  base: what to subtract from
    // scores; returns the factor of the sums so far.
    __device__ float advance(float top, float &base) {
        top = half_max(top) * factor();
        const float before = m;
        if constexpr (BEHIND == 0) m = fmaxf(m, top);
        else m = top > m + float(BEHIND) ? top : m;
        base = m == -kInf ? 0.f : m;
        return __builtin_amdgcn_exp2f(before - base);
    }

    // The weights of the keys from j0 on, from their products x, as operands;
    // advances the maximum and the sum.  Returns what the output so far is to
    // be multiplied by.
    template <int NB>
    __device__ float weights(f32x16_t *x, typename M::Frag *p, int j0) {
        const float away = float(place - j0 - 4 * h);
        const int left = limit - j0 - 4 * h;
        float top = -kInf;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = b * 32 + 8 * (r >> 2) + (r & 3);
                x[b][r] = key < left ? scored(x[b][r], key, away) : -kInf;
                top = fmaxf(top, x[b][r]);
            }
        float base, sum = 0.f;
        const float f = advance(top, base);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[b][r] = __builtin_amdgcn_exp2f(fmaf(x[b][r], factor(), -base));
                sum += x[b][r];
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = x[b][8 * s + e];
                p[2 * b + s] = M::pack(v);
            }
        }
        l = fmaf(l, f, sum);
        return f;
    }

    // f may be anything where there is nothing to multiply yet
    __device__ void rescale(float f) {
        if (__any(f != 1.f)) {
#pragma unroll
            for (int t = 0; t < D / 32; ++t) acc[t] *= f;
        }
    }

    // One tile, keys j0 .. j0 + 32 NB - 1 of the sequence, part after part.
    template <int NB>
    __device__ void step(const AttnArgs &a, uint32_t kt, uint32_t vt, int j0) {
        f32x16_t x[NB];
        typename M::Frag p[2 * NB];
        products<NB>(x, kt);
        rescale(weights<NB>(x, p, j0));
        const bool look = a.causal && j0 + 32 * NB > first_limit;
        Product<T, D, 2 * NB, true>::add(acc, p, vt, lane, look, [&](int j) { return j0 + j < limit; });
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
// Keys of a tile of `tiles`.
template <typename T, int D>
constexpr int kTileKeys = sizeof(T) == 2 && D <= 64 ? 64 : 32;
constexpr int kLeastShare = 128;  // keys


template <typename T, int D, Cap CAP, bool BIAS>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void k_tiles(AttnArgs a, Shares sh) {
    constexpr int N = kTileKeys<T, D>;
    constexpr uint32_t kBytes = N * Tile<T, D>::kRowBytes;
    extern __shared__ __align__(1024) unsigned char lds[];
    Seq sq;
    if (!find_tile<false>(a, tile_of(a), kTileColumns, sq)) return;
    const int kvh = head_of(a), wave = threadIdx.x >> 6;
    const int64_t columns = int64_t(sq.nq) * a.group;
    // the last tiles of a causal sequence have the most keys: first
    const int mine = a.causal ? int((columns + kTileColumns - 1) / kTileColumns) - 1 - sq.tile : sq.tile;
    const int64_t c0 = int64_t(mine) * kTileColumns;

    Columns<T, D, CAP, BIAS, 8> col;
    col.init(a, sq, kvh, c0 + wave * 32);
    const int64_t c_last = min(c0 + kTileColumns, columns) - 1;
    const int keys = limit_of(a, sq, int(c_last / a.group));
    int t0, t1;
    share((keys + N - 1) / N, sh.splits, blockIdx.y, kLeastShare / N, t0, t1);

    const T *k = static_cast<const T *>(a.k) + sq.k0 * a.k_s[0] + kvh * a.k_s[1];
    const T *v = static_cast<const T *>(a.v) + sq.k0 * a.v_s[0] + kvh * a.v_s[1];
    Stager<T, D, N, 256> ks, vs;
    ks.init(threadIdx.x, a.k_s[0], a.dim);
    vs.init(threadIdx.x, a.v_s[0], a.dim);
    const uint32_t base = lds_offset(lds);
    // buffers: K 0, K 1, V 0, V 1
    auto load_k = [&](int t, int buffer) {
        ks.load(k + int64_t(t) * N * a.k_s[0], keys - t * N, base + buffer * kBytes, threadIdx.x);
    };
    auto load_v = [&](int t, int buffer) {
        vs.load(v + int64_t(t) * N * a.v_s[0], keys - t * N, base + (2 + buffer) * kBytes, threadIdx.x);
    };
    constexpr int NB = N / 32;
    int t = t0;
    // Tiles that every column of the block sees whole, an even number of them,
    // in turns that run three tiles at once: the products of the next, the
    // weights of this one and the output of the last, so that the matrix cores
    // and the vector units have independent work from one wave.
    const int whole = max(0, min(t1, limit_of(a, sq, int(c0 / a.group)) / N) - t0) & ~1;
    if constexpr (sizeof(T) == 2) {
        f32x16_t x0[NB], x1[NB];
        bf16x8_t p0[2 * NB] = {}, p1[2 * NB] = {};
        Lanes<T, D> at;
        Walk<Stager<T, D, N, 256>, N> kw, vw;
        at.init(col.lane, base);
        auto turn = [&](f32x16_t *x, f32x16_t *next, bf16x8_t *p, bf16x8_t *last, int now, auto which) {
            constexpr int buffer = decltype(which)::value, other = buffer ^ 1;
            wait_loads();
            barrier();
            if (now + 2 < t0 + whole) kw.template load<buffer * kBytes>(ks);
            vw.template load<(2 + buffer) * kBytes>(vs);
            // H products of the next tile and H of the last, a share of this
            // tile's vector work after each; reads from LDS run ahead
            constexpr int H = NB * D / 16, E = NB * 16, W = D / 32;
            constexpr int kAhead = H < 4 ? H : 4;
            bf16x8_t f[2 * H];
            auto read = [&](int i) {
                f[i] = i < H ? at.row_frag(other * kBytes, i % NB, i / NB)
                             : at.col_frag((2 + other) * kBytes, (i - H) / W, (i - H) % W);
            };
#pragma unroll
            for (int i = 0; i < kAhead; ++i) read(i);
            __builtin_amdgcn_sched_barrier(0);
            const float away = float(col.place - now * N - 4 * col.h);
            float top = -kInf, base = 0.f, less = 1.f, sum = 0.f;
            // plain scores: the maximum first, the weights beside all products;
            // others: the scores beside the first half, the weights beside the
            // second
            auto raise = [&](int e) {
                const float y = col.scored(x[e / 16][e % 16], e / 16 * 32 + 8 * (e % 16 >> 2) + (e & 3), away);
                x[e / 16][e % 16] = y;
                top = fmaxf(top, y);
            };
            uint32_t words[E / 2];
            float even = 0.f;
            auto weigh = [&](int e) {
                const float w = __builtin_amdgcn_exp2f(fmaf(x[e / 16][e % 16], col.factor(), -base));
                sum += w;
                const bf16x2_t two = {__bf16(even), __bf16(w)};
                if (e % 2) words[e / 2] = Lanes<T, D>::opaque(__builtin_bit_cast(uint32_t, two));
                even = w;
            };
            if constexpr (CAP == kNone && !BIAS) {
#pragma unroll
                for (int e = 0; e < E; ++e) raise(e);
                less = col.advance(top, base);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) next[b] = f32x16_t{};
#pragma unroll
            for (int i = 0; i < 2 * H; ++i) {
                if (i < H) next[i % NB] = Op<T>::mma(f[i], col.q[i / NB], next[i % NB]);
                else col.acc[(i - H) % W] = Op<T>::mma(f[i], last[(i - H) / W], col.acc[(i - H) % W]);
                if (i + kAhead < 2 * H) read(i + kAhead);
                if constexpr (CAP == kNone && !BIAS) {
#pragma unroll
                    for (int e = i * E / (2 * H); e < (i + 1) * E / (2 * H); ++e) weigh(e);
                } else {
#pragma unroll
                    for (int e = i % H * E / H; e < (i % H + 1) * E / H; ++e) {
                        if (i < H) raise(e);
                        else weigh(e);
                    }
                    if (i == H - 1) less = col.advance(top, base);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < 2 * NB; ++i) {
                const u32x4_t u = {words[4 * i], words[4 * i + 1], words[4 * i + 2], words[4 * i + 3]};
                p[i] = __builtin_bit_cast(bf16x8_t, u);
            }
            col.l = fmaf(col.l, less, sum);
            col.rescale(less);
        };
        if (whole > 0) {
            kw.init(ks, k + int64_t(t) * N * a.k_s[0], threadIdx.x, base);
            vw.init(vs, v + int64_t(t) * N * a.v_s[0], threadIdx.x, base);
            kw.template load<0>(ks);
            vs.load(v, 0, base + 3 * kBytes, threadIdx.x);  // zeros, the values of a tile before the first
            wait_loads();
            barrier();
            kw.template load<kBytes>(ks);
            col.template products<NB>(x0, base);
            for (; t < t0 + whole; t += 2) {
                turn(x0, x1, p0, p1, t, std::integral_constant<int, 0>());
                turn(x1, x0, p1, p0, t + 1, std::integral_constant<int, 1>());
            }
            wait_loads();
            barrier();
            Product<T, D, 2 * NB, false>::add(col.acc, p1, base + 3 * kBytes, col.lane, false, [](int) { return true; });
            barrier();
        }
    }
    if (t < t1) load_k(t, 0), load_v(t, 0);
    for (int buffer = 0; t < t1; ++t, buffer ^= 1) {
        wait_loads();
        barrier();
        if (t + 1 < t1) load_k(t + 1, buffer ^ 1), load_v(t + 1, buffer ^ 1);
        if (t * N < col.last_limit)
            col.template step<NB>(a, base + buffer * kBytes, base + (2 + buffer) * kBytes, t * N);
    }
    col.store(a, sh, blockIdx.y);
}

// Waves of a block of `few`: as many as the LDS holds two buffers of.
template <typename T, int D>
constexpr int kFewWaves = sizeof(T) == 4 && D == 128 ? 2 : 4;

template <typename T, int D, Cap CAP, bool BIAS>
__global__ __launch_bounds__((64 * kFewWaves<T, D>), 1) void k_few(AttnArgs a, Shares sh) {
    constexpr int W = kFewWaves<T, D>, N = 32;
    constexpr uint32_t kBytes = N * Tile<T, D>::kRowBytes;
    extern __shared__ __align__(1024) unsigned char lds[];
    Seq sq;
    if (!find_tile<false>(a, tile_of(a), kFewColumns, sq)) return;
    const int kvh = head_of(a), wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t columns = int64_t(sq.nq) * a.group, c0 = int64_t(sq.tile) * kFewColumns;

    Columns<T, D, CAP, BIAS, 0> col;
    col.init(a, sq, kvh, c0);
    const int keys = col.last_limit;
    int t0, t1;
    share((keys + N - 1) / N, sh.splits, blockIdx.y, kLeastShare / N * W, t0, t1);

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
        col.template step<1>(a, at, at + kBytes, t * N);
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
__global__ __launch_bounds__(256) void k_join(AttnArgs a, Shares sh) {
    Seq sq;
    if (!find_tile<false>(a, tile_of(a), kJoinColumns, sq)) return;
    const int kvh = head_of(a), lane = threadIdx.x & 63;
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
    int64_t blocks;
    int splits;
};

Plan plan_of(const AttnArgs &a) {
    Plan p;
    const int64_t columns = int64_t(a.q_rows) * a.group;
    p.few = columns <= int64_t(kFewColumns) * a.n_seqs;
    p.blocks = column_blocks(a, p.few ? kFewColumns : kTileColumns);
    const int64_t wanted = int64_t(compute_units()) * (p.few ? 4 : 2);
    const int64_t keys = (a.k_rows + a.n_seqs - 1) / std::max(a.n_seqs, 1);
    int64_t s = std::min<int64_t>((wanted + p.blocks - 1) / p.blocks, (keys + 255) / 256);
    p.splits = int(std::max<int64_t>(1, std::min<int64_t>(s, 64)));
    return p;
}

template <typename T, int D, Cap CAP, bool BIAS>
hipError_t run(const AttnArgs &a, const Plan &p, hipStream_t s) {
    Shares sh{};
    sh.splits = p.splits;
    const int64_t rows = int64_t(p.splits) * a.q_heads * a.q_rows;
    if (p.splits > 1) {
        sh.o = static_cast<float *>(a.workspace);
        sh.ml = reinterpret_cast<float2 *>(sh.o + rows * D);
    }
    constexpr int W = kFewWaves<T, D>;
    const Fold f = fold(p.blocks, p.few ? 64 * W : 256);
    const dim3 grid(f.x, p.splits, f.z);
    if (p.few) {
        constexpr int stage = W * 4 * 32 * Tile<T, D>::kRowBytes, ends = W * 32 * (8 + (D + 4) * 4);
        constexpr int lds = stage > ends ? stage : ends;
        const hipError_t e = max_lds(k_few<T, D, CAP, BIAS>, lds);
        if (e != hipSuccess) return e;
        k_few<T, D, CAP, BIAS><<<grid, 64 * W, lds, s>>>(a, sh);
    } else {
        constexpr int lds = 4 * kTileKeys<T, D> * Tile<T, D>::kRowBytes;
        const hipError_t e = max_lds(k_tiles<T, D, CAP, BIAS>, lds);
        if (e != hipSuccess) return e;
        k_tiles<T, D, CAP, BIAS><<<grid, 256, lds, s>>>(a, sh);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) {
        const Fold j = fold(column_blocks(a, kJoinColumns), 256);
        k_join<T, D><<<dim3(j.x, 1, j.z), 256, 0, s>>>(a, sh);
        e = hipGetLastError();
    }
    return e;
}

template <typename T, int D>
hipError_t run(const AttnArgs &a, const Plan &p, hipStream_t s) {
    return with_terms<T>(a, [&](auto cap, auto bias) { return run<T, D, cap.value, bias.value>(a, p, s); });
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
