// Layer norm of a residual stream on gfx950, and its gradient.
//
//   s = x + residual,  n = (s - mean(s)) r,  r = 1 / sqrt(var(s) + eps),
//   y = n w + b
//   g = dy w;  ds = r (g - mean(g) - n mean(g n)) + dsum
//   dw = sum over rows of dy n,  db = sum over rows of dy
//
// G threads hold one row in registers, V times eight channels each (thread l:
// channels 8 (l + G v) ..), so every tensor is read once.  The mean is taken twice: its
// first sum is off by some 2^-20 of it, which is much beside the spread of a row far
// from zero (n of a row of one value would be up to 1).  The differences from it are
// exact there, and their sum, beside that of their squares, gives what is left of the
// mean and the variance without it.  Rows of up to 2,048 channels
// (of the gradient 1,536, of float32 with a gradient past the norm 1,024) stay within a
// wave (G <= 64: sums by exchanges), longer ones take a block of 256 or 512 threads
// (sums through LDS).  Bandwidth bound: 32,768 rows of 384 channels, bf16, with
// residual: 20.5 us, 4.9 TB/s, the rate of a copy; the gradient with the one past the
// norm 22 us and 4 for the weights' sums (4.7 TB/s); float32 gradient of 4,577 rows of
// 4,104 channels 47 + 7 us.
#include <algorithm>

#include <hip/hip_runtime.h>

#include "compute_units.hpp"
#include "token_ops.hpp"

namespace rtcc {
namespace kern {

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// 8 consecutive elements as they lie in memory, so that a row's loads are all
// under way before the first is used
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
    u32x4_t u;
    __device__ void load(const uint16_t *p) { u = *reinterpret_cast<const u32x4_t *>(p); }
    __device__ float operator[](int e) const {
        return __uint_as_float(e & 1 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
    }
};
template <>
struct Eight<float> {
    f32x4_t a, b;
    __device__ void load(const float *p) {
        a = reinterpret_cast<const f32x4_t *>(p)[0];
        b = reinterpret_cast<const f32x4_t *>(p)[1];
    }
    __device__ float operator[](int e) const { return e < 4 ? a[e] : b[e - 4]; }
};
__device__ inline void store8(uint16_t *p, const float *v) {
    bf16x8_t f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __bf16(v[e]);
    *reinterpret_cast<bf16x8_t *>(p) = f;
}
__device__ inline void store8(float *p, const float *v) {
    f32x4_t a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = v[e], b[e] = v[e + 4];
    reinterpret_cast<f32x4_t *>(p)[0] = a;
    reinterpret_cast<f32x4_t *>(p)[1] = b;
}
// of a weight: float32 at any address of a float
__device__ inline void load8_weight(const float *p, float *v) {
    const f32x4_any_t a = reinterpret_cast<const f32x4_any_t *>(p)[0], b = reinterpret_cast<const f32x4_any_t *>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = a[e], v[e + 4] = b[e];
}

// x of another lane, by a pattern within its row of 16.
template <int PATTERN>
__device__ inline float from_lane(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), PATTERN, 0xf, 0xf, true));
}
// Sum over the G <= 64 lanes of a group, in all of them: within rows of 16 by the
// neighbour, the neighbouring pair and the mirrored half and row (whose lanes hold
// equal sums), then rows by exchanges.  Through LDS a step would take 100 cycles.
template <int G>
__device__ inline float lane_sum(float x) {
    if constexpr (G >= 2) x += from_lane<0xb1>(x);
    if constexpr (G >= 4) x += from_lane<0x4e>(x);
    if constexpr (G >= 8) x += from_lane<0x141>(x);
    if constexpr (G >= 16) x += from_lane<0x140>(x);
    if constexpr (G >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (G >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return x;
}

// Sums of N values over the G threads of a row; `part` is LDS of a block's waves
// (G > 64), used again only after the caller's next barrier.
template <int G, int N>
__device__ inline void row_sums(float (&x)[N], float (*part)[2]) {
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = lane_sum<(G < 64 ? G : 64)>(x[n]);
    if constexpr (G > 64) {
        const int wave = threadIdx.x / 64;
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) part[wave][n] = x[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            x[n] = 0.f;
#pragma unroll
            for (int w = 0; w < G / 64; ++w) x[n] += part[w][n];
        }
    }
}

// A row's first mean, rounded before it is taken from the row's values: the difference
// of one with the unrounded product would itself be rounded.
__device__ inline float first_mean(float sum, float over) {
#pragma clang fp contract(off)
    return sum * over;
}
// sum / channels, over = 1 / channels: exact where that is a float (equal differences),
// in 3 instructions for a division's 10, which a row would wait for.
__device__ inline float second_mean(float sum, float channels, float over) {
    const float q = sum * over;
    return fmaf(fmaf(-q, channels, sum), over, q);
}
// Sum of squares of a row's differences from its mean, from `left`, the sums of those
// from the first mean and of their squares, and rest, the mean of the former.
__device__ inline float square_sum(const float (&left)[2], float rest) { return fmaxf(fmaf(-rest, left[0], left[1]), 0.f); }

template <int G>
constexpr int kThreads = G > 256 ? G : 256;

template <typename T, int G, int V>
__global__ __launch_bounds__(kThreads<G>) void k_layer_norm(LayerNormArgs a) {
    constexpr int kRows = kThreads<G> / G;
    __shared__ float part[2][G > 64 ? G / 64 : 1][2];
    const uint32_t place = (blockIdx.z * gridDim.x + blockIdx.x) * uint32_t(kRows) + threadIdx.x / G;
    if (place >= uint32_t(a.rows)) return;  // all of a row's threads
    const int64_t row = place;
    const int l = threadIdx.x % G;
    const float over = 1.f / float(a.channels);
    Eight<T> x[V], r[V];
    const T *px = static_cast<const T *>(a.x) + row * a.x_s, *pr = static_cast<const T *>(a.residual) + row * a.residual_s;
    float s[V][8], sum[1] = {}, left[2] = {};
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = 8 * (l + G * v);
        if (c < a.channels) {
            x[v].load(px + c);
            if (a.residual) r[v].load(pr + c);
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const bool on = 8 * (l + G * v) < a.channels;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[v][e] = on ? (a.residual ? x[v][e] + r[v][e] : x[v][e]) : 0.f;
            sum[0] += s[v][e];
        }
        if (on && a.sum_out) store8(static_cast<T *>(a.sum_out) + row * a.sum_s + 8 * (l + G * v), s[v]);
    }
    row_sums<G>(sum, part[0]);
    const float mean = first_mean(sum[0], over);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[v][e] = 8 * (l + G * v) < a.channels ? s[v][e] - mean : 0.f;
            left[0] += s[v][e];
            left[1] = fmaf(s[v][e], s[v][e], left[1]);
        }
    row_sums<G>(left, part[1]);
    const float rest = second_mean(left[0], float(a.channels), over);
    const float scale = rsqrtf(fmaf(square_sum(left, rest), over, a.eps));
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = 8 * (l + G * v);
        if (c >= a.channels) continue;
        float w[8], b[8];
        if (a.weight) load8_weight(a.weight + c, w);
        if (a.bias) load8_weight(a.bias + c, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[v][e] = (s[v][e] - rest) * scale;
            s[v][e] = fmaf(s[v][e], a.weight ? w[e] : 1.f, a.bias ? b[e] : 0.f);
        }
        store8(static_cast<T *>(a.out) + row * a.out_s + c, s[v]);
    }
}

// A block walks rows and keeps the sums of its channels' dw and db in registers;
// the next row's loads are under way while a row's sums are made (32,768 rows of 384:
// 22 us; with sums by shuffles and each row's loads at its turn 34).  partial:
// [blocks][2][channels].  PAST: with dsum.
template <typename T, int G, int V, bool PAST>
__global__ __launch_bounds__(kThreads<G>, 2) void k_layer_norm_grad(LayerNormArgs a) {
    constexpr int kRows = kThreads<G> / G;
    constexpr int kTensors = PAST ? 3 : 2;
    // what fits the registers
    constexpr bool kAhead = sizeof(T) == 2 ? V <= 3 : V * kTensors <= 6;
    __shared__ float part[3][G > 64 ? G / 64 : 1][2];
    const int l = threadIdx.x % G;
    const float over = 1.f / float(a.channels);
    float dw[V][8] = {}, db[V][8] = {}, w[V][8];
    Eight<T> x[V] = {}, dy[V] = {}, ds[V] = {};
    auto fetch = [&](int64_t row) {
        const T *px = static_cast<const T *>(a.x) + row * a.x_s, *pg = static_cast<const T *>(a.dout) + row * a.dout_s;
        const T *pd = PAST ? static_cast<const T *>(a.residual) + row * a.residual_s : nullptr;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = 8 * (l + G * v);
            if (c < a.channels) {
                x[v].load(px + c);
                dy[v].load(pg + c);
                if (PAST) ds[v].load(pd + c);
            }
        }
    };
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = 8 * (l + G * v);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[v][e] = 1.f;
        if (a.weight && c < a.channels) load8_weight(a.weight + c, w[v]);
    }
    int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / G;
    const int64_t ahead = int64_t(gridDim.x) * kRows;
    if (kAhead && row < a.rows) fetch(row);
    for (; row < a.rows; row += ahead) {
        if (!kAhead) {
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = dy[v] = ds[v] = Eight<T>{};  // not kept over the row
            fetch(row);
        }
        // channels past the end hold zeros
        float n[V][8], y[V][8], past[V][8], sum[1] = {}, left[2] = {}, dots[2] = {};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                n[v][e] = x[v][e];
                y[v][e] = dy[v][e];
                if (PAST) past[v][e] = ds[v][e];
                sum[0] += n[v][e];
            }
        if (kAhead && row + ahead < a.rows) fetch(row + ahead);
        row_sums<G>(sum, part[0]);
        const float mean = first_mean(sum[0], over);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                n[v][e] = 8 * (l + G * v) < a.channels ? n[v][e] - mean : 0.f;
                left[0] += n[v][e];
                left[1] = fmaf(n[v][e], n[v][e], left[1]);
            }
        row_sums<G>(left, part[1]);
        const float rest = second_mean(left[0], float(a.channels), over);
        const float scale = rsqrtf(fmaf(square_sum(left, rest), over, a.eps));
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                n[v][e] = (n[v][e] - rest) * scale;
                dw[v][e] = fmaf(y[v][e], n[v][e], dw[v][e]);
                db[v][e] += y[v][e];
                y[v][e] *= w[v][e];
                dots[0] += y[v][e];
                dots[1] = fmaf(y[v][e], n[v][e], dots[1]);
            }
        row_sums<G>(dots, part[2]);
        const float m0 = dots[0] * over, m1 = dots[1] * over;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = 8 * (l + G * v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[v][e] = scale * (y[v][e] - fmaf(n[v][e], m1, m0));
                if (PAST) y[v][e] += past[v][e];
            }
            if (c < a.channels) store8(static_cast<T *>(a.out) + row * a.out_s + c, y[v]);
        }
        if constexpr (G > 64) __syncthreads();  // the sums' LDS before the next row
    }
    if (!a.partial) return;
    float *to = a.partial + int64_t(blockIdx.x) * 2 * a.channels;
    if constexpr (G >= 256) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = 8 * (l + G * v);
            if (c >= a.channels) continue;
            store8(to + c, dw[v]);
            store8(to + a.channels + c, db[v]);
        }
    } else {
        // the rows of a wave, then the four waves
        __shared__ float both[4][2][V * G * 8];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int d = G; d < 64; d <<= 1) {
                    dw[v][e] += __shfl_xor(dw[v][e], d);
                    db[v][e] += __shfl_xor(db[v][e], d);
                }
                if (threadIdx.x % 64 < G) {
                    both[threadIdx.x / 64][0][8 * (l + G * v) + e] = dw[v][e];
                    both[threadIdx.x / 64][1][8 * (l + G * v) + e] = db[v][e];
                }
            }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * a.channels; i += 256) {
            const int k = i >= a.channels, c = i - k * a.channels;
            to[i] = (both[0][k][c] + both[1][k][c]) + (both[2][k][c] + both[3][k][c]);
        }
    }
}

// Adds up the blocks' sums, in a fixed order: kSumThreads threads a channel take
// every kSumThreads-th block, then halves are added.
constexpr int kSumChannels = 16, kSumThreads = 64;
__global__ __launch_bounds__(kSumChannels *kSumThreads) void k_layer_norm_sums(LayerNormArgs a, int blocks) {
    __shared__ float part[kSumThreads][kSumChannels];
    const int x = threadIdx.x % kSumChannels, l = threadIdx.x / kSumChannels;
    const int at = int(blockIdx.x) * kSumChannels + x;  // 2 channels is a multiple of 16
    float sum = 0.f;
#pragma unroll 4
    for (int b = l; b < blocks; b += kSumThreads) sum += a.partial[int64_t(b) * 2 * a.channels + at];
    part[l][x] = sum;
    for (int half = kSumThreads / 2; half > 0; half /= 2) {
        __syncthreads();
        if (l < half) part[l][x] += part[l + half][x];
    }
    if (l == 0) {
        if (at < a.channels) {
            if (a.dweight) a.dweight[at] = part[0][x];
        } else if (a.dbias) {
            a.dbias[at - a.channels] = part[0][x];
        }
    }
}

// Threads of a row and eights of channels each: the fewest threads that hold the row
// in at most `most` eights, or, of the longest rows, in four.
struct Cut {
    int g, v;
};
constexpr Cut cut(int channels, int most) {
    const int eights = channels / 8;
    for (int g : {8, 16, 32, 64, 256, 512})
        if (eights <= most * g) return {g, (eights + g - 1) / g};
    return {512, (eights + 511) / 512};
}
// Three eights, of float32 with a gradient past the norm two: then the next row's fit
// the registers beside this one's and the sums (2,281 rows of 7,712 channels, bf16, 512
// threads with two: 40 us, 256 with four 86; 16,384 of 2,048: 58 us, 64 threads with
// four 99).
constexpr int grad_most(bool bf16, bool past) { return !bf16 && past ? 2 : 3; }
Cut grad_cut(const LayerNormArgs &a) { return cut(a.channels, grad_most(a.bf16, a.residual)); }
// Whether a row of some width is cut so: kernels of other cuts are not built.
constexpr bool is_cut(int g, int v, int most) {
    for (int channels = 8; channels <= kMaxNormChannels; channels += 8) {
        const Cut c = cut(channels, most);
        if (c.g == g && c.v == v) return true;
    }
    return false;
}

// Two blocks a CU, one of 512 threads: as many as fit it, and their sums stay small.
int grad_blocks(const LayerNormArgs &a) {
    const Cut c = grad_cut(a);
    return int(std::min<int64_t>(row_tiles(a.rows, std::max(1, 256 / c.g)), (c.g > 256 ? 1 : 2) * compute_units()));
}

template <typename T, int G, int V>
hipError_t run(const LayerNormArgs &a, int grad_blocks, hipStream_t s) {
    constexpr bool kBf16 = sizeof(T) == 2;
    constexpr bool kForward = is_cut(G, V, 4), kPast = is_cut(G, V, grad_most(kBf16, true)),
                   kAlone = is_cut(G, V, grad_most(kBf16, false));
    if (grad_blocks && a.residual) {
        if constexpr (kPast) k_layer_norm_grad<T, G, V, true><<<grad_blocks, kThreads<G>, 0, s>>>(a);
    } else if (grad_blocks) {
        if constexpr (kAlone) k_layer_norm_grad<T, G, V, false><<<grad_blocks, kThreads<G>, 0, s>>>(a);
    } else if constexpr (kForward) {
        const Fold f = fold(row_tiles(a.rows, kThreads<G> / G), kThreads<G>);
        k_layer_norm<T, G, V><<<dim3(f.x, 1, f.z), kThreads<G>, 0, s>>>(a);
    }
    return hipGetLastError();
}

template <typename T, int G>
hipError_t run(const LayerNormArgs &a, int v, int grad_blocks, hipStream_t s) {
    switch (v) {
        case 1: return run<T, G, 1>(a, grad_blocks, s);
        case 2: return run<T, G, 2>(a, grad_blocks, s);
        case 3: return run<T, G, 3>(a, grad_blocks, s);
        default: return run<T, G, 4>(a, grad_blocks, s);
    }
}

template <typename T>
hipError_t run(const LayerNormArgs &a, int grad_blocks, hipStream_t s) {
    const Cut c = grad_blocks ? grad_cut(a) : cut(a.channels, 4);
    switch (c.g) {
        case 8: return run<T, 8>(a, c.v, grad_blocks, s);
        case 16: return run<T, 16>(a, c.v, grad_blocks, s);
        case 32: return run<T, 32>(a, c.v, grad_blocks, s);
        case 64: return run<T, 64>(a, c.v, grad_blocks, s);
        case 256: return run<T, 256>(a, c.v, grad_blocks, s);
        default: return run<T, 512>(a, c.v, grad_blocks, s);
    }
}

}  // namespace

int layer_norm(const LayerNormArgs &a, void *stream) {
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.bf16 ? run<uint16_t>(a, 0, s) : run<float>(a, 0, s);
}

size_t layer_norm_grad_workspace(const LayerNormArgs &a) {
    if (a.rows == 0 || !(a.dweight || a.dbias)) return 0;
    return size_t(grad_blocks(a)) * 2 * a.channels * sizeof(float);
}

int layer_norm_grad(const LayerNormArgs &args, void *stream) {
    LayerNormArgs a = args;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool sums = a.dweight || a.dbias;
    if (!sums) a.partial = nullptr;
    const int blocks = a.rows > 0 ? grad_blocks(a) : 0;  // the sums over no rows are zero
    if (blocks) {
        const hipError_t e = a.bf16 ? run<uint16_t>(a, blocks, s) : run<float>(a, blocks, s);
        if (e != hipSuccess) return e;
    }
    if (!sums) return hipSuccess;
    k_layer_norm_sums<<<2 * a.channels / kSumChannels, kSumChannels * kSumThreads, 0, s>>>(a, blocks);
    return hipGetLastError();
}

}  // namespace kern
}  // namespace rtcc
