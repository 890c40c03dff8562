// Norm and rotation of queries and keys on gfx950, and its gradient.
//
//   n = x r w,  r = 1 / sqrt(mean(x^2) + eps);  y = R n
//   g = R^T dy;  dx = r (g w - x r mean(g w x r));  dw = sum over rows (and
//   heads) of g x r
//
// G lanes hold one head of one row, 16 channels each, laid out so that both
// channels of a rotated pair are in one lane: [8 l, 8 l + 8) and the same in
// the upper half, or, with interleaved pairs, [16 l, 16 l + 16).  A pair's
// sine and cosine depend on the row alone: a lane computes its eight once and
// uses them for all heads of its chunk of heads.  Bandwidth bound: every
// element is read once and written once.  32,768 rows of 12 heads of 64, bf16:
// 30 us, 3.4 TB/s.
#include <algorithm>

#include <hip/hip_runtime.h>

#include "compute_units.hpp"
#include "token_ops.hpp"

namespace rtcc {
namespace kern {

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// 8 consecutive elements
__device__ inline void load8(const uint16_t *p, float *v) {
    const u32x4_t u = *reinterpret_cast<const u32x4_t *>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(u[e] << 16);
        v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
}
__device__ inline void load8(const float *p, float *v) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
// of a weight: float32 at any address of a float
__device__ inline void load8_weight(const float *p, float *v) {
    typedef float f32x4_t __attribute__((ext_vector_type(4), aligned(4)));
    const f32x4_t a = reinterpret_cast<const f32x4_t *>(p)[0], b = reinterpret_cast<const f32x4_t *>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = a[e], v[e + 4] = b[e];
}
__device__ inline void store8(uint16_t *p, const float *v) {
    typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
    bf16x8_t f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __bf16(v[e]);
    *reinterpret_cast<bf16x8_t *>(p) = f;
}
__device__ inline void store8(float *p, const float *v) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// Sum over the G lanes of a group (G a power of two).
template <int G>
__device__ inline float group_sum(float x) {
#pragma unroll
    for (int d = 1; d < G; d <<= 1) x += __shfl_xor(x, d);
    return x;
}

// A lane's 16 channels: v[0 .. 8) and v[8 .. 16) start at channels `lo` and
// `hi`; pair p = first + e has its members at v[one(e)], v[two(e)].
template <bool IL>
struct Lane {
    int lo, hi, first;
    bool on;
    __device__ Lane(int l, int dim) {
        on = 16 * l < dim;
        first = 8 * l;
        lo = IL ? 16 * l : 8 * l;
        hi = IL ? 16 * l + 8 : 8 * l + dim / 2;
    }
    __device__ static constexpr int one(int e) { return IL ? 2 * e : e; }
    __device__ static constexpr int two(int e) { return IL ? 2 * e + 1 : e + 8; }
};

// Cosine and sine of the lane's eight pairs in one row.  The angle in turns,
// float64, so that positions of any size keep their fraction.
__device__ inline void angles(const NormRopeArgs &a, int row, int first, bool on, float *cs, float *sn) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int p = first + e;
        cs[e] = 1.f;
        sn[e] = 0.f;
        if (on && p < a.section_end[2]) {
            const int axis = p < a.section_end[0] ? 0 : p < a.section_end[1] ? 1 : 2;
            const double turns =
                double(a.positions[int64_t(row) * a.n_axes + axis]) * double(a.inv_freq[p]) * 0.15915494309189535;
            sincospif(2.f * float(turns - rint(turns)), &sn[e], &cs[e]);
        }
    }
}

// Heads are cut into chunks, the queries' first; grid.y is a chunk.  Copies of
// v are a further kind of head.
struct Chunk {
    int kind, head, end;  // kind 0: q, 1: k, 2: v
    __device__ Chunk(const NormRopeArgs &a, int per, int c) {
        const int cq = (a.q_heads + per - 1) / per, ck = (a.kv_heads + per - 1) / per;
        kind = c < cq ? 0 : c < cq + ck ? 1 : 2;
        c -= kind == 0 ? 0 : kind == 1 ? cq : cq + ck;
        head = c * per;
        end = min(head + per, kind == 0 ? a.q_heads : a.kv_heads);
    }
};

template <typename T, int G, bool IL>
__global__ __launch_bounds__(256) void k_norm_rope(NormRopeArgs a, int per) {
    const uint32_t place = (blockIdx.z * gridDim.x + blockIdx.x) * (256u / G) + threadIdx.x / G;
    if (place >= uint32_t(a.rows)) return;
    const int row = int(place);
    const Lane<IL> lane(threadIdx.x % G, a.dim);
    const Chunk c(a, per, blockIdx.y);
    int64_t out_row = row;
    if (c.kind > 0 && a.slots) {
        out_row = a.slots[row];
        if (out_row < 0 || out_row >= a.slot_rows) return;
    }
    const bool q = c.kind == 0, v = c.kind == 2;
    const T *x = static_cast<const T *>(q ? a.q : v ? a.v : a.k) + row * (q ? a.q_s[0] : v ? a.v_s[0] : a.k_s[0]);
    T *y = static_cast<T *>(q ? a.q_out : v ? a.v_out : a.k_out) +
           out_row * (q ? a.qo_s[0] : v ? a.vo_s[0] : a.ko_s[0]);
    const int64_t xh = q ? a.q_s[1] : v ? a.v_s[1] : a.k_s[1], yh = q ? a.qo_s[1] : v ? a.vo_s[1] : a.ko_s[1];
    if (v) {
        if (!lane.on) return;
        for (int h = c.head; h < c.end; ++h) {
            float u[16];
            load8(x + h * xh + lane.lo, u);
            load8(x + h * xh + lane.hi, u + 8);
            store8(y + h * yh + lane.lo, u);
            store8(y + h * yh + lane.hi, u + 8);
        }
        return;
    }
    float cs[8], sn[8];
    angles(a, row, lane.first, lane.on, cs, sn);
    const float *weight = q ? a.q_weight : a.k_weight;
    const int wh = q ? a.q_weight_stride : a.k_weight_stride;
    for (int h = c.head; h < c.end; ++h) {
        float u[16] = {}, w[16];
        if (lane.on) {
            load8(x + h * xh + lane.lo, u);
            load8(x + h * xh + lane.hi, u + 8);
        }
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) ss = fmaf(u[e], u[e], ss);
        const float r = rsqrtf(group_sum<G>(ss) / float(a.dim) + a.eps);
        if (!lane.on) continue;
        if (weight) {
            load8_weight(weight + h * wh + lane.lo, w);
            load8_weight(weight + h * wh + lane.hi, w + 8);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] *= weight ? r * w[e] : r;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float f = u[lane.one(e)], s = u[lane.two(e)];
            u[lane.one(e)] = f * cs[e] - s * sn[e];
            u[lane.two(e)] = s * cs[e] + f * sn[e];
        }
        store8(y + h * yh + lane.lo, u);
        store8(y + h * yh + lane.hi, u + 8);
    }
}

// partial: [blocks][chunks][dim] sums of dw over the block's rows and the
// chunk's heads.
template <typename T, int G, bool IL>
__global__ __launch_bounds__(256) void k_norm_rope_grad(NormRopeArgs a, int per) {
    const Lane<IL> lane(threadIdx.x % G, a.dim);
    const Chunk c(a, per, blockIdx.y);
    const bool q = c.kind == 0;
    const int64_t xr = q ? a.q_s[0] : a.k_s[0], xh = q ? a.q_s[1] : a.k_s[1];
    const int64_t gr = q ? a.dqo_s[0] : a.dko_s[0], gh = q ? a.dqo_s[1] : a.dko_s[1];
    const int64_t yr = q ? a.qo_s[0] : a.ko_s[0], yh = q ? a.qo_s[1] : a.ko_s[1];
    const float *weight = q ? a.q_weight : a.k_weight;
    const int wh = q ? a.q_weight_stride : a.k_weight_stride;
    float dw[16] = {};
    for (int64_t row = int64_t(blockIdx.x) * (256 / G) + threadIdx.x / G; row < a.rows;
         row += int64_t(gridDim.x) * (256 / G)) {
        float cs[8], sn[8];
        angles(a, int(row), lane.first, lane.on, cs, sn);
        const T *x = static_cast<const T *>(q ? a.q : a.k) + row * xr;
        const T *dy = static_cast<const T *>(q ? a.dq_out : a.dk_out) + row * gr;
        T *dx = static_cast<T *>(q ? a.q_out : a.k_out) + row * yr;
        for (int h = c.head; h < c.end; ++h) {
            float u[16] = {}, g[16] = {}, w[16];
            if (lane.on) {
                load8(x + h * xh + lane.lo, u);
                load8(x + h * xh + lane.hi, u + 8);
                load8(dy + h * gh + lane.lo, g);
                load8(dy + h * gh + lane.hi, g + 8);
                if (weight) {
                    load8_weight(weight + h * wh + lane.lo, w);
                    load8_weight(weight + h * wh + lane.hi, w + 8);
                }
            }
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) ss = fmaf(u[e], u[e], ss);
            const float r = rsqrtf(group_sum<G>(ss) / float(a.dim) + a.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float f = g[lane.one(e)], s = g[lane.two(e)];
                g[lane.one(e)] = f * cs[e] + s * sn[e];
                g[lane.two(e)] = s * cs[e] - f * sn[e];
            }
            float dot = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                u[e] *= r;
                dw[e] = fmaf(g[e], u[e], dw[e]);
                if (weight) g[e] *= lane.on ? w[e] : 0.f;
                dot = fmaf(g[e], u[e], dot);
            }
            dot = group_sum<G>(dot) / float(a.dim);
            if (lane.on) {
#pragma unroll
                for (int e = 0; e < 16; ++e) g[e] = r * fmaf(-u[e], dot, g[e]);
                store8(dx + h * yh + lane.lo, g);
                store8(dx + h * yh + lane.hi, g + 8);
            }
        }
    }
    if (!a.partial) return;
    // lanes of one place in their group, then the four waves
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int d = G; d < 64; d <<= 1) dw[e] += __shfl_xor(dw[e], d);
    __shared__ float part[4][128];
    if ((threadIdx.x & 63) < G && lane.on) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            part[threadIdx.x >> 6][lane.lo + e] = dw[e];
            part[threadIdx.x >> 6][lane.hi + e] = dw[e + 8];
        }
    }
    __syncthreads();
    const int d = threadIdx.x;
    if (d < a.dim)
        a.partial[(int64_t(blockIdx.x) * gridDim.y + blockIdx.y) * a.dim + d] =
            (part[0][d] + part[1][d]) + (part[2][d] + part[3][d]);
}

// A block adds up 16 channels of a result row (a head's weight, or the shared
// one; the results are grid.x) over the parts of its chunks, in a fixed order:
// 64 threads a channel take every 64th part, then halves are added.  One block
// a result instead waited for each of its loads: whole calls of 32,768 rows, 9
// heads of 128, 196 us; so 60 us.
constexpr int kSumChannels = 16, kSumThreads = 64;
__global__ __launch_bounds__(kSumChannels *kSumThreads) void k_weight_grad(NormRopeArgs a, int per, int blocks,
                                                                            int chunks, int q_results) {
    const bool q = int(blockIdx.x) < q_results;
    const int cq = (a.q_heads + per - 1) / per;
    const int which = int(blockIdx.x) - (q ? 0 : q_results);
    const bool shared = (q ? a.q_weight_stride : a.k_weight_stride) == 0;
    const int c0 = (q ? 0 : cq) + (shared ? 0 : which), n = shared ? (q ? cq : chunks - cq) : 1;
    float *out = (q ? a.dq_weight : a.dk_weight);
    if (!out) return;
    __shared__ float part[kSumThreads][kSumChannels];
    const int x = threadIdx.x % kSumChannels, l = threadIdx.x / kSumChannels;
    const int d = int(blockIdx.y) * kSumChannels + x;  // dim is a multiple of 16
    float sum = 0.f;
    for (int c = 0; c < n; ++c) {
#pragma unroll 4
        for (int b = l; b < blocks; b += kSumThreads) sum += a.partial[(int64_t(b) * chunks + c0 + c) * a.dim + d];
    }
    part[l][x] = sum;
    for (int half = kSumThreads / 2; half > 0; half /= 2) {
        __syncthreads();
        if (l < half) part[l][x] += part[l + half][x];
    }
    if (l == 0) out[int64_t(which) * a.dim + d] = part[0][x];
}

struct Cut {
    int per, chunks, blocks;
};

int ceil_div(int a, int b) { return (a + b - 1) / b; }
int group_of(int dim) { return dim <= 16 ? 1 : dim <= 32 ? 2 : dim <= 64 ? 4 : 8; }

// Heads a chunk: all of a tensor's, fewer where the rows alone leave compute
// units without eight waves each.
Cut forward_cut(const NormRopeArgs &a) {
    Cut c;
    c.blocks = int(row_tiles(a.rows, 256 / group_of(a.dim)));
    c.per = std::max(std::max(a.q_heads, a.kv_heads), 1);
    auto chunks = [&](int per) {
        return ceil_div(a.q_heads, per) + ceil_div(a.kv_heads, per) * (a.v ? 2 : 1);
    };
    while (c.per > 1 && int64_t(c.blocks) * chunks(c.per) < 2 * compute_units()) c.per = (c.per + 1) / 2;
    c.chunks = chunks(c.per);
    return c;
}

Cut gradient_cut(const NormRopeArgs &a) {
    Cut c;
    const bool per_head = (a.dq_weight && a.q_weight_stride) || (a.dk_weight && a.k_weight_stride);
    c.blocks = int(row_tiles(a.rows, 256 / group_of(a.dim)));
    c.per = per_head ? 1 : std::max(std::max(a.q_heads, a.kv_heads), 1);
    auto chunks = [&](int per) { return ceil_div(a.q_heads, per) + ceil_div(a.kv_heads, per); };
    while (c.per > 1 && int64_t(c.blocks) * chunks(c.per) < 2 * compute_units()) c.per = (c.per + 1) / 2;
    c.chunks = chunks(c.per);
    // enough blocks to fill the device, few enough that their sums stay small
    c.blocks = std::max(1, std::min(c.blocks, ceil_div(8 * compute_units(), c.chunks)));
    return c;
}

template <typename T, int G>
hipError_t run(const NormRopeArgs &a, bool grad, const Cut &c, hipStream_t s) {
    const Fold f = fold(c.blocks, 256);  // the gradient's blocks are few
    const dim3 grid(f.x, c.chunks, f.z);
    if (grad) {
        if (a.interleaved) k_norm_rope_grad<T, G, true><<<grid, 256, 0, s>>>(a, c.per);
        else k_norm_rope_grad<T, G, false><<<grid, 256, 0, s>>>(a, c.per);
    } else {
        if (a.interleaved) k_norm_rope<T, G, true><<<grid, 256, 0, s>>>(a, c.per);
        else k_norm_rope<T, G, false><<<grid, 256, 0, s>>>(a, c.per);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t run(const NormRopeArgs &a, bool grad, const Cut &c, hipStream_t s) {
    switch (group_of(a.dim)) {
        case 1: return run<T, 1>(a, grad, c, s);
        case 2: return run<T, 2>(a, grad, c, s);
        case 4: return run<T, 4>(a, grad, c, s);
        default: return run<T, 8>(a, grad, c, s);
    }
}

}  // namespace

int norm_rope(const NormRopeArgs &a, void *stream) {
    const Cut c = forward_cut(a);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.bf16 ? run<uint16_t>(a, false, c, s) : run<float>(a, false, c, s);
}

size_t norm_rope_grad_workspace(const NormRopeArgs &a) {
    if (a.rows == 0 || !(a.dq_weight || a.dk_weight)) return 0;
    const Cut c = gradient_cut(a);
    return size_t(c.blocks) * c.chunks * a.dim * sizeof(float);
}

int norm_rope_grad(const NormRopeArgs &args, void *stream) {
    NormRopeArgs a = args;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool sums = a.dq_weight || a.dk_weight;
    if (!sums) a.partial = nullptr;
    Cut c = gradient_cut(a);
    if (a.rows > 0) {
        const hipError_t e = a.bf16 ? run<uint16_t>(a, true, c, s) : run<float>(a, true, c, s);
        if (e != hipSuccess) return e;
    } else {
        c.blocks = 0;  // the weights' gradients of no rows are zero
    }
    if (!sums) return hipSuccess;
    const int q_results = !a.q_heads ? 0 : a.q_weight_stride ? a.q_heads : 1;
    const int k_results = !a.kv_heads ? 0 : a.k_weight_stride ? a.kv_heads : 1;
    k_weight_grad<<<dim3(q_results + k_results, a.dim / kSumChannels), kSumChannels * kSumThreads, 0, s>>>(
        a, c.per, c.blocks, c.chunks, q_results);
    return hipGetLastError();
}

const char *launch_error(int e) { return hipGetErrorString(hipError_t(e)); }

}  // namespace kern
}  // namespace rtcc
