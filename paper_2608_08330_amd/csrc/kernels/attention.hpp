// Device code shared by the attention kernels (attention.hip,
// attention_grad.hip): matrix operands from LDS tiles, staging, sequences.
//
// All products run on 32 x 32 tiles with 16 contracted values a step.  Lane l
// holds row (or column) l % 32 of an operand and, with h = l / 32, the eight
// contracted values 8 h .. 8 h + 7 of the step; of a result it holds column
// l % 32 and, in register r, row 8 (r / 4) + 4 h + r % 4.  The scores of a
// tile are computed with the softmax's long axis on the rows, so each lane has
// 16 of its column's 32 scores in registers and the statistics are one
// register reduction and one exchange with lane l ^ 32.  The weights go into
// the next product from the registers they are in: registers 8 s .. 8 s + 7
// are the step s of an operand whose contracted order is 4 h + e (e < 4) and
// 8 + 4 h + e - 4 (e >= 4), and the other operand is read in that order.
// float32 uses the 2-value products of the same layout, eight to a step.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "token_ops.hpp"

namespace rtcc {
namespace kern {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
typedef __attribute__((address_space(3))) float lds_f32;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();

template <typename T>
struct Op;

template <>
struct Op<uint16_t> {
    typedef bf16x8_t Frag;
    static constexpr int kPerChunk = 8;  // elements of 16 bytes
    __device__ static f32x16_t mma(Frag a, Frag b, f32x16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    // eight float32 values as an operand, rounded to nearest even
    __device__ static Frag pack(const float *v) {
        Frag f;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __bf16(v[e]);
        return f;
    }
    __device__ static bool finite(Frag f, int e) {
        return (__builtin_bit_cast(uint16_t, __bf16(f[e])) & 0x7f80u) != 0x7f80u;
    }
    __device__ static float widen(Frag f, int e) { return float(f[e]); }
};

template <>
struct Op<float> {
    typedef f32x8_t Frag;
    static constexpr int kPerChunk = 4;
    __device__ static f32x16_t mma(Frag a, Frag b, f32x16_t c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    __device__ static Frag pack(const float *v) {
        Frag f;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = v[e];
        return f;
    }
    __device__ static bool finite(Frag f, int e) {
        return (__float_as_uint(f[e]) & 0x7f800000u) != 0x7f800000u;
    }
    __device__ static float widen(Frag f, int e) { return f[e]; }
};

// A tile in LDS: rows of D elements without padding (the direct loads write 16
// bytes a lane, lane after lane).  16-byte chunk c of row r is stored at c ^
// turn(r), so that both kinds of reads spread over the 64 banks: sixteen rows
// of one chunk (operand rows), and four neighbouring rows of 64 bytes
// (transposed reads).
template <typename T, int D>
struct Tile {
    static constexpr int kRowBytes = D * int(sizeof(T));
    static constexpr int kChunks = kRowBytes / 16;  // of a row: 4, 8, 16 or 32

    __device__ static constexpr uint32_t turn(uint32_t r) {
        if constexpr (kChunks == 4) return (r >> 2) & 3;
        else if constexpr (kChunks == 8) return ((r & 2) << 1) | ((r >> 2) & 3);
        else if constexpr (sizeof(T) == 2) return ((r & 3) << 2) | ((r >> 2) & 3);
        else return ((r & 4) << 1) | ((r & 3) << 1) | ((r >> 3) & 1);  // float32, 16 or 32 chunks
    }

    // Operand with rows of the tile as its rows: row `row` (the lane's),
    // values 16 kk + 8 h ..
    __device__ static typename Op<T>::Frag row_frag(uint32_t tile, uint32_t row, int kk, int h) {
        const uint32_t base = tile + row * kRowBytes, t = turn(row);
        if constexpr (sizeof(T) == 2) {
            const u32x4_t u = *(lds_u32x4 *)(base + (((2 * kk + h) ^ t) << 4));
            return __builtin_bit_cast(bf16x8_t, u);
        } else {
            const u32x4_t u0 = *(lds_u32x4 *)(base + (((4 * kk + 2 * h) ^ t) << 4));
            const u32x4_t u1 = *(lds_u32x4 *)(base + (((4 * kk + 2 * h + 1) ^ t) << 4));
            f32x8_t f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[e] = __uint_as_float(u0[e]);
                f[e + 4] = __uint_as_float(u1[e]);
            }
            return f;
        }
    }

    // Channels d .. d + 3 of row r, d a multiple of 4.
    __device__ static void four(uint32_t tile, uint32_t r, uint32_t d, float *v) {
        const uint32_t b = d * sizeof(T), at = tile + r * kRowBytes + (((b >> 4) ^ turn(r)) << 4) + (b & 15);
        if constexpr (sizeof(T) == 2) {
            const s16x4_t u = *(lds_s16x4 *)at;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(uint32_t(uint16_t(u[e])) << 16);
        } else {
            const u32x4_t u = *(lds_u32x4 *)at;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(u[e]);
        }
    }

    // Operand with columns 32 dt .. of the tile as its rows and tile rows as
    // the contracted values: rows 16 s + 4 h + e (e < 4), 16 s + 8 + 4 h + e - 4.
    __device__ static typename Op<T>::Frag col_frag(uint32_t tile, int s, int dt, int lane) {
        const int h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // a transposed read of 16 lanes: lane i gives row i / 4, columns
            // 4 (i % 4) ..; it receives column i of the four rows
            const uint32_t r = 4 * h + ((lane & 15) >> 2);
            const uint32_t c = dt * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
            const uint32_t at = tile + (16 * s + r) * kRowBytes + (lane & 1) * 8;
            const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + ((c ^ turn(r)) << 4)));
            const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s16x4 *)(at + 8 * kRowBytes + ((c ^ turn(r + 8)) << 4)));
            typedef short s16x8_t __attribute__((ext_vector_type(8)));
            const s16x8_t both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(bf16x8_t, both);
        } else {
            f32x8_t f;
            const uint32_t c = dt * 8 + ((lane & 31) >> 2);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t r = (e < 4 ? 0 : 8) + 4 * h + (e & 3);
                f[e] = *(lds_f32 *)(tile + (16 * s + r) * kRowBytes + ((c ^ turn(r)) << 4) + (lane & 3) * 4);
            }
            return f;
        }
    }
};

// Reads operands from tiles at constant LDS addresses: what depends on the lane
// is computed once, the rest of an address is a constant of the instruction.
template <typename T, int D>
struct Lanes {
    typedef Tile<T, D> L;
    int lane;
    uint32_t at;
    // first: LDS address of tile 0
    __device__ void init(int l, uint32_t first) {
        lane = l;
        at = first;
    }
    // Tile::row_frag of row 32 b + lane % 32, and Tile::col_frag
    __device__ typename Op<T>::Frag row_frag(uint32_t tile, int b, int kk) const {
        return L::row_frag(at + tile, b * 32 + (lane & 31), kk, lane >> 5);
    }
    __device__ typename Op<T>::Frag col_frag(uint32_t tile, int s, int t) const {
        return L::col_frag(at + tile, s, t, lane);
    }
    // To the other of two buffers, `bytes` (a power of two) apart.
    __device__ void flip(uint32_t bytes) { at ^= bytes; }
};

template <int D>
struct Lanes<uint16_t, D> {
    typedef Tile<uint16_t, D> L;
    uint32_t row[D / 16], col[D / 32][2];
    __device__ void init(int lane, uint32_t first) {
        const uint32_t h = lane >> 5, r = lane & 31, rc = 4 * h + ((lane & 15) >> 2);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
            row[kk] = opaque(first + r * L::kRowBytes + (((2 * kk + h) ^ L::turn(r)) << 4));
#pragma unroll
        for (int t = 0; t < D / 32; ++t) {
            const uint32_t c = t * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
            const uint32_t at = first + rc * L::kRowBytes + (lane & 1) * 8;
            col[t][0] = opaque(at + ((c ^ L::turn(rc)) << 4));
            col[t][1] = opaque(at + 8 * L::kRowBytes + ((c ^ L::turn(rc + 8)) << 4));
        }
    }
    __device__ bf16x8_t row_frag(uint32_t tile, int b, int kk) const {
        return __builtin_bit_cast(bf16x8_t, *(lds_u32x4 *)(row[kk] + (tile + b * 32 * L::kRowBytes)));
    }
    __device__ bf16x8_t col_frag(uint32_t tile, int s, int t) const {
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(col[t][0] + (tile + 16 * s * L::kRowBytes)));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(col[t][1] + (tile + 16 * s * L::kRowBytes)));
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    __device__ void flip(uint32_t bytes) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) row[kk] ^= bytes;
#pragma unroll
        for (int t = 0; t < D / 32; ++t) col[t][0] ^= bytes, col[t][1] ^= bytes;
    }
    // not to be computed again at its uses
    __device__ static uint32_t opaque(uint32_t x) {
        asm volatile("" : "+v"(x));
        return x;
    }
};

// Tile row of element e of a column operand's step s in half h.
__device__ inline int col_row(int s, int e, int h) { return 16 * s + (e < 4 ? 0 : 8) + 4 * h + (e & 3); }
// Tile row of result register r in half h.
__device__ inline int res_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

__device__ inline uint32_t lds_offset(const void *p) {
    return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void *)p));
}

// The value of the lane's column in the other half.
__device__ inline float other_half(float x, bool upper) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(upper ? r[0] : r[1]);
}
__device__ inline float half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Copies ROWS rows of one head from global memory into an LDS tile, straight
// (no registers): THREADS threads, 16 bytes each a load.  Rows past the end and
// channels past `dim` become zero: the hardware returns zero beyond the
// buffer's length, and channels of padding are given an offset beyond it.
template <typename T, int D, int ROWS, int THREADS>
struct Stager {
    typedef Tile<T, D> L;
    static constexpr int kLoads = ROWS * L::kChunks / THREADS;
    static_assert(kLoads >= 1 && ROWS * L::kChunks % THREADS == 0, "whole loads");
    static constexpr int kPass = THREADS / L::kChunks;  // rows of one load of all threads
    // Rows 16 apart are stored alike: then one offset serves all loads.
    static constexpr bool kOne = kPass % 16 == 0;
    static constexpr uint32_t kBytes = THREADS * 16;  // of one load of all threads
    uint32_t off[kOne ? 1 : kLoads];
    uint32_t row_bytes, head_bytes;

    // thread: 0 .. THREADS - 1
    __device__ void init(int thread, int64_t row_stride, int dim) {
        row_bytes = __builtin_amdgcn_readfirstlane(uint32_t(row_stride * sizeof(T)));
        head_bytes = uint32_t(dim * sizeof(T));
#pragma unroll
        for (int n = 0; n < (kOne ? 1 : kLoads); ++n) {
            const uint32_t id = uint32_t(n) * THREADS + thread, row = id / L::kChunks;
            const uint32_t c = (id % L::kChunks) ^ L::turn(row);
            off[n] = c * 16 < head_bytes ? row * row_bytes + c * 16 : 0x80000000u;
        }
    }
    // Of load n.  A tile's bytes stay below 2^31; offsets of padding stay past
    // that: 2^31 and at most ROWS - kPass rows more, in 32 bits.
    static constexpr int64_t kMaxRowBytes = kMaxRowStride * int64_t(sizeof(T));
    static_assert((ROWS - 1) * kMaxRowBytes + L::kRowBytes <= (int64_t(1) << 31), "a tile past 32-bit offsets");
    static_assert((int64_t(1) << 31) + (ROWS - kPass) * kMaxRowBytes < (int64_t(1) << 32), "padding wraps");
    __device__ uint32_t offset(int n) const { return kOne ? off[0] + uint32_t(n * kPass) * row_bytes : off[kOne ? 0 : n]; }
    // The wave's part of a tile.
    __device__ static uint32_t part(int thread) {
        return __builtin_amdgcn_readfirstlane(uint32_t(thread >> 6) * 1024u);
    }
    // rows: how many exist from `src` on (wave-uniform, as src and lds).  The
    // s_nop is the wait state that m0 needs before a load reads it; the
    // compiler adds none inside inline assembly.
    __device__ void load(const T *src, int rows, uint32_t lds, int thread) const {
        const uint64_t p = reinterpret_cast<uint64_t>(src);
        const uint32_t len = rows <= 0 ? 0u : uint32_t(min(rows, ROWS) - 1) * row_bytes + head_bytes;
        u32x4_t rsrc;
        rsrc[0] = __builtin_amdgcn_readfirstlane(uint32_t(p));
        rsrc[1] = __builtin_amdgcn_readfirstlane(uint32_t(p >> 32) & 0xffffu);
        rsrc[2] = __builtin_amdgcn_readfirstlane(len);
        rsrc[3] = 0x00020000u;
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds) + part(thread);
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset(n)), "s"(rsrc),
                         "s"(at + uint32_t(n) * kBytes)
                         : "memory", "m0");
        }
    }
};

// A Stager's tiles one after another, all of them whole: the scalar work of a
// tile is one addition.
template <typename S, int ROWS>
struct Walk {
    u32x4_t rsrc;
    uint64_t step;
    uint32_t at;  // the wave's part of a tile at the block's first LDS address
    template <typename T>
    __device__ void init(const S &s, const T *src, int thread, uint32_t first) {
        const uint64_t p = reinterpret_cast<uint64_t>(src);
        rsrc[0] = __builtin_amdgcn_readfirstlane(uint32_t(p));
        rsrc[1] = __builtin_amdgcn_readfirstlane(uint32_t(p >> 32) & 0xffffu);
        rsrc[2] = __builtin_amdgcn_readfirstlane(uint32_t(ROWS - 1) * s.row_bytes + s.head_bytes);
        rsrc[3] = 0x00020000u;
        const uint64_t bytes = uint64_t(ROWS) * s.row_bytes;
        step = uint64_t(__builtin_amdgcn_readfirstlane(uint32_t(bytes >> 32))) << 32 |
               __builtin_amdgcn_readfirstlane(uint32_t(bytes));
        at = __builtin_amdgcn_readfirstlane(first) + S::part(thread);
    }
    // The next tile, to the address TO past the first (s_nop: as in Stager).
    template <uint32_t TO>
    __device__ void load(const S &s) {
#pragma unroll
        for (int n = 0; n < S::kLoads; ++n) {
            asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(s.offset(n)), "s"(rsrc),
                         "s"(at), "i"(TO + uint32_t(n) * S::kBytes)
                         : "memory", "m0", "scc");
        }
        const uint64_t p = (uint64_t(rsrc[1]) << 32 | rsrc[0]) + step;
        rsrc[0] = uint32_t(p);
        rsrc[1] = uint32_t(p >> 32);
    }
};

// All direct loads of this wave have arrived.
__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
template <int N>
__device__ inline void wait_loads_but() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Registers loaded from global memory have arrived.  Said to the compiler: it
// cannot count the direct loads, and a register load that it still takes to be
// on its way where a loop begins costs a wait for all of them in every turn.
__device__ inline void wait_registers() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // vmcnt(0) alone
// This wave's reads of a tile are done: direct loads may write over it.
__device__ inline void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ inline void barrier() {
    wait_reads();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// One sequence, clamped to the buffers.
struct Seq {
    int s, q0, nq, k0, nk, prefix, tile;
};

__device__ inline int clamp_to(int x, int lo, int hi) { return min(max(x, lo), hi); }

__device__ inline void q_range(const AttnArgs &a, int s, int &q0, int &nq) {
    q0 = clamp_to(a.q_offsets[s], 0, a.q_rows);
    nq = clamp_to(a.q_offsets[s + 1], q0, a.q_rows) - q0;
}
__device__ inline void k_range(const AttnArgs &a, int s, int &k0, int &nk) {
    k0 = clamp_to(a.k_offsets[s], 0, a.k_rows);
    const int64_t end = a.k_lens ? int64_t(k0) + max(a.k_lens[s], 0) : int64_t(a.k_offsets[s + 1]);
    nk = int(min(max(end, int64_t(k0)), int64_t(a.k_rows))) - k0;
}

__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Sequence and tile within it of tile `t` of the batch, a tile being `per`
// units: columns (queries x heads of a group) with KEYS = false, keys with
// KEYS = true.  False past the last tile.  Every wave of a block gets the same
// answer, in scalar registers.  Sums of 64 sequences' tiles (of at least 64
// units where there are many) reach 2^31 at most, where lists overlap.
template <bool KEYS>
__device__ inline bool find_tile(const AttnArgs &a, int tile, int per, Seq &q) {
    const int lane = threadIdx.x & 63;
    uint32_t t = tile;  // less the tiles of the sequences looked at
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
        const int s = s0 + lane;
        uint32_t n = 0;
        if (s < a.n_seqs) {
            int from, len;
            if constexpr (KEYS) k_range(a, s, from, len);
            else q_range(a, s, from, len);
            const int64_t units = KEYS ? len : int64_t(len) * a.group;
            n = uint32_t((units + per - 1) / per);
        }
        uint32_t sum = n;  // inclusive over the lanes
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t up = __shfl_up(sum, d);
            if (lane >= d) sum += up;
        }
        const uint32_t total = __builtin_amdgcn_readlane(sum, 63);
        if (t < total) {
            const unsigned long long past = __ballot(sum > t);
            const int at = __builtin_ctzll(past);
            q.s = s0 + at;
            q.tile = int(t - (at ? uint32_t(__builtin_amdgcn_readlane(sum, at - 1)) : 0u));
            q.s = uniform(q.s);
            q.tile = uniform(q.tile);
            q_range(a, q.s, q.q0, q.nq);
            k_range(a, q.s, q.k0, q.nk);
            q.prefix = a.prefix_lens ? clamp_to(a.prefix_lens[q.s], 0, q.nk) : 0;
            q.q0 = uniform(q.q0);
            q.nq = uniform(q.nq);
            q.k0 = uniform(q.k0);
            q.nk = uniform(q.nk);
            q.prefix = uniform(q.prefix);
            return true;
        }
        t -= total;
    }
    return false;
}

// Keys that query i of a sequence sees: [0, limit).  Does not fall with i.
__device__ inline int limit_of(const AttnArgs &a, const Seq &q, int i) {
    return a.causal ? clamp_to(q.nk - q.nq + i + 1, q.prefix, q.nk) : q.nk;
}

// Products of a tile's columns with weights: acc[t] += tile[:, 32 t ..]^T w, the
// weights of 16 tile rows a step.  A weight of 0 times a value that is not
// finite would still reach the sum; with `look` (where MASK allows it), rows
// that hold such values are taken one by one, for the lanes (columns of the
// result) that see them.
template <typename T, int D, int STEPS, bool MASK>
struct Product {
    typedef Op<T> M;
    typedef Tile<T, D> L;

    template <typename SEEN>
    __device__ static void add(f32x16_t *acc, const typename M::Frag *w, uint32_t tile, int lane, bool look,
                               const SEEN &seen) {
        if (MASK && look) {
            const unsigned long long bad = not_finite(tile, lane);
            if (bad) {
                apart(acc, w, tile, lane, bad, seen);
                return;
            }
        }
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int s = 0; s < STEPS; ++s) acc[t] = M::mma(L::col_frag(tile, s, t, lane), w[s], acc[t]);
    }

    // Rows of the tile that hold an infinity or a NaN, as a bit each.
    __device__ static unsigned long long not_finite(uint32_t tile, int lane) {
        bool bad = false;
        if (lane < 16 * STEPS) {
#pragma unroll 1
            for (int c = 0; c < L::kChunks; ++c) {
                const u32x4_t u = *(lds_u32x4 *)(tile + lane * L::kRowBytes + c * 16);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    bad |= (u[w] & 0x7f800000u) == 0x7f800000u;
                    if constexpr (sizeof(T) == 2) bad |= (u[w] & 0x7f80u) == 0x7f80u;
                }
            }
        }
        return __ballot(bad);
    }

    template <typename SEEN>
    __device__ static void apart(f32x16_t *acc, const typename M::Frag *w, uint32_t tile, int lane,
                                 unsigned long long bad, const SEEN &seen) {
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
                acc[t] = M::mma(only(L::col_frag(tile, s, t, lane), s, lane, ~bad), w[s], acc[t]);
#pragma unroll 1
        for (; bad; bad &= bad - 1) {
            const int j = __builtin_ctzll(bad), h = lane >> 5;
            const float f = weight(w, j, h);
            const bool see = seen(j);
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float v[4];
                    L::four(tile, j, 32 * t + 8 * g + 4 * h, v);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][4 * g + e] = see ? fmaf(f, v[e], acc[t][4 * g + e]) : acc[t][4 * g + e];
                }
        }
    }
    // The weight of tile row j in the lane's column.
    __device__ static float weight(const typename M::Frag *w, int j, int h) {
        const int step = j >> 4, place = (j >> 3 & 1) * 4 + (j & 3);
        float f = 0.f;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (s == step && e == place) f = M::widen(w[s], e);
        const float other = other_half(f, h != 0);
        return (j >> 2 & 1) == h ? f : other;
    }
    __device__ static typename M::Frag only(typename M::Frag f, int s, int lane, unsigned long long keep) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!(keep >> col_row(s, e, lane >> 5) & 1)) f[e] = 0;
        return f;
    }
};

// A lane's part of a row as operands: row `src`, channels 16 kk + 8 h .., zero
// past `dim`.
template <typename T, int D>
__device__ inline void load_row(const T *src, int dim, int h, typename Op<T>::Frag *f) {
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
        f[kk] = typename Op<T>::Frag{};
        if (kk * 16 < dim) {
            const u32x4_t *p = reinterpret_cast<const u32x4_t *>(src + kk * 16 + h * 8);
            if constexpr (sizeof(T) == 2) {
                f[kk] = __builtin_bit_cast(bf16x8_t, p[0]);
            } else {
                const u32x4_t u0 = p[0], u1 = p[1];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f[kk][e] = __uint_as_float(u0[e]);
                    f[kk][e + 4] = __uint_as_float(u1[e]);
                }
            }
        }
    }
}

// Stores a lane's column of transposed results (32 t + 8 g + 4 h .. of a row).
template <typename T, int D>
__device__ inline void store_column(T *dst, int dim, int h, const f32x16_t *acc, float f) {
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * t + 8 * g + 4 * h;
            if (d >= dim) continue;
            if constexpr (sizeof(T) == 2) {
                typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
                bf16x4_t v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __bf16(acc[t][4 * g + e] * f);
                *reinterpret_cast<bf16x4_t *>(dst + d) = v;
            } else {
                *reinterpret_cast<float4 *>(dst + d) = make_float4(acc[t][4 * g] * f, acc[t][4 * g + 1] * f,
                                                                   acc[t][4 * g + 2] * f, acc[t][4 * g + 3] * f);
            }
        }
}

// A lane's column of a tile of columns: query i of head `head`.
struct Column {
    int i, row, head;
    bool valid;
    // c0: the wave's first; the last column stands in for those past it
    __device__ void init(const AttnArgs &a, const Seq &sq, int kvh, int64_t c0) {
        const uint32_t n = uint32_t(sq.nq) * uint32_t(a.group);
        const uint32_t c = uint32_t(c0) + (threadIdx.x & 31);
        valid = c < n;
        const uint32_t cc = valid ? c : n - 1;
        const uint32_t q = a.group == 1 ? cc : cc / uint32_t(a.group);
        i = int(q);
        row = sq.q0 + i;
        head = kvh * a.group + int(cc - q * a.group);
    }
};

// The cap's forms.  kShort: cap tanh(y) as cap - 2 cap / (exp2(2 y log2 e) + 1),
// whose error is 2^-22 of the cap wherever the score lies.  kExact: the same
// from |y| = 0.63 on and y P(y^2) below, 3 roundings of the score itself; P is
// tanh(y) / y fitted to 1.1e-8 (float32 coefficients).  bf16 keeps to the short
// form up to caps of kShortCap: 2^-16 of a weight, where the weight's own
// rounding is 2^-9.  The exact form takes 13 more vector operations a score in
// loops that those bound: 8,192 causal tokens, 6 heads of 128, 183 us in the
// short form and 218 us in the exact one; forward and gradients of four
// histories of up to 4,096 tokens, 6 heads of 64, 405 and 523 us.
enum Cap { kNone, kShort, kExact };
constexpr float kShortCap = 64.f;

// What turns a product <q, k> into a score in units of log 2.
//   plain:  x * c1
//   capped: cap tanh(y) with y = x scale / cap = x c3, 2 y log2 e = x c2
// and the distance bias, slope * |p - j|.
struct Score {
    float c1, c2, c3, capl;
    __device__ void init(const AttnArgs &a) {
        // factors past float32's range would make NaN of products of 0 or
        // infinity: the tanh is its argument or +-1 there
        constexpr float kLow = 1.17549435e-38f, kHigh = 3.40282347e38f;
        c1 = a.scale * kLog2e;
        c2 = fminf(fmaxf(2.f * kLog2e * a.scale / a.softcap, kLow), kHigh);
        c3 = fminf(fmaxf(a.scale / a.softcap, kLow), kHigh);
        capl = fminf(a.softcap * kLog2e, kHigh);
    }
    // The capped score; th: its tanh, in [-1, 1].
    template <Cap CAP>
    __device__ float capped(float x, float &th) const {
        th = fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * c2) + 1.f), 1.f);
        if constexpr (CAP == kShort) return capl * th;
        const float y = x * c3, t = y * y;
        float p = fmaf(t, -5.6482954e-3f, 2.0589806e-2f);
        p = fmaf(t, p, -5.3725120e-2f);
        p = fmaf(t, p, 1.33312747e-1f);
        p = fmaf(t, p, -3.33332747e-1f);
        p = fmaf(t, p, 1.f);
        const bool near = t < 0.4f;
        th = near ? y * p : th;
        return near ? x * c1 * p : capl * th;
    }
};

// Block b (counted over x and z, see fold) takes tile b / kv_heads of key head b % kv_heads: the heads' longest
// tiles start first, and every XCD (block b runs on XCD b % 8) gets tiles of
// all lengths.  Runs of one head's tiles on one XCD, for its L2, were slower by
// 11% (16,384 tokens, 6 heads of 64) to 33% (8,192 tokens, causal, 6 heads of
// 128): the XCDs' shares of a causal batch differ, and a head's keys and values
// of these sizes are near in the shared cache anyway.
__device__ inline int block() { return int(blockIdx.z * gridDim.x + blockIdx.x); }
__device__ inline int tile_of(const AttnArgs &a) { return block() / a.kv_heads; }
__device__ inline int head_of(const AttnArgs &a) { return block() % a.kv_heads; }

// The tile width of a head: its channels are padded with zeros to this.
inline int padded(int dim) { return dim <= 32 ? 32 : dim <= 64 ? 64 : 128; }

// Calls f with the score's terms of a call as constants: Cap and whether there
// is a distance bias.
template <typename T, typename F>
inline hipError_t with_terms(const AttnArgs &a, const F &f) {
    auto with = [&](auto cap) { return a.slopes ? f(cap, std::true_type()) : f(cap, std::false_type()); };
    if (a.softcap == 0.f) return with(std::integral_constant<Cap, kNone>());
    if constexpr (sizeof(T) == 2) {
        if (a.softcap <= kShortCap) return with(std::integral_constant<Cap, kShort>());
    }
    return with(std::integral_constant<Cap, kExact>());
}

template <typename F>
inline hipError_t max_lds(F kernel, int bytes) {
    return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

}  // namespace
}  // namespace kern
}  // namespace rtcc
