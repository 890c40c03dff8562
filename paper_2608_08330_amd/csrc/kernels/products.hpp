// Device code of the matrix products of gated_ffn.hip: panels of an operand
// staged in LDS straight from global memory, and fragments read from them.
//
// A step of the contracted axis is 128 bytes: 64 bf16 or 32 float32 values.  A panel
// holds ROWS rows (or columns) of one operand over such a step.  Two layouts, by how
// the operand lies in memory:
//   K contiguous: [ROWS][step]; the panel's rows are the operand's
//   K in rows:    [step][ROWS]; fragments are read transposed
// Lane l has fr = l % 16 and fk = l / 16; a fragment is the lane's 16 bytes of
// row fr: contracted values 8 fk .. 8 fk + 7 of 32 (bf16) or 4 fk .. 4 fk + 3 of
// 16 (float32).  Results: the operands are given to the instruction in turned
// order, so a lane holds four neighbouring columns 4 fk .. of row fr.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "token_ops.hpp"

namespace rtcc {
namespace kern {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
typedef __attribute__((address_space(3))) float lds_f32;

// Steps of a product of two fragments, and one of them: c += a . b.  The float32
// instruction takes one value of a lane's four; neighbouring instructions of a step
// are better of different results (they need not wait for each other).
template <typename T>
constexpr int kMmaSteps = sizeof(T) == 2 ? 1 : 4;
__device__ inline f32x4_t mma(uint16_t, int, u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0,
                                                   0);
}
__device__ inline f32x4_t mma(float, int e, u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
}

// Eight neighbouring values of a row.
__device__ inline void store8(uint16_t *p, const float *v) {
    bf16x8_t b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = __bf16(v[e]);
    *reinterpret_cast<bf16x8_t *>(p) = b;
}
__device__ inline void store8(float *p, const float *v) {
    f32x4_t a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = v[e], b[e] = v[e + 4];
    reinterpret_cast<f32x4_t *>(p)[0] = a;
    reinterpret_cast<f32x4_t *>(p)[1] = b;
}
// As they lie in memory, so that many loads fit the registers before any is used.
template <typename T>
struct Eight {
    u32x4_t raw[sizeof(T) / 2];
    __device__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < int(sizeof(T) / 2); ++i) raw[i] = reinterpret_cast<const u32x4_t *>(p)[i];
    }
    __device__ float operator[](int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(raw[e / 4][e % 4]);
        else return __uint_as_float(e & 1 ? raw[0][e / 2] & 0xffff0000u : raw[0][e / 2] << 16);
    }
};
// Four of them.
__device__ inline void store4(uint16_t *p, f32x4_t v) {
    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
    bf16x4_t b;
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = __bf16(v[e]);
    *reinterpret_cast<bf16x4_t *>(p) = b;
}
__device__ inline void store4(float *p, f32x4_t v) { *reinterpret_cast<f32x4_t *>(p) = v; }
// Two results side by side, x and y, as eight neighbouring columns a lane: of x
// where fk is even and of y where it is odd, from column 8 (fk / 2) on.
__device__ inline void pair_up(f32x4_t x, f32x4_t y, float *v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[e]), __float_as_uint(y[e]), false, false);
        v[e] = __uint_as_float(r[0]);
        v[e + 4] = __uint_as_float(r[1]);
    }
}

// The 16-byte chunk c of row r of a panel is stored at c ^ turn(r), so that the
// lanes of a read spread over the 64 banks.
template <typename T, bool KC, int ROWS>
struct Panel {
    static constexpr int kStep = 128 / int(sizeof(T));
    static constexpr int kBytes = ROWS * 128;
    static constexpr int kLine = KC ? 128 : ROWS * int(sizeof(T));  // bytes of a panel's row
    static constexpr int kChunks = kLine / 16;
    static constexpr int kLines = KC ? ROWS : kStep;

    __device__ static constexpr uint32_t turn(uint32_t r) {
        if constexpr (KC) return (r >> 1) & 7;  // 16 rows of one chunk
        // transposed: four neighbouring rows, and those 8 further, of 32 bytes
        else if constexpr (sizeof(T) == 2)
            return 2 * (kLine >= 256 ? (r & 3) | ((r >> 1) & 4) : kLine == 128 ? ((r >> 1) & 1) | ((r >> 2) & 2) : (r >> 3) & 1);
        // four rows, 4 apart, of 64 bytes
        else return 4 * ((r >> 2) & (kLine >= 256 ? 3 : 1));
    }

    // Lane constants of the fragments of N tiles of 16 rows, from row `first`.
    template <int N>
    struct Lanes {
        uint32_t at[KC ? 2 : N];
        __device__ void init(int lane, uint32_t lds, int first) {
            const uint32_t fr = lane & 15, fk = lane >> 4;
            if constexpr (KC) {
#pragma unroll
                for (uint32_t s = 0; s < 2; ++s) at[s] = lds + (first + fr) * 128 + (((4 * s + fk) ^ turn(fr)) << 4);
            } else if constexpr (sizeof(T) == 2) {
                // a transposed read of 16 lanes: lane i gives row i / 4, columns
                // 4 (i % 4) ..; it receives column i of the four rows
                const uint32_t k = 8 * fk + (fr >> 2);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const uint32_t c = (first / 16 + n) * 2 + ((fr & 3) >> 1);
                    at[n] = lds + k * kLine + ((c ^ turn(k)) << 4) + (fr & 1) * 8;
                }
            } else {
                const uint32_t k = 4 * fk;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const uint32_t c = (first / 16 + n) * 4 + (fr >> 2);
                    at[n] = lds + k * kLine + ((c ^ turn(k)) << 4) + (fr & 3) * 4;
                }
            }
        }
        // Tile n, half s of the contracted values, of a panel `to` bytes further.
        __device__ u32x4_t frag(int n, int s, uint32_t to) const {
            if constexpr (KC) {
                return *(lds_u32x4 *)(at[s] + (to + n * 16 * 128));
            } else if constexpr (sizeof(T) == 2) {
                const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at[n] + (to + 32 * s * kLine)));
                const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at[n] + (to + (32 * s + 4) * kLine)));
                return __builtin_bit_cast(u32x4_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            } else {
                u32x4_t f;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    f[e] = __float_as_uint(*(lds_f32 *)(at[n] + (to + (16 * s + e) * kLine)));
                return f;
            }
        }
    };

    // Fills the panel with THREADS threads, 16 bytes each a load, step after step.
    // What lies past the operand becomes zero: the hardware returns zero beyond the
    // buffer's length, and lanes past the end of a line get an offset beyond it.
    // The state but off and chunk is wave-uniform; a step costs a few scalar
    // instructions a panel.
    template <int THREADS>
    struct Feed {
        static constexpr int kLoads = kLines * kChunks / THREADS;
        static_assert(kLoads >= 1 && kLines * kChunks % THREADS == 0, "whole loads");
        static constexpr int kPass = THREADS / kChunks;  // lines of one load of all threads
        // Lines kPass apart are stored alike: one offset serves all loads.
        static constexpr bool kOne = turn(kPass) == 0 && turn(2 * kPass) == 0 && turn(4 * kPass) == 0;
        static_assert(kLoads <= 8, "turns of the passes");
        static constexpr int64_t kMaxRowBytes = kMaxRowStride * int64_t(sizeof(T));
        static_assert((kLines - 1) * kMaxRowBytes + kLine <= (int64_t(1) << 31), "a panel past 32-bit offsets");
        static_assert((int64_t(1) << 31) + (kLines - kPass) * kMaxRowBytes < (int64_t(1) << 32), "padding wraps");
        static constexpr uint32_t kBeyond = 0x80000000u;
        uint32_t off[kOne ? 1 : kLoads], chunk;
        uint64_t at, ahead;  // the next step's first byte, and from step to step
        uint32_t row, size;  // bytes between rows; K contiguous: of all rows but the last, else: of a line

        // base: the operand.  row_bytes: between its rows.  first: the panel's first
        // row (K in rows: column).  rows: how many exist from there on, any number.
        // step: the first one.
        __device__ void init(int thread, const char *base, uint32_t row_bytes, int64_t first, int rows, int64_t step) {
            row = row_bytes;
            const int here = max(0, min(rows, ROWS));
            if constexpr (KC) {
                at = reinterpret_cast<uint64_t>(base) + first * row + step * 128;
                ahead = 128;
                size = here ? uint32_t(here - 1) * row : 0u;
            } else {
                at = reinterpret_cast<uint64_t>(base) + first * int(sizeof(T)) + step * kStep * row;
                ahead = uint64_t(kStep) * row;
                size = uint32_t(here) * uint32_t(sizeof(T));
            }
#pragma unroll
            for (int n = 0; n < (kOne ? 1 : kLoads); ++n) {
                const uint32_t id = uint32_t(n) * THREADS + thread, line = id / kChunks;
                const uint32_t c = ((id % kChunks) ^ turn(line)) * 16;
                off[n] = (KC ? here > 0 : c < size) ? line * row + c : kBeyond;
                if (n == 0) chunk = c;
            }
        }
        // The step's buffer descriptor; k: its contracted values, 0 .. kStep (none:
        // zeros are stored).  To the next step.
        __device__ u32x4_t next(int k) {
            u32x4_t rsrc;
            rsrc[0] = uint32_t(at);
            rsrc[1] = uint32_t(at >> 32);  // an address has 48 bits: the others, the stride, are zero
            // said to be uniform here: where offsets use them too, the compiler keeps
            // them in vector registers, which a descriptor cannot be in
            const uint32_t z = __builtin_amdgcn_readfirstlane(size), r = __builtin_amdgcn_readfirstlane(row);
            k = __builtin_amdgcn_readfirstlane(k);
            rsrc[2] = KC ? z + uint32_t(k) * uint32_t(sizeof(T)) : uint32_t(max(0, k * int(r) - int(r - z)));
            rsrc[3] = 0x00020000u;
            at += ahead;
            return rsrc;
        }
        // Load n of the step.  lds: the panel, the wave's part of it.  The s_nop is
        // the wait state that m0 needs before a load reads it; the compiler adds
        // none inside inline assembly.
        __device__ void load(int n, u32x4_t rsrc, int k, uint32_t lds) const {
            uint32_t o = kOne ? off[0] + uint32_t(n * kPass) * row : off[kOne ? 0 : n];
            if constexpr (KC) o = int(chunk) < k * int(sizeof(T)) ? o : kBeyond;
            asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(o), "s"(rsrc),
                         "s"(lds + uint32_t(n * THREADS * 16))
                         : "memory", "m0");
        }
    };
};

// Contracted values of the steps of one slice, as the loads go through them.
struct Steps {
    int left, more;  // values of the segment from the next step on; steps of the slice from there on
    template <int STEP>
    __device__ int next() {
        const int k = more > 0 ? min(left, STEP) : 0;
        left -= STEP;
        --more;
        return k;
    }
};

__device__ inline uint32_t lds_offset(const void *p) {
    return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void *)p));
}

}  // namespace
}  // namespace kern
}  // namespace rtcc
