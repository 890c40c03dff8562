// Arguments and launchers of the token operators (norm_rope.hip,
// attention.hip, attention_grad.hip).  Host code only, free of HIP headers so
// that the argument checks build into the host test library, which has
// launchers of its own that refuse.  A launcher checks nothing: token_ops.cpp
// has validated the descriptor.  Return value: a hipError_t as int.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace rtcc {
namespace kern {

struct NormRopeArgs {
    bool bf16, interleaved;
    int32_t rows, q_heads, kv_heads, dim, n_axes;
    int32_t section_end[3];  // pairs before the end of each axis' section
    float eps;
    int64_t slot_rows;
    // forward: x -> y (and v copied); gradient: x and dy -> dx
    const void *q, *k, *v;
    const void *dq_out, *dk_out;
    void *q_out, *k_out, *v_out;
    int64_t q_s[2], k_s[2], v_s[2], qo_s[2], ko_s[2], vo_s[2], dqo_s[2], dko_s[2];
    const float *q_weight, *k_weight;
    int32_t q_weight_stride, k_weight_stride;  // head_dim or 0
    const float *positions, *inv_freq;
    const int64_t *slots;
    float *dq_weight, *dk_weight;
    float *partial;  // gradient: [blocks][chunks][dim] sums
};

struct AttnArgs {
    bool bf16, causal;
    int32_t n_seqs, q_heads, kv_heads, group, dim;
    int32_t q_rows, k_rows;
    float scale, softcap;
    const int32_t *q_offsets, *k_offsets, *k_lens, *prefix_lens;
    const float *slopes;
    const void *q, *k, *v;
    void *out;
    float *lse;
    int64_t q_s[2], k_s[2], v_s[2], o_s[2];
    // gradient
    const void *dout;
    void *dq, *dk, *dv;
    int64_t do_s[2], dq_s[2], dk_s[2], dv_s[2];
    void *workspace;
};

// Blocks of a launch, of which a kernel counts blockIdx.z * gridDim.x +
// blockIdx.x: HIP takes fewer than 2^32 threads an axis.  The description's
// limits keep every number of blocks below 2^31.
struct Fold {
    uint32_t x, z;
};
inline Fold fold(int64_t blocks, int threads) {
    const int64_t most = ((int64_t(1) << 32) - 1) / threads, z = std::max<int64_t>(1, (blocks + most - 1) / most);
    return {uint32_t((blocks + z - 1) / z), uint32_t(z)};
}
// Tiles of `per` rows.
inline int64_t row_tiles(int64_t rows, int per) { return (rows + per - 1) / per; }
// Tiles of `per` columns (queries x heads of a group) or keys, for all key
// heads: at least the sum over the sequences of their rounded tiles.
inline int64_t column_blocks(const AttnArgs &a, int per) {
    return (int64_t(a.q_rows) * a.group / per + a.n_seqs) * a.kv_heads;
}
inline int64_t key_blocks(const AttnArgs &a, int per) {
    return (int64_t(a.k_rows) / per + a.n_seqs) * a.kv_heads;
}
// Between rows: up to 128 rows of a tile lie within 32-bit offsets of its first
// (attention.hpp checks this).
constexpr int64_t kMaxRowStride = int64_t(1) << 22;
// Of the gradient's smallest tiles of a long batch (64 keys): 2^29 + 2^26 blocks.
constexpr int64_t kMaxGradKeys = int64_t(1) << 35;  // k_rows * kv_heads

size_t norm_rope_grad_workspace(const NormRopeArgs &a);
int norm_rope(const NormRopeArgs &a, void *stream);
int norm_rope_grad(const NormRopeArgs &a, void *stream);
size_t attention_workspace(const AttnArgs &a);
int attention(const AttnArgs &a, void *stream);
size_t attention_grad_workspace(const AttnArgs &a);
int attention_grad(const AttnArgs &a, void *stream);
// Text of a launcher's error; null from the host test library's launchers.
const char *launch_error(int e);

}  // namespace kern
}  // namespace rtcc
