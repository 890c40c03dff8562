// Entry points of the token operators (rtcc_norm_rope, rtcc_attention and
// their gradients): argument checks and marshalling; the work is in
// kernels/norm_rope.hip, attention.hip and attention_grad.hip.
#include <cmath>
#include <string>

#include "../../include/rtcc.h"
#include "kernels/token_ops.hpp"

namespace rtcc {
void set_thread_error(const std::string &msg);
}

namespace {

constexpr int64_t kMaxRows = 2147483647;
// Of attention: a place up to a tile past the last row is still an int.
constexpr int64_t kMaxPlaces = 2147483648 - 256;
constexpr int64_t kMaxRowStride = rtcc::kern::kMaxRowStride, kMaxHeadStride = int64_t(1) << 40;
constexpr int32_t kMaxHeads = 1024, kMaxSeqs = 65536;

// First failed check of a call; empty while all hold.
struct Checks {
    std::string why;
    void need(bool ok, const char *msg) {
        if (!ok && why.empty()) why = msg;
    }
    void tensor(const void *p, const int64_t *stride, int64_t rows, int32_t heads, int32_t dim, int32_t elem,
                const char *name) {
        if (!why.empty() || rows == 0 || heads == 0) return;
        if (!p) {
            why = std::string(name) + " is NULL";
            return;
        }
        if (reinterpret_cast<uintptr_t>(p) % 16) why = std::string(name) + " is not 16-byte aligned";
        for (int i = 0; i < 2; ++i) {
            if ((i == 0 ? rows : int64_t(heads)) == 1) continue;  // a stride that is never taken
            if (stride[i] < dim || stride[i] > (i == 0 ? kMaxRowStride : kMaxHeadStride))
                why = std::string(name) + ": a stride is out of range";
            else if (stride[i] * elem % 16)
                why = std::string(name) + ": a stride breaks the 16-byte alignment of the heads";
        }
    }
};

rtcc_status fail(rtcc_status s, const std::string &msg) {
    // the message is best effort where memory is short
    try {
        rtcc::set_thread_error(msg);
    } catch (...) {
    }
    return s;
}

rtcc_status launched(int e, const char *what) {
    if (e == 0) return RTCC_OK;
    const char *text = rtcc::kern::launch_error(e);
    if (!text) return fail(RTCC_E_STATE, std::string(what) + " needs the GPU library");
    return fail(RTCC_E_HIP, std::string(what) + " failed: " + text);
}

// No C++ exception crosses the ABI.
template <class F>
rtcc_status guarded(F &&f) {
    try {
        return f();
    } catch (const std::bad_alloc &) {
        return RTCC_E_NOMEM;
    } catch (...) {
        return RTCC_E_INTERNAL;
    }
}

// A stride of an axis with one entry is never taken: any value will do.
void copy_stride(int64_t *to, const int64_t *from, int64_t rows, int32_t heads, int32_t dim) {
    to[0] = rows > 1 ? from[0] : dim;
    to[1] = heads > 1 ? from[1] : dim;
}

void check_common(Checks &c, int32_t abi_version, int32_t precision, int32_t head_dim) {
    c.need(abi_version == RTCC_ABI_VERSION, "abi_version mismatch");
    c.need(precision == RTCC_PREC_FP32 || precision == RTCC_PREC_BF16, "unknown precision");
    c.need(head_dim >= 16 && head_dim <= 128 && head_dim % 16 == 0, "head_dim must be a multiple of 16 in [16, 128]");
}

// The part of a norm_rope call that forward and gradient share.
Checks check_norm_rope(const rtcc_norm_rope_desc &d, rtcc::kern::NormRopeArgs &a) {
    Checks c;
    check_common(c, d.abi_version, d.precision, d.head_dim);
    c.need(d.rows >= 0 && d.rows <= kMaxRows, "rows out of range");
    c.need(d.q_heads >= 0 && d.q_heads <= kMaxHeads && d.kv_heads >= 0 && d.kv_heads <= kMaxHeads &&
               d.q_heads + d.kv_heads > 0,
           "q_heads and kv_heads must be in [0, 1024], not both 0");
    c.need(d.interleaved == 0 || d.interleaved == 1, "interleaved must be 0 or 1");
    c.need(d.n_axes >= 1 && d.n_axes <= RTCC_MAX_AXES, "n_axes must be in [1, 3]");
    c.need(std::isfinite(d.eps) && d.eps >= 0.f, "eps must be finite and >= 0");
    c.need((d.q_weight_per_head | 1) == 1 && (d.k_weight_per_head | 1) == 1, "a weight_per_head is not 0 or 1");
    if (!c.why.empty()) return c;
    int64_t pairs = 0;
    for (int i = 0; i < RTCC_MAX_AXES; ++i) {
        const int64_t s = i < d.n_axes ? d.sections[i] : 0;
        c.need(s >= 0 && s <= d.head_dim, "a section is out of range");
        pairs += s;
        a.section_end[i] = int32_t(pairs);
    }
    c.need(pairs <= d.head_dim / 2, "the sections hold more than head_dim / 2 pairs");
    if (!c.why.empty()) return c;
    const int32_t elem = d.precision == RTCC_PREC_BF16 ? 2 : 4;
    c.tensor(d.q, d.q_stride, d.rows, d.q_heads, d.head_dim, elem, "q");
    c.tensor(d.k, d.k_stride, d.rows, d.kv_heads, d.head_dim, elem, "k");
    if (d.rows > 0) {
        c.need(d.positions || pairs == 0, "positions is NULL");
        c.need(d.inv_freq || pairs == 0, "inv_freq is NULL");
    }
    a.bf16 = d.precision == RTCC_PREC_BF16;
    a.interleaved = d.interleaved != 0;
    a.rows = int32_t(d.rows);
    a.q_heads = d.q_heads;
    a.kv_heads = d.kv_heads;
    a.dim = d.head_dim;
    a.n_axes = d.n_axes;
    a.eps = d.eps;
    a.q = d.q;
    a.k = d.k;
    copy_stride(a.q_s, d.q_stride, d.rows, d.q_heads, d.head_dim);
    copy_stride(a.k_s, d.k_stride, d.rows, d.kv_heads, d.head_dim);
    a.q_weight = d.q_weight;
    a.k_weight = d.k_weight;
    // without a weight the flag says nothing: its gradient is one row
    a.q_weight_stride = d.q_weight && d.q_weight_per_head ? d.head_dim : 0;
    a.k_weight_stride = d.k_weight && d.k_weight_per_head ? d.head_dim : 0;
    a.positions = d.positions;
    a.inv_freq = d.inv_freq;
    return c;
}

Checks check_norm_rope_grad(const rtcc_norm_rope_grad_desc &d, rtcc::kern::NormRopeArgs &a) {
    Checks c = check_norm_rope(d.fwd, a);
    if (!c.why.empty()) return c;
    const rtcc_norm_rope_desc &f = d.fwd;
    const int32_t elem = f.precision == RTCC_PREC_BF16 ? 2 : 4;
    c.tensor(d.dq_out, d.dq_out_stride, f.rows, f.q_heads, f.head_dim, elem, "dq_out");
    c.tensor(d.dk_out, d.dk_out_stride, f.rows, f.kv_heads, f.head_dim, elem, "dk_out");
    c.tensor(d.dq, d.dq_stride, f.rows, f.q_heads, f.head_dim, elem, "dq");
    c.tensor(d.dk, d.dk_stride, f.rows, f.kv_heads, f.head_dim, elem, "dk");
    a.dq_out = d.dq_out;
    a.dk_out = d.dk_out;
    a.q_out = d.dq;
    a.k_out = d.dk;
    copy_stride(a.dqo_s, d.dq_out_stride, f.rows, f.q_heads, f.head_dim);
    copy_stride(a.dko_s, d.dk_out_stride, f.rows, f.kv_heads, f.head_dim);
    copy_stride(a.qo_s, d.dq_stride, f.rows, f.q_heads, f.head_dim);
    copy_stride(a.ko_s, d.dk_stride, f.rows, f.kv_heads, f.head_dim);
    a.dq_weight = f.q_heads ? d.dq_weight : nullptr;
    a.dk_weight = f.kv_heads ? d.dk_weight : nullptr;
    return c;
}

Checks check_attention(const rtcc_attn_desc &d, rtcc::kern::AttnArgs &a) {
    Checks c;
    check_common(c, d.abi_version, d.precision, d.head_dim);
    c.need(d.n_seqs >= 0 && d.n_seqs <= kMaxSeqs, "n_seqs must be in [0, 65536]");
    c.need(d.kv_heads >= 1 && d.kv_heads <= kMaxHeads && d.q_heads >= 1 && d.q_heads <= kMaxHeads,
           "q_heads and kv_heads must be in [1, 1024]");
    if (!c.why.empty()) return c;
    c.need(d.q_heads % d.kv_heads == 0, "q_heads must be a multiple of kv_heads");
    c.need(d.causal == 0 || d.causal == 1, "causal must be 0 or 1");
    c.need(std::isfinite(d.scale) && d.scale > 0.f, "scale must be finite and > 0");
    c.need(std::isfinite(d.softcap) && d.softcap >= 0.f, "softcap must be finite and >= 0");
    c.need(d.q_rows >= 0 && d.q_rows <= kMaxPlaces / d.q_heads, "q_rows * q_heads out of range");
    c.need(d.k_rows >= 0 && d.k_rows <= kMaxPlaces, "k_rows out of range");
    c.need(!d.prefix_lens || d.causal, "prefix_lens without causal");
    if (!c.why.empty()) return c;
    const int32_t elem = d.precision == RTCC_PREC_BF16 ? 2 : 4;
    if (d.n_seqs > 0) {
        c.need(d.q_offsets, "q_offsets is NULL");
        c.need(d.k_offsets, "k_offsets is NULL");
        c.tensor(d.q, d.q_stride, d.q_rows, d.q_heads, d.head_dim, elem, "q");
        c.tensor(d.k, d.k_stride, d.k_rows, d.kv_heads, d.head_dim, elem, "k");
        c.tensor(d.v, d.v_stride, d.k_rows, d.kv_heads, d.head_dim, elem, "v");
        c.tensor(d.out, d.out_stride, d.q_rows, d.q_heads, d.head_dim, elem, "out");
    }
    a.bf16 = d.precision == RTCC_PREC_BF16;
    a.causal = d.causal != 0;
    a.n_seqs = d.n_seqs;
    a.q_heads = d.q_heads;
    a.kv_heads = d.kv_heads;
    a.group = d.q_heads / d.kv_heads;
    a.dim = d.head_dim;
    a.q_rows = int32_t(d.q_rows);
    a.k_rows = int32_t(d.k_rows);
    a.scale = d.scale;
    a.softcap = d.softcap;
    a.q_offsets = d.q_offsets;
    a.k_offsets = d.k_offsets;
    a.k_lens = d.k_lens;
    a.prefix_lens = d.prefix_lens;
    a.slopes = d.slopes;
    a.q = d.q;
    a.k = d.k;
    a.v = d.v;
    a.out = d.out;
    a.lse = d.lse;
    copy_stride(a.q_s, d.q_stride, d.q_rows, d.q_heads, d.head_dim);
    copy_stride(a.k_s, d.k_stride, d.k_rows, d.kv_heads, d.head_dim);
    copy_stride(a.v_s, d.v_stride, d.k_rows, d.kv_heads, d.head_dim);
    copy_stride(a.o_s, d.out_stride, d.q_rows, d.q_heads, d.head_dim);
    return c;
}

Checks check_attention_grad(const rtcc_attn_grad_desc &d, rtcc::kern::AttnArgs &a) {
    Checks c = check_attention(d.fwd, a);
    if (!c.why.empty()) return c;
    const rtcc_attn_desc &f = d.fwd;
    if (f.n_seqs > 0) {
        const int32_t elem = f.precision == RTCC_PREC_BF16 ? 2 : 4;
        c.need(f.lse || f.q_rows == 0, "lse is NULL");
        c.need(f.k_rows * f.kv_heads < rtcc::kern::kMaxGradKeys, "k_rows * kv_heads out of range");
        c.tensor(d.dout, d.dout_stride, f.q_rows, f.q_heads, f.head_dim, elem, "dout");
        c.tensor(d.dq, d.dq_stride, f.q_rows, f.q_heads, f.head_dim, elem, "dq");
        c.tensor(d.dk, d.dk_stride, f.k_rows, f.kv_heads, f.head_dim, elem, "dk");
        c.tensor(d.dv, d.dv_stride, f.k_rows, f.kv_heads, f.head_dim, elem, "dv");
    }
    a.dout = d.dout;
    a.dq = d.dq;
    a.dk = d.dk;
    a.dv = d.dv;
    copy_stride(a.do_s, d.dout_stride, f.q_rows, f.q_heads, f.head_dim);
    copy_stride(a.dq_s, d.dq_stride, f.q_rows, f.q_heads, f.head_dim);
    copy_stride(a.dk_s, d.dk_stride, f.k_rows, f.kv_heads, f.head_dim);
    copy_stride(a.dv_s, d.dv_stride, f.k_rows, f.kv_heads, f.head_dim);
    return c;
}

bool workspace_ok(const void *workspace, size_t given, size_t needed) {
    return needed == 0 || (workspace && given >= needed && reinterpret_cast<uintptr_t>(workspace) % 16 == 0);
}

constexpr const char *kBadWorkspace = "the workspace is NULL, too small or not 16-byte aligned";

}  // namespace

extern "C" {

rtcc_status rtcc_norm_rope(const rtcc_norm_rope_desc *desc, void *hip_stream) {
    return guarded([&]() -> rtcc_status {
        if (!desc) return fail(RTCC_E_ARG, "desc is NULL");
        const rtcc_norm_rope_desc &d = *desc;
        rtcc::kern::NormRopeArgs a{};
        Checks c = check_norm_rope(d, a);
        if (c.why.empty()) {
            const int32_t elem = a.bf16 ? 2 : 4;
            c.need(!d.slots || (d.slot_rows >= 0 && d.slot_rows <= kMaxRows), "slot_rows out of range");
            c.need(!d.v || d.slots, "v without slots");
            c.tensor(d.q_out, d.q_out_stride, d.rows, d.q_heads, d.head_dim, elem, "q_out");
            const int64_t kv_rows = !d.slots ? d.rows : d.rows > 0 ? d.slot_rows : 0;
            c.tensor(d.k_out, d.k_out_stride, kv_rows, d.kv_heads, d.head_dim, elem, "k_out");
            if (d.v) {
                c.tensor(d.v, d.v_stride, d.rows, d.kv_heads, d.head_dim, elem, "v");
                c.tensor(d.v_out, d.v_out_stride, kv_rows, d.kv_heads, d.head_dim, elem, "v_out");
            }
            a.slot_rows = d.slot_rows;
            a.slots = d.slots;
            a.v = d.v;
            a.q_out = d.q_out;
            a.k_out = d.k_out;
            a.v_out = d.v_out;
            copy_stride(a.v_s, d.v_stride, d.rows, d.kv_heads, d.head_dim);
            copy_stride(a.qo_s, d.q_out_stride, d.rows, d.q_heads, d.head_dim);
            copy_stride(a.ko_s, d.k_out_stride, kv_rows, d.kv_heads, d.head_dim);
            copy_stride(a.vo_s, d.v_out_stride, kv_rows, d.kv_heads, d.head_dim);
        }
        if (!c.why.empty()) return fail(RTCC_E_ARG, c.why);
        if (d.rows == 0) return RTCC_OK;
        return launched(rtcc::kern::norm_rope(a, hip_stream), "rtcc_norm_rope");
    });
}

rtcc_status rtcc_norm_rope_grad_workspace(const rtcc_norm_rope_grad_desc *desc, size_t *bytes) {
    return guarded([&]() -> rtcc_status {
        if (!desc || !bytes) return fail(RTCC_E_ARG, "desc or bytes is NULL");
        *bytes = 0;
        rtcc::kern::NormRopeArgs a{};
        const Checks c = check_norm_rope_grad(*desc, a);
        if (!c.why.empty()) return fail(RTCC_E_ARG, c.why);
        *bytes = rtcc::kern::norm_rope_grad_workspace(a);
        return RTCC_OK;
    });
}

rtcc_status rtcc_norm_rope_grad(const rtcc_norm_rope_grad_desc *desc, void *workspace, size_t workspace_bytes,
                                void *hip_stream) {
    return guarded([&]() -> rtcc_status {
        if (!desc) return fail(RTCC_E_ARG, "desc is NULL");
        rtcc::kern::NormRopeArgs a{};
        const Checks c = check_norm_rope_grad(*desc, a);
        if (!c.why.empty()) return fail(RTCC_E_ARG, c.why);
        if (!workspace_ok(workspace, workspace_bytes, rtcc::kern::norm_rope_grad_workspace(a)))
            return fail(RTCC_E_ARG, kBadWorkspace);
        a.partial = static_cast<float *>(workspace);
        return launched(rtcc::kern::norm_rope_grad(a, hip_stream), "rtcc_norm_rope_grad");
    });
}

rtcc_status rtcc_attention_workspace(const rtcc_attn_desc *desc, size_t *bytes) {
    return guarded([&]() -> rtcc_status {
        if (!desc || !bytes) return fail(RTCC_E_ARG, "desc or bytes is NULL");
        *bytes = 0;
        rtcc::kern::AttnArgs a{};
        const Checks c = check_attention(*desc, a);
        if (!c.why.empty()) return fail(RTCC_E_ARG, c.why);
        *bytes = rtcc::kern::attention_workspace(a);
        return RTCC_OK;
    });
}

rtcc_status rtcc_attention(const rtcc_attn_desc *desc, void *workspace, size_t workspace_bytes, void *hip_stream) {
    return guarded([&]() -> rtcc_status {
        if (!desc) return fail(RTCC_E_ARG, "desc is NULL");
        rtcc::kern::AttnArgs a{};
        const Checks c = check_attention(*desc, a);
        if (!c.why.empty()) return fail(RTCC_E_ARG, c.why);
        if (!workspace_ok(workspace, workspace_bytes, rtcc::kern::attention_workspace(a)))
            return fail(RTCC_E_ARG, kBadWorkspace);
        a.workspace = workspace;
        if (a.n_seqs == 0 || a.q_rows == 0) return RTCC_OK;
        return launched(rtcc::kern::attention(a, hip_stream), "rtcc_attention");
    });
}

rtcc_status rtcc_attention_grad_workspace(const rtcc_attn_grad_desc *desc, size_t *bytes) {
    return guarded([&]() -> rtcc_status {
        if (!desc || !bytes) return fail(RTCC_E_ARG, "desc or bytes is NULL");
        *bytes = 0;
        rtcc::kern::AttnArgs a{};
        const Checks c = check_attention_grad(*desc, a);
        if (!c.why.empty()) return fail(RTCC_E_ARG, c.why);
        *bytes = rtcc::kern::attention_grad_workspace(a);
        return RTCC_OK;
    });
}

rtcc_status rtcc_attention_grad(const rtcc_attn_grad_desc *desc, void *workspace, size_t workspace_bytes,
                                void *hip_stream) {
    return guarded([&]() -> rtcc_status {
        if (!desc) return fail(RTCC_E_ARG, "desc is NULL");
        rtcc::kern::AttnArgs a{};
        const Checks c = check_attention_grad(*desc, a);
        if (!c.why.empty()) return fail(RTCC_E_ARG, c.why);
        if (!workspace_ok(workspace, workspace_bytes, rtcc::kern::attention_grad_workspace(a)))
            return fail(RTCC_E_ARG, kBadWorkspace);
        a.workspace = workspace;
        if (a.n_seqs == 0) return RTCC_OK;
        return launched(rtcc::kern::attention_grad(a, hip_stream), "rtcc_attention_grad");
    });
}

}  // extern "C"
