"""GPU token operators at the edges of their descriptions: buffers of exactly
the stated size, sizes and places near the limits, caps of every size.

Tolerances as in test_gpu_tokens.py: U and B are one rounding to float32 and
bf16; each test says what it adds."""

import numpy as np
import pytest

from oracle import tokens as T
from paper_2608_08330_amd import rtcc as R
from tests.test_gpu_tokens import B, PRECISIONS, U, Case, Rope, _f64, _workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("precision", PRECISIONS)
def test_gradient_of_an_absent_weight_is_one_row(precision):
    """Without a weight its gradient has head_dim values, whatever the flag for
    weights of every head says: what lies behind them is not written."""
    import torch
    rows, heads, dim = 90, (5, 3), 48
    c = Rope(precision, rows, *heads, dim, (8, 8, 8), False, weights="none")
    dy = [g.cuda() for g in c.dy]
    dx = [torch.empty_like(g) for g in dy]
    dw = [torch.full((h, dim), 7.0, device="cuda") for h in heads]
    g = R.norm_rope_grad_desc(c.desc(c.gx), dy[0], dy[1], dx[0], dx[1], dw[0][0], dw[1][0])
    g.fwd.q_weight_per_head = g.fwd.k_weight_per_head = 1
    n = R.rtcc_norm_rope_grad_workspace(g)
    space = _workspace(n)
    R.rtcc_norm_rope_grad(g, space.data_ptr(), n)
    torch.cuda.synchronize()
    for i in range(2):
        assert (dw[i][1:] == 7.0).all()
        want = T.norm_rope_grad(_f64(c.x[i]), None, c.angle, c.eps, False, _f64(c.dy[i]))[1].sum(0)
        x = _f64(c.x[i])
        # terms g x r: |g| of a pair's length, rms-normed x
        size = (np.linalg.norm(_f64(c.dy[i]), axis=-1, keepdims=True) * np.abs(x) /
                np.sqrt((x * x).mean(-1, keepdims=True) + c.eps)).sum((0, 1))
        assert (np.abs(_f64(dw[i][0]) - want) <= (dim + 64 + 2 * np.sqrt(rows * heads[i])) * U * size).all()


class Capped(Case):
    """A case whose allowed error of a score follows the score, not the cap:
    the product's dim + 8 roundings and 8 more of the tanh.  bf16 with caps up
    to 64 has the header's 2^-22 of the cap instead."""

    def errors(self):
        cap, self.softcap = self.softcap, 0.0
        s, _p = super().errors()
        self.softcap = cap
        q, k = np.abs(_f64(self.q)), np.abs(_f64(self.k))
        g = q.shape[1] // k.shape[1]
        most = max((q[q0:q0 + nq, h] @ k[k0:k0 + nk, h // g].T).max() for q0, nq, k0, nk, _p in self.seqs
                   for h in range(q.shape[1]))
        s += cap * 2.0 ** -22 if self.precision == "bf16" and cap <= 64 else 8 * U * self.scale * most
        return s, 2 * s + max(nk for _a, _b, _c, nk, _p in self.seqs) * U + 2.0 ** -20


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("dim,bias,causal", [(64, False, False), (32, True, True), (128, True, False)])
@pytest.mark.parametrize("cap", [2.0 ** -130, 1e-3, 2.5, 50.0, 64.0, 100.0, 1e4, 1e6, 1e8, 3e38])
def test_caps_of_every_size(cap, dim, bias, causal, precision):
    c = Capped(precision, [(150, 150, 0), (33, 200, 0)], 4, 2, dim, causal=causal, bias=bias,
               softcap=float(np.float32(cap)))
    o = c.oracle()
    c.to_gpu().forward().check_forward(o).backward().check_backward(o)


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("cap", [50.0, 1e6])
def test_caps_for_single_tokens(cap, precision):
    """The kernel for few queries."""
    c = Capped(precision, [(1, 300, 0), (2, 90, 0), (1, 1, 0)], 4, 1, 64, causal=True, softcap=cap)
    c.to_gpu().forward().check_forward()


def test_more_blocks_than_one_axis_holds():
    """16,400 sequences of one token with 1,024 heads: 17.3 M blocks.  A token
    that sees itself alone returns its value and its output's gradient, and has
    no gradient of its score."""
    import torch
    n, heads, dim = 16400, 1024, 16
    gen = torch.Generator(device="cuda").manual_seed(0)
    q, k, v, do = (torch.randn(n, heads, dim, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    out, dq, dk, dv = (torch.full_like(q, float("nan")) for _ in range(4))
    lse = torch.empty(heads, n, device="cuda")
    offsets = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    d = R.attention_desc(q, k, v, out, offsets, offsets, lse=lse)
    assert R.rtcc_attention_workspace(d) == 0
    R.rtcc_attention(d, 0, 0)
    torch.cuda.synchronize()
    assert torch.equal(out, v)
    g = R.attention_grad_desc(d, do, dq, dk, dv)
    m = R.rtcc_attention_grad_workspace(g)
    space = _workspace(m)
    R.rtcc_attention_grad(g, space.data_ptr(), m)
    torch.cuda.synchronize()
    assert torch.equal(dv, do)
    # two orders of a product of 16 terms, each at most 6^2 in size, and a weight's 2^-20
    worst = ((2 * 16 + 8) * U * 16 + 2.0 ** -20) * 36 * 6 * dim ** -0.5
    assert dq.abs().max().item() <= worst and dk.abs().max().item() <= worst


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("weights", ["shared", "per_head"])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_weights_inside_a_larger_buffer(shift, weights, precision):
    """Weights and their gradients at 4-byte aligned addresses: the same bits as
    at aligned ones."""
    import torch
    rows, heads, dim = 70, (3, 2), 80
    c = Rope(precision, rows, *heads, dim, (10, 10, 10), True, weights=weights)
    dy = [g.cuda() for g in c.dy]

    def run(shift):
        def inside(w):
            buffer = torch.full((w.numel() + 8,), float("nan"), device="cuda")
            at = buffer[shift:shift + w.numel()].view(w.shape)
            return at.copy_(w)
        c.gw = [inside(w) for w in c.w]
        out = [torch.empty_like(g) for g in dy]
        d = c.desc(out)
        R.rtcc_norm_rope(d)
        dx, dw = [torch.empty_like(g) for g in dy], [inside(torch.zeros_like(w)) for w in c.w]
        g = R.norm_rope_grad_desc(d, dy[0], dy[1], dx[0], dx[1], dw[0], dw[1])
        n = R.rtcc_norm_rope_grad_workspace(g)
        space = _workspace(n)
        R.rtcc_norm_rope_grad(g, space.data_ptr(), n)
        torch.cuda.synchronize()
        return out + dx + dw

    for a, b in zip(run(0), run(shift)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("nq", [2, 200])
def test_distances_in_a_history_past_2_to_24(nq):
    """The distance bias of queries at places that float32 does not hold: with
    a slope of 0.7 the last 300 keys are all that counts (the others' weights
    are below e^-70), and the oracle sees only those."""
    import torch
    dim, n, rows = 16, 300, (1 << 24) + 333
    tail = Case("bf16", [(nq, n, 0)], 2, 1, dim, causal=True, bias=True, seed=nq)
    tail.slopes = torch.full((2,), 0.7)
    o = tail.oracle()
    c = Case("bf16", [(nq, nq, 0)], 2, 1, dim, causal=True, bias=True, seed=nq)
    c.q, c.do = tail.q, tail.do
    c.k, c.v = (torch.zeros(rows, 1, dim, dtype=torch.bfloat16) for _ in range(2))
    c.k[-n:], c.v[-n:] = tail.k, tail.v
    c.lists.update(k_lens=torch.tensor([rows], dtype=torch.int32, device="cuda"),
                   slopes=tail.slopes.cuda())
    c.to_gpu().forward()
    s, p = tail.errors()
    lse, out = _f64(c.lse), _f64(c.out)
    assert (np.abs(lse - o.lse) <= s + n * U + 2.0 ** -20 + 4 * U * np.abs(o.lse)).all()
    assert (np.abs(out - o.out) <= (p + B) * o.out_abs + (B + U) * np.abs(o.out)).all()
    c.backward()
    grads, sizes = o.grad(_f64(c.do))
    rel = p + (2 * dim + 16 + 2 * nq) * U + 3 * B
    for got, want, size in ((c.dq, grads[0], sizes[0]), (c.dk[-n:], grads[1], sizes[1]), (c.dv[-n:], grads[2], sizes[2])):
        assert (np.abs(_f64(got) - want) <= rel * size + (B + U) * np.abs(want) + 1e-30).all()
    # keys further away: at most e^-70 of the queries' sizes
    assert c.dk[:-n].abs().max().item() < 1e-20 and c.dv[:-n].abs().max().item() < 1e-20


# Long enough that tiles which all columns see whole run in turns, several of
# them.  "shares": few blocks, so the keys are cut into shares (three or more,
# turns start past the first key in all but one) and joined; "one": short
# sequences beside a long one, which keep every row to one share.
TURNS = {
    "shares": [(150, 700, 64), (131, 1333, 500)],
    "one": [(300, 705, 250)] + [(33, 20, 5)] * 3,
    "square": [(330, 330, 40), (530, 530, 0)],
}
TERMS = {"plain": {}, "cap": dict(softcap=3.0), "wide_cap": dict(softcap=1e3), "bias": dict(bias=True),
         "cap_bias": dict(softcap=3.0, bias=True)}


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("terms", sorted(TERMS))
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("seqs", sorted(TURNS))
def test_whole_tiles(seqs, dim, terms, causal, precision):
    """Forward and gradients where whole tiles run in turns, with every term."""
    c = Case(precision, TURNS[seqs], 2, 1, dim, causal=causal, gap=3, **TERMS[terms])
    o = c.oracle()
    c.to_gpu().forward()
    # shares need a workspace; without one there are none
    assert (R.rtcc_attention_workspace(c.d) > 0) == (seqs != "one")
    c.check_forward(o).backward().check_backward(o)


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("dim", [48, 96])
def test_whole_tiles_of_padded_heads(dim, precision):
    c = Case(precision, TURNS["shares"], 4, 2, dim, causal=True, layout="heads", gap=1)
    o = c.oracle()
    c.to_gpu().forward().check_forward(o).backward().check_backward(o)


@pytest.mark.parametrize("precision", PRECISIONS)
def test_caches_in_any_order(precision):
    """Key ranges that lie in another order than the queries."""
    c = Case(precision, [(70, 90, 3), (40, 300, 0), (5, 33, 33)], 2, 2, 64, causal=True, gap=7)
    (a, na, ka, la, pa), (b, nb, kb, lb, pb), (d, nd, kd, ld, pd) = c.seqs
    c.seqs = [(a, na, kd, ld, pa), (b, nb, ka, la, pb), (d, nd, kb, lb, pd)]
    for name in ("k_offsets", "k_lens"):
        x = c.lists[name]
        c.lists[name] = x[[2, 0, 1]].contiguous()
    o = c.oracle()
    c.to_gpu().forward().check_forward(o).backward().check_backward(o)


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("lists", [
    dict(q_offsets=[0, 10, 30, 2 ** 31 - 1], k_offsets=[0, 10, 2 ** 31 - 7], k_lens=[10, 20, 2 ** 31 - 1]),
    dict(q_offsets=[-5, 30, 12, 36]), dict(k_offsets=[-9, 40, -2 ** 31]), dict(k_lens=[-1, 5, 1000]),
    dict(q_offsets=[36, 0, 36, 0], k_offsets=[35, 1, 0], k_lens=[500, 500, 500]),
    dict(prefix_lens=[2 ** 31 - 1, -2 ** 31, 7]),
])
def test_nothing_is_written_past_the_buffers(lists, precision):
    """Whatever the lists hold: results lie inside larger buffers whose other
    rows keep what they hold, forward and backward, in both kinds of kernels."""
    import torch
    for rows in ((10, 20, 6), (1, 1, 2)):
        c = Case(precision, [(r, 3 * r, 1) for r in rows], 2, 1, 64, causal=True)
        for name, values in lists.items():
            if name != "prefix_lens" and rows != (10, 20, 6):
                values = [v if abs(v) > 1000 else v // 10 for v in values]
            c.lists[name] = torch.tensor(values, dtype=torch.int32, device="cuda")
        c.to_gpu()
        guard, held = 200, []

        def inside(x):
            """A tensor like x, of 7s, between rows of 5s that are to stay."""
            flat = torch.full((x.numel() + 2 * guard * 64,), 5.0, dtype=x.dtype, device="cuda")
            held.append((flat, x.numel()))
            return flat[guard * 64:guard * 64 + x.numel()].view(x.shape).fill_(7.0)

        out, lse, dq, dk, dv = (inside(x) for x in (c.q, c.lse, c.q, c.k, c.k))
        d = R.attention_desc(c.gq, c.gk, c.gv, out, lse=lse, causal=True, scale=c.scale, **c.lists)
        n = R.rtcc_attention_workspace(d)
        space = inside(torch.empty(max(n // 4, 4)))
        R.rtcc_attention(d, space.data_ptr(), n)
        g = R.attention_grad_desc(d, c.gdo, dq, dk, dv)
        n = R.rtcc_attention_grad_workspace(g)
        space = inside(torch.empty(n // 4))
        R.rtcc_attention_grad(g, space.data_ptr(), n)
        torch.cuda.synchronize()
        for flat, size in held:
            assert (flat[:guard * 64] == 5).all() and (flat[guard * 64 + size:] == 5).all()


@pytest.mark.parametrize("late", [False, True])
def test_the_largest_weight_of_a_single_token_is_not_rounded(late):
    """bf16, one query, one key that takes most of the weight, 1 to 7.9 powers
    of 2 above the one before (in a tile 128 keys before or in its own): its
    weight is 1 before the sums are divided, so the output carries its own rounding and
    that of the other weights only."""
    import torch
    n, dim, count = 150, 64, 96
    c = Case("bf16", [(1, n, 0)] * count, 2, 2, dim)
    c.scale = 0.125
    c.q.zero_()
    c.q[..., 0] = 8.0
    c.k.zero_()
    c.k[..., 0] = -60.0
    top = (torch.arange(1, count + 1) * 5.4 / count).bfloat16()
    for s in range(count):
        c.k[s * n + (0 if late else n - 2), :, 0] = 0.0
        c.k[s * n + n - 1, :, 0] = top[s]
    c.to_gpu().forward()
    o = c.oracle()
    got = _f64(c.out)
    v = _f64(c.v).reshape(count, n, 2, dim)
    less = np.exp(-_f64(top))[:, None, None]  # of the other key's weight and the largest one
    other = less / (1 + less) * np.abs(v[:, 0 if late else n - 2])
    p = 2 * (dim + 8) * U * 8 + n * U + 2.0 ** -20  # of a weight: scores of up to 60 are exact here
    assert (np.abs(got - o.out) <= B * np.abs(o.out) + B * other + p * o.out_abs).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_key_gradients_do_not_see_the_rounding_of_out(dim):
    """bf16, values that differ by one step of bf16: dS is what those steps leave
    of dP - delta, and a delta from the rounded output would be off by as much.
    Scores are whole numbers times the scale, exact but for it."""
    import torch
    n = 200
    c = Case("bf16", [(n, n, 0)], 2, 2, dim, causal=True)
    c.q, c.k = c.q.sign(), c.k.sign()
    c.scale = 0.1
    steps = (c.v > 0).float() + torch.arange(dim) % 64
    c.v = (1 + steps / 128).bfloat16()
    o = c.oracle()
    c.to_gpu().forward().backward()
    (_dq, dk, _dv), (_sq, size, _sv) = o.grad(_f64(c.do))
    rounded = np.zeros_like(dk)  # dS, each rounded to bf16
    for h, row, keys, p, _lse, _x, bend in o.rows():
        dp = o.v[keys, h] @ _f64(c.do)[row, h]
        rounded[keys, h] += np.outer(np.abs(p * (dp - p @ dp)) * c.scale, np.abs(o.q[row, h]))
    rel = 2 * (4 * U * c.scale * dim) + n * U + 2.0 ** -20 + (2 * dim + 16 + n) * U
    assert (np.abs(_f64(c.dk) - dk) <= rel * size + B * rounded + (B + U) * np.abs(dk) + 1e-30).all()
