"""GPU token operators (rtcc_norm_rope, rtcc_attention and their gradients)
against the fp64 oracle on the same inputs.

Tolerances are bounds, element by element: U = 2^-24 and B = 2^-8 are the
relative errors of one rounding to float32 and bf16.  A score of D products
carries D + 8 roundings of its absolute terms (and, capped, the error of a
float32 tanh, 2^-22 of the cap; with a bias, one rounding of it); a weight
twice that plus the sum's n roundings and 2^-20 for exp2, log2 and the
reciprocal; bf16 adds B for the weight itself and B for the result.  In the
gradients delta carries B of sum |dout| |out|, as out is read back rounded."""

import numpy as np
import pytest

from oracle import tokens as T
from paper_2608_08330_amd import rtcc as R

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
PRECISIONS = ["fp32", "bf16"]


def _dtype(precision):
    import torch
    return torch.bfloat16 if precision == "bf16" else torch.float32


def _rand(gen, shape, precision, scale=1.0):
    """A CPU tensor whose values the dtype holds."""
    import torch
    return (torch.randn(*shape, generator=gen) * scale).to(_dtype(precision))


def _f64(x):
    return x.double().cpu().numpy()


def _strided(x, how):
    """The values of x on the GPU with other strides: a slice of a wider row, or
    heads outside of rows."""
    import torch
    g = x.cuda()
    if how == "packed":
        return g
    if how == "wide":
        wide = torch.full((x.shape[0], x.shape[1] + 2, x.shape[2]), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, 1:-1] = g
        return wide[:, 1:-1]
    return g.permute(1, 0, 2).contiguous().permute(1, 0, 2)  # "heads"


def _empty(shape, precision, how="packed"):
    import torch
    return _strided(torch.full(shape, float("nan"), dtype=_dtype(precision)), how)


def _workspace(nbytes):
    import torch
    return torch.full((max(nbytes, 1),), 255, dtype=torch.uint8, device="cuda")  # float NaN throughout


# -------------------------------------------------------------- norm, rotation

class Rope:
    def __init__(self, precision, rows, q_heads, kv_heads, dim, sections, interleaved, weights="shared", layout="packed",
                 far=False, seed=0):
        import torch
        gen = torch.Generator().manual_seed(seed)
        self.precision, self.dim, self.il, self.sections, self.eps = precision, dim, interleaved, sections, 1e-5
        self.heads = (q_heads, kv_heads)
        self.x = [_rand(gen, (rows, h, dim), precision) for h in self.heads]
        self.dy = [_rand(gen, (rows, h, dim), precision) for h in self.heads]
        self.w = [None if weights == "none" else
                  1 + 0.2 * torch.randn(*((h, dim) if weights == "per_head" else (dim,)), generator=gen)
                  for h in self.heads]
        self.pos = torch.randint(0, 1 << 24 if far else 600, (rows, len(sections)), generator=gen).float()
        self.freq = torch.rand(sum(sections), generator=gen)
        self.gx = [_strided(x, layout) if x.shape[1] else None for x in self.x]
        self.gw = [None if w is None else w.cuda() for w in self.w]
        self.layout = layout
        self.angle = T.angles(self.pos.numpy(), self.freq.numpy(), sections, dim)

    def desc(self, out, **kw):
        self.keep = (self.pos.cuda(), self.freq.cuda())
        return R.norm_rope_desc(self.gx[0], self.gx[1], out[0], out[1], self.gw[0] if self.heads[0] else None,
                                self.gw[1] if self.heads[1] else None, self.keep[0], self.keep[1], self.sections,
                                eps=self.eps, interleaved=self.il, **kw)

    def expected(self, i):
        return T.norm_rope(_f64(self.x[i]), None if self.w[i] is None else self.w[i].numpy(), self.angle, self.eps,
                           self.il)

    def bound(self, y):
        """Norm (D / 2 + 4 roundings), rotation of a pair (sum of both members),
        and the angle's rounding to float32 turns (2 pi U of both members)."""
        i, j = T._pairs(self.dim, self.il)
        pair = np.empty_like(y)
        pair[..., i] = pair[..., j] = np.hypot(y[..., i], y[..., j]) * np.sqrt(2)
        return (self.dim / 2 + 16) * U * pair + (B if self.precision == "bf16" else U) * np.abs(y) + 1e-30


ROPE = [
    # rows, q heads, kv heads, dim, sections, interleaved, weights, layout
    (1, 1, 1, 16, (8,), False, "shared", "packed"),
    (1, 3, 2, 128, (10, 27, 27), True, "none", "wide"),
    (37, 6, 2, 48, (0, 8, 8), False, "per_head", "packed"),
    (129, 8, 8, 80, (13, 7, 20), True, "shared", "heads"),
    (300, 5, 1, 96, (1, 0, 3), False, "shared", "wide"),
    (1000, 12, 4, 32, (4, 6, 6), True, "per_head", "heads"),
    (2049, 2, 2, 64, (32,), False, "none", "packed"),
    (70, 0, 3, 64, (8, 12, 12), False, "shared", "packed"),
    (70, 3, 0, 112, (8, 12, 12), True, "per_head", "packed"),
]


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("rows,hq,hk,dim,sections,il,weights,layout", ROPE)
def test_norm_rope(precision, rows, hq, hk, dim, sections, il, weights, layout):
    import torch
    c = Rope(precision, rows, hq, hk, dim, sections, il, weights, layout)
    out = [_empty((rows, h, dim), precision, layout) if h else None for h in (hq, hk)]
    R.rtcc_norm_rope(c.desc(out))
    torch.cuda.synchronize()
    for i, o in enumerate(out):
        if o is not None:
            y = c.expected(i)
            assert (np.abs(_f64(o) - y) <= c.bound(y)).all()


@pytest.mark.parametrize("precision", PRECISIONS)
def test_norm_rope_in_place_and_far_positions(precision):
    """Positions up to 2^24 with frequencies near 1: the angle's fraction of a
    turn needs more than float32."""
    import torch
    c = Rope(precision, 211, 3, 2, 64, (8, 12, 12), False, far=True)
    c.gx = [x.clone() for x in c.gx]
    R.rtcc_norm_rope(c.desc(c.gx))
    torch.cuda.synchronize()
    for i in range(2):
        y = c.expected(i)
        assert (np.abs(_f64(c.gx[i]) - y) <= c.bound(y)).all()


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("rows", [1, 7, 300])
def test_norm_rope_slots(precision, rows):
    """Rows go to their slots, with v; slots outside the cache are skipped and
    all other rows of the cache keep what they hold."""
    import torch
    c = Rope(precision, rows, 4, 2, 32, (4, 6, 6), True, layout="wide")
    v = _rand(torch.Generator().manual_seed(9), (rows, 2, 32), precision)
    n = 2 * rows + 3
    slots = torch.randperm(n, generator=torch.Generator().manual_seed(1))[:rows].clone()
    if rows > 3:
        slots[1], slots[3] = -1, n
        slots[2] = 1 << 40
    q_out, k_out, v_out = _empty((rows, 4, 32), precision), _empty((n, 2, 32), precision), _empty((n, 2, 32), precision)
    k_out.fill_(3.0)
    v_out.fill_(5.0)
    s = slots.cuda()
    R.rtcc_norm_rope(c.desc((q_out, k_out), v=_strided(v, "heads"), v_out=v_out, slots=s))
    torch.cuda.synchronize()
    y = c.expected(0)
    assert (np.abs(_f64(q_out) - y) <= c.bound(y)).all()
    y, ko, vo = c.expected(1), _f64(k_out), _f64(v_out)
    left = np.ones(n, bool)
    for r, at in enumerate(slots.tolist()):
        if 0 <= at < n:
            assert (np.abs(ko[at] - y[r]) <= c.bound(y)[r]).all()
            assert (vo[at] == _f64(v)[r]).all()
            left[at] = False
    assert (ko[left] == 3).all() and (vo[left] == 5).all()


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("rows,hq,hk,dim,sections,il,weights,layout", ROPE)
def test_norm_rope_gradient(precision, rows, hq, hk, dim, sections, il, weights, layout):
    import torch
    c = Rope(precision, rows, hq, hk, dim, sections, il, weights, layout)
    dy = [_strided(g, layout) if g.shape[1] else None for g in c.dy]
    dx = [_empty((rows, h, dim), precision, layout) if h else None for h in (hq, hk)]
    dw = [torch.full((h, dim) if weights == "per_head" else (dim,), float("nan"), device="cuda") if h else None
          for h in (hq, hk)]
    g = R.norm_rope_grad_desc(c.desc(c.gx), dy[0], dy[1], dx[0], dx[1], dw[0], dw[1])
    n = R.rtcc_norm_rope_grad_workspace(g)
    space = _workspace(n)
    R.rtcc_norm_rope_grad(g, space.data_ptr(), n)
    torch.cuda.synchronize()
    again = [None if x is None else x.clone() for x in dw]
    R.rtcc_norm_rope_grad(g, space.data_ptr(), n)
    torch.cuda.synchronize()
    for i in range(2):
        if dx[i] is None:
            continue
        w = None if c.w[i] is None else c.w[i].numpy()
        ex, ew = T.norm_rope_grad(_f64(c.x[i]), w, c.angle, c.eps, il, _f64(c.dy[i]))
        # dx is r (g w - n mean(g w n)): terms of size r |g w| and r |n| mean |g w n|
        gabs = np.abs(T.rotate(_f64(c.dy[i]), -c.angle, il))
        gabs = gabs + c.bound(_f64(c.dy[i])) / U * U
        x = _f64(c.x[i])
        r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + c.eps)
        pair = np.linalg.norm(_f64(c.dy[i]), axis=-1, keepdims=True)
        gw = (gabs + U * pair) * (1 if w is None else np.abs(w))
        terms = r * (gw + np.abs(x) * r * (gw * np.abs(x) * r).mean(-1, keepdims=True))
        slack = (dim + 32) * U * (terms + r * pair * (1 if w is None else np.abs(w)))
        assert (np.abs(_f64(dx[i]) - ex) <= slack + (B if precision == "bf16" else U) * np.abs(ex)).all()
        tw = ((gabs + pair) * np.abs(x) * r).sum(0)
        if weights != "per_head":
            ew, tw = ew.sum(0), tw.sum(0)
        # sums in the order of lanes, waves and blocks: at most the number of
        # rows a lane adds up, and the later joins
        assert (np.abs(_f64(dw[i]) - ew) <= (dim + 64 + 2 * np.sqrt(rows * c.heads[i])) * U * tw).all()
        assert torch.equal(again[i], dw[i])


def test_norm_rope_gradient_without_rows_or_weights():
    import torch
    c = Rope("fp32", 0, 2, 1, 32, (16,), False)
    dw = [torch.full((32,), 7.0, device="cuda") for _ in range(2)]
    e = [_empty((0, h, 32), "fp32") for h in (2, 1)]
    g = R.norm_rope_grad_desc(c.desc(e), e[0], e[1], e[0], e[1], dw[0], dw[1])
    R.rtcc_norm_rope_grad(g, 0, R.rtcc_norm_rope_grad_workspace(g))
    torch.cuda.synchronize()
    assert (dw[0] == 0).all() and (dw[1] == 0).all()
    # no weight gradients wanted, in place of the outputs' gradients
    c = Rope("bf16", 50, 2, 1, 32, (16,), False)
    dy = [g.cuda() for g in c.dy]
    g = R.norm_rope_grad_desc(c.desc(c.gx), dy[0], dy[1], dy[0], dy[1])
    assert R.rtcc_norm_rope_grad_workspace(g) == 0
    R.rtcc_norm_rope_grad(g, 0, 0)
    torch.cuda.synchronize()
    ex, _ = T.norm_rope_grad(_f64(c.x[0]), c.w[0].numpy(), c.angle, c.eps, False, _f64(c.dy[0]))
    assert np.abs(_f64(dy[0]) - ex).max() <= 2 * B * np.abs(ex).max()


# ------------------------------------------------------------------ attention

class Case:
    """One attention call.  seqs: (nq, nk, prefix) each; gap: rows of k and v
    between sequences (and after the last) that belong to none, holding NaN."""

    def __init__(self, precision, seqs, q_heads, kv_heads, dim, causal=False, softcap=0.0, bias=False, gap=0,
                 layout="packed", lens=True, seed=0):
        import torch
        gen = torch.Generator().manual_seed(seed)
        self.precision, self.causal, self.softcap = precision, causal, softcap
        q0, k0, self.seqs, qo, ko, kl = 0, 0, [], [0], [], []
        for nq, nk, prefix in seqs:
            self.seqs.append((q0, nq, k0, nk, prefix))
            q0 += nq
            qo.append(q0)
            ko.append(k0)
            kl.append(nk)
            k0 += nk + gap
        if not lens:
            ko.append(k0)
        self.q = _rand(gen, (q0, q_heads, dim), precision, 1.5)
        self.k, self.v = (_rand(gen, (k0, kv_heads, dim), precision) for _ in range(2))
        self.do = _rand(gen, (q0, q_heads, dim), precision)
        used = torch.zeros(k0, dtype=torch.bool)
        for _q0, _nq, at, nk, _p in self.seqs:
            used[at:at + nk] = True
        self.k[~used] = float("nan")
        self.v[~used] = float("nan")
        self.used = used.numpy()
        self.slopes = torch.rand(q_heads, generator=gen) * 0.2 if bias else None
        self.scale = 0.8 / dim ** 0.5
        self.layout = layout
        i32 = dict(dtype=torch.int32, device="cuda")
        self.lists = dict(q_offsets=torch.tensor(qo, **i32), k_offsets=torch.tensor(ko, **i32),
                          k_lens=torch.tensor(kl, **i32) if lens else None,
                          prefix_lens=torch.tensor([p for _a, _b, p in seqs], **i32)
                          if causal and any(p for _a, _b, p in seqs) else None,
                          slopes=None if self.slopes is None else self.slopes.cuda())

    def to_gpu(self):
        import torch
        self.gq, self.gk, self.gv, self.gdo = (_strided(x, self.layout) for x in (self.q, self.k, self.v, self.do))
        self.out = _empty(self.q.shape, self.precision, self.layout)
        self.lse = torch.full((self.q.shape[1], self.q.shape[0]), float("nan"), device="cuda")
        self.d = R.attention_desc(self.gq, self.gk, self.gv, self.out, lse=self.lse, causal=self.causal,
                                  scale=self.scale, softcap=self.softcap, **self.lists)
        return self

    def forward(self, stream=0):
        import torch
        n = R.rtcc_attention_workspace(self.d)
        self.space = _workspace(n)
        torch.cuda.synchronize()
        R.rtcc_attention(self.d, self.space.data_ptr(), n, stream)
        torch.cuda.synchronize()
        return self

    def backward(self):
        import torch
        self.dq = _empty(self.q.shape, self.precision, self.layout)
        self.dk, self.dv = (_empty(self.k.shape, self.precision, self.layout) for _ in range(2))
        self.g = R.attention_grad_desc(self.d, self.gdo, self.dq, self.dk, self.dv)
        n = R.rtcc_attention_grad_workspace(self.g)
        self.space = _workspace(n)
        torch.cuda.synchronize()
        R.rtcc_attention_grad(self.g, self.space.data_ptr(), n)
        torch.cuda.synchronize()
        return self

    def oracle(self):
        return T.Attention(_f64(self.q), _f64(self.k), _f64(self.v), self.seqs, self.causal,
                           None if self.slopes is None else self.slopes.double().numpy(), float(np.float32(self.scale)),
                           self.softcap)

    def errors(self):
        """Absolute error of a score, and relative error of a weight."""
        q, k = np.nan_to_num(np.abs(_f64(self.q))), np.nan_to_num(np.abs(_f64(self.k)))
        g = q.shape[1] // k.shape[1]
        most = max([(q[q0:q0 + nq, h] @ k[k0:k0 + nk, h // g].T).max() for q0, nq, k0, nk, _p in self.seqs if nq and nk
                    for h in range(q.shape[1])] or [0.0])
        n = max([nk for _a, _b, _c, nk, _p in self.seqs] + [1])
        far = max([max(nk, abs(nk - nq)) for _a, nq, _c, nk, _p in self.seqs] + [1])
        s = (q.shape[2] + 8) * U * self.scale * most + self.softcap * 2.0 ** -22
        s += 4 * U * (float(self.slopes.max()) * far if self.slopes is not None else 0.0)
        return s, 2 * s + n * U + 2.0 ** -20

    def check_forward(self, o=None):
        o = self.oracle() if o is None else o
        s, p = self.errors()
        r = B if self.precision == "bf16" else 0.0
        got, lse = _f64(self.out), _f64(self.lse)
        assert (np.isnan(got) == np.isnan(o.out)).all()
        ok = ~np.isnan(o.out)
        assert (np.abs(got - o.out)[ok] <= ((p + r) * o.out_abs + (r + U) * np.abs(o.out))[ok]).all()
        empty = o.lse == -np.inf
        assert (lse[empty] == -np.inf).all()
        real = np.isfinite(o.lse)
        n = max([nk for _a, _b, _c, nk, _p in self.seqs] + [1])
        assert (np.abs(lse - o.lse)[real] <= s + n * U + 2.0 ** -20 + 4 * U * np.abs(o.lse[real])).all()
        return self

    def check_backward(self, o=None):
        o = self.oracle() if o is None else o
        grads, sizes = o.grad(_f64(self.do))
        _s, p = self.errors()
        r = B if self.precision == "bf16" else 0.0
        n = max([nq for _a, nq, _c, _k, _p in self.seqs] + [1]) * self.q.shape[1]
        for name, got, want, size, rounds in (("dq", self.dq, grads[0], sizes[0], 3), ("dk", self.dk, grads[1], sizes[1], 3),
                                              ("dv", self.dv, grads[2], sizes[2], 1)):
            got = _f64(got)
            # delta and dP: D + 8 roundings each; rounds: of dS, delta's o and P
            rel = p + (2 * self.q.shape[2] + 16 + n) * U + rounds * r
            used = np.ones(len(got), bool) if name == "dq" else self.used
            assert np.isnan(got[~used]).all(), name
            bad = ~(np.abs(got - want) <= rel * size + (r + U) * np.abs(want) + 1e-30)[used]
            assert not bad.any(), (name, np.abs(got - want)[used].max())
        return self


# nq, nk, prefix of the sequences; heads; dim; terms
ATTENTION = {
    "one_token": dict(seqs=[(1, 1, 0)], q_heads=1, kv_heads=1, dim=16),
    "none": dict(seqs=[(0, 0, 0), (0, 5, 0), (3, 0, 0)], q_heads=2, kv_heads=2, dim=32, gap=3),
    "pairs": dict(seqs=[(2, 2, 0)] * 5, q_heads=3, kv_heads=1, dim=48, causal=True),
    "edges": dict(seqs=[(63, 63, 0), (64, 64, 0), (65, 65, 0), (127, 33, 0), (31, 129, 0)], q_heads=2, kv_heads=1,
                  dim=64, gap=1, layout="wide"),
    "causal": dict(seqs=[(200, 200, 0), (1, 90, 0), (130, 70, 0)], q_heads=2, kv_heads=2, dim=128, causal=True, gap=7),
    "prefix": dict(seqs=[(150, 150, 40), (97, 97, 97), (40, 10, 4), (5, 9, 100), (33, 80, -5)], q_heads=4, kv_heads=2,
                   dim=80, causal=True, layout="heads"),
    "cap": dict(seqs=[(70, 140, 0), (129, 129, 0)], q_heads=3, kv_heads=3, dim=96, softcap=2.5),
    "bias": dict(seqs=[(66, 100, 0), (100, 66, 0)], q_heads=4, kv_heads=2, dim=32, bias=True, layout="heads"),
    "all_terms": dict(seqs=[(180, 180, 20), (0, 7, 0), (3, 300, 250), (90, 40, 8)], q_heads=6, kv_heads=2, dim=64,
                      causal=True, softcap=4.0, bias=True, gap=5),
    "shared_by_8": dict(seqs=[(9, 75, 0), (17, 17, 0)], q_heads=8, kv_heads=1, dim=112, causal=True, bias=True),
    "tokens": dict(seqs=[(1, 700, 0), (1, 1, 0), (1, 33, 0), (1, 0, 0), (1, 2000, 0)], q_heads=6, kv_heads=2, dim=128,
                   causal=True, gap=64),
    "few": dict(seqs=[(5, 400, 0), (3, 2, 0), (7, 1100, 0)], q_heads=4, kv_heads=1, dim=64, causal=True, softcap=3.0,
                bias=True, gap=2, layout="wide"),
    "offsets_only": dict(seqs=[(40, 40, 0), (0, 0, 0), (70, 70, 0)], q_heads=2, kv_heads=1, dim=64, lens=False),
}


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("name", sorted(ATTENTION))
def test_attention(name, precision):
    Case(precision, **ATTENTION[name]).to_gpu().forward().check_forward()


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("name", sorted(ATTENTION))
def test_attention_gradient(name, precision):
    import torch
    c = Case(precision, **ATTENTION[name]).to_gpu().forward().backward().check_backward()
    first = [x.clone() for x in (c.dq, c.dk, c.dv)]
    c.backward()
    for a, b in zip(first, (c.dq, c.dk, c.dv)):
        assert torch.equal(a.view(torch.uint8) if a.is_contiguous() else a.contiguous().view(torch.uint8),
                           b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_attention_gradient_of_many_sequences(dim, precision):
    """Enough sequences that a block's waves share its columns and keys in pairs."""
    seqs = [(i % 41, (7 * i) % 67, i % 9) for i in range(130)]
    Case(precision, seqs, 4, 4, dim, causal=True, softcap=3.0, bias=True, gap=1).to_gpu().forward().backward() \
        .check_forward().check_backward()


def test_attention_gradient_against_differences():
    """<grad, step> against the difference of the forward pass itself along a
    random step of q, k and v, in float32: the loss sum(dout out) carries
    about 2^-20 of sum |dout| |out|, the difference of order h^2 of its third
    derivative."""
    import torch
    kw = dict(seqs=[(40, 40, 5), (9, 30, 0)], q_heads=4, kv_heads=2, dim=32, causal=True, softcap=5.0, bias=True)
    c = Case("fp32", **kw).to_gpu().forward().backward()
    gen = torch.Generator().manual_seed(5)
    steps = [_rand(gen, x.shape, "fp32") for x in (c.q, c.k, c.v)]
    want = sum((g.cpu().double() * s.double()).sum().item() for g, s in zip((c.dq, c.dk, c.dv), steps))
    h = 2.0 ** -7
    loss = []
    for sign in (1, -1):
        e = Case("fp32", **kw)
        e.q, e.k, e.v = (x + sign * h * s for x, s in zip((e.q, e.k, e.v), steps))
        e.to_gpu().forward()
        loss.append((e.out.cpu().double() * c.do.double()).sum().item())
    size = (c.out.cpu().double().abs() * c.do.double().abs()).sum().item()
    assert abs((loss[0] - loss[1]) / (2 * h) - want) <= 2.0 ** -20 * size / h + 100 * h * h * size / 10


@pytest.mark.parametrize("precision", PRECISIONS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_hidden_keys_take_no_part(precision, bad):
    """Infinities and NaN in keys and values after a query's place: the queries
    before them are as if they were not there, forward and in dq."""
    c = Case(precision, [(100, 100, 0), (40, 40, 8), (2, 600, 0)], 4, 2, 64, causal=True, gap=3)
    for at in (37, 99, 103 + 30):
        c.v[at, :, 5] = bad
        c.k[at, 1, 7] = bad
    c.v[146 + 599, 0, 1] = bad  # the last key of the third, seen by its second query only
    clean = Case(precision, [(100, 100, 0), (40, 40, 8), (2, 600, 0)], 4, 2, 64, causal=True, gap=3)
    for x, y in ((c, clean),):
        x.to_gpu().forward().backward()
        y.to_gpu().forward().backward()
    rows = list(range(37)) + list(range(100, 130)) + [140]
    o = clean.oracle()
    s, p = clean.errors()
    r = B if precision == "bf16" else 0.0
    got = _f64(c.out)[rows]
    assert (np.abs(got - o.out[rows]) <= (p + r) * o.out_abs[rows] + (r + U) * np.abs(o.out[rows])).all()
    assert np.isfinite(_f64(c.lse)[:, rows]).all()
    # rows that see them carry them
    assert not np.isfinite(_f64(c.out)[37, :, 5]).any() and not np.isfinite(_f64(c.out)[141, 0, 1]).any()
    # the gradient of rows that do not see them
    grads, sizes = o.grad(_f64(clean.do))
    got, want = _f64(c.dq)[rows], grads[0][rows]
    assert (np.abs(got - want) <= (p + 1000 * U + 3 * r) * sizes[0][rows] + (r + U) * np.abs(want) + 1e-30).all()


@pytest.mark.parametrize("precision", PRECISIONS)
def test_hidden_queries_take_no_part_in_key_gradients(precision):
    """NaN in a query and its output's gradient: keys after its place do not see
    it."""
    kw = dict(seqs=[(120, 120, 0)], q_heads=2, kv_heads=1, dim=64, causal=True)
    c, clean = Case(precision, **kw), Case(precision, **kw)
    c.q[50] = float("nan")
    c.do[50] = float("inf")
    c.to_gpu().forward().backward()
    o = clean.oracle()
    grads, sizes = o.grad(_f64(clean.do))
    _s, p = clean.errors()
    r = B if precision == "bf16" else 0.0
    for got, want, size in ((c.dk, grads[1], sizes[1]), (c.dv, grads[2], sizes[2])):
        g = _f64(got)
        assert (np.abs(g - want)[51:] <= ((p + 1000 * U + 3 * r) * size + (r + U) * np.abs(want))[51:]).all()
        assert np.isnan(g[:51]).any()


def test_scores_of_any_size():
    """Scores of thousands, all of one row equal, and -inf: no overflow."""
    import torch
    c = Case("fp32", [(4, 70, 0)], 1, 1, 32)
    c.q[0] *= 1e4
    c.q[1] = 0
    c.k[:] = c.k.abs() + 0.1
    c.q[2], c.q[3] = -float("inf"), -3e38
    c.to_gpu().forward()
    o = _f64(c.out)
    assert np.isfinite(o[:2]).all()
    assert np.abs(o[1, 0] - _f64(c.v).mean(0)[0]).max() < 1e-5
    best = (_f64(c.k)[:, 0] @ _f64(c.q)[0, 0]).argmax()
    assert np.abs(o[0, 0] - _f64(c.v)[best, 0]).max() < 1e-3
    assert (o[2] == 0).all() and c.lse[0, 2].item() == -float("inf")  # every score is -inf
    assert torch.isfinite(c.lse[0, :2]).all()


def test_lists_are_clamped_to_the_buffers():
    """Offsets and lengths that lead outside, overlap or fall stay inside: other
    sequences are right, and nothing is written past the buffers."""
    import torch
    c = Case("bf16", [(10, 10, 0), (20, 20, 0), (6, 6, 0)], 2, 1, 64, causal=True)
    c.lists["k_lens"][2] = 2 ** 31 - 1
    c.lists["k_offsets"][2] = 2 ** 31 - 7
    c.lists["q_offsets"][3] = 2 ** 31 - 1
    c.to_gpu().forward()
    o = c.oracle()
    got = _f64(c.out)
    assert np.abs(got[:30] - o.out[:30]).max() < 0.05
    assert (got[30:] == 0).all()  # no keys are left there
    for name, values in (("q_offsets", [-5, 30, 12, 36]), ("k_offsets", [-9, 40, -2 ** 31]), ("k_lens", [-1, 5, 1000])):
        e = Case("bf16", [(10, 10, 0), (20, 20, 0), (6, 6, 0)], 2, 1, 64)
        e.lists[name] = torch.tensor(values, dtype=torch.int32, device="cuda")
        e.to_gpu().forward().backward()


@pytest.mark.parametrize("precision", PRECISIONS)
def test_attention_in_a_graph_and_on_a_stream(precision):
    """Captured with its workspace and replayed on new inputs, beside eager
    calls; and on a stream of the caller."""
    import torch
    c = Case(precision, [(1, 900, 0), (1, 50, 0)], 4, 2, 64, causal=True).to_gpu().forward()
    n = R.rtcc_attention_workspace(c.d)
    space = _workspace(n)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        R.rtcc_attention(c.d, space.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
    for seed in range(3):
        new = _rand(torch.Generator().manual_seed(seed), c.q.shape, precision)
        c.q, _ = new, c.gq.copy_(new)
        c.out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        graph_out = c.out.clone()
        c.forward()
        assert torch.equal(graph_out, c.out)
        c.check_forward()
    s = torch.cuda.Stream()
    c.out.fill_(float("nan"))
    c.forward(s.cuda_stream).check_forward()


def test_training_step_in_a_graph():
    import torch
    c = Case("bf16", [(150, 150, 10), (60, 60, 0)], 4, 2, 64, causal=True, softcap=5.0).to_gpu().forward().backward()
    n = R.rtcc_attention_grad_workspace(c.g)
    m = R.rtcc_attention_workspace(c.d)
    space, fspace = _workspace(n), _workspace(m)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s = torch.cuda.current_stream().cuda_stream
        R.rtcc_attention(c.d, fspace.data_ptr(), m, s)
        R.rtcc_attention_grad(c.g, space.data_ptr(), n, s)
    for seed in range(3):
        c.gk.copy_(_rand(torch.Generator().manual_seed(seed), c.k.shape, "bf16"))
        for x in (c.out, c.dq, c.dk, c.dv):
            x.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        first = [x.clone() for x in (c.out, c.dq, c.dk, c.dv)]
        R.rtcc_attention(c.d, fspace.data_ptr(), m)
        R.rtcc_attention_grad(c.g, space.data_ptr(), n)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (c.out, c.dq, c.dk, c.dv)))


def test_cache_past_32_bits():
    """A sequence at the end of a cache of more than 2^31 elements (4.3 GB a
    tensor), and one of its rows written there."""
    import torch
    heads, dim = 8, 128
    rows = (1 << 31) // (heads * dim) + 300
    k, v = (torch.empty(rows, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gen = torch.Generator().manual_seed(0)
    n = 200
    tail = [_rand(gen, (n, heads, dim), "bf16") for _ in range(2)]
    k[-n:], v[-n:] = tail[0].cuda(), tail[1].cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    for nq in (1, 150):
        q = _rand(gen, (nq, heads, dim), "bf16")
        gq, out = q.cuda(), _empty(q.shape, "bf16")
        lse = torch.empty(heads, nq, device="cuda")
        qo, ko, kl = torch.tensor([0, nq], **i32), torch.tensor([rows - n], **i32), torch.tensor([n], **i32)
        d = R.attention_desc(gq, k, v, out, qo, ko, k_lens=kl, lse=lse, causal=True)
        m = R.rtcc_attention_workspace(d)
        space = _workspace(m)
        R.rtcc_attention(d, space.data_ptr(), m)
        torch.cuda.synchronize()
        o = T.Attention(_f64(q), _f64(tail[0]), _f64(tail[1]), [(0, nq, 0, n, 0)], causal=True, scale=dim ** -0.5)
        assert (np.abs(_f64(out) - o.out) <= (B + 1e-4) * (o.out_abs + np.abs(o.out))).all()
    x = _rand(gen, (1, heads, dim), "bf16")
    gx, pos, freq = x.cuda(), torch.zeros(1, 1, device="cuda"), torch.ones(64, device="cuda")
    slots = torch.tensor([rows - 1], device="cuda")
    R.rtcc_norm_rope(R.norm_rope_desc(None, gx, None, k, None, None, pos, freq, (64,), v=gx, v_out=v, slots=slots))
    torch.cuda.synchronize()
    want = T.norm_rope(_f64(x), None, np.zeros((1, 64)), 1e-6, False)
    assert np.abs(_f64(k[-1:]) - want).max() <= 2 * B * np.abs(want).max()
    assert torch.equal(v[-1:].cpu(), x)


def test_workspace_refusals():
    c = Case("bf16", [(1, 5000, 0)], 2, 1, 64).to_gpu()
    n = R.rtcc_attention_workspace(c.d)
    assert n > 0
    space = _workspace(n)
    for pointer, size in ((0, n), (space.data_ptr(), n - 1), (space.data_ptr() + 4, n)):
        with pytest.raises(R.RtccError) as e:
            R.rtcc_attention(c.d, pointer, size)
        assert e.value.status == R.RTCC_E_ARG and "workspace" in str(e.value)
    assert np.isnan(_f64(c.out)).all()
