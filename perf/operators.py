"""Performance cases of the token operators: the norm and rotation of queries
and keys, and attention over packed sequences and caches.

After the detector's join a perception server keeps tokens of the fused
bird's-eye-view map (patches of cells, frame after frame, of up to eight
agents) and lets them attend to each other.  Every token has a time and a cell
(row, column), so its queries and keys are rotated by three positions; the
heads are normed before that.  A sequence is one scene: its tokens attend to
their own scene only, in full (one map), causally in time, or causally with a
prefix of scene tokens that all may see; scores may be capped by a tanh and get
a bias that falls with the distance in the sequence.  A server appends the
newest frame's tokens to a cache and attends to it; a fine-tuning step needs
the gradients.

Kinds of cases:
  rotate         norm + rotation of q and k
  append         the same for a few new tokens, with k and v written to their
                 rows of the cache
  rotate_grad    gradients of rotate with respect to q, k and both norm weights
  attend         attention of packed sequences to themselves: outputs and the
                 rows' log-sum-exp
  train          attend and its gradients with respect to q, k and v
  step           the newest `tokens` tokens of every request attend to its cache

Head layouts split the channel counts of the repository's networks (256 and
384); the token counts are those of its grids (64 x 64 up to 512 x 512 cells)
in patches, and the ranges between.
"""

import math
import random

import torch

own = False

NEG = float("-inf")


def _rotate(**kw):
    c = dict(kind="rotate", precision="bf16", rows=4096, q_heads=6, kv_heads=6, dim=64, sec_t=8, sec_y=12, sec_x=12,
             interleaved=False)
    c.update(kw)
    return c


def _attend(**kw):
    c = dict(kind="attend", precision="bf16", seqs=1, len_min=4096, len_max=4096, spread=1, tokens=0, q_heads=6,
             kv_heads=6, dim=64, causal=False, prefix=0, softcap=0.0, bias=False)
    c.update(kw)
    return c


def listed():
    return [
        # tokens of eight agents' 64 x 64 patch grids, 384 channels, before
        # they attend to each other
        _rotate(name="rotate_map", rows=32768),
        # sixteen streams, one new scene token each: a server's step, where
        # the launch is what counts; k and v go to the caches
        _rotate(name="append_step", kind="append", rows=16, capacity=2048, q_heads=8, kv_heads=2, dim=32, sec_t=4,
                sec_y=6, sec_x=6),
        # the backward pass of a fine-tuning step over 32 k tokens, wide heads
        # shared by pairs of queries, pairs of neighbouring channels rotated
        _rotate(name="rotate_grad_map", kind="rotate_grad", rows=32768, q_heads=6, kv_heads=3, dim=128, sec_t=16,
                sec_y=24, sec_x=24, interleaved=True),
        # float32 network, eight scenes of 44 x 13 patches and one row more;
        # two axes, part of the channels left as they are
        _rotate(name="rotate_grad_fp32", kind="rotate_grad", precision="fp32", rows=4577, q_heads=8, kv_heads=8,
                dim=48, sec_t=0, sec_y=8, sec_x=8),
        # two agents' 8 x 8 patches, float32, one head: the smallest workload
        _attend(name="attend_pair_fp32", precision="fp32", len_min=128, len_max=128, q_heads=1, kv_heads=1, dim=32),
        # one large map: four agents' 64 x 64 patches, all see all
        _attend(name="attend_map", len_min=16384, len_max=16384),
        # frames of one scene in time order, capped scores, wide shared heads
        _attend(name="attend_history", len_min=8192, len_max=8192, q_heads=6, kv_heads=3, dim=128, causal=True,
                softcap=30.0),
        # 35 scenes of all sizes in one batch, scene tokens first
        _attend(name="attend_scenes", seqs=35, len_min=100, len_max=1200, q_heads=12, kv_heads=4, dim=32, causal=True,
                prefix=64, bias=True),
        # a fine-tuning step over four scenes' histories with every term of
        # the score
        _attend(name="train_history", kind="train", seqs=4, len_min=1000, len_max=4096, causal=True, prefix=128,
                softcap=30.0, bias=True),
        # fine-tuning a float32 network, five scenes of at most 44 x 13 patches
        _attend(name="train_fp32", kind="train", precision="fp32", seqs=5, len_min=33, len_max=572, q_heads=8,
                kv_heads=2, dim=32),
        # one stream, one new token, a short history
        _attend(name="step_one", kind="step", tokens=1, len_min=512, len_max=512, q_heads=6, kv_heads=2, causal=True),
        # 64 streams with histories up to 32 k tokens, one new token each
        _attend(name="step_many", kind="step", seqs=64, tokens=1, len_min=1024, len_max=32768, q_heads=6, kv_heads=2,
                dim=128, causal=True, softcap=30.0, bias=True),
    ]


# --------------------------------------------------------------------- sizes

def _lengths(case):
    """Keys of every sequence: fixed by the case, spread evenly in the
    logarithm between its limits (the longest is always there)."""
    rng = random.Random(case["spread"])
    lo, hi = math.log(case["len_min"]), math.log(case["len_max"])
    lens = [min(case["len_max"], max(case["len_min"], round(math.exp(rng.uniform(lo, hi))))) for _ in range(case["seqs"])]
    lens[rng.randrange(len(lens))] = case["len_max"]
    return lens


def _queries(case, lens):
    return [case["tokens"] for _ in lens] if case["tokens"] else list(lens)


def _prefixes(case, lens):
    rng = random.Random(case["spread"] + 1)
    return [min(n, rng.randint(0, case["prefix"])) for n in lens]


def work(case):
    def visible_pairs(lens):  # (query, key) pairs of one head
        total = 0
        for nk, nq, pre in zip(lens, _queries(case, lens), _prefixes(case, lens)):
            if not case["causal"]:
                total += nq * nk
                continue
            # query i sees max(nk - nq + i + 1, pre) keys, at least none
            first, last = nk - nq + 1, nk
            flat = max(0, min(nq, pre - first + 1))  # queries that see the prefix only
            total += flat * pre
            a, n = first + flat, nq - flat
            total += n * (a + last) // 2 if n > 0 else 0
        return total

    el = 2 if case["precision"] == "bf16" else 4
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    if case["kind"] in ("rotate", "append", "rotate_grad"):
        n = case["rows"] * (hq + hk) * d
        axes = sum(1 for s in ("sec_t", "sec_y", "sec_x") if case[s])
        small = case["rows"] * axes * 4 + 2 * d * 4
        if case["kind"] == "rotate":
            return {"bytes": 2 * n * el + small, "flops": 8 * n}
        if case["kind"] == "append":
            return {"bytes": 2 * (n + case["rows"] * hk * d) * el + small + 8 * case["rows"], "flops": 8 * n}
        return {"bytes": 3 * n * el + small + 2 * d * 4, "flops": 18 * n}
    lens = _lengths(case)
    nk, nq = sum(lens), sum(_queries(case, lens))
    fwd_bytes = (2 * nq * hq * d + 2 * nk * hk * d) * el + nq * hq * 4
    pairs = visible_pairs(lens) * hq
    if case["kind"] == "train":
        # the forward's, then dO in and dq, dk, dv out
        return {"bytes": fwd_bytes + (2 * nq * hq * d + 2 * nk * hk * d) * el, "flops": 14 * pairs * d}
    return {"bytes": fwd_bytes, "flops": 4 * pairs * d}


def _cost(case):
    """Work in units of bf16 matrix operations: float32 products run at a
    sixteenth of the rate; a byte weighs 300 of them."""
    w = work(case)
    return w["flops"] * (16 if case["precision"] == "fp32" else 1) + 300 * w["bytes"]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _draw_once(rng):
    precision = "fp32" if rng.random() < 0.3 else "bf16"
    kind = rng.choice(["rotate", "append", "rotate_grad", "attend", "attend", "train", "train", "step", "step"])
    dim = rng.choice([16, 32, 32, 48, 64, 64, 64, 80, 96, 128, 128])
    kv = rng.choice([1, 2, 3, 4, 6, 8])
    q = kv * rng.choice([1, 1, 2, 3, 4, 8])
    if kind in ("rotate", "append", "rotate_grad"):
        pairs = dim // 2
        used = rng.choice([pairs, pairs, max(1, pairs // 2)])
        t = rng.randint(0, used // 2)
        y = rng.randint(0, used - t)
        c = _rotate(kind=kind, precision=precision, rows=_log(rng, 1, 65536), q_heads=q, kv_heads=kv, dim=dim, sec_t=t,
                    sec_y=y, sec_x=used - t - y, interleaved=rng.random() < 0.5)
        if kind == "append":
            c["rows"] = _log(rng, 1, 256)
            c["capacity"] = rng.choice([64, 129, 512, 1000])
        return c
    c = _attend(kind=kind, precision=precision, seqs=_log(rng, 1, 64), q_heads=q, kv_heads=kv, dim=dim,
                spread=rng.randrange(1 << 20), causal=rng.random() < 0.6, softcap=rng.choice([0.0, 0.0, 20.0, 50.0]),
                bias=rng.random() < 0.4)
    c["len_max"] = _log(rng, 1, 32768 if kind == "step" else 8192)
    c["len_min"] = _log(rng, 1, c["len_max"])
    if c["causal"] and rng.random() < 0.4:
        c["prefix"] = _log(rng, 1, 512)
    if kind == "step":
        c["tokens"] = rng.choice([1, 1, 1, 2, 5, 16, 64, 100])
    return c


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw_once(rng)
        w = c.get("len_max", 0)
        # the plain form holds the scores of the padded batch
        scores = c.get("seqs", 1) * c["q_heads"] * (c["tokens"] or w) * w if w else 0
        rows = c.get("seqs", 1) * w * c["kv_heads"] * c["dim"] if w else 0
        if _cost(c) <= most and scores <= 16384 * 16384 * 6 and rows <= 64 * 32768 * 256:
            return c


# -------------------------------------------------------------------- inputs

def _inverse_frequencies(case):
    parts = [[10000.0 ** (-i / n) for i in range(n)] for n in (case["sec_t"], case["sec_y"], case["sec_x"])]
    return torch.tensor([f for p in parts for f in p], dtype=torch.float32)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dtype = torch.bfloat16 if case["precision"] == "bf16" else torch.float32
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]

    def rand(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device=dev, dtype=dtype).mul_(scale)

    s = {"case": case, "dtype": dtype}
    if case["kind"] in ("rotate", "append", "rotate_grad"):
        n = case["rows"]
        # a fused projection's rows: queries, keys and values side by side
        qkv = rand(n, hq + 2 * hk, d, scale=1.5)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        s["q_weight"] = 1.0 + 0.1 * torch.randn(d, generator=gen, device=dev)
        s["k_weight"] = 1.0 + 0.1 * torch.randn(d, generator=gen, device=dev)
        secs = [case["sec_t"], case["sec_y"], case["sec_x"]]
        axes = [a for a in range(3) if secs[a]]
        s["sections"] = tuple(secs[a] for a in axes)
        top = (200, 512, 512)  # frames, rows and columns of cells
        s["positions"] = torch.stack(
            [torch.randint(0, top[a], (n,), generator=gen, device=dev).float() for a in axes], dim=1).contiguous()
        s["inv_freq"] = _inverse_frequencies(case).to(dev)
        s["q_out"] = torch.empty(n, hq, d, device=dev, dtype=dtype)
        if case["kind"] == "append":
            cap = case["capacity"]
            s["k_out"], s["v_out"] = rand(n * cap, hk, d), rand(n * cap, hk, d)
            at = torch.randint(0, cap, (n,), generator=gen, device=dev)
            s["slots"] = torch.arange(n, device=dev) * cap + at  # one stream a row
        else:
            s["k_out"] = torch.empty(n, hk, d, device=dev, dtype=dtype)
        if case["kind"] == "rotate_grad":
            s["dq_out"], s["dk_out"] = rand(n, hq, d, scale=0.1), rand(n, hk, d, scale=0.1)
            dqkv = torch.empty(n, hq + hk, d, device=dev, dtype=dtype)
            s["dq"], s["dk"] = dqkv[:, :hq], dqkv[:, hq:]
            s["dq_weight"] = torch.empty(d, device=dev)
            s["dk_weight"] = torch.empty(d, device=dev)
        return s

    lens = _lengths(case)
    nqs = _queries(case, lens)
    tq = sum(nqs)
    q_offsets = [0]
    for x in nqs:
        q_offsets.append(q_offsets[-1] + x)
    s["q_offsets"] = torch.tensor(q_offsets, dtype=torch.int32, device=dev)
    s["q_max"], s["k_max"] = max(nqs), max(lens)
    s["q"] = rand(tq, hq, d, scale=1.5)
    if case["tokens"]:
        # caches of one capacity; rows past a stream's length hold what an
        # earlier stream left there
        cap = (max(lens) + 63) // 64 * 64
        s["k"], s["v"] = rand(len(lens) * cap, hk, d), rand(len(lens) * cap, hk, d)
        s["k_offsets"] = torch.arange(len(lens), dtype=torch.int32, device=dev) * cap
    else:
        s["k"], s["v"] = rand(tq, hk, d), rand(tq, hk, d)
        s["k_offsets"] = s["q_offsets"][:-1].contiguous()
    s["k_lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    s["prefix_lens"] = (torch.tensor(_prefixes(case, lens), dtype=torch.int32, device=dev)
                        if case["prefix"] else None)
    # slopes that halve from head to head, as far as 2 ** -8
    s["slopes"] = (torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], device=dev)
                   if case["bias"] else None)
    s["scale"] = 1.0 / math.sqrt(d)
    s["out"] = torch.empty(tq, hq, d, device=dev, dtype=dtype)
    s["lse"] = torch.empty(hq, tq, device=dev)
    if case["kind"] == "train":
        s["dout"] = rand(tq, hq, d, scale=0.1)
        s["dq"] = torch.empty(tq, hq, d, device=dev, dtype=dtype)
        s["dk"] = torch.empty(tq, hk, d, device=dev, dtype=dtype)
        s["dv"] = torch.empty(tq, hk, d, device=dev, dtype=dtype)
    return s


# --------------------------------------------------------------- plain forms

def _angles(s, real):
    """cos, sin [rows, pairs] of the rotated pairs, 1 and 0 for the others."""
    n, pairs = s["positions"].shape[0], s["case"]["dim"] // 2
    counts = torch.tensor(s["sections"])
    axis = torch.repeat_interleave(torch.arange(len(counts)), counts).to(s["positions"].device)
    a = s["positions"].to(real)[:, axis] * s["inv_freq"].to(real)
    a = torch.cat([a, a.new_zeros(n, pairs - a.shape[1])], dim=1)[:, None, :]
    return torch.cos(a), torch.sin(a)


def _turn(x, cos, sin, interleaved):
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _norm_turn(x, w, cos, sin, interleaved, real):
    x = x.to(real)
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6)
    return _turn(x * r * w.to(real), cos, sin, interleaved)


def _norm_turn_grad(dy, x, w, cos, sin, interleaved, real):
    x, w = x.to(real), w.to(real)
    g = _turn(dy.to(real), cos, -sin, interleaved)
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6)
    n = x * r
    dn = g * w
    dx = r * (dn - n * (dn * n).mean(dim=-1, keepdim=True))
    return dx, (g * n).sum(dim=(0, 1))


def _plain_rotate(s):
    c = s["case"]
    cos, sin = _angles(s, torch.float32)
    il = c["interleaved"]
    if c["kind"] == "rotate_grad":
        dq, dwq = _norm_turn_grad(s["dq_out"], s["q"], s["q_weight"], cos, sin, il, torch.float32)
        dk, dwk = _norm_turn_grad(s["dk_out"], s["k"], s["k_weight"], cos, sin, il, torch.float32)
        return dq.to(s["dtype"]), dk.to(s["dtype"]), dwq, dwk
    q = _norm_turn(s["q"], s["q_weight"], cos, sin, il, torch.float32).to(s["dtype"])
    k = _norm_turn(s["k"], s["k_weight"], cos, sin, il, torch.float32).to(s["dtype"])
    if c["kind"] == "rotate":
        return q, k
    s["k_out"].index_copy_(0, s["slots"], k)
    s["v_out"].index_copy_(0, s["slots"], s["v"])
    return q, s["k_out"], s["v_out"]


def _plain_attention(s):
    """The padded batch: [sequence, kv head, query head of it, query, key]."""
    c, dev = s["case"], s["q"].device
    hk, g, d = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    n, mq, mk = c["seqs"], s["q_max"], s["k_max"]
    iq, ik = torch.arange(mq, device=dev), torch.arange(mk, device=dev)
    qo, nk = s["q_offsets"].long(), s["k_lens"].long()
    nq = qo[1:] - qo[:-1]
    qrow = torch.clamp(qo[:-1, None] + iq, max=s["q"].shape[0] - 1)
    krow = torch.clamp(s["k_offsets"].long()[:, None] + ik, max=s["k"].shape[0] - 1)

    def heads_of(x):  # [tokens, q_heads, d] -> [n, hk, g * mq, d]
        return x.float()[qrow].view(n, mq, hk, g, d).permute(0, 2, 3, 1, 4).reshape(n, hk, g * mq, d)

    real_key = (ik < nk[:, None])[:, None, :, None]
    q = heads_of(s["q"])
    k = torch.where(real_key, s["k"][krow].float().permute(0, 2, 1, 3), 0.0)
    v = torch.where(real_key, s["v"][krow].float().permute(0, 2, 1, 3), 0.0)
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(s["scale"]).view(n, hk, g, mq, mk)
    if c["softcap"]:
        score.div_(c["softcap"]).tanh_()
        slope_of_cap = 1.0 - score * score if c["kind"] == "train" else None
        score.mul_(c["softcap"])
    at = nk[:, None] - nq[:, None] + iq  # the queries' places among the keys
    if s["slopes"] is not None:
        far = (at[:, :, None] - ik).abs().float()
        score.sub_(s["slopes"].view(1, hk, g, 1, 1) * far[:, None, None])
    seen = (ik < nk[:, None])[:, None, :] & (iq < nq[:, None])[:, :, None]
    if c["causal"]:
        past = ik <= at[:, :, None]
        if s["prefix_lens"] is not None:
            past = past | (ik < s["prefix_lens"][:, None])[:, None, :]
        seen = seen & past
    score.masked_fill_(~seen[:, None, None], NEG)
    top = score.amax(dim=-1, keepdim=True)
    top = torch.where(top == NEG, torch.zeros_like(top), top)
    p = score.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)
    p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    flat = p.view(n, hk, g * mq, mk)
    out = torch.matmul(flat, v)

    # back to packed rows
    row = torch.arange(s["q"].shape[0], device=dev)
    seq = torch.bucketize(row, qo[1:], right=True)
    place = row - qo[seq]

    def packed(x):  # [n, hk, g * mq, d] -> [tokens, q_heads, d]
        x = x.view(n, hk, g, mq, d).permute(0, 3, 1, 2, 4).reshape(n, mq, hk * g, d)
        return x[seq, place].to(s["dtype"])

    out = packed(out)
    lse = lse.permute(0, 3, 1, 2).reshape(n, mq, hk * g)[seq, place].t().contiguous()
    if c["kind"] != "train":
        return out, lse
    do = torch.where((iq < nq[:, None])[:, None, None, :, None],
                     heads_of(s["dout"]).view(n, hk, g, mq, d), 0.0).view(n, hk, g * mq, d)
    dv = torch.matmul(flat.transpose(-1, -2).contiguous(), do)
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = dp.sub_((flat * dp).sum(dim=-1, keepdim=True)).mul_(flat)
    if c["softcap"]:
        ds = ds.mul_(slope_of_cap.view(n, hk, g * mq, mk))
    ds.mul_(s["scale"])
    dq = packed(torch.matmul(ds, k))
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q)
    dk, dv = (x.permute(0, 2, 1, 3)[seq, place].to(s["dtype"]) for x in (dk, dv))
    return out, lse, dq, dk, dv


# ----------------------------------------------------------------------- run

def _own_rotate(s):
    from paper_2608_08330_amd import rtcc as R

    c = s["case"]
    stream = torch.cuda.current_stream().cuda_stream
    append = c["kind"] == "append"
    d = R.norm_rope_desc(s["q"], s["k"], s["q_out"], s["k_out"], s["q_weight"], s["k_weight"], s["positions"],
                         s["inv_freq"], s["sections"], eps=1e-6, interleaved=c["interleaved"],
                         v=s["v"] if append else None, v_out=s["v_out"] if append else None,
                         slots=s["slots"] if append else None)
    if c["kind"] == "rotate_grad":
        g = R.norm_rope_grad_desc(d, s["dq_out"], s["dk_out"], s["dq"], s["dk"], s["dq_weight"], s["dk_weight"])
        space = torch.empty(R.rtcc_norm_rope_grad_workspace(g), dtype=torch.uint8, device="cuda")
        R.rtcc_norm_rope_grad(g, space.data_ptr(), space.numel(), stream)
        return s["dq"], s["dk"], s["dq_weight"], s["dk_weight"]
    R.rtcc_norm_rope(d, stream)
    return (s["q_out"], s["k_out"], s["v_out"]) if append else (s["q_out"], s["k_out"])


def _own_attention(s):
    from paper_2608_08330_amd import rtcc as R

    c = s["case"]
    stream = torch.cuda.current_stream().cuda_stream
    d = R.attention_desc(s["q"], s["k"], s["v"], s["out"], s["q_offsets"], s["k_offsets"], k_lens=s["k_lens"],
                         prefix_lens=s["prefix_lens"], slopes=s["slopes"], lse=s["lse"], causal=c["causal"],
                         scale=s["scale"], softcap=c["softcap"])
    space = torch.empty(R.rtcc_attention_workspace(d), dtype=torch.uint8, device="cuda")
    R.rtcc_attention(d, space.data_ptr(), space.numel(), stream)
    if c["kind"] != "train":
        return s["out"], s["lse"]
    g = R.attention_grad_desc(d, s["dout"], s["dq"], s["dk"], s["dv"])
    space = torch.empty(R.rtcc_attention_grad_workspace(g), dtype=torch.uint8, device="cuda")
    R.rtcc_attention_grad(g, space.data_ptr(), space.numel(), stream)
    return s["out"], s["lse"], s["dq"], s["dk"], s["dv"]


def run(state):
    if state["case"]["kind"] in ("rotate", "append", "rotate_grad"):
        return _own_rotate(state) if own else _plain_rotate(state)
    return _own_attention(state) if own else _plain_attention(state)


# --------------------------------------------------------------------- exact

def exact(case, seed):
    def rotate(s):
        """Every pair as a complex number times exp(i angle), in 64 bits."""
        c, dev = s["case"], s["q"].device
        d, n = c["dim"], c["rows"]
        angle = torch.zeros(n, d // 2, dtype=torch.float64, device=dev)
        at = 0
        for a, count in enumerate(s["sections"]):
            angle[:, at:at + count] = s["positions"][:, a:a + 1].double() * s["inv_freq"][at:at + count].double()
            at += count
        unit = torch.polar(torch.ones_like(angle), angle)[:, None, :]
        first = torch.arange(0, d, 2, device=dev) if c["interleaved"] else torch.arange(d // 2, device=dev)
        second = first + 1 if c["interleaved"] else first + d // 2

        def turned(x, by):
            z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * by
            y = torch.empty_like(x)
            y[..., first], y[..., second] = z.real, z.imag
            return y

        def length(x):  # root of the mean square, eps inside
            return ((x.square().sum(-1, keepdim=True) / d) + 1e-6).sqrt()

        def forward(x, w):
            x = x.double()
            return turned(x / length(x) * w.double(), unit)

        if c["kind"] == "rotate_grad":
            res = []
            for x, w, dy in ((s["q"], s["q_weight"], s["dq_out"]), (s["k"], s["k_weight"], s["dk_out"])):
                x, g = x.double(), turned(dy.double(), unit.conj())
                ln = length(x)
                gw = g * w.double()
                dx = gw / ln - x * (gw * x).sum(-1, keepdim=True) / (d * ln ** 3)
                res.append((dx, (g * x / ln).sum(1).sum(0)))
            return res[0][0], res[1][0], res[0][1], res[1][1]
        q, k = forward(s["q"], s["q_weight"]), forward(s["k"], s["k_weight"])
        if c["kind"] == "rotate":
            return q, k
        ko, vo = s["k_out"].double(), s["v_out"].double()
        ko[s["slots"]] = k
        vo[s["slots"]] = s["v"].double()
        return q, ko, vo

    def attention(s):
        """Sequence by sequence and head by head, in 64 bits."""
        c, dev = s["case"], s["q"].device
        lens = _lengths(c)
        nqs, pres = _queries(c, lens), _prefixes(c, lens)
        starts = s["k_offsets"].tolist()
        g, train = c["q_heads"] // c["kv_heads"], c["kind"] == "train"
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
        lse = torch.full(s["lse"].shape, NEG, dtype=torch.float64, device=dev)
        dq = torch.zeros_like(out)
        dk, dv = (torch.zeros(s["k"].shape if train else (1, 1, 1), dtype=torch.float64, device=dev) for _ in range(2))
        q0 = 0
        for nk, nq, pre, k0 in zip(lens, nqs, pres, starts):
            j = torch.arange(nk, device=dev)
            place = torch.arange(nk - nq, nk, device=dev)[:, None]
            hidden = (j > place) & (j >= pre) if c["causal"] else None
            for h in range(c["q_heads"]):
                kh = h // g
                qs = s["q"][q0:q0 + nq, h].double()
                ks, vs = s["k"][k0:k0 + nk, kh].double(), s["v"][k0:k0 + nk, kh].double()
                x = qs @ ks.t() * s["scale"]
                bend = None
                if c["softcap"]:
                    t = torch.tanh(x / c["softcap"])
                    x, bend = c["softcap"] * t, 1.0 - t ** 2
                if c["bias"]:
                    x = x - s["slopes"][h].double() * (place - j).abs()
                if hidden is not None:
                    x = x.masked_fill(hidden, NEG)
                z = torch.logsumexp(x, dim=1)
                p = torch.exp(x - torch.where(z == NEG, torch.zeros_like(z), z)[:, None])
                o = p @ vs
                out[q0:q0 + nq, h], lse[h, q0:q0 + nq] = o, z
                if train:
                    do = s["dout"][q0:q0 + nq, h].double()
                    ds = p * (do @ vs.t() - (do * o).sum(1, keepdim=True)) * s["scale"]
                    ds = ds if bend is None else ds * bend
                    dq[q0:q0 + nq, h] = ds @ ks
                    dk[k0:k0 + nk, kh] += ds.t() @ qs
                    dv[k0:k0 + nk, kh] += p.t() @ do
            q0 += nq
        return (out, lse, dq, dk, dv) if train else (out, lse)

    s = prepare(case, seed)
    return rotate(s) if case["kind"] in ("rotate", "append", "rotate_grad") else attention(s)
