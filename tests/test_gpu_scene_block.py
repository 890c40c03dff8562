"""The block over scene tokens: norm, attention, norm of the sum and gated
feed-forward unit run together, in training and frame by frame."""

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _reference(p, x, positions, lens, attention, eps=1e-5):
    """The block from its definition, in float64, by torch on the CPU."""
    import torch
    h, kv, d = attention.q_heads, attention.kv_heads, attention.dim

    def norm(t, i):
        c = t - t.mean(1, keepdim=True)
        return c / (c.square().mean(1, keepdim=True) + eps).sqrt() * p["weight%d" % i] + p["bias%d" % i]

    def turned(t, weight):
        t = t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() * weight
        axis = torch.repeat_interleave(torch.arange(3), torch.tensor(attention.sections))
        angle = (positions[:, axis] * attention.inv_freq.double().cpu())[:, None]
        one, two = t.chunk(2, -1)
        return torch.cat([one * angle.cos() - two * angle.sin(), two * angle.cos() + one * angle.sin()], -1)

    q, k, v = (norm(x, 1) @ p["qkv"]).view(x.shape[0], -1, d).split([h, kv, kv], 1)
    q, k = turned(q, p["q_norm"]), turned(k, p["k_norm"])
    k, v = k.repeat_interleave(h // kv, 1), v.repeat_interleave(h // kv, 1)
    outs, at = [], 0
    for n in lens:
        s = torch.einsum("ihd,jhd->hij", q[at:at + n], k[at:at + n]) * d ** -0.5
        s = attention.softcap * torch.tanh(s / attention.softcap)
        s = s.masked_fill(torch.ones(n, n).triu(1).bool(), float("-inf")).softmax(-1)
        outs.append(torch.einsum("hij,jhd->ihd", s, v[at:at + n]))
        at += n
    y = x + torch.cat(outs).reshape(x.shape[0], -1) @ p["proj"]
    b = norm(y, 2)
    g = b @ p["w_gate"].T
    return y + (g * torch.sigmoid(g) * (b @ p["w_up"].T)) @ p["w_down"].T


def test_gradients_of_the_block():
    """float32, two scenes, against differentiation in float64.  A value comes
    through at most 12 operators, each with sums of at most 144 terms that are at
    most 8 times the largest result: 12 * 144 * 8 U of the largest value."""
    import torch
    from paper_2608_08330_amd import scene_tokens as S
    lens, channels = (17, 30), 72
    block = S.SceneBlock(channels, 4, 2, 32, 136, softcap=5.0, dtype=torch.float32, seed=3)
    gen = torch.Generator().manual_seed(4)
    for name in ("weight1", "bias1", "weight2", "bias2", "q_norm", "k_norm"):
        block.p[name].add_(0.3 * torch.randn(block.p[name].shape, generator=gen).cuda())
    n = sum(lens)
    x, dy = torch.randn(n, channels, generator=gen), torch.randn(n, channels, generator=gen)
    positions = torch.randint(0, 30, (n, 3), generator=gen).float()
    out, grads = block.train(x.cuda(), positions.cuda(), torch.tensor([0, 17, 47], dtype=torch.int32, device="cuda"), dy.cuda())
    leaves = {k: t.double().cpu().requires_grad_() for k, t in block.p.items()}
    leaves["x"] = x.double().requires_grad_()
    ref = _reference(leaves, leaves["x"], positions.double(), lens, block.attention)
    wanted = dict(zip(leaves, torch.autograd.grad(ref, list(leaves.values()), dy.double())))
    assert set(grads) == set(wanted)
    for got, want in [(out, ref.detach())] + [(grads[k], wanted[k]) for k in grads]:
        assert got.shape == want.shape
        assert (got.double().cpu() - want).abs().max() <= 12 * 144 * 8 * U * want.abs().max()


@pytest.mark.parametrize("frames,patches,hidden", [(1, 1, 8), (3, 5, 1000), (4, 8, 1536)])
def test_served_frames_are_the_history(frames, patches, hidden):
    """The stream is a sum of values of about 1 (at most 16); the two ways round
    their bf16 values apart (2^-8) some six times: 6 * 16 * 2^-8 = 0.375."""
    from paper_2608_08330_amd import scene_tokens
    argv = ["--frames", str(frames), "--patches", str(patches), "--hidden", str(hidden)]
    assert scene_tokens.main(argv) <= 0.375


def test_the_block_in_a_graph():
    """Training steps captured and replayed with other tokens, with eager steps
    between: the same bits."""
    import torch
    from paper_2608_08330_amd import scene_tokens as S
    block = S.SceneBlock(384, 6, 2, 64, 520)
    n = 150
    x, dy = (torch.zeros(n, 384, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    positions = torch.arange(3 * n, device="cuda").view(n, 3).float()
    offsets = torch.tensor([0, 60, n], dtype=torch.int32, device="cuda")

    def fill(seed):
        gen = torch.Generator().manual_seed(seed)
        for t in (x, dy):
            t.copy_(torch.randn(n, 384, generator=gen))

    fill(0)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        block.train(x, positions, offsets, dy)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, grads = block.train(x, positions, offsets, dy)
    for seed in (1, 2, 3):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        first = [out.clone()] + [grads[k].clone() for k in sorted(grads)]
        again, more = block.train(x, positions, offsets, dy)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, [again] + [more[k] for k in sorted(more)]))
