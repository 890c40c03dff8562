"""One attention layer over tokens of the bird's-eye-view map, frame after frame.

  python -m paper_2608_08330_amd.scene_tokens [--frames F] [--patches P]

Runs the token operators together as a program uses them: `train` normalises
and rotates queries and keys by (time, row, column), attends causally over the
scene's packed history and takes the gradients back to the projection;
`serve` appends the newest frame's tokens to a cache and attends to it.  The
projections are torch products.  A served token sees what it saw in `train`,
so both answers agree up to the stored type's rounding; main() prints how far
they differ.
"""

import argparse

import torch

from . import rtcc as R


def _space(nbytes, device):
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)


class SceneAttention:
    """Fused projection [channels, (q_heads + 2 kv_heads) dim] and the norm
    weights of one layer; `softcap` as in rtcc_attention."""

    def __init__(self, channels, q_heads, kv_heads, dim, softcap=30.0, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator().manual_seed(seed)
        width = (q_heads + 2 * kv_heads) * dim
        self.q_heads, self.kv_heads, self.dim, self.softcap = q_heads, kv_heads, dim, softcap
        self.weight = (torch.randn(channels, width, generator=gen) * channels ** -0.5).to("cuda", dtype)
        self.q_norm, self.k_norm = torch.ones(dim, device="cuda"), torch.ones(dim, device="cuda")
        t = dim // 8
        y = (dim // 2 - t) // 2
        self.sections = (t, y, dim // 2 - t - y)
        self.inv_freq = torch.tensor([10000.0 ** (-i / n) for n in self.sections for i in range(n)], device="cuda")

    def _split(self, x):
        x = x.view(x.shape[0], -1, self.dim)
        return x[:, :self.q_heads], x[:, self.q_heads:-self.kv_heads], x[:, -self.kv_heads:]

    def _attend(self, q, k, v, q_offsets, k_offsets, k_lens):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[1], q.shape[0], device=q.device)
        d = R.attention_desc(q, k, v, out, q_offsets, k_offsets, k_lens=k_lens, lse=lse, causal=True,
                             softcap=self.softcap)
        space = _space(R.rtcc_attention_workspace(d), q.device)
        R.rtcc_attention(d, space.data_ptr(), space.numel(), torch.cuda.current_stream().cuda_stream)
        return out, lse, d

    def train(self, tokens, positions, offsets, dout):
        """tokens [n, channels] of packed scenes, positions float32 [n, 3],
        offsets int32 [scenes + 1], dout [n, q_heads, dim]: outputs, and the
        gradients of the projection and of both norm weights."""
        stream = torch.cuda.current_stream().cuda_stream
        q, k, v = self._split(tokens @ self.weight)
        qr, kr = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(k.shape, dtype=k.dtype, device="cuda")
        rope = R.norm_rope_desc(q, k, qr, kr, self.q_norm, self.k_norm, positions, self.inv_freq, self.sections)
        R.rtcc_norm_rope(rope, stream)
        out, _lse, d = self._attend(qr, kr, v, offsets, offsets, None)
        flat = torch.empty(tokens.shape[0], self.weight.shape[1], dtype=q.dtype, device="cuda")
        dq, dk, dv = self._split(flat)
        g = R.attention_grad_desc(d, dout, dq, dk, dv)
        space = _space(R.rtcc_attention_grad_workspace(g), "cuda")
        R.rtcc_attention_grad(g, space.data_ptr(), space.numel(), stream)
        dwq, dwk = torch.empty_like(self.q_norm), torch.empty_like(self.k_norm)
        g = R.norm_rope_grad_desc(rope, dq, dk, dq, dk, dwq, dwk)  # in place
        space = _space(R.rtcc_norm_rope_grad_workspace(g), "cuda")
        R.rtcc_norm_rope_grad(g, space.data_ptr(), space.numel(), stream)
        return out, tokens.t().contiguous() @ flat, dwq, dwk

    def serve(self, tokens, positions, cache_k, cache_v, length):
        """Append tokens [n, channels] after `length` rows of a scene's cache
        [capacity, kv_heads, dim] and attend to all of it."""
        n = tokens.shape[0]
        if length < 0 or length + n > cache_k.shape[0]:
            raise ValueError("the cache holds %d rows, %d are needed" % (cache_k.shape[0], length + n))
        q, k, v = self._split(tokens @ self.weight)
        qr = torch.empty(q.shape, dtype=q.dtype, device="cuda")
        slots = torch.arange(length, length + n, device="cuda")
        R.rtcc_norm_rope(R.norm_rope_desc(q, k, qr, cache_k, self.q_norm, self.k_norm, positions, self.inv_freq,
                                          self.sections, v=v, v_out=cache_v, slots=slots),
                         torch.cuda.current_stream().cuda_stream)
        i32 = dict(dtype=torch.int32, device="cuda")
        return self._attend(qr, cache_k, cache_v, torch.tensor([0, n], **i32), torch.zeros(1, **i32),
                            torch.tensor([length + n], **i32))[0]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--frames", type=int, default=4)
    ap.add_argument("--patches", type=int, default=8, help="patches a side of the map")
    ap.add_argument("--channels", type=int, default=384)
    a = ap.parse_args(argv)
    per, n = a.patches ** 2, a.frames * a.patches ** 2
    gen = torch.Generator().manual_seed(1)
    layer = SceneAttention(a.channels, 6, 2, 64)
    tokens = torch.randn(n, a.channels, generator=gen).to("cuda", torch.bfloat16)
    i = torch.arange(n, device="cuda")
    positions = torch.stack([i // per, i % per // a.patches, i % a.patches], dim=1).float()
    dout = torch.randn(n, 6, 64, generator=gen).to("cuda", torch.bfloat16)
    out, dw, _dwq, _dwk = layer.train(tokens, positions, torch.tensor([0, n], dtype=torch.int32, device="cuda"), dout)
    cache = [torch.zeros(n, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    served = torch.cat([layer.serve(tokens[f:f + per], positions[f:f + per], cache[0], cache[1], f)
                        for f in range(0, n, per)])
    far = (served.float() - out.float()).abs().max().item()
    print("%d tokens of %d frames: served and trained outputs differ by at most %.2e; projection gradient %.3e"
          % (n, a.frames, far, dw.float().norm().item()))
    return far


if __name__ == "__main__":
    main()
