"""What the Python descriptions of the token operators refuse before an address
reaches a kernel (no GPU: tensors of one other device are stood in for)."""

import pytest
import torch

from paper_2608_08330_amd import rtcc as R


class On:
    """A tensor that says it is on a GPU."""

    def __init__(self, x):
        self.x = x

    def get_device(self):
        return 0

    def __getattr__(self, name):
        return getattr(self.x, name)


def _attention(**on_host):
    t = dict(q=torch.zeros(4, 2, 32), k=torch.zeros(6, 1, 32), v=torch.zeros(6, 1, 32), out=torch.zeros(4, 2, 32),
             q_offsets=torch.tensor([0, 4], dtype=torch.int32), k_offsets=torch.tensor([0], dtype=torch.int32),
             k_lens=torch.tensor([6], dtype=torch.int32), prefix_lens=torch.tensor([1], dtype=torch.int32),
             slopes=torch.zeros(2), lse=torch.zeros(2, 4))
    t = {name: x if name in on_host else On(x) for name, x in t.items()}
    return R.attention_desc(causal=True, **t)


def _rope(host=()):
    x = {name: torch.zeros(4, 2, 32) for name in ("q", "k", "q_out", "v")}
    x.update(k_out=torch.zeros(9, 2, 32), v_out=torch.zeros(9, 2, 32), q_weight=torch.ones(32), k_weight=torch.ones(2, 32),
             positions=torch.zeros(4, 1), inv_freq=torch.zeros(16), slots=torch.zeros(4, dtype=torch.int64))
    return R.norm_rope_desc(sections=(16,), **{name: t if name in host else On(t) for name, t in x.items()})


@pytest.mark.parametrize("name", ["q", "k", "v", "out", "q_offsets", "k_offsets", "k_lens", "prefix_lens", "slopes", "lse"])
def test_attention_tensors_of_two_devices(name):
    _attention()
    with pytest.raises(ValueError, match="another device"):
        _attention(**{name: True})


@pytest.mark.parametrize("name", ["q", "k", "v", "q_out", "k_out", "v_out", "q_weight", "k_weight", "positions",
                                  "inv_freq", "slots"])
def test_norm_rope_tensors_of_two_devices(name):
    _rope()
    with pytest.raises(ValueError, match="another device"):
        _rope((name,))


def test_gradient_tensors_of_two_devices():
    x, w = torch.zeros(4, 2, 32), torch.zeros(6, 1, 32)
    R.attention_grad_desc(_attention(), On(x), On(x), On(w), On(w))
    for i in range(4):
        with pytest.raises(ValueError, match="another device"):
            R.attention_grad_desc(_attention(), *(t if j == i else On(t) for j, t in enumerate((x, x, w, w))))
    for i in range(4):
        with pytest.raises(ValueError, match="another device"):
            R.norm_rope_grad_desc(_rope(), *(x if j == i else On(x) for j in range(4)))


def test_host_tensors_reach_the_host_library_only():
    q, off = torch.zeros(4, 2, 32), torch.tensor([0, 4], dtype=torch.int32)
    lse = torch.zeros(2, 4)
    d = R.attention_desc(q, q, q, torch.zeros_like(q), off, off, lse=lse)
    g = R.attention_grad_desc(d, q, q, q, q)
    n = R.norm_rope_desc(q, q, q, q, None, None, torch.zeros(4, 1), torch.zeros(16), (16,))
    ng = R.norm_rope_grad_desc(n, q, q, q, q)
    for call, desc, rest in ((R.rtcc_attention, d, (0, 0)), (R.rtcc_attention_grad, g, (0, 0)), (R.rtcc_norm_rope, n, ()),
                             (R.rtcc_norm_rope_grad, ng, (0, 0))):
        with pytest.raises(ValueError, match="host memory"):
            call(desc, *rest)
        with pytest.raises(R.RtccError) as e:
            call(desc, *rest, kind="host")
        assert e.value.status == R.RTCC_E_STATE


def test_missing_or_flat_tensors():
    x, pos, f = torch.zeros(4, 2, 32), torch.zeros(4, 1), torch.zeros(16)
    slots, off = torch.zeros(4, dtype=torch.int64), torch.tensor([0, 4], dtype=torch.int32)
    rest = (None, None, pos, f, (16,))
    for args, kw in (((x, None, x, None), dict(slots=slots)), ((x, x, x, None), dict(slots=slots)),
                     ((x, x, x, x), dict(v=x, slots=slots)), ((x, x, x, x), dict(v=x, v_out=x)),
                     ((x[0], x, x, x), {}), ((x[0, 0], None, x, None), {})):
        with pytest.raises(ValueError):
            R.norm_rope_desc(*args, *rest, **kw)
    with pytest.raises(ValueError, match="dk is None"):
        R.norm_rope_grad_desc(R.norm_rope_desc(x, x, x, x, *rest), x, x, x, None)
    for q, k in ((x[0], x), (x, x[0]), (x, x[0, 0])):
        with pytest.raises(ValueError, match="rows, heads"):
            R.attention_desc(q, k, k, x, off, off)
