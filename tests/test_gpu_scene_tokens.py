"""The layer over scene tokens: frames served from a cache against the whole
history at once."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("frames,patches", [(1, 1), (3, 5), (4, 8)])
def test_served_frames_are_the_history(frames, patches):
    """Outputs are averages of values of about 1 (at most 8); the projections of
    a frame and of the history may round a bf16 apart (2^-8 of queries, keys and
    values), the outputs are rounded to bf16, and a few such steps of 8 * 2^-8
    are 0.125."""
    from paper_2608_08330_amd import scene_tokens
    assert scene_tokens.main(["--frames", str(frames), "--patches", str(patches)]) <= 0.125


def test_full_cache_is_refused():
    import torch
    from paper_2608_08330_amd import scene_tokens
    layer = scene_tokens.SceneAttention(64, 2, 1, 32)
    cache = [torch.zeros(3, 1, 32, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    x, p = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 3, device="cuda")
    with pytest.raises(ValueError, match="cache holds 3"):
        layer.serve(x, p, cache[0], cache[1], 2)
