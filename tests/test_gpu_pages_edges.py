"""Edges of the calls on pages: score rows exactly as wide as their prompts.
"""
import pytest

from test_gpu_pages import BAD_INDEX, INVALID, Prompts, _check_score
from test_gpu_pages import gpu  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


# ---- weights: rows of scores no wider than the prompts ----------------------------------------------------------------
@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 64, 8, 2), ("bf16", 128, 2, 2), ("f32", 64, 4, 1)])
@pytest.mark.parametrize("past,new,stride", [([4096], [100], 1024), ([64, 120], [64, 8], 64), ([2047, 0, 900], [1, 500, 0], 500), ([0, 0], [3, 700], 1500),
                                             ([0, 5], [0, 1], 40)])
@pytest.mark.parametrize("add", [False, True])
def test_scores_as_wide_as_the_longest_prompt(gpu, dtype, d, hq, hkv, past, new, stride, add):
    """A chunk padded to a wider buffer, and short chunks behind long pasts beside long ones behind short pasts, without max_past."""
    import torch

    P = Prompts(gpu, dtype, d, hq, hkv, 16, past, new, stride, seed=sum(past) + stride)
    _, lse = P.attend()
    steps = max(p + n for p, n in zip(past, new))
    s = torch.full((len(past), hkv, steps), 7.0, device="cuda")
    before = s.clone()
    P.kv.paged_score(P.q, lse, P.kp, P.table, P.past_dev, s, lens=new, add=add)
    assert P.kv.stats()["device_error"] == 0
    _check_score(P, lse, s, before if add else None)
    for b, (p, n) in enumerate(zip(past, new)):
        assert bool((s[b, :, p + n if n else 0:] == 7).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_sequence_that_reaches_past_its_scores_sits_out(gpu, dtype):
    """Whatever max_past says: it would write into the next rows."""
    import torch

    P = Prompts(gpu, dtype, 64, 4, 2, 16, [126, 64, 90, 5], [8, 64, 38, 1], 64)
    _, lse = P.attend()
    for bound in (None, 126, 127, 128):
        P.kv.reset()
        s = torch.full((4, 2, 128), 7.0, device="cuda")
        if bound == 128:      # no sequence of the call could have that many
            with pytest.raises(gpu.TreeKVError) as e:
                P.kv.paged_score(P.q, lse, P.kp, P.table, P.past_dev, s, lens=P.new, max_past=bound)
            assert e.value.status == INVALID and bool((s == 7).all())
            continue
        P.kv.paged_score(P.q, lse, P.kp, P.table, P.past_dev, s, lens=P.new, max_past=bound)
        st = P.kv.stats(check=False)
        assert st["device_error"] == BAD_INDEX and st["status"] == INVALID
        assert bool((s[0] == 7).all())
        Q = Prompts(gpu, dtype, 64, 4, 2, 16, [126, 64, 90, 5], [0, 64, 38, 1], 64)
        Q.K, Q.q = P.K, P.q
        _check_score(Q, lse, s)
