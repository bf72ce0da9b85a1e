"""Rows of the slab that hold no token of a sequence may hold anything - an earlier request's values, an evicted token's, the
next sequence's - and none of it may reach a result.  Two contexts take the same calls; in one of them the values that must
not be seen are NaN or infinity.
"""
import math

import pytest

from test_gpu_state import _image_parts

pytestmark = pytest.mark.gpu

HQ, HKV, D, B, BUDGET = 4, 2, 128, 3, 100


@pytest.fixture(scope="module")
def gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2501_04987_b200 import _build

    _build.build()
    from paper_2501_04987_b200 import binding

    return binding


def _tokens(kv, g, shape):
    import torch

    return [torch.randn(shape + (h, D), generator=g, device="cuda").to(kv.tdtype) for h in (HQ, HKV, HKV)]


def _steps(pair, g, n, active, bad=None):
    """n decode steps; in the first context the value of the token that bad(step, b) names is not finite."""
    import torch

    junk = (math.nan, math.inf)
    for s in range(n):
        q, k, v = _tokens(pair[0], g, (B,))
        w = v.clone()
        for b in range(B):
            if bad is not None and bad(s, b):
                w[b] = junk[(s + b) % 2]
        for kv, x in zip(pair, (w, v)):
            kv.decode_step(q, k, x, active=[1 if b in active else 0 for b in range(B)])


@pytest.mark.parametrize("path,split", [(1, 0), (2, 0), (3, 1), (3, 2)])
@pytest.mark.parametrize("chunk", [24, 128])
@pytest.mark.parametrize("how", ["freed", "overwritten", "reset", "neighbour", "evicted"])
def test_prefill_sees_no_dead_row(gpu, path, split, chunk, how):
    import torch

    pair = [gpu.TreeKV(BUDGET, HQ, HKV, D, "bf16", B, chunk) for _ in range(2)]
    for kv in pair:
        kv.set_rule(gpu.RULE_KEEP_LEFT)
        kv.set_option(gpu.OPT_PREFILL_PATH, path)
        if path == 3:
            kv.set_option(gpu.OPT_PREFILL_KEY_SPLIT, split)
    g = torch.Generator(device="cuda").manual_seed(chunk + path)
    mine = 1
    if how == "neighbour":        # tiles that end behind the slab of sequence 0 reach into sequence 1, which is full of them
        mine = 0
        _steps(pair, g, 2 * BUDGET - 3, (0, 1), lambda s, b: b == 1)
    elif how == "evicted":        # the right token of the last pair that was decided: its row is not reused yet
        _steps(pair, g, BUDGET + 5, (1,), lambda s, b: s == 9)
    else:
        _steps(pair, g, 30, (0,))
        _steps(pair, g, 2 * BUDGET + 37, (1,), lambda s, b: True)
        for kv in pair:
            if how == "reset":
                kv.reset()
            else:
                kv.fork_sequences([0, -1 if how == "freed" else 0, 2])
    q, k, v = _tokens(pair[0], g, (B, chunk))
    got = []
    for kv in pair:
        lens = [chunk if b == mine else 0 for b in range(B)]
        outs = [kv.prefill_chunk(q, k, v, chunk_lens=lens)[mine] for _ in range(2)]
        image, _ = kv.export_state()
        got.append(outs + [x[mine] for x in _image_parts(torch, kv, image)])
    assert bool(torch.isfinite(got[1][0]).all())
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert all(kv.stats()["device_error"] == 0 for kv in pair)
