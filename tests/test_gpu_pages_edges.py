"""Edges of the calls on pages and of the path of a draft: score rows exactly as wide as their prompts, keys that are NaN for a whole
share of a row's keys, little mass behind rejected children, the smallest temperatures.
"""
import math

import numpy as np
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


# ---- attention: a share of the keys that holds nothing but NaN ---------------------------------------------------------
@pytest.mark.parametrize("dtype,hq,hkv,past,n", [
    ("bf16", 4, 1, 20000, 1), ("bf16", 4, 1, 6912, 4), ("bf16", 32, 32, 1280, 2), ("bf16", 16, 8, 4096, 3),            # up to 16 rows
    ("bf16", 4, 1, 20000, 16), ("bf16", 8, 1, 6912, 5), ("bf16", 32, 32, 1280, 30), ("bf16", 32, 8, 4096, 20),         # up to 128
    ("bf16", 4, 1, 6912, 300), ("bf16", 4, 1, 1280, 70), ("bf16", 16, 4, 4096, 200),                                   # beyond
    ("f32", 4, 1, 20000, 2), ("f32", 4, 4, 6912, 1), ("f32", 8, 2, 20000, 9), ("f32", 4, 4, 640, 5)])
def test_shares_of_nan_keys(gpu, dtype, hq, hkv, past, n):
    """Wherever the keys of a row are cut: keys of NaN reach every row that sees one, and no other."""
    import torch

    P = Prompts(gpu, dtype, 64, hq, hkv, 64, [past], [n], n, seed=past + n)
    clean, k = P.kp.clone(), P.k.clone()
    plain = P.attend(max_past=past)
    assert bool(plain[0].isfinite().all()) and bool(plain[1].isfinite().all())
    pages = P.table[0].long()

    def poison(a, b):       # keys [a, b) of the past
        for x in range(a // 64, -(-b // 64)):
            P.kp[pages[x], :, max(0, a - 64 * x):min(64, b - 64 * x)] = math.nan

    ranges = [(0, past // 2), (0, past - 128), (past - 128, past), (past // 128 * 64, past), (0, 16), (past - 32, past), (0, past)]
    ranges += [(0, x) for x in range(512, past, 512)]
    for a, b in ranges:
        P.kp.copy_(clean)
        P.k.copy_(k)
        poison(a, b)
        for bound in (past, None):
            out, lse = P.attend(max_past=bound)
            assert bool(out.isnan().all()) and bool(lse.isnan().all()), (a, b, bound)
    for first in {0, 1, n // 2, n - 1} & set(range(n)):
        for last in {first + 1, n}:
            P.kp.copy_(clean)
            P.k.copy_(k)
            P.k[0, first:last] = math.nan
            for bound in (past, None):
                out, lse = P.attend(max_past=bound)
                assert bool(out[0, first:].isnan().all()) and bool(lse[0, first:].isnan().all()), (first, last, bound)
                assert bool(out[0, :first].isfinite().all()) and bool(lse[0, :first].isfinite().all()), (first, last, bound)
    assert P.kv.stats()["device_error"] == 0


# ---- the path of a draft ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [50, 1000, 40001, 128000])
@pytest.mark.parametrize("left", [[1e-3], [1e-5], [1e-6], [0.5, 1e-3], [0.1, 1e-2, 1e-4], [0.7, 0.6, 0.5, 0.3, 0.1, 0.01, 1e-3, 1e-4, 1e-5]])
def test_little_mass_behind_rejected_children(gpu, dtype, V, left):
    """A star whose first children are certain tokens and turned down by the largest number below one; left[i] is the mass behind the
    i-th.  The child after them has half of what is left: numbers one in a thousand beside that decide (its share is off by its
    exponential's argument of at most 20, 20 x 2^-24, the sums' some 2^-20 of what is held, and what is held by at most 16 times that)."""
    import torch

    m, heavy, B = len(left), 7, 64
    tokens = [3 + 2 * i for i in range(m)] + [heavy + 2 * m]
    masses = [1.0 - left[0]] + [left[i - 1] - left[i] for i in range(1, m)]
    p = np.full(V, 0.5 * left[-1] / (V - m - 1))
    p[tokens[:m]], p[tokens[m]] = masses, 0.5 * left[-1]
    row = torch.tensor(np.log(p), device="cuda").float().to(torch.float32 if dtype == "f32" else torch.bfloat16)
    r = np.exp(row.double().cpu().numpy())
    r /= r.sum()
    kept, rest = [], r.copy()
    for i in range(m):      # children that can be turned down: the largest number below one is above their share, told in 32 bits
        share = rest[tokens[i]] / rest.sum()
        if 1.0 - share > 4e-7:
            kept.append(tokens[i])
            rest[tokens[i]] = 0.0
    share = rest[tokens[m]] / rest.sum()
    n = len(kept) + 2
    if n == 2 or not 0.01 < share < 0.99:
        return              # (bf16 logits of a large vocabulary leave another distribution)
    rng = np.random.default_rng(V)
    u = share * (1.0 + np.where(np.arange(B) % 2, 1, -1) * np.exp(rng.uniform(math.log(1e-3), math.log(0.5), B)))
    u = np.minimum(u, 0.999)
    uniform = torch.full((B, n), 1.0 - 2.0 ** -24, device="cuda")
    uniform[:, n - 1] = torch.tensor(u, device="cuda").float()
    logits = row.expand(B, n, V).contiguous()
    tok = torch.tensor([[0] + kept + [tokens[m]]], dtype=torch.int32, device="cuda").expand(B, n).contiguous()
    mask = torch.tensor([[1] + [1 | 2 << i for i in range(n - 1)]], dtype=torch.int64, device="cuda").expand(B, n).contiguous()
    noise = torch.ones((B, V), device="cuda")
    kv = gpu.TreeKV(16, 2, 2, 64, "bf16", B, 0)
    path, count, after = (x.cpu().numpy() for x in kv.pick_path(logits, tok, uniform, noise, mask=mask))
    taken = u < share
    assert np.array_equal(count == 2, taken)
    assert (path[taken, 1] == n - 1).all()
    rest[tokens[m]] = 0.0
    if np.partition(rest, -2)[-2] < 0.99 * rest.max():
        assert (after[~taken] == int(np.argmax(rest))).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("temperature", [1e-30, 1e-38, 4e-39, 1e-41, 1.4e-45])
def test_temperatures_next_to_zero(gpu, dtype, given, temperature):
    """The one largest logit has all the mass."""
    import torch

    B, T, V = 3, 4, 5000
    g = torch.Generator(device="cuda").manual_seed(4)
    logits = torch.randn((B, T, V), generator=g, device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    logits[:, :, 100] = -math.inf
    best = torch.tensor([[17, 4000, 3, 4999], [0, 1, 2, 3], [88, 89, 90, 91]], device="cuda")
    logits.scatter_(2, best[..., None], 20.0)
    tokens = torch.zeros((B, T), dtype=torch.int32, device="cuda")
    tokens[0, 1:] = best[0, :3].int()      # a chain that is accepted
    tokens[1, 1], tokens[1, 2] = 0, 2      # accepted, then turned down
    uniform, noise = torch.full((B, T), 0.5, device="cuda"), torch.empty((B, V), device="cuda").exponential_(generator=g)
    q = torch.full((B, T, V), 1.0 / V, device="cuda") if given else None
    kv = gpu.TreeKV(16, 2, 2, 64, "bf16", B, 0)
    path, count, after = (x.tolist() for x in kv.pick_path(logits, tokens, uniform, noise, draft=q, temperature=temperature))
    assert count == [4, 2, 1] and after == [4999, 1, 88]
    assert path == [[0, 1, 2, 3], [0, 1, -1, -1], [0, -1, -1, -1]]
