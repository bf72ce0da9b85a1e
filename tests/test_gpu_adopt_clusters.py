"""Eviction of long prompts where a cluster of 2, 4, 8 or 16 blocks, or one block whose weights do not fit its shared memory, takes a KV
head: ragged batches with empty and short sequences, averages, protected tokens, equal weights, NaN.
"""
import numpy as np
import pytest

from test_gpu_pages import _image_parts
from test_gpu_pages import gpu  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def _kept(w, n, c, ns, nr):
    """Tokens that stay of one KV head, in order; w: the weights that decide, float32."""
    if n <= c:
        return np.arange(n)
    free = np.arange(ns, n - nr)
    x = w[ns:n - nr]
    none = np.isnan(x)
    order = np.lexsort((free, -np.where(none, 0.0, x.astype(np.float64)), none))   # numbers first, the largest first, of equal ones the older
    return np.concatenate([np.arange(ns), np.sort(free[order[:c - ns - nr]]), np.arange(n - nr, n)])


@pytest.mark.parametrize("lens,hkv,budget,protect", [
    ([13000, 16001, 0, 12289, 40, 700, 15000, 99, 98, 14999], 5, 100, None),                   # 50 units: two blocks each
    ([20000, 12500, 0, 13003, 64, 8000], 4, 500, (4, 30)),                                      # 24 units: four
    ([41000, 0, 300, 33000], 3, 1000, (0, 64)), ([100003, 5, 60000], 2, 2048, (1, 0)),          # 12 units: eight; 6 units: sixteen
    ([50001, 0, 7, 49300, 60000, 12288, 700] + [49200] * 12, 4, 33, (2, 7)),                    # 76 units: one block each, weights read again
    ([12288, 12289] * 8, 4, 12000, None),                                                       # 64 units, nearly all stay
])
@pytest.mark.parametrize("average", [True, False])
@pytest.mark.parametrize("weights", ["even", "few values", "equal"])
def test_adopt_by_clusters(gpu, lens, hkv, budget, protect, average, weights):
    import torch

    B, d, page, pool = len(lens), 64, 64, 40
    g = torch.Generator(device="cuda").manual_seed(sum(lens) + hkv)
    kv = gpu.TreeKV(budget, hkv, hkv, d, "bf16", B, 0)
    ns, nr = protect or (0, 0)
    kv.set_protection(ns, nr)
    if not average:
        kv.set_rule(gpu.RULE_ACCUMULATED)
    width = -(-max(lens) // page)
    kp, vp = (torch.randn((pool, hkv, page, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.randint(0, pool, (B, width), generator=g, device="cuda", dtype=torch.int32)   # pages that sequences share, and meet again
    s = torch.rand((B, hkv, max(lens) + 3), generator=g, device="cuda")
    if weights == "few values":
        s = torch.round(s * 6) / 6
        s[:, 0, 5::1000] = float("nan")
        s[:, -1, 7::997] = -0.0
        s[:, -1, 9::4001] = float("inf")
    elif weights == "equal":
        s.fill_(0.375)
    first = [max(0, n - 1000) if i % 2 else 0 for i, n in enumerate(lens)]
    kv.adopt_pages(kp, vp, table, s, lens, first=first)
    img, seen = kv.export_state()
    K, V, S, pos = _image_parts(kv, img)[:4]
    sc = s.cpu().numpy()
    pages = table.long()
    for b, n in enumerate(lens):
        assert seen[b] == n
        w = sc[b, :, :n]
        if average and n:
            w = w / (n - np.maximum(np.arange(n), first[b])).astype(np.float32)
        for h in range(hkv):
            kept = _kept(w[h], n, budget, ns, nr)
            L = len(kept)
            assert np.array_equal(pos[b, h, :L], kept) and (pos[b, h, L:] == -1).all(), (b, h)
            assert np.array_equal(S[b, h, :L], sc[b, h, kept], equal_nan=True)
            at = torch.tensor(kept, device="cuda")
            rows = pages[b, at // page], at % page
            for got, src in ((K, kp), (V, vp)):
                assert np.array_equal(got[b, h, :L], src[rows[0], h, rows[1]].float().cpu().numpy())
    assert kv.stats()["device_error"] == 0
