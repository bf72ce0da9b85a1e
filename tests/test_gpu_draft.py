"""Drafted decoding on the GPU: projection split with norms and rotation, attention of a drafted tree, the accepted path's
way into the cache, copies between sequences.  References are 64-bit; tolerances are derived where they stand.
"""
import math

import numpy as np
import pytest

import workloads as W
from lockstep import NEAR_TIE, Report, compare_state, evicted_total, run_prefill, step_decode
from test_gpu_state import _image_parts

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24                       # half a step of fp32, relative
HALF = {"bf16": 2.0 ** -8, "f32": U32}  # half a step of the element type
BAD_INDEX = 256


@pytest.fixture(scope="module")
def gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2501_04987_b200 import _build

    _build.build()
    from paper_2501_04987_b200 import binding

    return binding


def _tables(slots, d, base=1e4):
    import torch

    cos, sin = W.rope_tables(slots, d, base)
    return torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()


# ---- projection split, norms, rotation -------------------------------------------------------------------------------
def _norm_rope_ref(kv, qkv, wq, wk, cos, sin, pos, eps):
    """(value, scale of the terms that were added) of q and k in 64 bits, and v."""
    import torch

    n, d, Hq, Hkv = qkv.shape[0], kv.head_dim, kv.n_heads, kv.n_kv_heads
    x = qkv.double().reshape(n, Hq + 2 * Hkv, d)
    res = []
    for part, w in ((x[:, :Hq], wq), (x[:, Hq:Hq + Hkv], wk)):
        y = part
        if w is not None:
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * w.double()
        a, b = y[..., :d // 2], y[..., d // 2:]
        mag = torch.cat([a.abs() + b.abs()] * 2, -1)
        if cos is not None:
            c, s = cos[pos.long()].double()[:, None], sin[pos.long()].double()[:, None]
            y = torch.cat([a * c - b * s, b * c + a * s], -1)
        res.append((y, mag))
    return res, x[:, Hq + Hkv:]


def _norm_rope_close(got, ref, mag, dtype, d):
    # fp32 arithmetic: the mean of d squares is off by at most (d + 2) U32 relative, half of that after the root, which the
    # library function adds 4 U32 to; two products and a weight, then two operations of the rotation: under (d / 2 + 12) U32
    # of |n1| + |n2|; one rounding to the element type
    lim = HALF[dtype] * ref.abs() + (d / 2 + 12) * U32 * mag * (1 + HALF[dtype]) + 1e-38
    err = (got.double() - ref).abs()
    assert bool((err <= lim).all()), "off by %.3g of the limit" % float((err / lim).max())


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 32, 8), ("bf16", 128, 3, 3), ("bf16", 64, 8, 1), ("f32", 64, 4, 4),
                                            ("f32", 128, 6, 3)])
@pytest.mark.parametrize("tokens", [1, 2, 33, 700])
def test_norm_rope(gpu, dtype, d, hq, hkv, tokens):
    import torch

    kv = gpu.TreeKV(16, hq, hkv, d, dtype, 1, 0)
    g = torch.Generator(device="cuda").manual_seed(tokens * 1000 + d + hq)
    wide = (torch.randn((tokens, (hq + 2 * hkv) * d + 64), generator=g, device="cuda") * 3).to(kv.tdtype)
    cos, sin = _tables(97, d)
    pos = torch.randint(0, 97, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    wq, wk = ((1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(kv.tdtype) for _ in range(2))
    for qkv in (wide[:, :-64], wide[:, :-64].contiguous(), wide[:, 64:]):
        for w1, w2, cs in ((wq, wk, True), (None, None, True), (wq, None, True), (wq, wk, False), (None, None, False)):
            args = dict(q_weight=w1, k_weight=w2)
            if cs:
                args.update(cos=cos, sin=sin, positions=pos)
            q, k, v = kv.norm_rope(qkv, eps=1e-5, **args)
            (rq, rk), rv = _norm_rope_ref(kv, qkv, w1, w2, cos if cs else None, sin, pos, 1e-5)
            _norm_rope_close(q, *rq, dtype, d)
            _norm_rope_close(k, *rk, dtype, d)
            assert torch.equal(v.double(), rv)
    assert kv.stats()["device_error"] == 0


def test_norm_rope_padding_bad_positions_and_missing_v(gpu):
    import torch

    hq, hkv, d, n = 4, 2, 64, 9
    kv = gpu.TreeKV(16, hq, hkv, d, "bf16", 1, 0)
    cos, sin = _tables(8, d)
    qkv = torch.randn((n, (hq + 2 * hkv) * d), device="cuda").to(kv.tdtype)
    pos = torch.tensor([0, -1, 7, 3, -5, 1, 2, -(2 ** 31), 5], dtype=torch.int32, device="cuda")
    mark = lambda h: torch.full((n, h, d), 7.0, device="cuda", dtype=kv.tdtype)
    q, k, v = kv.norm_rope(qkv, cos=cos, sin=sin, positions=pos, q=mark(hq), k=mark(hkv), v=mark(hkv))
    assert kv.stats()["device_error"] == 0
    (rq, _), rv = _norm_rope_ref(kv, qkv, None, None, cos, sin, pos.clamp(min=0), 1e-6)
    for i in range(n):
        if pos[i] < 0:
            assert bool((q[i] == 7).all() and (k[i] == 7).all() and (v[i] == 7).all())
        else:
            _norm_rope_close(q[i], rq[0][i], rq[1][i], "bf16", d)
            assert torch.equal(v[i].double(), rv[i])
    # v not wanted: nothing but q and k is written
    q2, k2 = mark(hq), mark(hkv)
    assert gpu.treekv_norm_rope(kv._h, qkv.data_ptr(), qkv.stride(0), None, None, 1e-6, cos.data_ptr(), sin.data_ptr(), 8,
                                pos.data_ptr(), q2.data_ptr(), k2.data_ptr(), None, n, kv._stream()) == 0
    assert torch.equal(q2, q) and torch.equal(k2, k)
    # a position past the tables is not followed, and shows
    pos[3] = 8
    q, k, v = kv.norm_rope(qkv, cos=cos, sin=sin, positions=pos, q=mark(hq), k=mark(hkv), v=mark(hkv))
    assert bool((q[3] == 7).all() and (k[3] == 7).all() and (v[3] == 7).all()) and torch.equal(q[8], q2[8])
    with pytest.raises(gpu.TreeKVError):
        kv.stats()
    st = kv.stats(check=False)
    assert st["status"] == 1 and st["device_error"] == BAD_INDEX
    kv.reset()
    assert kv.stats()["device_error"] == 0


def test_norm_rope_of_zero_tokens_and_refusals(gpu):
    import torch

    kv = gpu.TreeKV(16, 4, 2, 64, "bf16", 1, 0)
    row = 8 * 64
    q, k, v = kv.norm_rope(torch.empty((0, row), device="cuda", dtype=kv.tdtype))
    assert q.shape == (0, 4, 64) and v.shape == (0, 2, 64)
    buf = torch.zeros(4 * row, device="cuda", dtype=kv.tdtype)
    p = buf.data_ptr()
    call = lambda qkv=p, stride=row, wq=None, eps=1e-6, cos=None, sin=None, slots=0, pos=None, q=p, k=p, v=p, n=1: gpu.treekv_norm_rope(
        kv._h, qkv, stride, wq, None, eps, cos, sin, slots, pos, q, k, v, n, kv._stream())
    before = kv.stats()["kernel_launches"]
    assert call(qkv=None) == 1 and call(q=None) == 1 and call(k=None) == 1          # missing tensors
    assert call(qkv=p + 2) == 1 and call(v=p + 8) == 1 and call(wq=p + 2) == 1      # misaligned
    assert call(stride=row - 8) == 1 and call(stride=row + 4) == 1                  # overlapping rows; rows off the 16 bytes
    assert call(cos=p) == 1 and call(cos=p, sin=p, slots=4) == 1                    # half a table; no positions
    assert call(cos=p, sin=p, slots=0, pos=p) == 1 and call(n=-1) == 1 and call(eps=-1.0) == 1 and call(eps=float("nan")) == 1
    assert kv.stats()["kernel_launches"] == before                                  # nothing was enqueued
    with pytest.raises(ValueError):
        kv.norm_rope(buf.view(4, row)[:, :-64])


# ---- a cache to draft on ---------------------------------------------------------------------------------------------
def _filled(gpu, dtype, d, hq, hkv, budget, seen, max_chunk=0, seed=1, rule=None):
    """A context whose sequences have seen that many tokens, and its K, V, S, positions in cache order."""
    import torch

    B = len(seen)
    kv = gpu.TreeKV(budget, hq, hkv, d, dtype, B, max_chunk)
    g = torch.Generator(device="cuda").manual_seed(seed)
    image, _ = kv.export_state()
    K, V, S, P, N = _image_parts(torch, kv, image)
    for b, n in enumerate(seen):
        L = min(n, budget)
        K[b, :, :L] = (1.5 * torch.randn((hkv, L, d), generator=g, device="cuda")).to(kv.tdtype)
        V[b, :, :L] = torch.randn((hkv, L, d), generator=g, device="cuda").to(kv.tdtype)
        for h in range(hkv):
            p = torch.randperm(n, generator=g, device="cuda")[:L].sort().values
            if L:
                p[-1] = n - 1
            P[b, h, :L] = p.int()
        S[b, :, :L] = (n - P[b, :, :L]) * torch.rand((hkv, L), generator=g, device="cuda") / max(L, 1)
        N[b] = n
    kv.import_state(image, list(seen))
    return kv, (K, V, S, P)


def _draft(kv, T, seed=2):
    import torch

    g = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda h, s: (s * torch.randn((kv.batch, T, h, kv.head_dim), generator=g, device="cuda")).to(kv.tdtype)
    return make(kv.n_heads, 1.0), make(kv.n_kv_heads, 1.5), make(kv.n_kv_heads, 1.0)


def _masks(B, T, kind, seed=3):
    """Python ints; a tree of ancestors and self, random words, empty words, or a chain."""
    r = np.random.default_rng(seed)
    rows = []
    for _ in range(B):
        bits = []
        for i in range(T):
            if kind == "tree":
                up = int(r.integers(max(-1, i - 5), i)) if i else -1
                bits.append((bits[up] if up >= 0 else 0) | 1 << i)
            elif kind == "any":
                bits.append(int(r.integers(0, 2 ** 63)) << 1 | int(r.integers(0, 2)))
            elif kind == "none":
                bits.append(0)
            else:
                bits.append((1 << (i + 1)) - 1)
        rows.append(bits)
    return rows


def _mask_tensor(rows):
    import torch

    return torch.tensor([[m - (1 << 64) if m >> 63 else m for m in row] for row in rows], dtype=torch.int64, device="cuda")


def _attend_ref(kv, cache, L, q, k, v, sees, b, h, rope=None):
    """Head h of sequence b in 64 bits: outputs, log-sum-exps and their limits; `sees` [T, T] drafted visibility."""
    import torch

    K, V = cache
    d, G = kv.head_dim, kv.n_heads // kv.n_kv_heads
    kh, T = h // G, sees.shape[0]
    keys = torch.cat([K[b, kh, :L].double(), k[b, :T, kh].double()])
    vals = torch.cat([V[b, kh, :L].double(), v[b, :T, kh].double()])
    qq = q[b, :T, h].double()
    if rope is not None:   # cached token j at slot j, a drafted one behind the cache by its depth; rounded as the library does
        cos, sin = rope
        depth = (sees.sum(1) - 1).clamp(min=0)
        slots = torch.cat([torch.arange(L, device="cuda"), L + depth])

        def turn(x, at):
            a, c = x[:, :d // 2].float(), x[:, d // 2:].float()
            cs, sn = cos[at], sin[at]
            # fma(x, cos, +-(y sin)) with the product rounded first: 64-bit products of 32-bit factors are exact
            y1 = (a.double() * cs.double() - (c * sn).double()).float()
            y2 = (c.double() * cs.double() + (a * sn).double()).float()
            return torch.cat([y1, y2], 1).to(kv.tdtype).double()

        keys, qq = turn(keys, slots), turn(qq, L + depth)
    see = torch.cat([torch.ones((T, L), dtype=torch.bool, device="cuda"), sees], 1)
    s = (qq @ keys.T) / math.sqrt(d)
    s = torch.where(see, s, -math.inf)
    terms = torch.where(see, (qq.abs() @ keys.abs().T) / math.sqrt(d), 0.0).amax(1) if see.shape[1] else torch.zeros(T, device="cuda")
    lse = torch.logsumexp(s, 1)
    p = torch.where(see, torch.exp(s - torch.where(lse.isinf(), 0.0, lse)[:, None]), 0.0)
    vals = torch.where(see.any(0)[:, None], vals, 0.0)   # a drafted token that nobody sees has no say, whatever it holds
    out = p @ vals
    # A logit is off by at most (d + 4) U32 of the sum of its terms' magnitudes (two more factors for the scale and its
    # products with log2 e); so a weight by twice that relative, plus 4 U32 for the exponential, plus - where the weights go
    # to the matrix units in bf16 - half a bf16 step; the sums over n keys by (n + 8) U32 relative.
    n = see.shape[1]
    delta = 2 * (d + 8) * U32 * terms + (n + 12) * U32
    lim = (p @ vals.abs()) * (2 * delta + (HALF["bf16"] if kv.tdtype == torch.bfloat16 else 0.0))[:, None]
    lim = lim * 1.01 + HALF["bf16" if kv.tdtype == torch.bfloat16 else "f32"] * out.abs() * 1.01 + 1e-30
    return out, lse, lim, delta + 2 * U32 * lse.abs().nan_to_num(0, 0, 0)


def _check_verify(kv, cache, seen, draft, rows, lens, out, lse, rope=None, heads=None):
    import torch

    q, k, v = draft
    for b in range(kv.batch):
        T = lens[b]
        if T == 0:
            continue
        sees = torch.tensor([[m >> j & 1 for j in range(T)] for m in rows[b][:T]], dtype=torch.bool, device="cuda")
        for h in range(kv.n_heads) if heads is None else heads:
            ro, rl, lim, llim = _attend_ref(kv, cache, min(seen[b], kv.budget), q, k, v, sees, b, h, rope)
            err = (out[b, :T, h].double() - ro).abs()
            assert bool((err <= lim).all()), (b, h, float((err / lim).max()))
            same = lse[b, :T, h].double() == rl                       # also minus infinity for a token that sees nothing
            assert bool((same | ((lse[b, :T, h].double() - rl).abs() <= llim)).all()), (b, h)


_SHAPES = [("bf16", 128, 8, 2), ("bf16", 128, 2, 2), ("bf16", 128, 8, 1), ("bf16", 128, 4, 2), ("bf16", 64, 8, 2), ("f32", 64, 4, 4),
           ("f32", 128, 4, 1)]


@pytest.mark.parametrize("dtype,d,hq,hkv", _SHAPES)
@pytest.mark.parametrize("T", [1, 5, 17, 33, 64])
def test_verify_trees(gpu, dtype, d, hq, hkv, T):
    """Empty, filling, just full and wrapped caches in one batch; draft lengths from nothing to all."""
    budget = 150
    seen = [0, 1, 63, 150, 151, 222, 299, 300, 437]
    lens = [T, T, max(1, T // 2), T, 0, T, 1, T, max(1, T - 1)]
    import torch

    kv, (K, V, S, P) = _filled(gpu, dtype, d, hq, hkv, budget, seen)
    draft = _draft(kv, T)
    for kind in ("tree", "any", "none", "chain"):
        rows = _masks(len(seen), T, kind)
        out = torch.full_like(draft[0], 7.0)
        lse = torch.full((len(seen), T, hq), 7.0, device="cuda")
        kv.verify_tree(*draft, mask=None if kind == "chain" else _mask_tensor(rows), lens=lens, out=out, lse=lse)
        _check_verify(kv, (K, V), seen, draft, rows, lens, out, lse)
        for b, n in enumerate(lens):
            assert bool((out[b, n:] == 7).all() and (lse[b, n:] == 7).all())   # rows behind the draft are left as they were
    if T == 5:   # the empty cache under an empty word
        rows = _masks(len(seen), T, "none")
        out, lse = kv.verify_tree(*draft, mask=_mask_tensor(rows), lens=lens)
        assert bool((out[0] == 0).all() and (lse[0] == -math.inf).all())
    # nothing of the cache has moved
    image, tokens = kv.export_state()
    K2, V2, S2, P2, _ = _image_parts(torch, kv, image)
    assert tokens == seen and torch.equal(K, K2) and torch.equal(V, V2) and torch.equal(S, S2) and torch.equal(P, P2)
    assert kv.stats()["device_error"] == 0


@pytest.mark.parametrize("dtype,d,hq,hkv,budget,B", [("bf16", 128, 8, 2, 1500, 1), ("bf16", 128, 32, 8, 700, 5), ("bf16", 64, 4, 1, 2048, 2),
                                                     ("f32", 128, 4, 2, 900, 1), ("f32", 64, 8, 1, 700, 3), ("f32", 128, 32, 16, 333, 6)])
@pytest.mark.parametrize("T", [2, 24, 64])
def test_verify_long_caches(gpu, dtype, d, hq, hkv, budget, B, T):
    seen = [budget * 2 + 77 * b + 5 for b in range(B)]
    kv, (K, V, S, P) = _filled(gpu, dtype, d, hq, hkv, budget, seen, seed=5)
    draft = _draft(kv, T, 6)
    rows = _masks(B, T, "tree", 7)
    out, lse = kv.verify_tree(*draft, mask=_mask_tensor(rows))
    _check_verify(kv, (K, V), seen, draft, rows, [T] * B, out, lse, heads=range(0, hq, 3))
    again, lse2 = kv.verify_tree(*draft, mask=_mask_tensor(rows))
    assert torch_equal(out, again) and torch_equal(lse, lse2)   # no sum depends on the order of execution
    assert kv.stats()["device_error"] == 0


def torch_equal(a, b):
    import torch

    return torch.equal(a, b)


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 4, 2), ("bf16", 64, 4, 1), ("f32", 64, 2, 2), ("f32", 128, 4, 1)])
def test_verify_with_values_that_must_not_spread(gpu, dtype, d, hq, hkv):
    """NaN and infinity in drafted tokens that a row does not see, behind the draft, and in rows of the cache that hold no
    token any more; large logits."""
    import torch

    seen, T = [70, 130, 40], 20
    lens = [20, 13, 6]
    kv, _ = _filled(gpu, dtype, d, hq, hkv, 100, [100 + 37, 260, 200], seed=8)
    # a used slab, every row of it NaN, before the real content comes in
    junk = torch.full((3, hkv, d), math.nan, device="cuda", dtype=kv.tdtype)
    for _ in range(230):
        kv.decode_step(torch.zeros((3, hq, d), device="cuda", dtype=kv.tdtype), junk, junk)
    kv2, (K, V, S, P) = _filled(gpu, dtype, d, hq, hkv, 100, seen, seed=9)
    image, tokens = kv2.export_state()
    kv.import_state(image, tokens)
    q, k, v = _draft(kv, T, 10)
    q *= 6.0
    rows = _masks(3, T, "tree", 11)
    bad = 4                                                   # a node whose value is not finite
    for b in range(3):
        rows[b][bad] = 1 << bad
        for i in range(T):
            if i != bad:
                rows[b][i] &= ~(1 << bad)
    k[0, bad], v[0, bad] = math.nan, math.nan
    v[1, bad] = math.inf
    k[2, bad] = -math.inf
    v[2, bad, :, ::2] = math.nan
    for b in range(3):
        k[b, lens[b]:], v[b, lens[b]:], q[b, lens[b]:] = math.nan, math.nan, math.nan
    out, lse = kv.verify_tree(q, k, v, mask=_mask_tensor(rows), lens=lens)
    kc, vc = k.clone(), v.clone()
    for x in (kc, vc):
        x[:, bad] = 0.0
    for b in range(3):
        keep = [i for i in range(lens[b]) if i != bad]
        sees = torch.tensor([[rows[b][i] >> j & 1 for j in range(lens[b])] for i in range(lens[b])], dtype=torch.bool, device="cuda")
        for h in range(hq):
            ro, rl, lim, llim = _attend_ref(kv, (K, V), min(seen[b], kv.budget), q, kc, vc, sees, b, h)
            assert bool(((out[b, keep, h].double() - ro[keep]).abs() <= lim[keep]).all()), (b, h)
            assert bool(((lse[b, keep, h].double() - rl[keep]).abs() <= llim[keep]).all()), (b, h)
    assert bool(out[0, bad].isnan().all())                    # the one that sees it gets it
    assert bool((out[1, bad] == math.inf).all())
    assert kv.stats()["device_error"] == 0


@pytest.mark.parametrize("dtype,d,hq,hkv,max_chunk,budget", [
    ("bf16", 128, 8, 2, 16, 90), ("bf16", 128, 2, 2, 0, 90), ("bf16", 64, 4, 2, 16, 90), ("f32", 64, 4, 2, 0, 90),
    ("bf16", 128, 8, 1, 0, 900), ("bf16", 64, 16, 4, 0, 1500), ("bf16", 128, 32, 8, 0, 450), ("f32", 128, 4, 2, 0, 700)])
def test_verify_with_in_cache_positions(gpu, dtype, d, hq, hkv, max_chunk, budget):
    import torch

    seen, T = [0, 37, budget, 2 * budget + 20], 21
    lens = [21, 8, 21, 20]
    kv2, (K, V, S, P) = _filled(gpu, dtype, d, hq, hkv, budget, seen, max_chunk, seed=12)
    image, tokens = kv2.export_state()
    kv = gpu.TreeKV(budget, hq, hkv, d, dtype, 4, max_chunk)
    cos, sin = _tables(budget + 21, d)
    kv.set_positions(cos, sin)
    kv.import_state(image, tokens)
    draft = _draft(kv, T, 13)
    for kind in ("tree", "chain"):
        rows = _masks(4, T, kind, 14)
        out, lse = kv.verify_tree(*draft, mask=_mask_tensor(rows) if kind == "tree" else None, lens=lens)
        _check_verify(kv, (K, V), seen, draft, rows, lens, out, lse, rope=(cos, sin))
    wide = _draft(kv, 22, 13)
    with pytest.raises(gpu.TreeKVError) as e:                 # the tables end before the deepest node could sit
        kv.verify_tree(*wide)
    assert e.value.status == 4


def test_verify_refusals(gpu):
    import torch

    kv = gpu.TreeKV(16, 4, 2, 64, "bf16", 2, 0)
    buf = torch.zeros(65 * 2 * 4 * 64, device="cuda", dtype=kv.tdtype)
    p = buf.data_ptr()
    call = lambda q=p, k=p, v=p, m=None, o=p, l=p, lens=None, stride=3: gpu.treekv_verify_tree(kv._h, q, k, v, m, o, l, lens, stride, kv._stream())
    before = kv.stats()["kernel_launches"]
    assert call(q=None) == 1 and call(k=None) == 1 and call(v=None) == 1 and call(o=None) == 1
    assert call(q=p + 2) == 1 and call(o=p + 8) == 1 and call(l=p + 4) == 1 and call(m=p + 4) == 1
    assert call(stride=0) == 1 and call(stride=65) == 1
    assert call(lens=[3, 4]) == 1 and call(lens=[-1, 0]) == 1
    assert call(lens=[0, 0]) == 0                              # nobody takes part
    assert kv.stats()["kernel_launches"] == before
    q, k, v = _draft(kv, 3)
    with pytest.raises(ValueError):
        kv.verify_tree(q, k, v, mask=torch.zeros((2, 3), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        kv.verify_tree(q, k[:, :2], v)
    with pytest.raises(ValueError):
        kv.verify_tree(q, k, v, lens=[3])
    # the accepted path needs rows for more than one new token
    lse = torch.zeros((2, 3, 4), device="cuda")
    path = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    with pytest.raises(gpu.TreeKVError) as e:
        kv.accept_path(q, k, v, lse, path)
    assert e.value.status == 2


def test_verify_in_a_graph_follows_the_cache(gpu):
    """Captured once, replayed on other inputs and after the cache has moved on."""
    import torch

    kv, _ = _filled(gpu, "bf16", 128, 8, 2, 200, [200, 511, 77], seed=15)
    twin, _ = _filled(gpu, "bf16", 128, 8, 2, 200, [200, 511, 77], seed=15)
    q, k, v = _draft(kv, 12, 16)
    mask = _mask_tensor(_masks(3, 12, "tree", 17))
    wide = torch.randn((36, 12 * 128), device="cuda").to(kv.tdtype)
    cos, sin = _tables(64, 128)
    pos = torch.randint(0, 64, (36,), device="cuda", dtype=torch.int32)
    qn, kn, vn = torch.empty((36, 8, 128), device="cuda", dtype=kv.tdtype), *(torch.empty((36, 2, 128), device="cuda", dtype=kv.tdtype) for _ in range(2))
    out, lse = torch.empty_like(q), torch.empty((3, 12, 8), device="cuda")
    path = torch.zeros((3, 1), dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        kv.verify_tree(q, k, v, mask=mask, out=out, lse=lse)
        kv.norm_rope(wide, cos=cos, sin=sin, positions=pos, q=qn, k=kn, v=vn)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            kv.norm_rope(wide, cos=cos, sin=sin, positions=pos, q=qn, k=kn, v=vn)
            kv.verify_tree(q, k, v, mask=mask, out=out, lse=lse)
            for call in (lambda: kv.fork_sequences([0, 0, 0]), lambda: kv.accept_path(q, k, v, lse, path, [1, 0, 1])):
                with pytest.raises(gpu.TreeKVError) as e:
                    call()
                assert e.value.status == 2
    torch.cuda.synchronize()
    for step in range(3):
        q.copy_(torch.randn_like(q)); wide.copy_(torch.randn_like(wide))
        graph.replay()
        torch.cuda.synchronize()
        a, b = twin.verify_tree(q, k, v, mask=mask)
        assert torch.equal(a, out) and torch.equal(b, lse)
        assert all(torch.equal(x, y) for x, y in zip(twin.norm_rope(wide, cos=cos, sin=sin, positions=pos), (qn, kn, vn)))
        tok = [torch.randn((3, h, 128), device="cuda").to(kv.tdtype) for h in (8, 2, 2)]
        kv.decode_step(*tok); twin.decode_step(*tok)
        torch.cuda.synchronize()


# ---- the accepted path -----------------------------------------------------------------------------------------------
def _path_rows(B, T, lens, took, seed):
    """Trees in which path[b] (took[b] nodes, ascending) is a way from a root down."""
    r = np.random.default_rng(seed)
    rows, paths = [], []
    for b in range(B):
        way = sorted(r.choice(lens[b], took[b], replace=False).tolist()) if took[b] else []
        bits = []
        for i in range(T):
            up = int(r.integers(max(-1, i - 4), i)) if i else -1
            if i in way:
                up = way[way.index(i) - 1] if i != way[0] else -1
            bits.append((bits[up] if up >= 0 else 0) | 1 << i)
        rows.append(bits)
        paths.append(way)
    return rows, paths


@pytest.mark.parametrize("dtype,d,hq,hkv,budget,chunk,protect,rope,rule", [
    ("bf16", 128, 8, 2, 96, 32, None, False, 0), ("bf16", 128, 2, 2, 40, 16, None, False, 0), ("bf16", 128, 8, 1, 60, 16, (4, 20), False, 0),
    ("bf16", 64, 4, 2, 64, 16, None, False, 3), ("f32", 64, 4, 4, 50, 16, None, False, 0), ("f32", 128, 4, 1, 70, 64, (3, 9), True, 0),
    ("bf16", 128, 2, 1, 2, 16, None, False, 0), ("f32", 64, 2, 2, 3, 8, None, False, 0), ("bf16", 64, 8, 1, 5, 64, (1, 2), False, 0),
    ("bf16", 128, 4, 1, 80, 16, None, True, 0), ("bf16", 64, 2, 2, 33, 16, None, True, 0), ("bf16", 128, 4, 2, 20, 16, None, False, 1)])
def test_drafted_decoding_in_lock_step(gpu, dtype, d, hq, hkv, budget, chunk, protect, rope, rule):
    """Prefill, then drafted steps with decode steps between them, against the oracle, for which an accepted path is a chunk:
    outputs of the accepted tokens, scores and retained positions after every call."""
    import torch
    from oracle import Oracle

    B, T = 4, 24
    w = W.parity_slice(W.CONFIGS["cfg4"], layers=1, batch=B, n_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype, budget=budget, chunk=chunk,
                       rotate=not rope)
    ns, nr = protect or (0, 0)
    kv = gpu.TreeKV(budget, hq, hkv, d, dtype, B, chunk)
    orc = Oracle(budget, hq, hkv, d, B, n_sink=ns, n_recent=nr, rule=rule)
    kv.set_rule(rule)
    if protect:
        kv.set_protection(ns, nr)
    cos = sin = None
    if rope:
        cos, sin = W.rope_tables(budget + max(T, chunk), d, w.rope_base)
        kv.set_positions(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
        orc.set_rope(cos, sin, round_bf16=dtype == "bf16")
    rep = Report()
    start = [3 * chunk + 5, 2 * chunk, chunk - 3, 0]
    run_prefill(kv, orc, w, rep, start, chunk)
    r = np.random.default_rng(budget + d)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda().to(kv.tdtype)
    f64 = lambda x: x.double().cpu().numpy()
    for step in range(14):
        lens = [int(x) for x in r.integers(1, T + 1, B)]
        took = [int(min(x, y)) for x, y in zip(lens, r.integers(0, min(T, chunk) + 1, B) if step == 5 else r.integers(0, 7, B))]
        if step == 3:
            lens[1] = took[1] = 0
        rows, paths = _path_rows(B, T, lens, took, 100 * step + d)
        q, k, v = (dev(W.round_to(s * r.standard_normal((B, T, h, d)).astype(np.float32), dtype)) for h, s in ((hq, 1.0), (hkv, 1.5), (hkv, 1.0)))
        seen = [kv.tokens_seen(b) for b in range(B)]
        out, lse = kv.verify_tree(q, k, v, mask=_mask_tensor(rows), lens=lens)
        if step % 5 == 0:
            image, _ = kv.export_state()
            Kc, Vc, _, _, _ = _image_parts(torch, kv, image)
            tabs = (torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()) if rope else None
            _check_verify(kv, (Kc, Vc), seen, (q, k, v), rows, lens, out, lse, rope=tabs)
        P = max(1, max(took))
        path = torch.tensor([(p + [T - 1] * P)[:P] for p in paths], dtype=torch.int32, device="cuda")
        kv.accept_path(q, k, v, lse, path, took)
        pick = path.long()
        seq = torch.arange(B, device="cuda")[:, None]
        out_o = orc.prefill_attend(f64(q[seq, pick]), f64(k[seq, pick]), f64(v[seq, pick]), took)
        pos_g, cnt_g = kv.retained_positions()
        ev0 = evicted_total(orc)
        rep.tally(orc, ev0, *orc.evict(pos_g.cpu().numpy(), cnt_g.cpu().numpy(), NEAR_TIE))
        og = f64(out[seq, pick])
        for b in range(B):
            assert kv.tokens_seen(b) == seen[b] + took[b]
            if took[b]:
                assert np.abs(og[b, :took[b]] - out_o[b, :took[b]]).max() <= (2e-2 if dtype == "bf16" else 1e-4)
        compare_state(kv, orc, rep)
        if step % 4 == 2:
            tok = [W.round_to(r.standard_normal((B, h, d)).astype(np.float32), dtype) for h in (hq, hkv, hkv)]
            step_decode(kv, orc, *tok, dtype, rep)
    st = kv.stats()
    assert st["device_error"] == 0 and st["evictions"] == evicted_total(orc) and rep.decisions > 0


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 8, 2), ("bf16", 64, 4, 4), ("f32", 128, 4, 2)])
def test_accept_equals_a_chunk(gpu, dtype, d, hq, hkv):
    """Long caches, paths of 1 to 64 tokens that wrap the cycle: the rows and positions of a prefill chunk under a rule that
    does not look at scores, and its scores within the error of two ways to compute a weight."""
    import torch

    budget, T, chunk = 700, 64, 64
    seen = [700 * 2 - 3, 700 + 690, 650, 0, 5, 1399]
    took = [64, 40, 64, 64, 1, 2]
    ctx = []
    for _ in range(2):
        kv, _ = _filled(gpu, dtype, d, hq, hkv, budget, seen, chunk, seed=21)
        kv.set_rule(gpu.RULE_KEEP_LEFT)
        ctx.append(kv)
    kv, twin = ctx
    q, k, v = _draft(kv, T, 22)
    rows, paths = _path_rows(6, T, [T] * 6, took, 23)
    out, lse = kv.verify_tree(q, k, v, mask=_mask_tensor(rows))
    path = torch.tensor([(p + [0] * 64)[:64] for p in paths], dtype=torch.int32, device="cuda")
    kv.accept_path(q, k, v, lse, path, took)
    pick, seq = path.long(), torch.arange(6, device="cuda")[:, None]
    out2 = twin.prefill_chunk(*(x[seq, pick].contiguous() for x in (q, k, v)), chunk_lens=took)
    (a, n1), (b, n2) = kv.export_state(), twin.export_state()
    A, B2 = _image_parts(torch, kv, a), _image_parts(torch, twin, b)
    assert n1 == n2 and all(torch.equal(A[i], B2[i]) for i in (0, 1, 3, 4))
    # both sides' weights are within delta (see _attend_ref) of the exact ones; terms of a logit sum to under 60 here
    lim = 2 * (2 * (2 * (d + 8) * U32 * 60 + (budget + 100) * U32)) * A[2].abs() + 1e-12
    assert bool(((A[2].double() - B2[2].double()).abs() <= lim).all())
    for s in range(6):
        # two kernels' roundings of the output and of the weights in bf16 (fp32: none), around values of at most 5
        tol = 5 * 4 * HALF[dtype] if dtype == "bf16" else 1e-4
        assert float((out[s, paths[s]].double() - out2[s, :took[s]].double()).abs().max()) <= tol
    # the same call twice gives the same bits
    kv2, _ = _filled(gpu, dtype, d, hq, hkv, budget, seen, chunk, seed=21)
    kv2.set_rule(gpu.RULE_KEEP_LEFT)
    kv2.accept_path(q, k, v, lse, path, took)
    c, _ = kv2.export_state()
    assert torch.equal(a, c)


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 4, 2), ("bf16", 64, 3, 3), ("f32", 64, 3, 3), ("f32", 128, 2, 1)])
def test_accept_of_rows_and_keys_that_weigh_nothing(gpu, dtype, d, hq, hkv):
    """A path token that saw nothing adds to no score, and a key whose logits are minus infinity gains exactly nothing, in
    calls whose rows do not fill a tile."""
    import torch

    kv = gpu.TreeKV(40, hq, hkv, d, dtype, 2, 8)
    q, k, v = _draft(kv, 3, 30)
    blind = torch.tensor([[0, 2, 6], [1, 3, 7]], dtype=torch.int64, device="cuda")  # sequence 0: the first sees nothing
    out, lse = kv.verify_tree(q, k, v, mask=blind)
    assert bool((lse[0, 0] == -math.inf).all()) and bool((out[0, 0] == 0).all())
    kv.accept_path(q, k, v, lse, torch.tensor([[0], [0]], dtype=torch.int32, device="cuda"))
    S = kv.scores()
    assert bool((S[0, :, 0] == 0).all()) and float((S[1, :, 0] - 1).abs().max()) <= (d + 16) * U32 * 60
    q[..., 0] = q[..., 0].abs() + 0.5
    k[:, 1, :, 0] = -math.inf                      # the path's second token: logits of minus infinity from every query
    for _ in range(2):                             # as a token of the path, then as a cached one
        out, lse = kv.verify_tree(q, k, v)
        assert bool(torch.isfinite(lse[:, 0]).all()) and not bool(torch.isnan(out).any())
        kv.accept_path(q, k, v, lse, torch.tensor([[0, 1, 2], [0, 1, 2]], dtype=torch.int32, device="cuda"))
        S = kv.scores()
        assert bool(torch.isfinite(S).all()) and bool((S[:, :, 2] == 0).all())
    assert kv.stats()["device_error"] == 0


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 8, 2), ("bf16", 64, 2, 2), ("f32", 64, 4, 1)])
def test_a_draft_of_one_is_a_decode_step(gpu, dtype, d, hq, hkv):
    """One drafted token, accepted: the cache of a decode step, and its output."""
    import torch

    seen = [0, 5, 99, 100, 101, 250]
    pair = [_filled(gpu, dtype, d, hq, hkv, 100, seen, 4, seed=51)[0] for _ in range(2)]
    path = torch.zeros((6, 1), dtype=torch.int32, device="cuda")
    for step in range(5):
        q, k, v = _draft(pair[0], 1, 52 + step)
        out, lse = pair[0].verify_tree(q, k, v)
        pair[0].accept_path(q, k, v, lse, path)
        want = pair[1].decode_step(q[:, 0].contiguous(), k[:, 0].contiguous(), v[:, 0].contiguous())
        # two kernels' roundings around values of at most 5 (the output's, and the weights' where those go to bf16)
        tol = 5 * 4 * HALF[dtype] if dtype == "bf16" else 5e-5
        assert float((out[:, 0].double() - want.double()).abs().max()) <= tol
        a, b = (x.retained_positions() for x in pair)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        sa, sb = (x.scores() for x in pair)
        assert float((sa - sb).abs().max()) <= 1e-5 * float(sb.abs().max())
    assert [pair[0].tokens_seen(b) for b in range(6)] == [n + 5 for n in seen]


def test_drafts_behind_a_pending_eviction(gpu):
    """The eviction of a chunk on the context's own stream is waited for."""
    import torch

    pair = [_filled(gpu, "bf16", 128, 4, 2, 96, [96, 300, 20], 32, seed=60)[0] for _ in range(2)]
    pair[0].set_option(gpu.OPT_EVICTION_STREAM, 1)
    x = [torch.randn((3, 32, h, 128), device="cuda").to(pair[0].tdtype) for h in (4, 2, 2)]
    q, k, v = _draft(pair[0], 9, 61)
    rows, paths = _path_rows(3, 9, [9] * 3, [3, 4, 2], 62)
    path = torch.tensor([(p + [0] * 4)[:4] for p in paths], dtype=torch.int32, device="cuda")
    got = []
    for kv in pair:
        kv.prefill_chunk(*x)
        out, lse = kv.verify_tree(q, k, v, mask=_mask_tensor(rows))
        kv.prefill_chunk(*x)
        kv.accept_path(q, k, v, lse, path, [3, 4, 2])
        got.append((out, lse, kv.export_state()[0]))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_offsets_beyond_32_bits(gpu):
    """Slabs of more than 2^32 bytes: the last sequence's rows lie behind them."""
    import torch

    B, hkv, d, budget, T = 56, 8, 128, 20480, 20
    kv = gpu.TreeKV(budget, hkv, hkv, d, "bf16", B, 8)
    assert B * hkv * (2 * budget + 8) * d * 2 > 2 ** 32
    image, _ = kv.export_state()
    K, V, S, P, N = _image_parts(torch, kv, image)
    seen = [0] * (B - 2) + [budget + 77, 3 * budget + 11]
    g = torch.Generator(device="cuda").manual_seed(70)
    for b in (B - 2, B - 1):
        K[b] = torch.randn((hkv, budget, d), generator=g, device="cuda").to(kv.tdtype)
        V[b] = torch.randn((hkv, budget, d), generator=g, device="cuda").to(kv.tdtype)
        P[b] = torch.arange(seen[b] - budget, seen[b], device="cuda", dtype=torch.int32)
        S[b] = torch.rand((hkv, budget), generator=g, device="cuda") + 0.5
        N[b] = seen[b]
    kv.import_state(image, seen)
    keep = [x[B - 2:].clone() for x in (K, V, S, P)]
    draft = _draft(kv, T, 71)
    rows, paths = _path_rows(B, T, [0] * (B - 2) + [T, T], [0] * (B - 2) + [5, 6], 72)
    lens = [0] * (B - 2) + [T, T]
    out, lse = kv.verify_tree(*draft, mask=_mask_tensor(rows), lens=lens)
    _check_verify(kv, (K, V), seen, draft, rows, lens, out, lse, heads=[0, 7])
    path = torch.tensor([(p + [0] * 6)[:6] for p in paths], dtype=torch.int32, device="cuda")
    kv.accept_path(*draft, lse, path, [0] * (B - 2) + [5, 6])
    kv.fork_sequences([B - 1] + list(range(1, B - 1)) + [B - 2])
    pos, cnt = kv.retained_positions()
    assert bool((cnt[[0, B - 2, B - 1]] == budget).all()) and kv.tokens_seen(0) == seen[-1] + 6 and kv.tokens_seen(B - 1) == seen[-2] + 5
    image, _ = kv.export_state()
    K2, V2, S2, P2, _ = _image_parts(torch, kv, image)
    where = {0: 1, B - 2: 0, B - 1: 0}        # sequence -> which of the two its content was
    for b, x in where.items():
        took = 6 if x else 5
        for h in (0, 7):
            # Algorithm 1 lets one of each of `took` adjacent pairs go: all other rows are the old ones, the path's behind them
            old = {int(p): i for i, p in enumerate(keep[3][x, h].tolist())}
            now = P2[b, h].tolist()
            assert now[-took:] == list(range(seen[B - 2 + x], seen[B - 2 + x] + took)) and len(set(now)) == budget
            idx = torch.tensor([old[p] for p in now[:-took]], device="cuda")
            assert torch.equal(K2[b, h, :-took], keep[0][x, h, idx]) and torch.equal(V2[b, h, :-took], keep[1][x, h, idx])
            nodes = torch.tensor(paths[B - 2 + x], device="cuda")
            assert torch.equal(K2[b, h, -took:], draft[1][B - 2 + x, nodes, h]) and torch.equal(V2[b, h, -took:], draft[2][B - 2 + x, nodes, h])
    assert kv.stats()["device_error"] == 0


def test_accept_of_a_bad_path_and_refusals(gpu):
    import torch

    kv, _ = _filled(gpu, "bf16", 128, 4, 2, 64, [100, 30], 8, seed=24)
    q, k, v = _draft(kv, 10, 25)
    out, lse = kv.verify_tree(q, k, v)
    image, tokens = kv.export_state()
    before = kv.stats()["kernel_launches"]
    path = torch.tensor([[0, 1, 2], [0, 1, 2]], dtype=torch.int32, device="cuda")
    p, l, w = q.data_ptr(), lse.data_ptr(), path.data_ptr()
    call = lambda q=p, lse=l, stride=10, path=w, ps=3, lens=None: gpu.treekv_accept_path(kv._h, q, p, p, lse, stride, path, ps, lens, kv._stream())
    assert call(q=None) == 1 and call(lse=None) == 1 and call(path=None) == 1
    assert call(q=p + 2) == 1 and call(lse=l + 4) == 1 and call(path=w + 2) == 1
    assert call(stride=0) == 1 and call(stride=65) == 1 and call(ps=0) == 1
    assert call(lens=[4, 0]) == 1 and call(lens=[-1, 0]) == 1 and call(ps=9, lens=[9, 0]) == 1   # more than max_chunk
    assert call(stride=2, lens=[3, 0]) == 1                                                     # more than the draft
    assert call(lens=[0, 0]) == 0
    assert kv.stats()["kernel_launches"] == before and kv.tokens_seen(0) == 100
    path[1, 1], path[0, 2] = 10, -1
    kv.accept_path(q, k, v, lse, path, [2, 2])         # sequence 0 stops before the bad index
    status, s = gpu.treekv_get_stats(kv._h, kv._stream())
    assert status == 1 and s.device_error == BAD_INDEX
    kv.reset()
    kv.import_state(image, tokens)
    kv.accept_path(q, k, v, lse, torch.tensor([[0, 1], [0, 1]], dtype=torch.int32, device="cuda"))
    assert kv.stats()["device_error"] == 0 and kv.tokens_seen(0) == 102


# ---- copies between sequences ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d,hkv,budget,B", [("bf16", 128, 2, 70, 9), ("bf16", 64, 3, 33, 9), ("f32", 128, 1, 50, 9), ("f32", 64, 2, 64, 90),
                                                  ("bf16", 128, 1, 300, 70)])
def test_fork_sequences(gpu, dtype, d, hkv, budget, B):
    import torch

    r = np.random.default_rng(B + d)
    seen = [int(x) for x in r.integers(0, 4 * budget, B)]
    seen[:5] = [0, 1, budget, budget + 1, 2 * budget]
    kv, _ = _filled(gpu, dtype, d, 2 * hkv, hkv, budget, seen, 4, seed=30)
    before = kv.stats()["evictions"]
    for source in (r.permutation(B), [0] * B, r.integers(0, B, B), r.integers(-1, B, B), np.roll(np.arange(B), 1), np.arange(B),
                   [b ^ 1 if b ^ 1 < B else b for b in range(B)], [4] * (B - 1) + [-1]):
        source = [int(x) for x in source]
        image, n0 = kv.export_state()
        old = [x.clone() for x in _image_parts(torch, kv, image)]
        kv.fork_sequences(source)
        image, n1 = kv.export_state()
        new = _image_parts(torch, kv, image)
        assert n1 == [0 if s < 0 else n0[s] for s in source] == [kv.tokens_seen(b) for b in range(B)]
        for b, s in enumerate(source):
            for i in range(5):
                if s >= 0:
                    assert torch.equal(new[i][b], old[i][s]), (b, s, i)
        # copies of one sequence stay equal under equal inputs, whatever else the batch does
        one = [torch.randn((1, h, d), device="cuda").to(kv.tdtype).expand(B, h, d).contiguous() for h in (2 * hkv, hkv, hkv)]
        out = kv.decode_step(*one)
        for b, s in enumerate(source):
            if s >= 0:
                twin = source.index(s)
                assert torch.equal(out[b], out[twin])
    assert kv.stats()["device_error"] == 0 and before >= 0


def test_fork_after_a_pending_eviction_and_refusals(gpu):
    import torch

    kv, _ = _filled(gpu, "bf16", 128, 4, 2, 64, [64, 200, 10], 32, seed=31)
    ref, _ = _filled(gpu, "bf16", 128, 4, 2, 64, [64, 200, 10], 32, seed=31)
    kv.set_option(gpu.OPT_EVICTION_STREAM, 1)
    x = [torch.randn((3, 32, h, 128), device="cuda").to(kv.tdtype) for h in (4, 2, 2)]
    for c in (kv, ref):
        c.prefill_chunk(*x)
        c.fork_sequences([2, 0, 1])
    (a, n1), (b, n2) = kv.export_state(), ref.export_state()
    assert n1 == n2 and torch.equal(a, b)
    assert gpu.treekv_fork_sequences(kv._h, [0, 3, 0], kv._stream()) == 1
    assert gpu.treekv_fork_sequences(kv._h, [0, -2, 0], kv._stream()) == 1
    assert gpu.treekv_fork_sequences(kv._h, None, kv._stream()) == 1
    with pytest.raises(ValueError):
        kv.fork_sequences([0, 1])
    # a sequence that was prefilled in one shot keeps its scoring start in its copies
    kv.set_option(gpu.OPT_EVICTION_STREAM, 0)
    kv.reset()
    kv.prefill_oneshot(*x, block=8, lens=[32, 16, 0])
    kv.fork_sequences([1, 0, 0])
    s = kv.scores()
    kv.fork_sequences([1, 0, -1])
    s2 = kv.scores()
    assert torch.equal(s[1], s2[0]) and torch.equal(s[0], s2[1]) and torch.equal(s[2], s[1]) and bool((s2[2] == 0).all())


def test_a_drafted_step_from_projection_to_cache(gpu):
    """The calls as a program uses them: one prompt, four samples of it, drafted steps on all of them."""
    import torch

    hq, hkv, d, budget, T, B = 8, 2, 128, 128, 10, 4
    kv = gpu.TreeKV(budget, hq, hkv, d, "bf16", B, 64)
    cos, sin = _tables(2048, d)
    g = torch.Generator(device="cuda").manual_seed(40)
    wq, wk = (torch.ones(d, device="cuda", dtype=kv.tdtype) for _ in range(2))
    new = lambda n: torch.randn((n, (hq + 2 * hkv) * d), generator=g, device="cuda").to(kv.tdtype)
    prompt = 190
    for c0 in range(0, prompt, 64):        # the prompt enters sequence 2 only; the others' rows are padding
        m = min(64, prompt - c0)
        pos = torch.full((B, 64), -1, dtype=torch.int32, device="cuda")
        pos[2, :m] = torch.arange(c0, c0 + m, device="cuda")
        q, k, v = kv.norm_rope(new(B * 64), wq, wk, cos, sin, pos.view(-1))
        kv.prefill_chunk(q.view(B, 64, hq, d), k.view(B, 64, hkv, d), v.view(B, 64, hkv, d), chunk_lens=[0, 0, m, 0])
    kv.fork_sequences([2] * B)
    assert [kv.tokens_seen(b) for b in range(B)] == [prompt] * B
    for step in range(12):
        rows, paths = _path_rows(B, T, [T] * B, [1 + (b + step) % 4 for b in range(B)], 50 + step)
        depth = torch.tensor([[bin(m).count("1") - 1 for m in row] for row in rows], dtype=torch.int32, device="cuda")
        seen = torch.tensor([kv.tokens_seen(b) for b in range(B)], dtype=torch.int32, device="cuda")
        q, k, v = kv.norm_rope(new(B * T), wq, wk, cos, sin, (seen[:, None] + depth).view(-1))
        q, k, v = q.view(B, T, hq, d), k.view(B, T, hkv, d), v.view(B, T, hkv, d)
        image, _ = kv.export_state()
        K, V, _, P, _ = _image_parts(torch, kv, image)
        out, lse = kv.verify_tree(q, k, v, mask=_mask_tensor(rows))
        _check_verify(kv, (K, V), seen.tolist(), (q, k, v), rows, [T] * B, out, lse, heads=[0, 5])
        took = [len(p) for p in paths]
        path = torch.tensor([(p + [0] * 4)[:4] for p in paths], dtype=torch.int32, device="cuda")
        kv.accept_path(q, k, v, lse, path, took)
        pos, cnt = kv.retained_positions()
        assert bool((pos[:, :, -1].long() == (seen + torch.tensor(took, device="cuda")).long()[:, None] - 1).all())
        kv.fork_sequences([b if (b + step) % 3 else (b + 1) % B for b in range(B)])
    st = kv.stats()
    assert st["device_error"] == 0


# ---- copies after replays of captured steps --------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d,hkv,budget,B,steps", [("bf16", 128, 2, 40, 5, 31), ("bf16", 64, 1, 300, 3, 9), ("f32", 64, 2, 33, 70, 50),
                                                        ("f32", 128, 1, 90, 2, 700)])
def test_fork_after_replayed_steps(gpu, dtype, d, hkv, budget, B, steps):
    """The copies follow the caches as they are, which replays of a captured step move without the host's counts: a twin takes
    the same steps by calls."""
    import torch

    r = np.random.default_rng(steps)
    seen = [int(x) for x in r.integers(0, 2 * budget, B)]
    seen[0] = 0
    kv, _ = _filled(gpu, dtype, d, 2 * hkv, hkv, budget, seen, 4, seed=80)
    twin, _ = _filled(gpu, dtype, d, 2 * hkv, hkv, budget, seen, 4, seed=80)
    g = torch.Generator(device="cuda").manual_seed(81)
    tok = [torch.randn((B, h, d), generator=g, device="cuda").to(kv.tdtype) for h in (2 * hkv, hkv, hkv)]
    out = torch.empty_like(tok[0])
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        kv.decode_step(*tok, out=out)
    at = 0
    for source in ([int(x) for x in r.permutation(B)], [int(x) for x in r.integers(-1, B, B)], [B - 1] * B, [(b + 1) % B for b in range(B)]):
        for _ in range(steps):
            for x in tok:
                x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
            graph.replay()
            want = twin.decode_step(*tok)
            assert torch.equal(out, want), at
            at += 1
        for c in (kv, twin):
            c.fork_sequences(source)
        (a, _), (b, _) = kv.export_state(), twin.export_state()
        assert torch.equal(a, b), source
    assert kv.stats()["device_error"] == 0


def test_fork_keeps_the_count_of_evictions(gpu):
    kv, _ = _filled(gpu, "bf16", 64, 4, 2, 30, [100, 7, 0], 4, seed=82)
    before = kv.stats()["evictions"]
    assert before == 70
    for source in ([1, 0, 2], [0, 0, 0], [-1, -1, 0], [2, 2, -1]):
        kv.fork_sequences(source)
        assert kv.stats()["evictions"] == before


def test_caches_survive_a_bad_position_as_an_image(gpu):
    import torch

    kv, _ = _filled(gpu, "bf16", 64, 4, 2, 30, [100, 7, 0], 4, seed=83)
    cos, sin = _tables(8, 64)
    kv.norm_rope(torch.zeros((1, 8 * 64), device="cuda", dtype=kv.tdtype), cos=cos, sin=sin,
                 positions=torch.tensor([8], dtype=torch.int32, device="cuda"))
    assert kv.stats(check=False)["device_error"] == BAD_INDEX
    image, tokens = kv.export_state()
    kv.reset()
    kv.import_state(image, tokens)
    assert kv.stats()["device_error"] == 0
    again, tokens2 = kv.export_state()
    assert tokens2 == tokens and torch.equal(again, image)


@pytest.mark.parametrize("dtype,d,hkv", [("bf16", 128, 2), ("bf16", 64, 1), ("f32", 128, 1)])
def test_fork_of_caches_that_only_replays_have_filled(gpu, dtype, d, hkv):
    """The host has counted one step, the caches hold hundreds of tokens: many more rows than the launch was sized for."""
    import torch

    B, budget = 4, 250
    kv, twin = (gpu.TreeKV(budget, hkv, hkv, d, dtype, B, 0) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(84)
    tok = [torch.randn((B, hkv, d), generator=g, device="cuda").to(kv.tdtype) for _ in range(3)]
    out = torch.empty_like(tok[0])
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        kv.decode_step(*tok, out=out)
    for source in ([1, 2, 3, 0], [2, 2, 2, 2], [-1, 0, -1, 1], [1, 0, 3, 2]):
        for _ in range(310):
            for x in tok:
                x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
            graph.replay()
            twin.decode_step(*tok)
        for c in (kv, twin):
            c.fork_sequences(source)
        (a, n), (b, _) = kv.export_state(), twin.export_state()
        assert torch.equal(a, b), source
        assert max(n) <= 1
    assert kv.stats()["device_error"] == 0
