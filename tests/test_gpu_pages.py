"""Prompts in pages on the GPU: attention of chunks over pages, what rows gave to tokens, eviction by accumulated weight into
the cache.  References are 64-bit; tolerances are derived where they stand.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24                       # half a step of fp32, relative
HALF = {"bf16": 2.0 ** -8, "f32": U32}  # half a step of the element type
BAD_INDEX = 256
INVALID, BAD_STATE, UNSUPPORTED = 1, 2, 4


@pytest.fixture(scope="module")
def gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2501_04987_b200 import _build

    _build.build()
    from paper_2501_04987_b200 import binding

    return binding


def _image_parts(kv, image):
    """K, V (as float32), S, positions, tokens seen, scoring start of a state image, as numpy arrays."""
    units, c, d, B = kv.batch * kv.n_kv_heads, kv.budget, kv.head_dim, kv.batch
    e = 4 if kv.dtype_code == 0 else 2
    got, at = [], 0
    for size in (units * c * d * e, units * c * d * e, units * c * 4, units * c * 4, B * 4, B * 4):
        got.append(image[at:at + size])
        at += -(-size // 256) * 256
    t = kv.torch
    shape = (B, kv.n_kv_heads, c)
    return ([x.view(kv.tdtype).view(*shape, d).float().cpu().numpy() for x in got[:2]] + [got[2].view(t.float32).view(shape).cpu().numpy()] +
            [got[3].view(t.int32).view(shape).cpu().numpy()] + [x.view(t.int32).cpu().numpy() for x in got[4:]])


class Prompts:
    """Pools, tables and the tokens in them: sequence b has past[b] tokens; everything else in the pools is NaN."""

    def __init__(self, gpu, dtype, d, hq, hkv, page, past, new, stride, seed=0, spare=3, scale=1.0):
        import torch

        g = torch.Generator(device="cuda").manual_seed(seed)
        self.kv = gpu.TreeKV(16, hq, hkv, d, dtype, len(past), 0)
        self.dtype, self.dt, self.page, self.past, self.new, self.stride = dtype, self.kv.tdtype, page, past, new, stride
        B = len(past)
        need = [-(-(p + n) // page) for p, n in zip(past, new)]
        self.width = max(max(need), 1) + 1
        self.n_pages = sum(need) + spare
        order = torch.randperm(self.n_pages, generator=g, device="cuda").to(torch.int32).tolist()
        table = [[-7] * self.width for _ in range(B)]       # entries behind the last token are not followed
        for b in range(B):
            for x in range(need[b]):
                table[b][x] = order.pop()
        self.table = torch.tensor(table, dtype=torch.int32, device="cuda")
        self.past_dev = torch.tensor(past, dtype=torch.int32, device="cuda")
        self.K, self.V = ([torch.randn((hkv, p + n, d), generator=g, device="cuda").mul(scale).to(self.dt) for p, n in zip(past, new)] for _ in range(2))
        self.kp, self.vp = (torch.full((self.n_pages, hkv, page, d), math.nan, device="cuda", dtype=self.dt) for _ in range(2))
        for b, p in enumerate(past):
            for x in range(-(-p // page)):
                m = min(page, p - x * page)
                self.kp[table[b][x], :, :m] = self.K[b][:, x * page:x * page + m]
                self.vp[table[b][x], :, :m] = self.V[b][:, x * page:x * page + m]
        self.q = torch.full((B, stride, hq, d), math.nan, device="cuda", dtype=self.dt)
        self.k, self.v = (torch.full((B, stride, hkv, d), math.nan, device="cuda", dtype=self.dt) for _ in range(2))
        for b, n in enumerate(new):
            self.q[b, :n] = torch.randn((n, hq, d), generator=g, device="cuda").mul(scale).to(self.dt)
            self.k[b, :n] = self.K[b][:, past[b]:].transpose(0, 1)
            self.v[b, :n] = self.V[b][:, past[b]:].transpose(0, 1)

    def logits(self, b):
        """[Hq, n, tokens] in 64 bits, minus infinity where a row does not see; and a bound of their error in fp32."""
        import torch

        p, n = self.past[b], self.new[b]
        G, d = self.kv.n_heads // self.kv.n_kv_heads, self.kv.head_dim
        K = self.K[b].double().repeat_interleave(G, 0)
        q = self.q[b, :n].double().transpose(0, 1)
        x = q @ K.transpose(1, 2) / math.sqrt(d)
        # d products and additions in fp32, the scale and the change to base 2: (d + 4) roundings of at most the sum of the
        # absolute terms
        err = (d + 4) * U32 * (q.abs() @ K.abs().transpose(1, 2)) / math.sqrt(d)
        sees = torch.arange(p + n, device="cuda") <= p + torch.arange(n, device="cuda")[:, None]
        return x.masked_fill(~sees, -math.inf), torch.where(sees, err, 0.0).amax(-1, keepdim=True)

    def attend(self, **kw):
        return self.kv.paged_attend(self.q, self.k, self.v, self.kp, self.vp, self.table, self.past_dev, lens=self.new, **kw)


def _check_attend(P, out, lse, finite=True):
    import torch

    G = P.kv.n_heads // P.kv.n_kv_heads
    for b, n in enumerate(P.new):
        if n == 0:
            continue
        x, err = P.logits(b)
        z = torch.logsumexp(x, -1, keepdim=True)
        w = torch.exp(x - z)
        V = P.V[b].double().repeat_interleave(G, 0)
        ref, mag = (w @ V).transpose(0, 1), (w @ V.abs()).transpose(0, 1)
        # a weight is off by its logit's error and the reference's, each once in it and once in the sum, the exponential (2^-21 of
        # the value, with the rounding of its argument) and the running sums (one rounding for each 32 keys and step); as an
        # operand it is rounded to the element type; then the output
        tokens = P.past[b] + n
        rel = 4 * err.transpose(0, 1) + 2.0 ** -19 + (tokens / 32 + 64) * U32
        lim = (HALF[P.dtype] * (1 + rel) + rel) * mag + HALF[P.dtype] * ref.abs() * (1 + HALF[P.dtype]) + 1e-30
        diff = (out[b, :n].double() - ref).abs()
        assert bool((diff <= lim).all()), "output %d off by %.3g of the limit" % (b, float((diff / lim).max()))
        lz = (2 * err + 2.0 ** -19 + (tokens / 32 + 64) * U32)[..., 0] + 4 * U32 * z[..., 0].abs()
        assert bool(((lse[b, :n].double().transpose(0, 1) - z[..., 0]).abs() <= lz).all())


def _check_pages(P):
    """The new tokens are in their pages; nothing else has changed."""
    import torch

    kp, vp = (torch.full_like(P.kp, math.nan) for _ in range(2))
    table = P.table.tolist()
    for b in range(len(P.past)):
        for t0 in range(0, P.past[b] + P.new[b], P.page):
            m = min(P.page, P.past[b] + P.new[b] - t0)
            kp[table[b][t0 // P.page], :, :m] = P.K[b][:, t0:t0 + m]
            vp[table[b][t0 // P.page], :, :m] = P.V[b][:, t0:t0 + m]
    for got, want in ((P.kp, kp), (P.vp, vp)):
        assert bool(((got == want) | (got.isnan() & want.isnan())).all())


LENGTHS = [
    ([0], [1]), ([0], [64]), ([63], [1]), ([64], [1]), ([1000], [1]), ([5], [130]),
    ([0, 17, 300, 64, 129], [3, 0, 1, 66, 2]),
    ([700, 0, 33], [40, 257, 1]),
]


@pytest.mark.parametrize("dtype,d,hq,hkv,page", [("bf16", 128, 8, 2, 16), ("bf16", 64, 3, 3, 32), ("bf16", 128, 8, 1, 64), ("bf16", 64, 4, 2, 256),
                                                 ("bf16", 128, 2, 2, 128), ("f32", 64, 4, 4, 16), ("f32", 128, 8, 1, 64), ("f32", 128, 6, 3, 256)])
@pytest.mark.parametrize("past,new", LENGTHS)
def test_attend(gpu, dtype, d, hq, hkv, page, past, new):
    import torch

    P = Prompts(gpu, dtype, d, hq, hkv, page, past, new, max(new) + 2, seed=len(past) * 1000 + sum(past))
    out = torch.full((len(past), P.stride, hq, d), 7.0, device="cuda", dtype=P.dt)
    lse = torch.full((len(past), P.stride, hq), 7.0, device="cuda")
    got = P.attend(out=out, lse=lse, max_past=max(past))
    assert got[0] is out and got[1] is lse
    _check_attend(P, out, lse)
    _check_pages(P)
    for b, n in enumerate(new):          # rows behind a sequence's tokens stay as they were
        assert bool((out[b, n:] == 7).all()) and bool((lse[b, n:] == 7).all())
    assert P.kv.stats()["device_error"] == 0


@pytest.mark.parametrize("dtype,d,hq,hkv,past,new,page", [
    ("bf16", 128, 8, 2, [9000], [1], 16), ("bf16", 128, 32, 8, [2500, 40, 3100], [300, 700, 1], 64), ("bf16", 128, 8, 8, [0], [2049], 128),
    ("bf16", 64, 8, 1, [5001], [600], 32), ("f32", 128, 8, 2, [4100, 1], [2, 70], 16), ("f32", 64, 8, 1, [20000], [2], 64), ("f32", 128, 2, 1, [9000, 17, 0], [9, 0, 30], 16), ("f32", 64, 2, 2, [70], [900], 64),
    ("bf16", 128, 8, 8, [130, 7] * 20, [200, 260] * 20, 64)])
def test_attend_long(gpu, dtype, d, hq, hkv, past, new, page):
    P = Prompts(gpu, dtype, d, hq, hkv, page, past, new, max(new), seed=7, scale=1.5)
    out, lse = P.attend()
    _check_attend(P, out, lse)
    _check_pages(P)


@pytest.mark.parametrize("d,hq,hkv,page", [(128, 16, 16, 16), (64, 32, 8, 64), (128, 32, 4, 128)])
@pytest.mark.parametrize("longest,count", [(3000, 48), (700, 48), (130, 100), (9000, 5)])
def test_attend_steps_of_ragged_batches(gpu, d, hq, hkv, page, longest, count):
    """Blocks take many short units, parts of long ones, and both."""
    past = [(7919 * i * i + 131 * i) % (longest + 1) for i in range(count)]
    past[0] = longest
    new = [1 if i % 5 else 2 for i in range(count)]
    new[count // 2] = 0
    P = Prompts(gpu, "bf16", d, hq, hkv, page, past, new, 2, seed=longest)
    for bound in (longest, None):
        out, lse = P.attend(max_past=bound)
        _check_attend(P, out, lse)
    _check_pages(P)
    assert P.kv.stats()["device_error"] == 0


@pytest.mark.parametrize("d,hq,hkv,page", [(128, 16, 4, 16), (64, 8, 8, 64), (64, 16, 2, 256), (128, 2, 2, 32)])
@pytest.mark.parametrize("longest,count,tokens", [(3000, 24, 16), (300, 60, 16), (9000, 3, 15), (2000, 30, 9), (40, 30, 32), (6000, 2, 128), (1500, 9, 60)])
def test_attend_short_chunks_of_ragged_batches(gpu, d, hq, hkv, page, longest, count, tokens):
    """17 rows a KV head and more: blocks take whole units, parts of one, ends and starts; sequences with nothing new between them."""
    past = [(7919 * i * i + 131 * i) % (longest + 1) for i in range(count)]
    past[0] = longest
    new = [(37 * i * i + 11 * i) % (tokens + 1) for i in range(count)]
    new[-1] = tokens
    P = Prompts(gpu, "bf16", d, hq, hkv, page, past, new, tokens, seed=longest)
    for bound in (longest, None):
        out, lse = P.attend(max_past=bound)
        _check_attend(P, out, lse)
    _check_pages(P)
    assert P.kv.stats()["device_error"] == 0


@pytest.mark.parametrize("d,hq,hkv", [(128, 4, 1), (64, 8, 4), (128, 8, 1)])
@pytest.mark.parametrize("past,n", [(20000, 5), (20000, 16), (20000, 33), (20000, 129), (7000, 300), (1100, 65), (1100, 257)])
def test_attend_of_one_user(gpu, d, hq, hkv, past, n):
    """Few units: the keys of each are shared by many blocks, also by more than there are tiles to share."""
    P = Prompts(gpu, "bf16", d, hq, hkv, 64, [past], [n], n + 1, seed=past + n)
    for bound in (past, 60000 if past < 5000 else None):
        out, lse = P.attend(max_past=min(bound, P.width * 64) if bound else None)
        _check_attend(P, out, lse)
    _check_pages(P)
    assert P.kv.stats()["device_error"] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new", [[3, 2], [60, 5]])
def test_tables_of_millions_of_tokens(gpu, dtype, new):
    """A table's width, and with it the largest past a launch has to expect, says nothing about how long its sequences are."""
    import torch

    P = Prompts(gpu, dtype, 64, 4, 2, 64, [700, 90], new, max(new), seed=1)
    wide = torch.full((2, 70000), -7, dtype=torch.int32, device="cuda")
    wide[:, :P.width] = P.table
    P.table = wide
    out, lse = P.attend()
    _check_attend(P, out, lse)
    s = torch.full((2, 2, 70000 * 64 + max(new)), 7.0, device="cuda")
    P.kv.paged_score(P.q, lse, P.kp, P.table, P.past_dev, s, lens=new)
    _check_score(P, lse, s)
    for b, (p, n) in enumerate(zip(P.past, new)):
        assert bool((s[b, :, p + n:] == 7).all())
    P.kv.adopt_pages(P.kp, P.vp, P.table, s, [p + n for p, n in zip(P.past, new)])
    assert P.kv.stats()["device_error"] == 0


def test_the_largest_batch(gpu):
    import torch

    for n, hq in ((1, 4), (32, 4), (40, 4), (17, 1)):
        past = [i % 90 for i in range(1024)]
        new = [(5 * i) % (n + 1) for i in range(1024)]
        new[3] = n
        P = Prompts(gpu, "bf16", 128, hq, 1, 16, past, new, n, seed=n)
        out, lse = P.attend(max_past=89)
        torch.cuda.synchronize()
        assert P.kv.stats()["device_error"] == 0
        keep = [b for b in range(1024) if b % 37 < 2 or b == 3]
        for x in ("past", "new", "K", "V"):
            setattr(P, x, [getattr(P, x)[b] for b in keep])
        P.q, out, lse = P.q[keep], out[keep], lse[keep]
        _check_attend(P, out, lse)


@pytest.mark.parametrize("dtype,new", [("bf16", [2, 1, 0]), ("bf16", [40, 3, 17]), ("bf16", [200, 300, 1]), ("f32", [3, 40, 2])])
def test_calls_on_two_streams_at_once(gpu, dtype, new):
    """Calls that overlap have nothing in common but the context: each gives what it gives alone, to the bit."""
    import torch

    P = [Prompts(gpu, dtype, 64, 8, 2, 16, [3000, 77, 500], new, max(new), seed=s) for s in range(2)]
    alone = [p.attend() for p in P]
    P[1].kv = P[0].kv
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in P]
    got = [[], []]
    for _ in range(8):
        for x, (p, s) in enumerate(zip(P, streams)):
            with torch.cuda.stream(s):
                got[x].append(p.attend())
    torch.cuda.synchronize()
    for p, one, many in zip(P, alone, got):
        for out, lse in many:
            for b, n in enumerate(p.new):
                assert torch.equal(out[b, :n], one[0][b, :n]) and torch.equal(lse[b, :n], one[1][b, :n])


def test_two_captured_calls_share_nothing(gpu):
    """Two graphs of calls that leave parts behind, replayed in turns and at once."""
    import torch

    P = [Prompts(gpu, "bf16", 128, 8, 2, 64, [9000], [n], n, seed=n) for n in (2, 30)]
    P.append(Prompts(gpu, "bf16", 128, 8, 2, 64, [5000], [150], 150, seed=3))
    alone = [p.attend() for p in P]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for p in P:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(p.attend())
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in P]
    for _ in range(3):
        for o in outs:
            o[0].zero_(), o[1].zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for a, b in zip(alone, outs):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 64), ("bf16", 64, 16), ("f32", 128, 32)])
@pytest.mark.parametrize("past,n", [(0, 200), (70, 7), (300, 150), (64, 64), (9000, 6), (9000, 40), (9000, 150)])
def test_values_that_are_not_finite(gpu, dtype, d, page, past, n):
    """A value of infinity or NaN reaches the rows that see its token and no other."""
    import torch

    P = Prompts(gpu, dtype, d, 4, 2, page, [past], [n], n, seed=past + n)
    at = {0: math.inf, n // 2: math.nan, n - 1: -math.inf}
    for j, x in at.items():
        P.v[0, j, 0, 5] = x
        P.V[0][0, past + j, 5] = x
    out, lse = P.attend()
    clean = P.V[0].clone()
    P.V[0][0, past:, 5] = torch.where(P.V[0][0, past:, 5].isfinite(), P.V[0][0, past:, 5], 0.0)
    rows = torch.arange(n, device="cuda")
    first = min(at)
    hit = rows >= first                    # rows of KV head 0 from here on see an infinity or a NaN in channel 5
    got = out[0, :, :2, 5].double()
    w = None
    bad = torch.zeros(n, dtype=torch.float64, device="cuda")
    for j, x in sorted(at.items()):
        bad[j:] += x
    assert bool(torch.where(hit[:, None], (got == bad[:, None]) | (got.isnan() & bad.isnan()[:, None]), got.isfinite()).all())
    ok = out.clone()
    ok[0, :, :2, 5] = 0.0
    assert bool(ok.isfinite().all())
    P.V[0] = clean
    P.V[0][0, :, 5] = 0.0                   # everything else is as without them
    ok2 = ok.clone()
    _check_attend(P, ok2, lse)


def test_infinite_keys_behind_a_row(gpu):
    """Keys of NaN or infinity leave the rows in front of them alone."""
    import torch

    for dtype in ("bf16", "f32"):
        P = Prompts(gpu, dtype, 64, 2, 1, 16, [20], [100], 100)
        P.k[0, 50, 0, 3], P.k[0, 51, 0, 4] = math.nan, math.inf
        out, lse = P.attend()
        got = out[0, :50].clone(), lse[0, :50].clone()
        Q = Prompts(gpu, dtype, 64, 2, 1, 16, [20], [100], 100)
        ref = Q.attend()
        assert torch.equal(got[0], ref[0][0, :50]) and torch.equal(got[1], ref[1][0, :50])
        s = torch.zeros((1, 1, 120), device="cuda")
        lens = [50]
        P.kv.paged_score(P.q, lse, P.kp, P.table, P.past_dev, s, lens=lens)
        assert bool(s.isfinite().all()) and bool((s[0, 0, 70:] == 0).all())


@pytest.mark.parametrize("dtype,n", [("bf16", 3), ("bf16", 40), ("bf16", 300), ("f32", 40)])
def test_keys_that_are_nan_or_infinite_reach_every_row_that_sees_them(gpu, dtype, n):
    """Wherever in a tile the key stands."""
    import torch

    for at in (0, 2, 5, 6, 7, 31, 63, 64, 70, 127, 133):
        P = Prompts(gpu, dtype, 64, 2, 1, 16, [134], [n], n, seed=at)
        P.kp[P.table[0, at // 16], 0, at % 16, 3] = math.nan
        out, lse = P.attend()
        assert bool(out.isnan().all()) and bool(lse.isnan().all())
        s = torch.zeros((1, 1, 134 + n), device="cuda")
        P.kv.paged_score(P.q, torch.full_like(lse, 3.0), P.kp, P.table, P.past_dev, s)
        want = torch.zeros(134 + n, dtype=torch.bool, device="cuda")
        want[at] = True
        assert torch.equal(s[0, 0].isnan(), want)


def test_shared_pages_and_an_identical_table(gpu):
    """Sequences that share the pages of a prefix, and the first page used twice by one."""
    import torch

    P = Prompts(gpu, "bf16", 128, 4, 1, 16, [64, 64, 32], [5, 9, 1], 9)
    P.table[1, :4] = P.table[0, :4]
    P.table[2, :2] = P.table[0, 0]
    P.K[1][:, :64], P.V[1][:, :64] = P.K[0][:, :64], P.V[0][:, :64]
    for x in (P.K, P.V):
        x[2][:, :16] = x[0][:, :16]
        x[2][:, 16:32] = x[0][:, :16]
    out, lse = P.attend()
    _check_attend(P, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_pages_and_lengths_are_not_followed(gpu, dtype):
    import torch

    P = Prompts(gpu, dtype, 64, 4, 2, 16, [40, 40, 40, 40], [3, 3, 3, 3], 3)
    P.table[0, 2] = P.n_pages          # the page the new tokens go to, and are read from
    P.table[1, 0] = -1
    P.past_dev[2] = 5000
    before = P.kp.clone()
    out, lse = torch.full((4, 3, 4, 64), 7.0, device="cuda", dtype=P.dt), torch.full((4, 3, 4), 7.0, device="cuda")
    P.attend(out=out, lse=lse, max_past=41)
    st = P.kv.stats(check=False)
    assert st["device_error"] == BAD_INDEX and st["status"] == INVALID
    assert bool((out[2] == 7).all()) and bool((lse[2] == 7).all())     # the sequence sat the call out
    changed = ((P.kp != before) & ~(P.kp.isnan() & before.isnan())).any(-1).any(1).any(1)
    table = P.table.tolist()
    assert set(changed.nonzero()[:, 0].tolist()) == {table[1][2], table[3][2]}
    P.past, P.new = [40], [3]
    P.K, P.V, P.q = [P.K[3]], [P.V[3]], P.q[3:]
    _check_attend(P, out[3:], lse[3:])
    kv = P.kv
    kv.reset()
    s = torch.full((4, 2, 48), 7.0, device="cuda")
    q = torch.randn((4, 3, 4, 64), device="cuda").to(P.dt)
    kv.paged_score(q, torch.zeros((4, 3, 4), device="cuda"), P.kp, P.table, P.past_dev, s, lens=[0, 0, 3, 0], max_past=41)
    assert kv.stats(check=False)["device_error"] == BAD_INDEX and bool((s == 7).all())


def test_captured_call_replays_while_the_sequence_grows(gpu):
    """Two captured steps that share the pool, replayed; beside them an eager call on another stream."""
    import torch

    for dtype in ("bf16", "f32"):
        P = Prompts(gpu, dtype, 128, 4, 2, 16, [30, 0, 100], [4, 4, 4], 4)
        out, lse = torch.zeros((3, 1, 4, 128), device="cuda", dtype=P.dt), torch.zeros((3, 1, 4), device="cuda")
        q, k, v = (torch.zeros_like(x[:, :1]) for x in (P.q, P.k, P.v))
        past = P.past_dev.clone()
        whole = P.attend()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            P.kv.paged_attend(q, k, v, P.kp, P.vp, P.table, past, out=out, lse=lse, max_past=110)
            past.add_(1)
        for i in range(4):
            for dst, src in ((q, P.q), (k, P.k), (v, P.v)):
                dst.copy_(src[:, i:i + 1])
            graph.replay()
            # same keys and values, other splits of the work: each within the limits of _check_attend, here with a sum of |q k| /
            # sqrt d of at most 16 and of weighted |v| of at most 4
            err = 132 * U32 * 16
            rel = 4 * err + 2.0 ** -18
            assert bool(((out[:, 0].float() - whole[0][:, i].float()).abs() <= 2 * 4 * (2 * HALF[dtype] + rel)).all())
            assert bool(((lse[:, 0] - whole[1][:, i]).abs() <= 2 * (2 * err + 2.0 ** -18)).all())
        assert past.tolist() == [34, 4, 104]
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            again = P.attend()
        other.synchronize()
        assert torch.equal(again[0], whole[0]) and torch.equal(again[1], whole[1])


def test_offsets_beyond_32_bits(gpu):
    """Pages whose elements lie beyond 2^32, read, written, weighed and adopted."""
    import torch

    page, hkv, d = 256, 8, 128
    n_pages = 2 ** 32 // (page * hkv * d) + 8
    kv = gpu.TreeKV(64, 8, hkv, d, "bf16", 1, 0)
    kp, vp = (torch.empty((n_pages, hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    P = Prompts(gpu, "bf16", d, 8, hkv, page, [300], [20], 20)
    table = torch.tensor([[n_pages - 1, n_pages - 3, 0]], dtype=torch.int32, device="cuda")
    for x in range(2):
        m = min(page, 300 - x * page)
        kp[table[0, x], :, :m], vp[table[0, x], :, :m] = P.K[0][:, x * page:x * page + m], P.V[0][:, x * page:x * page + m]
    out, lse = kv.paged_attend(P.q, P.k, P.v, kp, vp, table, P.past_dev)
    _check_attend(P, out, lse)
    s = torch.zeros((1, hkv, 320), device="cuda")
    kv.paged_score(P.q, lse, kp, table, P.past_dev, s)
    _check_score(P, lse, s)
    kv.adopt_pages(kp, vp, table, s, [320])
    img, _ = kv.export_state()
    K, V, S, pos = _image_parts(kv, img)[:4]
    for h in range(hkv):
        at = torch.tensor(pos[0, h], device="cuda").long()
        assert np.array_equal(K[0, h], P.K[0][h, at].float().cpu().numpy()) and np.array_equal(V[0, h], P.V[0][h, at].float().cpu().numpy())


# ---- what rows gave ---------------------------------------------------------------------------------------------------
def _check_score(P, lse, s, before=None):
    import torch

    G = P.kv.n_heads // P.kv.n_kv_heads
    for b, n in enumerate(P.new):
        if n == 0:
            continue
        x, err = P.logits(b)
        w = torch.exp(x - lse[b, :n].transpose(0, 1)[..., None].double())
        ref = w.view(-1, G * n, w.shape[-1]).sum(1) / G
        # each weight: its logit's error, the exponential (2^-21), the roundings of its argument - the log-sum-exp in base 2, the
        # factor and the result; sums of at most 128 in one rounding each, then compensated; the mean and the addition
        far = torch.where(x.isinf(), 0.0, x).abs() + 2 * lse[b, :n].transpose(0, 1)[..., None].double().abs()
        mag = w * (2 * err + 2.0 ** -21 + (2 * far + 140) * U32)
        lim = mag.view(-1, G * n, w.shape[-1]).sum(1) / G + 1e-30
        want = ref if before is None else ref + before[b, :, :P.past[b] + n].double()
        lim = lim + 2 * U32 * want.abs()
        diff = (s[b, :, :P.past[b] + n].double() - want).abs()
        assert bool((diff <= lim).all()), "weights %d off by %.3g of the limit" % (b, float((diff / lim).max()))


@pytest.mark.parametrize("dtype,d,hq,hkv,page", [("bf16", 128, 8, 2, 16), ("bf16", 64, 3, 3, 32), ("bf16", 128, 8, 1, 64), ("bf16", 64, 4, 2, 256),
                                                 ("f32", 64, 4, 4, 16), ("f32", 128, 8, 1, 128)])
@pytest.mark.parametrize("past,new", LENGTHS + [([900], [1100]), ([3000, 10], [40, 300]), ([40, 7] * 25, [33, 1] * 25)])
def test_score(gpu, dtype, d, hq, hkv, page, past, new):
    import torch

    P = Prompts(gpu, dtype, d, hq, hkv, page, past, new, max(new) + 1, seed=sum(new))
    _, lse = P.attend()
    top = max(p + n for p, n in zip(past, new)) + 3 + max(new)
    s = torch.full((len(past), hkv, top), 7.0, device="cuda")
    P.kv.paged_score(P.q, lse, P.kp, P.table, P.past_dev, s, lens=new, max_past=max(past))
    _check_score(P, lse, s)
    for b, n in enumerate(new):
        assert bool((s[b, :, past[b] + n if n else 0:] == 7).all())
    again = s.clone()
    P.kv.paged_score(P.q, lse, P.kp, P.table, P.past_dev, again, lens=new, max_past=max(past))
    assert torch.equal(again, s)         # one order of additions
    before = torch.rand(s.shape, device="cuda")
    more = before.clone()
    P.kv.paged_score(P.q, lse, P.kp, P.table, P.past_dev, more, lens=new, add=True)
    _check_score(P, lse, more, before)
    assert P.kv.stats()["device_error"] == 0


def test_score_of_rows_that_give_nothing(gpu):
    import torch

    for dtype in ("bf16", "f32"):
        P = Prompts(gpu, dtype, 64, 4, 2, 16, [30], [40], 40)
        _, lse = P.attend()
        lse[0, 10:30] = math.inf
        lse[0, 30:] = -math.inf
        s = torch.empty((1, 2, 70), device="cuda")
        P.kv.paged_score(P.q, lse, P.kp, P.table, P.past_dev, s)
        P.new, P.K = [10], [P.K[0][:, :40]]
        _check_score(P, lse, s)
        assert bool((s[0, :, 40:] == 0).all())


# ---- eviction by accumulated weight -----------------------------------------------------------------------------------
def _adopt_ref(s, n, first, c, ns, nr, average):
    """Tokens that stay, in order, of one KV head."""
    w = np.asarray(s[:n], dtype=np.float32)
    if average:
        w = w / (n - np.maximum(np.arange(n), first)).astype(np.float32)
    if n <= c:
        return list(range(n))
    key = [(1, 0.0) if math.isnan(x) else (0, -float(x)) for x in w]
    free = sorted(range(ns, n - nr), key=lambda t: key[t] + (t,))[:c - ns - nr]
    return list(range(ns)) + sorted(free) + list(range(n - nr, n))


@pytest.mark.parametrize("dtype,d,hq,hkv,page", [("bf16", 128, 8, 2, 16), ("bf16", 64, 3, 3, 64), ("f32", 64, 4, 4, 256), ("f32", 128, 8, 1, 32)])
@pytest.mark.parametrize("budget,protect,lens", [(16, None, [0, 1, 15, 16, 17, 40]), (64, (4, 20), [500, 64, 65, 3, 0, 2000]),
                                                 (33, (2, 0), [9000, 10, 34, 100, 66, 67]), (300, (0, 298), [301, 900, 0, 299, 6000, 300])])
@pytest.mark.parametrize("average", [True, False])
def test_adopt(gpu, dtype, d, hq, hkv, page, budget, protect, lens, average):
    import torch

    B = len(lens)
    P = Prompts(gpu, dtype, d, hq, hkv, page, lens, [0] * B, 1)
    kv = gpu.TreeKV(budget, hq, hkv, d, dtype, B, 0)
    if protect:
        kv.set_protection(*protect)
    if not average:
        kv.set_rule(gpu.RULE_ACCUMULATED)
    q, k, v = (torch.randn((B, h, d), device="cuda").to(P.dt) for h in (hq, hkv, hkv))
    for _ in range(3):                       # caches that hold something: a prompt takes its place, a length of zero leaves it
        kv.decode_step(q, k, v)
    held = _image_parts(kv, kv.export_state()[0])
    first = [max(0, n - 30) if i % 2 else 0 for i, n in enumerate(lens)]
    s = torch.rand((B, hkv, max(lens) + 5), device="cuda").pow(3)
    s[:, :, ::3] = torch.round(s[:, :, ::3] * 8) / 8       # many equal ones
    s[:, 0, 7::50] = math.nan
    s[:, -1, 9::41] = math.inf
    s[:, -1, 11::43] = -0.0
    s[:, -1, 12::43] = 0.0
    s[:, -1, 13::47] = -3.5
    kv.adopt_pages(P.kp, P.vp, P.table, s, lens, first=first)
    img, seen = kv.export_state()
    K, V, S, pos, seen_dev, w0 = _image_parts(kv, img)
    sc = s.cpu().numpy()
    ns, nr = protect or (0, 0)
    for b, n in enumerate(lens):
        if n == 0:
            assert seen[b] == 3 and np.array_equal(pos[b], held[3][b]) and np.array_equal(K[b], held[0][b]) and np.array_equal(S[b], held[2][b])
            continue
        assert seen[b] == n == seen_dev[b] and w0[b] == first[b] and kv.tokens_seen(b) == n
        for h in range(hkv):
            kept = _adopt_ref(sc[b, h], n, first[b], budget, ns, nr, average)
            L = len(kept)
            assert pos[b, h, :L].tolist() == kept and (pos[b, h, L:] == -1).all()
            assert np.array_equal(S[b, h, :L], sc[b, h, kept], equal_nan=True)
            at = torch.tensor(kept, device="cuda")
            assert np.array_equal(K[b, h, :L], P.K[b][h, at].float().cpu().numpy())
            assert np.array_equal(V[b, h, :L], P.V[b][h, at].float().cpu().numpy())
    assert kv.stats()["device_error"] == 0


@pytest.mark.parametrize("n,value", [(50000, None), (70001, 0.25), (20000, 0.0), (9000, None), (450000, None), (900000, None), (900000, 0.5)])
def test_adopt_long_and_equal_weights(gpu, n, value):
    """Few units: clusters share one; all weights equal: the oldest stay."""
    import torch

    P = Prompts(gpu, "bf16", 64, 2, 1, 256, [n], [0], 1)
    kv = gpu.TreeKV(777, 2, 1, 64, "bf16", 1, 0)
    kv.set_rule(gpu.RULE_ACCUMULATED)
    s = torch.rand((1, 1, n), device="cuda") if value is None else torch.full((1, 1, n), value, device="cuda")
    kv.adopt_pages(P.kp, P.vp, P.table, s, [n])
    pos, count = kv.retained_positions()
    assert pos[0, 0].tolist() == _adopt_ref(s[0, 0].cpu().numpy(), n, 0, 777, 0, 0, False) and int(count) == 777


# ---- refusals ----------------------------------------------------------------------------------------------------------
def test_refusals(gpu):
    import torch

    P = Prompts(gpu, "bf16", 64, 4, 2, 16, [20, 5], [2, 2], 2)
    kv = P.kv
    good = dict(q=P.q, k=P.k, v=P.v, k_pages=P.kp, v_pages=P.vp, table=P.table, past=P.past_dev)
    for name, wrong in (("q", P.q.float()), ("k", P.k[:, :1]), ("v", P.v.transpose(1, 2)), ("k_pages", P.kp[:, :1]), ("v_pages", P.vp[:-1]),
                        ("table", P.table.long()), ("table", P.table[:1]), ("past", P.past_dev.long()), ("past", P.past_dev.cpu())):
        with pytest.raises(ValueError):
            kv.paged_attend(**dict(good, **{name: wrong}))
    with pytest.raises(ValueError):
        kv.paged_attend(**good, lens=[1])
    for kw in (dict(lens=[3, 0]), dict(lens=[-1, 0]), dict(max_past=-1), dict(max_past=P.width * 16 + 1)):
        with pytest.raises(gpu.TreeKVError) as e:
            kv.paged_attend(**good, **kw)
        assert e.value.status == INVALID
    for page in (8, 24, 512):
        pool = torch.zeros((4, 2, page, 64), device="cuda", dtype=torch.bfloat16)
        with pytest.raises(gpu.TreeKVError) as e:
            kv.paged_attend(**dict(good, k_pages=pool, v_pages=pool))
        assert e.value.status == UNSUPPORTED
    lse = torch.zeros((2, 2, 4), device="cuda")
    with pytest.raises(gpu.TreeKVError) as e:                # rows would reach past the scores
        kv.paged_score(P.q, lse, P.kp, P.table, P.past_dev, torch.zeros((2, 2, 21), device="cuda"), max_past=20)
    assert e.value.status == INVALID
    s = torch.zeros((2, 2, 64), device="cuda")
    for lens, first in (([64 + 1, 0], None), ([-1, 0], None), ([10, 0], [10, 0]), ([10, 0], [-1, 0])):
        with pytest.raises(gpu.TreeKVError) as e:
            kv.adopt_pages(P.kp, P.vp, P.table, s, lens, first=first)
        assert e.value.status == INVALID
    with pytest.raises(ValueError):
        kv.adopt_pages(P.kp, P.vp, P.table, s, None)
    kv.set_rule(gpu.RULE_KEEP_LEFT)
    with pytest.raises(gpu.TreeKVError) as e:
        kv.adopt_pages(P.kp, P.vp, P.table, s, [10, 0])
    assert e.value.status == UNSUPPORTED
    kv.set_rule(gpu.RULE_SCORES)
    cos = torch.ones((64, 32), device="cuda")
    kv.set_positions(cos, cos)
    with pytest.raises(gpu.TreeKVError) as e:
        kv.adopt_pages(P.kp, P.vp, P.table, s, [10, 0])
    assert e.value.status == UNSUPPORTED
    kv.set_positions(None, None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(gpu.TreeKVError) as e:
            kv.adopt_pages(P.kp, P.vp, P.table, s, [10, 0])
        x = s + 1
    assert e.value.status == BAD_STATE
    assert kv.stats()["device_error"] == 0 and kv.tokens_seen(0) == 0 and kv.stats()["kernel_launches"] == 1
    kv.paged_attend(**good, lens=[0, 0])                     # nothing to do is no error
    kv.adopt_pages(P.kp, P.vp, P.table, s, [0, 0])
    assert kv.stats()["kernel_launches"] == 1
