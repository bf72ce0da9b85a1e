"""The accepted path of a draft on the GPU, against its definition in 64 bits and against the distribution that it must leave;
and a prompt's whole way: pages, weights, eviction into the cache, drafted decoding.
"""
import math

import numpy as np
import pytest

from test_gpu_pages import BAD_INDEX, INVALID, UNSUPPORTED, Prompts, _adopt_ref, _check_attend, _check_score

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2501_04987_b200 import _build

    _build.build()
    from paper_2501_04987_b200 import binding

    return binding


def _ref(logits, tokens, uniform, noise, parents, q, temperature):
    """One sequence: (path, next token), and whether a comparison was too close to tell in 32 bits."""
    n, path, close = len(parents), [0], False
    V = logits.shape[1]
    while True:
        x = logits[path[-1]].astype(np.float64)
        kids = [i for i in range(n) if parents[i] == path[-1] and i > path[-1]]
        if temperature == 0:
            if np.isnan(x).any() or not (x > -np.inf).any():
                return path, -1, close
            best = int(np.argmax(x))
            hit = [i for i in kids if tokens[i] == best]
            if not hit:
                return path, best, close
            path.append(hit[0])
            continue
        top = x.max()
        if not np.isfinite(top):
            return path, -1, close
        r = np.exp((x - top) / temperature)
        r /= r.sum()
        hit = None
        for i in kids:
            t = tokens[i]
            if not 0 <= t < V:
                continue
            a, b = uniform[i] * (1.0 if q is None else q[path[-1], t]) * r.sum(), r[t]
            close |= abs(a - b) <= 1e-4 * max(a, b)
            if a < b:
                hit = i
                break
            if q is None:
                r = r.copy()
                r[t] = 0.0
            else:
                r = np.maximum(r / r.sum() - q[path[-1]], 0.0)
        if hit is not None:
            path.append(hit)
            continue
        z = r / noise
        best = int(np.argmax(z))
        second = np.partition(z, -2)[-2] if V > 1 else 0.0
        close |= second >= (1 - 1e-4) * z[best]
        return path, best, close


def _trees(rng, B, T, kind):
    lens, parents = [], []
    for b in range(B):
        n = int(rng.integers(0, T + 1)) if b % 3 else T
        lens.append(n)
        parents.append([-1 if i == 0 else i - 1 if kind == "chain" else 0 if kind == "star" else int(rng.integers(max(-1, i - 5), i)) for i in range(n)])
    return lens, parents


def _masks(parents, T):
    rows = []
    for up in parents:
        bits = []
        for i, p in enumerate(up):
            bits.append((bits[p] if p >= 0 else 0) | (1 << i))
        rows.append([x - (1 << 64) if x >> 63 else x for x in bits + [0] * (T - len(up))])
    return rows


@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (1, 8, 2), (5, 3, 50), (7, 64, 333), (3, 16, 4099), (40, 7, 1000), (2, 5, 40001), (1, 33, 128000), (300, 4, 70), (2, 3, 300001), (150, 2, 20001)])
@pytest.mark.parametrize("kind", ["chain", "tree", "star"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("given,temperature", [(False, 1.0), (True, 1.0), (False, 0.6), (True, 1.7), (False, 0.0)])
def test_path(gpu, B, T, V, kind, dtype, given, temperature):
    import torch

    rng = np.random.default_rng(B * 100000 + T * 1000 + V)
    lens, parents = _trees(rng, B, T, kind)
    g = torch.Generator(device="cuda").manual_seed(V + T)
    logits = (2 * torch.randn((B, T, V), generator=g, device="cuda"))
    tokens = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
    own = torch.rand((B, T), generator=g, device="cuda") < 0.5       # half of the drafted tokens are likely
    for i in range(1, T):
        up = [p[i] if i < len(p) else 0 for p in parents]
        for b in range(B):
            if own[b, i] and up[b] >= 0:
                logits[b, up[b], tokens[b, i].long()] = math.log(V) + 2.0
    logits = logits.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    q = torch.softmax(1.5 * torch.randn((B, T, V), generator=g, device="cuda"), -1) if given else None
    if q is not None:
        q[:, ::2] = torch.softmax(logits[:, ::2].float() + 0.3 * q[:, ::2] * V, -1)
    uniform = torch.rand((B, T), generator=g, device="cuda")
    noise = torch.empty((B, V), device="cuda").exponential_(generator=g)
    kv = gpu.TreeKV(16, 2, 2, 64, "bf16", B, 0)
    mask = None if kind == "chain" else torch.tensor(_masks(parents, T), dtype=torch.int64, device="cuda")
    warm = temperature > 0
    path, count, after = (x.cpu().numpy() for x in kv.pick_path(logits, tokens, uniform if warm else None, noise if warm else None, mask=mask,
                                                                lens=lens, draft=q, temperature=temperature))
    l, t, u, e = (x.float().cpu().numpy() if x.dtype != torch.int32 else x.cpu().numpy() for x in (logits, tokens, uniform, noise))
    told = 0
    for b in range(B):
        if lens[b] == 0:
            assert count[b] == 0 and after[b] == -1 and (path[b] == -1).all()
            continue
        way, best, close = _ref(l[b], t[b], u[b].astype(np.float64), e[b].astype(np.float64), parents[b],
                                None if q is None else q[b].double().cpu().numpy(), temperature)
        if close:       # (within 1e-4 of a draw: 32 bits may fall on the other side)
            continue
        told += 1
        assert path[b].tolist() == way + [-1] * (T - len(way)) and count[b] == len(way) and after[b] == best, b
    assert told >= 0.9 * sum(n > 0 for n in lens) - 1
    assert kv.stats()["device_error"] == 0


@pytest.mark.parametrize("given", [False, True])
def test_first_token_is_distributed_as_the_target(gpu, given):
    """Two children of the root, drawn from q: the token that follows the root - the accepted child's, or the next one - has the
    target's distribution."""
    import torch

    B, V, rounds = 1024, 6, 200
    kv = gpu.TreeKV(16, 2, 2, 64, "bf16", B, 0)
    g = torch.Generator(device="cuda").manual_seed(1)
    row, qrow = torch.tensor([0.3, -1.0, 1.2, 0.0, -0.4, 0.9], device="cuda"), torch.tensor([0.4, 0.1, 0.05, 0.25, 0.1, 0.1], device="cuda")
    logits = row.expand(B, 3, V).contiguous()
    draft = qrow.expand(B, 3, V).contiguous() if given else None
    mask = torch.tensor([[1, 3, 5]], dtype=torch.int64, device="cuda").expand(B, 3).contiguous()
    seen = torch.zeros(V, device="cuda")
    for _ in range(rounds):
        tokens = torch.multinomial(qrow, B * 3, replacement=True, generator=g).view(B, 3).to(torch.int32)
        uniform, noise = torch.rand((B, 3), generator=g, device="cuda"), torch.empty((B, V), device="cuda").exponential_(generator=g)
        path, count, after = kv.pick_path(logits, tokens, uniform, noise, mask=mask, draft=draft)
        first = torch.where(count > 1, tokens.gather(1, path[:, 1:2].clamp(min=0).long())[:, 0], after)
        seen += torch.bincount(first.long(), minlength=V).float()
    p = torch.softmax(row.double(), 0).cpu()
    N = B * rounds
    # a binomial count strays by more than five standard deviations about once in two million
    assert bool(((seen.double().cpu() - N * p).abs() <= 5 * (N * p * (1 - p)).sqrt()).all())


def test_rows_that_hold_no_choice(gpu):
    """NaN and infinite logits, rows of minus infinity, tokens outside the vocabulary, a distribution equal to the draft's."""
    import torch

    B, T, V = 6, 3, 1000
    kv = gpu.TreeKV(16, 2, 2, 64, "bf16", B, 0)
    logits = torch.randn((B, T, V), device="cuda")
    tokens = torch.full((B, T), 5, dtype=torch.int32, device="cuda")
    logits[0, 0, 77] = math.nan
    logits[1, 0, 78] = math.inf
    logits[2, 0] = -math.inf
    tokens[3, 1] = V
    tokens[4, 1] = -1
    logits[5, 0] = -math.inf
    logits[5, 0, 5], logits[5, 0, 6] = 1.0, 1.0
    uniform, noise = torch.full((B, T), 0.999, device="cuda"), torch.ones((B, V), device="cuda")
    uniform[5, 1] = 0.25
    for t in (1.0, 0.0):
        kv.reset()
        path, count, after = (x.tolist() for x in kv.pick_path(logits, tokens, uniform, noise, temperature=t))
        assert after[:3] == [-1, -1 if t else 78, -1] and count[:3] == [1, 1, 1]
        for b in (3, 4):
            assert count[b] == 1 and after[b] == int(logits[b, 0].argmax())
        assert count[5] >= 2 and path[5][:2] == [0, 1]
        st = kv.stats(check=False)
        assert st["device_error"] == BAD_INDEX and st["status"] == INVALID
    # the draft's distribution is the target's: accepted whatever the number, or, rounded the other way, another token of it
    kv.reset()
    q = torch.softmax(logits, -1)
    q[:3] = 1.0 / V
    logits[:3] = 0.0
    tokens.clamp_(0, V - 1)
    path, count, after = kv.pick_path(logits, tokens, torch.full((B, T), 1.0 - 2.0 ** -24, device="cuda"), noise, draft=q)
    assert bool(((after >= 0) & (after < V)).all()) and kv.stats()["device_error"] == 0
    # T so small that one logit is all, and an odd row start
    path, count, after = kv.pick_path(logits[..., :333].contiguous(), tokens, uniform, noise[:, :333].contiguous(), temperature=1e-6)
    assert bool((after >= 0).all())


def test_pick_refusals_and_capture(gpu):
    import torch

    kv = gpu.TreeKV(16, 2, 2, 64, "bf16", 2, 0)
    L, t, u, e = torch.randn((2, 4, 50), device="cuda"), torch.zeros((2, 4), dtype=torch.int32, device="cuda"), torch.rand((2, 4), device="cuda"), torch.rand((2, 50), device="cuda") + 0.1
    for kw in (dict(logits=L.half()), dict(logits=L[:, :3]), dict(tokens=t.long()), dict(uniform=u[:1]), dict(noise=e.double()), dict(noise=e[:, :49]),
               dict(mask=t), dict(draft=L.bfloat16()), dict(lens=[1])):
        with pytest.raises(ValueError):
            kv.pick_path(**dict(dict(logits=L, tokens=t, uniform=u, noise=e), **kw))
    for kw in (dict(lens=[5, 0]), dict(lens=[0, -1]), dict(temperature=-1.0), dict(temperature=math.nan), dict(uniform=None), dict(noise=None)):
        with pytest.raises(gpu.TreeKVError) as err:
            kv.pick_path(**dict(dict(logits=L, tokens=t, uniform=u, noise=e), **kw))
        assert err.value.status == INVALID
    big = torch.zeros((2, 65, 50), device="cuda")
    with pytest.raises(gpu.TreeKVError):
        kv.pick_path(big, torch.zeros((2, 65), dtype=torch.int32, device="cuda"), torch.zeros((2, 65), device="cuda"), e)
    want = [x.clone() for x in kv.pick_path(L, t, u, e)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = kv.pick_path(L, t, u, e)
    for x in got:
        x.fill_(9)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 8, 2, 128), ("f32", 4, 4, 64)])
def test_prompt_to_drafted_decoding(gpu, dtype, hq, hkv, d):
    """A prompt chunk by chunk into pages, its window's weights, eviction into the cache, a drafted step with the path that the
    logits give - and the cache goes on as one that was given the same tokens through a state image."""
    import torch

    B, budget, page, window, T, V = 2, 96, 16, 24, 6, 211
    total = [260, 75]
    P = Prompts(gpu, dtype, d, hq, hkv, page, [0, 0], total, max(total), seed=5)
    kv, other = (gpu.TreeKV(budget, hq, hkv, d, dtype, B, 16) for _ in range(2))
    for x in (kv, other):
        x.set_protection(2, 8)
    out, lse = torch.zeros((B, P.stride, hq, d), device="cuda", dtype=P.dt), torch.zeros((B, P.stride, hq), device="cuda")
    done = 0
    while done < max(total):
        m = min(100, max(total) - done)
        lens = [max(0, min(m, n - done)) for n in total]
        part = [x[:, done:done + m].contiguous() for x in (P.q, P.k, P.v)]
        past = torch.tensor([min(done, n) for n in total], dtype=torch.int32, device="cuda")
        o, z = kv.paged_attend(*part, P.kp, P.vp, P.table, past, lens=lens)
        for b in range(B):
            out[b, done:done + lens[b]], lse[b, done:done + lens[b]] = o[b, :lens[b]], z[b, :lens[b]]
        done += m
    _check_attend(P, out, lse)
    first = [n - window for n in total]
    qw, lw = (torch.stack([x[b, first[b]:total[b]] for b in range(B)]) for x in (P.q, lse))
    s = torch.zeros((B, hkv, max(total)), device="cuda")
    kv.paged_score(qw, lw, P.kp, P.table, torch.tensor(first, dtype=torch.int32, device="cuda"), s)
    P.past, P.new, q_all, P.q = first, [window] * B, P.q, qw
    _check_score(P, lw, s)
    kv.adopt_pages(P.kp, P.vp, P.table, s, total, first=first)
    pos, count = kv.retained_positions()
    for b in range(B):
        for h in range(hkv):
            kept = _adopt_ref(s[b, h].cpu().numpy(), total[b], first[b], budget, 2, 8, True)
            assert pos[b, h, :len(kept)].tolist() == kept
    image, seen = kv.export_state()
    other.import_state(image, seen)
    g = torch.Generator(device="cuda").manual_seed(3)
    head = torch.randn((hq * d, V), generator=g, device="cuda") * 0.1
    for step in range(3):
        q, k, v = (torch.randn((B, T, h, d), generator=g, device="cuda").to(P.dt) for h in (hq, hkv, hkv))
        tokens = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
        uniform, noise = torch.rand((B, T), generator=g, device="cuda") * 0.02, torch.empty((B, V), device="cuda").exponential_(generator=g)
        mask = torch.tensor(_masks([[-1, 0, 0, 1, 2, 4]] * B, T), dtype=torch.int64, device="cuda")
        res = []
        for x in (kv, other):
            o, z = x.verify_tree(q, k, v, mask=mask)
            logits = o.float().view(B, T, hq * d) @ head
            path, cnt, after = x.pick_path(logits, tokens, uniform, noise, mask=mask)
            x.accept_path(q, k, v, z, path.clamp(min=0), cnt.tolist())
            res.append((o, z, path, cnt, after, *x.retained_positions(), x.scores()))
        assert all(torch.equal(a, b) for a, b in zip(*res))
        up = [-1, 0, 0, 1, 2, 4]
        for b in range(B):
            way, best, close = _ref(logits[b].cpu().numpy(), tokens[b].tolist(), uniform[b].double().cpu().numpy(), noise[b].double().cpu().numpy(), up, None, 1.0)
            assert close or (path[b, :len(way)].tolist() == way and int(cnt[b]) == len(way) and int(after[b]) == best)
    assert kv.tokens_seen(0) > total[0] and kv.stats()["device_error"] == 0
