"""Measured cases of the operators around drafted decoding on the fixed-budget cache.

Four operators, named by the case's "op":

  qk      split of a packed projection row into q, k, v with a norm of every query and key head and the position
          rotation in the same pass
  verify  attention of a tree of drafted tokens over the cache, which it leaves as it is
  step    verify, then the accepted path of the tree enters the cache: append, score update, evictions of Algorithm 1
  fork    sequences of a batch become copies of others (beam reorder, one prompt for many samples), or are freed

With `own` false, run() computes them with elementary torch operations in 32 bits; with `own` true it makes the
library's calls.  The cache is kept in the library's slab layout for the operators that change it: with N tokens seen and
budget c, L = min(N, c) tokens are cached, i = max(N - c, 0) mod c evictions of the running cycle are done, and the live
rows of a slab are [0, i) and [2i, L + i) in cache order.
"""
import math
import random

import torch

own = False

ALIGN = 256          # parts of the workspace and of a state image start on such a boundary
EPS = 1e-6
BASE = 5e5           # rotary base


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    gqa = dict(batch=32, heads=32, kv_heads=8, dim=128, budget=2048, dtype="bf16")
    mha = dict(batch=8, heads=32, kv_heads=32, dim=128, budget=1024, dtype="bf16")
    return [
        # one decode step of 32 sequences, grouped heads: latency
        dict(name="qk_step", op="qk", tokens=32, heads=32, kv_heads=8, dim=128, dtype="bf16", slots=16384, pad=0, norm=True),
        # four sequences' chunks of 1024 tokens
        dict(name="qk_chunk", op="qk", tokens=4096, heads=32, kv_heads=8, dim=128, dtype="bf16", slots=131072, pad=0, norm=True),
        # a ragged batch in 32 bits, head dimension 64, rows inside a wider projection
        dict(name="qk_ragged_f32", op="qk", tokens=1531, heads=4, kv_heads=4, dim=64, dtype="f32", slots=2048, pad=64, norm=True),
        # a "tree" of one token for each of eight sequences: the step of an undrafted batch
        dict(name="verify_single", op="verify", draft=1, ragged=0, **mha),
        # trees of up to 16 tokens, full and filling caches
        dict(name="verify_tree16", op="verify", draft=16, ragged=1, **gqa),
        # the widest tree: 64 tokens for each of 32 sequences
        dict(name="verify_tree64", op="verify", draft=64, ragged=0, **gqa),
        # one user, long cache
        dict(name="verify_one_user", op="verify", draft=24, ragged=0, batch=1, heads=32, kv_heads=8, dim=128, budget=4096, dtype="bf16"),
        # 32 bits, head dimension 64, small cache
        dict(name="verify_f32", op="verify", draft=13, ragged=0, batch=1, heads=4, kv_heads=4, dim=64, budget=256, dtype="f32"),
        # a whole drafted step: verify, then up to six tokens enter
        dict(name="step_gqa", op="step", draft=16, accept=6, ragged=1, **gqa),
        dict(name="step_mha", op="step", draft=7, accept=4, ragged=0, **mha),
        # one prompt becomes eight samples
        dict(name="fork_samples", op="fork", kind="samples", ragged=0, **mha),
        # beams: every sequence takes a random parent's cache, some end
        dict(name="fork_beams", op="fork", kind="beams", ragged=1, **gqa),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = max(_cost(c) for c in listed())
    while True:
        case = _draw_any(rng)
        if _cost(case) <= largest:
            return case


def _draw_any(rng):
    op = rng.choice(["qk", "verify", "verify", "step", "step", "fork"])
    group = rng.choice([1, 2, 4, 8])
    kv_heads = rng.choice([1, 2, 3, 4, 8, 16])
    case = dict(op=op, heads=group * kv_heads, kv_heads=kv_heads, dim=rng.choice([64, 128, 128]),
                dtype=rng.choice(["bf16", "bf16", "f32"]))
    if op == "qk":
        return dict(case, tokens=_spread(rng, 1, 8192), slots=_spread(rng, 1024, 131072), pad=rng.choice([0, 8, 256]),
                    norm=rng.random() < 0.8)
    case.update(batch=_spread(rng, 2 if op == "fork" else 1, 48), budget=_spread(rng, 80, 4096), ragged=rng.randrange(1, 1 << 20))
    if op == "fork":
        return dict(case, kind=rng.choice(["samples", "beams"]))
    case["draft"] = _spread(rng, 1, 64)
    if op == "step":
        case["accept"] = rng.randint(1, min(12, case["draft"]))
    return case


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _lengths(case):
    """Tokens seen, drafted and accepted by each sequence: ragged = 0: full caches somewhere in a cycle, full drafts."""
    r = random.Random("%d %d %d" % (case["ragged"], case["batch"], case["budget"]))
    c, B, T, A = case["budget"], case["batch"], case.get("draft", 1), case.get("accept", 0)
    seen, lens, took = [], [], []
    for b in range(B):
        full = case["ragged"] == 0 or r.random() < 0.7
        seen.append(c + r.randrange(0, 3 * c) if full else r.randrange(0, c + 1))
        lens.append(T if case["ragged"] == 0 else r.randint(1, T))
        took.append(min(lens[b], A if case["ragged"] == 0 else r.randint(0, A)))
    if case["ragged"] and B > 3:
        lens[r.randrange(B)] = 0     # a sequence that sits this call out
        took = [min(t, n) for t, n in zip(took, lens)]
    return seen, lens, took


def _sources(case):
    r = random.Random("%d sources %d" % (case["ragged"], case["batch"]))
    B = case["batch"]
    if case["kind"] == "samples":
        return [0] * B
    return [-1 if r.random() < 0.06 else b if r.random() < 0.25 else r.randrange(B) for b in range(B)]


def _live_rows(n, c):
    L = min(n, c)
    return L, (max(n - c, 0) % c)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    Hq, Hkv, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "qk":
        row = (Hq + 2 * Hkv) * d
        return {"bytes": case["tokens"] * (2 * row * e + 2 * (d // 2) * 4 + 4), "flops": case["tokens"] * (Hq + Hkv) * d * 7}
    seen, lens, took = _lengths(case)
    c = case["budget"]
    cached = [min(n, c) for n in seen]
    if case["op"] == "fork":
        src = _sources(case)
        token = Hkv * (2 * d * e + 8)
        read = sum(cached[s] for s in {s for b, s in enumerate(src) if s not in (b, -1)})
        write = sum(cached[s] for b, s in enumerate(src) if s not in (b, -1))
        return {"bytes": (read + write) * token + 1, "flops": 0}
    bytes_, flops = 0, 0
    for L, T in zip(cached, lens):
        if T:
            bytes_ += L * Hkv * 2 * d * e + T * (2 * Hq + 2 * Hkv) * d * e + T * (Hq * 4 + 8)
            flops += 4 * d * Hq * T * (L + (T + 1) / 2)
    if case["op"] == "step":
        for n, L, A in zip(seen, cached, took):
            if A:
                moved = max(0, L + A - c)
                bytes_ += L * Hkv * (d * e + 8) + A * (Hq * d * e + 4 * Hkv * d * e) + moved * Hkv * (4 * d * e + 24)
                flops += 2 * d * Hq * A * (L + (A + 1) / 2)
    return {"bytes": bytes_, "flops": flops}


# ---- inputs --------------------------------------------------------------------------------------------------------
def _trees(lens, took, T, r):
    """Ancestor bits of random trees - a node hangs under an earlier one or is a first token of its own - and in each
    the way to an accepted node."""
    masks, paths = [], []
    for n, a in zip(lens, took):
        way = sorted(r.sample(range(n), a))
        bits = []
        for i in range(T):
            under = r.randrange(max(-1, i - 6), i) if i else -1
            if i in way:
                under = way[way.index(i) - 1] if i != way[0] else -1
            bits.append((bits[under] if under >= 0 else 0) | (1 << i))
        masks.append([x - (1 << 64) if x >> 63 else x for x in bits])
        paths.append(way)
    return masks, paths


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dtype(case)
    Hq, Hkv, d = case["heads"], case["kv_heads"], case["dim"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if case["op"] == "qk":
        n, row = case["tokens"], (Hq + 2 * Hkv) * d
        wide = (normal(n, row + case["pad"]) * (0.5 + 2 * torch.rand((n, 1), generator=g, device="cuda"))).to(dt)
        freq = BASE ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
        angle = torch.arange(case["slots"], device="cuda", dtype=torch.float64)[:, None] * freq
        s = dict(case=case, qkv=wide[:, :row], cos=angle.cos().float(), sin=angle.sin().float(),
                 wq=(1 + 0.2 * normal(d)).to(dt) if case["norm"] else None,
                 wk=(1 + 0.2 * normal(d)).to(dt) if case["norm"] else None,
                 pos=torch.randint(0, case["slots"], (n,), generator=g, device="cuda", dtype=torch.int32))
        if own:
            from paper_2501_04987_b200 import TreeKV

            s["kv"] = TreeKV(64, Hq, Hkv, d, case["dtype"], 1, 0)
        return s

    B, c = case["batch"], case["budget"]
    seen, lens, took = _lengths(case)
    s = dict(case=case, seen=seen)
    peak = torch.ones(d, device="cuda")
    peak[d // 2 - 1] = peak[d - 1] = 8.0   # a few strong key channels, as trained models have
    N = torch.tensor(seen, device="cuda", dtype=torch.int64)[:, None]
    L = N.clamp(max=c)
    slot = torch.arange(c, device="cuda")[None]
    held = slot < L                                                   # [B, c]
    back = (L - 1 - slot).clamp(min=0)                                # tokens from the newest
    thin = (back.double() / (c - 1)).square() * (N - L)               # old context is sparse, recent context dense
    pos = torch.where(held, N - 1 - back - thin.long(), -1).to(torch.int32)[:, None].expand(B, Hkv, c).contiguous()
    K = ((normal(B, Hkv, c, d) * peak) * held[:, None, :, None]).to(dt)
    V = (normal(B, Hkv, c, d) * held[:, None, :, None]).to(dt)
    count = (N[:, None] - pos).float()
    S = torch.where(held[:, None], count / L.clamp(min=1)[:, None] * torch.exp(0.7 * normal(B, Hkv, c)), 0.0)
    room = 0
    if case["op"] in ("verify", "step"):
        T = case["draft"]
        masks, paths = _trees(lens, took, T, random.Random(seed))
        s["mask"] = torch.tensor(masks, dtype=torch.int64, device="cuda")
        s["q"] = normal(B, T, Hq, d).to(dt)
        s["k"] = (normal(B, T, Hkv, d) * peak).to(dt)
        s["v"] = normal(B, T, Hkv, d).to(dt)
        s["out"] = torch.zeros((B, T, Hq, d), device="cuda", dtype=dt)
        s["lse"] = torch.zeros((B, T, Hq), device="cuda")
        s["lens"], s["lens_dev"] = lens, torch.tensor(lens, device="cuda")
        if case["op"] == "step":
            room = case["accept"]
            s["took"], s["took_dev"] = took, torch.tensor(took, device="cuda")
            s["path"] = torch.tensor([(w + [0] * room)[:room] for w in paths], dtype=torch.int32, device="cuda")
    else:
        s["source"] = _sources(case)
        s["source_dev"] = torch.tensor(s["source"], device="cuda")
    s["N"] = N[:, 0]
    s["room"] = room
    if own:
        _open(s, K, V, S, pos)
    elif case["op"] == "verify":
        s["K"], s["V"] = K, V
    else:
        _slabs(s, K, V, S, pos)
    return s


def _slabs(s, K, V, S, pos):
    """The cache as it lies in memory: slabs of 2 * budget + room rows, zeros where no token was ever written."""
    B, Hkv, c, d = K.shape
    R = 2 * c + s["room"]
    rows, held = _rows(s["N"], c)
    to = torch.where(held, rows, R)[:, None].expand(B, Hkv, c)        # slots without a token land in a spare row
    s["K"] = torch.zeros((B, Hkv, R + 1, d), device="cuda", dtype=K.dtype).scatter_(2, to[..., None].expand(-1, -1, -1, d), K)[:, :, :R].contiguous()
    s["V"] = torch.zeros((B, Hkv, R + 1, d), device="cuda", dtype=V.dtype).scatter_(2, to[..., None].expand(-1, -1, -1, d), V)[:, :, :R].contiguous()
    s["S"] = torch.zeros((B, Hkv, R + 1), device="cuda").scatter_(2, to, S)[:, :, :R].contiguous()
    s["pos"] = torch.zeros((B, Hkv, R + 1), device="cuda", dtype=torch.int32).scatter_(2, to, pos)[:, :, :R].contiguous()
    s["n"] = s["N"][:, None].expand(B, Hkv).to(torch.int32).contiguous()


def _open(s, K, V, S, pos):
    """The library's handle with this cache in it, and its slabs as views of the workspace that the program owns."""
    from paper_2501_04987_b200 import TreeKV

    case = s["case"]
    B, Hkv, c, d = K.shape
    kv = TreeKV(c, case["heads"], Hkv, d, case["dtype"], B, s["room"])
    seen = s["N"].to(torch.int32)
    parts = [K, V, S.float(), pos, seen, torch.zeros_like(seen)]
    image = _bytes([p.contiguous().view(-1).view(torch.uint8) for p in parts])
    kv.import_state(image, s["seen"])
    s["kv"] = kv
    R, at = 2 * c + s["room"], (-kv.workspace.data_ptr()) % ALIGN

    def view(dtype, *shape):
        nonlocal at
        size = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
        got = kv.workspace[at:at + size].view(dtype).view(shape)
        at += -(-size // ALIGN) * ALIGN
        return got

    s["K"], s["V"] = view(K.dtype, B, Hkv, R, d), view(K.dtype, B, Hkv, R, d)
    if K.dtype == torch.bfloat16 and d == 128 and s["room"]:
        view(K.dtype, B, Hkv, R, d)                                   # keys encoded at their slots: not in use
    s["S"], s["pos"], s["n"] = view(torch.float32, B, Hkv, R), view(torch.int32, B, Hkv, R), view(torch.int32, B, Hkv)


def _bytes(parts):
    """Byte strings one after another, each padded to the alignment."""
    return torch.cat([torch.nn.functional.pad(p, (0, (-p.numel()) % ALIGN)) for p in parts])


# ---- a pass --------------------------------------------------------------------------------------------------------
def run(s):
    return {"qk": _run_qk, "verify": _run_verify, "step": _run_step, "fork": _run_fork}[s["case"]["op"]](s)


def _run_qk(s):
    if own:
        return s["kv"].norm_rope(s["qkv"], q_weight=s["wq"], k_weight=s["wk"], cos=s["cos"], sin=s["sin"],
                                 positions=s["pos"], eps=EPS)
    case = s["case"]
    Hq, Hkv, d = case["heads"], case["kv_heads"], case["dim"]
    dt, n = s["qkv"].dtype, case["tokens"]
    q, k, v = (x.reshape(n, -1, d) for x in s["qkv"].split([Hq * d, Hkv * d, Hkv * d], dim=1))
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]

    def turn(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(dt)

    return turn(q, s["wq"]), turn(k, s["wk"]), v.contiguous()


def _rows(N, c):
    """Slab rows of the cached tokens in cache order, [B, c], and which of them exist."""
    L, i = N.clamp(max=c)[:, None], ((N - c).clamp(min=0) % c)[:, None]
    slot = torch.arange(c, device="cuda")[None]
    return slot + torch.where(slot >= i, i, 0), slot < L


def _attend(s, K, V, N):
    """Attention of the drafted tokens over the cached ones (K, V in cache order) and the drafted ones of their mask."""
    case = s["case"]
    B, Hkv, c, d = K.shape
    T, G = case["draft"], case["heads"] // Hkv
    q = s["q"].float().view(B, T, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, d)
    keys = torch.cat([K.float(), s["k"].float().transpose(1, 2)], 2)
    values = torch.cat([V.float(), s["v"].float().transpose(1, 2)], 2)
    logits = (q @ keys.transpose(2, 3)) * (d ** -0.5)
    held = (torch.arange(c, device="cuda")[None] < N.clamp(max=c)[:, None])[:, None].expand(B, T, c)
    node = torch.arange(T, device="cuda")
    real = node[None] < s["lens_dev"][:, None]
    tree = ((s["mask"][:, :, None] >> node) & 1).bool() & real[:, None]
    sees = torch.cat([held, tree], 2)[:, None, :, None].expand(B, 1, T, G, c + T).reshape(B, 1, T * G, c + T)
    logits = logits.masked_fill(~sees, -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top.isinf(), 0.0, top)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    o = (p @ values) / torch.where(total > 0, total, 1.0)
    o = o.view(B, Hkv, T, G, d).permute(0, 2, 1, 3, 4).reshape(B, T, Hkv * G, d)
    lse = (top + torch.log(total)).view(B, Hkv, T, G).permute(0, 2, 1, 3).reshape(B, T, Hkv * G)
    s["out"].copy_(torch.where(real[..., None, None], o.to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(real[..., None], lse, s["lse"]))
    return s["out"], s["lse"]


def _run_verify(s):
    if own:
        return s["kv"].verify_tree(s["q"], s["k"], s["v"], mask=s["mask"], lens=s["lens"], out=s["out"], lse=s["lse"])
    return _attend(s, s["K"], s["V"], s["N"])


def _run_step(s):
    if own:
        out, lse = s["kv"].verify_tree(s["q"], s["k"], s["v"], mask=s["mask"], lens=s["lens"], out=s["out"], lse=s["lse"])
        s["kv"].accept_path(s["q"], s["k"], s["v"], lse, s["path"], s["took"])
        return out, lse, s["K"], s["V"], s["S"], s["pos"], s["n"]
    c, d = s["case"]["budget"], s["case"]["dim"]
    N = s["n"][:, 0].long()
    rows, held = _rows(N, c)
    B, Hkv = s["n"].shape
    at = rows[:, None].expand(B, Hkv, c)
    K, V = (s[x].gather(2, at[..., None].expand(-1, -1, -1, d)) for x in "KV")
    out, lse = _attend(s, K, V, N)
    _accept(s, K, at, held, N)
    return out, lse, s["K"], s["V"], s["S"], s["pos"], s["n"]


def _accept(s, K, at, held, N):
    """The accepted path enters the cache: append, score update, evictions."""
    case = s["case"]
    B, Hkv, c, d = K.shape
    A, G = case["accept"], case["heads"] // Hkv
    step = torch.arange(A, device="cuda")
    took = s["took_dev"]
    real = step[None] < took[:, None]                                             # [B, A]
    pick = s["path"].long()
    seq = torch.arange(B, device="cuda")[:, None]
    q, k, v, lse = (s[x][seq, pick] for x in ("q", "k", "v", "lse"))              # [B, A, heads, ...]
    k, v = k.transpose(1, 2), v.transpose(1, 2)
    # what the accepted rows gave to every cached token and to one another
    qf = q.float().view(B, A, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, A * G, d)
    keys = torch.cat([K.float(), k.float()], 2)
    logits = (qf @ keys.transpose(2, 3)) * (d ** -0.5)
    p = torch.exp(logits - lse.view(B, A, Hkv, G).permute(0, 2, 1, 3).reshape(B, Hkv, A * G, 1))
    sees = torch.cat([held[:, None].expand(B, A, c), (step[None] <= step[:, None])[None].expand(B, A, A)], 2) & real[..., None]
    p = torch.where(sees[:, None, :, None].expand(B, 1, A, G, c + A).reshape(B, 1, A * G, c + A), p, 0.0)
    given = p.sum(2) / G                                                          # [B, Hkv, c + A]
    L, i = N.clamp(max=c), (N - c).clamp(min=0) % c
    S, P = s["S"], s["pos"]
    S.scatter_add_(2, at, torch.where(held[:, None], given[..., :c], 0.0))
    new = (L + i)[:, None] + step                                                 # rows of the appended tokens
    _put(s, new, real, k, v, given[..., c:], (N[:, None] + step).to(torch.int32)[:, None].expand(B, Hkv, A))
    # evictions: the pairs up to the end of the cycle, then the rows behind the last pair move down, then the rest
    now = (N + took)[:, None, None]
    out = (L + took - c).clamp(min=0)
    first = torch.minimum(out, c - i)
    rest = out - first
    _drop(s, i[:, None] + step, step[None] < first[:, None], now)
    _move(s, 2 * c + step[None].expand(B, A), c + step[None].expand(B, A), step[None] < rest[:, None])
    _drop(s, step[None].expand(B, A), step[None] < rest[:, None], now)
    s["n"].copy_((N + took)[:, None].expand(B, Hkv))


def _drop(s, pair, real, now):
    """Of rows 2 * pair and 2 * pair + 1 the one with the larger S / C stays (the right one at a tie), in row pair."""
    B, Hkv = s["n"].shape
    left = torch.where(real, 2 * pair, 0)[:, None].expand(B, Hkv, -1)
    score = [s["S"].gather(2, left + x) / (now - s["pos"].gather(2, left + x)).float() for x in (0, 1)]
    _move(s, left + torch.where(score[0] > score[1], 0, 1), pair, real)


def _move(s, src, dst, real):
    B, Hkv = s["n"].shape
    src = (torch.where(real[:, None], src, 0) if src.dim() == 3 else torch.where(real, src, 0)[:, None]).expand(B, Hkv, -1)
    wide = src[..., None].expand(-1, -1, -1, s["case"]["dim"])
    _put(s, dst, real, s["K"].gather(2, wide), s["V"].gather(2, wide), s["S"].gather(2, src), s["pos"].gather(2, src))


def _put(s, rows, real, k, v, score, pos):
    """Writes the real ones of the given rows, which are all different; the others keep what they hold."""
    B, Hkv = s["n"].shape
    rows, real = rows[:, None].expand(B, Hkv, -1), real[:, None].expand(B, Hkv, -1)
    wide = rows[..., None].expand(-1, -1, -1, s["case"]["dim"])
    for x, new in (("K", k), ("V", v)):
        s[x].scatter_(2, wide, torch.where(real[..., None], new, s[x].gather(2, wide)))
    for x, new in (("S", score), ("pos", pos)):
        s[x].scatter_(2, rows, torch.where(real, new, s[x].gather(2, rows)))


def _run_fork(s):
    if own:
        s["kv"].fork_sequences(s["source"])
        return s["K"], s["V"], s["S"], s["pos"], s["n"]
    c = s["case"]["budget"]
    src = s["source_dev"].clamp(min=0)
    moves = (s["source_dev"] >= 0) & (s["source_dev"] != torch.arange(len(s["source"]), device="cuda"))
    N = s["n"][:, 0].long()[src]
    L, i = N.clamp(max=c)[:, None], ((N - c).clamp(min=0) % c)[:, None]
    row = torch.arange(s["S"].shape[2], device="cuda")[None]
    live = ((row < i) | ((row >= 2 * i) & (row < L + i))) & moves[:, None]        # [B, R]
    for x in ("K", "V"):
        s[x].copy_(torch.where(live[:, None, :, None], s[x][src], s[x]))
    for x in ("S", "pos"):
        s[x].copy_(torch.where(live[:, None], s[x][src], s[x]))
    s["n"].copy_(torch.where((s["source_dev"] >= 0)[:, None], s["n"][src], 0))
    return s["K"], s["V"], s["S"], s["pos"], s["n"]


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"qk": _exact_qk, "verify": _exact_verify, "step": _exact_step, "fork": _exact_fork}[case["op"]](s)


def _exact_qk(s):
    case = s["case"]
    d, n, Hq, Hkv = case["dim"], case["tokens"], case["heads"], case["kv_heads"]
    x = s["qkv"].double().reshape(n, Hq + 2 * Hkv, d)
    out = x.clone()
    c, sn = s["cos"].double()[s["pos"].long()], s["sin"].double()[s["pos"].long()]
    for h in range(Hq + Hkv):
        w = s["wq"] if h < Hq else s["wk"]
        y = x[:, h]
        if w is not None:
            y = y / torch.sqrt((y * y).sum(1, keepdim=True) / d + EPS) * w.double()
        z = torch.complex(y[:, :d // 2], y[:, d // 2:]) * torch.complex(c, sn)
        out[:, h] = torch.cat([z.real, z.imag], 1)
    return out[:, :Hq].contiguous(), out[:, Hq:Hq + Hkv].contiguous(), out[:, Hq + Hkv:].contiguous()


def _exact_heads(s, b, K, V, L):
    """One sequence: outputs and log-sum-exps of its drafted tokens; K, V its cached tokens [Hkv, L, d]."""
    case = s["case"]
    Hkv, d, T = case["kv_heads"], case["dim"], s["lens"][b]
    G = case["heads"] // Hkv
    bits = s["mask"][b, :T].tolist()
    tree = torch.tensor([[bool(m >> j & 1) for j in range(T)] for m in bits], device="cuda").view(T, T)
    hide = torch.cat([torch.zeros((T, L), dtype=torch.bool, device="cuda"), ~tree], 1)
    o = torch.empty((T, case["heads"], d), dtype=torch.float64, device="cuda")
    z = torch.empty((T, case["heads"]), dtype=torch.float64, device="cuda")
    for h in range(Hkv):
        kk = torch.cat([K[h], s["k"][b, :T, h].double()])
        vv = torch.cat([V[h], s["v"][b, :T, h].double()])
        a = torch.einsum("tgd,nd->gtn", s["q"][b, :T, h * G:(h + 1) * G].double(), kk) / math.sqrt(d)
        a = a.masked_fill(hide, -math.inf)
        z[:, h * G:(h + 1) * G] = torch.logsumexp(a, 2).T
        o[:, h * G:(h + 1) * G] = (torch.softmax(a, 2) @ vv).transpose(0, 1)
    return o, z


def _exact_verify(s):
    out, lse = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["seen"]):
        if s["lens"][b]:
            L = min(n, s["case"]["budget"])
            out[b, :s["lens"][b]], lse[b, :s["lens"][b]] = _exact_heads(s, b, s["K"][b, :, :L].double(), s["V"][b, :, :L].double(), L)
    return out, lse


def _exact_step(s):
    case = s["case"]
    c, d, Hkv = case["budget"], case["dim"], case["kv_heads"]
    G = case["heads"] // Hkv
    out, lse = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    S = s["S"].double()
    head = torch.arange(Hkv, device="cuda")
    for b, n in enumerate(s["seen"]):
        T, A = s["lens"][b], s["took"][b]
        if not T:
            continue
        L, i = _live_rows(n, c)
        rows = list(range(i)) + list(range(2 * i, L + i))
        K, V, P = s["K"][b], s["V"][b], s["pos"][b]
        out[b, :T], lse[b, :T] = _exact_heads(s, b, K[:, rows].double(), V[:, rows].double(), L)
        for t in range(A):   # the tokens are appended one by one, each scores what it sees
            node, row = int(s["path"][b, t]), L + i + t
            K[:, row], V[:, row] = s["k"][b, node], s["v"][b, node]
            P[:, row], S[b, :, row] = n + t, 0.0
            rows.append(row)
            a = torch.einsum("hgd,hnd->hgn", s["q"][b, node].double().view(Hkv, G, d), K[:, rows].double()) / math.sqrt(d)
            S[b][:, rows] += torch.exp(a - lse[b, node].view(Hkv, G, 1)).mean(1)
        held = L + A
        while held > c:      # Algorithm 1's branch, one pair at a time, the scores as they stand
            l, r = 2 * i, 2 * i + 1
            stays = torch.where(S[b, :, l] / (n + A - P[:, l]) > S[b, :, r] / (n + A - P[:, r]), l, r)
            K[:, i], V[:, i], P[:, i], S[b, :, i] = K[head, stays], V[head, stays], P[head, stays], S[b][head, stays]
            i, held = i + 1, held - 1
            if i == c:
                for x in range(held - c):
                    K[:, c + x], V[:, c + x], P[:, c + x], S[b, :, c + x] = K[:, 2 * c + x].clone(), V[:, 2 * c + x].clone(), P[:, 2 * c + x].clone(), S[b, :, 2 * c + x].clone()
                i = 0
        s["n"][b] += A
    return out, lse, s["K"], s["V"], S, s["pos"], s["n"]


def _exact_fork(s):
    c = s["case"]["budget"]
    was = {x: s[x].clone() for x in ("K", "V", "S", "pos", "n")}
    for b, a in enumerate(s["source"]):
        if a < 0:
            s["n"][b] = 0
        elif a != b:
            L, i = _live_rows(s["seen"][a], c)
            for rows in (slice(0, i), slice(2 * i, L + i)):
                for x in ("K", "V", "S", "pos"):
                    s[x][b, :, rows] = was[x][a, :, rows]
            s["n"][b] = was["n"][a]
    return s["K"], s["V"], s["S"].double(), s["pos"], s["n"]
