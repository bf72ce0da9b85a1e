"""Measured cases of the operators that keep a prompt whole in pages, evict it into the fixed-budget cache and find the
accepted path of a draft.

Four operators, named by the case's "op":

  attend  attention of a chunk of new tokens over a paged cache, which the chunk enters
  score   what the rows of a chunk (an observation window, or all of a prompt's last chunk) gave to every token of the pages
  adopt   the heaviest tokens of paged prompts become the cache of a budget: eviction by accumulated attention weight
  pick    verification of drafted trees against the target's probabilities from given random numbers

Pages lie [page][KV head][token of the page][channel]; table[b, x] is the page of the tokens [x * page, (x + 1) * page) of
sequence b.  With `own` false, run() computes the operators with elementary torch operations; with `own` true it makes the
library's calls.
"""
import math
import random

import torch

own = False

ALIGN = 256          # parts of the cache's workspace start on such a boundary


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    gqa = dict(heads=32, kv_heads=8, dim=128, dtype="bf16")
    mha = dict(heads=32, kv_heads=32, dim=128, dtype="bf16")
    return [
        # one decode step of 32 sequences of different lengths while their prompts are still whole
        dict(name="attend_step", op="attend", batch=32, tokens=1, past=4096, page=16, ragged=1, **gqa),
        # one user, one token, a long context: the work has to be split along it
        dict(name="attend_one_user", op="attend", batch=1, tokens=1, past=100000, page=64, ragged=0, **gqa),
        # a few tokens behind a short prompt in 32 bits: latency
        dict(name="attend_few_f32", op="attend", batch=3, tokens=5, past=203, page=16, ragged=1, heads=4, kv_heads=4, dim=64, dtype="f32"),
        # the next 1024 tokens of four prompts
        dict(name="attend_chunk", op="attend", batch=4, tokens=1024, past=8192, page=64, ragged=0, **gqa),
        # whole prompts, nothing cached before them
        dict(name="attend_prompt", op="attend", batch=2, tokens=4096, past=0, page=128, ragged=0, **mha),
        # the last 32 tokens of eight prompts weigh all their tokens
        dict(name="score_window", op="score", batch=8, tokens=32, past=8160, page=64, ragged=0, **gqa),
        # every row of a chunk of 1024 counts
        dict(name="score_chunk", op="score", batch=4, tokens=1024, past=4096, page=64, ragged=1, **gqa),
        # eight prompts shrink to a budget of 1024
        dict(name="adopt_batch", op="adopt", batch=8, past=8192, budget=1024, page=64, rule="accumulated", sinks=4, recent=64, ragged=1, **gqa),
        # one long prompt shrinks to 2048, the weights averaged over the rows that saw the token
        dict(name="adopt_one_user", op="adopt", batch=1, past=100000, budget=2048, page=64, rule="average", sinks=0, recent=0, ragged=0, **gqa),
        # a chain of seven tokens from a drafter that is certain of each, one user
        dict(name="pick_chain", op="pick", batch=1, draft=8, accept=4, vocab=32000, logits="f32", given=False, warm=1.0, ragged=0),
        # trees of 16 for 32 sequences, drawn from a draft model's probabilities, large vocabulary
        dict(name="pick_tree", op="pick", batch=32, draft=16, accept=5, vocab=128000, logits="bf16", given=True, warm=0.8, ragged=1),
        # greedy: the path follows the largest logit; an odd vocabulary, so rows start anywhere
        dict(name="pick_greedy", op="pick", batch=8, draft=24, accept=6, vocab=50257, logits="bf16", given=False, warm=0.0, ragged=1),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = max(_cost(c) for c in listed())
    while True:
        case = _draw_any(rng)
        if _cost(case) <= largest and _held(case) <= 4e9:
            return case


def _draw_any(rng):
    op = rng.choice(["attend", "attend", "attend", "score", "score", "adopt", "pick", "pick"])
    ragged = rng.randrange(1, 1 << 20)
    if op == "pick":
        draft = _spread(rng, 1, 64)
        return dict(op=op, batch=_spread(rng, 1, 64), draft=draft, accept=rng.randint(1, min(8, draft)), vocab=_spread(rng, 500, 200000),
                    logits=rng.choice(["bf16", "f32"]), given=rng.random() < 0.5, warm=rng.choice([0.0, 0.7, 1.0, 1.0]), ragged=ragged)
    kv_heads = rng.choice([1, 2, 3, 4, 8, 16])
    case = dict(op=op, heads=rng.choice([1, 2, 4, 8]) * kv_heads, kv_heads=kv_heads, dim=rng.choice([64, 128, 128]),
                dtype=rng.choice(["bf16", "bf16", "f32"]), page=rng.choice([16, 32, 64, 128, 256]), batch=_spread(rng, 1, 48),
                past=_spread(rng, 1, 100000), ragged=ragged)
    if op == "adopt":
        budget = _spread(rng, 16, 4096)
        sinks, recent = (rng.randint(0, 4), rng.randint(0, budget // 4)) if rng.random() < 0.5 else (0, 0)
        return dict(case, budget=budget, rule=rng.choice(["accumulated", "average"]), sinks=sinks, recent=recent)
    case["tokens"] = _spread(rng, 1, 4096 if op == "attend" else 1024)
    return case


def _cost(case):
    """Time as bytes: what is moved, or the operations at the rate of the type's units."""
    w = work(case)
    return max(w["bytes"], w["flops"] / (8 if case.get("dtype") == "f32" else 185))


def _held(case):
    """Bytes of the pages, or of the logits."""
    if case["op"] == "pick":
        return case["batch"] * case["draft"] * case["vocab"] * ((4 if case["logits"] == "f32" else 2) + (4 if case["given"] else 0))
    return case["batch"] * (case["past"] + case.get("tokens", 0)) * case["kv_heads"] * case["dim"] * 2 * (4 if case["dtype"] == "f32" else 2)


def _lengths(case):
    """Tokens cached and new ones of each sequence: ragged = 0: all as long as the case says."""
    r = random.Random("%d %d %d" % (case["ragged"], case["batch"], case["past"]))
    past, new = [], []
    for b in range(case["batch"]):
        T = case.get("tokens", 0)
        full = case["ragged"] == 0
        past.append(case["past"] if full or b == 0 else r.randint(0, case["past"]))
        new.append(T if full or b == 0 else r.randint(1, T) if T else 0)
    if case["ragged"] and case["batch"] > 3:
        at = r.randrange(1, case["batch"])       # a sequence that sits this call out
        if case["op"] == "adopt":
            past[at] = 0
        else:
            new[at] = 0
    return past, new


def _trees(case):
    """Parents of the drafted tokens (node 0 is the token that the draft hangs on) and the way to the last accepted one."""
    r = random.Random("%d %d %d" % (case["ragged"], case["batch"], case["draft"]))
    T, A = case["draft"], case["accept"]
    lens, parents, ways = [], [], []
    for b in range(case["batch"]):
        n = T if case["ragged"] == 0 or b == 0 else r.randint(1, T)
        if case["ragged"] and case["batch"] > 3 and b == 2:
            n = 0
        took = 0 if n == 0 else min(n, A) if case["ragged"] == 0 or b == 0 else r.randint(1, min(n, A))
        way = [0] + sorted(r.sample(range(1, n), took - 1)) if took else []
        if case["ragged"] == 0:
            up, way = [i - 1 for i in range(n)], list(range(took))
        else:
            up = [-1]
            for i in range(1, n):
                up.append(way[way.index(i) - 1] if i in way else r.randrange(max(0, i - 6), i))
            up = up[:n]
        lens.append(n)
        parents.append(up)
        ways.append(way)
    return lens, parents, ways


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    if case["op"] == "pick":
        lens, parents, ways = _trees(case)
        e = 4 if case["logits"] == "f32" else 2
        V, rows, draft_rows = case["vocab"], sum(len(w) for w in ways), 0
        if case["given"] and case["warm"] > 0:
            for n, up, way in zip(lens, parents, ways):
                # draft probabilities count where a child is turned down
                draft_rows += sum(1 for x in way if [c for c in range(x + 1, n) if up[c] == x and (c not in way or min(k for k in range(n) if up[k] == x) != c)])
        noise = sum(1 for n in lens if n) if case["warm"] > 0 else 0
        return {"bytes": rows * V * e + draft_rows * V * 4 + noise * V * 4 + sum(lens) * 16, "flops": rows * V * 4}
    e = 4 if case["dtype"] == "f32" else 2
    Hq, Hkv, d = case["heads"], case["kv_heads"], case["dim"]
    past, new = _lengths(case)
    if case["op"] == "adopt":
        kept = [min(n, case["budget"]) for n in past]
        return {"bytes": sum(past) * Hkv * 4 + sum(kept) * Hkv * (4 * d * e + 8), "flops": 0}
    seen = sum(n * p + n * (n + 1) // 2 for p, n in zip(past, new))
    live = sum(p for p, n in zip(past, new) if n)
    if case["op"] == "score":
        return {"bytes": (live + sum(new)) * Hkv * (d * e + 4) + sum(new) * Hq * (d * e + 4), "flops": 2 * d * Hq * seen}
    return {"bytes": live * Hkv * 2 * d * e + sum(new) * (Hq * (2 * d * e + 4) + 4 * Hkv * d * e), "flops": 4 * d * Hq * seen}


# ---- inputs --------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return _prepare_pick(case, g, seed) if case["op"] == "pick" else _prepare_pages(case, g)


def _prepare_pages(case, g):
    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    B, Hq, Hkv, d, page = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["page"]
    dt = _dtype(case["dtype"])
    past, new = _lengths(case)
    T = case.get("tokens", 0)
    need = [-(-(p + n) // page) for p, n in zip(past, new)]
    width = max(need)
    total = sum(need) + 2                                            # two pages that nobody has
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    peak = torch.ones(d, device="cuda")
    peak[d // 2 - 1] = peak[d - 1] = 4.0                              # a few strong key channels, as trained models have
    kp, vp = (torch.empty((total, Hkv, page, d), device="cuda", dtype=dt) for _ in range(2))
    step = max(1, (1 << 26) // (Hkv * page * d))
    for x in range(0, total, step):                                  # (rows that hold no token keep what earlier requests left)
        n = min(step, total - x)
        kp[x:x + n] = (normal(n, Hkv, page, d) * peak).to(dt)
        vp[x:x + n] = normal(n, Hkv, page, d).to(dt)
    s = dict(case=case, past=past, new=new, table=table, kp=kp, vp=vp, width=width,
             past_dev=torch.tensor(past, dtype=torch.int32, device="cuda"))
    if case["op"] == "attend":
        s["q"], s["k"], s["v"] = normal(B, T, Hq, d).to(dt), (normal(B, T, Hkv, d) * peak).to(dt), normal(B, T, Hkv, d).to(dt)
        s["out"], s["lse"] = torch.zeros((B, T, Hq, d), device="cuda", dtype=dt), torch.zeros((B, T, Hq), device="cuda")
    elif case["op"] == "score":
        s["q"] = normal(B, T, Hq, d).to(dt)
        s["scores"] = torch.zeros((B, Hkv, width * page), device="cuda")
        s["lse"] = _sums(s)
    else:
        # a token's weight: a heavy tail, and for the older ones more rows that saw them
        age = (torch.tensor(past, device="cuda")[:, None] - torch.arange(width * page, device="cuda")).clamp(min=1)
        s["first"] = [max(0, n - 64) if case["rule"] == "average" else 0 for n in past]
        if case["rule"] == "average":
            age = age.clamp(max=64)
        s["scores"] = age[:, None] / max(past) * torch.exp(1.5 * normal(B, Hkv, width * page))
        _prepare_cache(s)
    if own:
        from paper_2501_04987_b200 import TreeKV, binding

        if case["op"] == "adopt":
            s["kv"] = TreeKV(case["budget"], Hq, Hkv, d, case["dtype"], B, 0)
            if case["sinks"] or case["recent"]:
                s["kv"].set_protection(case["sinks"], case["recent"])
            if case["rule"] == "accumulated":
                s["kv"].set_rule(binding.RULE_ACCUMULATED)
            _views(s)
        else:
            s["kv"] = TreeKV(64, Hq, Hkv, d, case["dtype"], B, 0)
    return s


def _sums(s):
    """Log-sum-exps of the rows over what they see, as their attention left them."""
    case = s["case"]
    B, T, Hq, d = s["q"].shape
    Hkv = case["kv_heads"]
    lse = torch.zeros((B, T, Hq), device="cuda")
    for b, (p, n) in enumerate(zip(s["past"], s["new"])):
        if n:
            K = _rows(s, s["kp"], b, p + n).float()
            for h in range(Hkv):
                x = _logits(s, b, h, K[h], p, 0, n)
                lse[b, :n, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)] = torch.logsumexp(x, -1)
    return lse


def _prepare_cache(s):
    """The cache as it lies in memory: slabs of 2 * budget rows, zeros where no token was ever written."""
    case = s["case"]
    B, Hkv, R, d = case["batch"], case["kv_heads"], 2 * case["budget"], case["dim"]
    if own:
        return
    dt = _dtype(case["dtype"])
    s["K"], s["V"] = (torch.zeros((B, Hkv, R, d), device="cuda", dtype=dt) for _ in range(2))
    s["S"] = torch.zeros((B, Hkv, R), device="cuda")
    s["pos"] = torch.zeros((B, Hkv, R), device="cuda", dtype=torch.int32)
    s["n"] = torch.zeros((B, Hkv), device="cuda", dtype=torch.int32)


def _views(s):
    """The slabs of the library's cache as views of the workspace that the program owns."""
    case, kv = s["case"], s["kv"]
    B, Hkv, R, d = case["batch"], case["kv_heads"], 2 * case["budget"], case["dim"]
    at = (-kv.workspace.data_ptr()) % ALIGN

    def view(dtype, *shape):
        nonlocal at
        size = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
        got = kv.workspace[at:at + size].view(dtype).view(shape)
        at += -(-size // ALIGN) * ALIGN
        return got

    s["K"], s["V"] = view(kv.tdtype, B, Hkv, R, d), view(kv.tdtype, B, Hkv, R, d)
    s["S"], s["pos"], s["n"] = view(torch.float32, B, Hkv, R), view(torch.int32, B, Hkv, R), view(torch.int32, B, Hkv)


def _prepare_pick(case, g, seed):
    B, T, V = case["batch"], case["draft"], case["vocab"]
    lens, parents, ways = _trees(case)
    logits = torch.empty((B, T, V), device="cuda", dtype=_dtype(case["logits"]))
    given = torch.zeros((B, T, V), device="cuda") if case["given"] else None
    tokens = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
    uniform = torch.rand((B, T), generator=g, device="cuda")
    noise = torch.empty((B, V), device="cuda").exponential_(generator=g)
    picked = tokens.tolist()
    heavy = math.log(V) + 2.0                                        # a token with this logit outweighs the rest of the row
    for b in range(B):
        for i in range(T):
            row = 2.0 * torch.randn(V, generator=g, device="cuda")
            below = [c for c in range(i + 1, lens[b]) if parents[b][c] == i]
            if i < lens[b] and below and given is not None:          # the drafter was fairly sure of the children it drew
                drawn = torch.randn(V, generator=g, device="cuda")
                drawn[[picked[b][c] for c in below]] = math.log(V)
                given[b, i] = torch.softmax(drawn, -1)
            ahead = [c for c in below if c in ways[b]] if i in ways[b] else []
            if ahead:                                                # the target agrees with one of them
                row[picked[b][ahead[0]]] = heavy + 4.0
            logits[b, i] = row.to(logits.dtype)
    for b in range(B):
        for i in range(1, lens[b]):                                  # accepted ones need not be lucky, the others are not
            uniform[b, i] = 0.5 * uniform[b, i] if i in ways[b] else 0.5 + 0.5 * uniform[b, i]
    masks = []
    for b in range(B):
        bits = []
        for i in range(lens[b]):
            bits.append((bits[parents[b][i]] if parents[b][i] >= 0 else 0) | (1 << i))
        masks.append([x - (1 << 64) if x >> 63 else x for x in bits + [0] * (T - lens[b])])
    s = dict(case=case, lens=lens, parents=parents, logits=logits, given=given, tokens=tokens, uniform=uniform, noise=noise,
             mask=torch.tensor(masks, dtype=torch.int64, device="cuda") if case["ragged"] else None)
    if own:
        from paper_2501_04987_b200 import TreeKV

        s["kv"] = TreeKV(64, 4, 4, 64, "bf16", B, T)
    return s


# ---- a pass --------------------------------------------------------------------------------------------------------
def run(s):
    return {"attend": _run_attend, "score": _run_score, "adopt": _run_adopt, "pick": _run_pick}[s["case"]["op"]](s)


def _rows(s, pool, b, n):
    """The first n tokens of sequence b: [KV heads, n, channels]."""
    page = s["case"]["page"]
    got = pool[s["table"][b, :-(-n // page)].long()]
    return got.permute(1, 0, 2, 3).reshape(pool.shape[1], -1, pool.shape[3])[:, :n]


def _logits(s, b, h, K, past, r0, r1, dtype=torch.float32):
    """Scaled products of the new tokens [r0, r1) of sequence b, of the heads of KV head h, with its tokens; minus infinity
    behind each.  [rows, heads of the group, tokens]."""
    case = s["case"]
    G, d = case["heads"] // case["kv_heads"], case["dim"]
    q = s["q"][b, r0:r1, h * G:(h + 1) * G].to(dtype)
    x = (q.reshape(-1, d) @ K.T).view(r1 - r0, G, -1) * (d ** -0.5)
    hide = torch.arange(K.shape[0], device="cuda")[None] > past + torch.arange(r0, r1, device="cuda")[:, None]
    return x.masked_fill(hide[:, None], -math.inf)


def _run_attend(s):
    if own:
        s["kv"].paged_attend(s["q"], s["k"], s["v"], s["kp"], s["vp"], s["table"], s["past_dev"], lens=s["new"],
                             max_past=max(s["past"]), out=s["out"], lse=s["lse"])
        return s["out"], s["lse"], s["kp"], s["vp"]
    case = s["case"]
    Hkv, page = case["kv_heads"], case["page"]
    G = case["heads"] // Hkv
    for b, (p, n) in enumerate(zip(s["past"], s["new"])):
        if n == 0:
            continue
        t = torch.arange(p, p + n, device="cuda")
        to = s["table"][b, t // page].long()
        s["kp"][to, :, t % page] = s["k"][b, :n]
        s["vp"][to, :, t % page] = s["v"][b, :n]
        K, V = _rows(s, s["kp"], b, p + n).float(), _rows(s, s["vp"], b, p + n).float()
        for h in range(Hkv):
            x = _logits(s, b, h, K[h], p, 0, n)
            top = x.amax(-1, keepdim=True)
            w = torch.exp(x - top)
            total = w.sum(-1, keepdim=True)
            s["out"][b, :n, h * G:(h + 1) * G] = ((w @ V[h]) / total).to(s["out"].dtype)
            s["lse"][b, :n, h * G:(h + 1) * G] = (top + torch.log(total))[..., 0]
    return s["out"], s["lse"], s["kp"], s["vp"]


def _run_score(s):
    if own:
        return s["kv"].paged_score(s["q"], s["lse"], s["kp"], s["table"], s["past_dev"], s["scores"], lens=s["new"],
                                   max_past=max(s["past"]))
    Hkv = s["case"]["kv_heads"]
    G = s["case"]["heads"] // Hkv
    for b, (p, n) in enumerate(zip(s["past"], s["new"])):
        if n == 0:
            continue
        K = _rows(s, s["kp"], b, p + n).float()
        for h in range(Hkv):
            w = torch.exp(_logits(s, b, h, K[h], p, 0, n) - s["lse"][b, :n, h * G:(h + 1) * G, None])
            s["scores"][b, h, :p + n] = w.sum((0, 1)) / G
    return s["scores"]


def _run_adopt(s):
    if own:
        s["kv"].adopt_pages(s["kp"], s["vp"], s["table"], s["scores"], s["past"], first=s["first"])
    else:
        _adopt(s, s["scores"], s["kp"], s["vp"])
    return s["K"], s["V"], s["S"], s["pos"], s["n"]


def _adopt(s, scores, kp, vp):
    case = s["case"]
    c, ns, nr = case["budget"], case["sinks"], case["recent"]
    for b, n in enumerate(s["past"]):
        if n == 0:
            continue
        token = torch.arange(n, device="cuda")
        weight = scores[b, :, :n]
        if case["rule"] == "average":
            weight = weight / (n - token.clamp(min=s["first"][b])).float()
        weight = torch.where((token < ns) | (token >= n - nr), math.inf, weight)
        L = min(n, c)
        kept = torch.sort(weight, dim=1, descending=True, stable=True).indices[:, :L].sort(dim=1).values     # [heads, L]
        i = max(n - c, 0) % (c - ns - nr)
        slot = torch.arange(L, device="cuda")
        row = torch.where(slot < ns + i, slot, slot + i)
        wide = kept[..., None].expand(-1, -1, case["dim"])
        s["K"][b, :, row] = _rows(s, kp, b, n).gather(1, wide)
        s["V"][b, :, row] = _rows(s, vp, b, n).gather(1, wide)
        s["S"][b, :, row] = scores[b, :, :n].gather(1, kept)
        s["pos"][b, :, row] = kept.to(torch.int32)
        s["n"][b] = n


def _run_pick(s):
    if own:
        warm = s["case"]["warm"]
        return s["kv"].pick_path(s["logits"], s["tokens"], s["uniform"] if warm else None, s["noise"] if warm else None, mask=s["mask"],
                                 lens=s["lens"], draft=s["given"] if warm else None, temperature=warm)
    B, T = s["tokens"].shape
    path = torch.full((B, T), -1, dtype=torch.int32, device="cuda")
    count = torch.zeros(B, dtype=torch.int32, device="cuda")
    after = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    warm = s["case"]["warm"]
    for b, n in enumerate(s["lens"]):
        at, depth = (0, 1) if n else (-1, 0)
        if n:
            path[b, 0] = 0
        while at >= 0:
            children = [i for i in range(at + 1, n) if s["parents"][b][i] == at]
            row = s["logits"][b, at].double()        # (64 bits: the draws are compared with values next to them)
            if warm == 0:
                best = torch.where(row == row.max(), torch.arange(len(row), device="cuda"), len(row)).min()   # (the first of equals)
                hit = next((i for i in children if s["tokens"][b, i] == best), -1)
                if hit < 0:
                    after[b] = best
            else:
                e = torch.exp((row - row.max()) / warm)
                left = e / e.sum()
                hit = -1
                for i in children:
                    x = s["tokens"][b, i].long()
                    q = 1.0 if s["given"] is None else s["given"][b, at, x].double()
                    if s["uniform"][b, i].double() * q * left.sum() < left[x]:
                        hit = i
                        break
                    if s["given"] is None:
                        left = left.clone()
                        left[x] = 0.0
                    else:
                        left = (left / left.sum() - s["given"][b, at].double()).clamp(min=0)
                if hit < 0:
                    after[b] = (left / s["noise"][b].double()).argmax()
            if hit >= 0:
                path[b, depth] = hit
                depth += 1
            at = hit
        count[b] = depth
    return path, count, after


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] in ("attend", "score") and work(case)["flops"] > 3e13:
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"attend": _exact_attend, "score": _exact_score, "adopt": _exact_adopt, "pick": _exact_pick}[case["op"]](s)


def _token_rows(s, pool, b, h, n):
    """Tokens 0..n-1 of one KV head, fetched one by one from where they lie, in 64 bits."""
    t = torch.arange(n, device="cuda")
    page = s["case"]["page"]
    return pool[s["table"][b].long()[t // page], h, t % page].double()


def _exact_attend(s):
    case = s["case"]
    B, T, Hq, d = s["q"].shape
    Hkv, page = case["kv_heads"], case["page"]
    G = Hq // Hkv
    out = torch.zeros((B, T, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, T, Hq), dtype=torch.float64, device="cuda")
    for b in range(B):
        for i in range(s["new"][b]):
            x = s["past"][b] + i
            s["kp"][s["table"][b, x // page], :, x % page] = s["k"][b, i]
            s["vp"][s["table"][b, x // page], :, x % page] = s["v"][b, i]
    for b in range(B):
        p, n = s["past"][b], s["new"][b]
        for h in range(Hkv if n else 0):
            K, V = _token_rows(s, s["kp"], b, h, p + n), _token_rows(s, s["vp"], b, h, p + n)
            for g in range(G):
                for r in range(0, n, 512):
                    q = s["q"][b, r:min(n, r + 512), h * G + g].double()
                    a = torch.einsum("td,nd->tn", q, K) / math.sqrt(d)
                    own_at = p + r + torch.arange(len(q), device="cuda")
                    a = torch.where(torch.arange(p + n, device="cuda")[None] <= own_at[:, None], a, -math.inf)
                    z = torch.logsumexp(a, 1)
                    lse[b, r:r + len(q), h * G + g] = z
                    out[b, r:r + len(q), h * G + g] = torch.exp(a - z[:, None]) @ V
    return out, lse, s["kp"], s["vp"]


def _exact_score(s):
    case = s["case"]
    B, T, Hq, d = s["q"].shape
    Hkv = case["kv_heads"]
    G = Hq // Hkv
    got = torch.zeros(s["scores"].shape, dtype=torch.float64, device="cuda")
    for b in range(B):
        p, n = s["past"][b], s["new"][b]
        for h in range(Hkv if n else 0):
            K = _token_rows(s, s["kp"], b, h, p + n)
            for g in range(G):
                a = torch.einsum("td,nd->tn", s["q"][b, :n, h * G + g].double(), K) / math.sqrt(d) - s["lse"][b, :n, h * G + g, None].double()
                got[b, h, :p + n] += torch.tril(torch.exp(a), p).sum(0) / G
    return got


def _exact_adopt(s):
    case = s["case"]
    c, ns, nr = case["budget"], case["sinks"], case["recent"]
    for b, n in enumerate(s["past"]):
        if not n:
            continue
        L, i = min(n, c), max(n - c, 0) % (c - ns - nr)
        rows = [x if x < ns + i else x + i for x in range(L)]
        for h in range(case["kv_heads"]):
            # the definition compares the sums, or the averages as 32-bit numbers
            weight = s["scores"][b, h, :n].double().cpu()
            if case["rule"] == "average":
                weight = torch.stack([weight, n - torch.arange(n).clamp(min=s["first"][b]).double()])
                weight = (weight[0] / weight[1]).float().double()
            w = weight.tolist()
            free = range(min(ns, n), max(n - nr, min(ns, n)))
            if n > c:
                best = sorted(free, key=lambda t: (-w[t], t))[:c - ns - nr]
                kept = list(range(ns)) + sorted(best) + list(range(n - nr, n))
            else:
                kept = list(range(n))
            kept = torch.tensor(kept, device="cuda")
            page = s["table"][b].long()[kept // case["page"]]
            s["K"][b, h, rows], s["V"][b, h, rows] = s["kp"][page, h, kept % case["page"]], s["vp"][page, h, kept % case["page"]]
            s["S"][b, h, rows], s["pos"][b, h, rows] = s["scores"][b, h, kept], kept.to(torch.int32)
        s["n"][b] = n
    return s["K"], s["V"], s["S"], s["pos"], s["n"]


def _exact_pick(s):
    import numpy as np

    case = s["case"]
    B, T, V = s["logits"].shape
    path, count, after = np.full((B, T), -1, np.int32), np.zeros(B, np.int32), np.full(B, -1, np.int32)
    tokens, uniform = s["tokens"].cpu().numpy(), s["uniform"].cpu().double().numpy()
    for b in range(B):
        if not s["lens"][b]:
            continue
        way, done = [0], False
        while not done:
            row = s["logits"][b, way[-1]].cpu().double().numpy()
            below = [i for i, up in enumerate(s["parents"][b]) if up == way[-1]]
            if case["warm"] == 0:
                best = int(np.flatnonzero(row == row.max())[0])
                same = [i for i in below if tokens[b, i] == best]
                way, after[b], done = (way + same[:1], -1, False) if same else (way, best, True)
                continue
            row = row / case["warm"]
            p = np.exp(row - (row.max() + np.log(np.sum(np.exp(row - row.max())))))
            q = None if s["given"] is None else s["given"][b, way[-1]].cpu().double().numpy()
            done = True
            for i in below:
                x, mass = tokens[b, i], p.sum()
                if uniform[b, i] < (p[x] / mass if q is None else p[x] / mass / q[x]):
                    way.append(i)
                    done = False
                    break
                p = np.where(np.arange(V) == x, 0.0, p) if q is None else np.maximum(p / mass - q, 0.0)
            if done:
                after[b] = int(np.argmax(p / s["noise"][b].cpu().double().numpy()))
        path[b, :len(way)], count[b] = way, len(way)
    return tuple(torch.from_numpy(x).cuda() for x in (path, count, after))
