"""Drafted decoding at the sizes that choose the other kernel variants: projections of whole prompts, and accepted paths of few
sequences with long caches, whose units are owned by clusters of two, four and eight blocks.
"""
import pytest

from test_gpu_draft import U32, _draft, _filled, _mask_tensor, _norm_rope_close, _norm_rope_ref, _path_rows, _tables
from test_gpu_state import _image_parts

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


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("hq,hkv", [(3, 3), (8, 2), (32, 8), (1, 1)])
def test_norm_rope_of_a_prompt(gpu, dtype, d, hq, hkv):
    """Calls large enough for four heads per lane; head counts that do not fill a warp's groups, padding among the tokens."""
    import torch

    n = 4 * 148 * 32 // 3 if hq == 32 else 4801    # at least 32 warps for each of 148 SMs whatever the heads a warp takes
    kv = gpu.TreeKV(16, hq, hkv, d, dtype, 1, 0)
    g = torch.Generator(device="cuda").manual_seed(d + hq)
    qkv = (torch.randn((n, (hq + 2 * hkv) * d + 64), generator=g, device="cuda") * 3).to(kv.tdtype)[:, 64:]
    cos, sin = _tables(1500, d)
    pos = torch.randint(0, 1500, (n,), generator=g, device="cuda", dtype=torch.int32)
    pos[::7] = -1
    wq, wk = ((1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(kv.tdtype) for _ in range(2))
    mark = lambda h: torch.full((n, h, d), 7.0, device="cuda", dtype=kv.tdtype)
    real = pos >= 0
    for w1, w2, cs in ((wq, wk, True), (None, wk, True), (wq, None, False)):
        args = dict(q_weight=w1, k_weight=w2, positions=pos)
        if cs:
            args.update(cos=cos, sin=sin)
        q, k, v = kv.norm_rope(qkv, eps=1e-5, q=mark(hq), k=mark(hkv), v=mark(hkv), **args)
        (rq, rk), rv = _norm_rope_ref(kv, qkv, w1, w2, cos if cs else None, sin, pos.clamp(min=0), 1e-5)
        _norm_rope_close(q[real], rq[0][real], rq[1][real], dtype, d)
        _norm_rope_close(k[real], rk[0][real], rk[1][real], dtype, d)
        assert torch.equal(v[real].double(), rv[real])
        assert all(bool((x[~real] == 7).all()) for x in (q, k, v))
    assert kv.stats()["device_error"] == 0


def _with_positions(gpu, kv, chunk, tables, protect):
    """The content of kv in a context with in-cache positions and protected tokens."""
    image, tokens = kv.export_state()
    other = gpu.TreeKV(kv.budget, kv.n_heads, kv.n_kv_heads, kv.head_dim, kv.tdtype, kv.batch, chunk)
    if protect:
        other.set_protection(*protect)
    if tables:
        other.set_positions(*tables)
    other.import_state(image, tokens)
    return other


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 8, 2), ("bf16", 128, 2, 2), ("bf16", 128, 8, 1), ("bf16", 64, 8, 1), ("f32", 128, 4, 2),
                                            ("f32", 128, 8, 1), ("f32", 64, 8, 1)])
@pytest.mark.parametrize("budget", [300, 700, 1500])
@pytest.mark.parametrize("rope,protect", [(False, None), (True, None), (True, (4, 40)), (False, (4, 40))])
def test_accept_of_few_long_sequences(gpu, dtype, d, hq, hkv, budget, rope, protect):
    """One and two sequences, paths of 1 to 64 tokens over the end of a cycle, three drafts in a row: rows and positions of prefill
    chunks under a rule that does not look at scores, scores within the error of two ways to compute a weight."""
    import torch

    T = chunk = 64
    middle = budget - sum(protect or (0, 0))
    tables = _tables(budget + chunk, d) if rope else None
    for seen, took in (([budget + middle - 30], [[64], [1], [37]]), ([budget - 20, 2 * budget + 11], [[33, 64], [64, 5], [0, 1]])):
        B = len(seen)
        src, _ = _filled(gpu, dtype, d, hq, hkv, budget, seen, chunk, seed=90)
        kv, twin = (_with_positions(gpu, src, chunk, tables, protect) for _ in range(2))
        for x in (kv, twin):
            x.set_rule(gpu.RULE_KEEP_LEFT)
        for step, n in enumerate(took):
            q, k, v = _draft(kv, T, 91 + step)
            rows, paths = _path_rows(B, T, [T] * B, n, 95 + step)
            out, lse = kv.verify_tree(q, k, v, mask=_mask_tensor(rows))
            path = torch.tensor([(p + [0] * T)[:T] for p in paths], dtype=torch.int32, device="cuda")
            kv.accept_path(q, k, v, lse, path, n)
            pick, seq = path.long(), torch.arange(B, device="cuda")[:, None]
            twin.prefill_chunk(*(x[seq, pick].contiguous() for x in (q, k, v)), chunk_lens=n)
            (a, n1), (b, n2) = kv.export_state(), twin.export_state()
            A, B2 = _image_parts(torch, kv, a), _image_parts(torch, twin, b)
            assert n1 == n2 and all(torch.equal(A[i], B2[i]) for i in (0, 1, 3, 4)), step
            # every step so far added weights that both sides have within delta of the exact ones: (d + 8) rounding steps of a
            # logit's terms, whose magnitudes sum to under 60 here, twice, and one step per key for the sums
            lim = 2 * (2 * (2 * (d + 8) * U32 * 60 + (budget + 100) * U32)) * A[2].abs() + 1e-12
            assert bool(((A[2].double() - B2[2].double()).abs() <= lim).all()), step
        assert kv.stats()["device_error"] == 0 and twin.stats()["device_error"] == 0
        # a cluster's blocks leave the same bits every time
        again = _with_positions(gpu, src, chunk, tables, protect)
        again.set_rule(gpu.RULE_KEEP_LEFT)
        for step, n in enumerate(took):
            q, k, v = _draft(again, T, 91 + step)
            rows, paths = _path_rows(B, T, [T] * B, n, 95 + step)
            out, lse = again.verify_tree(q, k, v, mask=_mask_tensor(rows))
            again.accept_path(q, k, v, lse, torch.tensor([(p + [0] * T)[:T] for p in paths], dtype=torch.int32, device="cuda"), n)
        assert torch.equal(again.export_state()[0], a)
