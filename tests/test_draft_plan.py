"""Host side of drafted decoding: the order in which sequences are copied within a batch, and refusals that need no GPU."""
import itertools
import random

import pytest

KEPT, EMPTY = 65535, 65534


@pytest.fixture(scope="module")
def binding():
    from paper_2501_04987_b200 import _build

    _build.build()
    from paper_2501_04987_b200 import binding as b

    return b


def _play(ops, n):
    """What the kernel does with a plan: each component has registers of its own for one loaded and one kept value."""
    held = list(range(n))                      # content of every sequence, named by its first owner; -1 empty
    loads, last = 0, None
    kept = {}
    for comp, src, dst, seen in ops:
        if src == EMPTY:
            assert seen == 0
            held[dst], last = -1, None
            continue
        if src == KEPT:
            value = kept[comp]
        elif last is not None and last[0] == (comp, src):
            value = last[1]                    # the loaded value serves all copies that follow one another
        else:
            value, loads = held[src], loads + 1
        assert seen == 100 + value             # the geometry that belongs to the content
        if dst == KEPT:
            assert comp not in kept            # one kept value per component
            kept[comp] = value
        else:
            held[dst] = value
        last = ((comp, src), value)
    return held, loads


def _check(binding, source):
    n = len(source)
    ops = binding.treekv_selftest_fork_plan(source, [100 + b for b in range(n)])
    assert len(ops) <= n + n // 2
    held, loads = _play(ops, n)
    assert held == [-1 if s < 0 else s for s in source], (source, ops)
    used = {s for b, s in enumerate(source) if s >= 0 and s != b}
    assert loads == len(used), "every source is read once"
    # components are independent: no sequence occurs in two of them
    owner = {}
    for comp, src, dst, _ in ops:
        for x in (src, dst):
            if x < EMPTY:
                assert owner.setdefault(x, comp) == comp
    assert sorted({c for c, _, _, _ in ops}) == list(range(len({c for c, _, _, _ in ops})))


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5])
def test_every_map_of_a_small_batch(binding, n):
    for source in itertools.product(range(-1, n), repeat=n):
        _check(binding, list(source))


@pytest.mark.parametrize("n", [31, 64, 65, 1000, 1024])
def test_random_maps_of_a_large_batch(binding, n):
    r = random.Random(n)
    for kind in range(6):
        if kind == 0:
            source = r.sample(range(n), n)                                     # rings only
        elif kind == 1:
            source = [r.randrange(-1, n) for _ in range(n)]
        elif kind == 2:
            source = [max(0, b - 1) for b in range(n)]                         # one chain
        elif kind == 3:
            source = [n - 1] * n                                               # one source
        elif kind == 4:
            source = [(b ^ 1) if (b ^ 1) < n else b for b in range(n)]         # as many rings as there can be
        else:
            source = [-1] * n
        _check(binding, source)


def test_bad_plans_are_refused(binding):
    assert binding.treekv_selftest_fork_plan([0, 2], [1, 1]) is None
    assert binding.treekv_selftest_fork_plan([-2], [1]) is None
    assert binding.treekv_selftest_fork_plan([0] * 1025, [1] * 1025) is None


def test_null_context_is_an_error_not_a_crash(binding):
    assert binding.treekv_norm_rope(None, 16, 64, 0, 0, 1e-6, 0, 0, 0, 0, 16, 16, 16, 1) == 1
    assert binding.treekv_verify_tree(None, 16, 16, 16, 0, 16, 16, None, 1) == 1
    assert binding.treekv_accept_path(None, 16, 16, 16, 16, 1, 16, 1, None) == 1
    assert binding.treekv_fork_sequences(None, [0]) == 1


def test_stats_that_could_not_be_read_raise(binding):
    """check=False reports what the device recorded; a call on a closed context has nothing to report."""
    import types

    closed = types.SimpleNamespace(_h=None, _stream=lambda: 0)
    for check in (True, False):
        with pytest.raises(binding.TreeKVError) as e:
            binding.TreeKV.stats(closed, check=check)
        assert e.value.status == 1
