"""The calls on pages and the path of a draft without a GPU: what the host turns down before it asks for a device."""
import ctypes as C

import pytest

INVALID = 1


@pytest.fixture(scope="module")
def binding():
    from paper_2501_04987_b200 import _build

    _build.build()
    from paper_2501_04987_b200 import binding as b

    return b


def test_no_context(binding):
    lib, some = binding.lib, C.c_void_p(4096)
    assert lib.treekv_paged_scratch_bytes(None, 4) == 0
    lens = (C.c_int32 * 1)(1)
    pages = (some, some, 4, 16, some, 2)
    assert lib.treekv_paged_attend(None, some, some, some, *pages, some, 16, some, some, lens, 1, some, 1 << 20, None) == INVALID
    assert lib.treekv_paged_score(None, some, some, some, 4, 16, some, 2, some, 16, some, 32, 0, lens, 1, None) == INVALID
    assert lib.treekv_adopt_pages(None, *pages, some, 32, lens, None, None) == INVALID
    assert lib.treekv_pick_path(None, some, binding.TREEKV_BF16, 100, some, None, None, 1.0, some, some, some, some, some, lens, 1, None) == INVALID


def test_the_calls_are_part_of_the_class(binding):
    for name in ("paged_attend", "paged_score", "adopt_pages", "pick_path"):
        assert getattr(binding.TreeKV, name).__doc__
