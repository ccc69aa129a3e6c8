"""The language backbone's operators at the edges of what their arguments may be, as far as that shows without a GPU."""
import glob
import os
import re

import numpy as np
import pytest

import paper_2607_12287_gb300 as pkg
from tests.test_backbone_checks import bf, ints, lib, rope, rope_backward  # noqa: F401 (lib: a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_asynchronous_copies_take_no_l2_policy():
    # 16-byte asynchronous copies with a policy operand have faulted, for a reason that was not found
    sources = glob.glob(os.path.join(ROOT, "paper_2607_12287_gb300", "csrc", "*.cu*"))
    assert sources
    for path in sources:
        assert not re.search(r"cp\.async\.c[ag]\.[a-z.:0-9_]*cache_hint", open(path).read(), re.I), path


@pytest.mark.parametrize("rows", [None, 0x10000, np.zeros(4, np.int32)])
def test_write_needs_its_rows(monkeypatch, rows):
    # how many rows there are is known from this tensor alone
    monkeypatch.setattr(pkg, "load", lambda *a: pytest.fail("library reached"))
    caches = bf(3, 4, 16, 2, 64)
    with pytest.raises(TypeError, match="rows"):
        pkg.ivit_kv_write(pkg.make_cache_layout(caches[0]), bf(3, 6, 2, 64), bf(3, 6, 2, 64), rows, ints(4), caches, caches)


@pytest.mark.parametrize("rows", [2 ** 30 + 1, 2 ** 31 - 1])
def test_rotation_refuses_rows_that_its_index_does_not_hold(lib, rows):  # noqa: F811
    cfg = pkg.make_rope_config(8, 2, 64)
    assert rope(lib, cfg, n=rows) == rope_backward(lib, cfg, n=rows) == pkg.IVIT_ERR_SHAPE
