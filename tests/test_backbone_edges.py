"""The language backbone's operators at the edges of what their arguments may be, as far as that shows without a GPU."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_asynchronous_copies_take_no_l2_policy():
    # 16-byte asynchronous copies with a policy operand have faulted, for a reason that was not found
    sources = glob.glob(os.path.join(ROOT, "paper_2607_12287_gb300", "csrc", "*.cu*"))
    assert sources
    for path in sources:
        assert not re.search(r"cp\.async\.c[ag]\.[a-z.:0-9_]*cache_hint", open(path).read(), re.I), path
