"""The bounded wait for a CTA's copies after an aborted wait, against a model of its barriers."""
import os
import re

from paper_2602_08329_b200 import build as B
from tests.test_chunk_host import compiled, run


def test_the_drain_waits_for_each_slots_latest_fill(tmp_path_factory):
    run(compiled(tmp_path_factory, "drain"))


def test_no_kernel_waits_for_either_parity():
    """A barrier is always past the parity that is not under way: such a wait returns at once, whatever is in flight."""
    for name in os.listdir(B.CSRC):
        text = open(os.path.join(B.CSRC, name)).read()
        assert not re.search(r"mbar_try_wait\([^;]*, 0\) && !mbar_try_wait\([^;]*, 1\)", text), name
