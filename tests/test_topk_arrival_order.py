"""In the operators on records of top logits too, what a workgroup posts is in
place before its arrival at the counter is issued (read from the assembly)."""
import os

import pytest

from paper_2310_07177_amd import build
from tests.test_arrival_order import ARRIVAL, WAIT_ALL, WRITE, assembly


@pytest.mark.parametrize("src,least", [("verify_topk.hip", 4), ("distill_topk.hip", 12)])
def test_posts_before_arrival(src, least, tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("needs hipcc")
    lines = assembly(src, str(tmp_path / "out.s"))
    arrivals = [k for k, l in enumerate(lines) if ARRIVAL.match(l)]
    assert len(arrivals) >= least
    for k in arrivals:
        for j in range(k - 1, -1, -1):
            if WAIT_ALL.match(lines[j]):
                break
            assert not WRITE.match(lines[j]), f"{src}: no wait between\n{lines[j]}\nand\n{lines[k]}"
