"""osd_cache_append refuses rotated queries over the queries, tokens at one distance or
at two (no GPU needed)."""
import pytest

from tests.test_cache_abi import P, append

Q = 0x1000000  # 2 x 3 tokens of 512 bytes


@pytest.mark.parametrize("qs,qos,at", [
    (256, 256, 16), (256, 256, -16), (256, 256, 5 * 512 + 496), (256, 256, -(5 * 512 + 496)),
    (1024, 1024, 496), (1024, 1024, -496), (1024, 1024, 2048 - 496), (1024, 1024, 5 * 2048 + 496), (1024, 1024, -5 * 2048 - 496),
    (1024, 1024, 2048), (1024, 512, 512), (512, 1024, 512), (256, 512, 0), (1024, 256, 512),
])
def test_outputs_over_queries_are_refused(qs, qos, at):
    assert append(vc=P(0x10000000), q=P(Q), qs=qs, qo=P(Q + at), qos=qos) == -1
