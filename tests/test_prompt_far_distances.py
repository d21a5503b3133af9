"""CPU checks of bucket starts for distances far past any sequence: the starts come at
once, and a plan whose last bucket begins too far away is refused."""
import pytest

import paper_2502_21079_amd as ad


@pytest.mark.timeout(20)
@pytest.mark.parametrize("n,far,both", [(32, 10 ** 9, True), (32, 1 << 40, False), (64, 10 ** 8, True), (3, 10 ** 12, False)])
def test_starts_of_far_distances(n, far, both):
    starts = ad.relative_bucket_starts(n, far, both)
    side = n // 2 if both else n
    e = side // 2
    assert len(starts) == side and starts[:e + 1] == tuple(range(e + 1))
    for m in range(1, side - e):
        reached = lambda d: d ** (side - e) * e ** m >= far ** m * e ** (side - e)  # noqa: E731
        assert reached(starts[e + m]) and not reached(starts[e + m] - 1)


@pytest.mark.timeout(20)
@pytest.mark.parametrize("n,far,both", [(32, 10 ** 9, True), (3, ((1 << 32) + 5) ** 2, False)])
def test_a_plan_that_reaches_too_far_is_refused(n, far, both):
    """Also where a start would wrap to a small one."""
    assert ad.rel_bias_attn_workspace((1, 2, 100, 64), (1, 2, 100, 64), n, max_distance=far, bidirectional=both) == 0
