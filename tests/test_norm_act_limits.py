"""The most tokens of GroupNorm with its activation: what the kernels' row
numbers and the prefetch behind the last one hold.  Every call here fails
validation before anything would be enqueued."""

import pytest

from tests.test_norm_act_abi import _norm

MOST = 1 << 30


@pytest.mark.parametrize("channels,groups", [(8, 1), (16, 2), (32, 32), (64, 8)])
@pytest.mark.parametrize("tokens", [MOST + 1, 2147479809, 2147481600, (1 << 31) - 3000, (1 << 31) - 1])
def test_more_tokens_are_refused(tokens, channels, groups):
    from paper_2412_02962_amd import pcpp
    over = dict(batch=1, tokens=tokens, channels=channels, groups=groups, drop=0.0)
    for backward in (False, True):
        assert _norm(pcpp, backward, over, wsb=1 << 40) == pcpp.PCPP_EINVAL
    assert pcpp.pcpp_group_norm_act_workspace_size(pcpp.make_norm_act_geom(**over)) == 0


@pytest.mark.parametrize("dtype", ["BF16", "F32"])
@pytest.mark.parametrize("channels,groups", [(8, 1), (16, 2), (32, 32), (64, 8)])
def test_the_most_tokens_have_a_workspace(channels, groups, dtype):
    """512 chunks of records and of two columns' sums, and the merged records."""
    from paper_2412_02962_amd import pcpp
    g = pcpp.make_norm_act_geom(1, MOST, channels, groups, dtype=getattr(pcpp, "PCPP_DTYPE_" + dtype))
    merged = -(-3 * groups // 4) * 4
    want = 4 * max(merged + 512 * 3 * groups, merged + 512 * 2 * groups + 512 * 2 * channels)
    assert pcpp.pcpp_group_norm_act_workspace_size(g) == want
    # the rows that a thread has on their way behind its last: 2 x 8 of as many as stand side by side
    assert MOST + 2 * 8 * (512 // (channels // 8)) < 1 << 31
