"""Host-only: the launches of w2l_groupnorm_fwd / _bwd at sizes up to the limits that w2l.h states.  A launch holds fewer than 2^32 threads along each axis (of the second and third at
most 65535 workgroups) and at most 160 KB of LDS a workgroup."""
import pytest

import paper_1812_07625_amd as P
from launches import build, launches

# (B, T, C, G, act, dtype): many short utterances and long ones in runs of frames; groups of 16 KB, a workgroup each; the longest utterance; all of a launch's limits at once
SIZES = [(65, 1 << 23, 32, 32, 2, 1), (65534, 8200, 32, 32, 3, 1), (65534, 32768, 64, 1, 0, 0), (1, 1 << 24, 8192, 8192, 2, 1), (127, 1 << 24, 512, 512, 1, 0), (65534, 1024, 2048, 256, 2, 1),
         (65534, 1024, 2048, 256, 3, 0), (60000, 4096, 2, 2, 3, 0), (2, 40, 24, 4, 3, 1), (1, 3, 8192, 8192, 2, 1)]


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    return build(tmp_path_factory.mktemp("recorder"))


def call(B, T, C, G, act, dtype):
    """Both calls, with operands at addresses of their own that nothing reads."""
    return """
B, T, C, G, act, dtype = %r
at = lambda i: i << 50
n = P.w2l_groupnorm_workspace_bytes(B, T, C, G, act, dtype)
assert n > 0
assert P.raw.w2l_groupnorm_fwd(at(1), at(2), at(3), at(4), at(5), at(6), at(7), B, T, C, G, 1e-5, act, dtype, at(8), n, None) == 0
print("backward")
assert P.raw.w2l_groupnorm_bwd(at(1), at(2), at(3), at(4), at(5), at(6), at(7), at(8), at(9), at(10), B, T, C, G, act, dtype, 0, at(11), n, None) == 0
""" % ((B, T, C, G, act, dtype),)


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_every_launch_is_one_that_can_be_made(recorder, size):
    all_ = launches(recorder, call(*size))
    assert all_
    for grid, block, lds in all_:
        assert grid[0] > 0 and 0 < grid[1] < 1 << 16 and grid[2] == 1 and block[1:] == (1, 1)
        assert grid[0] * block[0] < 1 << 32 and 64 <= block[0] <= 512 and lds <= 160 << 10, (grid, block, lds)


def test_one_launch_each_where_they_fit(recorder):
    """(parts are for sizes that need them: a batch of training has its launches, and no more)"""
    assert len(launches(recorder, call(16, 1500, 2048, 1, 2, 1))) == 4 and len(launches(recorder, call(8, 750, 1536, 32, 3, 1))) == 3
    assert len(launches(recorder, call(65, 1 << 23, 32, 32, 2, 1))) == 18  # three parts of 32 utterances, six launches each
    assert P.w2l_groupnorm_launch_config(65, 1 << 23, 32, 32, 2, 1) == (0, 1)


@pytest.mark.parametrize("size", [(1, 131072, 64, 32, 2, 1), (1, 1 << 24, 32, 32, 2, 1), (4, 60000, 512, 32, 3, 1), (1, 1 << 22, 512, 512, 2, 0), (2, 100000, 8, 1, 0, 0)], ids=str)
def test_runs_of_long_utterances_are_joined_once(recorder, size):
    """Not by each workgroup that needs their sums, which would be the square of an utterance's length: a launch that gives up to eight groups of an utterance a workgroup, each way."""
    B, T, C, G, act, dtype = size
    assert P.w2l_groupnorm_launch_config(*size)[0] == 0
    all_ = launches(recorder, call(*size))
    assert len(all_) == 6
    for grid, block, _ in (all_[1], all_[4]):
        assert grid == (-(-G // 8), B, 1) and block[0] == 256


@pytest.mark.parametrize("size", [(32, 700, 80, 80, 2, 1), (1, 3000, 512, 32, 2, 1)], ids=str)
def test_few_sums_cost_no_launch(recorder, size):
    assert P.w2l_groupnorm_launch_config(*size)[0] == 0 and len(launches(recorder, call(*size))) == 4
