"""Attention where its warps, tiles and types come to their ends."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2503_05330_b200 import binding  # noqa: E402,F401
import model_ref as ref  # noqa: E402,F401
from test_gpu_attend import DEV, KINDS, check, make_cache  # noqa: E402,F401


@pytest.mark.parametrize("kind,q_type", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,T,group,keys", [(5, 13, 2, 500), (7, 5, 4, 2000), (10, 16, 1, 129), (23, 7, 1, 128), (3, 64, 1, 300), (193, 1, 1, 40000), (7, 32, 1, 700)])
def test_rows_that_leave_warps_of_the_second_half_without_one(kind, q_type, d, N, T, group, keys):
    """129 to 224 rows: of the second 128 some warps' 32 have nobody, and those warps run ahead of the others.  The same bits every time."""
    att, args = check(1, N, T, group, 1, d, kind, q_type, 0, None, prefix_cap=keys + 3, prefix_lens=[keys], seed=N + T)
    first = args[1].clone()
    for _ in range(100):
        args[1].fill_(7.0)
        att(*args)
        assert torch.equal(args[1], first)
    assert not att.timed_out()


@pytest.mark.parametrize("kind,q_type", KINDS)
def test_own_rows_that_leave_warps_without_one(kind, q_type):
    att, args = check(1, 6, 33, 4, 1, 128, kind, q_type, 300, [0, 90, 128, 200, 267, 100], seed=70)          # 132 rows a path
    first = args[1].clone()
    for _ in range(100):
        args[1].fill_(7.0)
        att(*args)
        assert torch.equal(args[1], first)
