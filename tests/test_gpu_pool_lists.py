"""Forks of a small pool into more children than half of its pages: every child
has its own copy of its parent's last page."""
import numpy as np
import pytest
import torch

from test_gpu_pool import Pair

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.mark.parametrize("n_children,spare", [(63, 0), (63, 1), (63, 40), (62, 200), (15, 2),
                                              (3, 0), (1, 0)])
def test_more_children_than_half_of_the_pages(n_children, spare):
    """One parent of two pages: a copy for every child."""
    S = n_children + 1
    p = Pair(S, 3, 2 + n_children + spare)
    p.grow([20])
    print("[pool] fork into", n_children, flush=True)
    p.fork([0] * n_children, list(range(1, S)), [20] * S)
    p.check()
    assert p.ref.refused == 0


@pytest.mark.parametrize("n_pages", [60, 65, 70, 127, 128, 129])
def test_several_parents_and_pages_that_run_out(n_pages):
    """Twelve parents of two pages, forked at different lengths into 52
    children: the pages suffice for some of the copies, or for all."""
    S, n = 64, 12
    p = Pair(S, 2, n_pages, seed=n_pages)
    p.grow([17 + i for i in range(n)])
    rng = np.random.default_rng(n_pages)
    parents = [int(x) for x in rng.integers(0, n, S - n)]
    length = [17 + i for i in range(n)] + [0] * (S - n)
    print("[pool] fork of", n_pages, flush=True)
    p.fork(parents, [int(c) for c in n + rng.permutation(S - n)], length)
    p.check()
    p.release(list(range(0, S, 2)))
    p.compact()
    p.check()
    torch.cuda.synchronize()
