"""mkv_chunk_attention: a wait that runs out is reported, and the pool stays usable."""
import pytest
import torch

import paper_2608_23834_b200 as M
from test_gpu_chunk import Cache, run

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("d,group,requests", [
    (256, 6, [(2000, 40)]), (256, 1, [(30, 1), (300, 7)]),
    (128, 8, [(900, 40), (1000, 33)]),                            # two row tiles
    (128, 4, [(700, 3), (40, 1), (260, 5)])])                     # key tiles by turns, two accumulators joined
def test_a_limit_of_zero_gives_up_and_says_so(d, group, requests):
    c = Cache(d, 2, group, requests, 2, seed=51)
    pool = c.pool()
    ref = c.reference()
    for _ in range(3):
        pool.set_wait_limit_ns(0)
        run(c, pool)
        assert pool.status() == M.E_TIMEOUT and pool.status() == M.OK
        pool.set_wait_limit_ns(20_000_000)
        out, lse, _ = run(c, pool)
        assert pool.status() == M.OK
        c.check(out, lse, ref)


@gpu
def test_a_call_without_tokens_has_nothing_to_wait_for():
    c = Cache(128, 1, 4, [(0, 3), (0, 1)], seed=1)
    pool = c.pool()
    pool.set_wait_limit_ns(0)
    out, lse, _ = run(c, pool)
    assert pool.status() == M.OK and not out.any() and lse.isneginf().all()
