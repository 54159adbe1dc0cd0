"""mkv_chunk_attention with queries far from 1: a power of two in the queries and its reciprocal in the scale change no bit."""
import pytest
import torch

import paper_2608_23834_b200 as M
from test_gpu_chunk import Cache, run

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("d,group,fmt", [(128, 8, 1), (128, 2, 2), (256, 5, 2)])
@pytest.mark.parametrize("power", [-104, -60, 60, 98, 103, 112])
def test_a_power_of_two_moved_from_the_scale_to_the_queries(d, group, fmt, power):
    c = Cache(d, 1, group, [(300, 40), (77, 1)], fmt, seed=101)
    c.q = torch.where(c.q.abs() < 2.0 ** -12, 0, c.q)              # (times 2^-104 they are normal numbers of bf16 then)
    want, want_lse, pool = run(c)
    c.check(want, want_lse, c.reference())
    c.q = (c.q.double() * 2.0 ** power).bfloat16()
    out, lse, _ = run(c, pool, scale=c.scale * 2.0 ** -power)
    assert pool.status() == M.OK
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@gpu
@pytest.mark.parametrize("d", [128, 256])
def test_infinite_and_zero_queries(d):
    c = Cache(d, 1, 2, [(90, 4)], seed=102)
    c.q[0, 0] = 0
    ref = c.reference()
    c.q[2, 1, 5] = float("inf")
    out, lse, pool = run(c)
    bad = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
    bad[2, 1] = True
    assert out[bad].isnan().all() and lse[bad].isnan().all()
    c.check(torch.where(bad[..., None], torch.from_numpy(ref[0]).cuda().bfloat16(), out),
            torch.where(bad, torch.from_numpy(ref[1]).cuda().float(), lse), ref)
