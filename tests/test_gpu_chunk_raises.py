"""mkv_chunk_attention where a row's reference is raised inside key tiles: what is in tensor memory already is read back,
scaled down and read back again.

Every query is a head's factor times one pattern of signs and every FP8 key a level times that pattern, so a token's score is its
level; levels are small integers (exact in e4m3) that step up every 32 tokens, the columns of a softmax step.  Values of the later
steps are zero in a part of the channels, which leaves the outputs there to what was scaled down."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_chunk import STALE, Cache, run

gpu = pytest.mark.gpu


def set_fp8(c, b, levels, values, pattern):
    """Keys levels[t] * pattern and values[t] for the tokens of request b that lie in FP8 pages."""
    for p in range(-(-int(c.lens[b]) // 16)):
        if c.tags[b, p] == STALE:
            continue
        at, m = 16 * p, min(16, int(c.lens[b]) - 16 * p)
        for h in range(c.hkv):
            k, v = np.zeros((16, c.d), np.float32), np.zeros((16, c.d), np.float32)
            k[:m] = levels[at:at + m, None] * pattern * c.k_scale
            v[:m] = values[at:at + m]
            rec = oracle.fp8_pack_block(k, v, m, c.k_scale, c.v_scale)
            c.fp8[c.table[b, p], h] = rec
            kf, vf = oracle.fp8_unpack_block_f32(rec, c.d, 1, c.k_scale, c.v_scale)
            c.k[b][at:at + m, h], c.v[b][at:at + m, h] = kf[:m], vf[:m]


def set_queries(c, pattern):
    """+-1 and +-1/2 by turns of the heads."""
    factor = np.where(np.arange(c.q.shape[1]) % 2, 0.5, 1.0)[:, None]
    c.q = torch.from_numpy(np.ascontiguousarray(np.broadcast_to(factor * pattern, c.q.shape), np.float32)).bfloat16()


def octaves(c, n):
    """scale at which two levels are n octaves apart for a head of factor 1."""
    return n * np.log(2) / (c.d * c.k_scale)


@gpu
@pytest.mark.parametrize("d,hkv,group", [(128, 1, 8), (128, 2, 2), (256, 1, 6), (256, 2, 1)])
@pytest.mark.parametrize("step", [9, 10, 19])
def test_a_raise_at_every_step_of_a_tile(d, hkv, group, step):
    c = Cache(d, hkv, group, [(512, 140), (509, 5), (130, 130), (400, 64)], 1, seed=91, stale=0.0)
    rng = np.random.RandomState(5)
    pattern = rng.randint(0, 2, d) * 2.0 - 1
    set_queries(c, pattern)
    for b in range(4):
        n = int(c.lens[b])
        stairs = np.arange(n) // 32
        values = rng.randn(n, d).astype(np.float32)
        last = stairs[-1]
        for k in range(1, 4):                                        # a quarter of the channels each: none, one, two or three steps empty
            values[np.ix_(stairs > last - k, np.arange(k, d, 4))] = 0
        set_fp8(c, b, stairs, values, pattern)
    scale = octaves(c, step)
    out, lse, pool = run(c, scale=scale)
    assert pool.status() == 0
    c.check(out, lse, c.reference(scale, far=True))


@gpu
@pytest.mark.parametrize("d,hkv,group", [(128, 1, 8), (128, 2, 2), (256, 1, 6), (256, 2, 1)])
@pytest.mark.parametrize("fmt,v_scale", [(1, 0.7), (2, 3.0)])
def test_a_raise_in_the_tile_that_changes_the_format(d, hkv, group, fmt, v_scale):
    """The accumulator goes from the Stale values' unit to the FP8 values' and is scaled again for the higher scores behind."""
    c = Cache(d, hkv, group, [(512 + 140, 140), (1003, 5), (300, 64)], fmt, seed=92, stale=1.0, v_scale=v_scale, loud=False)
    rng = np.random.RandomState(6)
    pattern = rng.randint(0, 2, d) * 2.0 - 1
    set_queries(c, pattern)
    for b in range(3):
        n, first = int(c.lens[b]), int(np.flatnonzero(c.tags[b] != STALE)[0]) * 16
        stairs = 1 + np.maximum(np.arange(n) - first, 0) // 32
        values = (rng.randn(n, d) * v_scale).astype(np.float32)
        values[:, 1::2] = 0                                          # Stale values alone, of a weight of 2^-10 and less
        set_fp8(c, b, stairs, values, pattern)
    scale = octaves(c, 10)
    out, lse, pool = run(c, scale=scale)
    assert pool.status() == 0
    c.check(out, lse, c.reference(scale, far=True))


@gpu
@pytest.mark.parametrize("d,hkv,group", [(128, 1, 8), (128, 2, 2), (256, 1, 6), (256, 2, 1)])
@pytest.mark.parametrize("rise", [14, 24, 26, 28, 30])
def test_a_raise_by_many_octaves_keeps_what_the_reference_lagged_behind(d, hkv, group, rise):
    """A probability of 2^14 against the reference (seven octaves above it no raise is due) is 2^(14 - rise) after a raise, which
    fp16 holds also where it does not hold 2^-rise."""
    c = Cache(d, hkv, group, [(160, 4), (420, 9)], 1, seed=93, stale=0.0)
    rng = np.random.RandomState(7)
    pattern = rng.randint(0, 2, d) * 2.0 - 1
    set_queries(c, pattern)
    for b, first in ((0, 0), (1, 128)):                              # in a unit's first key tile, and in a later one
        n = int(c.lens[b])
        levels, values = np.zeros(n), rng.randn(n, d).astype(np.float32)
        levels[first + 40], levels[first + 64:] = 7, rise
        values[:, 1::2] = 0
        values[first + 40, 1::2] = 448
        set_fp8(c, b, levels, values, pattern)
    scale = octaves(c, 1)
    out, lse, pool = run(c, scale=scale)
    assert pool.status() == 0
    c.check(out, lse, c.reference(scale, far=True))
