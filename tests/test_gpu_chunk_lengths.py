"""mkv_chunk_attention at the last lengths that an int32 holds: 2^31 - 1 tokens, whose pages are the same few again and again."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_23834_b200 as M

gpu = pytest.mark.gpu
LAST = (1 << 31) - 1


def make(d, page, pages, seed):
    """A pool of `pages` FP8 pages of one KV head, and what they hold: keys, values [pages][page][d]."""
    rng = np.random.RandomState(seed)
    k, v = rng.randn(pages, page, d).astype(np.float32), (rng.randn(pages, page, d) + 1).astype(np.float32)
    recs = [oracle.fp8_pack_block(k[i], v[i], page, 1.0, 1.0) for i in range(pages)]
    pool = M.Pool(d, 1, 2, pages, 1, np.ones(d, np.int8), max_batch=1, page_tokens=page)
    pool.fp8_arena[:pages * page * 2 * d] = torch.from_numpy(np.stack(recs).ravel()).cuda()
    kv = [oracle.fp8_unpack_block_f32(r, d, page // 16, 1.0, 1.0) for r in recs]
    return pool, [np.stack([x[i] for x in kv]).astype(np.float64) for i in (0, 1)]


def call(pool, q, new, table, tags):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    lse = torch.zeros(q.shape[:2], device="cuda")
    out = pool.chunk_attention(q, i32([0, new]), table[None], tags[None], i32([LAST]), pool.d ** -0.5, lse=lse)
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def reference(q, k, v, counts):
    """counts[row][page][token]: how often the row sees that token."""
    q, d = q.double().cpu().numpy(), q.shape[-1]
    out, lse, spread = np.zeros(q.shape), np.zeros(q.shape[:2]), np.zeros(q.shape)
    for i in range(q.shape[0]):
        for h in range(q.shape[1]):
            s = d ** -0.5 * (k @ q[i, h])
            w = counts[i] * np.exp(s - s.max())
            lse[i, h] = s.max() + np.log(w.sum())
            w /= w.sum()
            out[i, h], spread[i, h] = np.einsum("pt,ptc->c", w, v), np.einsum("pt,ptc->c", w, np.abs(v))
    return out, lse, spread


@gpu
@pytest.mark.parametrize("d,page", [(128, 1792), (256, 4096)])
def test_two_pages_of_the_longest_row(d, page):
    """All entries but the first and the last are invalid: skipped and flagged."""
    pool, (k, v) = make(d, page, 2, d)
    width, new = LAST // page + 1, 3
    table = torch.full((width,), -1, dtype=torch.int32, device="cuda")
    table[0], table[-1] = 1, 0
    q = torch.randn(new, 2, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    out, lse = call(pool, q, new, table, torch.zeros_like(table, dtype=torch.uint8))
    assert pool.status() == M.E_BOUNDS and pool.status() == M.OK
    counts = np.ones((new, 2, page))
    for i in range(new):
        counts[i, 0, LAST % page - new + i + 1:] = 0
    want, want_lse, spread = reference(q, k, v, counts)
    # fp16 probabilities 2^-11, fp32 sums of a few hundred terms 2^-13, bf16 output 2^-8 (no Stale pages: the rest is exact)
    assert (np.abs(out - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -13) * spread).all()
    assert (np.abs(lse - want_lse) <= 2.0 ** -16 * (1 + np.abs(want_lse))).all()


@gpu
def test_every_page_of_the_longest_row():
    """Every entry is page 0.  A block's accumulators take 2^24 key tiles / 148 / 2 each, eight products of 16 keys a tile: 4.5e5
    sums in fp32, each off by at most 2^-23 of what is there (0.055 in all), the row's sum four a tile and 2^-24 each."""
    d, page, new = 128, 1792, 2
    pool, (k, v) = make(d, page, 1, 9)
    width = LAST // page + 1
    table = torch.zeros(width, dtype=torch.int32, device="cuda")
    q = torch.randn(new, 2, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).bfloat16()
    out, lse = call(pool, q, new, table, torch.zeros_like(table, dtype=torch.uint8))
    assert pool.status() == M.OK
    counts = np.full((new, 1, page), width - 1.0)
    for i in range(new):
        counts[i, 0, :LAST % page - new + i + 1] += 1
    want, want_lse, spread = reference(q, k, v, counts)
    assert (np.abs(out - want) <= 2.0 ** -8 * np.abs(want) + 0.07 * spread).all()
    assert (np.abs(lse - want_lse) <= 0.014 + 2.0 ** -16 * (1 + np.abs(want_lse))).all()
