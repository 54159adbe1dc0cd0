"""NaN values in units that a block meets one behind the other (mkv_chunk_attention).

A block notes the channels of NaN values among masked places for one unit at a time.  The units here are small (one or two key
tiles, and rows for one to all of the softmax warps), every KV head of every request has a NaN in its chunk, and there are
several times as many units as blocks: the next unit's notes come while the rows of the one before are being written.

The rows that see a NaN are NaN in its channel; everything else has the bits that it has with a zero in the NaN's place."""
import numpy as np
import pytest
import torch

import paper_2608_23834_b200 as M

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("d,hkv,group", [(128, 4, 2), (128, 8, 1), (128, 4, 8), (256, 4, 3), (256, 8, 1), (256, 4, 6)])
@pytest.mark.parametrize("longest", [40, 130, 250])
@pytest.mark.parametrize("most_new", [3, 16])
def test_nan_in_every_unit_of_a_block(d, hkv, group, longest, most_new):
    rng = np.random.RandomState(longest + most_new + d + group)
    gen = torch.Generator(device="cuda").manual_seed(longest)
    n = 160
    lens = rng.randint(most_new, longest + 1, n)
    new = rng.randint(1, most_new + 1, n)
    starts = np.concatenate([[0], np.cumsum(new)])
    n_pages = -(-lens // 16)
    table = np.full((n, n_pages.max() + 1), -1, np.int32)
    ids = rng.permutation(n_pages.sum())
    for b in range(n):
        table[b, :n_pages[b]] = ids[n_pages[:b].sum():][:n_pages[b]]
    pool = M.Pool(d, hkv, hkv * group, len(ids), 1, np.ones(d, np.int8), max_batch=n)
    store = torch.randn(len(ids) * hkv * 32 * d, generator=gen, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)
    pool.fp8_arena[:store.numel()] = store
    pages = pool.fp8_arena[:store.numel()].view(len(ids), hkv, 32 * d)
    values = pages[..., 16 * d:].unflatten(-1, (d, 16))
    for b in range(n):                                               # what no token fills is NaN in any case
        if lens[b] % 16:
            values[table[b, n_pages[b] - 1], :, :, lens[b] % 16:] = 0x7F
    want = torch.zeros((starts[-1], hkv * group, d), dtype=torch.bool)
    at = []
    for b in range(n):
        for h in range(hkv):
            i, ch = int(rng.randint(0, new[b])), int(rng.randint(0, d))      # row i of the chunk and those behind it see the NaN
            token = lens[b] - new[b] + i
            at.append((table[b, token // 16], h, ch, token % 16))
            want[starts[b] + i:starts[b + 1], h * group:(h + 1) * group, ch] = True
    at, want = tuple(torch.tensor(x, device="cuda") for x in zip(*at)), want.cuda()
    q = torch.randn(want.shape, generator=gen, device="cuda").bfloat16()
    args = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (starts, table)]
    args += [torch.zeros(table.shape, dtype=torch.uint8, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")]
    ws, lse = pool.chunk_workspace(n, table.shape[1]), torch.zeros(q.shape[:2], device="cuda")
    values[at] = 0
    clean = pool.chunk_attention(q, *args, d ** -0.5, out=torch.zeros_like(q), lse=lse, workspace=ws)
    lse_clean = lse.clone()
    values[at] = 0x7F
    assert clean.isfinite().all()
    outs = [torch.zeros_like(q) for _ in range(50)]
    for out in outs:
        pool.chunk_attention(q, *args, d ** -0.5, out=out, lse=lse, workspace=ws)
    assert pool.status() == M.OK and torch.equal(lse, lse_clean)
    for out in outs:
        assert torch.equal(out.isnan(), want)
        assert torch.equal(torch.where(want, 0, out), torch.where(want, 0, clean))
