"""mkv_chunk_attention against dense attention in 64 bits over the cache's own numbers (unpacked by the oracle).

Tolerance, element by element, from the roundings on the way (each at most half a step):
  scores    FP8 pages: keys and the query are exact in fp16, products are summed in fp32.  Stale pages: the rotated query
            and level * g are rounded to fp16, 2^-11 each, so a score is off by at most
            E_t = 2^-10 |scale| sum_i |q'_i| |k'_ti| (and its square, covered by the 5 % on top), a weight by exp(2 E) - 1;
  weights   fp16, 2^-11, and exponential, row sum and products in fp32: 2^-13 in all for the lengths here;
  values    Stale: code * scale + zero in fp16, 2^-11;
  output    bf16, 2^-8 of the element.
So |out - exact| <= 2^-8 |exact| + (expm1(2 E) + 2^-10 + 2^-13) sum_t w_t |v_t|, and |lse - exact| <= E + 2^-16 (1 + |lse|)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_23834_b200 as M

gpu = pytest.mark.gpu
RECENT, ANCHOR, STALE = 0, 1, 2


class Cache:
    """Requests with random pages in both stores; `rows`: per request (length, new tokens)."""

    def __init__(self, d, hkv, group, requests, fmt=1, page=16, seed=0, k_scale=1.0, v_scale=1.0, stale=0.6, stale_new=False,
                 spare=3, loud=True):
        rng = np.random.RandomState(seed)
        self.d, self.hkv, self.group, self.page, self.fmt = d, hkv, group, page, fmt
        self.k_scale, self.v_scale = k_scale, v_scale
        self.lens = np.array([r[0] for r in requests], np.int32)
        self.new = np.array([r[1] for r in requests], np.int32)
        self.starts = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        B, tiles = len(requests), page // 16
        n_pages = [-(-int(n) // page) for n in self.lens]
        width = max(1, max(n_pages)) + 1
        self.tags = np.full((B, width), 77, np.uint8)                 # unused entries hold rubbish
        self.table = np.full((B, width), -5, np.int32)
        for b, n in enumerate(n_pages):
            first_new = max(0, int(self.lens[b] - self.new[b])) // page
            for p in range(n):
                full = (p + 1) * page <= self.lens[b]
                may = full and (stale_new or p < first_new)
                self.tags[b, p] = STALE if may and rng.rand() < stale else rng.choice([RECENT, ANCHOR])
        used = np.arange(width)[None] < np.array(n_pages)[:, None]
        is3 = used & (self.tags == STALE)
        n3, n8 = int(is3.sum()) + spare, int((used & ~is3).sum()) + spare
        self.table[is3] = rng.permutation(n3)[:int(is3.sum())]
        self.table[used & ~is3] = rng.permutation(n8)[:int((used & ~is3).sum())]
        self.sigma = (rng.randint(0, 2, d) * 2 - 1).astype(np.int8)
        old = oracle.get_format()
        oracle.set_format(fmt)
        self.fp8 = rng.randint(0, 256, (n8, hkv, tiles * 32 * d)).astype(np.uint8)   # rubbish in spare pages, NaN among it
        self.tq3 = np.zeros((n3, hkv, oracle.tq3_block_bytes(d, tiles)), np.uint8)
        factor = np.ones(d, np.float32)
        if loud:
            factor[rng.permutation(d)[:3]] = 8
        self.k = [np.zeros((int(n), hkv, d)) for n in self.lens]      # what the pages stand for
        self.v = [np.zeros((int(n), hkv, d)) for n in self.lens]
        self.kr = [np.zeros((int(n), hkv, d)) for n in self.lens]     # |k'| of Stale tokens, rotated; zero for FP8 ones
        for b in range(B):
            for p in range(n_pages[b]):
                at, n = p * page, min(page, int(self.lens[b]) - p * page)
                for h in range(hkv):
                    k, v = (rng.randn(page, d).astype(np.float32) * factor * s for s in (k_scale, v_scale))
                    if self.tags[b, p] == STALE:
                        rec = oracle.tq3_block_from_f32(k, v, self.sigma)
                        self.tq3[self.table[b, p], h] = rec
                        kc, g, vc, sc, zp = oracle.tq3_unpack_block(rec, d, tiles)
                        gf, scf, zpf = (x.view(np.float16).astype(np.float64) for x in (g, sc, zp))
                        levels = oracle.codebook()[0].astype(np.float64)
                        self.k[b][at:at + n, h] = np.stack([oracle.tq3_decode_key(kc[t], g[t], self.sigma) for t in range(page)])
                        self.kr[b][at:at + n, h] = levels[kc & 3] * gf[:, None]
                        self.v[b][at:at + n, h] = vc * scf + zpf
                    else:
                        rec = oracle.fp8_pack_block(k, v, n, k_scale, v_scale)
                        kf, vf = oracle.fp8_unpack_block_f32(rec, d, tiles, k_scale, v_scale)
                        # what no token fills is rubbish, NaN among it
                        whole = rec.reshape(tiles, 32 * d)
                        for t in range(n, page):
                            whole[t // 16, 16 * d:].reshape(d, 16)[:, t % 16] = 0x7F
                            whole[t // 16, :16 * d].reshape(16, d)[t % 16] = 0xFF
                        self.fp8[self.table[b, p], h] = whole.ravel()
                        self.k[b][at:at + n, h], self.v[b][at:at + n, h] = kf[:n], vf[:n]
        oracle.set_format(old)
        self.q = rng.randn(int(self.starts[-1]), hkv * group, d).astype(np.float32)
        self.q = torch.from_numpy(self.q).bfloat16()
        self.scale = d ** -0.5

    def pool(self):
        p = M.Pool(self.d, self.hkv, self.hkv * self.group, self.fp8.shape[0], self.tq3.shape[0], self.sigma, self.k_scale,
                   self.v_scale, max_batch=max(1, len(self.lens)), page_tokens=self.page, tq3_format=self.fmt)
        p.upload_arenas(self.fp8, self.tq3)
        return p

    def device(self):
        self.dev = [torch.from_numpy(x).cuda() for x in (self.starts, self.table, self.tags, self.lens)]
        return self.dev

    def reference(self, scale=None, far=False):
        """(out, lse, tolerance of out, tolerance of lse) in 64 bits.  far: scores so far apart that two more terms count.  A score
        is d / 16 additions in fp32, each off by at most 2^-24 of sum |q k|.  A probability below 2^-14 is off by up to 2^-25, half of
        fp16's least step, where the row's largest is 2^6 at least: 2^-31 of a weight of at most 1."""
        scale = self.scale if scale is None else scale
        n, hq, d = self.q.shape
        out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
        tol, tol_lse = np.zeros((n, hq, d)), np.zeros((n, hq))
        had = np.ones((1, 1))
        while had.shape[0] < d:
            had = np.kron([[1, 1], [1, -1]], had)
        q = self.q.double().numpy()
        qr = np.abs((q * self.sigma) @ had) * d ** -0.5
        for b in range(len(self.lens)):
            for i in range(int(self.new[b])):
                p, r = int(self.lens[b] - self.new[b]) + i, int(self.starts[b]) + i
                if p < 0:
                    continue
                for h in range(hq):
                    k, v, kr = (x[b][:p + 1, h // self.group] for x in (self.k, self.v, self.kr))
                    s = scale * (k @ q[r, h])
                    m = s.max()
                    w = np.exp(s - m)
                    lse[r, h] = m + np.log(w.sum())
                    w /= w.sum()
                    out[r, h] = w @ v
                    e = 1.05 * 2.0 ** -10 * abs(scale) * (kr @ qr[r, h]).max()
                    if far:
                        e += self.d / 16 * 2.0 ** -24 * abs(scale) * (np.abs(k) @ np.abs(q[r, h])).max()
                    tol[r, h] = 2.0 ** -8 * np.abs(out[r, h]) + (np.expm1(2 * e) + 2.0 ** -10 + 2.0 ** -13) * (w @ np.abs(v)) + 1e-30
                    if far:
                        tol[r, h] += 2.0 ** -31 * np.abs(v).sum(0)
                    tol_lse[r, h] = e + 2.0 ** -16 * (1 + abs(lse[r, h]))
        return out, lse, tol, tol_lse

    def check(self, out, lse, ref, rows=slice(None)):
        o, l, tol, tol_l = (x[rows] for x in ref)
        out, lse = out.double().cpu().numpy()[rows], lse.double().cpu().numpy()[rows]
        off = np.abs(out - o) - tol
        assert np.isfinite(out).all() and off.max(initial=-1) <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))
        empty = np.isneginf(l)
        assert (np.isneginf(lse) == empty).all() and not out[empty].any()
        assert (np.abs(lse[~empty] - l[~empty]) <= tol_l[~empty]).all()


def run(c, pool=None, scale=None, **kw):
    pool = pool or c.pool()
    starts, table, tags, lens = c.device()
    lse = torch.full(c.q.shape[:2], 9.0, device="cuda")
    out = pool.chunk_attention(c.q.cuda(), starts, table, tags, lens, c.scale if scale is None else scale, lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse, pool


SHAPES = [(128, 1, 8), (128, 2, 4), (128, 1, 1), (128, 1, 5), (256, 1, 6), (256, 2, 3), (256, 1, 7), (256, 1, 1)]


@gpu
@pytest.mark.parametrize("d,hkv,group", SHAPES)
@pytest.mark.parametrize("fmt,page", [(1, 16), (2, 16), (1, 48), (2, 832)])
def test_against_dense_attention(d, hkv, group, fmt, page):
    # single tokens, an empty chunk, a page's border, chunks that end inside a page, one row of pages longer than a key tile
    c = Cache(d, hkv, group, [(1, 1), (517, 1), (300, 0), (160, 37), (33, 33), (1000, 5), (129, 128), (96, 17)], fmt, page, seed=d + group)
    out, lse, pool = run(c)
    assert pool.status() == M.OK
    c.check(out, lse, c.reference())


@gpu
@pytest.mark.parametrize("d,group", [(128, 8), (128, 3), (256, 6), (256, 4)])
@pytest.mark.parametrize("stale", [0.0, 0.5, 1.0])
def test_units_shared_by_many_blocks(d, group, stale):
    """One request whose key tiles are spread over the whole grid: partials of every block are joined."""
    c = Cache(d, 1, group, [(6007, 3)], 1 + group % 2, seed=3, stale=stale)
    out, lse, pool = run(c)
    ref = c.reference()
    c.check(out, lse, ref)
    again, lse2, _ = run(c, pool)
    assert torch.equal(out, again) and torch.equal(lse, lse2) and pool.status() == M.OK


@gpu
@pytest.mark.parametrize("d", [128, 256])
def test_many_rows_and_units(d):
    c = Cache(d, 2, 4, [(700, 300), (333, 333), (90, 1)], 2, seed=5)
    out, lse, pool = run(c)
    c.check(out, lse, c.reference())


@gpu
@pytest.mark.parametrize("d,fmt", [(128, 1), (128, 2), (256, 1), (256, 2)])
def test_stale_pages_within_the_chunk(d, fmt):
    """Nothing keeps a page of the chunk from being Stale (a chunk whose pages have been demoted already): masks go by position."""
    c = Cache(d, 1, 4, [(400, 350), (64, 64), (170, 100)], fmt, seed=9, stale_new=True, stale=0.7)
    out, lse, pool = run(c)
    c.check(out, lse, c.reference())
    c = Cache(d, 1, 2, [(300, 250)], fmt, page=48, seed=10, stale_new=True, stale=0.7)
    out, lse, pool = run(c)
    c.check(out, lse, c.reference())


@gpu
@pytest.mark.parametrize("k_scale,v_scale", [(0.02, 0.003), (3.0, 40.0), (0.7, 1.9)])
@pytest.mark.parametrize("scale", [0.0, -0.05, 0.2])
def test_pool_scales_and_signs(k_scale, v_scale, scale):
    scale = scale / k_scale
    for d, fmt in ((128, 2), (256, 1)):
        c = Cache(d, 1, 3, [(190, 20), (50, 50)], fmt, seed=12, k_scale=k_scale, v_scale=v_scale)
        out, lse, pool = run(c, scale=scale)
        c.check(out, lse, c.reference(scale))


@gpu
@pytest.mark.parametrize("d", [128, 256])
def test_rows_that_see_nothing_and_rows_of_nobody(d):
    # more new tokens than cached ones: the first rows have negative positions; a length of zero
    c = Cache(d, 2, 3, [(5, 9), (0, 4), (40, 6)], seed=2)
    c.q = torch.cat([torch.full((2,) + c.q.shape[1:], float("nan")).bfloat16(), c.q, torch.full((3,) + c.q.shape[1:], float("nan")).bfloat16()])
    c.starts = c.starts + 2
    ref = c.reference()
    pool, dev = c.pool(), c.device()
    out = torch.full(c.q.shape, 3.5, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(c.q.shape[:2], 9.0, device="cuda")
    pool.chunk_attention(c.q.cuda(), *dev, c.scale, out=out, lse=lse, workspace=pool.chunk_workspace(3, c.table.shape[1]))
    assert pool.status() == M.OK
    c.check(out, lse, ref, slice(2, -3))
    for rows in (slice(0, 2), slice(-3, None)):
        assert (out[rows] == 3.5).all() and (lse[rows] == 9).all()


@gpu
def test_rows_of_a_fused_projection():
    c = Cache(256, 2, 3, [(100, 40), (300, 1)], 2, seed=4)
    pool, dev = c.pool(), c.device()
    want = pool.chunk_attention(c.q.cuda(), *dev, c.scale)
    wide = torch.full((41, 10, 256), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:7] = c.q.cuda()
    assert torch.equal(pool.chunk_attention(wide[:, 1:7], *dev, c.scale), want)
    out = torch.zeros_like(want)
    pool.chunk_attention(wide[:, 1:7], *dev, c.scale, out=out, workspace=pool.chunk_workspace(2, c.table.shape[1]))
    assert torch.equal(out, want)


@gpu
@pytest.mark.parametrize("d", [128, 256])
def test_nan_reaches_the_rows_that_see_it(d):
    """A NaN value or key of the chunk itself: rows before it are as without it, rows from it on are NaN (a value: in its
    channel)."""
    c = Cache(d, 1, 4, [(200, 90), (40, 3)], seed=6, stale=0.5)
    ref = c.reference()
    token = 150                                                     # row 40 of the chunk
    page, at = c.table[0, token // 16], token % 16
    assert c.tags[0, token // 16] != STALE
    clean = c.fp8[page].copy()
    c.fp8[page, 0, 16 * d:].reshape(d, 16)[7, at] = 0x7F
    out, lse, pool = run(c)
    bad = out.isnan()
    assert bad[40:90, :, 7].all() and bad.sum() == 50 * 4
    fixed = torch.where(bad, torch.from_numpy(ref[0]).cuda().bfloat16(), out)
    c.check(fixed, lse, ref)
    c.fp8[page] = clean
    c.fp8[page, 0, :16 * d].reshape(16, d)[at, 5] = 0xFF
    out, lse, pool = run(c)
    assert out[40:90].isnan().all() and lse[40:90].isnan().all()
    c.check(out, lse, ref, slice(0, 40))
    c.check(out, lse, ref, slice(90, None))


@gpu
def test_bad_entries_are_skipped_and_flagged():
    c = Cache(128, 1, 4, [(150, 20), (64, 5)], seed=8, stale=0.5)
    c.tags[0, 1], c.table[0, 1] = RECENT, 1 << 28                  # beyond the store
    c.tags[0, 3] = 9                                                # no such tier
    c.table[0, 4] = -1
    c.lens[1] = 10 ** 6                                             # beyond the table's row
    for p in (1, 3, 4):
        c.k[0][16 * p:16 * p + 16] = np.nan
    keep = np.ones(150, bool)
    keep[16:32] = keep[48:80] = False
    out, lse, pool = run(c)
    assert pool.status() == M.E_BOUNDS and pool.status() == M.OK
    for b in (0,):
        sub_k, sub_v = c.k[0][keep], c.v[0][keep]
        q = c.q.double().numpy()
        for i in (0, 7, 19):
            n = keep[:130 + i + 1].sum()
            s = c.scale * sub_k[:n, 0] @ q[i, 2]
            w = np.exp(s - s.max())
            want = (w / w.sum()) @ sub_v[:n, 0]
            assert np.abs(out[i, 2].double().cpu().numpy() - want).max() < 0.05
    # a request whose rows lie outside q is left out
    c = Cache(128, 1, 2, [(50, 3), (60, 4)], seed=8)
    pool, (starts, *rest) = c.pool(), c.device()
    good, bad = torch.zeros(7, 2, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(7, 2, 128, dtype=torch.bfloat16, device="cuda")
    ws = pool.chunk_workspace(2, c.table.shape[1])
    pool.chunk_attention(c.q.cuda(), starts, *rest, c.scale, out=good, workspace=ws)
    pool.chunk_attention(c.q.cuda(), torch.tensor([0, 3, 8], dtype=torch.int32, device="cuda"), *rest, c.scale, out=bad, workspace=ws)
    assert pool.status() == M.E_BOUNDS
    assert torch.equal(bad[:3], good[:3]) and not bad[3:].any()
    # a Stale page that is not full
    c = Cache(128, 1, 2, [(40, 4)], seed=8, stale=0)
    c.tags[0, 2], c.table[0, 2] = STALE, 0
    run_out, _, pool = run(c)
    assert pool.status() == M.E_BOUNDS and run_out.isfinite().all()


@gpu
def test_one_new_token_is_decode():
    """The same row through decode_attention: both are within their tolerance of the exact result."""
    c = Cache(256, 2, 6, [(700, 1), (33, 1), (1, 1)], 2, seed=11)
    out, lse, pool = run(c)
    dec = torch.zeros(3, 12, 256, device="cuda")
    dl = torch.zeros(3, 12, device="cuda")
    starts, table, tags, lens = c.dev
    pool.decode_attention(c.q.cuda(), table, tags, lens, c.scale, out=dec, lse=dl)
    ref = c.reference()
    c.check(out, lse, ref)
    assert (np.abs(out.double().cpu().numpy() - dec.double().cpu().numpy()) <= ref[2] + 2e-3).all()


@gpu
def test_graph_replay_reads_the_present_tables():
    """A captured call with another batch's lengths, tables and pages behind it at replay; two graphs with a workspace each."""
    a = Cache(128, 1, 4, [(200, 8), (70, 8)], 2, seed=21)
    b = Cache(128, 1, 4, [(90, 8), (203, 8)], 2, seed=22)
    width = max(a.table.shape[1], b.table.shape[1])
    n8, n3 = (max(getattr(x, s).shape[0] for x in (a, b)) for s in ("fp8", "tq3"))
    for x in (a, b):
        pad = width - x.table.shape[1]
        x.table, x.tags = np.pad(x.table, ((0, 0), (0, pad))), np.pad(x.tags, ((0, 0), (0, pad)))
        x.fp8, x.tq3 = (np.concatenate([y, np.zeros((n - y.shape[0],) + y.shape[1:], np.uint8)]) for y, n in ((x.fp8, n8), (x.tq3, n3)))
        x.sigma_ref = x.sigma
    pools = [x.pool() for x in (a, b)]
    state, graphs = [], []
    for x, pool in zip((a, b), pools):
        q, dev, out, ws = x.q.cuda(), x.device(), torch.zeros(x.q.shape, dtype=torch.bfloat16, device="cuda"), pool.chunk_workspace(2, width)
        lse = torch.zeros(x.q.shape[:2], device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pool.chunk_attention(q, *dev, x.scale, out=out, lse=lse, workspace=ws)
        state.append((q, dev, out, lse, ws))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for x, (q, dev, out, lse, ws) in zip((a, b), state):
        x.check(out, lse, x.reference())
    # other lengths at replay: the chunk of request 0 a token earlier (its last token is not there yet)
    a.lens[0] -= 1
    for x in (a.k, a.v, a.kr):
        x[0] = x[0][:-1]
    state[0][1][3].copy_(torch.from_numpy(a.lens))
    graphs[0].replay()
    torch.cuda.synchronize()
    a.check(state[0][2], state[0][3], a.reference())


@gpu
def test_many_requests_and_back_to_back_calls():
    rng = np.random.RandomState(0)
    c = Cache(128, 1, 2, [(int(n), int(min(n, m))) for n, m in zip(rng.randint(0, 90, 300), rng.randint(0, 4, 300))], 1, seed=31)
    pool, dev, q = c.pool(), c.device(), c.q.cuda()
    ws = pool.chunk_workspace(300, c.table.shape[1])
    outs = [torch.zeros(c.q.shape, dtype=torch.bfloat16, device="cuda") for _ in range(5)]
    lse = torch.zeros(c.q.shape[:2], device="cuda")
    for o in outs:
        pool.chunk_attention(q, *dev, c.scale, out=o, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    c.check(outs[0], lse, c.reference())
    assert all(torch.equal(o, outs[0]) for o in outs)


@gpu
def test_pages_behind_four_gigabytes():
    c = Cache(256, 4, 2, [(120, 20)], 1, seed=41, stale=0.5)
    far8, far3 = 140_000, 270_000                                   # 32,768 and 16,512 bytes a page
    pool = M.Pool(256, 4, 8, far8 + c.fp8.shape[0], far3 + c.tq3.shape[0], c.sigma, max_batch=1)
    f, t = pool.fp8_arena, pool.tq3_arena
    f[far8 * 32768:far8 * 32768 + c.fp8.size] = torch.from_numpy(c.fp8.ravel()).cuda()
    t[far3 * 16512:far3 * 16512 + c.tq3.size] = torch.from_numpy(c.tq3.ravel()).cuda()
    c.table = np.where(c.table < 0, c.table, c.table + np.where(c.tags == STALE, far3, far8)).astype(np.int32)
    out, lse, _ = run(c, pool)
    assert pool.status() == M.OK
    c.check(out, lse, c.reference())


@gpu
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right():
    c = Cache(256, 1, 6, [(2000, 40)], 2, seed=51)
    pool = c.pool()
    pool.set_wait_limit_ns(0)
    run(c, pool)
    assert pool.status() in (M.OK, M.E_TIMEOUT)
    pool.set_wait_limit_ns(20_000_000)
    out, lse, _ = run(c, pool)
    assert pool.status() == M.OK
    c.check(out, lse, c.reference())


@gpu
def test_refusals_on_a_device_pool():
    c = Cache(128, 2, 2, [(40, 4)], seed=1)
    pool, dev, q = c.pool(), c.device(), c.q.cuda()
    starts, table, tags, lens = dev
    ws = pool.chunk_workspace(1, table.shape[1])
    out = torch.full(c.q.shape, 2.0, dtype=torch.bfloat16, device="cuda")
    ok = dict(q=q, q_starts=starts, block_table=table, tier_tag=tags, seq_lens=lens, scale=0.1, out=out, workspace=ws)
    for bad in (dict(q=q.half()), dict(q=q[:, :2]), dict(q=q.transpose(0, 1)), dict(q_starts=starts.long()), dict(q_starts=starts[:1]),
                dict(block_table=table.long()), dict(tier_tag=tags[:, :1]), dict(seq_lens=lens.float()), dict(out=out.float()),
                dict(out=out[:2]), dict(lse=torch.zeros(4, 4, device="cuda", dtype=torch.float64)), dict(workspace=ws.float()),
                dict(seq_lens=lens.cpu()), dict(q=q[..., ::2].repeat(1, 1, 2)[..., ::2])):
        with pytest.raises((AssertionError, M.MkvError)):
            pool.chunk_attention(**{**ok, **bad})
    same = torch.zeros(2 * q.numel(), dtype=torch.bfloat16, device="cuda")
    for bad in (dict(scale=float("nan")), dict(scale=float("inf")), dict(workspace=ws[:1024]), dict(out=q),
                dict(q=same[:q.numel()].view(q.shape), out=same[512:512 + q.numel()].view(q.shape))):
        with pytest.raises(M.MkvError) as e:
            pool.chunk_attention(**{**ok, **bad})
        assert e.value.code == M.E_INVALID
    torch.cuda.synchronize()
    assert (out == 2).all() and not same.any() and pool.status() == M.OK
    # a row of its own has no stride to speak of
    one = pool.chunk_attention(q[3:].as_strided((1, 4, 128), (8, 128, 1)), torch.tensor([0, 1], dtype=torch.int32, device="cuda"), table, tags, lens, 0.1)
    assert torch.equal(one[0], pool.chunk_attention(q, starts, table, tags, lens, 0.1)[3]) and pool.status() == M.OK
    empty = pool.chunk_attention(q[:0], torch.zeros(2, dtype=torch.int32, device="cuda"), table, tags, lens, 0.1)
    assert empty.shape == (0, 4, 128)


@gpu
@pytest.mark.parametrize("d,group", [(128, 4), (128, 8), (256, 6)])
def test_many_calls_give_the_same_bits(d, group):
    """Units of every size, 200 calls in a row on one workspace and on two streams with a workspace each."""
    c = Cache(d, 2, group, [(517, 1), (1030, 5), (300, 40), (700, 33), (1, 1), (0, 3), (140, 140)], 2, seed=61, stale=0.6)
    pool, dev, q = c.pool(), c.device(), c.q.cuda()
    ws = [pool.chunk_workspace(7, c.table.shape[1]) for _ in range(2)]
    want = pool.chunk_attention(q, *dev, c.scale, out=torch.empty_like(q), workspace=ws[0])
    outs = [torch.zeros_like(q) for _ in range(8)]
    different = torch.zeros((), dtype=torch.int64, device="cuda")
    for i in range(200):
        pool.chunk_attention(q, *dev, c.scale, out=outs[i % 8], workspace=ws[0])
        if i % 8 == 7:
            different += sum((o != want).sum() for o in outs)
    streams = [torch.cuda.Stream() for _ in ws]
    torch.cuda.synchronize()
    for i in range(60):
        for k, s in enumerate(streams):
            pool.chunk_attention(q, *dev, c.scale, out=outs[4 * k + i % 4], workspace=ws[k], stream=s)
    torch.cuda.synchronize()
    different += sum((o != want).sum() for o in outs)
    assert different.item() == 0 and pool.status() == M.OK


@gpu
@pytest.mark.parametrize("d,group", [(128, 2), (128, 8), (256, 3)])
def test_nan_in_several_units_of_a_block(d, group):
    """NaN values in the chunks of many short requests: every block meets several such units one behind the other."""
    rng = np.random.RandomState(4)
    c = Cache(d, 4, group, [(int(n), int(min(n, 3 + n % 20))) for n in rng.randint(20, 200, 160)], 1, seed=71, stale=0.3)
    marks = []
    for b in range(0, 160, 2):
        token = int(c.lens[b] - c.new[b]) + b % int(c.new[b])          # a token of the chunk: rows before it do not see it
        page, at, h, ch = c.table[b, token // 16], token % 16, b % 4, (7 * b) % d
        c.fp8[page, h, 16 * d:].reshape(d, 16)[ch, at] = 0x7F
        marks.append((int(c.starts[b]) + b % int(c.new[b]), int(c.starts[b + 1]), h, ch))
    want = torch.zeros(c.q.shape, dtype=torch.bool)
    for r0, r1, h, ch in marks:
        want[r0:r1, h * group:(h + 1) * group, ch] = True
    for _ in range(3):
        out, lse, pool = run(c)
        assert pool.status() == M.OK and torch.equal(out.isnan().cpu(), want) and lse.isfinite().all()
    ref = c.reference()
    c.check(torch.where(want.cuda(), torch.from_numpy(ref[0]).cuda().bfloat16(), out), lse, ref)


@gpu
@pytest.mark.parametrize("d,group", [(128, 8), (128, 3), (256, 5)])
@pytest.mark.parametrize("scale", [1.5, -0.6])
def test_scores_that_keep_rising_and_falling(d, group, scale):
    """Scores hundreds of nats apart: every row's reference is raised many times, what lies far below it vanishes."""
    c = Cache(d, 1, group, [(900, 5), (300, 300), (2600, 2), (40, 40)], 1, seed=81, stale=0.0)
    ramp = lambda n: np.float32(2.0) ** np.round(np.linspace(-6, 3, n))[:, None]
    for b, up in enumerate((True, False, True, True)):
        n = int(c.lens[b])
        factor = ramp(n) if up else ramp(n)[::-1]                      # powers of two: e4m3 holds the products or their rounding
        for p in range(-(-n // 16)):
            at, m = 16 * p, min(16, n - 16 * p)
            k = np.zeros((16, d), np.float32)
            k[:m] = c.k[b][at:at + m, 0] * factor[at:at + m]
            v = np.zeros((16, d), np.float32)
            v[:m] = c.v[b][at:at + m, 0]
            rec = oracle.fp8_pack_block(k, v, m, 1.0, 1.0)
            c.fp8[c.table[b, p], 0] = rec
            kf, vf = oracle.fp8_unpack_block_f32(rec, d, 1, 1.0, 1.0)
            c.k[b][at:at + m, 0], c.v[b][at:at + m, 0] = kf[:m], vf[:m]
    out, lse, pool = run(c, scale=scale)
    assert pool.status() == M.OK
    ref = c.reference(scale, far=True)
    assert np.ptp(ref[1][np.isfinite(ref[1])]) > 100
    c.check(out, lse, ref)
