"""mkv_append_rotary against the rotation in 64 bits, and against Append for everything but the rotation.

Tolerance: the angle is off by 2^-32 of a turn and half a unit of its fp32 value (at most pi 2^-24), sine and cosine by
2^-22, and two products and a sum round by 2^-24 each: a turned dim, before its last rounding, is within
m 2^-20 (|x| + |y|) =: e of m (x cos - y sin).  Queries then round to bf16 (2^-8 of the element).  Keys: e4m3 rounds
monotonically, so the stored number lies between the e4m3 roundings of (exact - e) / k_scale and (exact + e) / k_scale."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_23834_b200 as M

gpu = pytest.mark.gpu
E = 2.0 ** -20


def frequencies(pairs, base=1e4):
    return base ** (-np.arange(pairs) / pairs)


def exact(x, positions, inv_freq, axes, interleaved, mscale):
    """x turned in 64 bits, and the bound e of every element."""
    x = x.double().cpu().numpy()
    p = np.atleast_2d(np.asarray(positions, np.float64))
    r = 2 * len(inv_freq)
    ang = (p[np.zeros(len(inv_freq), int) if axes is None else axes] * inv_freq[:, None]).T[:, None]
    i, j = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y, e = x.copy(), np.zeros_like(x)
    a, b = x[..., i], x[..., j]
    y[..., i], y[..., j] = mscale * (a * np.cos(ang) - b * np.sin(ang)), mscale * (b * np.cos(ang) + a * np.sin(ang))
    e[..., i] = e[..., j] = abs(mscale) * E * (np.abs(a) + np.abs(b))
    return y, e


def check_q(got, want):
    y, e = want
    off = np.abs(got.double().cpu().numpy() - y) - (2.0 ** -8 * np.abs(y) + 1.01 * e + 2.0 ** -133)
    assert off.max() <= 0, off.max()


def key_bytes(arena, pages, hkv, tiles, d):
    return arena[:pages * hkv * tiles * 32 * d].view(pages, hkv, tiles, 32 * d)


def check_k(pool, slots, want):
    y, e = want
    e = e / pool.cfg.k_scale + 2.0 ** -23 * np.abs(y) / pool.cfg.k_scale            # and the fp32 bounds' own rounding
    d, tiles = pool.d, pool.tiles
    rec = key_bytes(pool.fp8_arena, pool.cfg.fp8_pages, pool.hkv, tiles, d)
    keep = np.flatnonzero(slots >= 0)
    s = torch.from_numpy(slots[keep].astype(np.int64)).cuda()
    k = rec[..., :16 * d].unflatten(-1, (16, d))[s // (16 * tiles), :, s % (16 * tiles) // 16, s % 16]
    k = k.contiguous().view(torch.float8_e4m3fn).double().cpu().numpy()
    fp8 = lambda x: torch.from_numpy(x).float().clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy()
    z = y[keep] / pool.cfg.k_scale
    assert (k >= fp8(z - e[keep])).all() and (k <= fp8(z + e[keep])).all()


def scattered_slots(rng, n, page, pages, skip=0.1):
    """Runs of tokens in shuffled pages, some starting inside one, some single, some without a slot."""
    out, ids = [], list(rng.permutation(pages))
    while len(out) < n and ids:
        pid, at = ids.pop(), rng.randint(0, page) if rng.rand() < 0.5 else 0
        out += [pid * page + i for i in range(at, page if rng.rand() < 0.7 else rng.randint(at, page) + 1)]
    out = np.array(out[:n])
    assert len(out) == n
    out[rng.rand(n) < skip] = -1
    return out.astype(np.int32)


CASES = [  # d, hkv, group, rotary_dim, axes, interleaved
    (128, 2, 4, 128, 1, False), (128, 1, 8, 64, 1, True), (128, 3, 1, 16, 2, False), (256, 4, 6, 256, 1, False),
    (256, 1, 5, 96, 3, False), (256, 2, 8, 256, 3, True), (128, 8, 4, 128, 3, False)]


@gpu
@pytest.mark.parametrize("d,hkv,group,rotary_dim,n_axes,interleaved", CASES)
@pytest.mark.parametrize("n,page", [(1, 16), (2, 16), (37, 48), (255, 16), (256, 16), (271, 16), (700, 48), (1300, 832), (2300, 48)])
def test_against_the_rotation_in_64_bits(d, hkv, group, rotary_dim, n_axes, interleaved, n, page):
    check_case(d, hkv, group, rotary_dim, n_axes, interleaved, n, page)


@gpu
@pytest.mark.parametrize("d,hkv,group,rotary_dim,n_axes,interleaved,n,page", [
    (128, 1, 8, 64, 1, True, 9000, 16), (256, 1, 5, 96, 3, False, 4203, 48), (128, 3, 1, 16, 2, False, 2800, 16),
    (128, 2, 1, 128, 1, False, 4096, 16), (128, 2, 3, 128, 1, False, 4095, 16)])
def test_prompts_of_few_heads(d, hkv, group, rotary_dim, n_axes, interleaved, n, page):
    check_case(d, hkv, group, rotary_dim, n_axes, interleaved, n, page)


def check_case(d, hkv, group, rotary_dim, n_axes, interleaved, n, page):
    rng = np.random.RandomState(n + d + rotary_dim)
    pages = n // page * 3 + n // 4 + 4
    k_scale, v_scale, mscale = 0.5, 2.0, 1.25 if n % 2 else 1.0
    sigma = np.ones(d, np.int8)
    pool = M.Pool(d, hkv, hkv * group, pages, 1, sigma, k_scale, v_scale, page_tokens=page)
    plain = M.Pool(d, hkv, hkv * group, pages, 1, sigma, k_scale, v_scale, page_tokens=page)
    hq = hkv * group
    qkv = torch.from_numpy(rng.randn(n, hq + 2 * hkv, d).astype(np.float32)).bfloat16().cuda()
    q, k, v = qkv.split([hq, hkv, hkv], 1)
    slots = scattered_slots(rng, n, page, pages)
    positions = rng.randint(-1000, 1 << 20, (n_axes, n)).astype(np.int32)
    positions[:, 0] = (1 << 31) - 1                                        # the last position there is
    inv = frequencies(rotary_dim // 2)
    axes = None if n_axes == 1 else rng.randint(0, n_axes, rotary_dim // 2)
    if axes is not None:
        axes[-1] = n_axes - 1
    rot = M.Rotary(inv, axes, interleaved, mscale)
    sl, pos = torch.from_numpy(slots).cuda(), torch.from_numpy(positions if n_axes > 1 else positions[0]).cuda()
    before = qkv.clone()
    out = pool.append_rotary(q, k, v, sl, pos, rot)
    torch.cuda.synchronize()
    assert pool.status() == M.OK and torch.equal(qkv, before)
    check_q(out, exact(q, positions, inv, axes, interleaved, mscale))
    check_k(pool, slots, exact(k, positions, inv, axes, interleaved, mscale))
    # values, and what no token was written to, as Append leaves them
    plain.append(k.contiguous(), v.contiguous(), sl)
    a, b = (key_bytes(p.fp8_arena, pages, hkv, page // 16, d) for p in (pool, plain))
    assert torch.equal(a[..., 16 * d:], b[..., 16 * d:])
    # position 0 turns nothing: the whole store is Append's
    zero = torch.zeros_like(pos)
    pool.append_rotary(q, k, v, sl, zero, M.Rotary(inv, axes, interleaved))
    assert torch.equal(a, b)
    # in place, and through the native call
    wide = qkv.clone()
    wq = wide[:, :hq]
    assert pool.append_rotary(wq, wide[:, hq:hq + hkv], wide[:, hq + hkv:], sl, pos, rot, q_out=wq) is wq
    assert torch.equal(wq, out) and torch.equal(wide[:, hq:], qkv[:, hq:])


@gpu
@pytest.mark.parametrize("n", [5, 400, 4200])
def test_keys_only_and_queries_only(n):
    rng = np.random.RandomState(n)
    inv = frequencies(64)
    rot = M.Rotary(inv)
    a, b, c = (M.Pool(128, 2, 4, n // 16 + 15, 1, np.ones(128, np.int8)) for _ in range(3))
    q, k, v = (torch.from_numpy(rng.randn(n, h, 128).astype(np.float32)).bfloat16().cuda() for h in (4, 2, 2))
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda") + 77
    out = a.append_rotary(q, k, v, slots, pos, rot)
    assert b.append_rotary(None, k, v, slots, pos, rot) is None
    assert torch.equal(a.fp8_arena, b.fp8_arena)
    assert torch.equal(c.append_rotary(q, None, None, None, pos, rot), out) and not c.fp8_arena.any()
    assert a.append_rotary(q[:0], k[:0], v[:0], slots[:0], pos[:0], rot).shape == (0, 4, 128)


@gpu
@pytest.mark.parametrize("n", [20, 300, 8300])
def test_slots_beyond_the_store_are_flagged_and_saturation_and_nan(n):
    pages = max(30, n // 16 + 2)
    pool = M.Pool(128, 1, 1, pages, 1, np.ones(128, np.int8))
    q, k, v = (torch.ones(n, 1, 128, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    k[0], k[1, 0, 5], v[2] = 1e6, float("nan"), -1e6
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    slots[n - 1] = pages * 16
    slots[n - 2] = (1 << 31) - 1
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    rot = M.Rotary(frequencies(64))
    pool.append_rotary(q, k, v, slots, pos, rot)
    assert pool.status() == M.E_BOUNDS and pool.status() == M.OK
    rec = pool.fp8_arena[:pages * 4096].view(pages, 4096).view(torch.float8_e4m3fn).float()
    assert (rec[0, :128] == 448).all() and rec[0, 128 + 5].isnan() and (rec[0, 2048 + 2::16] == -448).all()
    written = rec[:, :2048].reshape(-1, 128)
    assert (written[2:n - 2] == 1).all() and not written[n - 2:].any()


@gpu
def test_captured_and_on_another_stream():
    n = 9
    rng = np.random.RandomState(3)
    pool, other = (M.Pool(256, 2, 6, 9, 1, np.ones(256, np.int8)) for _ in range(2))
    rot = M.Rotary(frequencies(128))
    q, k, v = (torch.from_numpy(rng.randn(n, h, 256).astype(np.float32)).bfloat16().cuda() for h in (6, 2, 2))
    slots = torch.from_numpy(rng.permutation(9 * 16)[:n].astype(np.int32)).cuda()
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pool.append_rotary(q, k, v, slots, pos, rot, q_out=out)
    pos.fill_(1234)
    g.replay()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    want = other.append_rotary(q, k, v, slots, pos, rot, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(pool.fp8_arena, other.fp8_arena)


@gpu
def test_refusals_on_a_device_pool():
    pool = M.Pool(128, 2, 4, 4, 1, np.ones(128, np.int8))
    rot = M.Rotary(frequencies(64))
    q, k, v = (torch.zeros(3, h, 128, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2))
    slots, pos = (torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2))
    ok = dict(q=q, k=k, v=v, slot_mapping=slots, positions=pos, rotary=rot, q_out=torch.zeros_like(q))
    for bad in (dict(q=q.float()), dict(k=k[:2]), dict(v=None), dict(q=None), dict(positions=pos.long()), dict(positions=pos[:2]),
                dict(positions=pos.cpu()), dict(slot_mapping=slots.long()), dict(q_out=torch.zeros_like(q).float()),
                dict(q=torch.zeros(3, 4, 132, dtype=torch.bfloat16, device="cuda")[..., :128]),
                dict(rotary=M.Rotary(frequencies(128))), dict(rotary=M.Rotary(frequencies(64), axes=np.arange(64) % 3))):
        with pytest.raises((AssertionError, M.MkvError)):
            pool.append_rotary(**{**ok, **bad})
    assert not pool.fp8_arena.any() and pool.status() == M.OK


@gpu
def test_outputs_that_overlap_inputs_are_refused_and_slices_of_one_buffer_are_not():
    n, hq, hkv, d = 5, 4, 2, 128
    pool, other = (M.Pool(d, hkv, hq, 4, 1, np.ones(d, np.int8)) for _ in range(2))
    rot = M.Rotary(frequencies(64))
    wide = torch.zeros(n, hq + 2 * hkv + hq + 1, d, dtype=torch.bfloat16, device="cuda")
    wide[:, :hq + 2 * hkv] = torch.randn(n, hq + 2 * hkv, d, device="cuda").bfloat16()
    before = wide.clone()
    q, k, v, room = wide.split([hq, hkv, hkv, hq + 1], 1)
    slots, pos = (torch.arange(n, dtype=torch.int32, device="cuda") for _ in range(2))
    flat = wide.view(-1)
    for bad in (wide[:, 1:1 + hq], wide[:, 5:5 + hq], flat[:n * hq * d].view(n, hq, d), flat[d:d + n * hq * d].view(n, hq, d)):
        with pytest.raises(M.MkvError) as e:
            pool.append_rotary(q, k, v, slots, pos, rot, q_out=bad)
        assert e.value.code == M.E_INVALID
    torch.cuda.synchronize()
    assert torch.equal(wide, before) and not pool.fp8_arena.any()
    want = other.append_rotary(q, k, v, slots, pos, rot)
    pool.append_rotary(q, k, v, slots, pos, rot, q_out=room[:, 1:])
    assert torch.equal(room[:, 1:], want) and torch.equal(wide[:, :hq + 2 * hkv], before[:, :hq + 2 * hkv])
    assert torch.equal(pool.fp8_arena, other.fp8_arena)


@gpu
@pytest.mark.parametrize("d,hkv,group,fmt", [(256, 2, 6, 2), (128, 2, 4, 1)])
def test_prompt_demotion_and_drafts_as_a_server_runs_them(d, hkv, group, fmt):
    """A prompt in chunks (rotated Append, chunk attention), its old pages demoted, then draft tokens and a decode step: every
    output against attention in 64 bits over what the store then holds."""
    rng = np.random.RandomState(7)
    hq, inv, total = hkv * group, frequencies(d // 2), 203
    sigma = (rng.randint(0, 2, d) * 2 - 1).astype(np.int8)
    pool = M.Pool(d, hkv, hq, 20, 20, sigma, tq3_format=fmt)
    rot, ws = M.Rotary(inv), pool.chunk_workspace(1, 20)
    seq = M.Seq(pool)
    qkv = torch.from_numpy(rng.randn(total + 5, hq + 2 * hkv, d).astype(np.float32)).bfloat16().cuda()
    scale, at = d ** -0.5, 0
    old = oracle.get_format()
    oracle.set_format(fmt)
    try:
        for step, (n, recent) in enumerate([(90, None), (113, 64), (4, None), (1, 32)]):
            q, k, v = qkv[at:at + n].split([hq, hkv, hkv], 1)
            slots = []
            for _ in range(n):
                page, slot, _ = seq.append()
                slots.append(page * 16 + slot)
            i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
            turned = pool.append_rotary(q, k, v, i32(slots), torch.arange(at, at + n, dtype=torch.int32, device="cuda"), rot,
                                        q_out=torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda"))
            at += n
            ids, tags = seq.row()
            args = [torch.from_numpy(ids.copy()[None]).cuda(), torch.from_numpy(tags.copy()[None]).cuda(), i32([at])]
            if step == 3:
                out = pool.decode_attention(turned, *args, scale, out=torch.empty(1, hq, d, device="cuda"))
            else:
                out = pool.chunk_attention(turned, i32([0, n]), *args, scale, out=torch.empty_like(turned), workspace=ws)
            torch.cuda.synchronize()
            keys, values = np.zeros((len(ids) * 16, hkv, d)), np.zeros((len(ids) * 16, hkv, d))
            for p, (pid, tag) in enumerate(zip(ids, tags)):
                raw = pool.page_read_raw(M.FMT_TQ3 if tag == M.TAG_STALE else M.FMT_FP8, int(pid)).reshape(hkv, -1)
                for h in range(hkv):
                    if tag == M.TAG_STALE:
                        kc, g, vc, sc, zp = oracle.tq3_unpack_block(raw[h], d, 1)
                        sc, zp = (x.view(np.float16).astype(np.float64) for x in (sc, zp))
                        keys[16 * p:16 * p + 16, h] = [oracle.tq3_decode_key(kc[t], g[t], sigma) for t in range(16)]
                        values[16 * p:16 * p + 16, h] = vc * sc + zp
                    else:
                        keys[16 * p:16 * p + 16, h], values[16 * p:16 * p + 16, h] = oracle.fp8_unpack_block_f32(raw[h], d, 1)
            for i in range(n):
                for hh in range(hq):
                    kk, vv = keys[:at - n + i + 1, hh // group], values[:at - n + i + 1, hh // group]
                    s = scale * (kk @ turned[i, hh].double().cpu().numpy())
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    # Stale scores are good to 2^-10 sum |q' k'| <= 2^-10 |q||k| scale (below 0.03 here), the rest to bf16
                    tol = 2.0 ** -8 * np.abs(w @ vv) + (np.expm1(2 * 2.0 ** -10 * scale * np.linalg.norm(kk, axis=1).max() *
                          np.linalg.norm(turned[i, hh].double().cpu().numpy())) + 2.0 ** -9) * (w @ np.abs(vv))
                    assert (np.abs(out[i, hh].double().cpu().numpy() - w @ vv) <= tol).all(), (step, i, hh)
            if recent is not None:
                moved = seq.age(recent)
                if moved:
                    pool.demote(i32([m[1] for m in moved]), i32([m[2] for m in moved]))
                    for m in moved:
                        seq.release(M.FMT_FP8, m[1])
        assert (seq.row()[1] == M.TAG_STALE).sum() >= 8 and pool.status() == M.OK
    finally:
        oracle.set_format(old)
