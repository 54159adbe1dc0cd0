"""Timed calls between a layer's QKV projection and its output: rotated Append, and attention of a chunk of new tokens.

Kinds of case:
  rotary  the queries, keys and values of some tokens as the projection leaves them: queries and keys are turned by
          their positions (one axis, or time / height / width), keys and values go to the FP8 pages of the cache
  chunk   attention of the last tokens of every request (a prompt's chunk, draft tokens to be verified, or a mixed
          batch) over the paged cache that holds them and everything before, FP8 and Stale pages under one softmax

Shapes are those of mkv_workloads: head_dim 128 and 256, 16-token pages and long pages, both record formats, first
tokens Anchor and a Recent window in FP8, the rest Stale.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
# query heads x head_dim x visible (query, key) pairs, and cached tokens x KV heads x head_dim, of a drawn case at most
MOST_PAIRS = 24 * 256 * 2048 * 57984
MOST_TOKENS = 2 * 59008 * 4 * 256
STALE = 2
LEVELS = {1: (0.2451171875, 0.755859375, 1.34375, 2.15234375), 2: (0.25, 0.75, 1.375, 2.25)}
BORDERS = {1: (0.50048828125, 1.0498046875, 1.748046875), 2: (0.5, 1.0625, 1.8125)}


def _rotary(name, tokens, requests, d, hkv, group, rotary_dim, axes=1, interleaved=False, fused=True, page=16, far=131072,
            skipped=0):
    return {"name": name, "kind": "rotary", "tokens": tokens, "requests": requests, "head_dim": d, "kv_heads": hkv,
            "group": group, "rotary_dim": rotary_dim, "axes": axes, "interleaved": interleaved, "fused": fused,
            "page": page, "far": far, "skipped": skipped}


def _chunk(name, batch, new_min, new_max, past_min, past_max, d, hkv, group, fmt, anchor, recent, page=16):
    return {"name": name, "kind": "chunk", "batch": batch, "new_min": new_min, "new_max": new_max, "past_min": past_min,
            "past_max": past_max, "head_dim": d, "kv_heads": hkv, "group": group, "format": fmt, "anchor": anchor,
            "recent": recent, "page": page}


def listed():
    return [
        # a decode step of a small batch: one token per request, nothing but latency
        _rotary("rotary_decode8", 8, 8, 128, 4, 8, 128),
        # a larger batch, a quarter of the head rotated in neighbouring pairs, two rows of a padded batch without a slot
        _rotary("rotary_decode64", 64, 64, 256, 4, 6, 64, interleaved=True, skipped=2),
        # a short odd prompt in long pages, tensors of their own
        _rotary("rotary_odd", 515, 2, 128, 4, 8, 128, fused=False, page=832),
        # the tokens of a video: time, height and width
        _rotary("rotary_video", 8191, 1, 128, 8, 4, 128, axes=3),
        # a prefill chunk of five requests, lengths that leave partial pages
        _rotary("rotary_prefill", 32768 + 77, 5, 256, 4, 6, 256),
        # four draft tokens of one short request to verify
        _chunk("verify_tiny", 1, 4, 4, 4092, 4092, 128, 1, 8, 1, 64, 256),
        # five draft tokens each of a small batch
        _chunk("verify_batch8", 8, 5, 5, 16384, 16384, 128, 4, 8, 2, 128, 1024),
        # a mixed batch: decoding requests beside the chunks of new ones, of very different lengths
        _chunk("mixed_ragged16", 16, 1, 700, 1, 20011, 128, 8, 4, 1, 64, 512),
        # prompts from the start: everything still in FP8
        _chunk("prefill_first", 3, 4097, 4097, 0, 0, 256, 4, 6, 1, 0, 4097),
        # a chunk in the middle of two prompts
        _chunk("chunk_middle", 2, 1000, 1000, 16384, 16384, 128, 8, 4, 2, 128, 1024),
        # pages of 1,792 tokens
        _chunk("chunk_blocks", 2, 513, 513, 58495, 58495, 256, 4, 6, 1, 1792, 5 * 1792, page=1792),
        # the last chunk of a long document: 59,008 tokens, almost everything Stale
        _chunk("chunk_long", 1, 2048, 2048, 56960, 56960, 256, 4, 6, 2, 256, 2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    d, hkv, group = rng.choice([(128, 1, 8), (128, 4, 8), (128, 8, 4), (128, 2, 3), (256, 4, 6), (256, 4, 6), (256, 2, 4), (256, 1, 1)])
    page = rng.choice([16] * 6 + [832, 1792])
    if rng.random() < 0.4:
        tokens = _log_int(rng, 1, 32768)
        axes = rng.choice([1, 1, 3])
        return {"kind": "rotary", "tokens": tokens, "requests": min(tokens, rng.randint(1, 9)), "head_dim": d, "kv_heads": hkv,
                "group": group, "rotary_dim": rng.choice([d, d, d // 2, 64]), "axes": axes, "interleaved": rng.random() < 0.3,
                "fused": rng.random() < 0.7, "page": page, "far": _log_int(rng, 4096, 1 << 22),
                "skipped": rng.choice([0, 0, 0, 1, min(tokens, 3)])}
    batch, new_max, past_max = _log_int(rng, 1, 32), _log_int(rng, 1, 4096), _log_int(rng, 1, 65536) - 1
    new_min = new_max if rng.random() < 0.5 else _log_int(rng, max(1, new_max // 64), new_max)
    past_min = past_max if rng.random() < 0.5 else past_max // rng.randint(2, 50)
    while (batch * new_max * (past_max + new_max // 2) * hkv * group * d > MOST_PAIRS
           or batch * (past_max + new_max + page) * hkv * d > MOST_TOKENS):
        if batch > 1:
            batch //= 2
        else:
            past_max, past_min = past_max // 2, past_min // 2
            new_max, new_min = max(1, new_max * 2 // 3), max(1, new_min * 2 // 3)
    recent = rng.choice([256, 512, 2048, 131072])
    anchor = rng.choice([0, 64, 256])
    if page > 16:
        anchor, recent = page * rng.choice([0, 1]), page * rng.randint(1, 5)
    return {"kind": "chunk", "batch": batch, "new_min": new_min, "new_max": new_max, "past_min": past_min,
            "past_max": past_max, "head_dim": d, "kv_heads": hkv, "group": group, "format": rng.choice([1, 2]),
            "anchor": anchor, "recent": recent, "page": page}


# ------------------------------------------------------------------------------------------- layout
def _spread(n, lo, hi, seed):
    """n lengths from lo to hi, spread over their logarithm, in a fixed shuffled order (zero allowed)."""
    x = np.random.RandomState(seed).permutation(n) / max(1, n - 1) if n > 1 else np.ones(1)
    return np.floor((lo + 1) * ((hi + 1) / (lo + 1)) ** x + 1e-6).astype(np.int64) - 1


def _requests(case):
    """(new tokens, cached tokens with the new ones, tier tag of every page) of the requests of a chunk case."""
    new = _spread(case["batch"], case["new_min"], case["new_max"], 7)
    lengths = new + _spread(case["batch"], case["past_min"], case["past_max"], 8)
    page, rows = case["page"], []
    for n, length in zip(new, lengths):
        tags = np.full(-(-int(length) // page), STALE, np.uint8)
        tags[:case["anchor"] // page] = 1
        tags[max(0, int(length) - max(case["recent"], int(n))) // page:] = 0
        rows.append(tags)
    return new, lengths, rows


def _key_bits(d, fmt):
    """Bit of a TQ3 tile record that holds bit b of the key code of token t, rotated dim i: [16, d, 3]."""
    t, i, b = np.meshgrid(np.arange(16), np.arange(d), np.arange(3), indexing="ij")
    if fmt == 2:
        s, k = i // 32, i % 32
        lane, j, e = 4 * (t % 8) + k % 16 // 4, s // 2, 4 * (s % 2) + 2 * (t // 8) + k // 16
        n, part = 4 * (e % 2) + k % 4, e // 2
    else:
        s = i % 16
        lane, j, n, part = 4 * (t % 8) + s % 8 // 2, i // 64, 2 * (t // 8 + 2 * (s // 8)) + s % 2, i // 16 % 4
    high = part >= 2                       # codes whose magnitude sits in the third word, their sign in the first or second
    word = 3 * j + np.where(high & (b < 2), 2, part % 2)
    bit = 4 * n + np.where(high, np.where(b < 2, 2 * (part % 2) + b, 3), b)
    return _word_bit(d, lane, word, bit)


def _value_bits(d):
    """The same of the value code of token t, channel c: [16, d, 3]."""
    t, c, b = np.meshgrid(np.arange(16), np.arange(d), np.arange(3), indexing="ij")
    words = np.array([[[0, 0, 1], [0, 0, 1]], [[1, 2, 2], [1, 2, 2]]])
    bytes_ = np.array([[[0, 1, 0], [2, 3, 2]], [[1, 0, 1], [3, 2, 3]]])
    block, row = c // 16, c % 16
    lane, r, half = 4 * (row % 8) + t % 8 // 2, row // 8 + 2 * (t // 8), t % 2
    group, at = block % 4 // 2, 3 * (4 * (block % 2) + r) + b
    return 48 * d + _word_bit(d, lane, 3 * (block // 4) + words[group, half, at // 8], 8 * bytes_[group, half, at // 8] + at % 8)


def _word_bit(d, lane, word, bit):
    per_lane = 3 * d // 64
    full = per_lane - 4 * (word // 4) >= 4
    return 8 * (word // 4 * 512 + lane * np.where(full, 16, 8) + word % 4 * 4) + bit


def _scale_half(d):
    """Half-word of the scale of every channel within the scale/zero section; its zero is two half-words on."""
    c = np.arange(d)
    return c // 32 * 64 + c % 8 * 8 + 4 * (c // 16 % 2) + c % 16 // 8


# ------------------------------------------------------------------------------------------- inputs
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE)


def _loud(seed, d):
    """Channel factors: two percent of the channels are eight times as large."""
    f = np.ones(d, np.float32)
    f[np.random.RandomState(seed % (1 << 31)).permutation(d)[:max(1, round(0.02 * d))]] = 8.0
    return torch.from_numpy(f).to(DEVICE)


def _fp8_pages(gen, pages, hkv, tiles, d, loud):
    """Keys [pages, hkv, tiles, 16, d] and values [pages, hkv, tiles, d, 16] in e4m3, as the FP8 store holds them."""
    k = (_normal(gen, pages, hkv, tiles, 16, d) * loud[0]).to(torch.float8_e4m3fn)
    v = (_normal(gen, pages, hkv, tiles, d, 16) * loud[1][:, None]).to(torch.float8_e4m3fn)
    return k, v


def _tq3_pages(gen, pages, hkv, tiles, d, fmt, loud):
    """Codes of Stale pages: keys and values [pages, hkv, tiles, 16, d] (0..7), norm corrections g
    [pages, hkv, tiles, 16], scales and zeros [pages, hkv, d] of the page."""
    x = _normal(gen, pages, hkv, tiles, 16, d)
    mag = torch.bucketize(x.abs(), torch.tensor(BORDERS[fmt], device=DEVICE))
    kc = (mag + 4 * (x < 0)).to(torch.uint8)
    # a rotated key has the norm of the key: its loud channels are spread over all dims
    spread = float((loud[0] ** 2).mean().sqrt())
    g = (spread * x.norm(dim=-1) / torch.tensor(LEVELS[fmt], device=DEVICE)[mag].norm(dim=-1)).half()
    v = _normal(gen, pages, hkv, tiles, 16, d) * loud[1]
    lo, hi = v.amin((2, 3)), v.amax((2, 3))
    scale, zero = ((hi - lo) / 7).half(), lo.half()
    vc = torch.round((v - zero.float()[:, :, None, None]) / scale.float()[:, :, None, None]).clamp(0, 7).to(torch.uint8)
    return kc, g, vc, scale, zero


def _bytes_of(bits):
    """[..., 8 n] truth values -> [..., n] bytes, lowest bit first."""
    return (bits.view(*bits.shape[:-1], -1, 8).to(torch.uint8) << torch.arange(8, device=DEVICE, dtype=torch.uint8)).sum(-1, dtype=torch.uint8)


def _records(kc, g, vc, scale, zero, d, fmt):
    """The bytes of the Stale pages: [pages, hkv, page bytes]."""
    pages, hkv, tiles = kc.shape[:3]
    three = torch.arange(3, device=DEVICE, dtype=torch.uint8)
    where = np.concatenate([_key_bits(d, fmt).ravel(), _value_bits(d).ravel()])
    from_ = torch.from_numpy(np.argsort(where)).to(DEVICE)
    out = torch.empty((pages, hkv, tiles * (12 * d + 32) + 4 * d), dtype=torch.uint8, device=DEVICE)
    for first in range(0, pages, max(1, 1024 // tiles)):
        part = slice(first, first + max(1, 1024 // tiles))
        bits = torch.cat([((c[part, ..., None] >> three) & 1).flatten(3) for c in (kc, vc)], -1)[..., from_]
        tile = torch.cat([_bytes_of(bits), g[part].contiguous().view(torch.uint8)], -1)
        out[part, :, :tiles * (12 * d + 32)] = tile.flatten(2)
    halves = torch.zeros((pages, hkv, 2 * d), dtype=torch.float16, device=DEVICE)
    at = torch.from_numpy(_scale_half(d)).to(DEVICE)
    halves[..., at], halves[..., at + 2] = scale, zero
    out[:, :, tiles * (12 * d + 32):] = halves.view(torch.uint8)
    return out


def _chunk_inputs(case, seed):
    """Everything a chunk case is made of, the pages both as what they stand for and as bytes."""
    d, hkv, group, page, fmt = (case[k] for k in ("head_dim", "kv_heads", "group", "page", "format"))
    new, lengths, rows = _requests(case)
    tiles, width = page // 16, max(1, max(len(r) for r in rows))
    rng = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    tags, used = np.zeros((case["batch"], width), np.uint8), np.zeros((case["batch"], width), bool)
    for b, r in enumerate(rows):
        tags[b, :len(r)], used[b, :len(r)] = r, True
    stale = used & (tags == STALE)
    n3, n8 = int(stale.sum()), int((used & ~stale).sum())
    table = np.full((case["batch"], width), -1, np.int32)
    table[stale], table[used & ~stale] = rng.permutation(n3), rng.permutation(n8)
    loud = _loud(seed, d), _loud(seed + 1, d)
    return {"sigma": rng.randint(0, 2, d) * 2 - 1, "new": new, "lengths": lengths, "rows": rows, "table": table, "tags": tags,
            "q": _normal(gen, int(new.sum()), hkv * group, d).bfloat16(),
            "fp8": _fp8_pages(gen, max(1, n8), hkv, tiles, d, loud), "tq3": _tq3_pages(gen, max(1, n3), hkv, tiles, d, fmt, loud)}


def _prepare_chunk(case, seed):
    d, hkv, page, fmt = case["head_dim"], case["kv_heads"], case["page"], case["format"]
    x = _chunk_inputs(case, seed)
    fp8 = torch.cat([t.flatten(3) for t in x["fp8"]], -1).flatten(2).view(torch.uint8)
    tq3 = _records(*x["tq3"], d, fmt)
    starts = np.concatenate([[0], np.cumsum(x["new"])]).astype(np.int32)
    s = {"kind": "chunk", "d": d, "page": page, "scale": d ** -0.5, "q": x["q"], "out": torch.zeros_like(x["q"]),
         "starts": torch.from_numpy(starts).to(DEVICE), "bt": torch.from_numpy(x["table"]).to(DEVICE),
         "tags": torch.from_numpy(x["tags"]).to(DEVICE), "lens": torch.from_numpy(x["lengths"].astype(np.int32)).to(DEVICE)}
    if own:
        import paper_2608_23834_b200 as M
        s["pool"] = M.Pool(d, hkv, hkv * case["group"], fp8.shape[0], tq3.shape[0], x["sigma"], max_batch=case["batch"],
                           device=DEVICE, page_tokens=page, tq3_format=fmt)
        s["pool"].fp8_arena[:fp8.numel()].copy_(fp8.view(-1))
        s["pool"].tq3_arena[:tq3.numel()].copy_(tq3.view(-1))
        s["workspace"] = s["pool"].chunk_workspace(case["batch"], x["table"].shape[1])
    else:
        hadamard = torch.ones((1, 1), device=DEVICE)
        while hadamard.shape[0] < d:
            hadamard = torch.kron(torch.tensor([[1.0, 1.0], [1.0, -1.0]], device=DEVICE), hadamard)
        s.update(fp8=fp8, tq3=tq3, new=x["new"].tolist(), lengths=x["lengths"].tolist(),
                 rotation=torch.from_numpy(x["sigma"]).float().to(DEVICE)[:, None] * hadamard * d ** -0.5,
                 levels=torch.tensor(LEVELS[fmt] + tuple(-v for v in LEVELS[fmt]), device=DEVICE),
                 key_bits=torch.from_numpy(_key_bits(d, fmt)).to(DEVICE), value_bits=torch.from_numpy(_value_bits(d)).to(DEVICE),
                 scale_half=torch.from_numpy(_scale_half(d)).to(DEVICE),
                 stale=[torch.from_numpy(np.flatnonzero(r == STALE)).to(DEVICE) for r in x["rows"]],
                 other=[torch.from_numpy(np.flatnonzero(r != STALE)).to(DEVICE) for r in x["rows"]])
    return s


def _rotary_inputs(case, seed):
    d, hkv, hq, n = case["head_dim"], case["kv_heads"], case["kv_heads"] * case["group"], case["tokens"]
    page, R, pairs = case["page"], case["requests"], case["rotary_dim"] // 2
    rng = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    if case["fused"]:
        q, k, v = _normal(gen, n, hq + 2 * hkv, d).bfloat16().split([hq, hkv, hkv], 1)
    else:
        q, k, v = (_normal(gen, n, h, d).bfloat16() for h in (hq, hkv, hkv))
    k.mul_(_loud(seed, d).bfloat16())
    v.mul_(_loud(seed + 1, d).bfloat16())
    # every request continues somewhere in its own shuffled pages, at a position of its own
    cuts = np.linspace(0, n, R + 1).astype(np.int64)
    inside = [int(np.random.RandomState(r).randint(0, page)) if r else 0 for r in range(R)]
    pages = [-(-(inside[r] + int(cuts[r + 1] - cuts[r])) // page) for r in range(R)]
    ids = rng.permutation(sum(pages)).astype(np.int64)
    slots, positions, first = [], [], 0
    for r in range(R):
        at = inside[r] + np.arange(cuts[r + 1] - cuts[r])
        slots.append(ids[first + at // page] * page + at % page)
        positions.append(at + rng.randint(0, case["far"]) // page * page)
        first += pages[r]
    slots, positions = np.concatenate(slots), np.concatenate(positions)
    if case["skipped"]:
        slots[n - case["skipped"]:] = -1
    if case["axes"] == 3:                   # frames of 28 x 36 patches
        positions = np.stack([positions // 1008, positions % 1008 // 36, positions % 36])
    inv_freq = 1e6 ** (-np.arange(pairs) / pairs)
    axis = np.minimum(np.arange(pairs) * 8 // pairs // 2, 2) if case["axes"] == 3 else np.zeros(pairs, np.int64)
    return q, k, v, slots, positions, inv_freq, axis, max(1, sum(pages)), rng.randint(0, 2, d) * 2 - 1


def _prepare_rotary(case, seed):
    d, hkv, page, hq = case["head_dim"], case["kv_heads"], case["page"], case["kv_heads"] * case["group"]
    q, k, v, slots, positions, inv_freq, axis, pages, sigma = _rotary_inputs(case, seed)
    s = {"kind": "rotary", "q": q, "k": k, "v": v, "slots": torch.from_numpy(slots.astype(np.int32)).to(DEVICE),
         "positions": torch.from_numpy(positions.astype(np.int32)).to(DEVICE),
         "q_out": torch.zeros((case["tokens"], hq, d), dtype=torch.bfloat16, device=DEVICE)}
    if own:
        import paper_2608_23834_b200 as M
        s["pool"] = M.Pool(d, hkv, hq, pages, 1, sigma, device=DEVICE, page_tokens=page)
        s["rotary"] = M.Rotary(inv_freq, axes=axis if case["axes"] > 1 else None, interleaved=case["interleaved"], device=DEVICE)
        s["kv"] = s["pool"].fp8_arena[:pages * hkv * page * 2 * d].view(torch.float8_e4m3fn)
    else:
        # one page more takes the tokens without a slot
        s["records"] = torch.zeros((pages + 1, hkv, page // 16, 32 * d), dtype=torch.uint8, device=DEVICE)
        s["kv"] = s["records"][:pages].view(-1).view(torch.float8_e4m3fn)
        s.update(page=page, pages=pages, interleaved=case["interleaved"], inv_freq=torch.from_numpy(inv_freq).to(DEVICE),
                 axis=torch.from_numpy(axis).to(DEVICE))
    return s


def prepare(case, seed):
    return _prepare_rotary(case, seed) if case["kind"] == "rotary" else _prepare_chunk(case, seed)


# ------------------------------------------------------------------------------------------ the pass
def _turned(x, cos, sin, interleaved):
    """The first 2 * pairs dims of every head turned, in 32 bits."""
    x, r = x.float(), 2 * cos.shape[-1]
    if interleaved:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., r:]], -1)
    a, b = x[..., :r // 2], x[..., r // 2:r]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., r:]], -1)


def _run_rotary(s):
    positions = s["positions"].double().reshape(-1, s["slots"].numel())
    angle = positions[s["axis"]].T * s["inv_freq"]
    cos, sin = (f(angle).float()[:, None] for f in (torch.cos, torch.sin))
    s["q_out"].copy_(_turned(s["q"], cos, sin, s["interleaved"]))
    k = _turned(s["k"], cos, sin, s["interleaved"]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    v = s["v"].float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    d, slots = k.shape[-1], s["slots"].long()
    slots = torch.where(slots < 0, s["pages"] * s["page"], slots)
    page, tile, at = slots // s["page"], slots % s["page"] // 16, slots % 16
    records = s["records"]
    records[..., :16 * d].unflatten(-1, (16, d))[page, :, tile, at] = k
    records[..., 16 * d:].unflatten(-1, (d, 16))[page, :, tile, :, at] = v
    return {"q": s["q_out"], "kv": s["kv"]}


def _codes(tiles, where):
    """3-bit codes of all records, [pages, hkv, tiles, 16, d]."""
    bits = (tiles[..., where // 8] >> (where % 8).to(torch.uint8)) & 1
    return bits[..., 0] + 2 * bits[..., 1] + 4 * bits[..., 2]


def _run_chunk(s):
    d, page = s["d"], s["page"]
    tiles, inside = page // 16, torch.arange(page, device=DEVICE)
    fp8 = s["fp8"].view(torch.float8_e4m3fn).unflatten(-1, (tiles, 32 * d))
    k8 = fp8[..., :16 * d].float().unflatten(-1, (16, d)).flatten(2, 3)                   # [pages, hkv, page, d]
    v8 = fp8[..., 16 * d:].float().unflatten(-1, (d, 16)).transpose(-1, -2).flatten(2, 3)
    tile = s["tq3"][..., :tiles * (12 * d + 32)].unflatten(-1, (tiles, 12 * d + 32))
    g = tile[..., 12 * d:].contiguous().view(torch.float16).float()
    k3 = (s["levels"][_codes(tile, s["key_bits"]).int()] * g[..., None]).flatten(2, 3)
    meta = s["tq3"][..., tiles * (12 * d + 32):].contiguous().view(torch.float16).float()
    scale, zero = meta[..., s["scale_half"]], meta[..., s["scale_half"] + 2]
    v3 = (_codes(tile, s["value_bits"]).float() * scale[:, :, None, None] + zero[:, :, None, None]).flatten(2, 3)
    hkv, first = k8.shape[1], 0
    for b, (new, length) in enumerate(zip(s["new"], s["lengths"])):
        lp3, lp8 = s["stale"][b], s["other"][b]
        id3, id8 = s["bt"][b][lp3].long(), s["bt"][b][lp8].long()
        q = s["q"][first:first + new].float().unflatten(1, (hkv, -1)).permute(1, 2, 0, 3).flatten(1, 2)     # [hkv, group * new, d]
        scores = torch.cat([(q @ s["rotation"]) @ k3[id3].transpose(0, 1).flatten(1, 2).transpose(1, 2),
                            q @ k8[id8].transpose(0, 1).flatten(1, 2).transpose(1, 2)], -1).mul_(s["scale"])
        at = torch.cat([lp3, lp8])[:, None] * page + inside
        seen = at.flatten() <= (torch.arange(new, device=DEVICE) + (length - new)).repeat(scores.shape[1] // new)[:, None]
        scores.masked_fill_(~seen, -math.inf).sub_(scores.amax(-1, keepdim=True)).exp_()
        # what no token of the request fills is not looked at
        values = torch.cat([v3[id3], v8[id8]]).transpose(0, 1).flatten(1, 2).masked_fill_((at.flatten() >= length)[:, None], 0)
        out = (scores @ values).div_(scores.sum(-1, keepdim=True))
        s["out"][first:first + new] = out.unflatten(1, (-1, new)).permute(2, 0, 1, 3).flatten(1, 2).bfloat16()
        first += new
    return s["out"]


def run(s):
    if s["kind"] == "rotary":
        if own:
            s["pool"].append_rotary(s["q"], s["k"], s["v"], s["slots"], s["positions"], s["rotary"], q_out=s["q_out"])
            return {"q": s["q_out"], "kv": s["kv"]}
        return _run_rotary(s)
    if own:
        return s["pool"].chunk_attention(s["q"], s["starts"], s["bt"], s["tags"], s["lens"], s["scale"], out=s["out"],
                                         workspace=s["workspace"])
    return _run_chunk(s)


def work(case):
    d, hkv, hq = case["head_dim"], case["kv_heads"], case["kv_heads"] * case["group"]
    if case["kind"] == "rotary":
        return {"bytes": case["tokens"] * (4 * hq * d + 6 * hkv * d + 4 * case["axes"] + 4), "flops": 0}
    new, lengths, rows = _requests(case)
    tiles, stale = case["page"] // 16, sum(int((r == STALE).sum()) for r in rows)
    pages = sum(len(r) for r in rows)
    nbytes = hkv * ((int(lengths.sum()) - stale * case["page"]) * 2 * d + stale * (tiles * (12 * d + 32) + 4 * d))
    pairs = int((new * (lengths - new) + new * (new + 1) // 2).sum())
    return {"bytes": nbytes + 5 * pages + 4 * hq * d * int(new.sum()), "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------------------- the same in 64 bits
def _exact_rotary(case, seed):
    q, k, v, slots, positions, inv_freq, axis, pages, _ = _rotary_inputs(case, seed)
    d, hkv, page, half = case["head_dim"], case["kv_heads"], case["page"], case["rotary_dim"] // 2
    turn = torch.from_numpy(np.atleast_2d(positions)[axis].astype(np.float64) * inv_freq[:, None]).to(DEVICE).T
    place = torch.exp(1j * turn)[:, None]
    pair = (torch.arange(half) * 2, torch.arange(half) * 2 + 1) if case["interleaved"] else (torch.arange(half), torch.arange(half) + half)
    turned = []
    for x in (q, k):
        x = x.double()
        z = torch.complex(x[..., pair[0]], x[..., pair[1]]) * place
        x[..., pair[0]], x[..., pair[1]] = z.real, z.imag
        turned.append(x)
    kv = torch.zeros((pages, hkv, page // 16, 32 * d), dtype=torch.float64, device=DEVICE)
    kept = np.flatnonzero(slots >= 0)
    p, t, a = (torch.from_numpy(x).to(DEVICE) for x in (slots[kept] // page, slots[kept] % page // 16, slots[kept] % 16))
    kept = torch.from_numpy(kept).to(DEVICE)
    kv[..., :16 * d].unflatten(-1, (16, d))[p, :, t, a] = turned[1][kept].clamp(-448, 448)
    kv[..., 16 * d:].unflatten(-1, (d, 16))[p, :, t, :, a] = v[kept].double().clamp(-448, 448)
    return {"q": turned[0], "kv": kv.view(-1)}


def _exact_chunk(case, seed):
    """Keys rotated back and values as real numbers, one request and head at a time."""
    x = _chunk_inputs(case, seed)
    d, page, group, fmt = case["head_dim"], case["page"], case["group"], case["format"]
    kc, g, vc, scale, zero = x["tq3"]
    levels = torch.tensor(LEVELS[fmt], dtype=torch.float64, device=DEVICE)
    i = torch.arange(d, device=DEVICE)
    odd = i[:, None] & i
    for shift in (4, 2, 1):
        odd = odd ^ (odd >> shift)
    back = (1.0 - 2.0 * (odd & 1)).double() * d ** -0.5 * torch.from_numpy(x["sigma"]).to(DEVICE)
    out, first = torch.zeros(x["q"].shape, dtype=torch.float64, device=DEVICE), 0
    for b, (new, length) in enumerate(zip(x["new"].tolist(), x["lengths"].tolist())):
        tags, ids = x["rows"][b], x["table"][b]
        for h in range(case["kv_heads"]):
            n = len(tags)
            keys = torch.zeros((n, page, d), dtype=torch.float64, device=DEVICE)
            values = torch.zeros_like(keys)
            at8, at3 = np.flatnonzero(tags != STALE), np.flatnonzero(tags == STALE)
            id8, id3 = (torch.from_numpy(ids[a].astype(np.int64)).to(DEVICE) for a in (at8, at3))
            keys[at8] = x["fp8"][0][id8, h].double().flatten(1, 2)
            values[at8] = x["fp8"][1][id8, h].double().transpose(-1, -2).flatten(1, 2)
            code = kc[id3, h].long()
            c = levels[code & 3] * (1 - 2 * (code >> 2)).double() * g[id3, h].double()[..., None]
            keys[at3] = (c @ back).flatten(1, 2)
            values[at3] = (scale[id3, h].double()[:, None, None] * vc[id3, h].double() + zero[id3, h].double()[:, None, None]).flatten(1, 2)
            keys, values = keys.view(-1, d)[:length], values.view(-1, d)[:length]
            for r in range(group):
                s = (x["q"][first:first + new, h * group + r].double() @ keys.T) * d ** -0.5
                s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(length - new + 1), -math.inf)
                out[first:first + new, h * group + r] = torch.softmax(s, -1) @ values
        first += new
    return out


def exact(case, seed):
    return _exact_rotary(case, seed) if case["kind"] == "rotary" else _exact_chunk(case, seed)
