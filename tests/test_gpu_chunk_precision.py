"""mkv_chunk_attention to the precision that its header states: tolerances element by element from the spread of its roundings.

Each rounding is off by u = 2^-11 of the value at most (fp16), and a value is rounded once:
  q'      the rotated query, one rounding per dim, the same for every key;
  k'      level * g of a Stale key, one rounding per magnitude of its codebook (four), the same for all its dims of that level;
  p       one rounding per probability;
  v       code * scale + zero of a Stale page, one rounding per channel and code, the same for all its tokens of that code.
To first order an output is off by sum_j a_j e_j over these roundings, |e_j| <= u, with
  a = scale q'_i sum_t w_t (v_t - out) k'_ti,   scale w_t (v_t - out) sum_(i of that level) q'_i k'_ti,   w_t v_t,   v sum_(t of that code) w_t.
Taken as independent and of mean zero, |sum| > L u sqrt(sum a^2) has a probability of at most 2 exp(-L^2 / 2) (Hoeffding); L = 7.5
leaves 1e-6 for the million elements looked at.  Second order: (7.5 u)^2 of the largest score variance, times sum w |v|.  FP8 pages and
plain queries are exact in fp16.  On top, as everywhere: bf16 output 2^-8 of the element, fp32 sums and exponentials 2^-13 of sum w |v|;
elements below fp16's normal numbers 2^-24 of the pool's value scale.  lse likewise, from the scores alone, and 2^-16 (1 + |lse|)."""
import numpy as np
import pytest

import oracle
import paper_2608_23834_b200 as M
from test_gpu_chunk import STALE, Cache, run

gpu = pytest.mark.gpu
U, L = 2.0 ** -11, 7.5


def hadamard(d):
    h = np.ones((1, 1))
    while h.shape[0] < d:
        h = np.kron([[1, 1], [1, -1]], h)
    return h


class Unpacked:
    """The tokens of one request and KV head: keys and values, and of the Stale ones what was rounded together."""

    def __init__(self, c, b, h):
        n, d = int(c.lens[b]), c.d
        self.k, self.v = c.k[b][:, h], c.v[b][:, h]
        self.stale = np.zeros(n, bool)
        self.kr, self.level = np.zeros((n, d)), np.zeros((n, d), int)      # rotated keys, magnitude of every dim
        self.code, self.page = np.zeros((n, d), int), np.arange(n) // c.page
        old = oracle.get_format()
        oracle.set_format(c.fmt)
        levels = oracle.codebook()[0].astype(np.float64)
        for p in np.flatnonzero(c.tags[b] == STALE):
            at, tiles = slice(p * c.page, (p + 1) * c.page), c.page // 16
            kc, g, vc, _, _ = oracle.tq3_unpack_block(c.tq3[c.table[b, p], h], d, tiles)
            self.stale[at] = True
            self.level[at] = kc & 3
            self.kr[at] = levels[kc & 3] * np.where(kc & 4, -1, 1) * g.view(np.float16).astype(np.float64)[:, None]
            self.code[at] = vc
        oracle.set_format(old)


def bounds(c, scale, rows, drop=None):
    """(out, lse, tolerances) of the given (request, row of its chunk, head).  drop: a token that is left out of the exact result."""
    had, res = hadamard(c.d), []
    seen = {}
    for b, i, head in rows:
        key = (b, head // c.group)
        if key not in seen:
            seen[key] = Unpacked(c, *key)
        x = seen[key]
        n = int(c.lens[b] - c.new[b]) + i + 1
        q = c.q[int(c.starts[b]) + i, head].double().numpy()
        qr = (q * c.sigma) @ had * c.d ** -0.5
        k, v, kr, stale, level = x.k[:n], x.v[:n], x.kr[:n], x.stale[:n], x.level[:n]
        keep = np.ones(n, bool)
        if drop is not None:
            keep[drop[drop < n]] = False
        s = np.where(keep, scale * (k @ q), -np.inf)
        w = np.exp(s - s.max())
        lse = s.max() + np.log(w.sum())
        w /= w.sum()
        out = w @ v
        a = w[:, None] * (v - out)
        same = np.stack([(qr * kr * (level == m)).sum(1) for m in range(4)], 1) * stale[:, None]      # [t][level]
        var = scale ** 2 * (qr ** 2) @ ((kr * stale[:, None]).T @ a) ** 2                             # q'
        var += scale ** 2 * (same ** 2).sum(1) @ a ** 2                                               # k'
        var += w ** 2 @ v ** 2                                                                        # p
        for p in np.unique(x.page[:n][stale]):                                                        # v
            t = np.flatnonzero(x.page[:n] == p)
            for code in range(8):
                var += ((w[t, None] * (x.code[t] == code) * v[t]).sum(0)) ** 2
        score = scale ** 2 * (((qr * kr) ** 2).sum(1) * stale + (same ** 2).sum(1))                   # variance of a score, in u^2
        second = (L * U) ** 2 * score.max(initial=0)
        spread = w @ np.abs(v)
        tol = 2.0 ** -8 * np.abs(out) + L * U * np.sqrt(var) + (second + 2.0 ** -13) * spread + 2.0 ** -24 * c.v_scale
        var_lse = scale ** 2 * ((qr ** 2) @ ((kr * stale[:, None]).T @ w) ** 2 + w ** 2 @ (same ** 2).sum(1))
        res.append((out, lse, tol, L * U * np.sqrt(var_lse) + second + 2.0 ** -16 * (1 + abs(lse))))
    return [np.array(x) for x in zip(*res)]


def some_rows(c, n, seed):
    rng = np.random.RandomState(seed)
    all_rows = [(b, i, h) for b in range(len(c.lens)) for i in range(int(c.new[b])) for h in range(c.hkv * c.group)
                if c.lens[b] - c.new[b] + i >= 0]
    return [all_rows[k] for k in rng.permutation(len(all_rows))[:n]]


CASES = [  # d, hkv, group, format, page, k_scale, v_scale
    (128, 1, 8, 1, 16, 1.0, 1.0), (128, 2, 4, 2, 16, 0.7, 3.0), (128, 1, 3, 2, 48, 1.0, 0.02), (256, 1, 6, 1, 16, 1.0, 1.0),
    (256, 2, 3, 2, 16, 3.0, 0.7), (256, 1, 1, 1, 48, 1.0, 1.0)]


def make(case, seed):
    d, hkv, group, fmt, page, ks, vs = case
    # short rows of few Stale tokens, and longer ones; one request that is all Stale but for its chunk
    return Cache(d, hkv, group, [(20 + page, 3), (40 + 2 * page, 9), (517, 6), (700, 40), (1300, 2)], fmt, page, seed=seed, k_scale=ks,
                 v_scale=vs, stale=0.9, loud=False)


@gpu
@pytest.mark.parametrize("case", CASES)
def test_within_the_spread_of_the_roundings(case):
    c = make(case, seed=case[0] + case[2])
    scale = c.scale / c.k_scale
    out, lse, pool = run(c, scale=scale)
    assert pool.status() == 0
    rows = some_rows(c, 150, 1)
    want, want_lse, tol, tol_lse = bounds(c, scale, rows)
    at = [int(c.starts[b]) + i for b, i, _ in rows], [h for _, _, h in rows]
    off = np.abs(out.double().cpu().numpy()[at] - want)
    off_lse = np.abs(lse.double().cpu().numpy()[at] - want_lse)
    assert (off <= tol).all(), (off / tol).max()
    assert (off_lse <= tol_lse).all(), (off_lse / tol_lse).max()


@gpu
@pytest.mark.parametrize("case", CASES)
def test_skipped_entries_within_the_same_tolerances(case):
    """Invalid entries in both formats, before the chunk and in it: the rows are those of the pages that are left."""
    c = make(case, seed=3 + case[0])
    c.lens, c.new, c.tags, c.table = c.lens[3:4], c.new[3:4], c.tags[3:4], c.table[3:4]
    c.starts = np.array([0, c.new[0]], np.int32)
    c.q, c.k, c.v = c.q[:c.new[0]], c.k[3:4], c.v[3:4]
    n_pages = -(-int(c.lens[0]) // c.page)
    stale, other = np.flatnonzero(c.tags[0, :n_pages] == STALE), np.flatnonzero(c.tags[0, :n_pages] != STALE)
    gone = np.array([stale[0], stale[len(stale) // 2], other[-2], other[-1]])
    whole, c.table = c.table, c.table.copy()
    c.table[0, gone] = [1 << 29, -1, -7, (1 << 31) - 1]
    scale = c.scale / c.k_scale
    out, lse, pool = run(c, scale=scale)
    assert pool.status() == M.E_BOUNDS and pool.status() == M.OK
    c.table = whole
    rows = some_rows(c, 60, 2)
    want, want_lse, tol, tol_lse = bounds(c, scale, rows, drop=(gone[:, None] * c.page + np.arange(c.page)).ravel())
    at = [i for _, i, _ in rows], [h for _, _, h in rows]
    assert (np.abs(out.double().cpu().numpy()[at] - want) <= tol).all()
    assert (np.abs(lse.double().cpu().numpy()[at] - want_lse) <= tol_lse).all()


@pytest.mark.parametrize("case", [CASES[0], CASES[4]])
@pytest.mark.parametrize("b,missing", [(0, 1), (1, 1), (2, 16)])
def test_the_tolerances_catch_missing_tokens(case, b, missing):
    """Mistakes planted in the oracle: a Stale token less of some 50 or 100, a page less of 500 tokens."""
    c = make(case, seed=case[0] + case[2])
    scale = c.scale / c.k_scale
    rows = [(b, int(c.new[b]) - 1, h) for h in range(c.hkv * c.group)]
    stale = np.flatnonzero(np.repeat(c.tags[b] == STALE, c.page))
    want, _, tol, _ = bounds(c, scale, rows)
    for first in (0, len(stale) // 32 * 16, len(stale) - 16):
        wrong = bounds(c, scale, rows, drop=stale[first:first + missing])[0]
        assert (np.abs(wrong - want) > tol).any(-1).all()
