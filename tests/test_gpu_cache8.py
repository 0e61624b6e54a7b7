"""Paged 8-bit caches and the verification of drafts against their definitions in 64 bits (B200 only)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

FULL, BAD_TABLE, BAD_PAGE = 1, 32, 64


def _t(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}[name]


E4M3 = None


def _codes():
    """Values of the 127 codes from 0 to 448."""
    global E4M3
    if E4M3 is None:
        c = np.arange(127)
        e, m = c >> 3, c & 7
        E4M3 = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    return E4M3


def nearest(y, fmt):
    """Codes (int8 as stored) of 64-bit quotients: nearest, ties to even, saturated, NaN gives 0."""
    y = np.where(np.isnan(y), 0.0, y)
    if fmt == "int8":
        return np.rint(np.clip(y, -127, 127)).astype(np.int8)
    v, a = _codes(), np.minimum(np.abs(y), 448.0)
    hi = np.minimum(np.searchsorted(v, a), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = v[hi] - a, a - v[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.where(np.signbit(y) & (code > 0), code - 128, code).astype(np.int8)


def values(codes, fmt):
    if fmt == "int8":
        return codes.astype(np.float64)
    c = codes.astype(np.int64) & 255
    v = np.append(_codes(), np.nan)[c & 127]
    return np.where(c >= 128, -v, v)


class Cache:
    """A cache on the GPU and its mirror (bytes and scales) on the host; pages start out full of garbage."""

    def __init__(self, seed, n_pages, hkv, page, hd, fmt):
        import torch
        from paper_2410_12513_b200 import Cache8
        rng = np.random.default_rng(seed)
        self.fmt, self.page, self.n = fmt, page, n_pages
        self.b = [rng.integers(-128, 128, (n_pages, hkv, page, hd)).astype(np.int8) for _ in "kv"]  # (NaN codes among them)
        self.s = [rng.uniform(0.5, 2.0, (n_pages, hkv)).astype(np.float32) for _ in "kv"]
        self.s[0][0], self.s[1][-1] = np.nan, np.inf
        self.t = [torch.from_numpy(x).cuda().view(_t(fmt)) for x in self.b]
        self.ts = [torch.from_numpy(x).cuda() for x in self.s]
        self.c = Cache8(*self.t, *self.ts)

    def fill(self, seed, spread=1.0):
        """Sensible values and scales everywhere; scales of pages differ by up to 10^(2 spread)."""
        import torch
        rng = np.random.default_rng(seed)
        for i in range(2):
            y = rng.standard_normal(self.b[i].shape)
            self.b[i] = nearest(y * (36 if self.fmt == "int8" else 100), self.fmt)
            self.s[i] = (10.0 ** rng.uniform(-spread, spread, self.s[i].shape) / (36 if self.fmt == "int8" else 100)).astype(np.float32)
            self.t[i].view(torch.int8).copy_(torch.from_numpy(self.b[i]))
            self.ts[i].copy_(torch.from_numpy(self.s[i]))

    def append(self, which, x, pages, before):
        """The definition: x [new][heads][hd] (64 bits) of one sequence."""
        b, s = self.b[which], self.s[which]
        top = np.float32(1) / np.float32(127 if self.fmt == "int8" else 448)
        for first in range(before // self.page * self.page, before + len(x), self.page):
            p = pages[first // self.page]
            lo, hi = max(before - first, 0), min(before + len(x) - first, self.page)
            new = x[first + lo - before:first + hi - before].transpose(1, 0, 2)
            amax = np.where(np.isfinite(new), np.abs(new), 0).max((1, 2)).astype(np.float32)
            held = s[p] if lo else np.zeros_like(s[p])
            now = np.maximum(held, amax * top)
            unit = np.where(now > 0, now, 1).astype(np.float64)[:, None, None]
            with np.errstate(invalid="ignore"):
                y = new / unit
            y = np.where((now > 0)[:, None, None], y, 0)
            grown = now > held
            old = nearest(values(b[p][:, :lo], self.fmt) * held.astype(np.float64)[:, None, None] / unit, self.fmt)
            b[p][:, :lo] = np.where(grown[:, None, None], old, b[p][:, :lo])
            b[p][:, lo:hi] = nearest(y, self.fmt)
            s[p] = now

    def check(self):
        import torch
        for i, name in enumerate("kv"):
            assert np.array_equal(self.ts[i].cpu().numpy(), self.s[i], equal_nan=True), f"{name} scales"
            got = self.t[i].view(torch.int8).cpu().numpy()
            if self.fmt == "e4m3":  # (a zero's sign is free)
                got, want = np.where(got == -128, 0, got), np.where(self.b[i] == -128, 0, self.b[i])
            else:
                want = self.b[i]
            assert np.array_equal(got, want), f"{name}: {(got != want).sum()} of {got.size} values differ"

    def rows(self, which, pages, n):
        """Values of a sequence's first n positions, 64 bits."""
        pos = np.arange(n)
        p = np.asarray(pages)[pos // self.page]
        return values(self.b[which][p, :, pos % self.page], self.fmt) * self.s[which][p].astype(np.float64)[..., None]


def _tables(rng, need, n_pages, extra=0):
    """Pages in random order for sequences that need `need` pages each -> [B][width] with -1 behind."""
    ids, at = rng.permutation(n_pages), 0
    out = np.full((len(need), max(max(need), 1) + extra), -1, np.int32)
    for b, n in enumerate(need):
        out[b, :n] = ids[at:at + n]
        at += n
    assert at <= n_pages
    return out


def _dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _view(x, layout):
    """[tokens][heads][hd] as a view of other storage."""
    import torch
    T, H, hd = x.shape
    if layout == "own":
        return x.contiguous()
    if layout == "fused":
        big = torch.empty(T, H + 3, hd, dtype=x.dtype, device="cuda")
        big[:, 2:2 + H] = x
        return big[:, 2:2 + H]
    if layout == "heads_first":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    big = torch.empty(T, H * hd + 3, dtype=x.dtype, device="cuda")  # "odd": rows between alignments
    big[:, 1:1 + H * hd] = x.reshape(T, H * hd)
    return big[:, 1:1 + H * hd].unflatten(1, (H, hd))


# ------------------------------------------------------------------ append and read back
APPENDS = [  # tokens before, new ones, heads, hd, page, layout
    ([0], [1], 1, 32, 16, "own"), ([15], [1], 2, 64, 16, "fused"), ([16], [1], 8, 128, 16, "own"), ([63, 64, 65, 1], [1, 1, 1, 1], 8, 128, 64, "fused"),
    ([5, 0, 127, 300], [3, 0, 8, 1], 2, 64, 128, "odd"), ([0, 0, 0], [130, 1, 64], 4, 128, 64, "own"), ([7, 33], [129, 200], 1, 32, 32, "heads_first"),
    ([100, 0, 31], [28, 500, 2], 3, 64, 32, "odd"), ([1], [4000], 2, 128, 128, "own")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append_and_read(case, fmt, dtype):
    import torch
    from paper_2410_12513_b200 import first_append8, first_read8
    before, n, H, hd, page, layout = APPENDS[case]
    rng = np.random.default_rng(case)
    need = [-(-(a + b) // page) for a, b in zip(before, n)]
    pages = _tables(rng, need, sum(need) + 2, extra=1)
    cache = Cache(case, sum(need) + 2, H, page, hd, fmt)
    held = [nearest(rng.standard_normal(x.shape) * 30, fmt) for x in cache.b]  # what the sequences held before are values
    for i in range(2):
        for b, p in enumerate(pages):
            for j in range(-(-before[b] // page)):
                cache.b[i][p[j]] = held[i][p[j]]
                cache.s[i][p[j]] = rng.uniform(0.01, 0.03, H).astype(np.float32)
        cache.t[i].view(torch.int8).copy_(torch.from_numpy(cache.b[i]))
        cache.ts[i].copy_(torch.from_numpy(cache.s[i]))
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    total = int(cu[-1]) + 2  # rows behind the last sequence: not stored
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = [torch.randn(total, H, hd, generator=torch.Generator().manual_seed(case + i)).to(_t(dtype)) for i in range(2)]
    if total > 8:  # values that are not finite, a page of zeros, wide spreads
        x[0][1, 0, 3], x[0][2, 0, 5], x[0][3, 0, 0] = math.nan, math.inf, -math.inf
        x[1][: total // 2] *= 1e-3
        x[1][total // 2:, 0] = 0.0
    for i in range(2):
        for b in range(len(n)):
            cache.append(i, x[i][cu[b]:cu[b + 1]].double().numpy(), pages[b], before[b])
    args = (_dev(pages), _dev(np.array(before, np.int32)))
    for again in range(2):  # storing the same tokens again changes nothing
        first_append8(_view(x[0].cuda(), layout), _view(x[1].cuda(), layout), cache.c, *args, cu_new=_dev(cu), max_new=max(n), flags=flags)
        cache.check()
    assert int(flags) == 0
    rows = [a + b for a, b in zip(before, n)]
    cr = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    out = [_view(torch.full((int(cr[-1]) + 1, H, hd), 7.0, dtype=_t(dtype), device="cuda"), layout) for _ in "kv"]
    first_read8(cache.c, args[0], torch.zeros_like(args[1]), *out, cu=_dev(cr), max_rows=max(rows), flags=flags)
    assert int(flags) == 0
    for i in range(2):
        want = np.concatenate([cache.rows(i, pages[b], rows[b]) for b in range(len(n))] + [np.full((1, H, hd), 7.0)])
        assert torch.equal(out[i].cpu().float(), torch.from_numpy(want).float().to(_t(dtype)).float())  # one product, rounded


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_tokens_one_by_one(fmt):
    """The step's use: a token a call, scales that grow on the way; rows without a table of rows."""
    import torch
    from paper_2410_12513_b200 import first_append8
    rng = np.random.default_rng(5)
    H, hd, page, steps = 2, 64, 16, 40
    before = np.array([0, 9, 31], np.int32)
    pages = _tables(rng, [3, 4, 5], 14)
    cache = Cache(1, 14, H, page, hd, fmt)
    cache.fill(2, 0.2)
    for i in range(steps):
        x = [torch.randn(3, H, hd, generator=torch.Generator().manual_seed(100 * i + w)) * (1.1 ** (i % 17)) for w in range(2)]
        for w in range(2):
            for b in range(3):
                cache.append(w, x[w][b:b + 1].double().numpy(), pages[b], int(before[b]))
        first_append8(x[0].cuda(), x[1].cuda(), cache.c, _dev(pages), _dev(before))
        before += 1
    cache.check()


@pytest.mark.parametrize("fmt,top", [("int8", 127), ("e4m3", 448)])
def test_quotients_on_and_next_to_ties(fmt, top):
    """Scale 1 exactly (the largest magnitude is its own number); values on ties, and one float32 step beside them."""
    import torch
    from paper_2410_12513_b200 import first_append8
    if fmt == "int8":
        ties = np.arange(-127, 127) + 0.5
    else:
        v = _codes()
        ties = np.concatenate([(v[1:] + v[:-1]) / 2, -(v[1:] + v[:-1]) / 2])
    ties = ties.astype(np.float32)
    x = np.concatenate([ties, np.nextafter(ties, np.float32(1e9)), np.nextafter(ties, np.float32(-1e9)), [-0.0, 1e-42, -1e-45]]).astype(np.float32)
    page, hd = 128, 128
    rows = np.zeros((-(-x.size // hd), 1, hd), np.float32)
    rows.reshape(-1)[:x.size] = x
    factor = np.float32(top) / (np.float32(top) * (np.float32(1) / np.float32(top)))
    for scale in (1.0, 3.0e-5, 1e-41, 2.0 ** 100):  # (scales that are not powers of two have hardly any ties, but neighbours)
        cache = Cache(0, 1, 1, page, hd, fmt)
        y = np.concatenate([rows * np.float32(scale), np.full((1, 1, hd), np.float32(top) * factor * np.float32(scale), np.float32)]).astype(np.float32)
        for w in range(2):
            cache.append(w, y.astype(np.float64), [0], 0)
        t = torch.from_numpy(y).cuda()
        first_append8(t, t, cache.c, _dev(np.zeros((1, 1), np.int32)), _dev(np.zeros(1, np.int32)),
                      cu_new=_dev(np.array([0, len(y)], np.int32)), max_new=len(y))
        cache.check()


def test_append_without_pages_and_bad_tables():
    import torch
    from paper_2410_12513_b200 import first_append8, first_read8
    H, hd, page = 1, 32, 16
    cache = Cache(3, 6, H, page, hd, "int8")
    pages = np.array([[0, -1], [1, 99], [2, -7], [3, 4], [5, -1]], np.int32)
    before = np.array([15, 15, 20, -1, 0], np.int32)
    x = torch.ones(10, H, hd)
    cu = np.array([0, 2, 4, 6, 8, 10], np.int32)
    for b in (0, 1):  # the first of the two finds its page
        for w in range(2):
            cache.append(w, x[:1].double().numpy(), pages[b], 15)
    for w in range(2):
        cache.append(w, x[:2].double().numpy(), pages[4], 0)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    first_append8(x.cuda(), x.cuda(), cache.c, _dev(pages), _dev(before), cu_new=_dev(cu), max_new=2, flags=flags)
    assert int(flags) == FULL | BAD_TABLE | BAD_PAGE
    cache.check()
    flags.zero_()
    first_append8(x.cuda(), x.cuda(), cache.c, _dev(pages), _dev(before), cu_new=_dev(cu), max_new=1, flags=flags)  # more than said
    assert int(flags) == BAD_TABLE
    for bad in ([0, 2, 1, 6, 8, 10], [-1, 0, 0, 0, 0, 0], [0, 0, 0, 0, 9, 11]):
        flags.zero_()
        first_append8(x.cuda(), x.cuda(), cache.c, _dev(pages[[4] * 5]), _dev(np.full(5, 40, np.int32)), cu_new=_dev(np.array(bad, np.int32)), max_new=9, flags=flags)
        assert int(flags) & BAD_TABLE
    cache.check()
    flags.zero_()
    out = torch.full((2, H, hd), 3.0, device="cuda")
    first_read8(cache.c, _dev(np.array([[0, -1]], np.int32)), _dev(np.array([15], np.int32)), out, out.clone(), cu=_dev(np.array([0, 2], np.int32)), max_rows=2, flags=flags)
    assert int(flags) == BAD_PAGE and (out[1] == 3.0).all() and np.allclose(out[0].cpu().numpy(), cache.rows(0, [0], 16)[15], equal_nan=True)  # (page 0 has a NaN scale)


# ------------------------------------------------------------------ attention
def attention(cache, q, pages, total, n, scale):
    """64 bits: q [n][Hq][hd], the last of `total` positions; pages < 0 are not there.  -> out, and for the tolerance the
    largest sum of |q k| and the largest |v| of every (row, head)."""
    hkv = cache.b[0].shape[1]
    G = q.shape[1] // hkv
    pos = np.arange(total)
    at = pos // cache.page
    have = (at < len(pages)) & (np.asarray(pages)[np.minimum(at, len(pages) - 1)] >= 0) if len(pages) else np.zeros(total, bool)
    pos = pos[have]
    p = np.asarray(pages)[pos // cache.page] if len(pos) else np.zeros(0, int)
    k, v = (values(cache.b[w][p, :, pos % cache.page], cache.fmt) * cache.s[w][p].astype(np.float64)[..., None] for w in range(2))
    out, size, peak = np.zeros(q.shape), np.zeros(q.shape[:2]), np.zeros(q.shape[:2])
    for i in range(n):
        see = pos <= total - n + i
        for h in range(q.shape[1]):
            kk, vv = k[see, h // G], v[see, h // G]
            if not len(kk):
                continue
            z = kk @ q[i, h] * scale
            w = np.exp(z - z.max())
            out[i, h] = w @ vv / w.sum()
            size[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * abs(scale)
            peak[i, h] = np.abs(vv).max()
    return out, size, peak


def _tolerance(out, size, peak, total, dtype):
    # float32 on the way.  A logit: its products are summed in steps of the tensor cores, hd / 16 (x 2 halves) of them, each
    # cutting at 2^-22 of the largest partial sum: 16 * 2^-22 of sum |q k|; the halves of q hold 22 bits and scales are two
    # more products: 2^-20 of sum |q k| in all covers them.  In units of log2 (x 1.45) that is a relative error of every weight (x ln 2), at
    # both ends of the quotient: 2 * (16 * 2^-22 + 2^-20) = 10 * 2^-20.  exp2: 2 * 2^-22.  Sums over total / 64 steps of a warp of
    # four, 2^-22 each, twice; 64 more for the joins.  Weights: 22 bits (hi + lo), or one half with bfloat16: half a step of a half is 2^-11
    # (eps 2^-10), and it is off in the numerator alone.  The result's rounding: half a step of bfloat16 is 2^-8 (eps 2^-7), of float32 2^-24.
    rel = 10 * 2.0 ** -20 * size + 2.0 ** -21 + 2 * (total / 64 + 64) * 2.0 ** -22
    if dtype == "bf16":
        rel = rel + 2.0 ** -11
    return (rel * peak)[..., None] + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(out) + 1e-30


ATTN = [  # lengths with the new ones, new ones, KV heads, group, hd, page, layout
    ([1], [1], 1, 1, 32, 16, "own"), ([15, 16, 17, 31, 32, 33], [1] * 6, 2, 4, 64, 16, "own"), ([700], [1], 8, 4, 128, 64, "own"),
    ([100, 1, 64, 65], [1] * 4, 8, 3, 128, 32, "fused"), ([5, 200, 0, 130], [5, 3, 0, 1], 2, 2, 128, 128, "odd"),
    ([40, 600], [8, 6], 1, 8, 128, 16, "heads_first"), ([300, 77], [33, 40], 2, 1, 64, 64, "own"), ([150], [100], 1, 4, 32, 32, "own"),
    ([2500, 3, 900], [2, 2, 2], 4, 8, 64, 64, "fused"), ([129, 128, 127], [1, 2, 4], 2, 5, 128, 128, "own"), ([4096, 5000], [4, 1], 1, 4, 128, 64, "odd"),
    ([64] * 40, [1] * 40, 8, 4, 128, 64, "own"), ([20], [20], 3, 7, 64, 16, "own"), ([1 + i % 40 for i in range(300)], [1] * 300, 1, 2, 32, 16, "own")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention(case, fmt, dtype):
    import torch
    from paper_2410_12513_b200 import first_attn8
    total, n, H, G, hd, page, layout = ATTN[case]
    rng = np.random.default_rng(100 + case)
    need = [-(-t // page) for t in total]
    cache = Cache(case, sum(need) + 2, H, page, hd, fmt)
    pages = _tables(rng, need, cache.n, extra=1)
    garbage = [x.copy() for x in cache.b]
    cache.fill(case, 0.5)
    for w in range(2):  # behind every sequence's last token: any bytes, NaN codes among them; pages of nobody: any scale
        for b, t in enumerate(total):
            if t % page:
                cache.b[w][pages[b, t // page], :, t % page:] = garbage[w][pages[b, t // page], :, t % page:]
        free = sorted(set(range(cache.n)) - set(pages.ravel().tolist()))
        cache.s[w][free] = np.nan
        cache.t[w].view(torch.int8).copy_(torch.from_numpy(cache.b[w]))
        cache.ts[w].copy_(torch.from_numpy(cache.s[w]))
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    q = torch.randn(int(cu[-1]) + 2, H * G, hd, generator=torch.Generator().manual_seed(case)) * 2
    q[0, 0] *= 1e-3
    q[-3] *= 30
    q = q.to(_t(dtype))
    scale = 0.7 / math.sqrt(hd)
    out = _view(torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda"), layout)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = np.array(total) - np.array(n)
    args = (_view(q.cuda(), layout), cache.c, _dev(pages), _dev(before.astype(np.int32)), out)
    first_attn8(*args, scale=scale, cu_new=_dev(cu), max_new=max(n), flags=flags)
    assert int(flags) == 0
    got = out.double().cpu().numpy()
    for b in range(len(n)):
        r = slice(cu[b], cu[b + 1])
        want, size, peak = attention(cache, q[r].double().numpy(), pages[b], total[b], n[b], scale)
        err, tol = np.abs(got[r] - want), _tolerance(want, size, peak, total[b], dtype)
        assert (err <= tol).all(), (b, (err / tol).max())
    assert (got[cu[-1]:] == 5.0).all()  # rows behind the last sequence
    first = out.clone()
    first_attn8(*args, scale=scale, cu_new=_dev(cu), max_new=max(n))
    assert torch.equal(first, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_over_missing_pages(dtype):
    """Pages that are -1 or outside the cache are not there, whatever the length says; a row that sees nothing gives zeros."""
    import torch
    from paper_2410_12513_b200 import first_attn8
    H, G, hd, page = 2, 2, 64, 16
    cache = Cache(0, 12, H, page, hd, "e4m3")
    cache.fill(0)
    pages = np.array([[0, -1, 1, 2], [-1, -1, -1, -1], [3, 4, 5, 99], [6, -1, -1, -1], [-1, 7, 8, 9]], np.int32)
    total = np.array([60, 50, 64, 1, 1000], np.int32)  # (the last one is longer than its table)
    q = torch.randn(5, H * G, hd, generator=torch.Generator().manual_seed(1)).to(_t(dtype))
    out = torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    first_attn8(q.cuda(), cache.c, _dev(pages), _dev(total - 1), out, flags=flags)
    assert int(flags) == BAD_PAGE
    pages[2, 3] = -1
    for b in range(5):
        want, size, peak = attention(cache, q[b:b + 1].double().numpy(), pages[b], int(total[b]), 1, 0.125)
        assert (np.abs(out[b:b + 1].double().cpu().numpy() - want) <= _tolerance(want, size, peak, 64, dtype)).all(), b
    assert (out[1] == 0).all()
    none = torch.empty(5, 0, dtype=torch.int32, device="cuda")  # no pages at all
    first_attn8(q.cuda(), cache.c, none, _dev(total - 1), out)
    assert (out == 0).all()
    out.fill_(5.0)
    flags.zero_()
    first_attn8(q.cuda(), cache.c, _dev(pages), _dev(np.array([-1, 2, 2, 2, 2 ** 31 - 1], np.int32)), out, flags=flags)
    assert int(flags) & BAD_TABLE and (out[0] == 5.0).all() and (out[4] == 5.0).all() and (out[2] != 5.0).any()


@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("fmt,dtype", [("int8", "f32"), ("e4m3", "bf16")])
def test_attention_over_a_workspace(fmt, dtype, n):
    """Few long sequences: cut among more of the GPU where there is room for unfinished results, whatever it holds; without enough
    room the call does without."""
    import torch
    from paper_2410_12513_b200 import first_attn8
    from paper_2410_12513_b200.binding import _workspace8
    H, G, hd, page, total = 1, 4, 128, 64, [20000, 9000, 70]
    rng = np.random.default_rng(n)
    need = [-(-t // page) for t in total]
    cache = Cache(n, sum(need), H, page, hd, fmt)
    cache.fill(n, 0.5)
    pages = _tables(rng, need, cache.n)
    q = (torch.randn(3 * n, H * G, hd, generator=torch.Generator().manual_seed(n)) * 2).to(_t(dtype))
    cu = _dev(np.arange(4, dtype=np.int32) * n)
    before = _dev(np.array(total, np.int32) - n)
    room = _workspace8(cache.c.sizes, H * G, 0 if dtype == "f32" else 1, 3 * n, pages.shape[1], 3, n)
    assert room > 0
    outs = []
    for ws in (None, torch.full((room // 4,), math.nan, device="cuda"), torch.empty(2, device="cuda")):
        out = torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda")
        first_attn8(q.cuda(), cache.c, _dev(pages), before, out, cu_new=cu, max_new=n, workspace=ws)
        outs.append(out)
        for b in range(3):
            want, size, peak = attention(cache, q[b * n:b * n + n].double().numpy(), pages[b], total[b], n, hd ** -0.5)
            err = np.abs(out[b * n:b * n + n].double().cpu().numpy() - want)
            assert (err <= _tolerance(want, size, peak, total[b], dtype)).all(), b
    assert torch.equal(outs[0], outs[1])


def test_attention_extremes():
    """Infinite and NaN queries give NaN in their own rows alone; the largest and smallest finite ones hold."""
    import torch
    from paper_2410_12513_b200 import first_attn8
    H, hd, page, T = 1, 128, 64, 300
    cache = Cache(0, 5, H, page, hd, "int8")
    cache.fill(3, 0.1)
    pages = np.arange(5, dtype=np.int32)[None]
    q = torch.randn(1, 8, hd, generator=torch.Generator().manual_seed(1))
    q[0, 1, 5], q[0, 2, 7] = math.nan, math.inf
    q[0, 3] *= 1e36  # logits far apart: the largest alone weighs
    q[0, 4] *= 1e-38
    q[0, 5] = 0.0
    out = torch.empty_like(q, device="cuda")
    first_attn8(q.cuda(), cache.c, _dev(pages), _dev(np.array([T - 1], np.int32)), out, scale=0.25)
    got = out.cpu().double().numpy()
    assert np.isnan(got[0, 1]).all() and np.isnan(got[0, 2]).all()
    ok = [0, 3, 4, 5, 6, 7]
    want, size, peak = attention(cache, q[:, ok].double().numpy(), pages[0], T, 1, 0.25)
    size[0, 1] = 0.0  # (one weight of 1, the others 0)
    assert (np.abs(got[:, ok] - want) <= _tolerance(want, size, peak, T, "f32")).all()
    # the definition's lowest logits: a scale of 0 weighs all alike, a negative one turns the order round
    for scale in (0.0, -0.25):
        first_attn8(q[:, ok].contiguous().cuda(), cache.c, _dev(pages), _dev(np.array([T - 1], np.int32)), out[:, :6], scale=scale)
        want, size, peak = attention(cache, q[:, ok].double().numpy(), pages[0], T, 1, scale)
        size[0, 1] = 0.0
        assert (np.abs(out[:, :6].cpu().double().numpy() - want) <= _tolerance(want, size, peak, T, "f32")).all()


def test_a_long_cache_beyond_32_bits():
    """Pages whose bytes lie beyond 2^32 of the cache's start."""
    import torch
    from paper_2410_12513_b200 import Cache8, first_append8, first_attn8, first_copy_pages, first_read8
    H, hd, page = 8, 128, 128
    n = (2 ** 32) // (H * hd * page) + 8
    k, v = (torch.zeros(n, H, page, hd, dtype=torch.int8, device="cuda") for _ in "kv")
    ks, vs = (torch.zeros(n, H, device="cuda") for _ in "kv")
    c = Cache8(k, v, ks, vs)
    pages = torch.tensor([[n - 1, n - 3]], dtype=torch.int32, device="cuda")
    x = torch.randn(200, H, hd, device="cuda")
    cu = torch.tensor([0, 200], dtype=torch.int32, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    first_append8(x, x, c, pages, zero, cu_new=cu, max_new=200)
    back, _ = torch.empty_like(x), torch.empty_like(x)
    first_read8(c, pages, zero, back, _, cu=cu, max_rows=200)
    assert (back - x).abs().max() <= x.abs().max() / 127 * 0.501
    assert (k[:4] == 0).all() and (ks[:n - 3] == 0).all()
    first_copy_pages([c], torch.tensor([[0, n - 1, 1], [0, n - 3, n - 5]], dtype=torch.int32, device="cuda"))
    out, out2 = torch.empty(1, H, hd, device="cuda"), torch.empty(1, H, hd, device="cuda")
    first_attn8(x[:1].contiguous(), c, pages, zero + 199, out)
    first_attn8(x[:1].contiguous(), c, torch.tensor([[1, n - 5]], dtype=torch.int32, device="cuda"), zero + 199, out2)
    assert torch.equal(out, out2) and out.abs().max() > 0


def test_streams_and_graphs():
    import torch
    from paper_2410_12513_b200 import first_append8, first_attn8
    H, G, hd, page = 2, 4, 64, 32
    cache = Cache(0, 40, H, page, hd, "int8")
    cache.fill(1)
    rng = np.random.default_rng(0)
    pages, ln = _dev(_tables(rng, [4] * 8, 40)), _dev(np.arange(8, dtype=np.int32) * 13)
    x, q = torch.randn(8, H, hd, device="cuda"), torch.randn(8, H * G, hd, device="cuda")
    out = torch.empty_like(q)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    first_append8(x, x, cache.c, pages, ln, stream=st)
    first_attn8(q, cache.c, pages, ln, out, stream=st)
    st.synchronize()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first_append8(x, x, cache.c, pages, ln)
        first_attn8(q, cache.c, pages, ln, out)
    out.zero_()
    graph.replay()
    assert torch.equal(out, want)
    q2 = q * 0.5  # the replay reads the tensors of its own time
    q.mul_(0.5)
    ln.add_(1)
    graph.replay()
    got = out.clone()
    first_attn8(q2, cache.c, pages, ln, out)
    assert torch.equal(got, out) and not torch.equal(got, want)


# ------------------------------------------------------------------ pages from place to place
@pytest.mark.parametrize("layers,n,H,page,hd,moves", [(1, 5, 1, 16, 32, 2), (3, 17, 5, 16, 32, 20), (2, 9, 8, 128, 128, 8), (32, 12, 3, 64, 64, 100)])
def test_copies(layers, n, H, page, hd, moves):
    import torch
    from paper_2410_12513_b200 import first_copy_pages
    rng = np.random.default_rng(moves)
    caches = [Cache(l, n, H, page, hd, "e4m3") for l in range(layers)]
    todo = []
    for l in range(layers):
        order = rng.permutation(n)
        for i in range(min(moves // layers, n // 2)):
            todo.append((l, int(order[2 * i]), int(order[2 * i + 1])))
    bad = [(layers, 0, 1), (-1, 0, 1), (0, n, 1), (0, -1, 1), (0, 1, n), (0, 0, -1), (0, n - 1, n - 1)]
    table = np.array(todo + bad, np.int32)[rng.permutation(len(todo) + len(bad))]
    for l, a, b in todo:
        for w in range(2):
            caches[l].b[w][b], caches[l].s[w][b] = caches[l].b[w][a], caches[l].s[w][a]
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    first_copy_pages([c.c for c in caches], _dev(table), flags=flags)
    assert int(flags) == BAD_PAGE
    for c in caches:
        for w in range(2):
            assert np.array_equal(c.t[w].view(torch.int8).cpu().numpy(), c.b[w])
            assert np.array_equal(c.ts[w].cpu().numpy(), c.s[w], equal_nan=True)
    first_copy_pages([c.c for c in caches], torch.empty(0, 3, dtype=torch.int32, device="cuda"))


# ------------------------------------------------------------------ verification
def probabilities(x, temp, probs):
    x = x.astype(np.float64)
    if probs:
        return np.where(np.isnan(x), 0, np.maximum(x, 0))
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, float(np.finfo(np.float32).max)))
    if x.max() == -np.inf:
        return np.zeros_like(x)
    if not temp > 0:
        return (np.arange(x.size) == x.argmax()).astype(np.float64)
    w = np.exp((x - x.max()) / min(max(float(temp), float(np.float32(1e-37))), float(np.float32(1e30))))
    return w / w.sum()


def _u(u):
    return min(max(float(u), 0.0), 1.0 - 2.0 ** -24) if u == u else 1.0 - 2.0 ** -24


def verified(target, draft, drafted, temp, u, w, probs):
    """-> tokens, accepted, whether every decision is clear of its border (2^-18 of the quantities compared; 2^-40 of the sum)."""
    n, clear = len(drafted), True
    V = target.shape[1]
    for i in range(n + 1):
        p = probabilities(target[i], temp, probs)
        if i < n and 0 <= drafted[i] < V:
            q = probabilities(draft[i], temp, probs) if draft is not None else (np.arange(V) == drafted[i]).astype(np.float64)
            a, b = _u(u[i]) * q[drafted[i]], p[drafted[i]]
            clear &= probs or abs(a - b) > 2.0 ** -18 * max(a, b) or (a == 0 and b == 0) or not temp > 0
            if a < b:
                continue
            rest = np.maximum(p - q, 0)
            p = rest if rest.sum() > 0 else p
        cum = np.cumsum(p)
        out = list(drafted[:i]) + [-1] * (n + 1 - i)
        if cum[-1] > 0:
            at = np.searchsorted(cum, _u(w) * cum[-1], side="right")
            out[i] = min(int(at), int(np.flatnonzero(p)[-1]))
            gap = np.abs(cum - _u(w) * cum[-1])
            clear &= float(gap[p > 0].min()) > 2.0 ** -40 * cum[-1] or not (temp is None or temp > 0 or probs)
        return out, i, clear


def _verify(target, draft, drafted, u, w, temp=None, probs=False, **kw):
    import torch
    from paper_2410_12513_b200 import first_verify
    B, rows, _ = target.shape
    tokens = torch.full((B, rows), -9, dtype=torch.int32, device="cuda")
    accepted = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    first_verify(target, drafted, u, w, tokens, accepted, draft=draft, temperature=temp, probs=probs, **kw)
    return tokens, accepted


CASES = [  # sequences, drafts, vocab, spread
    (1, 4, 128256, 2.5), (1, 0, 1000, 2.0), (3, 1, 1, 1.0), (5, 3, 2, 1.0), (4, 7, 31, 2.0), (2, 32, 500, 2.0), (9, 8, 4097, 3.0),
    (30, 5, 50257, 2.5), (70, 4, 5000, 2.0), (400, 3, 300, 1.5), (2, 2, 524288, 2.0), (12, 9, 8191, 2.0)]


@pytest.mark.parametrize("kind", ["logits", "probs", "lookup", "greedy"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_verify(case, kind):
    import torch
    B, n, V, spread = CASES[case]
    g = torch.Generator().manual_seed(case)
    pad = case % 4  # rows between alignments
    target = torch.full((B, n + 1, V + pad), 1e30)[:, :, pad // 2:pad // 2 + V]
    target.copy_(torch.randn(B, n + 1, V, generator=g) * spread)
    target[:, :, ::5] = -math.inf if V > 5 else 0.0
    draft = None if kind == "lookup" else target[:, :n].clone() + 0.4 * torch.randn(B, n, V, generator=g)
    temp = 0.5 + torch.rand(B, generator=g)
    probs = kind == "probs"
    if kind == "greedy":
        temp[::2] = 0.0
        temp[1::2] = math.nan
    if probs:
        target = torch.softmax(target, -1)
        draft = torch.softmax(draft, -1)
    if draft is None:
        drafted = target[:, :n].argmax(-1)
    else:
        e = -torch.log(torch.rand(B, n, V, generator=g).clamp(min=1e-30))
        drafted = (draft / e if probs else draft / temp[:, None, None].nan_to_num().clamp(min=0.1) - torch.log(e)).argmax(-1)
    if n > 1:
        drafted[::3, n - 1] = -1  # fewer drafts
        drafted[1::7, 0] = V
    u, w = torch.rand(B, n, generator=g), torch.rand(B, generator=g)
    u[::4] *= 0.1  # (some sequences get far)
    w[0] = 0.0
    dev = [None if x is None else x.cuda() for x in (target, draft, drafted.int(), u, w, temp)]
    tokens, accepted = _verify(dev[0], dev[1], dev[2], dev[3], dev[4], None if probs else dev[5], probs)
    tokens, accepted, seen = tokens.cpu().numpy(), accepted.cpu().numpy(), 0
    for b in range(B):
        out, a, clear = verified(target[b].numpy(), None if draft is None else draft[b].numpy(), drafted[b].tolist(), float(temp[b]) if not probs else None,
                                 u[b].tolist(), float(w[b]), probs)
        if clear or w[b] == 0:
            assert accepted[b] == a and tokens[b].tolist() == out, (b, accepted[b], a, tokens[b].tolist(), out)
            seen += 1
    assert seen >= 0.9 * B


def test_verify_odd_rows():
    """Rows without a candidate, NaN and infinite logits, draws outside [0, 1), temperatures at the ends, p below q everywhere."""
    import torch
    V, n = 1000, 2
    base = torch.randn(1, n + 1, V, generator=torch.Generator().manual_seed(3)) * 2
    rows, drafts, temps, us, ws = [], [], [], [], []

    def add(t, d, temp=1.0, u=0.5, w=0.5):
        rows.append(t), drafts.append(d), temps.append(temp), us.append([u, u]), ws.append(w)
    dr = base[:, :n] + 0.3 * torch.randn(1, n, V, generator=torch.Generator().manual_seed(4))
    add(torch.full_like(base, -math.inf), dr)                           # no candidate: -1
    add(base, torch.full_like(dr, -math.inf))                           # the draft had none: accepted where p > 0
    x = base.clone()
    x[:, :, ::2] = math.nan
    add(x, dr)
    x = base.clone()
    x[:, :, 77] = math.inf
    x[:, 1, 78] = math.inf
    add(x, dr, u=0.9999)
    for temp in (1e-40, 1e-30, 1e31, math.inf, math.nan, -1.0, 3e38):
        add(base, dr, temp)
    for u in (-1.0, 1.0, math.nan, 7.0, 0.0):
        add(base, dr, 1.0, u, u)
    add(base, base[:, :n], 1.0, 1.0, 0.3)                               # p = q
    t, d = torch.cat(rows), torch.cat(drafts)
    B = t.shape[0]
    drafted = torch.stack([torch.arange(B) * 13 % V, torch.arange(B) * 29 % V], 1).int()
    drafted[3] = torch.tensor([77, 77])
    drafted[0] = 5
    temp, u, w = torch.tensor(temps), torch.tensor(us), torch.tensor(ws)
    tokens, accepted = _verify(t.cuda(), d.cuda(), drafted.cuda(), u.cuda(), w.cuda(), temp.cuda())
    tokens, accepted = tokens.cpu().numpy(), accepted.cpu().numpy()
    assert tokens[0].tolist() == [-1, -1, -1] and accepted[0] == 0
    assert accepted[1] == 2
    for b in range(1, B):
        out, a, clear = verified(t[b].numpy(), d[b].numpy(), drafted[b].tolist(), float(temp[b]), u[b].tolist(), float(w[b]), False)
        if clear or not float(temp[b]) > 0 or float(w[b]) in (0.0, -1.0):
            assert accepted[b] == a and tokens[b].tolist() == out, (b, tokens[b].tolist(), out)
    # probabilities: negative and NaN count as 0, a row need not sum to 1, p <= q everywhere falls back to p
    p = torch.rand(4, n + 1, V, generator=torch.Generator().manual_seed(9))
    q = torch.rand(4, n, V, generator=torch.Generator().manual_seed(10))
    p[0, :, ::3], q[0, :, ::2] = -1.0, math.nan
    q[1] = p[1, :n] * 2
    p[2] = 0.0
    d2 = torch.tensor([[0, 3], [5, 5], [1, 1], [-1, 4]], dtype=torch.int32)
    uu, ww = torch.full((4, n), 0.6), torch.tensor([0.1, 0.9, 0.5, 0.999])
    tokens, accepted = _verify(p.cuda(), q.cuda(), d2.cuda(), uu.cuda(), ww.cuda(), probs=True)
    for b in range(4):
        out, a, _ = verified(p[b].numpy(), q[b].numpy(), d2[b].tolist(), None, uu[b].tolist(), float(ww[b]), True)
        assert tokens[b].tolist() == out and int(accepted[b]) == a, b


def test_verify_keeps_the_targets_distribution():
    """Of many sequences with the same rows, the first token comes out as the target has it (a chi-squared test)."""
    import torch
    V, B = 12, 20000
    g = torch.Generator().manual_seed(1)
    t, d = torch.randn(2, V, generator=g), torch.randn(1, V, generator=g)
    p = torch.softmax(t[0].double(), -1).numpy()
    drafted = torch.multinomial(torch.softmax(d[0], -1), B, replacement=True, generator=g).int()[:, None]
    tokens, accepted = _verify(t.expand(B, 2, V).contiguous().cuda(), d.expand(B, 1, V).contiguous().cuda(), drafted.cuda(),
                               torch.rand(B, 1, generator=g).cuda(), torch.rand(B, generator=g).cuda())
    seen = np.bincount(tokens[:, 0].cpu().numpy(), minlength=V)
    chi = ((seen - B * p) ** 2 / (B * p)).sum()
    assert chi < 45  # 11 degrees of freedom: a chance of 5e-6
    assert 0 < int(accepted.sum()) < B


def test_verify_on_a_stream_and_in_a_graph():
    import torch
    B, n, V = 5, 3, 3000
    target, draft = torch.randn(B, n + 1, V, device="cuda"), torch.randn(B, n, V, device="cuda")
    drafted = torch.randint(0, V, (B, n), device="cuda", dtype=torch.int32)
    u, w = torch.rand(B, n, device="cuda"), torch.rand(B, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    want = _verify(target, draft, drafted, u, w)
    from paper_2410_12513_b200 import first_verify
    tokens, accepted = torch.empty(B, n + 1, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    first_verify(target, drafted, u, w, tokens, accepted, draft=draft, stream=st)
    st.synchronize()
    assert torch.equal(tokens, want[0]) and torch.equal(accepted, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first_verify(target, drafted, u, w, tokens, accepted, draft=draft)
    w.fill_(0.25)
    graph.replay()
    want = _verify(target, draft, drafted, u, w)
    assert torch.equal(tokens, want[0]) and torch.equal(accepted, want[1])
