"""Attention over 8-bit pages where its bounds are tight (B200 only)."""
import numpy as np
import pytest

from test_gpu_cache8 import Cache, _dev, _t, _tables, _tolerance, attention, nearest

pytestmark = pytest.mark.gpu


def _fill(cache, k, v, k_unit, v_unit):
    """Numbers k, v [pages][heads][page][hd] (codes' values) with one scale everywhere."""
    import torch
    for w, (x, unit) in enumerate(((k, k_unit), (v, v_unit))):
        cache.b[w], cache.s[w] = nearest(x, cache.fmt), np.full(cache.s[w].shape, unit, np.float32)
        cache.t[w].view(torch.int8).copy_(torch.from_numpy(cache.b[w]))
        cache.ts[w].copy_(torch.from_numpy(cache.s[w]))


# query rows of a KV head: every tile of query rows that bfloat16 has
ROWS = [(1, 1), (4, 1), (8, 1), (4, 4), (3, 8), (8, 4), (5, 7)]


def _rounded(out, size, peak, total):
    """The bound of float32 queries, and then the result's rounding to bfloat16 (half a step: 2^-8)."""
    return _tolerance(out, size, peak, total, "f32") + 2.0 ** -8 * np.abs(out)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("G,n", ROWS)
def test_results_that_nearly_cancel(G, n, fmt):
    """Two kinds of tokens with opposite values and almost the same weight: what is left of them hangs on the weights' bits behind the 11th."""
    import torch
    from paper_2410_12513_b200 import first_attn8
    H, hd, page, T = 8, 64, 16, 32 + n - 1
    rng = np.random.default_rng(G * n)
    pages = np.arange(4, dtype=np.int32)[None]
    cache = Cache(0, 4, H, page, hd, fmt)
    k, v = (np.zeros((4, H, page, hd)) for _ in "kv")
    k[:] = 4.0
    k[:, :, 1::2, 0] = 5.0
    v[:, :, ::2] = np.rint(rng.standard_normal((1, H, 1, hd)) * 4) * 8
    v[:, :, 1::2] = -v[:, :, ::2]
    _fill(cache, k, v, 1 / 32, 1 / 64)
    q = torch.randn(n, H * G, hd, generator=torch.Generator().manual_seed(1)).to(_t("bf16"))
    out = torch.empty_like(q, device="cuda")
    first_attn8(q.cuda(), cache.c, _dev(pages), _dev(np.array([T - n], np.int32)), out, cu_new=_dev(np.array([0, n], np.int32)), max_new=n)
    want, size, peak = attention(cache, q.double().numpy(), pages[0], T, n, hd ** -0.5)
    err = np.abs(out.double().cpu().numpy() - want)
    tol = _rounded(want, size, peak, T)
    assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("c", [4, 64, 256, 1024, 16384])
@pytest.mark.parametrize("G,n", ROWS)
def test_queries_with_large_channels(G, n, c, fmt):
    """One channel of the queries is c times the others, and the keys have nothing there: the others decide."""
    import torch
    from paper_2410_12513_b200 import first_attn8
    H, hd, page, T = 2, 128, 64, 300
    rng = np.random.default_rng(c + n)
    pages = _tables(rng, [5], 6)
    cache = Cache(1, 6, H, page, hd, fmt)
    k, v = (rng.standard_normal(cache.b[0].shape) * 36 for _ in "kv")
    k[..., 5] = 0.0
    _fill(cache, k, v, 1 / 36, 1 / 36)
    q = torch.randn(n, H * G, hd, generator=torch.Generator().manual_seed(2))
    q[:, :, 5] = float(c)
    q = q.to(_t("bf16"))
    out = torch.empty_like(q, device="cuda")
    first_attn8(q.cuda(), cache.c, _dev(pages), _dev(np.array([T - n], np.int32)), out, scale=0.25, cu_new=_dev(np.array([0, n], np.int32)), max_new=n)
    want, size, peak = attention(cache, q.double().numpy(), pages[0], T, n, 0.25)
    err = np.abs(out.double().cpu().numpy() - want)
    tol = _rounded(want, size, peak, T)
    # (a query element is held to 2^-31 of its row's largest: a key's largest number is 127 / 36, 128 of them, in units of log2, at both ends)
    tol = tol + (2 * 128 * 127 / 36 * 0.25 * c * 2.0 ** -31 * peak)[..., None]
    assert (err <= tol).all(), (err / tol).max()
