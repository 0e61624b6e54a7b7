"""Attention over 8-bit pages where its bounds are tight (B200 only)."""
import math

import numpy as np
import pytest

import first_inputs as fi
import oracle
from harness import GpuKV, gpu_weights, logits_check, oracle_model
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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,G,n,hd,page,fmt", [
    (1, 1, 4, 1, 128, 64, "int8"), (1, 1, 1, 1, 32, 128, "e4m3"), (1, 2, 4, 1, 64, 32, "int8"), (2, 1, 4, 1, 64, 64, "e4m3"),
    (3, 1, 2, 1, 32, 64, "int8"), (1, 1, 8, 3, 64, 64, "e4m3"), (1, 1, 5, 4, 128, 16, "int8"), (2, 1, 16, 2, 32, 64, "int8")])
def test_one_and_two_items(B, H, G, n, hd, page, fmt, dtype):
    """As many splits as there can be, over a workspace full of NaN; the second sequence leaves most of them without a token."""
    import torch
    from paper_2410_12513_b200 import first_attn8
    from paper_2410_12513_b200.binding import _workspace8
    total = [40000, 100, 25000][:B]
    rng = np.random.default_rng(B + G)
    need = [-(-t // page) for t in total]
    cache = Cache(n, sum(need), H, page, hd, fmt)
    cache.fill(n, 0.3)
    pages = _tables(rng, need, cache.n)
    q = (torch.randn(B * n, H * G, hd, generator=torch.Generator().manual_seed(n)) * 4).to(_t(dtype))
    room = _workspace8(cache.c.sizes, H * G, 0 if dtype == "f32" else 1, B * n, pages.shape[1], B, n)
    assert room > 0
    outs = []
    for ws in (torch.full((room // 4,), math.nan, device="cuda"), None, torch.empty(1, device="cuda")):
        out = torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda")
        first_attn8(q.cuda(), cache.c, _dev(pages), _dev(np.array(total, np.int32) - n), out, cu_new=_dev(np.arange(B + 1, dtype=np.int32) * n), max_new=n,
                    workspace=ws)
        outs.append(out)
        for b in range(B):
            want, size, peak = attention(cache, q[b * n:b * n + n].double().numpy(), pages[b], total[b], n, hd ** -0.5)
            err = np.abs(out[b * n:b * n + n].double().cpu().numpy() - want)
            tol = _tolerance(want, size, peak, total[b], dtype)
            assert (err <= tol).all(), (b, (err / tol).max())
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("slots,heads", [(1, 1), (1, 2), (2, 1), (2, 2)])
def test_a_step_over_one_long_sequence(slots, heads):
    """A decode step that cuts its one sequence among the whole GPU: each query head finds few of 30000 tokens, wherever they are."""
    import torch
    from paper_2410_12513_b200 import Cache8, FirstContext, FirstPages
    from test_gpu_pages import _read
    shape = fi.ModelShape(2, 128, 4, heads, 64, 256, 512)
    w = fi.make_weights(shape, 7, False)
    ctx = FirstContext(shape, 0, 32, 64, gpu_weights(w))
    om = oracle_model(shape, w)
    n, page, L = 30000, 128, shape.n_layers
    stage = GpuKV(shape, [n], False)
    g = torch.Generator(device="cuda").manual_seed(3)
    for l in range(L):
        stage.k[l].copy_(torch.randn(stage.k[l].shape, generator=g, device="cuda") * 24)
        stage.v[l].copy_(torch.randn(stage.v[l].shape, generator=g, device="cuda") * 4)
    caches = []
    for l in range(L):
        kv = [torch.zeros(240, heads, page, 64, dtype=torch.int8, device="cuda") for _ in "kv"]
        caches.append(Cache8(*kv, *[torch.zeros(240, heads, device="cuda") for _ in "kv"]))
    mgr = FirstPages(ctx, slots, 240, caches)
    ctx.set_pages(mgr)
    s = mgr.join(np.ones(L, np.uint8), stage.c, 0, n)
    mgr.commit()
    logits = torch.empty(slots, shape.vocab, device="cuda")
    for step in range(4):
        mgr.extend()
        mgr.commit()
        okv = oracle.OracleKV(om.shape, [n + step + 1])
        for l in range(L):
            for dst, src in zip(okv.rows(l, 0), _read(mgr, l, s, n + step)):
                dst[:n + step] = src.reshape(n + step, -1)
            okv.len[l, 0] = n + step
        okv.pos[0] = n + step
        toks = np.array([17 * step + 5] * slots, np.int32)
        ref = oracle.decode_step(om, toks[:1], np.ones((1, L), np.uint8), okv)[0]
        ctx.decode_step(torch.from_numpy(toks).cuda(), None, logits)
        assert ctx.device_flags() == 0
        err, _ = logits_check(logits[s:s + 1].cpu().numpy(), ref[None])
        assert err.max() <= 2e-2, (step, err)
    ctx.set_pages(None)
    mgr.close()
