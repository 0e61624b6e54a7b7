"""Adapters of many requests, rotary positions and per-request sampling against their definitions in 64 bits, standalone
and inside the step (B200 only)."""
import math

import numpy as np
import pytest

import first_inputs as fi
import oracle
from harness import GpuKV, gpu_weights, logits_check, oracle_model, synthetic_caches, widen

pytestmark = pytest.mark.gpu

F32, BF16 = 0, 1
U32 = 2.0 ** -24  # half a step of float32


def _t(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


# ------------------------------------------------------------------ rotary positions
def _rope_ref(x, pos, inv, factor, interleaved):
    rot = 2 * len(inv)
    x = x.astype(np.float64).copy()
    ang = pos.astype(np.float64)[:, None, None] * inv
    c, s = factor * np.cos(ang), factor * np.sin(ang)
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., i].copy(), x[..., j].copy()
    mag = np.zeros_like(x)
    x[..., i], x[..., j] = a * c - b * s, b * c + a * s
    mag[..., i] = mag[..., j] = factor * (np.abs(a) + np.abs(b))
    return x, mag


ROPE_CASES = [  # tokens, q heads, k heads, head dim, rotated, buffer
    (1, 1, 1, 64, 64, "own"), (1, 32, 8, 128, 128, "fused"), (7, 3, 1, 96, 38, "own"), (33, 8, 2, 128, 64, "fused"),
    (129, 4, 4, 32, 32, "heads_first"), (5, 6, 2, 80, 2, "odd"), (300, 24, 8, 128, 128, "own"), (64, 2, 1, 256, 256, "fused"),
    (3000, 32, 8, 128, 128, "fused"), (50, 4, 0, 64, 16, "own"), (257, 5, 1, 100, 48, "odd"), (20, 40, 10, 64, 24, "own")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", ROPE_CASES, ids=str)
def test_rope(case, interleaved, dtype):
    import torch
    from paper_2410_12513_b200 import first_rope
    T, hq, hk, hd, rot, buf = case
    g = torch.Generator().manual_seed(T * 7 + hd)
    if buf == "fused":
        big = torch.randn(T, hq + 2 * hk, hd, generator=g).to(_t(dtype)).cuda()
        q, k = big[:, :hq], big[:, hq:hq + hk]
    elif buf == "heads_first":  # [heads][tokens][hd]
        big = torch.randn(hq + hk, T, hd, generator=g).to(_t(dtype)).cuda()
        q, k = big[:hq].transpose(0, 1), big[hq:].transpose(0, 1)
    elif buf == "odd":  # rows one element apart from any alignment
        big = torch.randn(T, (hq + hk) * hd + 1, generator=g).to(_t(dtype)).cuda()
        q, k = big[:, 1:1 + hq * hd].unflatten(1, (hq, hd)), big[:, 1 + hq * hd:].unflatten(1, (hk, hd))
    else:
        big = torch.randn(T, hq + hk, hd, generator=g).to(_t(dtype)).cuda()
        q, k = big[:, :hq].contiguous(), big[:, hq:].contiguous()
    pos = torch.randint(0, 1 << 20, (T,), generator=g, dtype=torch.int32)
    pos[0] = 0 if T > 1 else 1000003
    if T > 2:
        pos[1], pos[2] = 2 ** 31 - 1, -5
    inv = (10000.0 ** (-2.0 * np.arange(rot // 2) / rot))
    factor = 1.25
    before = big.float().cpu().numpy().copy()
    q0, k0 = q.float().cpu().numpy().copy(), k.float().cpu().numpy().copy()
    first_rope(q, k if hk else None, pos.cuda(), torch.from_numpy(inv).cuda(), factor=factor, interleaved=interleaved)
    for x0, x1 in ((q0, q), (k0, k)):
        if x0.size == 0:
            continue
        ref, mag = _rope_ref(x0, pos.numpy(), inv, factor, interleaved)
        got = x1.double().cpu().numpy()
        # float32 on the way: the angle as a fraction of a turn (2 pi 2^-26 = 1.6 units of 2^-24), sine and cosine
        # (1 unit), the factor (1), products and their sum (1.5); with the argument of the far positions' 64-bit
        # product (2^31 rad * 2^-53 = 4 units at the very largest): 10 units; then one rounding to the type
        tol = 10 * U32 * mag + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0)
        assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()
        assert np.array_equal(got[..., rot:], x0[..., rot:])  # elements beyond the rotated ones
    if buf == "fused":  # v between them is not touched
        assert np.array_equal(big.float().cpu().numpy()[:, hq + hk:], before[:, hq + hk:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hd,rot", [(8192, 8192), (8200, 8194), (6000, 4000), (2048, 2048)])
def test_rope_of_wide_heads(hd, rot, interleaved, dtype):
    """Heads that are wider than a block, aligned and not."""
    import torch
    from paper_2410_12513_b200 import first_rope
    g = torch.Generator().manual_seed(rot)
    q, k = torch.randn(5, 3, hd, generator=g).to(_t(dtype)).cuda(), torch.randn(5, 1, hd, generator=g).to(_t(dtype)).cuda()
    pos = torch.tensor([0, 1, 4097, 2 ** 31 - 1, 77], dtype=torch.int32)
    inv = 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    q0, k0 = q.float().cpu().numpy(), k.float().cpu().numpy()
    first_rope(q, k, pos.cuda(), torch.from_numpy(inv).cuda(), interleaved=interleaved)
    for x0, x1 in ((q0, q), (k0, k)):
        ref, mag = _rope_ref(x0, pos.numpy(), inv, 1.0, interleaved)
        tol = 10 * U32 * mag + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0)  # (as in test_rope)
        assert (np.abs(x1.double().cpu().numpy() - ref) <= tol).all()


def test_rope_of_an_empty_batch():
    import torch
    from paper_2410_12513_b200 import first_rope
    q, k = torch.empty(0, 4, 64, device="cuda"), torch.empty(0, 2, 64, device="cuda")
    pos, inv = torch.empty(0, dtype=torch.int32, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda")
    first_rope(q, k, pos, inv)
    first_rope(q, None, pos, inv, interleaved=True)


def test_rope_on_another_stream_and_in_a_graph():
    import torch
    from paper_2410_12513_b200 import first_rope
    q0 = torch.randn(40, 8, 64, device="cuda")
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    inv = torch.from_numpy(10000.0 ** (-np.arange(32) / 32.0)).cuda()
    want = q0.clone()
    first_rope(want, None, pos, inv)
    q = q0.clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    first_rope(q, None, pos, inv, stream=st)
    st.synchronize()
    assert torch.equal(q, want)
    q = q0.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first_rope(q, None, pos, inv)
    assert torch.equal(q, q0)
    graph.replay()
    assert torch.equal(q, want)
    pos.neg_()  # the replay reads the positions of its own time: turning back gives the input again
    graph.replay()
    assert (q - q0).abs().max() < 40 * U32 * q0.abs().max()  # two rotations' rounding


# ------------------------------------------------------------------ adapters
def _lora_ref(x, a, b, ids, y, scales, seg):
    x, a, b, y = (v.double().cpu().numpy() for v in (x, a, b, y))
    ids = ids.cpu().numpy()
    rank, mag = b.shape[2], np.abs(y)
    y = y.copy()
    for r, ad in enumerate(ids):
        if not 0 <= ad < a.shape[0]:
            continue
        sc = 1.0 if scales is None else float(scales[ad])
        h, hm = a[ad] @ x[r], np.abs(a[ad]) @ np.abs(x[r])
        for s in range(len(seg) - 1):
            f = slice(seg[s], seg[s + 1])
            y[r, f] += sc * (b[ad, f] @ h[s * rank:(s + 1) * rank])
            mag[r, f] += abs(sc) * (np.abs(b[ad, f]) @ hm[s * rank:(s + 1) * rank])
    return y, mag


LORA_CASES = [  # rows, adapters, rank, k, segments
    (1, 1, 8, 256, (0, 128)), (1, 3, 16, 4096, (0, 4096, 5120, 6144)), (2, 1, 8, 8, (0, 1)), (9, 2, 24, 264, (0, 16, 50)),
    (32, 16, 16, 2048, (0, 2048, 2560)), (33, 4, 128, 1000, (0, 48, 96, 160, 333)), (64, 64, 32, 688, (0, 255)),
    (257, 3, 8, 512, (0, 1024)), (100, 1, 64, 4096, (0, 512)), (1030, 7, 16, 256, (0, 96, 200)), (300, 500, 8, 128, (0, 64)),
    (40, 2, 48, 14336, (0, 64)), (17, 5, 72, 24, (0, 32, 48, 64))]


def _lora_inputs(case, xt, yt, wt, seed, whole=False):
    import torch
    rows, n, rank, k, seg = case
    g = torch.Generator().manual_seed(seed)

    def make(lo, *shape):
        if whole:
            return torch.randint(-lo, lo + 1, shape, generator=g).float()
        return torch.randn(*shape, generator=g)
    s = len(seg) - 1
    x, y = make(3, rows, k).to(xt).cuda(), make(8, rows, seg[-1]).to(yt).cuda()
    a, b = make(2, n, s * rank, k).to(wt).cuda(), make(2, n, seg[-1], rank).to(wt).cuda()
    ids = torch.randint(-1, n + 1, (rows,), generator=g, dtype=torch.int32)  # -1 and n: no adapter
    ids[rows // 2] = n - 1
    if rows > 4:
        ids[rows // 4: rows // 2] = 0  # a run
    return x, a, b, ids.cuda(), y, g


@pytest.mark.parametrize("types", [("bf16", "f32", "bf16"), ("f32", "f32", "bf16"), ("bf16", "bf16", "bf16"), ("f32", "f32", "f32"),
                                   ("f32", "bf16", "f32"), ("bf16", "f32", "f32")], ids=str)
@pytest.mark.parametrize("case", LORA_CASES, ids=str)
def test_lora(case, types):
    """Normal inputs, random scales."""
    import torch
    from paper_2410_12513_b200 import first_lora
    xt, yt, wt = (_t(v) for v in types)
    x, a, b, ids, y, g = _lora_inputs(case, xt, yt, wt, 11)
    rows, n, rank, k, seg = case
    scales = torch.rand(n, generator=g) * 2 - 1
    ref, mag = _lora_ref(x, a, b, ids, y, scales, seg)
    y0 = y.clone()
    first_lora(x, a, b, ids, y, scales=scales.cuda(), segments=seg)
    got = y.double().cpu().numpy()
    # sums in float32: no accumulator takes more than k/8 + 16 products one after the other (the rest meets in a tree),
    # then rank of them; every operand exact to 2^-24 at least.  That is a bound, so it is a loose one; what is rounded
    # to fewer bits on the way shows in test_lora_whole_numbers.
    tol = (k / 8 + rank + 24) * U32 * mag + (2.0 ** -8 * np.abs(ref) if types[1] == "bf16" else 0.0)
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) / tol).max()
    idle = ((ids < 0) | (ids >= n)).cpu().numpy()
    assert np.array_equal(got[idle], y0.double().cpu().numpy()[idle])


@pytest.mark.parametrize("wt", ["bf16", "f32"])
@pytest.mark.parametrize("xt", ["bf16", "f32"])
@pytest.mark.parametrize("case", LORA_CASES, ids=str)
def test_lora_whole_numbers(case, xt, wt):
    """Small whole numbers: every sum is a whole number below 2^24, so float32 arithmetic is exact in any order, and a
    value cut to fewer bits anywhere (A x needs up to 16 bits here) shows as a difference."""
    from paper_2410_12513_b200 import first_lora
    x, a, b, ids, y, _ = _lora_inputs(case, _t(xt), _t("f32"), _t(wt), 5, whole=True)
    ref, mag = _lora_ref(x, a, b, ids, y, None, case[4])
    if mag.max() >= 2 ** 24:
        x, y = x.clamp(-1, 1), y
        a, b = a.clamp(-1, 1), b.clamp(-1, 1)
        ref, mag = _lora_ref(x, a, b, ids, y, None, case[4])
    assert mag.max() < 2 ** 24
    first_lora(x, a, b, ids, y, segments=case[4])
    assert np.array_equal(y.double().cpu().numpy(), ref)


@pytest.mark.parametrize("types", [("bf16", "f32", "bf16"), ("f32", "bf16", "bf16"), ("bf16", "bf16", "f32"), ("f32", "f32", "f32")], ids=str)
@pytest.mark.parametrize("case", [(1000, 3, 24, 264, (0, 64, 176)), (960, 1, 128, 520, (0, 48, 208)), (960, 8, 56, 1032, (0, 1000)),
                                  (1500, 2, 8, 72, (0, 16, 32, 80, 96)), (300, 9, 40, 200, (0, 160, 431)), (700, 2, 16, 96, (0, 801))], ids=str)
def test_lora_many_rows(case, types):
    """Whole and ragged tiles of many rows, aligned and not; steps that end inside a segment."""
    import torch
    from paper_2410_12513_b200 import first_lora
    x, a, b, ids, y, g = _lora_inputs(case, *(_t(v) for v in types), 29)
    rows, n, rank, k, seg = case
    scales = torch.rand(n, generator=g) * 2 - 1
    ref, mag = _lora_ref(x, a, b, ids, y, scales, seg)
    y0 = y.clone()
    first_lora(x, a, b, ids, y, scales=scales.cuda(), segments=seg)
    tol = (k / 8 + rank + 24) * U32 * mag + (2.0 ** -8 * np.abs(ref) if types[1] == "bf16" else 0.0)  # (as in test_lora)
    assert (np.abs(y.double().cpu().numpy() - ref) <= tol).all()
    idle = (ids < 0) | (ids >= n)
    assert torch.equal(y[idle], y0[idle])


@pytest.mark.parametrize("types", [("bf16", "bf16", "bf16"), ("f32", "f32", "bf16"), ("bf16", "f32", "f32"), ("f32", "f32", "f32")], ids=str)
@pytest.mark.parametrize("n,rank,k,seg", [(8, 16, 520, (0, 1040, 2080)), (5, 24, 264, (0, 48, 1000)), (3, 8, 40, (0, 16, 2044)), (8, 16, 520, (0, 1041))], ids=str)
def test_lora_tiles_of_every_number_of_rows(n, rank, k, seg, types):
    """Tiles of 1 to 32 rows, some lanes of a warp without a row or a feature: every row as when it is alone, bit for bit, and
    rows without an adapter left alone."""
    import torch
    from paper_2410_12513_b200 import first_lora
    x, a, b, _, y, g = _lora_inputs((1024, n, rank, k, seg), *(_t(v) for v in types), 41)
    scales = (torch.rand(n, generator=g) * 2 - 1).cuda()
    for trial in range(6):
        count = torch.randint(1, 200, (n,), generator=g)
        count[-1] = 97 + trial
        ids = torch.cat([torch.full((int(c),), i) for i, c in enumerate(count)] + [torch.full((1024,), -1)])[:1024]
        ids = ids[torch.randperm(1024, generator=g)].to(torch.int32).cuda()
        got = y.clone()
        first_lora(x, a, b, ids, got, scales=scales, segments=seg)
        idle = ids < 0
        assert torch.equal(got[idle], y[idle])
        for r in torch.randperm(1024, generator=g)[:40].tolist():
            one = y[r:r + 1].clone()
            first_lora(x[r:r + 1], a, b, ids[r:r + 1], one, scales=scales, segments=seg)
            assert torch.equal(one, got[r:r + 1]), (trial, r)


def test_lora_padded_rows_empty_batch_and_bit_reproducible():
    import torch
    from paper_2410_12513_b200 import first_lora
    case = (50, 6, 16, 520, (0, 64, 133))
    x, a, b, ids, y, _ = _lora_inputs(case, _t("bf16"), _t("f32"), _t("bf16"), 3)
    want = y.clone()
    first_lora(x, a, b, ids, want, segments=case[4])
    xp = torch.full((50, 560), float("nan"), dtype=torch.bfloat16, device="cuda")
    yp = torch.full((50, 140), 7.0, device="cuda")
    xp[:, :520], yp[:, 3:136] = x, y
    first_lora(xp[:, :520], a, b, ids, yp[:, 3:136], segments=case[4])  # y aligned to its element only
    assert torch.equal(yp[:, 3:136], want) and (yp[:, :3] == 7).all() and (yp[:, 136:] == 7).all()
    # a row's result does not depend on the batch around it
    for r in (0, 17, 49):
        one = y[r:r + 1].clone()
        first_lora(x[r:r + 1], a, b, ids[r:r + 1], one, segments=case[4])
        assert torch.equal(one, want[r:r + 1])
    first_lora(x[:0], a, b, ids[:0], y[:0], segments=case[4])
    none = y.clone()
    first_lora(x, a, b, torch.full_like(ids, -1), none, segments=case[4])
    assert torch.equal(none, y)


@pytest.mark.parametrize("types", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "f32", "bf16")], ids=str)
@pytest.mark.parametrize("case", [(70, 2, 128, 264, (0, 64, 128, 192, 300)), (200, 1, 128, 72, (0, 48, 80, 97)), (1024, 64, 128, 32, (0, 33)),
                                  (40, 4096, 8, 32, (0, 40)), (40, 4097, 8, 32, (0, 40))], ids=str)
def test_lora_largest_ranks_segments_and_adapter_counts(case, types):
    """What takes the most shared memory, many adapters of which few are used, and more than a CTA counts."""
    import torch
    from paper_2410_12513_b200 import first_lora
    x, a, b, ids, y, g = _lora_inputs(case, *(_t(v) for v in types), 23)
    rows, n, rank, k, seg = case
    if n >= 4096:
        ids.copy_(torch.tensor([0, n - 1, 17, n - 1, -1, n, 4000, 2 ** 31 - 1] * 5, dtype=torch.int32))
    ref, mag = _lora_ref(x, a, b, ids, y, None, seg)
    first_lora(x, a, b, ids, y, segments=seg)
    tol = (k / 8 + rank + 24) * U32 * mag + (2.0 ** -8 * np.abs(ref) if types[1] == "bf16" else 0.0)  # (as in test_lora)
    assert (np.abs(y.double().cpu().numpy() - ref) <= tol).all()


def test_calls_of_several_threads_at_once():
    """Calls of different sizes from two host threads, each on a stream of its own."""
    import threading
    import torch
    from paper_2410_12513_b200 import first_lora, first_sample
    sizes = [((48, 2, 128, 264, (0, 64, 300)), 60000), ((200, 3, 8, 512, (0, 96)), 3000)]
    work, errors = [], []
    for case, v in sizes:
        x, a, b, ids, y, g = _lora_inputs(case, _t("bf16"), _t("f32"), _t("bf16"), 2)
        want = y.clone()
        first_lora(x, a, b, ids, want, segments=case[4])
        lg, u = torch.randn(20, v, generator=g).cuda(), torch.rand(20, generator=g).cuda()
        tok = torch.empty(20, dtype=torch.int32, device="cuda")
        first_sample(lg, u, tok)
        work.append((case, x, a, b, ids, y, want, lg, u, tok))
    torch.cuda.synchronize()

    def go(case, x, a, b, ids, y, want, lg, u, tok):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(50):
                    got, t = y.clone(), torch.empty_like(tok)
                    first_lora(x, a, b, ids, got, segments=case[4])
                    first_sample(lg, u, t)
                    assert torch.equal(got, want) and torch.equal(t, tok)
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=go, args=w) for w in work]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors, errors


def test_lora_rows_of_other_adapters_do_not_leak_nan():
    """NaN and infinities in rows without an adapter, or in adapters no row uses, reach nothing."""
    import torch
    from paper_2410_12513_b200 import first_lora
    case = (23, 5, 16, 264, (0, 80))
    x, a, b, ids, y, _ = _lora_inputs(case, _t("bf16"), _t("f32"), _t("bf16"), 9)
    ids[:] = torch.arange(23) % 3 - 1  # -1, 0, 1
    want = y.clone()
    first_lora(x, a, b, ids, want, segments=case[4])
    x[ids < 0] = float("nan")
    a[2:], b[2:] = float("nan"), float("inf")
    got = y.clone()
    first_lora(x, a, b, ids, got, segments=case[4])
    assert torch.equal(got, want)
    x[1] = float("inf")  # one row's own values stay its own
    got = y.clone()
    first_lora(x, a, b, ids, got, segments=case[4])
    keep = torch.arange(23, device="cuda") != 1
    assert torch.equal(got[keep], want[keep])


def _lora_same(got, ref, tol):
    """NaN where the definition has NaN, its infinities, and near it elsewhere."""
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf])
    ok = np.isfinite(ref)
    assert np.isfinite(got[ok]).all() and (np.abs(got - ref)[ok] <= tol[ok]).all()


@pytest.mark.parametrize("types", [("bf16", "f32", "bf16"), ("f32", "f32", "bf16"), ("bf16", "f32", "f32"), ("f32", "f32", "f32")], ids=str)
@pytest.mark.parametrize("case", [(1, 1, 8, 256, (0, 128)), (23, 2, 24, 264, (0, 80, 163)), (960, 2, 56, 72, (0, 64, 1040)), (40, 3, 16, 1000, (0, 1001))], ids=str)
@np.errstate(invalid="ignore", over="ignore")
def test_lora_infinities_and_nan_where_the_definition_has_them(case, types):
    """An infinity in x, in A or in B gives what the sums of the definition give, in its own rows and features only; the
    others keep their bits."""
    import torch
    from paper_2410_12513_b200 import first_lora
    rows, n, rank, k, seg = case
    x, a, b, ids, y, _ = _lora_inputs(case, *(_t(v) for v in types), 19)
    ids[:] = torch.arange(rows) % n
    plain = y.clone()
    first_lora(x, a, b, ids, plain, segments=seg)
    inf = float("inf")
    for where in ("x", "x two signs", "x nan", "a", "b", "b and a"):
        x1, a1, b1 = x.clone(), a.clone(), b.clone()
        hit = torch.zeros(rows, dtype=torch.bool, device="cuda")
        if where[0] == "x":
            hit[::7] = True
            x1[::7, k // 3] = float("nan") if "nan" in where else inf
            if "two" in where:
                x1[::7, k - 1] = -inf
        if "a" in where.split():
            a1[n - 1, 3, k // 2] = -inf
            hit |= ids == n - 1
        if where[0] == "b":
            b1[n - 1, seg[-1] - 2, rank - 1] = inf
            hit |= ids == n - 1
        ref, mag = _lora_ref(x1, a1, b1, ids, y, None, seg)
        got = y.clone()
        first_lora(x1, a1, b1, ids, got, segments=seg)
        _lora_same(got, ref, (k / 8 + rank + 24) * U32 * mag)  # (as in test_lora)
        assert torch.equal(got[~hit], plain[~hit])
        if where == "b":
            keep = torch.arange(seg[-1], device="cuda") != seg[-1] - 2
            assert torch.equal(got[:, keep], plain[:, keep])


@pytest.mark.parametrize("types", [("bf16", "bf16", "bf16"), ("f32", "f32", "f32")], ids=str)
@pytest.mark.parametrize("rows", [1, 40, 960])
def test_lora_rows_full_of_nan(rows, types):
    """Every fifth row NaN from end to end: NaN there, the other rows as without them."""
    import torch
    from paper_2410_12513_b200 import first_lora
    case = (rows, 2, 16, 4096, (0, 2048, 2600))
    x, a, b, ids, y, _ = _lora_inputs(case, *(_t(v) for v in types), 8)
    ids[:] = torch.arange(rows) % 2
    want = y.clone()
    first_lora(x, a, b, ids, want, segments=case[4])
    x[::5] = float("nan")
    first_lora(x, a, b, ids, y, segments=case[4])
    bad = torch.arange(rows, device="cuda") % 5 == 0
    assert y[bad].isnan().all() and torch.equal(y[~bad], want[~bad])


@pytest.mark.parametrize("rows", [1, 9, 960])
def test_lora_largest_float32_values(rows):
    """Finite float32 values that bfloat16 rounds to an infinity, in x, A, B and in A x."""
    import torch
    from paper_2410_12513_b200 import first_lora
    most = float(np.finfo(np.float32).max)
    case = (rows, 1, 8, 40, (0, 1040))
    for where in ("x", "a", "b", "h"):
        x, a, b, ids, y, _ = _lora_inputs(case, _t("f32"), _t("f32"), _t("f32"), 3)
        ids.zero_()
        if where == "x":
            x[:, 5] = -most
            a *= 1e-3
            b *= 1e-2
        elif where == "a":
            a[0, 2, 7] = 3.4e38
            x *= 1e-3
            b *= 1e-2
        elif where == "b":
            b[0, 33, 1] = most
            a *= 1e-4
        else:
            x.zero_()
            x[:, 0] = 1.0
            a.zero_()
            a[0, :, 0] = torch.tensor([3.4e38, -3.4e38, 1.0, most, 0.0, -most, 2.0, 1e38])
            b *= 1e-2
        ref, mag = _lora_ref(x, a, b, ids, y, None, case[4])
        assert np.isfinite(ref).all() and np.abs(ref).max() < most / 2
        first_lora(x, a, b, ids, y)
        _lora_same(y, ref, (40 / 8 + 8 + 24) * U32 * mag)


def test_lora_on_another_stream_and_in_a_graph():
    import torch
    from paper_2410_12513_b200 import first_lora
    case = (20, 4, 16, 512, (0, 256))
    x, a, b, ids, y, _ = _lora_inputs(case, _t("bf16"), _t("f32"), _t("bf16"), 4)
    want = y.clone()
    first_lora(x, a, b, ids, want)
    got = y.clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    first_lora(x, a, b, ids, got, stream=st)
    st.synchronize()
    assert torch.equal(got, want)
    got, other = y.clone(), y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first_lora(x, a, b, ids, got)
        first_lora(x, a, b, ids, other)
    graph.replay()
    assert torch.equal(got, want) and torch.equal(other, want)
    ids.copy_((ids + 1) % 4)  # the replay reads the ids of its own time
    got.copy_(y)
    graph.replay()
    want = y.clone()
    first_lora(x, a, b, ids, want)
    assert torch.equal(got, want)


# ------------------------------------------------------------------ sampling
def _sample_ref(x, u, temp, k, p, mp):
    """-> the tokens the definition allows: one, or neighbours where the draw, or the nucleus' border, is as near to a
    weight's border as float32 weights place it.  A weight is off by at most 2^-21 of itself: the exponential 2^-22, its
    argument's two roundings 2 * 2^-24 * 0.73, the rounding to 2^-23 of a value of at least exp(-1/2) 0.83 * 2^-23; in
    the open last bin the last two are at most 2^-22 of that bin's own weight.  So is every sum of weights; prefix
    sums themselves are 64-bit.  A border and the share of the sum it is compared with move by 2^-21 of the sum each."""
    V = x.size
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    order = np.lexsort((np.arange(V), -x))
    if x[order[0]] == -np.inf:
        return [-1]
    if not temp > 0:
        return [int(order[0])]
    order = order[x[order] > -np.inf]
    top = x[order[0]]
    with np.errstate(invalid="ignore"):
        d = np.where(x[order] == top, 0.0, x[order] - top)
        w = np.exp(d / temp) if np.isfinite(temp) else np.where(np.isneginf(d), 0.0, 1.0)
    if k > 0:
        w = w[:k]
    if mp > 0:
        w = w[w >= min(mp, 1.0)]
    eps = 2.0 ** -20 * w.sum()
    cum, below = np.cumsum(w), np.concatenate([[0.0], np.cumsum(w)[:-1]])
    one = float(np.float32(1) - np.float32(2.0 ** -24))
    u = one if not u == u else min(max(u, 0.0), one)

    def rank(off):  # of the token, everything shifted one way
        n = w.size
        if p < 1:
            n = max(1, int((below < max(p, 0.0) * cum[-1] + off).sum()))
        return min(int((cum[:n] <= u * cum[n - 1] + off).sum()), n - 1)
    lo, hi = rank(-eps), rank(eps)
    return [int(t) for t in order[lo:hi + 1]]


def _sample_check(x, u, temp=None, k=None, p=None, mp=None, pad=0):
    """Device tokens against the definition."""
    import torch
    from paper_2410_12513_b200 import first_sample
    B, V = x.shape
    dev = lambda v, t: None if v is None else torch.from_numpy(np.asarray(v, dtype=t)).cuda()  # noqa: E731
    buf = torch.full((B, V + pad), float("inf"), device="cuda")  # what lies behind a row is larger than all in it
    buf[:, :V] = torch.from_numpy(x)
    tok = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    first_sample(buf[:, :V], dev(u, np.float32), tok, temperature=dev(temp, np.float32), top_k=dev(k, np.int32), top_p=dev(p, np.float32),
                 min_p=dev(mp, np.float32))
    got = tok.cpu().numpy()
    f = lambda v, r, d: d if v is None else float(np.float32(v[r]))  # noqa: E731
    for r in range(B):
        want = _sample_ref(x[r], f(u, r, 0), f(temp, r, 1.0), 0 if k is None else int(k[r]), f(p, r, 1.0), f(mp, r, 0.0))
        assert got[r] in want, (r, got[r], want[:5])
    return got


def _sample_tokens(x, u, temp=None, k=None, p=None, mp=None):
    """The device's tokens."""
    import torch
    from paper_2410_12513_b200 import first_sample
    dev = lambda v, t: None if v is None else torch.from_numpy(np.asarray(v, dtype=t)).cuda()  # noqa: E731
    tok = torch.full((len(x),), -7, dtype=torch.int32, device="cuda")
    first_sample(torch.from_numpy(x).cuda(), dev(u, np.float32), tok, temperature=dev(temp, np.float32), top_k=dev(k, np.int32),
                 top_p=dev(p, np.float32), min_p=dev(mp, np.float32))
    return tok.cpu().numpy()


def _settings(B, g):
    return (np.where(g.random(B) < 0.1, 0.0, 0.3 + 1.5 * g.random(B)),
            np.choose(g.integers(0, 4, B), [np.zeros(B), 1 + g.integers(0, 20, B), 50 + g.integers(0, 400, B), 2000 + g.integers(0, 9000, B)]).astype(np.int32),
            np.where(g.random(B) < 0.3, 1.0, 0.5 + 0.5 * g.random(B)), np.where(g.random(B) < 0.5, 0.0, 0.2 * g.random(B)))


@pytest.mark.parametrize("B,V,pad", [(1, 1, 0), (3, 2, 1), (5, 31, 0), (7, 1000, 3), (16, 4099, 0), (4, 32000, 0), (9, 50257, 47), (40, 128256, 0),
                                     (2, 262144, 0), (2, 300001, 0), (1, 524288, 0)])
@pytest.mark.parametrize("spread", [0.5, 2.5, 8.0])
def test_sample_mixed_settings(B, V, pad, spread):
    g = np.random.default_rng(B * 1000 + V)
    x = (spread * g.standard_normal((B, V))).astype(np.float32)
    _sample_check(x, g.random(B).astype(np.float32), *_settings(B, g), pad=pad)


@pytest.mark.parametrize("B,V", [(24, 20011), (24, 40001), (160, 40001), (24, 70000), (160, 70000), (24, 140003)])
def test_sample_long_candidate_lists(B, V):
    """Thousands of candidates, which one CTA takes over from its cluster or not, by how many rows there are."""
    g = np.random.default_rng(B + V)
    x = (1.5 * g.standard_normal((B, V))).astype(np.float32)
    t = (0.6 + 0.9 * g.random(B)).astype(np.float32)
    k = np.where(np.arange(B) % 3 == 0, 0, g.integers(1500, 11000, B)).astype(np.int32)
    p = np.where(np.arange(B) % 4 == 3, 1.0, 0.4 + 0.6 * g.random(B)).astype(np.float32)
    _sample_check(x, g.random(B).astype(np.float32), t, k, p)
    x[:, ::2] = np.round(x[:, ::2])  # half of them in large ties, at the lists' borders too
    _sample_check(x, g.random(B).astype(np.float32), t, k, p)
    x = np.sort(x, axis=1)           # all in the cluster's last CTA
    _sample_check(x, g.random(B).astype(np.float32), t, k, p)


@pytest.mark.parametrize("which", ["temp", "k", "p", "mp", "plain"])
def test_sample_one_filter_alone(which):
    g = np.random.default_rng(3)
    B, V = 12, 20000
    x = (3 * g.standard_normal((B, V))).astype(np.float32)
    t, k, p, mp = _settings(B, g)
    _sample_check(x, g.random(B).astype(np.float32), t if which == "temp" else None, k if which == "k" else None,
                  p if which == "p" else None, mp if which == "mp" else None)


def test_sample_masked_rows_infinities_and_nan():
    g = np.random.default_rng(8)
    V = 5000
    x = g.standard_normal((12, V)).astype(np.float32)
    x[0] = -np.inf                                    # nothing to choose from
    x[1] = np.nan
    x[2, :] = -np.inf
    x[2, 4321] = -3.0                                 # one candidate
    x[3, ::2] = -np.inf
    x[4, 17:40] = np.inf                              # infinities tie among themselves
    x[5, ::3] = np.nan                                # NaN is no candidate
    x[6] = np.finfo(np.float32).min                   # all at the type's lowest value: a tie of all
    x[7, :] = np.finfo(np.float32).min
    x[7, 99] = 0.0
    x[8] = 3.25                                       # one value
    x[9, :] = np.where(np.arange(V) % 2, 0.0, -0.0)   # -0 = +0: a tie in index order
    x[10, :] = np.finfo(np.float32).max
    x[11, 2] = np.finfo(np.float32).max
    u = (g.random(12) * 0.999).astype(np.float32)
    for t in (None, np.full(12, 0.7), np.full(12, np.inf), np.full(12, 1e-30), np.zeros(12), np.full(12, -1.0), np.full(12, np.nan)):
        got = _sample_check(x, u, t)
        assert got[0] == got[1] == -1 and got[2] == 4321
        _sample_check(x, u, t, k=np.full(12, 37))
        _sample_check(x, u, t, p=np.full(12, 0.77))


@pytest.mark.parametrize("kind", ["equal", "two_values", "bf16", "close", "steps", "peak"])
def test_sample_ties_and_crowded_values(kind):
    """Thousands of equal or nearly equal logits: the order by index, and the search among one value's elements."""
    g = np.random.default_rng(21)
    B, V = 8, 40000
    x = g.standard_normal((B, V)).astype(np.float32)
    if kind == "equal":
        x[:] = -1.5
    elif kind == "two_values":
        x = np.where(g.random((B, V)) < 0.3, 1.0, 0.0).astype(np.float32)
    elif kind == "bf16":
        x = widen(fi.f32_to_bf16_bits(x))
    elif kind == "close":  # within a few steps of the type
        x = (100.0 + g.integers(0, 5, (B, V)) * np.float32(2.0 ** -17)).astype(np.float32)
    elif kind == "steps":
        x = np.floor(4 * x) / 4
    else:
        x[:, 777] = 60.0
    x = x.astype(np.float32)
    u = ((np.arange(B) + 0.37) / B).astype(np.float32)
    for s in ({}, {"k": np.full(B, 12345)}, {"p": np.full(B, 0.613)}, {"mp": np.full(B, 0.2)}, {"temp": np.full(B, 50.0)},
              {"k": np.full(B, 30000), "p": np.full(B, 0.9), "temp": np.full(B, 0.05)}):
        _sample_check(x, u, **s)


@pytest.mark.parametrize("V", [262144, 524288])
def test_sample_largest_vocabularies_all_at_a_bins_upper_end(V):
    """All candidates but one tie exactly where a histogram's bin begins, at its largest weight: sums of 2^19 of them."""
    x = np.full((2, V), -0.25, np.float32)  # half a bin's width below the maximum: the second bin's upper end
    x[:, 1000] = 0.0
    u = np.array([0.31, 0.999], np.float32)
    _sample_check(x, u)
    _sample_check(x, u, k=np.array([V - 5, 200000]), p=np.array([0.5, 0.9]))
    x[:, 1000] = -0.25
    _sample_check(x, u, temp=np.full(2, np.inf))


def test_sample_values_outside_their_ranges():
    g = np.random.default_rng(5)
    B, V = 6, 3000
    x = (2 * g.standard_normal((B, V))).astype(np.float32)
    u = np.array([-1.0, 0.0, 1.0, 7.0, np.nan, 0.99999994], np.float32)
    got = _sample_check(x, u)
    order = [np.lexsort((np.arange(V), -x[b])) for b in range(B)]
    assert got[0] == order[0][0] and got[1] == order[1][0]
    u = g.random(B).astype(np.float32)
    _sample_check(x, u, k=np.array([0, -1, V, V + 5, 2 ** 31 - 1, 1]))
    assert (_sample_check(x, u, p=np.array([0.0, -1.0, 1e-9, 0.0, 0.0, 0.0])) == [o[0] for o in order]).all()
    _sample_check(x, u, p=np.array([1.0, 2.0, np.inf, 1.5, 1.0, 3.0]))
    assert (_sample_check(x, u, mp=np.array([1.0, 2.0, np.inf, 1.0, 1.5, 1.0])) == [o[0] for o in order]).all()
    _sample_check(x, u, mp=np.array([0.0, -1.0, -np.inf, np.nan, 0.0, 0.0]))


def test_sample_min_p_above_one_keeps_the_first_candidate_alone():
    g = np.random.default_rng(6)
    for V in (900, 20000, 140003):
        x = np.floor(2 * g.standard_normal((6, V))).astype(np.float32)  # ties at the largest
        x[3] = 0.5
        x[4, ::7] = np.inf
        first = x.argmax(1)
        u = np.array([0.0, 0.3, 0.6, 0.9, 0.95, 0.999], np.float32)
        for temp in (None, np.full(6, 0.7), np.full(6, np.inf), np.full(6, 1e-6)):
            for mp in (1.5, np.inf, float(np.nextafter(np.float32(1), np.float32(2)))):
                assert (_sample_tokens(x, u, temp, mp=np.full(6, mp)) == first).all()
        got = _sample_tokens(x, u, mp=np.ones(6))  # at 1 all of the largest stay
        assert (x[np.arange(6), got] == x.max(1)).all() and (got != first).any()


def test_sample_agrees_with_top_k_sampling_of_the_batch():
    import torch
    from paper_2410_12513_b200 import first_sample, first_sample_topk
    g = torch.Generator(device="cuda").manual_seed(2)
    x = 2 * torch.randn(64, 32000, generator=g, device="cuda")
    u = torch.rand(64, generator=g, device="cuda")
    a, b = (torch.empty(64, dtype=torch.int32, device="cuda") for _ in range(2))
    first_sample_topk(x, 10, 0.8, u, a)
    first_sample(x, u, b, temperature=torch.full((64,), 0.8, device="cuda"), top_k=torch.full((64,), 10, dtype=torch.int32, device="cuda"))
    assert torch.equal(a, b)


def test_sample_draws_follow_the_distribution():
    """An even grid of draws over one row: every token's count is its probability, to one."""
    import torch
    from paper_2410_12513_b200 import first_sample
    n, V = 4096, 50
    x = torch.linspace(-3, 2, V, device="cuda")[torch.randperm(V, generator=torch.Generator().manual_seed(1))]
    u = (torch.arange(n, device="cuda") + 0.5) / n
    tok = torch.empty(n, dtype=torch.int32, device="cuda")
    first_sample(x.expand(n, V).contiguous(), u, tok)
    count = torch.bincount(tok.long(), minlength=V).double()
    assert (count - n * torch.softmax(x.double(), 0)).abs().max() <= 1.0 + 1e-6


def test_sample_on_another_stream_in_a_graph_and_bit_reproducible():
    import torch
    from paper_2410_12513_b200 import first_sample
    g = torch.Generator(device="cuda").manual_seed(4)
    x = 2 * torch.randn(33, 40001, generator=g, device="cuda")
    u, tp = torch.rand(33, generator=g, device="cuda"), 0.5 + 0.5 * torch.rand(33, generator=g, device="cuda")
    tok = lambda: torch.empty(33, dtype=torch.int32, device="cuda")  # noqa: E731
    want, got = tok(), tok()
    first_sample(x, u, want, top_p=tp)
    for _ in range(20):
        first_sample(x, u, got, top_p=tp)
        assert torch.equal(got, want)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    other = tok()
    st.wait_stream(torch.cuda.current_stream())
    first_sample(x, u, other, top_p=tp, stream=st)
    first_sample(x, u, got, top_p=tp)  # at the same time
    torch.cuda.synchronize()
    assert torch.equal(other, want) and torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first_sample(x, u, got, top_p=tp)
    u.copy_(torch.rand(33, generator=g, device="cuda"))
    graph.replay()
    first_sample(x, u, want, top_p=tp)
    assert torch.equal(got, want)


@pytest.mark.parametrize("V", [300, 1000, 2000, 4096, 16384, 20000, 40000, 70000, 128256])
@pytest.mark.parametrize("top", [0, 5])
def test_sample_top_k_cuts_a_run_of_equal_logits(V, top):
    """The k-th candidate stands inside a run of equal logits, of hundreds to thousands in one CTA or spread over a
    cluster, alone or below a few larger ones: those behind it are out, in every later search too."""
    g = np.random.default_rng(V + top)
    B = 12
    for n in (300, 800, 2000, 2500):
        n = min(n, V - top)
        x = (-3.0 - g.random((B, V))).astype(np.float32)
        for r in range(B):
            at = np.sort(g.choice(V, n + top, replace=False)) if r % 3 else np.arange(n + top) + int(g.integers(0, V - n - top + 1))
            x[r, at] = 0.25
            x[r, g.choice(at, top, replace=False)] = 0.5 + 0.1 * np.arange(top, dtype=np.float32)
        u = ((np.arange(B) + 0.37) / B).astype(np.float32)
        for k in (1 + top, 10, 100, 225):
            _sample_check(x, u, k=np.full(B, k))
            _sample_check(x, u, k=np.full(B, k), p=np.full(B, 0.7))
            _sample_check(x, u, k=np.full(B, k), temp=np.full(B, 4.0), mp=np.full(B, 0.01))


@pytest.mark.parametrize("V", [1000, 20000, 40000, 128256, 140003])
def test_sample_temperatures_of_a_few_steps_of_the_maximum(V):
    """Temperatures of 0.3 to 4096 steps of float32 at the maximum, with hundreds of candidates within a few of those
    steps: what rounds at the maximum's size must not move weights, nor the room that lists of candidates need."""
    g = np.random.default_rng(V)
    for m in (10.0, 12.0, 33.0, 100.0, 1.0000001, -7.3, 16384.5, 1e6):
        ulp = float(np.spacing(np.float32(abs(m))))
        steps = np.array([0.3, 0.6, 1.0, 1.7, 2.668, 4.0, 8.0, 16.0, 30.0, 64.0, 256.0, 4096.0])
        B = steps.size
        temp = (steps * ulp).astype(np.float32)
        u = np.where(np.arange(B) % 2, 0.98, g.random(B)).astype(np.float32)
        for n, crowd in ((270, 1), (900, 1), (900, 3), (900, 40)):
            x = np.full((B, V), m - 100 - abs(m), np.float32)
            for r in range(B):
                at = np.sort(g.choice(V, n + 1, replace=False)) if r % 3 else np.arange(n + 1)
                x[r, at] = (m - ulp * np.round(np.maximum(1, steps[r] * (0.3 + 0.6 * g.random())) + g.integers(0, crowd, n + 1))).astype(np.float32)
                x[r, at[0]] = m
            _sample_check(x, u, temp)
            _sample_check(x, u, temp, p=np.full(B, 0.8))
            _sample_check(x, u, temp, k=np.full(B, 500), p=np.full(B, 0.9))


def test_sample_hundreds_of_candidates_two_steps_below_the_maximum():
    x = np.full((1, 1000), -100, np.float32)
    x[0, 500] = 10
    x[0, 100:370] = 10 - 2 * np.spacing(np.float32(10))
    assert _sample_check(x, np.array([0.98], np.float32), np.array([2.5444e-6])) == [364]


@pytest.mark.parametrize("V", [777, 50257, 128256, 262144])
def test_sample_of_equal_weights_is_exact(V):
    """Equal weights: token floor(u n) of the n candidates, with no allowance, however small a share of the sum one is."""
    g = np.random.default_rng(V)
    x = np.full((64, V), 1.75, np.float32)
    n = np.full(64, V)
    for r in range(1, 64, 2):  # every second row: some of them, below a filter's limit the others
        n[r] = g.integers(1, V)
        x[r, g.choice(V, V - n[r], replace=False)] = -np.inf
    u = ((np.floor(g.random(64) * n) + 0.1 + 0.8 * g.random(64)) / n).astype(np.float32)
    u = np.minimum(u, np.float32(1 - 2.0 ** -24))
    at = u.astype(np.float64) * n
    clear = np.abs(at - np.round(at)) > 1e-6 * n * 2.0 ** -24  # (the sums are exact; u n has 64 bits)
    for temp in (None, np.full(64, 0.7), np.full(64, 1e-6), np.full(64, np.inf)):
        got = _sample_tokens(x, u, temp)
        for r in np.nonzero(clear)[0]:
            assert got[r] == np.nonzero(x[r] > -np.inf)[0][int(at[r])], r


@pytest.mark.parametrize("V", [50257, 262144])
@pytest.mark.parametrize("spread,temp", [(0.01, 1.0), (0.5, 1.0), (2.5, 0.6), (4.0, 1.3)])
def test_sample_is_as_fine_as_its_draws(V, spread, temp):
    """Draws next to tokens' borders: the token is that of a draw at most one step of float32 (2^-24) away."""
    g = np.random.default_rng(V)
    B = 32
    x = (spread * g.standard_normal((B, V))).astype(np.float32)
    order = np.argsort(-x, axis=1, kind="stable")
    xs = np.take_along_axis(x, order, 1).astype(np.float64)
    cum = np.cumsum(np.exp((xs - xs[:, :1]) / float(np.float32(temp))), 1)
    share = cum / cum[:, -1:]
    place = np.empty_like(order)
    np.put_along_axis(place, order, np.arange(V)[None], 1)
    for trial in range(6):
        j = np.array([min(int(np.searchsorted(share[b], g.random())), V - 2) for b in range(B)])
        u = share[np.arange(B), j].astype(np.float32)
        u = np.clip(np.nextafter(u, np.float32(trial % 2)) if trial % 3 else u, 0, np.float32(1 - 2.0 ** -24))
        got = place[np.arange(B), _sample_tokens(x, u, np.full(B, temp))]
        hi = share[np.arange(B), got]
        lo = np.where(got > 0, share[np.arange(B), np.maximum(got - 1, 0)], 0.0)
        assert np.maximum(u - hi, lo - u).max() <= 2.0 ** -24


@pytest.mark.parametrize("B,V", [(200, 128256), (96, 40001), (64, 20011)])
def test_sample_is_the_same_beside_other_work(B, V):
    """The exchanges inside a cluster and the hand-over to one CTA while other kernels delay some of its warps: every
    run gives the same tokens, and they are the definition's."""
    import torch
    g = np.random.default_rng(B)
    x = (1.7 * g.standard_normal((B, V))).astype(np.float32)
    u, (t, k, p, mp) = g.random(B).astype(np.float32), _settings(B, g)
    want = _sample_check(x, u, t, k, p, mp)
    from paper_2410_12513_b200 import first_sample
    dev = [torch.from_numpy(np.asarray(v, dtype=d)).cuda() for v, d in ((t, np.float32), (k, np.int32), (p, np.float32), (mp, np.float32))]
    xd, ud, tok = torch.from_numpy(x).cuda(), torch.from_numpy(u).cuda(), torch.empty(B, dtype=torch.int32, device="cuda")
    side, noise = torch.cuda.Stream(), torch.randn(1 << 22, device="cuda")
    for _ in range(30):
        with torch.cuda.stream(side):
            for _ in range(8):
                noise.mul_(1.0000001)
        first_sample(xd, ud, tok, *dev)
        assert np.array_equal(tok.cpu().numpy(), want)


# ------------------------------------------------------------------ inside the step
ADAPTED = fi.ModelShape(3, 256, 8, 2, 64, 352, 512, 10000.0)


def _ctx(shape, bf16, max_batch, max_tokens, w):
    from paper_2410_12513_b200 import FirstContext
    return FirstContext(shape, BF16 if bf16 else F32, max_batch, max_tokens, gpu_weights(w))


def _adapters(shape, n, rank, seed, bf16, targets=("qkv", "o", "gate_up", "down"), skip=()):
    """-> (device adapters, host float32 copies [target][layer] = (a, b))."""
    import torch
    D, F, qd, kv = shape.d_model, shape.ffn_dim, shape.q_dim, shape.kv_dim
    sizes = {"qkv": (3, D, qd + 2 * kv), "o": (1, qd, D), "gate_up": (2, D, 2 * F), "down": (1, F, D)}
    dev, host = {}, {}
    for t in targets:
        s, k, out = sizes[t]
        dev[t], host[t] = [], []
        for l in range(shape.n_layers):
            if (t, l) in skip:
                dev[t].append(None)
                host[t].append(None)
                continue
            a = fi.normal((n, s * rank, k), 0.05, seed, f"{t}_a{l}", bf16)
            b = fi.normal((n, out, rank), 0.05, seed, f"{t}_b{l}", bf16)
            host[t].append((widen(a), widen(b)))
            dev[t].append(tuple(torch.from_numpy(v.view(np.int16)).cuda().view(torch.bfloat16) if bf16 else torch.from_numpy(v).cuda()
                                for v in (a, b)))
    return dev, host


def _merged(shape, w, host, ad, rank, scale):
    """Weights with adapter `ad` merged in (float32)."""
    m = {k: ([None if v is None else widen(v).astype(np.float32) for v in x] if isinstance(x, list) else widen(x)) for k, x in w.items()}
    if ad is None:
        return m
    qd, kv, F = shape.q_dim, shape.kv_dim, shape.ffn_dim
    parts = {"qkv": [("wq", 0, qd), ("wk", qd, qd + kv), ("wv", qd + kv, qd + 2 * kv)], "o": [("wo", 0, shape.d_model)],
             "gate_up": [("wg", 0, F), ("wu", F, 2 * F)], "down": [("wd", 0, shape.d_model)]}
    for t, layers in host.items():
        for l, p in enumerate(layers):
            if p is None:
                continue
            a, b = p[0][ad].astype(np.float64), p[1][ad].astype(np.float64)
            for s, (name, f0, f1) in enumerate(parts[t]):
                m[name][l] = (m[name][l] + scale * (b[f0:f1] @ a[s * rank:(s + 1) * rank])).astype(np.float32)
    return m


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("targets,skip", [(("qkv", "o", "gate_up", "down"), ()), (("qkv",), (("qkv", 1),)), (("o", "down"), ()), (("gate_up",), ())])
def test_step_with_adapters_equals_merged_weights(bf16, targets, skip):
    """Prompt phase and decode steps of a mixed batch, every sequence with its own adapter (or none): each sequence's
    logits against an oracle run of its own, on weights with its adapter merged in."""
    import torch
    shape, rank, n = ADAPTED, 8, 3
    lens, ids = [9, 30, 17, 5, 21], [2, -1, 0, 1, 2]
    B, L = len(lens), shape.n_layers
    w = fi.make_weights(shape, 31, bf16)
    dev, host = _adapters(shape, n, rank, 77, bf16, targets, skip)
    scales = np.array([1.0, 0.5, 2.0], np.float32)
    mask = np.array([[1, 1, 1], [1, 0, 1], [1, 0, 1], [1, 1, 1], [0, 1, 1]], np.uint8)
    prompts = [fi.tokens(shape, m, 3, f"p{b}") for b, m in enumerate(lens)]
    oms = {a: oracle_model(shape, _merged(shape, w, host, None if a < 0 else a, rank, float(scales[a])), kv_bf16=bf16) for a in set(ids)}
    okv = [oracle.OracleKV(oms[-1].shape, [m + 4]) for m in lens]
    pre = [oracle.prefill(oms[ids[b]], okv[b], 0, prompts[b], want_router_in=False) for b in range(B)]

    ctx = _ctx(shape, bf16, 64, 64, w)
    seq = torch.full((64,), -1, dtype=torch.int32, device="cuda")
    seq[:B] = torch.tensor(ids, dtype=torch.int32)
    ctx.set_adapters(dev, seq, torch.from_numpy(scales).cuda())
    kv = GpuKV(shape, [m + 4 for m in lens], bf16)
    logits = torch.empty((B, shape.vocab), device="cuda")
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    ctx.prefill(torch.from_numpy(np.concatenate(prompts)).cuda(), cu, kv.c, logits=logits)
    tol = 2e-2 if bf16 else 1e-4
    ref = np.stack([np.asarray(p["logits"]).reshape(-1, shape.vocab)[0] for p in pre])
    err, _ = logits_check(logits.cpu().numpy(), ref)
    assert err.max() <= tol, err
    plain = logits.clone()
    ctx.set_mask(torch.from_numpy(mask).cuda())
    toks = oracle.argmax(ref)
    for _ in range(3):
        ref = np.concatenate([oracle.decode_step(oms[ids[b]], toks[b:b + 1], mask[b:b + 1], okv[b]) for b in range(B)])
        ctx.decode_step(torch.from_numpy(toks).cuda(), kv.c, logits)
        err, _ = logits_check(logits.cpu().numpy(), ref)
        assert err.max() <= tol, err
        toks = oracle.argmax(ref)
    assert ctx.device_flags() == 0
    # the ids are read when a step runs: with no adapter for anyone the prompt gives the plain model's logits, and so
    # it does once the adapters are taken off
    base = oracle_model(shape, w)
    refs = []
    for b in range(B):
        o = oracle.OracleKV(base.shape, [lens[b] + 4])
        refs.append(np.asarray(oracle.prefill(base, o, 0, prompts[b], want_router_in=False)["logits"]).reshape(-1, shape.vocab)[0])
    for off in ("ids", "none"):
        if off == "ids":
            seq.fill_(-1)
        else:
            seq[:B] = torch.tensor(ids, dtype=torch.int32)
            ctx.set_adapters(None)
        ctx.prefill(torch.from_numpy(np.concatenate(prompts)).cuda(), cu, kv.c, logits=logits)
        err, _ = logits_check(logits.cpu().numpy(), np.stack(refs))
        assert err.max() <= tol
    assert not torch.equal(plain, logits)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("fuse", [0, 1])
def test_step_with_other_frequencies(bf16, fuse):
    """first_set_rope: another base and a factor against an oracle model with that base whose q and k projections carry
    the factor; NULL gives the description's frequencies back, bit for bit (float32) as before."""
    import torch
    shape = fi.ModelShape(2, 256, 4, 2, 64, 352, 512, 10000.0)
    other = fi.ModelShape(2, 256, 4, 2, 64, 352, 512, 700.0)
    w = fi.make_weights(shape, 5, bf16)
    factor = 1.25
    wm = {k: ([widen(v).astype(np.float32) for v in x] if isinstance(x, list) else widen(x)) for k, x in w.items()}
    for l in range(2):
        wm["wq"][l], wm["wk"][l] = wm["wq"][l] * np.float32(factor), wm["wk"][l] * np.float32(factor)
    om = oracle_model(other, wm, kv_bf16=bf16)
    from paper_2410_12513_b200 import first_rope_freqs
    inv, _ = first_rope_freqs(64, 700.0)
    n = 40
    prompt = fi.tokens(shape, n, 3, "p")
    ctx = _ctx(shape, bf16, 64, 64, w)
    ctx.set_option("fuse_rope", fuse)
    logits = torch.empty((1, shape.vocab), device="cuda")
    kv = GpuKV(shape, [n + 4], bf16)

    def run(ref_model):
        okv = oracle.OracleKV(om.shape, [n + 4])
        ref = np.asarray(oracle.prefill(ref_model, okv, 0, prompt, want_router_in=False)["logits"]).reshape(-1, shape.vocab)[:1]
        ctx.prefill(torch.from_numpy(prompt).cuda(), np.array([0, n], np.int32), kv.c, logits=logits)
        outs, errs = [logits.clone()], [logits_check(logits.cpu().numpy(), ref)[0].max()]
        ctx.set_mask(torch.ones((1, 2), dtype=torch.uint8, device="cuda"))
        for _ in range(2):
            toks = oracle.argmax(ref)
            ref = oracle.decode_step(ref_model, toks, np.ones((1, 2), np.uint8), okv)
            ctx.decode_step(torch.from_numpy(toks).cuda(), kv.c, logits)
            outs.append(logits.clone())
            errs.append(logits_check(logits.cpu().numpy(), ref)[0].max())
        assert max(errs) <= (2e-2 if bf16 else 1e-4), errs
        return outs
    plain = oracle_model(shape, w)
    first = run(plain)
    ctx.set_rope(inv, factor)
    run(om)
    ctx.set_rope(None)
    again = run(plain)
    if not bf16:
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("factor", [1.0, 1.25])
def test_rope_turns_by_the_factors_of_the_step(factor):
    """The key that a step appends at a position against first_rope on the key it appends at position 0 (no rotation).  The
    second half of every key is zero, so that a rotated element is one product: equal bits are equal cosines and sines."""
    import torch
    from paper_2410_12513_b200 import first_rope
    shape = fi.ModelShape(1, 64, 2, 2, 64, 80, 32, 500000.0)
    B = 64
    w = fi.make_weights(shape, 3, False)
    w["wk"][0].reshape(2, 64, 64)[:, 32:] = 0.0
    inv = 500000.0 ** (-np.arange(32) / 32.0)
    g = np.random.default_rng(4)
    ctx = _ctx(shape, False, B, 8, w)
    ctx.set_mask(torch.ones((B, 1), dtype=torch.uint8, device="cuda"))
    tok = torch.arange(B, dtype=torch.int32, device="cuda") % 32

    def keys(pos):  # [B][heads][64] as appended at these positions
        _, kv = synthetic_caches(shape, [1] * B, [4] * B, 1, False)
        kv.pos.copy_(torch.from_numpy(pos.astype(np.int32)))
        ctx.decode_step(tok, kv.c)
        return kv.k[0].view(2, B, 4, 64)[:, :, 1].transpose(0, 1).contiguous()
    base = keys(np.zeros(B))
    ctx.set_rope(inv, factor)
    for far in (100, 5000, 1 << 20, 2 ** 31 - 1):
        pos = g.integers(0, far, B)
        pos[0] = far - 1
        q = base.clone()
        first_rope(q, None, torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(inv).cuda(), factor=factor)
        assert torch.equal(q, keys(pos)), far


def test_step_with_per_row_sampling():
    """next_tokens of a step = the definition on that step's logits; parameters and draws are read when the step runs
    (a recorded step is replayed with new ones); the last choice of sampling holds."""
    import torch
    from paper_2410_12513_b200 import first_sample
    shape = fi.ModelShape(2, 256, 4, 2, 64, 352, 3001, 10000.0)
    B = 6
    w = fi.make_weights(shape, 5, True)
    _, kv = synthetic_caches(shape, [10] * B, [60] * B, 1, True)
    ctx = _ctx(shape, True, B, 60, w)
    ctx.set_mask(torch.ones((B, 2), dtype=torch.uint8, device="cuda"))
    logits = torch.empty((B, shape.vocab), device="cuda")
    nxt = torch.empty(B, dtype=torch.int32, device="cuda")
    tok = torch.arange(B, dtype=torch.int32, device="cuda")
    u = torch.empty(B, device="cuda")
    temp = torch.tensor([0.0, 0.5, 1.0, 1.0, 0.2, 3.0], device="cuda")
    k = torch.tensor([0, 5, 0, 100, 50, 0], dtype=torch.int32, device="cuda")
    tp = torch.tensor([1.0, 0.9, 0.6, 0.95, 1.0, 0.3], device="cuda")
    mp = torch.tensor([0.0, 0.0, 0.05, 0.0, 0.1, 0.0], device="cuda")
    ctx.set_sampling_rows(u, temp, k, tp, mp)
    pos0 = kv.pos.clone()
    want = torch.empty_like(nxt)
    for t in range(6):
        u.copy_(torch.rand(B, generator=torch.Generator().manual_seed(t)))
        if t == 3:
            temp.fill_(0.9)
        ctx.decode_step(tok, kv.c, logits, nxt)
        first_sample(logits, u, want, temperature=temp, top_k=k, top_p=tp, min_p=mp)
        assert torch.equal(nxt, want)
        f = lambda v: v.cpu().numpy()  # noqa: E731
        for r in range(B):
            assert int(nxt[r]) in _sample_ref(f(logits)[r], float(u[r]), float(temp[r]), int(k[r]), float(tp[r]), float(mp[r]))
    assert torch.equal(kv.pos, pos0 + 6)
    ctx.set_sampling(3, 0.8, u)
    ctx.decode_step(tok, kv.c, logits, nxt)
    from paper_2410_12513_b200 import first_sample_topk
    first_sample_topk(logits, 3, 0.8, u, want)
    assert torch.equal(nxt, want)
    ctx.set_sampling_rows(u)
    ctx.set_sampling_rows(None)
    ctx.decode_step(tok, kv.c, logits, nxt)
    assert np.array_equal(nxt.cpu().numpy(), oracle.argmax(logits.cpu().numpy()))


def test_operators_together():
    """One mixed batch as it is served: adapters, scaled frequencies and per-request sampling set on the context,
    sequences joining a pool with the ids of their slots; against per-sequence oracle runs on merged weights."""
    import torch
    from paper_2410_12513_b200 import FirstPool
    shape, rank = ADAPTED, 16
    base = fi.ModelShape(3, 256, 8, 2, 64, 352, 512, 3000.0)
    w = fi.make_weights(shape, 13, False)
    dev, host = _adapters(shape, 2, rank, 5, False)
    lens, ids = [12, 25, 7], [1, 0, -1]
    mask = np.array([[1, 1, 0], [1, 0, 1], [1, 1, 1]], np.uint8)
    oms = {a: oracle_model(base, _merged(shape, w, host, None if a < 0 else a, rank, 1.0)) for a in ids}
    prompts = [fi.tokens(shape, m, 3, f"p{b}") for b, m in enumerate(lens)]
    okv = [oracle.OracleKV(oms[-1].shape, [m + 8]) for m in lens]
    pre = [np.asarray(oracle.prefill(oms[ids[b]], okv[b], 0, prompts[b], want_router_in=False)["logits"]).reshape(-1, 512)[0] for b in range(3)]
    ctx = _ctx(shape, False, 32, 40, w)
    from paper_2410_12513_b200 import first_rope_freqs
    ctx.set_rope(*first_rope_freqs(64, 3000.0))
    seq = torch.full((32,), -1, dtype=torch.int32, device="cuda")
    seq[:3] = torch.tensor(ids, dtype=torch.int32)
    ctx.set_adapters(dev, seq)
    u = torch.tensor([0.3, 0.6, 0.9], device="cuda")
    temp, tp = torch.tensor([0.7, 1.0, 0.0], device="cuda"), torch.tensor([0.9, 0.8, 1.0], device="cuda")
    k = torch.tensor([0, 40, 0], dtype=torch.int32, device="cuda")
    ctx.set_sampling_rows(u, temp, k, tp)
    stage = GpuKV(shape, [m + 8 for m in lens], False)
    logits, nxt = torch.empty((3, 512), device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    ctx.prefill(torch.from_numpy(np.concatenate(prompts)).cuda(), np.array([0, 12, 37, 44], np.int32), stage.c, logits=logits, next_tokens=nxt)
    assert logits_check(logits.cpu().numpy(), np.stack(pre))[0].max() <= 1e-4
    for b in range(3):
        assert int(nxt[b]) in _sample_ref(logits[b].cpu().numpy(), float(u[b]), float(temp[b]), int(k[b]), float(tp[b]), 0.0)
    pk = [torch.zeros((2, 120, 64), device="cuda") for _ in range(3)]
    pool = FirstPool(ctx, 5, pk, [torch.zeros_like(t) for t in pk])
    slots = [pool.join(mask[b], lens[b] + 8, src=stage.c, src_seq=b, n_tokens=lens[b]) for b in (2, 0, 1)]
    at = {2: slots[0], 0: slots[1], 1: slots[2]}
    pool.commit()
    seq.fill_(-1)
    u5, t5, p5, k5 = torch.zeros(5, device="cuda"), torch.zeros(5, device="cuda"), torch.ones(5, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    tok = torch.zeros(5, dtype=torch.int32, device="cuda")
    for b in range(3):
        s = at[b]
        seq[s], u5[s], t5[s], p5[s], k5[s], tok[s] = ids[b], u[b], temp[b], tp[b], k[b], nxt[b]
    ctx.set_sampling_rows(u5, t5, k5, p5)
    lg, nt = torch.empty((5, 512), device="cuda"), torch.empty(5, dtype=torch.int32, device="cuda")
    for _ in range(3):
        host_tok = tok.cpu().numpy()
        ctx.decode_step(tok, pool.kv, lg, nt)
        for b in range(3):
            s = at[b]
            ref = oracle.decode_step(oms[ids[b]], host_tok[s:s + 1], mask[b:b + 1], okv[b])
            assert logits_check(lg[s:s + 1].cpu().numpy(), ref)[0].max() <= 1e-4
            assert int(nt[s]) in _sample_ref(lg[s].cpu().numpy(), float(u5[s]), float(t5[s]), int(k5[s]), float(p5[s]), 0.0)
        tok.copy_(nt)
    assert ctx.device_flags() == 0
    pool.close()


def test_context_checks_the_length_of_what_it_borrows():
    import torch
    shape = fi.ModelShape(2, 64, 2, 2, 32, 80, 32)
    _, kv = synthetic_caches(shape, [3, 3, 3], [9] * 3, 1, False)
    ctx = _ctx(shape, False, 3, 9, fi.make_weights(shape, 1, False))
    dev, _ = _adapters(shape, 2, 8, 1, False)
    with pytest.raises(ValueError):
        ctx.set_adapters(dev, torch.zeros(2, dtype=torch.int32, device="cuda"))
    ctx.set_mask(torch.ones((3, 2), dtype=torch.uint8, device="cuda"))
    ctx.set_sampling_rows(torch.zeros(2, device="cuda"))
    tok, nxt = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        ctx.decode_step(tok, kv.c, None, nxt)
    with pytest.raises(ValueError):
        ctx.prefill(tok, np.array([0, 1, 2, 3], np.int32), kv.c, next_tokens=nxt)
    ctx.decode_step(tok, kv.c)  # (nothing is sampled)
    ctx.set_sampling_rows(torch.zeros(3, device="cuda"), temperature=torch.ones(3, device="cuda"))
    ctx.decode_step(tok, kv.c, None, nxt)


def test_context_setters_refuse():
    import ctypes as C
    import torch
    from paper_2410_12513_b200 import FirstError, lib
    from paper_2410_12513_b200.binding import AdaptersC, SamplingC
    shape = fi.ModelShape(2, 64, 2, 2, 32, 72, 32)  # ffn_dim 72: no multiple of 16
    ctx = _ctx(shape, False, 4, 8, fi.make_weights(shape, 1, False))
    L = lib()
    assert L.first_set_sampling_rows(ctx.h, C.byref(SamplingC())) == -1  # no draws
    seq = torch.zeros(4, dtype=torch.int32, device="cuda")
    dev, _ = _adapters(shape, 2, 8, 1, False)
    with pytest.raises(FirstError) as e:
        ctx.set_adapters(dev, seq)
    assert e.value.status == -3
    del dev["gate_up"]
    ctx.set_adapters(dev, seq)
    ok = AdaptersC(2, 8, None, seq.data_ptr())
    assert L.first_set_adapters(ctx.h, C.byref(ok)) == 0
    for n, r, s, rc in ((0, 8, seq.data_ptr(), -1), (2, 0, seq.data_ptr(), -1), (2, 8, None, -1), (2, 12, seq.data_ptr(), -3), (2, 256, seq.data_ptr(), -3)):
        assert L.first_set_adapters(ctx.h, C.byref(AdaptersC(n, r, None, s))) == rc
    half = AdaptersC(2, 8, None, seq.data_ptr())
    arr = (C.c_void_p * 2)(dev["o"][0][0].data_ptr(), dev["o"][1][0].data_ptr())
    half.o_a = C.cast(arr, C.POINTER(C.c_void_p))
    assert L.first_set_adapters(ctx.h, C.byref(half)) == -1  # a without b
    odd = (C.c_void_p * 2)(dev["o"][0][0].data_ptr() + 4, None)
    half.o_a, half.o_b = C.cast(odd, C.POINTER(C.c_void_p)), C.cast(odd, C.POINTER(C.c_void_p))
    assert L.first_set_adapters(ctx.h, C.byref(half)) == -3
    with pytest.raises(ValueError):
        ctx.set_rope(np.ones(5))
    for bad in (math.nan, math.inf):
        with pytest.raises(FirstError):
            ctx.set_rope(np.full(16, bad))
        with pytest.raises(FirstError):
            ctx.set_rope(np.ones(16), bad)
    ctx.set_rope(None)
