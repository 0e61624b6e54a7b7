"""Page managers given caches, plans and imports that do not fit them (B200 only)."""
import numpy as np
import pytest

import first_inputs as fi
from test_gpu_pages import ARG, STATE, _caches, _ctx

pytestmark = pytest.mark.gpu


def test_layers_that_share_memory_are_refused():
    """Each layer hands out page ids of its own: two layers over one memory would overwrite each other."""
    import torch
    from paper_2410_12513_b200 import Cache8, FirstError, FirstPages
    ctx, _ = _ctx()
    shape = fi.TINY
    L = shape.n_layers
    own = _caches(shape, [3] * L, 16, "int8")

    def status(caches):
        with pytest.raises(FirstError) as e:
            FirstPages(ctx, 2, 3, caches)
        return e.value.status
    assert status([own[0]] * L) == ARG
    assert status(own[:3] + [own[1]]) == ARG
    a, b = own[0], own[3]
    for names in ({"k": a.k}, {"v": a.v}, {"k": a.v}, {"k_scale": a.k_scale}, {"v_scale": a.k_scale}, {"v": b.k}, {"v_scale": b.k_scale}):
        kw = {"k": b.k, "v": b.v, "k_scale": b.k_scale, "v_scale": b.v_scale} | names
        assert status(own[:3] + [Cache8(**kw)]) == ARG, list(names)
    # one memory cut in parts: side by side it is fine, by a page less it is not
    pool = torch.zeros(2 * L * 3 + 1, *a.k.shape[1:], dtype=torch.int8, device="cuda")
    scales = torch.zeros(2 * L * 3, shape.n_kv_heads, device="cuda")
    parts = [Cache8(pool[6 * l:6 * l + 3], pool[6 * l + 3:6 * l + 6], scales[6 * l:6 * l + 3], scales[6 * l + 3:6 * l + 6]) for l in range(L)]
    FirstPages(ctx, 2, 3, parts).close()
    over = Cache8(pool[6 * L - 7:6 * L - 4], pool[6 * L - 3:6 * L], scales[6 * L - 6:6 * L - 3], scales[6 * L - 3:])
    assert status(parts[:3] + [over]) == ARG
    none = torch.zeros(0, *a.k.shape[1:], dtype=torch.int8, device="cuda")  # (a layer that nobody keeps has no pages)
    FirstPages(ctx, 2, 3, own[:3] + [Cache8(none, none, scales[:0], scales[:0])]).close()


def test_a_step_asks_for_the_managers_own_plan():
    """Another mask of as many rows, a prompt phase, another manager's commit: the step over pages waits for a commit again."""
    import torch
    from harness import GpuKV
    from paper_2410_12513_b200 import FirstError, FirstPages
    ctx, _ = _ctx()
    shape = fi.TINY
    L = shape.n_layers
    mgr, other = (FirstPages(ctx, 2, 4, _caches(shape, [6] * L, 16, "int8")) for _ in "12")
    ctx.set_pages(mgr)
    s = mgr.join([1, 0, 1, 1])
    toks, logits = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.empty(2, shape.vocab, device="cuda")

    def steps(n):
        mgr.extend()
        mgr.commit()
        ctx.decode_step(toks, None, logits)
        assert ctx.device_flags() == 0
        assert [int(mgr.layer(l)[2][s]) for l in range(L)] == [n, 0, n, n]

    def refused():
        with pytest.raises(FirstError) as e:
            ctx.decode_step(toks, None, logits)
        assert e.value.status == STATE
    refused()
    steps(1)
    ctx.set_mask_host(np.ones((2, L), np.uint8))
    refused()
    mgr.commit()
    ctx.set_mask(torch.ones(2, L, dtype=torch.uint8, device="cuda"))
    refused()
    steps(2)
    stage = GpuKV(shape, [8], False)
    ctx.prefill(toks, np.array([0, 2], np.int32), stage.c)
    refused()
    steps(3)
    other.join([1] * L)
    other.commit()
    refused()
    steps(4)
    mgr.compact()
    steps(5)
    ctx2, _ = _ctx()
    with pytest.raises(FirstError) as e:
        ctx2.set_pages(mgr)
    assert e.value.status == ARG
    ctx.set_pages(None)
    mgr.close()
    other.close()


def test_imports_of_more_than_a_slab_holds():
    """The lengths of slabs are on the device: an import beyond one is left out and flagged, whoever the neighbour is; others arrive."""
    from harness import GpuKV
    from paper_2410_12513_b200 import FirstPages
    from test_gpu_pages import _read
    ctx, _ = _ctx()
    shape = fi.TINY
    L = shape.n_layers
    stage = GpuKV(shape, [40, 20, 30], False)
    for l in range(L):
        stage.k[l].normal_()
        stage.v[l].normal_()
    for seq, n, bad in ((0, 40, False), (0, 41, True), (1, 21, True), (1, 20, False), (2, 31, True), (2, 90, True), (2, 30, False)):
        caches = _caches(shape, [12] * L, 16, "int8")
        for c in caches:
            c.k.zero_(), c.v.zero_(), c.k_scale.fill_(2.0), c.v_scale.fill_(2.0)
        mgr = FirstPages(ctx, 2, 6, caches)
        if bad:  # (another sequence is not touched by it)
            mgr.join([1] * L, stage.c, seq, n)
        s = mgr.join([1] * L, stage.c, 0, 17)
        good = s if bad else mgr.join([1] * L, stage.c, seq, n)
        mgr.commit()
        assert ctx.device_flags() == (32 if bad else 0), (seq, n)
        o, m = (0, 17) if bad else (int(stage.off[seq]), n)
        for l in range(L):
            for got, want in zip(_read(mgr, l, good, m), (stage.k[l], stage.v[l])):
                want = want[:, o:o + m].permute(1, 0, 2).cpu().numpy()
                assert np.abs(got - want).max() <= np.abs(want).max() / 127 * 0.501
            if bad:
                assert (caches[l].k_scale == 2.0).sum() == 10 * shape.n_kv_heads  # (the good one's two pages alone)
        mgr.close()
    mgr = FirstPages(ctx, 2, 6, _caches(shape, [12] * L, 16, "int8"))
    for seq in (-1, 3):
        with pytest.raises(ValueError):
            mgr.join([1] * L, stage.c, seq, 3)
    assert mgr.stats()[2] == 0
    mgr.close()


@pytest.mark.parametrize("commit", ["commit", "compact"])
def test_a_source_lives_until_its_import(commit):
    """The cache that a sequence joins from is held on to until the commit has read it, and no longer."""
    import gc
    import weakref

    import torch
    from harness import GpuKV
    from paper_2410_12513_b200 import FirstPages
    from test_gpu_pages import _read
    ctx, _ = _ctx()
    shape = fi.TINY
    L = shape.n_layers
    mgr = FirstPages(ctx, 2, 6, _caches(shape, [12] * L, 16, "int8"))
    stage = GpuKV(shape, [300], False)
    for l in range(L):
        stage.k[l].fill_(0.5)
        stage.v[l].fill_(0.25)
    size, ref = stage.k[0].shape, weakref.ref(stage.c)
    s = mgr.join([1] * L, stage.c, 0, 40)
    del stage
    gc.collect()
    others = [torch.full(size, 9.0, device="cuda") for _ in range(4 * L)]  # (memory that is given back is handed out again)
    getattr(mgr, commit)()
    for l in range(L):
        k, v = _read(mgr, l, s, 40)
        assert np.allclose(k, 0.5, rtol=1e-6) and np.allclose(v, 0.25, rtol=1e-6)
    gc.collect()
    assert ref() is None and len(others) == 4 * L
    mgr.close()
