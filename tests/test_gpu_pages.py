"""Sequences on paged 8-bit caches: the page manager (first_pages_*), decode steps over it, and a whole round of drafts --
append, attend, verify, trim -- against mirrors on the host and runs of the host oracle (B200 only)."""
import copy

import numpy as np
import pytest

import first_inputs as fi
import oracle
from harness import GpuKV, gpu_weights, logits_check, oracle_model
from test_gpu_cache8 import _tolerance, attention, nearest, values, verified

pytestmark = pytest.mark.gpu

ARG, SHAPE, CAPACITY, STATE = -1, -2, -4, -7


class Store:
    """One (sequence, layer)'s K or V on the host: numbers and scales page by page, by the definition of first_append8."""

    def __init__(self, H, page, hd, fmt):
        self.fmt, self.page, self.shape = fmt, page, (H, page, hd)
        self.b, self.s, self.n = [], [], 0

    def append(self, x):
        top = np.float32(1) / np.float32(127 if self.fmt == "int8" else 448)
        while len(x):
            i, lo = divmod(self.n, self.page)
            if lo == 0:
                self.b[i:], self.s[i:] = [np.zeros(self.shape, np.int8)], [np.zeros(self.shape[0], np.float32)]
            new, x = x[:self.page - lo].transpose(1, 0, 2), x[self.page - lo:]
            held = self.s[i] if lo else np.zeros_like(self.s[i])
            now = np.maximum(held, np.abs(new).max((1, 2)).astype(np.float32) * top)
            unit = np.where(now > 0, now, 1).astype(np.float64)[:, None, None]
            old = nearest(values(self.b[i][:, :lo], self.fmt) * held.astype(np.float64)[:, None, None] / unit, self.fmt)
            self.b[i] = self.b[i].copy()
            self.b[i][:, :lo] = np.where((now > held)[:, None, None], old, self.b[i][:, :lo])
            self.b[i][:, lo:lo + new.shape[1]] = nearest(new / unit, self.fmt)
            self.s[i] = now
            self.n += new.shape[1]

    def trim(self, n):
        self.n = n

    def rows(self):
        pos = np.arange(self.n)
        if not self.n:
            return np.zeros((0, self.shape[0], self.shape[2]))
        return values(np.stack(self.b)[pos // self.page, :, pos % self.page], self.fmt) * np.stack(self.s)[pos // self.page].astype(np.float64)[..., None]


def _caches(shape, n_pages, page, fmt):
    import torch
    from paper_2410_12513_b200 import Cache8
    dt = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}[fmt]
    out = []
    for n in n_pages:
        kv = [torch.randint(-128, 128, (n, shape.n_kv_heads, page, shape.head_dim), dtype=torch.int8, device="cuda").view(dt) for _ in "kv"]
        sc = [torch.full((n, shape.n_kv_heads), float("nan"), device="cuda") for _ in "kv"]
        out.append(Cache8(*kv, *sc))
    return out


def _read(mgr, l, slot, n):
    """Values of a sequence's first n tokens in layer l, [n][heads][hd] float32."""
    import torch
    from paper_2410_12513_b200 import first_read8
    cache, table, _ = mgr.layer(l)
    H, hd = cache.c.n_kv_heads, cache.c.head_dim
    k, v = (torch.zeros(n, H, hd, device="cuda") for _ in "kv")
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    first_read8(cache, table[slot:slot + 1].contiguous(), cu[:1].contiguous(), k, v, cu=cu, max_rows=n)
    return k.cpu().numpy(), v.cpu().numpy()


def _ctx(shape=fi.TINY, bf16=False, batch=16, tokens=512, seed=3):
    from paper_2410_12513_b200 import FirstContext
    w = fi.make_weights(shape, seed, bf16)
    return FirstContext(shape, 1 if bf16 else 0, batch, tokens, gpu_weights(w)), w


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_a_schedule_of_forks_trims_and_compactions(fmt):
    """Random joins, appends of a few tokens, attention over them, forks, trims (after verification), leaves and compactions:
    every sequence keeps exactly its own tokens, and no page is lost."""
    import torch
    from paper_2410_12513_b200 import FirstError, FirstPages, first_append8, first_attn8, first_verify
    shape, page, B, V = fi.TINY, 16, 6, 40
    L, H, hd, G = shape.n_layers, shape.n_kv_heads, shape.head_dim, shape.n_q_heads // shape.n_kv_heads
    ctx, _ = _ctx()
    n_pages = [34, 25, 40, 34]
    mgr = FirstPages(ctx, B, 9, _caches(shape, n_pages, page, fmt))
    rng = np.random.default_rng(11)
    seqs = {}  # slot -> (mask, stores[l] = (k, v), tokens)
    refused = forks = compactions = 0
    for step in range(140):
        what = rng.choice(["join", "fork", "leave", "compact", "drafts", "drafts", "drafts", "drafts"])
        if what == "join" or not seqs:
            try:
                mask = (rng.random(L) < 0.7).astype(np.uint8)
                slot = mgr.join(mask)
            except FirstError as e:
                assert e.status == CAPACITY and len(seqs) == B
                continue
            assert slot not in seqs
            seqs[slot] = (mask, [[Store(H, page, hd, fmt) for _ in "kv"] for _ in range(L)], 0)
        elif what == "fork":
            src = int(rng.choice(list(seqs)))
            try:
                slot = mgr.fork(src)
            except FirstError as e:
                assert e.status == CAPACITY and len(seqs) == B
                continue
            seqs[slot] = copy.deepcopy(seqs[src])
            forks += 1
        elif what == "leave":
            slot = int(rng.choice(list(seqs)))
            mgr.leave(slot)
            del seqs[slot]
        elif what == "compact":
            mgr.compact()
            held, top, live = mgr.stats()
            assert (top == held - 1).all() and live == len(seqs)
            compactions += 1
        else:  # a sequence (or all) gains k tokens, attends over them, and keeps some
            alone = rng.random() < 0.5
            who = [int(rng.choice(list(seqs)))] if alone else sorted(seqs)
            k = int(rng.integers(1, 8))
            try:
                mgr.extend(k, who[0] if alone else -1)
            except FirstError as e:
                assert e.status == CAPACITY
                refused += 1
                big = max(seqs, key=lambda s: seqs[s][2])  # make room
                mgr.leave(big)
                del seqs[big]
                continue
            mgr.commit()
            cu = np.zeros(B + 1, np.int32)
            for b in range(B):
                cu[b + 1] = cu[b] + (k if b in who else 0)
            rows = int(cu[-1])
            cud = torch.from_numpy(cu).cuda()
            for l in range(L):
                # rows of sequences that skip the layer are not brought along
                here = np.array([b for b in who if seqs[b][0][l]], int)
                cul = np.zeros(B + 1, np.int32)
                for b in range(B):
                    cul[b + 1] = cul[b] + (k if b in here else 0)
                n = int(cul[-1])
                if n == 0:
                    continue
                cache, table, ln = mgr.layer(l)
                assert (ln.cpu().numpy()[here] == [seqs[b][2] for b in here]).all()
                x = [rng.standard_normal((n, H, hd)).astype(np.float32) * 1.5 ** (step % 5) for _ in "kv"]
                q = rng.standard_normal((n, H * G, hd)).astype(np.float32)
                cd = torch.from_numpy(cul).cuda()
                first_append8(*[torch.from_numpy(t).cuda() for t in x], cache, table, ln, cu_new=cd, max_new=k)
                out = torch.empty(n, H * G, hd, device="cuda")
                first_attn8(torch.from_numpy(q).cuda(), cache, table, ln, out, cu_new=cd, max_new=k)
                got = out.double().cpu().numpy()
                for b in here:
                    for w in range(2):
                        seqs[b][1][l][w].append(x[w][cul[b]:cul[b + 1]].astype(np.float64))
                    if step % 4 == 0:
                        st = seqs[b][1][l]
                        fake = type("C", (), {"b": [np.stack(t.b) for t in st], "s": [np.stack(t.s) for t in st], "page": page, "fmt": fmt})
                        want, size, peak = attention(fake, q[cul[b]:cul[b + 1]].astype(np.float64), np.arange(len(st[0].b)), st[0].n, k, hd ** -0.5)
                        assert (np.abs(got[cul[b]:cul[b + 1]] - want) <= _tolerance(want, size, peak, st[0].n, "f32")).all()
            # verification of the last k - 1 of them
            target = rng.standard_normal((B, k, V)).astype(np.float32)
            drafted = np.stack([target[:, i].argmax(-1) for i in range(k - 1)], 1).astype(np.int32) if k > 1 else np.zeros((B, 0), np.int32)
            u, w = rng.random((B, k - 1)).astype(np.float32), rng.random(B).astype(np.float32)
            tok, acc = torch.empty(B, k, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
            dev = [torch.from_numpy(np.ascontiguousarray(t)).cuda() for t in (target, drafted, u, w)]
            first_verify(dev[0], dev[1], dev[2], dev[3], tok, acc)
            for b in who:
                want, a, _ = verified(target[b], None, drafted[b].tolist(), 1.0, u[b].tolist(), float(w[b]), False)
                assert int(acc[b]) == a and tok[b].tolist() == want
                keep = seqs[b][2] + 1 + a
                for l in range(L):
                    for t in seqs[b][1][l]:
                        t.trim(keep if seqs[b][0][l] else 0)
                mgr.trim(b, keep)
                seqs[b] = (seqs[b][0], seqs[b][1], keep)
                assert mgr.tokens(b) == keep
        mgr.commit()
        if step % 7 == 0 or what == "compact":
            for b, (mask, stores, n) in seqs.items():
                for l in range(L):
                    _, table, ln = mgr.layer(l)
                    assert int(ln[b]) == (n if mask[l] else 0)
                    if mask[l] and n:
                        for got, st in zip(_read(mgr, l, b, n), stores[l]):
                            assert np.array_equal(got, st.rows().astype(np.float32)), (step, what, b, l)
    assert forks > 3 and compactions > 3
    for b in list(seqs):
        mgr.leave(b)
    mgr.commit()
    held, top, live = mgr.stats()
    assert (held == 0).all() and (top == -1).all() and live == 0
    mgr.close()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("bf16", [False, True])
def test_steps_over_pages_against_the_oracle(bf16, fmt):
    """Prompts from first_prefill, imported; decode steps with kv=None, forks with other tokens, a trim, a leave and a
    compaction in between.  Before every step the oracle's cache takes the values that the pages hold."""
    import torch
    from paper_2410_12513_b200 import FirstPages
    shape = fi.ModelShape(3, 256, 8, 2, 64, 512, 1000, 500000.0) if bf16 else fi.TINY_GQA
    ctx, w = _ctx(shape, bf16, batch=32, tokens=200, seed=9)
    om = oracle_model(shape, w)
    L, page, B = shape.n_layers, 16, 5
    lens = [37, 16, 1, 60]
    prompts = [fi.tokens(shape, n, 9, f"p{i}") for i, n in enumerate(lens)]
    masks = np.array([[1] * L, [1, 0] + [1] * (L - 2), [0] + [1] * (L - 1), [1, 1] + [0] * (L - 2)], np.uint8)
    stage = GpuKV(shape, [n + 3 for n in lens], bf16)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    ctx.prefill(torch.from_numpy(np.concatenate(prompts).astype(np.int32)).cuda(), cu, stage.c)
    mgr = FirstPages(ctx, B, 12, _caches(shape, [40] * L, page, fmt))
    ctx.set_pages(mgr)
    slots = [mgr.join(masks[b], stage.c, b, lens[b]) for b in range(4)]
    mgr.commit()
    live = {slots[b]: (masks[b], lens[b]) for b in range(4)}
    for b in range(4):  # the import: half a step of 8 bits of the page's largest
        for l in range(L):
            if masks[b][l]:
                for got, want in zip(_read(mgr, l, slots[b], lens[b]), stage.rows_host(l, b)):
                    want = want[:lens[b]].reshape(got.shape)
                    top = np.abs(want).max()
                    assert (np.abs(got - want) <= (top / 127 * 0.501 if fmt == "int8" else 2.0 ** -4 * np.abs(want) + top / 448 * 2.0 ** -10)).all()
    logits = torch.empty(B, shape.vocab, device="cuda")
    nxt = torch.empty(B, dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(4)
    worst = 0.0
    for step in range(24):
        if step == 6:
            live[mgr.fork(slots[0])] = live[slots[0]]
        if step == 10:  # two tokens are taken back
            mgr.trim(slots[3], live[slots[3]][1] - 2)
            live[slots[3]] = (live[slots[3]][0], live[slots[3]][1] - 2)
        if step == 13:
            mgr.leave(slots[1])
            del live[slots[1]]
        if step == 15:
            mgr.compact()
            held, top, _ = mgr.stats()
            assert (top == held - 1).all()
        mgr.extend()
        mgr.commit()
        toks = np.zeros(B, np.int32)
        refs = {}
        for s, (mask, n) in live.items():
            okv = oracle.OracleKV(om.shape, [n + 1])
            for l in range(L):
                if mask[l]:
                    kr, vr = okv.rows(l, 0)
                    for dst, src in zip((kr, vr), _read(mgr, l, s, n)):
                        dst[:n] = src.reshape(n, -1)
                    okv.len[l, 0] = n
            okv.pos[0] = n
            toks[s] = rng.integers(0, shape.vocab)
            refs[s] = oracle.decode_step(om, toks[s:s + 1], mask[None], okv)[0]
        ctx.decode_step(torch.from_numpy(toks).cuda(), None, logits, nxt)
        assert ctx.device_flags() == 0
        got = logits.cpu().numpy()
        for s in list(live):
            # the new token's key and value, and earlier ones rounded anew, are off by up to half a step of 8 bits: held to the bar of
            # bfloat16 caches
            err, _ = logits_check(got[s:s + 1], refs[s][None])
            worst = max(worst, float(err.max()))
            assert err.max() <= 2e-2, (step, s, err)
            assert int(nxt[s]) == int(got[s].argmax())
            live[s] = (live[s][0], live[s][1] + 1)
        for l in range(L):
            ln = mgr.layer(l)[2].cpu().numpy()
            for s, (mask, n) in live.items():
                assert ln[s] == (n if mask[l] else 0)
    assert ctx.graph_count() < 12  # commits that change page lists alone find their recorded step again
    ctx.set_pages(None)
    mgr.close()


def test_a_step_without_room():
    """A step whose sequence was not extended: the token is not stored, the flag says so, its length stays."""
    import torch
    from paper_2410_12513_b200 import FirstError, FirstPages
    ctx, _ = _ctx()
    shape = fi.TINY
    mgr = FirstPages(ctx, 2, 4, _caches(shape, [6] * 4, 16, "int8"))
    ctx.set_pages(mgr)
    s = mgr.join(np.ones(4, np.uint8))
    mgr.commit()
    toks, logits = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.empty(2, shape.vocab, device="cuda")
    ctx.decode_step(toks, None, logits)
    assert ctx.device_flags() == 1 and (mgr.layer(0)[2].cpu() == 0).all()
    mgr.extend()
    mgr.commit()
    ctx.decode_step(toks, None, logits)
    assert ctx.device_flags() == 0 and int(mgr.layer(0)[2][s]) == 1
    assert torch.isfinite(logits[s]).all()
    ctx.set_mask_host(np.ones((1, 4), np.uint8))  # another plan: not the manager's
    with pytest.raises(FirstError) as e:
        ctx.decode_step(toks[:1].contiguous(), None, logits[:1])
    assert e.value.status == STATE
    ctx.set_pages(None)
    with pytest.raises(FirstError) as e:
        ctx.decode_step(toks, None, logits)
    assert e.value.status == ARG
    mgr.close()


def test_the_manager_refuses():
    import torch
    from paper_2410_12513_b200 import FirstError, FirstPages
    ctx, _ = _ctx()
    shape = fi.TINY

    def status(fn, *a):
        with pytest.raises(FirstError) as e:
            fn(*a)
        return e.value.status
    caches = _caches(shape, [3, 3, 3, 3], 16, "int8")
    assert status(FirstPages, ctx, 17, 4, caches) == CAPACITY
    assert status(FirstPages, ctx, 0, 4, caches) == ARG
    assert status(FirstPages, ctx, 4, 0, caches) == ARG
    assert status(FirstPages, ctx, 4, 70000, caches) == CAPACITY
    other = fi.ModelShape(4, 256, 4, 2, 64, 688, 1024)
    assert status(FirstPages, ctx, 4, 4, _caches(other, [3] * 4, 16, "int8")) == SHAPE
    assert status(FirstPages, ctx, 4, 4, caches[:3] + _caches(shape, [3], 32, "int8")) == SHAPE
    assert status(FirstPages, ctx, 4, 4, caches[:3] + _caches(shape, [3], 16, "e4m3")) == SHAPE
    with pytest.raises(ValueError):
        FirstPages(ctx, 4, 4, caches[:3])
    mgr = FirstPages(ctx, 3, 2, caches)
    a = mgr.join([1, 1, 0, 1])
    assert status(mgr.join, [2, 0, 0, 0]) == ARG
    assert status(mgr.leave, 2) == STATE and status(mgr.fork, 1) == STATE and status(mgr.trim, 1, 0) == STATE
    assert status(mgr.leave, 3) == ARG and status(mgr.extend, 1, 3) == ARG and status(mgr.extend, -1, a) == ARG
    assert status(mgr.extend, 33, a) == CAPACITY  # more than max_pages
    assert status(mgr.trim, a, 1) == ARG
    mgr.extend(20, a)
    assert status(mgr.fork, a) == STATE and status(mgr.trim, a, 0) == STATE  # those tokens are not there yet
    mgr.commit()
    b, c = mgr.fork(a), mgr.fork(a)
    assert status(mgr.fork, a) == CAPACITY and status(mgr.join, [0, 0, 0, 0]) == CAPACITY
    # one page a layer is left: one of the three may copy their shared last page, no more, and nothing is taken by a refused call
    before = mgr.stats()[0].tolist()
    assert before == [2, 2, 0, 2]
    assert status(mgr.extend, 1, -1) == CAPACITY
    assert mgr.stats()[0].tolist() == before and mgr.tokens(b) == 20
    mgr.extend(1, b)
    assert mgr.stats()[0].tolist() == [3, 3, 0, 3]
    mgr.leave(c)
    mgr.extend(1, -1)  # (everybody's last page is its own by now)
    mgr.commit()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        assert status(mgr.commit) == STATE
        torch.empty(1, device="cuda").zero_()
    mgr.close()


def test_imports_wait_for_the_commit():
    import torch
    from paper_2410_12513_b200 import FirstError, FirstPages
    ctx, _ = _ctx()
    shape = fi.TINY
    stage = GpuKV(shape, [40, 40], False)
    for l in range(shape.n_layers):
        stage.k[l].normal_()
        stage.v[l].normal_()
    mgr = FirstPages(ctx, 4, 4, _caches(shape, [12] * 4, 16, "e4m3"))
    s = mgr.join([1, 1, 1, 1], stage.c, 1, 33)
    for fn in (mgr.fork, lambda x: mgr.trim(x, 3)):
        with pytest.raises(FirstError) as e:
            fn(s)
        assert e.value.status == STATE
    gone = mgr.join([1, 0, 1, 0], stage.c, 0, 40)
    mgr.leave(gone)  # its import is forgotten
    mgr.commit()
    f = mgr.fork(s)
    mgr.extend(3, f)
    with pytest.raises(FirstError):
        mgr.fork(f)
    mgr.leave(s)  # the copy of the shared page is still to be made, from a page that nobody holds
    t = mgr.join([1, 1, 1, 1])
    mgr.extend(40, t)
    mgr.commit()
    for l in range(4):
        k, v = _read(mgr, l, f, 33)
        for got, want in ((k, stage.k[l]), (v, stage.v[l])):
            want = want[:, 40:73].permute(1, 0, 2).cpu().numpy()
            assert (np.abs(got - want) <= 2.0 ** -4 * np.abs(want) + np.abs(want).max() / 448 * 2.0 ** -10).all()
    # a fork of a fork before anything is copied
    g = mgr.fork(f)
    h = mgr.fork(g)
    mgr.extend(1, g)
    mgr.extend(1, h)
    mgr.commit()
    for l in range(4):
        for a, b in zip(_read(mgr, l, f, 33), _read(mgr, l, h, 33)):
            assert np.array_equal(a, b)
    mgr.close()


def test_a_copy_that_nobody_wants_gives_its_source_back():
    """A fork takes a page of its own, then both leave before the copy was made: all pages can be had again."""
    from paper_2410_12513_b200 import FirstPages
    ctx, _ = _ctx()
    L = fi.TINY.n_layers
    mgr = FirstPages(ctx, 3, 4, _caches(fi.TINY, [4] * L, 16, "int8"))
    a = mgr.join([1] * L)
    mgr.extend(17, a)
    mgr.commit()
    b = mgr.fork(a)
    mgr.commit()
    mgr.extend(1, b)
    mgr.leave(a)
    mgr.leave(b)
    mgr.extend(4 * 16, mgr.join([1] * L))
    mgr.commit()
    assert (mgr.stats()[0] == 4).all()


def test_pages_of_another_model_are_refused():
    import dataclasses
    from paper_2410_12513_b200 import FirstError, FirstPages
    shape = fi.TINY
    ctx, _ = _ctx()
    mgr = FirstPages(ctx, 3, 2, _caches(shape, [3] * shape.n_layers, 16, "int8"))
    for n in (shape.n_layers - 1, shape.n_layers + 2):  # fewer and more layers than there are caches
        other, _ = _ctx(dataclasses.replace(shape, n_layers=n))
        with pytest.raises(FirstError) as e:
            other.set_pages(mgr)
        assert e.value.status == SHAPE
    ctx.set_pages(mgr)
    mgr.close()
