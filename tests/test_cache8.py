"""What the calls on paged 8-bit caches and the verification of drafts refuse, without a GPU (a refused call launches
nothing and reads nothing, so any address will do)."""
import ctypes as C

import pytest

OK, ARG, SHAPE, UNSUPPORTED, CAPACITY = 0, -1, -2, -3, -4
P = 1 << 20  # a 16-byte aligned address that is never read


def _L():
    from paper_2410_12513_b200 import lib
    return lib()


def _cache(**kw):
    from paper_2410_12513_b200.binding import Cache8C
    d = {"format": 0, "n_pages": 10, "n_kv_heads": 2, "page": 32, "head_dim": 64, "k": P, "v": P, "k_scale": P, "v_scale": P} | kw
    return C.byref(Cache8C(*[d[n] for n, _ in Cache8C._fields_]))


CACHES = [({"format": 2}, ARG), ({"format": -1}, ARG), ({"n_pages": -1}, ARG), ({"n_kv_heads": 0}, ARG), ({"k": None}, ARG),
          ({"v": None}, ARG), ({"k_scale": None}, ARG), ({"v_scale": None}, ARG), ({"page": 8}, UNSUPPORTED),
          ({"page": 48}, UNSUPPORTED), ({"page": 256}, UNSUPPORTED), ({"head_dim": 96}, UNSUPPORTED),
          ({"head_dim": 256}, UNSUPPORTED), ({"n_kv_heads": 1025}, UNSUPPORTED), ({"k": P + 8}, UNSUPPORTED),
          ({"v": P + 1}, UNSUPPORTED), ({"k_scale": P + 2}, UNSUPPORTED), ({"v_scale": P + 1}, UNSUPPORTED)]


def _append(c=None, k=P, kt=128, kh=64, v=P, vt=128, vh=64, dt=1, cu=None, total=3, pages=P, width=4, ln=P, B=3, new=1):
    return _L().first_append8(c or _cache(), k, kt, kh, v, vt, vh, dt, cu, total, pages, width, ln, B, new, None, None)


def _read(c=None, k=P, kt=128, kh=64, v=P, vt=128, vh=64, dt=1, cu=None, total=3, pages=P, width=4, ln=P, B=3, new=1):
    return _L().first_read8(c or _cache(), pages, width, ln, cu, B, total, new, k, kt, kh, v, vt, vh, dt, None, None)


def _attn(c=None, q=P, qt=256, qh=64, hq=4, dt=1, cu=None, total=3, pages=P, width=4, ln=P, B=3, new=1, out=P, ot=256, oh=64, ws=None, room=0):
    return _L().first_attn8(c or _cache(), q, qt, qh, hq, dt, 0.1, cu, total, pages, width, ln, B, new, out, ot, oh, ws, room, None, None)


@pytest.mark.parametrize("call", [_append, _read, _attn])
def test_caches_and_batches_are_checked(call):
    for kw, want in CACHES:
        assert call(c=_cache(**kw)) == want, kw
    assert _L().first_append8(None, P, 0, 0, P, 0, 0, 1, None, 0, P, 1, P, 0, 1, None, None) == ARG
    for kw in ({"B": -1}, {"total": -1}, {"width": -1}, {"new": -1}, {"pages": None}, {"ln": None}, {"dt": 2}, {"dt": -1}):
        assert call(**{"cu": P, **kw}) == ARG, kw
    assert call(total=4) == SHAPE  # one row a sequence, where there is no table of rows
    assert call(width=1 << 26) == CAPACITY
    for kw in ({"B": 0, "total": 0}, {"cu": P, "total": 0}, {"new": 0}):
        assert call(**kw) == OK, kw
    assert call(c=_cache(n_pages=0, k=None, v=None, k_scale=None, v_scale=None), B=0, total=0) == OK


def test_append_and_read_refuse():
    for call in (_append, _read):
        for kw in ({"k": None}, {"v": None}):
            assert call(**kw) == ARG, kw
        for kw in ({"kt": -128}, {"kh": -64}, {"vt": -1}, {"vh": -1}):
            assert call(**kw) == SHAPE, kw
        for kw in ({"k": P + 1}, {"v": P + 1}, {"dt": 0, "k": P + 2}, {"dt": 0, "v": P + 6}):
            assert call(**kw) == UNSUPPORTED, kw
    for kw in ({"kt": 127}, {"kh": 63}, {"vt": 64}, {"kt": 64, "kh": 191}):  # rows that are written do not overlap
        assert _read(**kw) == SHAPE, kw
    assert _append(cu=P, total=1 << 24, new=1 << 24, c=_cache(page=16)) == CAPACITY
    assert _read(B=70000, total=70000) == CAPACITY


def test_attention_refuses():
    for kw in ({"q": None}, {"out": None}, {"hq": 0}, {"hq": -4}, {"ws": P, "room": -1}):
        assert _attn(**kw) == ARG, kw
    for kw in ({"hq": 5}, {"qt": -256}, {"qh": -64}, {"ot": 255}, {"oh": 63}, {"ot": 0}):
        assert _attn(**kw) == SHAPE, kw
    for kw in ({"q": P + 1}, {"out": P + 1}, {"dt": 0, "q": P + 2}, {"dt": 0, "out": P + 2}, {"ws": P + 2, "room": 64}):
        assert _attn(**kw) == UNSUPPORTED, kw
    assert _attn(cu=P, total=1 << 20, new=1 << 20) == CAPACITY


def test_copies_refuse():
    L = _L()
    from paper_2410_12513_b200.binding import Cache8C
    one = [0, 10, 2, 32, 64, P, P, P, P]

    def call(layers=((),), n=None, moves=P, count=4, **kw):
        arr = (Cache8C * max(len(layers), 1))(*[Cache8C(*one) for _ in layers])
        for i, kv in enumerate(layers):
            for name, value in kv:
                setattr(arr[i], name, value)
        return L.first_copy_pages(C.byref(arr), len(layers) if n is None else n, moves, count, None, None)
    assert call(count=0) == OK and call(count=0, moves=None) == OK
    assert call(n=0) == ARG and call(moves=None) == ARG and call(count=-1) == ARG
    assert L.first_copy_pages(None, 1, P, 1, None, None) == ARG
    for name, value in (("format", 1), ("n_kv_heads", 4), ("page", 64), ("head_dim", 128)):  # layers that differ
        assert call(layers=((), ((name, value),))) == SHAPE, name
    assert call(layers=((), (("page", 24),))) == UNSUPPORTED
    assert call(layers=((),) * 97) == UNSUPPORTED
    assert call(count=1 << 40) == CAPACITY


def test_verify_refuses():
    L = _L()

    def call(target=P, ts=4000, tr=1000, draft=P, ds=3000, dr=1000, probs=0, drafted=P, B=2, n=3, V=1000, temp=None, u=P, w=P, tok=P, acc=P):
        return L.first_verify(target, ts, tr, draft, ds, dr, probs, drafted, B, n, V, temp, u, w, tok, acc, None)
    assert call(B=0) == OK and call(B=0, target=None, draft=None) == OK
    for kw in ({"B": -1}, {"n": -1}, {"V": 0}, {"target": None}, {"drafted": None}, {"u": None}, {"w": None}, {"tok": None}, {"acc": None}):
        assert call(**kw) == ARG, kw
    for kw in ({"ts": 999}, {"tr": 999}, {"ds": 999}, {"dr": 999}, {"ts": -4000}, {"dr": -1}):
        assert call(**kw) == SHAPE, kw
    for kw in ({"n": 33}, {"V": 524289}, {"target": P + 2}, {"draft": P + 1}):
        assert call(**kw) == UNSUPPORTED, kw
