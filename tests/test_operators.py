"""The operators around the step, without a GPU: rotary frequencies against an independent implementation, and what the
calls refuse (a refused call launches nothing and reads nothing, so any address will do)."""
import ctypes as C
import math

import numpy as np
import pytest

ARG, SHAPE, UNSUPPORTED, CAPACITY = -1, -2, -3, -4
P = 1 << 20  # a 16-byte aligned address that is never read


def _L():
    from paper_2410_12513_b200 import lib
    return lib()


# ------------------------------------------------------------------ rotary frequencies
@pytest.mark.parametrize("rot,base", [(64, 10000.0), (128, 500000.0), (96, 10000.0), (2, 10000.0)])
@pytest.mark.parametrize("scaling,kw", [
    ("none", {}), ("linear", {"factor": 4.0}), ("linear", {"factor": 1.0}),
    ("llama3", {"factor": 32.0, "low": 1.0, "high": 4.0, "trained_len": 8192}),
    ("llama3", {"factor": 8.0, "low": 2.0, "high": 9.0, "trained_len": 4096}),
    ("yarn", {"factor": 16.0, "low": 1.0, "high": 32.0, "trained_len": 8192}),
    ("yarn", {"factor": 4.0, "low": 1.0, "high": 32.0, "trained_len": 32768})])
def test_rope_frequencies_against_transformers(rot, base, scaling, kw):
    torch = pytest.importorskip("torch")
    rope = pytest.importorskip("transformers.modeling_rope_utils")
    from transformers import LlamaConfig
    from paper_2410_12513_b200 import first_rope_freqs
    inv, factor = first_rope_freqs(rot, base, scaling, **kw)
    if scaling == "none":
        want, wf = base ** (-2.0 * np.arange(rot // 2) / rot), 1.0
    elif scaling == "linear":
        want, wf = base ** (-2.0 * np.arange(rot // 2) / rot) / kw["factor"], 1.0
    else:
        if scaling == "yarn" and rot == 2:
            pytest.skip("one pair: the other side's ramp has no second point")
        params = {"rope_type": scaling, "rope_theta": base, "factor": kw["factor"], "original_max_position_embeddings": kw["trained_len"]}
        if scaling == "llama3":
            params |= {"low_freq_factor": kw["low"], "high_freq_factor": kw["high"]}
        else:
            params |= {"beta_slow": kw["low"], "beta_fast": kw["high"]}
        cfg = LlamaConfig(hidden_size=rot, num_attention_heads=1, head_dim=rot, max_position_embeddings=kw["trained_len"] * int(kw["factor"]),
                          rope_parameters=params)
        want, wf = rope.ROPE_INIT_FUNCTIONS[scaling](cfg, torch.device("cpu"))
        want = want.double().numpy()
    # the other side works in 32 bits: a handful of roundings of 2^-24 each, its power among them (exponent up to
    # ln(base) = 13: 13 * 2^-24), and its blend
    assert np.abs(inv / want - 1).max() < 24 * 2.0 ** -24
    assert abs(factor - wf) < 1e-12


def test_rope_scaling_limits():
    from paper_2410_12513_b200 import first_rope_freqs
    f = 500000.0 ** (-np.arange(64) / 64.0)
    inv, _ = first_rope_freqs(128, 500000.0, "llama3", factor=32.0, low=1.0, high=4.0, trained_len=8192)
    turns = 8192 * f / (2 * math.pi)
    assert np.allclose(inv[turns >= 4], f[turns >= 4], rtol=1e-15) and np.allclose(inv[turns <= 1], f[turns <= 1] / 32, rtol=1e-15)
    assert (np.diff(inv) < 0).all()


def test_rope_frequencies_refuse():
    from paper_2410_12513_b200.binding import RopeSpecC
    L, out, fac = _L(), (C.c_double * 64)(), C.c_double()

    def call(**kw):
        d = {"rot_dim": 128, "scaling": 2, "base": 1e4, "factor": 8.0, "low": 1.0, "high": 4.0, "trained_len": 8192} | kw
        return L.first_rope_freqs(C.byref(RopeSpecC(*[d[n] for n, _ in RopeSpecC._fields_])), out, C.byref(fac))
    assert call() == 0
    for bad in ({"rot_dim": 0}, {"rot_dim": 3}, {"scaling": 4}, {"scaling": -1}, {"base": 0.0}, {"base": math.nan}, {"factor": 0.5},
                {"factor": math.inf}, {"low": 0.0}, {"high": 1.0}, {"trained_len": 0}, {"scaling": 3, "base": 1.0}):
        assert call(**bad) == ARG, bad
    assert L.first_rope_freqs(None, out, C.byref(fac)) == ARG
    from paper_2410_12513_b200 import first_rope_freqs
    with pytest.raises(ValueError):
        first_rope_freqs(64, 1e4, "other")


# ------------------------------------------------------------------ refusals
def test_rope_refuses():
    L = _L()

    def call(q=P, qt=512, qh=128, hq=4, k=P, kt=256, kh=128, hk=2, dt=1, T=10, hd=128, rot=128, pos=P, inv=P, il=0):
        return L.first_rope(q, qt, qh, hq, k, kt, kh, hk, dt, T, hd, rot, pos, inv, 1.0, il, None)
    assert call(T=0) == 0 and call(hq=0, hk=0, q=None, k=None) == 0
    for bad in ({"q": None}, {"k": None}, {"pos": None}, {"inv": None}, {"dt": 2}, {"T": -1}, {"hq": -1}, {"hk": -1}, {"hq": 70000, "qt": 1 << 24}):
        assert call(**bad) == ARG, bad
    for bad in ({"rot": 129}, {"rot": 130}, {"rot": 0}, {"hd": 0}, {"qh": 64}, {"qt": 128}, {"qt": 0}, {"qt": -512}, {"qh": -128}, {"kt": 255},
                {"hq": 1, "qt": 100}):
        assert call(**bad) == SHAPE, bad
    assert call(hd=65538, rot=2, hq=1, hk=0, qt=1 << 20) == UNSUPPORTED
    assert call(T=1 << 40, qt=512, hk=0) == CAPACITY
    # [heads][tokens][hd] order is fine, heads overlapping in it is not
    assert call(T=10, qt=128, qh=1279, hk=0) == SHAPE


def test_lora_refuses_sizes_that_32_bits_cannot_round_up():
    L = _L()
    for k, n in ((2 ** 31 - 8, 100), (2 ** 30 + 8, 100), (256, 2 ** 31 - 1), (256, 2 ** 30 + 1)):
        seg = (C.c_int32 * 2)(0, n)
        assert L.first_lora(P, 1, k, P, P, 1, None, P, 4, 8, 1, seg, 1, k, n, P, 0, n, None) == UNSUPPORTED


def test_rope_refuses_addresses_between_elements():
    L = _L()
    for dt, q, k in ((1, P + 1, P), (1, P, P + 3), (0, P + 2, P), (0, P, P + 6), (0, P + 1, P)):
        assert L.first_rope(q, 512, 128, 4, k, 256, 128, 2, dt, 10, 128, 128, P, P, 1.0, 0, None) == UNSUPPORTED


def test_empty_batches_need_no_addresses():
    """An empty tensor's address is NULL: a batch of no rows does nothing, whatever the addresses are."""
    L = _L()
    assert L.first_rope(None, 512, 128, 4, None, 256, 128, 2, 1, 0, 128, 128, None, None, 1.0, 0, None) == 0
    assert L.first_rope(None, 512, 128, 4, None, 0, 0, 0, 0, 0, 128, 64, None, P, 1.0, 1, None) == 0
    assert L.first_rope(None, 0, 0, 0, None, 0, 0, 0, 0, 7, 128, 64, None, None, 1.0, 1, None) == 0
    assert L.first_rope(None, 512, 128, 4, None, 256, 128, 2, 1, 0, 128, 129, None, None, 1.0, 0, None) == SHAPE  # other checks stay
    assert L.first_lora(None, 1, 256, P, P, 1, None, None, 4, 8, 1, (C.c_int32 * 2)(0, 100), 0, 256, 100, None, 0, 100, None) == 0
    assert L.first_sample(None, 100, 0, 100, None, None, None, None, None, None, None) == 0


def test_lora_refuses():
    L = _L()
    seg = lambda *v: (C.c_int32 * len(v))(*v)  # noqa: E731

    def call(x=P, xd=1, ldx=256, a=P, b=P, wd=1, ids=P, n=4, rank=8, S=1, sg=seg(0, 100), rows=3, k=256, f=100, y=P, yd=0, ldy=100):
        return L.first_lora(x, xd, ldx, a, b, wd, None, ids, n, rank, S, sg, rows, k, f, y, yd, ldy, None)
    assert call(rows=0) == 0 and call(n=0) == 0
    for bad in ({"x": None}, {"a": None}, {"b": None}, {"ids": None}, {"y": None}, {"sg": None}, {"xd": 2}, {"wd": -1}, {"yd": 7},
                {"rows": -1}, {"n": -1}, {"rank": 0}, {"k": 0}, {"f": 0}, {"S": 0}):
        assert call(**bad) == ARG, bad
    for bad in ({"ldx": 255}, {"ldy": 99}, {"sg": seg(1, 100)}, {"sg": seg(0, 96)}, {"S": 2, "sg": seg(0, 0, 100)}, {"S": 2, "sg": seg(0, 112, 100)}):
        assert call(**bad) == SHAPE, bad
    for bad in ({"rank": 12}, {"rank": 136}, {"k": 252}, {"S": 2, "sg": seg(0, 40, 100)}, {"S": 5, "sg": seg(0, 16, 32, 48, 64, 100)},
                {"x": P + 8}, {"a": P + 2}, {"b": P + 4}, {"ldx": 260}, {"xd": 0, "ldx": 257}, {"y": P + 2}, {"yd": 1, "y": P + 1}):
        assert call(**bad) == UNSUPPORTED, bad


def test_sample_refuses():
    L = _L()

    def call(lg=P, ld=100, B=3, V=100, u=P, tok=P):
        return L.first_sample(lg, ld, B, V, None, None, None, None, u, tok, None)
    assert call(B=0) == 0
    for bad in ({"lg": None}, {"u": None}, {"tok": None}, {"B": -1}, {"V": 0}):
        assert call(**bad) == ARG, bad
    assert call(ld=99) == SHAPE
    assert call(V=524289, ld=524289) == UNSUPPORTED


def test_context_calls_refuse_a_missing_context():
    L = _L()
    assert L.first_set_sampling_rows(None, None) == ARG
    assert L.first_set_adapters(None, None) == ARG
    assert L.first_set_rope(None, None, 1.0) == ARG


def test_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    import paper_2410_12513_b200 as lib
    h = torch.zeros(2, 16)
    with pytest.raises(TypeError):
        lib.first_sample(h, torch.zeros(2), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        lib.first_lora(h, torch.zeros(1, 8, 16), torch.zeros(1, 4, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4))
    with pytest.raises(TypeError):
        lib.first_rope(torch.zeros(2, 1, 16), None, torch.zeros(2, dtype=torch.int32), torch.zeros(8, dtype=torch.float64))
