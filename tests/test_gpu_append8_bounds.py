"""Appending to 8-bit pages at the ends of float32 (B200 only)."""
import numpy as np
import pytest

from test_gpu_cache8 import Cache, _codes, _dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponent", [-99.0, -100.0, -100.3, -105.0, -112.7, -120.5, -122.6, -123.0, -126.0, 110.0, 118.4])
@pytest.mark.parametrize("fmt,top", [("int8", 127), ("e4m3", 448)])
def test_ties_of_tiny_and_huge_scales(fmt, top, exponent):
    """Values next to the middle between two numbers, at scales where that middle, or what a value differs by from it, is no normal float32."""
    import torch
    from paper_2410_12513_b200 import first_append8
    page, hd = 128, 128
    amax = np.float32(2.0 ** exponent * top)
    scale = np.float64(amax * (np.float32(1) / np.float32(top)))
    if fmt == "int8":
        middle = np.arange(0, 127) + 0.5
    else:
        v = _codes()
        middle = (v[1:] + v[:-1]) / 2
    x = (middle * scale).astype(np.float32)
    x = x[x < amax]
    x = np.concatenate([f for s in (1, -1) for f in (s * x, s * np.nextafter(x, np.float32(0)), s * np.nextafter(x, amax))] + [[amax]]).astype(np.float32)
    y = np.zeros((-(-x.size // hd), 1, hd), np.float32)
    y.reshape(-1)[:x.size] = x
    cache = Cache(0, 1, 1, page, hd, fmt)
    for w in range(2):
        cache.append(w, y.astype(np.float64), [0], 0)
    t = torch.from_numpy(y).cuda()
    first_append8(t, t, cache.c, _dev(np.zeros((1, 1), np.int32)), _dev(np.zeros(1, np.int32)), cu_new=_dev(np.array([0, len(y)], np.int32)), max_new=len(y))
    cache.check()
