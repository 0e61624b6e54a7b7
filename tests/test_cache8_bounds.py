"""What the calls on paged 8-bit caches and the verification of drafts refuse about addresses, without a GPU (a refused call
launches nothing and reads nothing, so any address will do)."""
import pytest

from test_cache8 import P, UNSUPPORTED, _L, _append, _attn, _cache, _read


@pytest.mark.parametrize("call", [_append, _read, _attn])
@pytest.mark.parametrize("name", ["pages", "ln", "cu"])
def test_tables_that_are_not_aligned(call, name):
    for off in (1, 2, 3):
        assert call(**{"cu": P, name: P + off}) == UNSUPPORTED


def test_flags_and_moves_that_are_not_aligned():
    L = _L()
    c = _cache()
    for off in (1, 2, 3):
        assert L.first_append8(c, P, 128, 64, P, 128, 64, 1, P, 3, P, 4, P, 3, 1, P + off, None) == UNSUPPORTED
        assert L.first_read8(c, P, 4, P, P, 3, 3, 1, P, 128, 64, P, 128, 64, 1, P + off, None) == UNSUPPORTED
        assert L.first_attn8(c, P, 256, 64, 4, 1, 0.1, P, 3, P, 4, P, 3, 1, P, 256, 64, None, 0, P + off, None) == UNSUPPORTED
        assert L.first_copy_pages(c, 1, P + off, 4, None, None) == UNSUPPORTED
        assert L.first_copy_pages(c, 1, P, 4, P + off, None) == UNSUPPORTED


@pytest.mark.parametrize("at", range(8))
def test_arrays_of_a_verification_that_are_not_aligned(at):
    for off in (1, 2, 3):
        a = [P + off if i == at else P for i in range(8)]  # target, draft, drafted, temperature, uniforms, draws, tokens, accepted
        rc = _L().first_verify(a[0], 4000, 1000, a[1], 3 * 1000, 1000, 0, a[2], 2, 3, 1000, a[3], a[4], a[5], a[6], a[7], None)
        assert rc == UNSUPPORTED
