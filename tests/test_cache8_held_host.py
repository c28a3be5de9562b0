"""cure_save_kv8 and cure_restore_kv8 without a GPU: the size they state, and what they refuse before anything is launched."""
import ctypes as C

import pytest

from test_cache8_host import DEV, NUL, ODD, UNALIGNED, _kv, _paged, lib  # noqa: F401


def test_size(lib):  # noqa: F811
    size = lib.cure_save_kv8_size
    assert size(1, 1, _kv()) == 2 * 2 * (16 * 128 + 4) and size(28, 32, _paged(16)) == 28 * 32 * size(1, 1, _kv())
    assert size(0, 3, _kv()) == 0 and size(128, 4096, _kv(heads_kv=8)) == 128 * 4096 * 4 * size(1, 1, _kv()) > 2 ** 32
    for bad in ((-1, 1, _kv()), (129, 1, _kv()), (1, -1, _kv()), (1, 1, _paged(8)), (1, 1, _kv(head_dim=64)), (1, 1, None)):
        assert size(*bad) == 0


@pytest.mark.parametrize("name", ["cure_save_kv8", "cure_restore_kv8"])
def test_refusals(lib, name):  # noqa: F811
    kc, vc, ks, vs = ((C.c_void_p * 2)(i << 20, (i + 1) << 20) for i in (1, 3, 5, 7))
    need = lib.cure_save_kv8_size(2, 3, _kv())
    ok = dict(layers=2, kc=kc, vc=vc, ks=ks, vs=vs, kv=_kv(), batch=3, cl=DEV, saved=DEV, bytes=need)

    def call(**kw):
        return getattr(lib, name)(*dict(ok, **kw).values(), None)
    missing, odd, unaligned = ((C.c_void_p * 2)(1 << 20, x) for x in (None, (1 << 20) + 8, (1 << 20) + 2))
    for kw in (dict(layers=-1), dict(layers=129), dict(batch=-1), dict(kv=None), dict(cl=NUL), dict(cl=UNALIGNED),
               dict(saved=NUL), dict(saved=ODD), *(dict([(a, b)]) for a in ("kc", "vc") for b in (None, missing, odd)),
               *(dict([(a, b)]) for a in ("ks", "vs") for b in (None, missing, unaligned))):
        assert call(**kw) == 1, kw
    assert call(kv=_paged(8)) == 5 and call(kv=_kv(head_dim=64)) == 5 and call(bytes=need - 1) == 2
    assert call(batch=0, cl=NUL, saved=NUL) == 0 and call(layers=0, kc=None, saved=NUL) == 0
