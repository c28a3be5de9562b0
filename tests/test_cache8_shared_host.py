"""Layers that share a cache in 8 bits are refused (what two of them write to a block has one scale), without a GPU."""
import ctypes as C

import pytest
import torch

from test_cache8_host import DEV, _kv, lib  # noqa: F401


def _calls(lib):  # noqa: F811
    at = lambda *x: (C.c_void_p * len(x))(*[i << 20 for i in x])  # noqa: E731
    ok = dict(layers=3, kc=at(1, 2, 3), vc=at(4, 5, 6), ks=at(7, 8, 9), vs=at(10, 11, 12))
    shared = (dict(kc=at(1, 2, 1)), dict(vc=at(5, 5, 6)), dict(kc=at(1, 2, 6)), dict(ks=at(7, 9, 9)), dict(vs=at(10, 11, 8)))

    def resync(**kw):
        a = dict(ok, **kw)
        return lib.cure_resync_kv8(*a.values(), _kv(), DEV, DEV, 1, 9, 8, *[DEV] * 9, None)

    def held(name, bytes=1 << 20):
        return lambda **kw: getattr(lib, name)(*dict(ok, **kw).values(), _kv(), 1, DEV, DEV, bytes, None)
    return at, shared, resync, held


def test_the_entry_points_refuse(lib):  # noqa: F811
    at, shared, resync, held = _calls(lib)
    for call in (resync, held("cure_save_kv8"), held("cure_restore_kv8")):
        for kw in shared:
            assert call(**kw) == 1, kw
    # the check is of the layers that there are: apart, the next one (a small workspace) answers
    for name in ("cure_save_kv8", "cure_restore_kv8"):
        assert held(name, 16)() == 2 and held(name, 16)(layers=2, kc=at(1, 2, 1)) == 2
    many = at(*range(1, 129)), at(*range(129, 257)), at(*range(257, 385)), at(*range(385, 513))
    assert lib.cure_save_kv8(128, *many, _kv(), 1, DEV, DEV, 16, None) == 2


def test_a_step_refuses(lib):  # noqa: F811
    """Before anything runs, whatever else it is given."""
    from paper_2608_00531_gb300 import cure
    from paper_2608_00531_gb300.step import RepairVerifyStep
    kv = cure.kv_desc(2, 128, 64)
    step = RepairVerifyStep(1, 4, 64, 3, 1.0, 2, 2, 1, 3, 4, kv, torch.device("cpu"), layer_map=[0, 1, 0])
    with pytest.raises(ValueError, match="share"):
        step.run(None, [None] * 2, [None] * 2, scales=([None] * 2, [None] * 2))
