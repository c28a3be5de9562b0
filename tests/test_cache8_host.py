"""The entry points over a cache in 8 bits and of rotations with several axes, without a GPU: what they refuse before
anything is launched, and the binding's own checks."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    try:
        __graft_entry__.build()
    except RuntimeError as e:  # no toolkit on this machine
        pytest.skip(f"cannot build libcure: {e}")
    from paper_2608_00531_gb300 import _lib
    return _lib.load()


DEV, ODD, NUL = C.c_void_p(1 << 20), C.c_void_p((1 << 20) + 8), None
UNALIGNED = C.c_void_p((1 << 20) + 2)


def _kv(**kw):
    from paper_2608_00531_gb300._lib import KVDesc
    return C.byref(KVDesc(**dict(dict(layout=0, heads_kv=2, head_dim=128, page_size=16, max_len=100, num_pages=0,
                                      block_table=None), **kw)))


def _paged(ps):
    return _kv(layout=1, page_size=ps, max_len=4, num_pages=4, block_table=1 << 20)


def test_axes(lib):
    from paper_2608_00531_gb300 import cure
    a = cure.rope_axes([0] * 16 + [1] * 24 + [2] * 24)
    assert a.axes == 3 and list(a.axis) == [0] * 16 + [1] * 24 + [2] * 24
    assert cure.rope_axes([0, 1]).axes == 2 and cure.rope_axes([7]).axes == 8
    for bad in ([], [0] * 65, [-1], [8]):
        with pytest.raises(ValueError):
            cure.rope_axes(bad)


def test_rope_axes_refusals(lib):
    from paper_2608_00531_gb300._lib import Rope, RopeAxes
    r = Rope(style=0, rot_dim=32, amplitude=1.0)
    ok = dict(q=DEV, k=DEV, v=DEV, ld_q=1024, ld_k=256, ld_v=256, rows=4, hq=8, hkv=2, D=128, pos=DEV,
              axes=C.byref(RopeAxes(axes=2)), rope=C.byref(r), qn=NUL, kn=NUL, eps=1e-6, qo=DEV, ko=DEV, vo=DEV, lqo=1024,
              lko=256, lvo=256)

    def call(**kw):
        return lib.cure_rope_qkv_axes(*dict(ok, **kw).values(), None)
    at = lambda i, v: (C.c_uint8 * 64)(*[v if j == i else 0 for j in range(64)])  # noqa: E731
    for kw in (dict(axes=C.byref(RopeAxes(axes=0))), dict(axes=C.byref(RopeAxes(axes=9))), dict(pos=NUL),
               dict(axes=C.byref(RopeAxes(axes=2, axis=at(15, 2)))), dict(rows=-1), dict(q=ODD), dict(pos=UNALIGNED)):
        assert call(**kw) == 1, kw
    # behind the rotated pairs nothing is read
    assert call(rows=0, axes=C.byref(RopeAxes(axes=2, axis=at(16, 2)))) == 0
    assert call(D=64) == 5 and call(rows=0, pos=NUL) == 0
    ok_a = dict(q=DEV, k=DEV, v=DEV, ld_q=1024, ld_k=256, ld_v=256, rows=4, hq=8, batch=1, rs=DEV, cl=DEV, pos=DEV,
                axes=C.byref(RopeAxes(axes=2)), kv=_kv(), kc=DEV, vc=DEV, rope=C.byref(r), qn=NUL, kn=NUL, eps=1e-6,
                qo=DEV, lqo=1024)

    def append(**kw):
        return lib.cure_append_kv_axes(*dict(ok_a, **kw).values(), None)
    for kw in (dict(pos=NUL), dict(axes=C.byref(RopeAxes(axes=-1))), dict(kc=NUL), dict(rs=NUL)):
        assert append(**kw) == 1, kw
    assert append(rows=0, pos=NUL) == 0


def test_append8_refusals(lib):
    from paper_2608_00531_gb300._lib import Rope, RopeAxes
    r = Rope(style=0, rot_dim=32, amplitude=1.0)
    ok = dict(q=DEV, k=DEV, v=DEV, ld_q=1024, ld_k=256, ld_v=256, rows=4, hq=8, batch=1, rs=DEV, cl=DEV, pos=NUL,
              axes=None, kv=_kv(), kc=DEV, vc=DEV, ks=DEV, vs=DEV, rope=C.byref(r), qn=NUL, kn=NUL, eps=1e-6, qo=DEV,
              lqo=1024)

    def call(**kw):
        return lib.cure_append_kv8(*dict(ok, **kw).values(), None)
    for kw in (dict(rows=-1), dict(batch=-1), dict(hq=0), dict(k=NUL), dict(v=NUL), dict(kc=NUL), dict(vc=ODD),
               dict(rs=NUL), dict(cl=NUL), dict(qo=NUL), dict(ld_v=248), dict(kv=None), dict(ks=NUL), dict(vs=NUL),
               dict(ks=UNALIGNED), dict(vs=UNALIGNED), dict(axes=C.byref(RopeAxes(axes=2))), dict(eps=float("nan"))):
        assert call(**kw) == 1, kw
    assert call(kv=_paged(8)) == 5 and call(kv=_paged(24)) == 5 and call(kv=_kv(head_dim=64)) == 5
    assert call(rows=0, k=NUL, v=NUL, ks=NUL, vs=NUL) == 0 and call(batch=0, rs=NUL, cl=NUL) == 0


def test_attention8_refusals(lib):
    need = lib.cure_prompt_attn8_workspace_size(4, 1, 8, _kv())
    assert need > 0 and need % 256 == 0 and lib.cure_tree_attn8_workspace_size(1, 4, 8, _kv()) == need
    ok = dict(q=DEV, kc=DEV, vc=DEV, ks=DEV, vs=DEV, kv=_kv(), rs=DEV, cl=DEV, rows=4, batch=1, hq=8, scale=0.1, out=DEV,
              ws=DEV, bytes=need)

    def prompt(**kw):
        return lib.cure_prompt_attn8(*dict(ok, **kw).values(), None)
    tree_ok = dict(q=DEV, kc=DEV, vc=DEV, ks=DEV, vs=DEV, kv=_kv(), cl=DEV, nn=DEV, anc=DEV, batch=1, n_max=4, hq=8,
                   scale=0.1, out=DEV, ws=DEV, bytes=need)

    def tree(**kw):
        return lib.cure_tree_attn8(*dict(tree_ok, **kw).values(), None)
    nan, inf = float("nan"), float("inf")
    for kw in (dict(batch=-1), dict(hq=0), dict(hq=7), dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(scale=inf),
               dict(q=NUL), dict(kc=NUL), dict(vc=NUL), dict(ks=NUL), dict(vs=NUL), dict(cl=NUL), dict(out=NUL),
               dict(ws=NUL), dict(q=ODD), dict(kc=ODD), dict(vc=ODD), dict(out=ODD), dict(ks=UNALIGNED),
               dict(vs=UNALIGNED), dict(cl=UNALIGNED), dict(ws=C.c_void_p((1 << 20) + 128)), dict(kv=None)):
        assert prompt(**kw) == 1, kw
        assert tree(**kw) == 1, kw
    assert prompt(rows=-1) == 1 and prompt(rs=NUL) == 1 and tree(nn=NUL) == 1 and tree(anc=NUL) == 1
    assert tree(n_max=0) == 1 and tree(anc=C.c_void_p((1 << 20) + 4)) == 1
    for call in (prompt, tree):
        assert call(batch=257) == 5 and call(hq=258) == 5 and call(bytes=need - 1) == 2
        assert call(kv=_paged(8)) == 5 and call(kv=_kv(head_dim=64)) == 5
        assert call(batch=0, q=NUL) == 0
    assert prompt(rows=0, q=NUL) == 0 and tree(n_max=257) == 5
    for size in (lib.cure_prompt_attn8_workspace_size, lib.cure_tree_attn8_workspace_size):
        assert size(4, 1, 8, _paged(8)) == 0 and size(4, 1, 7, _kv()) == 0


def test_resync8_refusals(lib):
    array = (C.c_void_p * 2)(1 << 20, 1 << 20)
    bad = (C.c_void_p * 2)(1 << 20, None)
    odd = (C.c_void_p * 2)(1 << 20, (1 << 20) + 2)
    ok = dict(layers=2, kc=array, vc=array, ks=array, vs=array, kv=_kv(), tk=DEV, tv=DEV, batch=1, n_max=9, block=8, path=DEV,
              a=DEV, d=DEV, tok=DEV, lin=DEV, lout=DEV, valid=DEV, replay=DEV, n=DEV)

    def call(**kw):
        return lib.cure_resync_kv8(*dict(ok, **kw).values(), None)
    for kw in (dict(layers=-1), dict(layers=129), dict(batch=-1), dict(n_max=8), dict(block=0), dict(block=33, n_max=40),
               dict(kc=bad), dict(vs=bad), dict(ks=odd), dict(vc=odd), dict(tk=NUL), dict(tv=NUL), dict(tv=ODD),
               dict(path=NUL), dict(a=NUL), dict(lin=NUL), dict(n=NUL), dict(kv=None), dict(ks=None)):
        assert call(**kw) == 1, kw
    assert call(kv=_paged(8)) == 5 and call(batch=0) == 0


def test_the_binding_refuses(lib):
    from paper_2608_00531_gb300 import cure
    kv = cure.kv_desc(2, 128, 40)
    assert cure.kv8_scale_shape(kv, 3) == (3, 3, 2)
    table = torch.zeros(2, 4, dtype=torch.int32)
    kv2 = cure.KVDesc(layout=1, heads_kv=4, head_dim=128, page_size=32, max_len=4, num_pages=7)
    assert cure.kv8_scale_shape(kv2, 2) == (7, 2, 4) and table.shape == (2, 4)
    pos = torch.zeros(2, 5, dtype=torch.int32)
    with pytest.raises(ValueError):
        cure._rows_of_axes(pos, cure.rope_axes([0, 1, 2]))
    with pytest.raises(ValueError):
        cure._rows_of_axes(pos[0], cure.rope_axes([0]))
    assert cure._rows_of_axes(pos, cure.rope_axes([0, 1])) == 5
