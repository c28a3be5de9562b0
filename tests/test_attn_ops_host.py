"""The attention operators' host side, without a GPU: the rotation's table of frequencies against decimal arithmetic,
and the arguments that the entry points refuse before anything is launched."""
import ctypes as C
import decimal
import math

import pytest


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    try:
        __graft_entry__.build()
    except RuntimeError as e:  # no toolkit on this machine
        pytest.skip(f"cannot build libcure: {e}")
    from paper_2608_00531_gb300 import _lib
    return _lib.load()


TWO_PI = decimal.Decimal("6.28318530717958647692528676655900576839433879875021164194988918461563")


@pytest.mark.parametrize("rot,base", [(128, 10000.0), (64, 500000.0), (16, 1.0e6)])
def test_frequencies_in_turns(lib, rot, base):
    """turns[i] 2^-64 is base^(-2i/rot) / 2 pi: a 64-bit power is off by 2^-52 of its value or so (pow within a unit, the
    exponent's rounding times the base's logarithm, at most 14), the quotient by half a unit."""
    from paper_2608_00531_gb300 import cure
    r = cure.rope_desc(rot, base)
    assert (r.style, r.rot_dim, r.amplitude) == (0, rot, 1.0)
    with decimal.localcontext() as ctx:
        ctx.prec = 60
        for i in range(rot // 2):
            want = decimal.Decimal(base) ** (decimal.Decimal(-2 * i) / rot) / TWO_PI
            got = decimal.Decimal(r.turns[i]) / 2 ** 64
            assert abs(got - want) <= want * decimal.Decimal(2.0 ** -48) + decimal.Decimal(2.0 ** -64), i
    assert all(t == 0 for t in r.turns[rot // 2:])


def test_own_frequencies_modulo_a_turn(lib):
    from paper_2608_00531_gb300 import cure
    two_pi = 2 * math.pi
    r = cure.rope_desc(16, freqs=[0.0, math.pi, two_pi, -math.pi / 2, 5 * math.pi, 1e-30, -1e-30, 3.0], style="interleaved")
    assert r.style == 1 and r.turns[0] == 0 and r.turns[1] == 1 << 63 and r.turns[2] == 0 and r.turns[3] == 3 << 62
    assert abs(r.turns[4] - (1 << 63)) <= 1 << 12 and r.turns[5] == 0 and r.turns[6] == 0
    assert abs(r.turns[7] / 2.0 ** 64 - 3.0 / two_pi) < 1e-15


def test_scalings(lib):
    """Each scaling's frequencies, as turns, against its formula."""
    from paper_2608_00531_gb300 import cure
    plain = [t / 2.0 ** 64 for t in cure.rope_desc(128, 1e4).turns]

    def turns(**sc):
        return [t / 2.0 ** 64 for t in cure.rope_desc(128, 1e4, scaling=sc).turns]
    for a, b in zip(plain, turns(kind="linear", factor=4.0)):
        assert abs(a / 4 - b) < 1e-14
    bands = turns(kind="bands", factor=8.0, low=1.0, high=4.0, original=8192)
    for a, b in zip(plain, bands):
        t = a * 8192
        g = min(1.0, max(0.0, (t - 1.0) / 3.0))
        assert abs(b - (g * a + (1 - g) * a / 8)) < 1e-14
    assert bands[0] == plain[0] and abs(bands[-1] - plain[-1] / 8) < 1e-15
    ramp = turns(kind="ramp", factor=4.0, slow=1.0, fast=32.0, original=4096)
    assert ramp[0] == plain[0] and abs(ramp[-1] - plain[-1] / 4) < 1e-15
    # slow and fast so close that the ramp has no width: a step
    step = turns(kind="ramp", factor=4.0, slow=31.9, fast=32.0, original=10.0)
    assert all(abs(s - p / 4) < 1e-14 or s == p for s, p in zip(step, plain))
    for a, b in zip([t / 2.0 ** 64 for t in cure.rope_desc(128, 1e4 * 2.0 ** (128 / 126)).turns],
                    turns(kind="base", factor=2.0)):
        assert abs(a - b) < 1e-13


def test_refusals(lib):
    from paper_2608_00531_gb300._lib import KVDesc, Rope, RopeScaling
    r, nul, dev = Rope(), None, C.c_void_p(1 << 20)
    init = lambda *a: lib.cure_rope_init(C.byref(r), *a)  # noqa: E731
    nan, inf = float("nan"), float("inf")
    assert init(0, 128, 1e4, None, 1.0) == 0
    for bad in ((2, 128, 1e4, None, 1.0), (-1, 128, 1e4, None, 1.0), (0, 0, 1e4, None, 1.0), (0, 130, 1e4, None, 1.0),
                (0, 17, 1e4, None, 1.0), (0, 128, 1.0, None, 1.0), (0, 128, nan, None, 1.0), (0, 128, inf, None, 1.0),
                (0, 128, 1e4, None, nan), (0, 128, 1e4, None, inf)):
        assert init(*bad) == 1, bad
    assert init(0, 24, 1e4, None, 1.0) == 5
    assert lib.cure_rope_init(None, 0, 128, 1e4, None, 1.0) == 1
    for sc in (RopeScaling(kind=5, factor=2.0), RopeScaling(kind=1, factor=0.0), RopeScaling(kind=2, factor=nan),
               RopeScaling(kind=3, factor=2.0, low=4.0, high=1.0, original=10.0),
               RopeScaling(kind=3, factor=2.0, low=0.0, high=1.0, original=10.0),
               RopeScaling(kind=4, factor=2.0, low=1.0, high=2.0, original=0.0),
               RopeScaling(kind=4, factor=2.0, low=1.0, high=inf, original=1.0)):
        assert init(0, 128, 1e4, C.byref(sc), 1.0) == 1
    freqs = (C.c_double * 64)(*([1.0] * 63 + [nan]))
    assert lib.cure_rope_init_freqs(C.byref(r), 0, 128, freqs, 1.0) == 1
    assert lib.cure_rope_init_freqs(C.byref(r), 0, 128, None, 1.0) == 1

    ok = dict(q=dev, k=dev, v=dev, ld_q=1024, ld_k=256, ld_v=256, rows=4, hq=8, hkv=2, D=128, pos=dev, rope=C.byref(r),
              qn=nul, kn=nul, eps=1e-6, qo=dev, ko=dev, vo=dev, lqo=1024, lko=256, lvo=256)

    def rope(**kw):
        a = dict(ok, **kw)
        return lib.cure_rope_qkv(*a.values(), None)
    odd = C.c_void_p((1 << 20) + 8)
    wrong = Rope(style=0, rot_dim=40, amplitude=1.0)
    for kw in (dict(rows=-1), dict(hq=-1), dict(eps=-1e-9), dict(eps=nan), dict(eps=inf), dict(q=odd), dict(vo=odd),
               dict(qn=odd), dict(ld_q=1023), dict(ld_q=1016), dict(lko=248), dict(ko=nul), dict(v=nul), dict(pos=nul),
               dict(rope=C.byref(wrong)), dict(rope=C.byref(Rope(style=7))), dict(D=0)):
        assert rope(**kw) == 1, kw
    assert rope(D=64) == 5 and rope(hq=5000, ld_q=1 << 20, lqo=1 << 20) == 5
    assert rope(rows=0, pos=nul) == 0 and rope(q=nul, k=nul, v=nul, qo=nul, ko=nul, vo=nul) == 0

    kv = KVDesc(layout=0, heads_kv=2, head_dim=128, page_size=16, max_len=100, num_pages=0, block_table=None)
    ok_a = dict(q=dev, k=dev, v=dev, ld_q=1024, ld_k=256, ld_v=256, rows=4, hq=8, batch=1, rs=dev, cl=dev, pos=nul,
                kv=C.byref(kv), kc=dev, vc=dev, rope=C.byref(r), qn=nul, kn=nul, eps=1e-6, qo=dev, lqo=1024)

    def append(**kw):
        a = dict(ok_a, **kw)
        return lib.cure_append_kv(*a.values(), None)
    for kw in (dict(rows=-1), dict(batch=-1), dict(hq=0), dict(k=nul), dict(v=nul), dict(kc=nul), dict(vc=odd),
               dict(rs=nul), dict(cl=nul), dict(qo=nul), dict(ld_v=248), dict(kv=None), dict(lqo=8)):
        assert append(**kw) == 1, kw
    bad_kv = KVDesc(layout=1, heads_kv=2, head_dim=128, page_size=12, max_len=4, num_pages=4, block_table=1 << 20)
    assert append(kv=C.byref(bad_kv)) == 5
    assert append(rows=0, k=nul, v=nul) == 0 and append(batch=0, rs=nul, cl=nul) == 0


def test_prompt_attn_refusals(lib):
    from paper_2608_00531_gb300._lib import KVDesc
    dev, nul, odd = C.c_void_p(1 << 20), None, C.c_void_p((1 << 20) + 8)
    kv = KVDesc(layout=0, heads_kv=2, head_dim=128, page_size=16, max_len=100, num_pages=0, block_table=None)
    need = lib.cure_prompt_attn_workspace_size(4, 1, 8, C.byref(kv))
    assert need > 0 and need % 256 == 0
    ok = dict(q=dev, kc=dev, vc=dev, kv=C.byref(kv), rs=dev, cl=dev, rows=4, batch=1, hq=8, scale=0.1, out=dev, ws=dev,
              bytes=need)

    def attn(**kw):
        return lib.cure_prompt_attn(*dict(ok, **kw).values(), None)
    for kw in (dict(rows=-1), dict(batch=-1), dict(hq=0), dict(hq=7), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(q=nul), dict(kc=nul), dict(vc=nul), dict(rs=nul),
               dict(cl=nul), dict(out=nul), dict(ws=nul), dict(q=odd), dict(kc=odd), dict(vc=odd), dict(out=odd),
               dict(ws=C.c_void_p((1 << 20) + 128)), dict(kv=None)):
        assert attn(**kw) == 1, kw
    assert attn(batch=257) == 5 and attn(hq=258) == 5 and attn(bytes=need - 1) == 2
    assert attn(rows=0, q=nul) == 0 and attn(batch=0, rs=nul) == 0
    kv64 = KVDesc(layout=0, heads_kv=2, head_dim=64, page_size=16, max_len=100, num_pages=0, block_table=None)
    assert attn(kv=C.byref(kv64)) == 5 and lib.cure_prompt_attn_workspace_size(4, 1, 8, C.byref(kv64)) == 0
    many = KVDesc(layout=0, heads_kv=4096, head_dim=128, page_size=16, max_len=100, num_pages=0, block_table=None)
    assert attn(kv=C.byref(many), rows=2 ** 31 - 1, hq=4096 * 128) == 5
