"""cure_rope_qkv and cure_append_kv on the GPU against their formulas in 64 bits.

Tolerance of a computed value y from the pair (a, b), both after the norm: it is
rounded to bf16 once (half a step: 2^-8 |y|); before that, in float32, the angle
is off by up to 2^-32 + 2^-25 turns (2^-22.3 radians), sincospif by 2 units of
2^-24, the norm's factor by about (128-term sum in 12 steps, rsqrtf 2 units)
2^-20, and four roundings of 2^-24 join the products: together below
2^-19 A (|a| + |b|), and half a step more where that crosses a rounding border:
2^-8 |y| + 2^-18 A (|a| + |b|).
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
D = 128


@pytest.fixture(scope="module")
def cure():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2608_00531_gb300 import cure as c
    torch.cuda.set_device(DEV)
    return c


def _freqs(rot, base, scaling=None):
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        return f / 4.0
    if scaling == "bands":
        t = f * 8192 / (2 * math.pi)
        g = np.clip((t - 1.0) / 3.0, 0.0, 1.0)
        return g * f + (1 - g) * f / 8.0
    return f


def _ref(x, pos, w, eps, style, rot, freqs, amp):
    """x float64 [rows][heads][D] -> (the value in 64 bits, |a| + |b| of its pair)."""
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    y, size = x.copy(), np.abs(x)
    if rot:
        ang = pos.astype(np.float64)[:, None] * freqs
        c, s = np.cos(ang)[:, None] * amp, np.sin(ang)[:, None] * amp
        ia = np.arange(rot // 2) if style == "half" else 2 * np.arange(rot // 2)
        ib = ia + rot // 2 if style == "half" else ia + 1
        a, b = x[..., ia], x[..., ib]
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        size[..., ia] = size[..., ib] = (np.abs(a) + np.abs(b)) * abs(amp)
    return y, size


def _close(got, y, size):
    g = got.double().cpu().numpy()
    assert np.all(np.abs(g - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -18 * size), np.max(np.abs(g - y) / (np.abs(y) + 1e-30))


def _randn(rng, *shape, std=1.0):
    return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32) * np.float32(std)).to(torch.bfloat16)


def _f64(t):
    return t.double().cpu().numpy()


FORMS = [("half", 128, None, 1.0, False), ("half", 128, None, 1.0, True), ("interleaved", 128, "bands", 1.0, True),
         ("half", 64, "linear", 1.25, False), ("interleaved", 64, None, 0.75, True), ("half", 16, None, 1.0, True),
         ("interleaved", 16, None, 1.0, False), ("half", 96, "bands", 1.0, False), ("half", 0, None, 1.0, True)]


@pytest.mark.parametrize("style,rot,scaling,amp,norm", FORMS)
@pytest.mark.parametrize("B,N,Hq,Hkv,fused", [(1, 1, 1, 1, False), (1, 25, 32, 8, True), (3, 33, 28, 4, True),
                                              (2, 49, 7, 7, False), (5, 9, 64, 3, True)])
def test_rope_qkv(cure, style, rot, scaling, amp, norm, B, N, Hq, Hkv, fused):
    rng = np.random.default_rng([B, N, Hq, rot])
    if fused:
        qkv = _randn(rng, B, N, Hq + 2 * Hkv, D).to(DEV)
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    else:
        q, k, v = (_randn(rng, B, N, h, D).to(DEV) for h in (Hq, Hkv, Hkv))
    pos = rng.integers(0, 9000, size=(B, N)).astype(np.int32)
    pos[:, N // 2:] = rng.integers(0, 2 ** 31 - 1, size=(B, N - N // 2))
    pos.reshape(-1)[0] = 0
    if N > 3:
        pos[:, -1], pos[:, -2], pos[0, 1] = -1, 2 ** 31 - 1, -7
    qn, kn = ((_randn(rng, D, std=0.2).to(DEV) + 1.0) if norm else None for _ in range(2))
    desc = None
    if rot:
        sc = {None: None, "linear": dict(kind="linear", factor=4.0),
              "bands": dict(kind="bands", factor=8.0, low=1.0, high=4.0, original=8192)}[scaling]
        desc = cure.rope_desc(rot, 10000.0, style=style, scaling=sc, amplitude=amp)
    out = tuple(torch.full((B, N, h, D), 3.5, dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv))
    got = cure.cure_rope_qkv(q, k, v, torch.from_numpy(pos).to(DEV), desc, q_norm=qn, k_norm=kn, eps=1e-5, out=out)
    keep = pos.reshape(-1) >= 0
    f = _freqs(rot, 10000.0, scaling) if rot else None
    for g, x, w in ((got[0], q, qn), (got[1], k, kn)):
        flat = g.reshape(B * N, -1, D)
        y, size = _ref(_f64(x).reshape(B * N, -1, D)[keep], pos.reshape(-1)[keep], None if w is None else _f64(w), 1e-5,
                       style, rot, f, amp)
        _close(flat[torch.from_numpy(keep).to(DEV)], y, size)
        assert torch.all(flat[torch.from_numpy(~keep).to(DEV)] == 3.5)
    kept = torch.from_numpy(keep.reshape(B, N)).to(DEV)
    assert torch.equal(got[2][kept], v[kept]) and torch.all(got[2][~kept] == 3.5)
    assert cure.cure_device_error() == 0


def test_rope_qkv_in_place_and_parts(cure):
    """Outputs that are the inputs; q alone, k alone, v alone."""
    rng = np.random.default_rng(3)
    T, Hq, Hkv = 70, 12, 2
    qkv = _randn(rng, T, Hq + 2 * Hkv, D).to(DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV) * 31
    desc = cure.rope_desc(128, 500000.0)
    parts = lambda t: (t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:])  # noqa: E731
    want = cure.cure_rope_qkv(*parts(qkv), pos, desc)
    here = qkv.clone()
    cure.cure_rope_qkv(*parts(here), pos, desc, out=parts(here))
    for w, h in zip(want, parts(here)):
        assert torch.equal(w, h)
    for i in range(3):
        only = [t if j == i else None for j, t in enumerate(parts(qkv))]
        got = cure.cure_rope_qkv(*only, pos, desc)
        assert torch.equal(got[i], want[i]) and all(g is None for j, g in enumerate(got) if j != i)


@pytest.mark.parametrize("style", ["half", "interleaved"])
def test_rope_qkv_infinities_and_nans_stay_with_their_pairs(cure, style):
    """A value that is not rotated passes through whatever lies around it, a pair's infinities and NaNs reach only the
    pair, v is copied bit for bit and rows without a position do not count."""
    rng = np.random.default_rng(9)
    T, rot = 20, 64
    q = _randn(rng, T, 3, D)
    q[2, 1, 100], q[3, 1, 70] = math.inf, math.nan          # not rotated
    q[5, 0, 3], q[6, 2, 17] = math.nan, -math.inf            # rotated
    q[7] = math.nan                                          # left out
    v = torch.from_numpy(rng.integers(-32768, 32768, size=(T, 2, D)).astype(np.int16)).view(torch.bfloat16)
    pos = torch.arange(1, T + 1, dtype=torch.int32)
    pos[7] = -1
    desc = cure.rope_desc(rot, 10000.0, style=style)
    out = (torch.zeros_like(q).to(DEV), None, torch.zeros_like(v).to(DEV))
    got, _, gv = cure.cure_rope_qkv(q.to(DEV), None, v.to(DEV), pos.to(DEV), desc, out=out)
    got, keep = got.float().cpu(), pos >= 0
    clean = cure.cure_rope_qkv(torch.nan_to_num(q, 0.5, 0.5, 0.5).to(DEV), None, None, pos.to(DEV), desc)[0].float().cpu()
    bad = torch.zeros(T, 3, D, dtype=torch.bool)
    bad[2, 1, 100] = bad[3, 1, 70] = True
    for r, h, d in ((5, 0, 3), (6, 2, 17)):
        bad[r, h, d] = True
        bad[r, h, (d + rot // 2) % rot if style == "half" else d ^ 1] = True
    assert torch.equal(~torch.isfinite(got[keep]), bad[keep])
    assert got[2, 1, 100] == math.inf and math.isnan(got[3, 1, 70])
    assert torch.equal(got[keep][~bad[keep]], clean[keep][~bad[keep]]) and torch.all(got[7] == 0)
    assert torch.equal(gv.cpu().view(torch.int16)[keep], v.view(torch.int16)[keep])


def test_rope_qkv_own_frequencies_and_ramp(cure):
    """The caller's own frequencies (above one turn and negative ones too), and the ramp's against its formula."""
    rng = np.random.default_rng(12)
    x = _randn(rng, 64, 2, D).to(DEV)
    pos = torch.from_numpy(rng.integers(0, 200000, size=64).astype(np.int32)).to(DEV)
    f = rng.uniform(-9.0, 9.0, size=64)
    f[0] = 0.0
    got = cure.cure_rope_qkv(x, None, None, pos, cure.rope_desc(128, freqs=f))[0]
    # the products' own rounding in 64 bits: 200000 * 9 * 2^-53 radians, far below 2^-22
    _close(got, *_ref(_f64(x), pos.cpu().numpy(), None, 0, "half", 128, f, 1.0))
    base, factor, orig, slow, fast = 1e6, 4.0, 32768, 1.0, 32.0
    d = lambda t: 128 * math.log(orig / (2 * math.pi * t)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(math.floor(d(fast)), 0), min(math.ceil(d(slow)), 127)
    g = np.clip((np.arange(64) - lo) / (hi - lo), 0, 1)
    f = _freqs(128, base)
    desc = cure.rope_desc(128, base, scaling=dict(kind="ramp", factor=factor, slow=slow, fast=fast, original=orig))
    got = cure.cure_rope_qkv(x, None, None, pos, desc)[0]
    _close(got, *_ref(_f64(x), pos.cpu().numpy(), None, 0, "half", 128, (1 - g) * f + g * f / factor, 1.0))
    desc = cure.rope_desc(128, base, scaling=dict(kind="base", factor=3.0))
    got = cure.cure_rope_qkv(x, None, None, pos, desc)[0]
    _close(got, *_ref(_f64(x), pos.cpu().numpy(), None, 0, "half", 128, _freqs(128, base * 3.0 ** (128 / 126)), 1.0))


# ---------------------------------------------------------------- append
def _cache(rng, lens, n, Hkv, ps):
    """Caches of a marker value, their table (None: contiguous) and a function from (sequence, slot) to the row."""
    ends = [a + b for a, b in zip(lens, n)]
    if ps == 0:
        shape, table, pages = (len(n), max(ends) + 3, Hkv, D), None, 0
        row = lambda b, s: b * shape[1] + s  # noqa: E731
    else:
        need = [-(-e // ps) for e in ends]
        pages = sum(need) + 3
        perm = rng.permutation(pages).astype(np.int32)
        table = np.full((len(n), max(max(need), 1)), -1, dtype=np.int32)
        o = 0
        for b, c in enumerate(need):
            table[b, :c] = perm[o:o + c]
            o += c
        shape = (pages, ps, Hkv, D)
        row = lambda b, s: int(table[b, s // ps]) * ps + s % ps  # noqa: E731
    k, v = (torch.full(shape, 2.25, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    return k, v, table, pages, row


def _desc(cure, k, table, pages, Hkv, ps):
    if table is None:
        return cure.kv_desc(Hkv, D, k.shape[1])
    return cure.kv_desc(Hkv, D, table.shape[1], block_table=torch.from_numpy(table).to(DEV), page_size=ps, num_pages=pages)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _check_append(q, k, v, got, kc, vc, row, lens, n, start, f, norm, desc_args, pos=None):
    style, rot, amp = desc_args
    T = k.shape[0]
    p = np.full(T, -1, dtype=np.int64)
    where = np.full(T, -1, dtype=np.int64)
    for b in range(len(n)):
        for i in range(n[b]):
            r = start[b] + i
            p[r] = lens[b] + i if pos is None else pos[r]
            where[r] = row(b, lens[b] + i)
    keep = p >= 0
    qn, kn = norm
    if q is not None:
        y, s = _ref(_f64(q)[keep], p[keep], None if qn is None else _f64(qn), 1e-6, style, rot, f, amp)
        _close(got[torch.from_numpy(keep).to(DEV)], y, s)
        assert torch.all(got[torch.from_numpy(~keep).to(DEV)] == 3.5)
    y, s = _ref(_f64(k)[keep], p[keep], None if kn is None else _f64(kn), 1e-6, style, rot, f, amp)
    Hkv = k.shape[1]
    at = torch.from_numpy(where[keep]).to(DEV)
    _close(kc.view(-1, Hkv, D)[at], y, s)
    assert torch.equal(vc.view(-1, Hkv, D)[at], v[torch.from_numpy(keep).to(DEV)])
    rest = torch.ones(kc.numel() // (Hkv * D), dtype=torch.bool, device=DEV)
    rest[at] = False
    assert torch.all(kc.view(-1, Hkv, D)[rest] == 2.25) and torch.all(vc.view(-1, Hkv, D)[rest] == 2.25)


@pytest.mark.parametrize("ps", [0, 8, 16, 32, 64])
@pytest.mark.parametrize("lens,n,Hq,Hkv,style,rot,norm", [
    ([0], [1], 8, 2, "half", 128, False),
    ([5, 0, 63, 17], [7, 0, 1, 90], 28, 4, "half", 128, True),
    ([0, 200, 64], [130, 3, 64], 3, 1, "interleaved", 32, False),
    ([3, 9, 0], [0, 0, 0], 4, 4, "half", 64, True),
])
def test_append_kv(cure, ps, lens, n, Hq, Hkv, style, rot, norm):
    rng = np.random.default_rng([ps, len(n), Hq])
    kc, vc, table, pages, row = _cache(rng, lens, n, Hkv, ps)
    pad = 2  # rows before the first sequence and behind the last one
    start = [pad] + [pad + int(x) for x in np.cumsum(n)]
    T = start[-1] + 3
    qkv = _randn(rng, T, Hq + 2 * Hkv, D).to(DEV)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    qn, kn = ((_randn(rng, D, std=0.2).to(DEV) + 1.0) if norm else None for _ in range(2))
    desc = cure.rope_desc(rot, 10000.0, style=style)
    out = torch.full((T, Hq, D), 3.5, dtype=torch.bfloat16, device=DEV)
    got = cure.cure_append_kv(k, v, kc, vc, _desc(cure, kc, table, pages, Hkv, ps), _i32(start), _i32(lens), desc, q=q,
                              q_norm=qn, k_norm=kn, out=out)
    _check_append(q, k, v, got, kc, vc, row, lens, n, start, _freqs(rot, 10000.0), (qn, kn), (style, rot, 1.0))
    assert cure.cure_device_error() == 0


def test_append_kv_many_sequences_without_q(cure):
    """More sequences than one round of the search covers, empty ones among them; K and V alone."""
    rng = np.random.default_rng(4)
    B, Hkv = 700, 2
    n = rng.integers(0, 4, size=B).tolist()
    lens = rng.integers(0, 50, size=B).tolist()
    kc, vc, table, pages, row = _cache(rng, lens, n, Hkv, 16)
    start = [0] + [int(x) for x in np.cumsum(n)]
    k, v = (_randn(rng, start[-1], Hkv, D).to(DEV) for _ in range(2))
    assert cure.cure_append_kv(k, v, kc, vc, _desc(cure, kc, table, pages, Hkv, 16), _i32(start), _i32(lens),
                               cure.rope_desc(128, 10000.0)) is None
    _check_append(None, k, v, None, kc, vc, row, lens, n, start, _freqs(128, 10000.0), (None, None), ("half", 128, 1.0))
    assert cure.cure_device_error() == 0


def test_append_kv_in_place_tree(cure):
    """The in-place tree layout: padded rows at slots L + j, the positions those of the tree, padding left out."""
    rng = np.random.default_rng(6)
    B, N, Hq, Hkv = 3, 11, 4, 2
    lens, n = [30, 0, 61], [N] * B
    nodes = [11, 1, 6]
    kc, vc, table, pages, row = _cache(rng, lens, n, Hkv, 16)
    q, k, v = (_randn(rng, B, N, h, D).to(DEV) for h in (Hq, Hkv, Hkv))
    pos = np.full((B, N), -1, dtype=np.int32)
    for b in range(B):
        pos[b, :nodes[b]] = lens[b] + np.minimum(np.arange(nodes[b]), 4)
    out = torch.full((B, N, Hq, D), 3.5, dtype=torch.bfloat16, device=DEV)
    got = cure.cure_append_kv(k, v, kc, vc, _desc(cure, kc, table, pages, Hkv, 16), _i32([0, N, 2 * N, 3 * N]), _i32(lens),
                              cure.rope_desc(128, 10000.0), q=q, pos=torch.from_numpy(pos).to(DEV), out=out)
    flat = lambda t: t.reshape(B * N, -1, D)  # noqa: E731
    _check_append(flat(q), flat(k), flat(v), flat(got), kc, vc, row, lens, n, [0, N, 2 * N, 3 * N], _freqs(128, 10000.0),
                  (None, None), ("half", 128, 1.0), pos=pos.reshape(-1))


def test_append_kv_bad_pages_and_slots(cure):
    """What only the device can see: the rows concerned are left out, the others written, a bit raised."""
    rng = np.random.default_rng(8)
    Hkv, ps = 2, 8
    table = np.array([[0, 1], [2, -1], [3, 99], [4, 5]], dtype=np.int32)
    kv = cure.kv_desc(Hkv, D, 2, block_table=torch.from_numpy(table).to(DEV), page_size=ps, num_pages=6)
    k, v = (_randn(rng, 12, Hkv, D).to(DEV) for _ in range(2))
    desc = cure.rope_desc(128, 10000.0)

    def run(start, lens):
        kc, vc = (torch.full((6, ps, Hkv, D), 2.25, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        cure.cure_append_kv(k, v, kc, vc, kv, _i32(start), _i32(lens), desc)
        bits = cure.cure_device_error()
        return bits, (vc.view(-1, Hkv, D) != 2.25).any(-1).any(-1).cpu().numpy().nonzero()[0].tolist()
    # rows 0..2 of each: sequence 1 crosses into a missing page, 2 into one that does not exist
    bits, at = run([0, 3, 6, 9, 12], [0, 6, 7, 8])
    assert bits == cure.DEVERR_PAGE and at == [0, 1, 2, 22, 23, 31, 40, 41, 42]
    # sequence 3 runs past its two pages, sequence 0 starts at a negative length
    bits, at = run([0, 3, 6, 9, 12], [-1, 0, 0, 15])
    assert bits == cure.DEVERR_SLOT and at == [0, 1, 16, 17, 18, 24, 25, 26, 47]
    # row_start that does not ascend: nothing outside the cache is touched and the bit is raised
    bits, _ = run([0, 9, 3, 12, 12], [0, 0, 0, 0])
    assert bits in (0, cure.DEVERR_NODES, cure.DEVERR_NODES | cure.DEVERR_PAGE, cure.DEVERR_PAGE)
    bits, _ = run([11, 2, 2, 2, 2], [0, 0, 0, 0])
    assert bits == 0  # every row lies behind the last sequence
    bits, _ = run([0, 0, 0, 11, 12], [0, 0, 0, 0])
    assert bits & ~(cure.DEVERR_SLOT | cure.DEVERR_PAGE) == 0


def test_append_kv_rows_of_no_sequence(cure):
    """Where row_start does not ascend, a row goes to a sequence whose range holds it or nowhere."""
    rng = np.random.default_rng(18)
    kv = cure.kv_desc(2, D, 16)
    k, v = (_randn(rng, 12, 2, D).to(DEV) for _ in range(2))

    def run(start):
        kc, vc = (torch.full((4, 16, 2, D), 2.25, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        cure.cure_append_kv(k, v, kc, vc, kv, _i32(start), _i32([0, 0, 0, 0]), cure.rope_desc(128, 10000.0))
        bits = cure.cure_device_error()
        return bits, (vc.view(-1, 2, D) != 2.25).any(-1).any(-1).cpu().numpy().nonzero()[0].tolist()
    assert run([0, 10, 2, 3, 3]) == (cure.DEVERR_NODES, [0, 1])
    assert run([-2, 3, 3, 3, 3]) == (cure.DEVERR_NODES, [])
    assert run([2, 3, 3, 5, 6]) == (0, [0, 32, 33, 48])


def test_empty_calls(cure):
    kv = cure.kv_desc(2, D, 8)
    kc, vc = (torch.full((1, 8, 2, D), 2.25, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    none = torch.empty(0, 2, D, dtype=torch.bfloat16, device=DEV)
    desc = cure.rope_desc(128, 10000.0)
    cure.cure_append_kv(none, none, kc, vc, kv, _i32([0, 0]), _i32([3]), desc)
    got = cure.cure_rope_qkv(none, none, none, _i32([]), desc)
    assert got[0].shape == (0, 2, D) and torch.all(kc == 2.25)


def test_graph_replay_and_streams(cure):
    """Captured once and replayed on other inputs, positions and lengths; on a stream of its own."""
    rng = np.random.default_rng(14)
    T, Hq, Hkv = 40, 8, 2
    desc = cure.rope_desc(128, 10000.0)
    q, k, v = (_randn(rng, T, h, D).to(DEV) for h in (Hq, Hkv, Hkv))
    pos, lens, start = _i32(list(range(T))), _i32([0, 10]), _i32([0, 15, 40])
    kc, vc = (torch.zeros(2, 64, Hkv, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    kv = cure.kv_desc(Hkv, D, 64)
    out = tuple(torch.zeros_like(t) for t in (q, k, v))
    q2 = torch.zeros_like(q)

    def call(stream=None):
        cure.cure_rope_qkv(q, k, v, pos, desc, out=out, stream=stream)
        cure.cure_append_kv(k, v, kc, vc, kv, start, lens, desc, q=q, out=q2, stream=stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed in range(2):
        for t in (q, k, v):
            t.copy_(_randn(np.random.default_rng(seed), *t.shape))
        pos.add_(17)
        lens.copy_(_i32([seed + 1, 3]))
        start.copy_(_i32([0, 9 + seed, 40]))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out, q2, kc, vc)]
        for t in (*out, q2):
            t.zero_()
        call()
        torch.cuda.synchronize()
        for a, b in zip(got, (*out, q2, kc, vc)):
            assert torch.equal(a, b)
    # a stream's own result: allocated there
    with torch.cuda.stream(side):
        fresh = cure.cure_rope_qkv(q, k, v, pos, desc, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(fresh, out))


def test_binding_refusals(cure):
    desc = cure.rope_desc(128, 10000.0)
    q = torch.zeros(4, 8, D, dtype=torch.bfloat16, device=DEV)
    k = torch.zeros(4, 2, D, dtype=torch.bfloat16, device=DEV)
    pos = _i32([0, 1, 2, 3])
    bad = [
        (TypeError, lambda: cure.cure_rope_qkv(q.float(), k, k, pos, desc)),
        (TypeError, lambda: cure.cure_rope_qkv(q, k, k, pos.long(), desc)),
        (ValueError, lambda: cure.cure_rope_qkv(q.cpu(), k, k, pos, desc)),
        (ValueError, lambda: cure.cure_rope_qkv(q, k, k, pos[:3], desc)),
        (ValueError, lambda: cure.cure_rope_qkv(q, k, k[:, :1], pos, desc)),
        (ValueError, lambda: cure.cure_rope_qkv(q.transpose(0, 1), k, k, pos, desc)),
        (ValueError, lambda: cure.cure_rope_qkv(q[..., ::2], None, None, pos, None)),
        (ValueError, lambda: cure.cure_rope_qkv(q, k, k, pos, desc, q_norm=torch.ones(64, dtype=torch.bfloat16, device=DEV))),
        (ValueError, lambda: cure.cure_rope_qkv(q, k, k, pos, desc, out=(q[:2], k, k))),
        (ValueError, lambda: cure.rope_desc(128, 1e4, style="whole")),
        (ValueError, lambda: cure.rope_desc(128, 1e4, scaling=dict(kind="other", factor=2.0))),
        (ValueError, lambda: cure.rope_desc(128, 1e4, scaling=dict(kind="bands", factor=2.0))),
        (ValueError, lambda: cure.rope_desc(64, freqs=[1.0] * 31)),
    ]
    kv = cure.kv_desc(2, D, 8)
    kc = torch.zeros(1, 8, 2, D, dtype=torch.bfloat16, device=DEV)
    bad += [
        (ValueError, lambda: cure.cure_append_kv(k, k, kc, kc.clone(), kv, _i32([0, 2, 4]), _i32([0]), desc)),
        (ValueError, lambda: cure.cure_append_kv(k, k, kc, kc.clone(), kv, _i32([0, 2, 4]), _i32([0, 0]), desc)),
        (ValueError, lambda: cure.cure_append_kv(q, q, kc, kc.clone(), kv, _i32([0, 4]), _i32([0]), desc)),
        (ValueError, lambda: cure.cure_append_kv(k, k, kc, kc.clone(), kv, _i32([0, 4]), _i32([0]), desc, pos=pos[:2])),
    ]
    for kind, f in bad:
        with pytest.raises(kind):
            f()
    from paper_2608_00531_gb300._lib import CureError
    for f in (lambda: cure.rope_desc(24, 1e4), lambda: cure.rope_desc(128, 1.0), lambda: cure.rope_desc(130, 1e4),
              lambda: cure.cure_rope_qkv(q[:, :, :64].contiguous(), None, None, pos, None),
              lambda: cure.cure_rope_qkv(q, None, None, pos, desc, eps=-1.0),
              lambda: cure.cure_rope_qkv(q[:1].expand(4, 8, D), None, None, pos, desc)):
        with pytest.raises(CureError):
            f()
    assert cure.cure_device_error() == 0
