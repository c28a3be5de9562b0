"""A cache held in 8 bits (e4m3 codes, a scale for each block of 16 slots and head): its append, the attention of packed
rows and of trees over it, and the commit of an accepted path, against their definitions in 64 bits.

Codes.  With s a power of two x / s is exact in float32, so that of V rows (and of K rows that are neither normed nor
rotated), and of values that a block held before, codes and scales must be the definition's to the bit.  A rotated K
value is off by the angle's error (2^-21 of a turn: 2^-18 of the pair's size) and some roundings of 2^-24; its code by
half a step more: 2^-4 of the value, or 2^-10 s where the value is below 2^-6 s.

Attention.  o = sum_j w_j v_j with weights w_j of sum 1.
  - q in two e4m3 parts is off by 2^-10 of a value that its row's power of two (above amax / 448, at most amax / 224)
    scales: at most 2^-10 amax / 224 < 2^-17 amax; 256 float32 products and sums: 256 * 2^-24 = 2^-16 of the sum of their sizes,
    which is at most (1 + 2^-4) times that of q's and k's. With both a score is off by
      e = scale (2^-17 amax(q) sum_d |k_d| + 2^-15 sum_d |q_d k_d|),
    a weight by a factor of exp(2 e) at most.
  - ex2 and the exponent's sum (of numbers below 2^8: 2^-17 ln 2) are off by less than 2^-16 of a weight, P' by its
    rounding to fp16, 2^-11; the sum of weights, the joins and the PV sums by less than 2^-14.
  - a weight below the smallest fp16 step, 2^-32 of the largest term's weight w v_scale: 2^-32 * 448 * keys of it at most
  - the output's rounding: 2^-8 |o|
In all |got - o| <= 2^-8 |o| + (2^-11 + 2^-13 + 4 e) sum_j w_j |v_j| + 2^-23 keys max_j (w_j vs_j), for e below 1/4.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
D, BLK = 128, 16
SCALE = 1.0 / math.sqrt(D)
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def cure():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2608_00531_gb300 import cure as c
    torch.cuda.set_device(DEV)
    return c


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Cache:
    """K and V of a layer in 8 bits. Unused slots hold NaN codes, unused blocks NaN scales."""

    def __init__(self, cure, ends, Hkv, ps, seed, slack=0, pow2=True):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rng = np.random.default_rng(seed)
        B, self.Hkv, self.ps = len(ends), Hkv, ps
        if ps == 0:
            self.cap = max(max(ends), 1) + slack
            self.blocks = -(-self.cap // BLK)
            shape, scales, self.table = (B, self.cap, Hkv, D), (B, self.blocks, Hkv), None
            self.kv = cure.kv_desc(Hkv, D, self.cap)
        else:
            need = [-(-e // ps) for e in ends]
            pages = sum(need) + 2
            perm = rng.permutation(pages).astype(np.int32)
            t = np.full((B, max(max(need), 1) + slack), -1, dtype=np.int32)
            o = 0
            for b, m in enumerate(need):
                t[b, :m] = perm[o:o + m]
                o += m
            self.table = t
            shape, scales = (pages, ps, Hkv, D), (pages, ps // BLK, Hkv)
            self.kv = cure.kv_desc(Hkv, D, t.shape[1], block_table=torch.from_numpy(t).to(DEV), page_size=ps,
                                   num_pages=pages)
        assert cure.kv8_scale_shape(self.kv, B) == scales
        self.codes = [torch.full(shape, 0x7f, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2)]
        self.scales = [torch.full(scales, math.nan, device=DEV) for _ in range(2)]
        for b, e in enumerate(ends):
            for codes, scale in zip(self.codes, self.scales):
                x = torch.empty(e, Hkv, D, device=DEV).normal_(0.0, 96.0, generator=g).clamp_(-448, 448).to(E4M3)
                codes.view(-1, Hkv, D).view(torch.uint8)[self.rows(b, range(e))] = x.view(torch.uint8)
                n = -(-e // BLK)
                s = torch.empty(n, Hkv, device=DEV).uniform_(-9.0, -5.0, generator=g)
                scale.view(-1, Hkv)[self.places(b, range(n))] = torch.exp2(s.round() if pow2 else s)

    def rows(self, b, slots):
        t = np.asarray(list(slots), dtype=np.int64)
        at = b * self.cap + t if self.table is None else self.table[b][t // self.ps].astype(np.int64) * self.ps + t % self.ps
        return torch.from_numpy(at).to(DEV)

    def places(self, b, blocks):
        t = np.asarray(list(blocks), dtype=np.int64)
        if self.table is None:
            return torch.from_numpy(b * self.blocks + t).to(DEV)
        per = self.ps // BLK
        return torch.from_numpy(self.table[b][t // per].astype(np.int64) * per + t % per).to(DEV)

    def values(self, which, b, end):
        """[end][Hkv][D] in 64 bits, and the scales [end][Hkv]."""
        x = self.codes[which].view(-1, self.Hkv, D)[self.rows(b, range(end))].double()
        s = self.scales[which].view(-1, self.Hkv)[self.places(b, range(-(-end // BLK)))].double()
        s = s.repeat_interleave(BLK, 0)[:end]
        return x * s[..., None], s

    def copy(self):
        return [t.view(torch.uint8).clone() for t in self.codes], [t.clone() for t in self.scales]

    def args(self):
        return (*self.codes, *self.scales, self.kv)


def _power_above(x):
    """The least power of two from 2^-40 to 2^40 that is not below x / 448 (64 bits)."""
    p = torch.ldexp(torch.ones(81, dtype=torch.float64), torch.arange(-40, 41)).to(DEV)
    return p[(448.0 * p < x[..., None]).sum(-1).clamp(max=80)]


# ---------------------------------------------------------------- append
def _packed(n, pad):
    return [pad + int(x) for x in np.concatenate([[0], np.cumsum(n)])]


def _check_append(c, before, lens, n, start, want, taken=None, exact=True):
    """Codes and scales of one of K (0) and V (1) after an append of the rows `want` [rows][Hkv][D] in 64 bits."""
    for which, x in enumerate(want):
        codes, scales = before[0][which].clone(), before[1][which].clone()
        H = c.Hkv
        fc, fs = codes.view(-1, H, D), scales.view(-1, H)
        got_c, got_s = c.codes[which].view(torch.uint8), c.scales[which]
        loose = []  # (rows, reference values, scale) of rotated rows
        for b in range(len(n)):
            for blk in range(lens[b] // BLK, -(-(lens[b] + n[b]) // BLK) if n[b] else 0):
                new = [t for t in range(max(lens[b], blk * BLK), min(lens[b] + n[b], blk * BLK + BLK))
                       if taken is None or taken[start[b] + t - lens[b]]]
                if not new:
                    continue
                held = list(range(blk * BLK, min(lens[b], blk * BLK + BLK)))
                place = c.places(b, [blk])[0]
                old = fc[c.rows(b, held)].view(E4M3).double() * fs[place].double()[None, :, None]
                y = x[[start[b] + t - lens[b] for t in new]].double()
                amax = torch.cat([old, y]).nan_to_num(nan=0.0, posinf=math.inf, neginf=-math.inf).abs().amax((0, 2))
                s = _power_above(amax)
                if not (exact or which == 1):  # where the largest value lies within its error of a border
                    near = (got_s.view(-1, H)[place].double() == _power_above(amax * (1 + 2.0 ** -17))) | (
                        got_s.view(-1, H)[place].double() == _power_above(amax * (1 - 2.0 ** -17)))
                    assert torch.all(near)
                    s = got_s.view(-1, H)[place].double()
                fs[place] = s.float()
                fc[c.rows(b, held)] = (old / s[None, :, None]).float().to(E4M3).view(torch.uint8)
                q = (y / s[None, :, None]).float().clamp(-448, 448).to(E4M3).view(torch.uint8)
                if exact or which == 1:
                    fc[c.rows(b, new)] = q
                else:
                    fc[c.rows(b, new)] = got_c.view(-1, H, D)[c.rows(b, new)]
                    loose.append((c.rows(b, new), y, s))
        assert torch.equal(got_s.nan_to_num(nan=-1.0), scales.nan_to_num(nan=-1.0)), which
        assert torch.equal(got_c, codes), which
        for at, y, s in loose:
            v = got_c.view(-1, H, D)[at].view(E4M3).double() * s[None, :, None]
            size = y.abs().amax(-1, keepdim=True)
            tol = torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * s[None, :, None]) + 2.0 ** -17 * size
            assert torch.all((v - y).abs() <= tol)


def _rotated(x, pos, rot, base, style, axis, norm=None, eps=1e-6):
    """Rows x [n][H][D] at positions pos [axes][n], in 64 bits."""
    x = x.double()
    if norm is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * norm.double()
    y, h = x.clone(), rot // 2
    for i in range(h):
        a = pos[axis[i]].double() * base ** (-2.0 * i / rot)
        c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
        p, q = (i, i + h) if style == "half" else (2 * i, 2 * i + 1)
        y[..., p], y[..., q] = x[..., p] * c - x[..., q] * s, x[..., q] * c + x[..., p] * s
    return y


LENS, ROWS = [0, 15, 16, 17, 0, 31, 100, 5, 64], [1, 1, 1, 16, 0, 33, 140, 12, 15]


@pytest.mark.parametrize("ps", [0, 16, 32, 64])
@pytest.mark.parametrize("Hq,Hkv", [(28, 4), (3, 3), (0, 1)])
def test_append_exact(cure, ps, Hq, Hkv):
    """Without norms and rotation: every code and scale, and everything else as it was."""
    c = Cache(cure, [a + b for a, b in zip(LENS, ROWS)], Hkv, ps, 7 + ps + Hq, slack=1)
    g = torch.Generator(device=DEV).manual_seed(ps)
    start = _packed(ROWS, 3)
    rows = start[-1] + 2
    k, v = (torch.empty(rows, Hkv, D, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g) for _ in range(2))
    k *= torch.exp2(torch.randint(-6, 7, (rows, 1, 1), device=DEV, generator=g).float()).bfloat16()  # scales that change
    v[:, :, 64:] = 0  # (also blocks of zeros)
    q = torch.randn(rows, Hq, D, device=DEV).bfloat16() if Hq else None
    before = c.copy()
    out = cure.cure_append_kv8(k, v, *c.args(), _i32(start), _i32(LENS), None, q=q)
    assert (out is None) if q is None else torch.equal(out[start[0]:start[-1]], q[start[0]:start[-1]])
    _check_append(c, before, LENS, ROWS, start, (k, v))
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("n", [[700, 9, 0, 801], [3] * 500, [1] * 300, [1], [17, 1, 16]])
@pytest.mark.parametrize("Hq,Hkv", [(28, 4), (5, 5), (2, 2)])
def test_append_many_and_few_rows(cure, n, Hq, Hkv):
    """Rows without a rotation: the values themselves, whatever heads meet at a time."""
    lens = [(7 * b) % 37 for b in range(len(n))]
    c = Cache(cure, [a + b for a, b in zip(lens, n)], Hkv, 16, len(n) + Hkv)
    start = _packed(n, 0)
    g = torch.Generator(device=DEV).manual_seed(6)
    k, v, q = (torch.empty(start[-1], h, D, dtype=torch.bfloat16, device=DEV).normal_(0.0, 2.0, generator=g)
               for h in (Hkv, Hkv, Hq))
    before = c.copy()
    got = cure.cure_append_kv8(k, v, *c.args(), _i32(start), _i32(lens), None, q=q)
    _check_append(c, before, lens, n, start, (k.double(), v.double()))
    assert torch.equal(got, q) and cure.cure_device_error() == 0


@pytest.mark.parametrize("style,rot,norm,axes", [("half", 128, False, None), ("interleaved", 128, True, None),
                                                 ("half", 64, True, "runs"), ("interleaved", 96, False, "turns"),
                                                 ("half", 128, True, "turns")])
def test_append_rotated(cure, style, rot, norm, axes):
    """Norms, rotation, parts of a fused projection, positions on three axes, rows that hold no token."""
    Hq, Hkv, base = 8, 2, 500000.0
    c = Cache(cure, [a + b for a, b in zip(LENS, ROWS)], Hkv, 16, rot, slack=1)
    g = torch.Generator(device=DEV).manual_seed(rot + norm)
    start = _packed(ROWS, 1)
    rows = start[-1] + 1
    qkv = torch.empty(rows, (Hq + 2 * Hkv) * D, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g).unflatten(
        -1, (-1, D))
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    w = [(1 + 0.1 * torch.randn(D, device=DEV, generator=g)).bfloat16() if norm else None for _ in range(2)]
    taken, pos, desc, axis = None, None, None, [0] * 64
    if axes is None:
        at = torch.zeros(1, rows, dtype=torch.long, device=DEV)
        for b, L in enumerate(LENS):
            at[0, start[b]:start[b + 1]] = L + torch.arange(ROWS[b], device=DEV)
    else:
        axis = [i % 3 for i in range(64)] if axes == "turns" else [0] * 10 + [1] * 12 + [2] * 42
        desc = cure.rope_axes(axis[:rot // 2])
        at = torch.randint(0, 5000, (3, rows), device=DEV, generator=g)
        taken = [True] * rows
        for r, a in ((start[3] + 4, 0), (start[5], 1), (start[6] + 139, 2), (start[8], 1)):
            at[a, r], taken[r] = -1, False
        pos = at.to(torch.int32)
    before = c.copy()
    out = torch.full((rows, Hq, D), 3.5, dtype=torch.bfloat16, device=DEV)
    cure.cure_append_kv8(k, v, *c.args(), _i32(start), _i32(LENS), cure.rope_desc(rot, base, style=style), q=q, pos=pos,
                         axes=desc, q_norm=w[0], k_norm=w[1], out=out)
    want_k, want_q = _rotated(k, at, rot, base, style, axis, w[1]), _rotated(q, at, rot, base, style, axis, w[0])
    _check_append(c, before, LENS, ROWS, start, (want_k, v), taken, exact=False)
    for r in range(rows):
        if start[0] <= r < start[-1] and (taken is None or taken[r]):
            size = want_q[r].abs().amax(-1, keepdim=True)
            assert torch.all((out[r].double() - want_q[r]).abs() <= 2.0 ** -8 * want_q[r].abs() + 2.0 ** -17 * size)
        else:
            assert torch.all(out[r] == 3.5)
    assert cure.cure_device_error() == 0


def test_append_token_by_token(cure):
    """Blocks that grow by one token a call, with a scale that rises and one that shrinks when a larger row is replaced."""
    Hkv = 2
    c = Cache(cure, [40], Hkv, 16, 1)
    for t in range(37):
        x = torch.randn(1, Hkv, D, device=DEV).bfloat16() * 2.0 ** (t % 7 - 3)
        before = c.copy()
        cure.cure_append_kv8(x, 3 * x, *c.args(), _i32([0, 1]), _i32([t]), None)
        _check_append(c, before, [t], [1], [0, 1], (x, 3 * x))
    # the same slot again with a smaller row: the block is what it holds now
    x = torch.full((1, Hkv, D), 1e-3, device=DEV).bfloat16()
    before = c.copy()
    cure.cure_append_kv8(x, x, *c.args(), _i32([0, 1]), _i32([32]), None)
    _check_append(c, before, [32], [1], [0, 1], (x, x))
    assert cure.cure_device_error() == 0


def test_append_extremes(cure):
    """NaN, infinities, the largest, the smallest and borders of the scale's steps."""
    Hkv = 1
    for value in (0.0, 448.0, 449.0, 450.0, 3.0 * 2.0 ** 120, 2.0 ** -133, 1.75, math.inf, -math.inf, 3.5 * 2.0 ** -40):
        c = Cache(cure, [20], Hkv, 0, 3)
        x = torch.zeros(20, Hkv, D, dtype=torch.bfloat16, device=DEV)
        x[3, 0, 5], x[17, 0, 9] = value, -value
        before = c.copy()
        cure.cure_append_kv8(x, x, *c.args(), _i32([0, 20]), _i32([0]), None)
        _check_append(c, before, [0], [20], [0, 20], (x, x))
    c = Cache(cure, [16], Hkv, 0, 3)
    x = torch.randn(16, Hkv, D, device=DEV).bfloat16()
    x[2, 0, 7] = math.nan
    cure.cure_append_kv8(x, x, *c.args(), _i32([0, 16]), _i32([0]), None)
    y, _ = c.values(0, 0, 16)
    assert torch.isnan(y[2, 0, 7]) and int(torch.isnan(y).sum()) == 1
    assert float(c.scales[0][0, 0, 0]) == float(_power_above(x.double().nan_to_num(0.0).abs().amax()))
    assert cure.cure_device_error() == 0


def test_append_errors(cure):
    """Slots past the capacity, missing pages, a row_start that does not ascend: left out and reported, the rest written."""
    Hkv = 2
    x = torch.randn(40, Hkv, D, device=DEV).bfloat16()
    c = Cache(cure, [40, 20], Hkv, 0, 5)  # capacity 40
    before = c.copy()
    cure.cure_append_kv8(x[:30], x[:30], *c.args(), _i32([0, 20, 30]), _i32([25, 3]), None)
    assert cure.cure_device_error() == cure.DEVERR_SLOT
    _check_append(c, before, [25, 3], [15, 10], [0, 20, 30], (x, x))
    c = Cache(cure, [64, 20], Hkv, 16, 6)
    c.table[0, 1], c.table[0, 3] = -1, 99
    c.kv._keep.copy_(torch.from_numpy(c.table))
    before = c.copy()
    cure.cure_append_kv8(x, x, *c.args(), _i32([0, 40, 40]), _i32([10, 0]), None)
    assert cure.cure_device_error() == cure.DEVERR_PAGE
    c.table[0, 1] = c.table[0, 0]  # (for the reference: blocks 0 and 2 are written)
    taken = [10 + r < 16 or 32 <= 10 + r < 48 for r in range(40)]
    c.table[0, 3] = c.table[0, 2]
    _check_append(c, before, [10, 0], [40, 0], [0, 40, 40], (x, x), taken)
    cure.cure_append_kv8(x, x, *c.args(), _i32([0, 30, 20]), _i32([0, 0]), None)
    cure.cure_device_error()
    cure.cure_append_kv8(x, x, *c.args(), _i32([-5, 3, 20]), _i32([0, 0]), None)
    assert cure.cure_device_error() & cure.DEVERR_NODES


def test_append_rows_without_tokens_need_no_place(cure):
    """Trees near the capacity, in place: rows behind a sequence's nodes may lie behind the cache and its pages."""
    Hkv, n_max = 2, 20
    for ps in (0, 16):
        c = Cache(cure, [40, 33], Hkv, ps, 17 + ps)
        lens, nodes = [c.kv.max_len * max(ps, 1) - 5, 28], [5, 5]
        if ps:
            c.table[1, 2:] = -1  # (sequence 1: 33 tokens in 3 pages, of which 2 hold what is written)
            c.kv._keep.copy_(torch.from_numpy(c.table))
            nodes[1] = 4
        x = torch.randn(2 * n_max, Hkv, D, device=DEV).bfloat16()
        pos = torch.full((2, n_max), -1, dtype=torch.int32, device=DEV)
        for b in range(2):
            pos[b, :nodes[b]] = lens[b]
        before = c.copy()
        cure.cure_append_kv8(x, x, *c.args(), _i32([0, n_max, 2 * n_max]), _i32(lens), None, pos=pos)
        assert cure.cure_device_error() == 0
        taken = [r % n_max < nodes[r // n_max] for r in range(2 * n_max)]
        _check_append(c, before, lens, nodes, [0, n_max, 2 * n_max], (x, x), taken)


# ---------------------------------------------------------------- attention
def _attention_ref(x, q, b, end, mask):
    """Rows q [n][Hq][D] over the first `end` keys of sequence b (mask [n][end]: not seen): output and tolerance."""
    c, Hq = x["cache"], q.shape[1]
    G = Hq // c.Hkv
    k, _ = c.values(0, b, end)
    v, vs = c.values(1, b, end)
    outs, tols = [], []
    for h in range(Hq):
        kk, vv, qq = k[:, h // G], v[:, h // G], q[:, h].double()
        s = (qq @ kk.T * SCALE).masked_fill(mask, -math.inf)
        w = torch.softmax(s, -1).nan_to_num(0.0)
        e = SCALE * (2.0 ** -17 * qq.abs().amax(-1, keepdim=True) * kk.abs().sum(-1)[None] + 2.0 ** -15 * (qq.abs() @ kk.abs().T))
        e = e.masked_fill(mask, 0.0).amax(-1, keepdim=True) if end else torch.zeros(len(qq), 1, device=DEV)
        assert float(e.max()) < 0.25 if e.numel() else True
        o = w @ vv
        big = (w * vs[:, h // G][None]).amax(-1, keepdim=True) if end else torch.zeros(len(qq), 1, device=DEV)
        outs.append(o)
        tols.append(2.0 ** -8 * o.abs() + (2.0 ** -11 + 2.0 ** -13 + 4 * e) * (w @ vv.abs()) + 2.0 ** -23 * end * big)
    return torch.stack(outs, 1), torch.stack(tols, 1)


def _prompt(cure, lens, n, Hq, Hkv, ps, seed, std=1.5, pad=0, slack=0, pow2=True):
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    start = _packed(n, pad)
    q = torch.empty(start[-1] + pad, Hq, D, dtype=torch.bfloat16, device=DEV).normal_(0.0, std, generator=g)
    c = Cache(cure, [a + b for a, b in zip(lens, n)], Hkv, ps, seed, slack, pow2)
    return dict(cache=c, q=q, lens=lens, n=n, start=start, row_start=_i32(start), cache_len=_i32(lens))


def _run(cure, x, out=None, **kw):
    if out is None:
        out = torch.full_like(x["q"], 3.5)
    return cure.cure_prompt_attn8(x["q"], *x["cache"].args(), x["row_start"], x["cache_len"], SCALE, out=out, **kw)


def _check(x, got, rows=None):
    assert torch.all(got[:x["start"][0]] == 3.5) and torch.all(got[x["start"][-1]:] == 3.5)
    for b, (n, L) in enumerate(zip(x["n"], x["lens"])):
        pick = range(n) if rows is None else sorted({r % n for r in rows if -n <= r < n} if n else set())
        i = torch.tensor(list(pick), dtype=torch.long, device=DEV)
        if not len(i):
            continue
        mask = torch.arange(L + n, device=DEV)[None] > (L + i)[:, None]
        o, tol = _attention_ref(x, x["q"][x["start"][b] + i], b, L + n, mask)
        off = (got[x["start"][b] + i].double() - o).abs()
        assert torch.all(off <= tol), (b, float((off / tol).max()))


@pytest.mark.parametrize("Hq,Hkv", [(28, 4), (8, 2), (3, 3), (5, 1)])
@pytest.mark.parametrize("ps", [0, 16, 32, 64])
def test_prompt_ragged(cure, ps, Hq, Hkv):
    """Whole prompts, chunks behind cached tokens, single tokens, empty sequences; rows around the batch's ends
    unwritten; NaN codes and scales wherever no key lies."""
    x = _prompt(cure, [0, 130, 0, 5, 127, 300, 64], [1, 40, 0, 123, 1, 129, 256], Hq, Hkv, ps, 100 + ps + Hq, pad=3, slack=1)
    _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 36, 37, 127, 128, 129, 255, 256, 257, 300])
def test_prompt_lengths_around_the_tiles(cure, n):
    for Hq, Hkv, L in ((28, 4, 0), (2, 2, 0), (8, 1, 127), (16, 1, 1)):
        x = _prompt(cure, [L], [n], Hq, Hkv, 16, n + Hq, pow2=n % 2 == 0)
        _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("G", [1, 2, 6, 9, 33, 64, 65, 127, 128])
def test_prompt_group_sizes(cure, G):
    x = _prompt(cure, [70, 0], [9, 131], G, 1, 32, G)
    _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("ps", [0, 16])
def test_prompt_long(cure, ps):
    """A long prompt and a chunk far into a long sequence, some rows of them; sharp and flat scores, any scales."""
    for std, pow2 in ((0.02, True), (1.5, False), (4.0, True)):
        x = _prompt(cure, [0, 9000], [5003, 700], 14, 2, ps, 7, std=std, pow2=pow2)
        _check(x, _run(cure, x), rows=[0, 1, 63, 127, 128, 129, 511, 640, 2047, 3333, 4999, -1, -2])
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("batch,L", [(1, 40000), (3, 20000), (64, 3000), (200, 300), (256, 1)])
def test_single_tokens(cure, batch, L):
    """Single tokens: few long sequences (cut into parts) to many short ones."""
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(0, L + 1, batch)]
    lens[0] = L
    x = _prompt(cure, lens, [1] * batch, 7, 1, 16, batch, std=2.0)
    _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


def test_few_tokens(cure):
    for n in (2, 5, 8, 18, 19):
        x = _prompt(cure, [700, 5000, 0, 129], [n, 1, n, n], 28, 4, 32, n)
        _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


def test_few_rows_on_average(cure):
    """Batches whose rows are few on average, all of them in one sequence: more units than one of it."""
    for n in ([16, 0, 0, 0, 0, 0, 0, 0], [0, 9, 0, 1, 0, 2, 0, 0], [100] + [0] * 7, [0, 37, 0, 0, 0, 1, 0, 100]):
        for Hq, Hkv in ((14, 2), (3, 3)):
            x = _prompt(cure, [700, 5, 0, 129, 0, 16, 0, 40], n, Hq, Hkv, 16, sum(n) + Hq)
            _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("ps", [0, 16, 64])
@pytest.mark.parametrize("batch,Hq,Hkv,L", [(90, 28, 4, 300), (256, 32, 8, 120), (200, 32, 2, 40), (256, 5, 5, 700),
                                            (256, 32, 32, 33), (256, 64, 8, 1)])
def test_many_short_sequences(cure, ps, batch, Hq, Hkv, L):
    """More units than there are warps, or fewer, of sequences of a few keys; none to a few rows each."""
    rng = np.random.default_rng(batch + ps)
    most = 16 // (Hq // Hkv)
    n = [int(v) for v in np.minimum(rng.choice([0, 1, 1, 1, 2, 3], batch), most)]
    n[0], n[-1] = 1, 0
    x = _prompt(cure, [int(v) for v in rng.integers(0, L + 1, batch)], n, Hq, Hkv, ps, batch + L, std=2.0, pad=2,
                pow2=bool(L % 2))
    got = _run(cure, x).clone()
    _check(x, got)
    assert cure.cure_device_error() == 0
    size = cure.cure_prompt_attn8_workspace_size(x["q"].shape[0], batch, Hq, x["cache"].kv)
    ws, out, graph = torch.empty(size, dtype=torch.uint8, device=DEV), torch.full_like(x["q"], 3.5), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _run(cure, x, out=out, workspace=ws)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[x["start"][0]:x["start"][-1]], got[x["start"][0]:x["start"][-1]])
    if ps:  # a sequence without its first page
        old = int(x["cache"].table[0, 0])
        x["cache"].kv._keep[0, 0] = -1
        bad = _run(cure, x)
        assert cure.cure_device_error() == cure.DEVERR_PAGE
        x["cache"].kv._keep[0, 0] = old
        assert torch.equal(bad[x["start"][1]:], got[x["start"][1]:]) and torch.isfinite(bad[x["start"][0]:x["start"][1]]).all()


def test_outputs_aligned_to_16_bytes(cure):
    """Outputs that begin 16 bytes behind a 32-byte boundary, in each form of the attention."""
    for lens, n, Hq in (([300, 0], [200, 70], 8), ([300, 1000, 50], [1, 1, 1], 8), ([1000, 30], [9, 12], 8)):
        x = _prompt(cure, lens, n, Hq, 2, 16, 5)
        buf = torch.full((x["q"].numel() + 8,), 3.5, dtype=torch.bfloat16, device=DEV)
        out = buf[8:].view(x["q"].shape)
        assert out.data_ptr() % 32 == 16
        _check(x, _run(cure, x, out=out))
        assert torch.all(buf[:8] == 3.5)
    x = _tree(cure, [100, 500], [20, 9], 20, 8, 2, 16, 3)
    want = _run_tree(cure, x)
    buf = torch.full((x["q"].numel() + 8,), 3.5, dtype=torch.bfloat16, device=DEV)
    got = cure.cure_tree_attn8(x["q"], *x["cache"].args(), x["cache_len"], x["n_nodes"], x["anc"], SCALE,
                               out=buf[8:].view(x["q"].shape))
    assert torch.equal(got, want) and torch.all(buf[:8] == 3.5) and cure.cure_device_error() == 0


def test_caches_past_32_bits(cure):
    """Pages whose codes lie 2^32 bytes and more behind the cache's beginning: append, attention of each form, commit."""
    Hkv, ps, pages = 8, 64, 70000  # 4.6 GB of codes each
    lens, n = [100, 200, 0], [30, 1, 300]
    small = Cache(cure, [160, 260, 400], Hkv, ps, 4)
    c = Cache.__new__(Cache)
    c.Hkv, c.ps, c.table = Hkv, ps, small.table.copy()
    c.table[c.table >= 0] += pages - small.codes[0].shape[0]
    c.codes = [torch.empty(pages, ps, Hkv, D, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2)]
    c.scales = [torch.empty(pages, ps // BLK, Hkv, device=DEV) for _ in range(2)]
    assert int(c.table[0, 0]) * ps * Hkv * D > 2 ** 32
    k = small.codes[0].shape[0]
    for w in (0, 1):
        c.codes[w].view(torch.uint8)[-k:] = small.codes[w].view(torch.uint8)
        c.scales[w][-k:] = small.scales[w]
    c.kv = cure.kv_desc(Hkv, D, c.table.shape[1], block_table=torch.from_numpy(c.table).to(DEV), page_size=ps, num_pages=pages)
    start = _packed(n, 0)
    x = torch.randn(start[-1], Hkv, D, device=DEV).bfloat16()
    tree = torch.randn(1, 3, 9, Hkv, D, device=DEV).bfloat16()
    acc = dict(path_nodes=_i32([[0, 1, 2, -1, -1, -1]] * 3), accept_len=_i32([2] * 3), diverge_depth=_i32([-1] * 3),
               out_tokens=_i32([[1] * 6] * 3))
    q = torch.randn(start[-1], 16, D, device=DEV).bfloat16()
    t = _tree(cure, [10, 20, 30], [9, 9, 9], 9, 16, Hkv, ps, 9)
    outs = []
    for at in (small, c):
        cure.cure_append_kv8(x, -x, *at.args(), _i32(start), _i32(lens), None)
        outs.append([cure.cure_prompt_attn8(q, *at.args(), _i32(start), _i32(lens), SCALE),
                     cure.cure_prompt_attn8(q[:3].contiguous(), *at.args(), _i32([0, 1, 2, 3]), _i32(lens), SCALE),
                     cure.cure_tree_attn8(t["q"], *at.args(), _i32(lens), t["n_nodes"], t["anc"], SCALE)])
        cure.cure_resync_kv8([at.codes[0]], [at.codes[1]], [at.scales[0]], [at.scales[1]], at.kv, tree, tree, acc,
                             _i32(lens), 4)
    assert cure.cure_device_error() == 0
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    for w in (0, 1):
        assert torch.equal(c.codes[w].view(torch.uint8)[-k:], small.codes[w].view(torch.uint8))
        assert torch.equal(c.scales[w][-k:].nan_to_num(nan=-1.0), small.scales[w].nan_to_num(nan=-1.0))


def test_two_calls_at_once(cure):
    """Calls of each form on two streams, with workspaces of their own."""
    forms = [_prompt(cure, [0, 3000], [700, 5], 28, 4, 16, 1), _prompt(cure, [4000, 9000, 20], [1, 1, 1], 28, 4, 16, 2)]
    want = [_run(cure, x).clone() for x in forms]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.full_like(x["q"], 3.5) for x in forms] for _ in streams]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o in zip(streams, outs):
            for x, out in zip(forms, o):
                cure.cure_prompt_attn8(x["q"], *x["cache"].args(), x["row_start"], x["cache_len"], SCALE, out=out, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(o, want))
    assert cure.cure_device_error() == 0


def test_scales_far_apart(cure):
    """Blocks whose values differ by 2^40, the large ones seen by none of the weight: relative to each row's own terms."""
    x = _prompt(cure, [600], [3], 4, 1, 0, 11)
    c = x["cache"]
    q = torch.zeros_like(x["q"])
    q[:, :, 0] = 40.0
    x["q"] = q
    k = c.codes[0].view(-1, 1, D).float()
    k[:, :, 0] = 0
    for blk, (ks0, vs) in enumerate([(-1.0, 2.0 ** 20)] + [(1.0, 2.0 ** -20)] * 37):
        at = slice(blk * BLK, blk * BLK + BLK)
        k[at, :, 0] = 200.0 * ks0
        c.scales[0].view(-1, 1)[blk] = 2.0 ** -4
        c.scales[1].view(-1, 1)[blk] = vs
    c.codes[0].view(torch.uint8).copy_(k.to(E4M3).view(c.codes[0].shape).view(torch.uint8))
    _check(x, _run(cure, x))
    # scales out of their range count as its ends, NaN as the lower one
    c.scales[1].view(-1)[1], c.scales[1].view(-1)[2] = math.nan, 0.0
    got = _run(cure, x)
    c.scales[1].view(-1)[1] = c.scales[1].view(-1)[2] = 2.0 ** -40
    assert torch.equal(got, _run(cure, x))


def test_prompt_errors(cure):
    """A sequence that does not fit, a row_start out of range, missing pages: reported, the others as ever."""
    x = _prompt(cure, [30, 200], [10, 20], 8, 2, 16, 12)
    full = _run(cure, x).clone()
    long = dict(x, cache_len=_i32([30, 100000]))
    got = _run(cure, long)
    assert cure.cure_device_error() == cure.DEVERR_SLOT
    assert torch.equal(got[:10], full[:10]) and torch.all(got[10:] == 3.5)
    got = _run(cure, dict(x, row_start=_i32([0, 10, 31])))
    assert cure.cure_device_error() == cure.DEVERR_NODES
    assert torch.equal(got[:10], full[:10]) and torch.all(got[10:] == 3.5)
    c = x["cache"]
    for page in (-1, 10 ** 6):  # the second page of sequence 0: zeros
        old = int(c.table[0, 1])
        c.kv._keep[0, 1] = page
        got = _run(cure, x)
        assert cure.cure_device_error() == cure.DEVERR_PAGE
        c.kv._keep[0, 1] = old
        y = dict(x, cache=Cache(cure, [40, 220], 2, 16, 12))
        for codes in y["cache"].codes:
            codes.view(torch.uint8)[old] = 0
        for s in y["cache"].scales:
            s[old] = 1.0
        o, tol = _attention_ref(y, x["q"][:10], 0, 40, torch.arange(40, device=DEV)[None] > 30 + torch.arange(10, device=DEV)[:, None])
        assert torch.all((got[:10].double() - o).abs() <= tol)


def test_same_bits_streams_and_graphs(cure):
    """Call after call, on another stream, in two graphs with workspaces of their own."""
    x = _prompt(cure, [0, 5000, 77], [600, 3, 1], 28, 4, 16, 21)
    first = _run(cure, x).clone()
    for _ in range(3):
        assert torch.equal(_run(cure, x), first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.full_like(x["q"], 3.5)
    torch.cuda.synchronize()
    got = cure.cure_prompt_attn8(x["q"], *x["cache"].args(), x["row_start"], x["cache_len"], SCALE, out=out, stream=s)
    s.synchronize()
    assert torch.equal(got, first)
    size = cure.cure_prompt_attn8_workspace_size(x["q"].shape[0], 3, 28, x["cache"].kv)
    graphs, outs = [], []
    for _ in range(2):
        ws, o = torch.empty(size, dtype=torch.uint8, device=DEV), torch.full_like(x["q"], 3.5)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _run(cure, x, out=o, workspace=ws)
        graphs.append((g, ws))
        outs.append(o)
    for _ in range(3):
        graphs[0][0].replay()
        graphs[1][0].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], first) and torch.equal(outs[1], first) and cure.cure_device_error() == 0


# ---------------------------------------------------------------- trees
def _tree(cure, lens, nodes, n_max, Hq, Hkv, ps, seed, empty=False):
    g = torch.Generator(device=DEV).manual_seed(seed + 2)
    rng = np.random.default_rng(seed)
    B, W = len(lens), (n_max + 63) // 64
    c = Cache(cure, [a + b for a, b in zip(lens, nodes)], Hkv, ps, seed)
    q = torch.empty(B, n_max, Hq, D, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.5, generator=g)
    seen = np.zeros((B, n_max, n_max), dtype=bool)
    for b, n in enumerate(nodes):
        for j in range(n):
            parent = int(rng.integers(0, j)) if j else -1
            if parent >= 0:
                seen[b, j] = seen[b, parent]
            seen[b, j, j] = True
        if empty:
            seen[b, :: 3] = False  # rows that see no node (and, without cached tokens, no key)
    anc = np.zeros((B, n_max, W), dtype=np.uint64)
    for w in range(W):
        for a in range(64 * w, min(n_max, 64 * w + 64)):
            anc[:, :, w] |= seen[:, :, a].astype(np.uint64) << np.uint64(a - 64 * w)
    return dict(cache=c, q=q, lens=lens, n=nodes, seen=seen, cache_len=_i32(lens), n_nodes=_i32(nodes),
                anc=torch.from_numpy(anc.view(np.int64)).to(DEV))


def _run_tree(cure, x, **kw):
    return cure.cure_tree_attn8(x["q"], *x["cache"].args(), x["cache_len"], x["n_nodes"], x["anc"], SCALE,
                                out=torch.full_like(x["q"], 3.5), **kw)


def _check_tree(x, got):
    for b, (n, L) in enumerate(zip(x["n"], x["lens"])):
        mask = torch.zeros(n, L + n, dtype=torch.bool, device=DEV)
        mask[:, L:] = ~torch.from_numpy(x["seen"][b, :n, :n]).to(DEV)
        o, tol = _attention_ref(x, x["q"][b, :n], b, L + n, mask)
        off = (got[b, :n].double() - o).abs()
        assert torch.all(off <= tol), (b, float((off / tol).max()))
        assert torch.all(got[b, n:] == 3.5)


@pytest.mark.parametrize("ps", [0, 16, 64])
@pytest.mark.parametrize("Hq,Hkv", [(28, 4), (8, 2), (2, 2), (128, 1)])
def test_tree(cure, ps, Hq, Hkv):
    x = _tree(cure, [100, 0, 127, 1000, 31, 64], [33, 17, 1, 25, 33, 32], 33, Hq, Hkv, ps, ps + Hq)
    _check_tree(x, _run_tree(cure, x))
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("n_max", [1, 31, 32, 63, 64, 65, 97, 128, 129, 200, 256])
def test_tree_sizes(cure, n_max):
    for L in (0, 1, 90, 128, 6000):
        x = _tree(cure, [L, 40], [n_max, max(1, n_max // 2)], n_max, 7, 1, 16, n_max + L)
        _check_tree(x, _run_tree(cure, x))
    assert cure.cure_device_error() == 0


def test_tree_rows_without_keys(cure):
    for L in ([0, 0], [0, 50]):
        x = _tree(cure, L, [20, 33], 40, 8, 2, 16, 5, empty=True)
        got = _run_tree(cure, x)
        _check_tree(x, got)
        assert torch.all(got[0, 0] == 0)
    assert cure.cure_device_error() == 0


def test_tree_long_batch_and_errors(cure):
    lens = [int(v) for v in np.random.default_rng(3).integers(1000, 9000, 16)]
    x = _tree(cure, lens, [33] * 16, 33, 14, 2, 16, 31)
    full = _run_tree(cure, x).clone()
    _check_tree(x, full)
    for bad in (0, -1, 34):
        got = _run_tree(cure, dict(x, n_nodes=_i32([33, bad] + [33] * 14)))
        assert cure.cure_device_error() == cure.DEVERR_NODES
        assert torch.all(got[1] == 3.5) and torch.allclose(got[2:].float(), full[2:].float(), atol=2e-2, rtol=2e-2)
    got = _run_tree(cure, dict(x, cache_len=_i32([10 ** 6] + lens[1:])))
    assert cure.cure_device_error() == cure.DEVERR_SLOT and torch.all(got[0] == 3.5)


@pytest.mark.parametrize("lens,n_max", [([4096], 25), ([3000, 100, 900, 0] * 4, 33), ([700], 200)])
def test_tree_same_bits_streams_and_graphs(cure, lens, n_max):
    """Call after call, on another stream, in two graphs with workspaces of their own."""
    x = _tree(cure, lens, [n_max] * len(lens), n_max, 28, 4, 16, n_max)
    first = _run_tree(cure, x).clone()
    _check_tree(x, first)
    assert torch.equal(_run_tree(cure, x), first)
    s, out = torch.cuda.Stream(), torch.full_like(x["q"], 3.5)
    torch.cuda.synchronize()
    args = (x["q"], *x["cache"].args(), x["cache_len"], x["n_nodes"], x["anc"], SCALE)
    cure.cure_tree_attn8(*args, out=out, stream=s)
    s.synchronize()
    assert torch.equal(out, first)
    size = cure.cure_tree_attn8_workspace_size(len(lens), n_max, 28, x["cache"].kv)
    graphs, outs = [], []
    for _ in range(2):
        ws, o = torch.empty(size, dtype=torch.uint8, device=DEV), torch.full_like(x["q"], 3.5)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cure.cure_tree_attn8(*args, out=o, workspace=ws)
        graphs.append((g, ws))
        outs.append(o)
    for _ in range(3):
        graphs[0][0].replay()
        graphs[1][0].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], first) and torch.equal(outs[1], first) and cure.cure_device_error() == 0


# ---------------------------------------------------------------- commit
@pytest.mark.parametrize("ps", [0, 16, 64])
@pytest.mark.parametrize("K,layers", [(16, 3), (32, 1), (1, 2), (1, 128)])
def test_commit(cure, ps, K, layers):
    """The path's rows as an append of them would write, lengths and replay lists as cure_resync_kv gives them."""
    B, Hkv, n_max = 5, 2, 2 * K + 1
    lens, rng = [0, 15, 16, 100, 37], np.random.default_rng(K)
    cs = [Cache(cure, [L + n_max for L in lens], Hkv, ps, 50 + l) for l in range(layers)]
    for c in cs[1:]:  # one table for all layers
        c.table, c.kv = cs[0].table, cs[0].kv
    tk, tv = (torch.randn(layers, B, n_max, Hkv, D, device=DEV).bfloat16() for _ in range(2))
    a = [int(v) for v in rng.integers(0, K + 1, B)]
    a[0], a[-1] = 0, K
    paths = [[0] + sorted(int(v) for v in rng.choice(np.arange(1, n_max), n, replace=False)) + [-1] * (K + 1 - n) for n in a]
    acc = dict(path_nodes=_i32(paths), accept_len=_i32(a), diverge_depth=_i32([-1, min(1, a[1]) or -1, -1, -1, 1]),
               out_tokens=torch.randint(0, 1000, (B, K + 2), dtype=torch.int32, device=DEV))
    before = [c.copy() for c in cs]
    r = cure.cure_resync_kv8([c.codes[0] for c in cs], [c.codes[1] for c in cs], [c.scales[0] for c in cs],
                             [c.scales[1] for c in cs], cs[0].kv, tk, tv, acc, _i32(lens), K)
    n = [v + 1 for v in a]
    start = _packed(n, 0)
    for l, c in enumerate(cs):
        want = [torch.cat([t[l, b, paths[b][:n[b]]] for b in range(B)]) for t in (tk, tv)]
        _check_append(c, before[l], lens, n, start, want)
    ref = cure.cure_resync_kv([], [], cs[0].kv, None, None, acc, _i32(lens), K)
    for name in ("cache_len", "draft_valid_len", "replay_tokens", "n_replay"):
        assert torch.equal(r[name], ref[name]), name
    # the new lengths over the old ones
    at = _i32(lens)
    r = cure.cure_resync_kv8([c.codes[0] for c in cs], [c.codes[1] for c in cs], [c.scales[0] for c in cs],
                             [c.scales[1] for c in cs], cs[0].kv, tk, tv, acc, at, K, cache_len_out=at)
    assert torch.equal(at, ref["cache_len"]) and cure.cure_device_error() == 0


def test_commit_errors(cure):
    B, Hkv, K, n_max = 2, 1, 4, 9
    c = Cache(cure, [30, 30], Hkv, 0, 9)  # capacity 30
    tk = torch.randn(1, B, n_max, Hkv, D, device=DEV).bfloat16()
    acc = dict(path_nodes=_i32([[0, 1, 99, 3, 4, -1], [0, 1, 2, 3, 4, -1]]), accept_len=_i32([4, 4]),
               diverge_depth=_i32([-1, -1]), out_tokens=_i32([[1] * 6] * 2))
    before = c.copy()
    args = ([c.codes[0]], [c.codes[1]], [c.scales[0]], [c.scales[1]], c.kv, tk, tk, acc)
    cure.cure_resync_kv8(*args, _i32([3, 10]), K)
    assert cure.cure_device_error() == cure.DEVERR_NODES
    rows = torch.cat([tk[0, 0, [0, 1, 1, 3, 4]], tk[0, 1, :5]])
    _check_append(c, before, [3, 10], [5, 5], [0, 5, 10], (rows, rows), [r != 2 for r in range(10)])
    before = c.copy()
    cure.cure_resync_kv8(*args, _i32([3, 27]), K)
    assert cure.cure_device_error() & cure.DEVERR_SLOT
    _check_append(c, before, [3, 27], [5, 3], [0, 5, 10], (rows, rows), [r != 2 for r in range(10)])


# ---------------------------------------------------------------- rotations with several axes
@pytest.mark.parametrize("style,rot,norm,axes", [("half", 128, False, 3), ("interleaved", 128, True, 2), ("half", 32, True, 8),
                                                 ("interleaved", 48, False, 1)])
@pytest.mark.parametrize("rows", [1, 33, 700])
def test_rope_axes(cure, style, rot, norm, axes, rows):
    Hq, Hkv, base = 12, 3, 10000.0
    g = torch.Generator(device=DEV).manual_seed(rows + rot)
    qkv = torch.empty(rows, (Hq + 2 * Hkv) * D, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g).unflatten(
        -1, (-1, D))
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    w = [(1 + 0.1 * torch.randn(D, device=DEV, generator=g)).bfloat16() if norm else None for _ in range(2)]
    axis = [(5 * i + 1) % axes for i in range(rot // 2)]
    axis[0] = axes - 1
    pos = torch.randint(0, 2 ** 20, (axes, rows), dtype=torch.int32, device=DEV, generator=g)
    out_of = sorted({0, rows // 2} - ({0} if rows == 1 else set()))
    for n, r in enumerate(out_of):
        pos[(n + 1) % axes, r] = -1
    outs = [torch.full_like(t, 3.5, memory_format=torch.contiguous_format) for t in (q, k, v)]
    cure.cure_rope_qkv(q, k, v, pos, cure.rope_desc(rot, base, style=style), axes=cure.rope_axes(axis), q_norm=w[0],
                       k_norm=w[1], out=tuple(outs))
    keep = torch.tensor([r not in out_of for r in range(rows)], device=DEV)
    for got, x, weight in ((outs[0], q, w[0]), (outs[1], k, w[1])):
        ref = _rotated(x, pos, rot, base, style, axis, weight)
        tol = 2.0 ** -8 * ref.abs() + 2.0 ** -17 * ref.abs().amax(-1, keepdim=True)
        assert torch.all(((got.double() - ref).abs() <= tol)[keep])
    assert torch.equal(outs[2][keep], v[keep])
    for got in outs:
        assert torch.all(got[~keep] == 3.5)
    # one axis for all pairs: the same bits as the rotation without axes
    if axes == 1:
        plain = cure.cure_rope_qkv(q, k, v, pos[0], cure.rope_desc(rot, base, style=style), q_norm=w[0], k_norm=w[1])
        assert all(torch.equal(a[keep], b[keep]) for a, b in zip(outs, plain))
    assert cure.cure_device_error() == 0


def test_append_axes_is_rope_axes(cure):
    """cure_append_kv with axes writes what cure_rope_qkv with axes gives, at the rows' slots."""
    Hq, Hkv, n, lens = 8, 2, [5, 0, 40], [3, 9, 100]
    start = _packed(n, 0)
    g = torch.Generator(device=DEV).manual_seed(1)
    q, k, v = (torch.empty(start[-1], h, D, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g) for h in (Hq, Hkv, Hkv))
    pos = torch.randint(0, 3000, (3, start[-1]), dtype=torch.int32, device=DEV, generator=g)
    pos[1, 7] = -1
    rope, axes = cure.rope_desc(128, 1e6), cure.rope_axes([0] * 16 + [1] * 24 + [2] * 24)
    kc, vc = (torch.full((3, 150, Hkv, D), 3.5, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    qo = torch.full_like(q, 3.5)
    cure.cure_append_kv(k, v, kc, vc, cure.kv_desc(Hkv, D, 150), _i32(start), _i32(lens), rope, q=q, pos=pos, axes=axes, out=qo)
    wq, wk, wv = (torch.full_like(t, 3.5) for t in (q, k, v))
    cure.cure_rope_qkv(q, k, v, pos, rope, axes=axes, out=(wq, wk, wv))
    assert torch.equal(qo, wq)
    for b in range(3):
        assert torch.equal(kc[b, lens[b]:lens[b] + n[b]], wk[start[b]:start[b + 1]])
        assert torch.equal(vc[b, lens[b]:lens[b] + n[b]], wv[start[b]:start[b + 1]])
        assert torch.all(kc[b, :lens[b]] == 3.5) and torch.all(kc[b, lens[b] + n[b]:] == 3.5)
    assert cure.cure_device_error() == 0


# ---------------------------------------------------------------- together
def test_prompt_then_steps(cure):
    """Prompts with images through PromptPass, then two repair-verify steps, all over caches in 8 bits: each stage's
    output against the definition on what the caches hold."""
    from paper_2608_00531_gb300.step import PromptPass, RepairVerifyStep, StepInputs
    B, K, V, R, layers, Hq, Hkv = 3, 8, 512, 6, 2, 8, 2
    n_max, lens, n = 1 + K + R, [0, 0, 0], [40, 7, 129]
    g = torch.Generator(device=DEV).manual_seed(77)
    rnd = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)  # noqa: E731
    start = _packed(n, 0)
    base = Cache(cure, [x + 60 for x in n], Hkv, 16, 8)
    caches = []
    for _ in range(layers):
        c = Cache(cure, [x + 60 for x in n], Hkv, 16, 8)
        c.kv, c.table = base.kv, base.table
        for t in c.codes:
            t.view(torch.uint8).fill_(0x7f)
        for t in c.scales:
            t.fill_(math.nan)
        caches.append(c)
    axes, rope = cure.rope_axes([i % 3 for i in range(64)]), cure.rope_desc(128, 1e6)
    pos = torch.randint(0, 200, (3, start[-1]), dtype=torch.int32, device=DEV, generator=g)
    p = PromptPass(start[-1], B, Hq, base.kv, rope, DEV)
    row_start, cache_len = _i32(start), _i32(lens)
    for l, c in enumerate(caches):
        qkv = rnd(start[-1], (Hq + 2 * Hkv) * D)
        out = p.layer(l, qkv, row_start, cache_len, *c.codes, scales=c.scales, pos=pos, axes=axes)
        q = p.q[:start[-1]].clone()
        x = dict(cache=c, q=q, lens=lens, n=n, start=start)
        _check(x, out)
    cache_len = p.advance(row_start, cache_len)
    step = RepairVerifyStep(B, K, V, 3, 1.0, R, 2, 1, layers, Hq, base.kv, DEV, rope=rope)
    ks, vs = [c.codes[0] for c in caches], [c.codes[1] for c in caches]
    scales = ([c.scales[0] for c in caches], [c.scales[1] for c in caches])
    for _ in range(2):
        L = cache_len.tolist()
        inputs = StepInputs(rnd(B, K, V), torch.zeros(B, dtype=torch.int32, device=DEV), cache_len, None, None, None, None,
                            rnd(B, n_max, V), rnd(layers, B, n_max, (Hq + 2 * Hkv) * D))
        held = [[c.values(w, b, L[b])[0] for b in range(B)] for c in caches for w in (0, 1)]
        r = step.run(inputs, ks, vs, scales=scales)
        tree, nn = r["tree"], r["tree"]["n_nodes"].tolist()
        q, tk, tv = step._rows
        anc = tree["anc"].cpu().numpy().view(np.uint64)
        a, path = r["acc"]["accept_len"].tolist(), r["acc"]["path_nodes"].tolist()
        # the tree rows as the step appended them, once more, for the attention's reference
        for l, c in enumerate(caches):
            t = Cache(cure, [x + 60 for x in n], Hkv, 16, 8)
            t.kv, t.table = base.kv, base.table
            for w in (0, 1):
                t.codes[w].view(torch.uint8).copy_(c.codes[w].view(torch.uint8))
                t.scales[w].copy_(c.scales[w])
            cure.cure_append_kv8(tk[l], tv[l], *t.args(), step._starts, cache_len, None, pos=tree["pos"])
            seen = np.zeros((B, n_max, n_max), dtype=bool)
            for j in range(n_max):
                seen[:, :, j] = (anc[:, :, j // 64] >> np.uint64(j % 64)) & np.uint64(1)
            x = dict(cache=t, lens=L, n=nn, seen=seen, q=q[l])
            got = r["attn"][l].clone()
            for b in range(B):
                got[b, nn[b]:] = 3.5
            _check_tree(x, got)
            # the accepted rows lie behind what was held, which is what it was but for roundings below the scale's range
            for w, tt in ((0, tk), (1, tv)):
                for b in range(B):
                    v, s = c.values(w, b, L[b] + a[b] + 1)
                    want = torch.cat([held[2 * l + w][b], tt[l, b, path[b][:a[b] + 1]].double()])
                    tol = torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -8 * s[..., None])
                    assert torch.all((v - want).abs() <= tol)
        cache_len = r["resync"]["cache_len"].clone()
        assert cache_len.tolist() == [x + y + 1 for x, y in zip(L, a)]
    assert cure.cure_device_error() == 0


def test_captured_passes_and_steps(cure):
    """A prompt's pass and the step behind it, captured and replayed, write and give what they do when called."""
    from paper_2608_00531_gb300.step import PromptPass, RepairVerifyStep, StepInputs
    B, K, V, R, layers, Hq, Hkv, n = 3, 8, 512, 6, 2, 8, 2, [40, 7, 129]
    n_max, start = 1 + K + R, _packed(n, 0)
    g = torch.Generator(device=DEV).manual_seed(78)
    rnd = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)  # noqa: E731
    caches = [Cache(cure, [x + 60 for x in n], Hkv, 0, 8 + l) for l in range(layers)]
    kv = caches[0].kv
    p = PromptPass(start[-1], B, Hq, kv, cure.rope_desc(128, 1e6), DEV)
    step = RepairVerifyStep(B, K, V, 3, 1.0, R, 2, 1, layers, Hq, kv, DEV)
    ks, vs = [c.codes[0] for c in caches], [c.codes[1] for c in caches]
    scales = ([c.scales[0] for c in caches], [c.scales[1] for c in caches])
    row_start, none, held = _i32(start), _i32([0] * B), _i32(n)
    qkv = [rnd(start[-1], (Hq + 2 * Hkv) * D) for _ in range(layers)]
    x = StepInputs(rnd(B, K, V), _i32([0] * B), held, None, rnd(layers, B, n_max, Hq, D), rnd(layers, B, n_max, Hkv, D),
                   rnd(layers, B, n_max, Hkv, D), rnd(B, n_max, V))
    outs = [torch.empty(start[-1], Hq, D, dtype=torch.bfloat16, device=DEV) for _ in range(layers)]

    def run():
        for l, c in enumerate(caches):
            p.layer(l, qkv[l], row_start, none, *c.codes, scales=c.scales, out=outs[l])
        return step.run(x, ks, vs, scales=scales)

    state = [t for c in caches for t in (*(k.view(torch.uint8) for k in c.codes), *c.scales)]
    fresh = [t.clone() for t in state]
    with pytest.raises(RuntimeError, match="before it is captured"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            run()
    r = run()
    nn = r["tree"]["n_nodes"].tolist()
    rows = [(l, b, slice(0, nn[b])) for l in range(layers) for b in range(B)]
    want = [t.clone() for t in (*outs, *(r["attn"][i] for i in rows), *state, *r["resync"].values())]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = run()
    for _ in range(2):
        for t, f in zip(state, fresh):
            t.copy_(f)
        for t in (*outs, r["attn"], *r["resync"].values()):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = (*outs, *(r["attn"][i] for i in rows), *state, *r["resync"].values())
        assert len(got) == len(want)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
    assert cure.cure_device_error() == 0
