"""cure_prompt_attn on the GPU against softmax attention in 64 bits.

Tolerance of an output value o = sum_j w_j v_j (weights w_j of sum 1): the
probabilities are rounded to bf16 before the product (each by up to 2^-8 of
itself: 2^-8 sum_j w_j |v_j|) and the output once more (2^-8 |o|); the float32
scores are off by 128 products' roundings (2^-17 of scale sum_d |q_d k_d|, which
the inputs here keep below 64), ex2 by 2^-22 of itself and the sums by less than
that: 2^-10 sum_j w_j |v_j| covers them.  In all
  |got - o| <= 2^-8 |o| + (2^-8 + 2^-10) sum_j w_j |v_j|.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
D = 128
SCALE = 1.0 / math.sqrt(D)


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


def _case(cure, lens, n, Hq, Hkv, ps, seed, std=1.5, pad=0, slack=0, stale=math.nan):
    """Rows, caches whose unused places hold `stale`, geometry and tables.  pad: rows before the first and behind
    the last sequence."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    rnd = lambda *s, std=1.0: torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(0.0, std, generator=g)  # noqa: E731
    B, ends = len(n), [a + b for a, b in zip(lens, n)]
    start = [pad] + [pad + int(x) for x in np.cumsum(n)]
    q = rnd(start[-1] + pad, Hq, D, std=std)
    if ps == 0:
        cap = max(max(ends), 1) + slack
        kc, vc = (torch.full((B, cap, Hkv, D), stale, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        kv, table = cure.kv_desc(Hkv, D, cap), None
        rows = lambda b: b * cap + np.arange(ends[b])  # noqa: E731
    else:
        need = [-(-e // ps) for e in ends]
        pages = sum(need) + 2
        perm = rng.permutation(pages).astype(np.int32)
        table = np.full((B, max(max(need), 1) + slack), -1, dtype=np.int32)
        o = 0
        for b, m in enumerate(need):
            table[b, :m] = perm[o:o + m]
            o += m
        kc, vc = (torch.full((pages, ps, Hkv, D), stale, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        kv = cure.kv_desc(Hkv, D, table.shape[1], block_table=torch.from_numpy(table).to(DEV), page_size=ps,
                          num_pages=pages)
        rows = lambda b: table[b][np.arange(ends[b]) // ps].astype(np.int64) * ps + np.arange(ends[b]) % ps  # noqa: E731
    at = [torch.from_numpy(np.asarray(rows(b), dtype=np.int64)).to(DEV) for b in range(B)]
    for b in range(B):
        kc.view(-1, Hkv, D)[at[b]] = rnd(ends[b], Hkv, D)
        vc.view(-1, Hkv, D)[at[b]] = rnd(ends[b], Hkv, D)
    return dict(q=q, kc=kc, vc=vc, kv=kv, at=at, lens=lens, n=n, start=start, Hq=Hq, Hkv=Hkv,
                row_start=_i32(start), cache_len=_i32(lens))


def _run(cure, x, out=None, **kw):
    if out is None:
        out = torch.full_like(x["q"], 3.5)
    return cure.cure_prompt_attn(x["q"], x["kc"], x["vc"], x["kv"], x["row_start"], x["cache_len"], SCALE, out=out, **kw)


def _check(x, got, seqs=None, rows=None):
    """rows: which rows of each sequence to compute in 64 bits (all of them by default)."""
    G = x["Hq"] // x["Hkv"]
    assert torch.all(got[:x["start"][0]] == 3.5) and torch.all(got[x["start"][-1]:] == 3.5)
    for b in range(len(x["n"])) if seqs is None else seqs:
        n, L = x["n"][b], x["lens"][b]
        pick = range(n) if rows is None else sorted({r % n for r in rows if -n <= r < n} if n else set())
        i = torch.tensor(list(pick), dtype=torch.long, device=DEV)
        if not len(i):
            continue
        for h in range(x["Hkv"]):
            k, v = (x[t].view(-1, x["Hkv"], D)[x["at"][b], h].double() for t in ("kc", "vc"))
            q = x["q"][x["start"][b] + i, h * G:(h + 1) * G].double()
            s = (q @ k.T) * SCALE
            s.masked_fill_(torch.arange(L + n, device=DEV)[None, None] > (L + i)[:, None, None], -math.inf)
            w = torch.softmax(s, -1)
            o = got[x["start"][b] + i, h * G:(h + 1) * G].double()
            ref, size = w @ v, w @ v.abs()
            assert torch.all((o - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -10) * size), (
                b, h, float(((o - ref).abs() / size).max()))


HEADS = [(28, 4), (8, 2), (3, 3), (5, 1)]


@pytest.mark.parametrize("Hq,Hkv", HEADS)
@pytest.mark.parametrize("ps", [0, 8, 16, 64])
def test_prompt_ragged(cure, ps, Hq, Hkv):
    """Whole prompts, chunks behind cached tokens, single tokens, empty sequences; rows around the batch's ends
    unwritten; NaN wherever no key lies."""
    x = _case(cure, [0, 130, 0, 5, 127, 300, 64], [1, 40, 0, 123, 1, 129, 256], Hq, Hkv, ps, 100 + ps + Hq, pad=3)
    _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("n", [1, 2, 17, 18, 19, 36, 37, 127, 128, 129, 255, 256, 257, 300])
def test_prompt_lengths_around_the_tiles(cure, n):
    for Hq, Hkv, L in ((28, 4, 0), (2, 2, 0), (8, 1, 127), (16, 1, 1)):
        x = _case(cure, [L], [n], Hq, Hkv, 16, n + Hq)
        _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("G", [1, 2, 6, 9, 33, 64, 65, 127, 128])
def test_prompt_group_sizes(cure, G):
    x = _case(cure, [70, 0], [9, 131], G, 1, 32, G)
    _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("ps", [0, 16])
def test_prompt_long(cure, ps):
    """A long prompt and a chunk far into a long sequence, some rows of them in 64 bits; sharp and flat scores."""
    for std in (0.02, 1.5, 4.0):
        x = _case(cure, [0, 9000], [5003, 700], 14, 2, ps, 7, std=std)
        _check(x, _run(cure, x), rows=[0, 1, 63, 127, 128, 129, 511, 640, 2047, 3333, 4999, -1, -2])
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("ps", [0, 16])
@pytest.mark.parametrize("Hq,Hkv", [(28, 4), (8, 8)])
def test_prompt_single_tokens(cure, ps, Hq, Hkv):
    """One token a sequence over caches of one to many tokens."""
    lens = [0, 1, 127, 128, 129, 1000, 4095, 20000]
    x = _case(cure, lens, [1] * len(lens), Hq, Hkv, ps, 5)
    _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


def test_prompt_one_token_on_a_long_cache(cure):
    x = _case(cure, [131071], [1], 28, 4, 16, 6)
    _check(x, _run(cure, x))
    x = _case(cure, [70000], [3], 8, 1, 0, 6)
    _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


def test_prompt_most_sequences(cure):
    """256 sequences, the most that a call takes, many of them empty or of one row."""
    rng = np.random.default_rng(2)
    n = [int(v) for v in rng.choice([0, 1, 1, 2, 5, 40], size=256)]
    lens = [int(v) for v in rng.integers(0, 300, size=256)]
    x = _case(cure, lens, n, 8, 2, 16, 11)
    _check(x, _run(cure, x))
    x = _case(cure, [0] * 256, [0] * 256, 8, 2, 16, 11, pad=1)
    _check(x, _run(cure, x))
    assert cure.cure_device_error() == 0


def test_prompt_growing_maxima(cure):
    """Scores that grow along the keys, so that the running maximum rises tile after tile, by little and by much."""
    for step in (0.02, 0.4):
        x = _case(cure, [0], [900], 2, 1, 0, 13)
        x["q"][:] = 0.0
        x["q"][:, :, 0] = 4.0
        x["kc"][0, :, 0] = 0.0
        x["kc"][0, :, 0, 0] = (torch.arange(900, device=DEV) * step).to(torch.bfloat16)
        _check(x, _run(cure, x))


def test_prompt_scores_of_minus_infinity(cure):
    """Keys whose scores are -inf weigh nothing, beside finite ones."""
    x = _case(cure, [0], [300], 2, 1, 16, 17)
    x["q"][:, :, 0] = 1.0
    k = x["kc"].view(-1, 1, D)
    k[x["at"][0][5:200:3], 0, 0] = -math.inf
    _check(x, _run(cure, x))


def test_prompt_bad_pages_slots_and_rows(cure):
    x = _case(cure, [0, 100, 20], [50, 60, 30], 8, 2, 16, 19)
    want = _run(cure, x)
    s = x["start"]
    # sequence 1 does not fit its capacity: its rows stay, the others are computed
    lens = x["cache_len"].clone()
    lens[1] = 16 * x["kv"].max_len - 59
    got = cure.cure_prompt_attn(x["q"], x["kc"], x["vc"], x["kv"], x["row_start"], lens, SCALE,
                                out=torch.full_like(want, 3.5))
    assert cure.cure_device_error() == cure.DEVERR_SLOT
    assert torch.all(got[s[1]:s[2]] == 3.5) and torch.equal(got[:s[1]], want[:s[1]]) and torch.equal(got[s[2]:], want[s[2]:])
    lens[1] = -1
    got = cure.cure_prompt_attn(x["q"], x["kc"], x["vc"], x["kv"], x["row_start"], lens, SCALE,
                                out=torch.full_like(want, 3.5))
    assert cure.cure_device_error() == cure.DEVERR_SLOT and torch.all(got[s[1]:s[2]] == 3.5)
    # row_start outside the rows, or descending
    for bad in ([0, 50, 110, 141], [-1, 50, 110, 140], [0, 120, 110, 140]):
        cure.cure_prompt_attn(x["q"], x["kc"], x["vc"], x["kv"], _i32(bad), x["cache_len"], SCALE,
                              out=torch.full_like(want, 3.5))
        assert cure.cure_device_error() & cure.DEVERR_NODES
    # missing and bad pages count as zeros
    table = x["kv"]._keep
    keep = table.clone()
    for bad in (-1, 1 << 20):
        table[1, 2] = bad
        got = _run(cure, x)
        assert cure.cure_device_error() == cure.DEVERR_PAGE
        assert torch.equal(got[:s[1]], want[:s[1]]) and torch.isfinite(got).all()
        table.copy_(keep)
    y = dict(x, kc=x["kc"].clone(), vc=x["vc"].clone())
    y["kc"][int(keep[1, 2])] = 0
    y["vc"][int(keep[1, 2])] = 0
    assert torch.equal(_run(cure, y), got)


def test_prompt_workspace_and_repeats(cure):
    """Whatever the workspace holds, call after call the same bits."""
    x = _case(cure, [0, 4000, 17], [700, 1, 90], 28, 4, 16, 23)
    want = _run(cure, x)
    size = cure.cure_prompt_attn_workspace_size(x["q"].shape[0], 3, 28, x["kv"])
    for fill in (0x00, 0xff, 0x7f):
        ws = torch.full((size,), fill, dtype=torch.uint8, device=DEV)
        for _ in range(3):
            assert torch.equal(_run(cure, x, workspace=ws), want)
    _check(x, want)


def test_prompt_graphs_and_streams(cure):
    """Two captured graphs on one workspace, replayed in turn on other inputs and lengths; a call on its own stream."""
    x = _case(cure, [600, 4000, 17], [200, 1, 90], 28, 4, 16, 29, stale=0.0)
    ws = torch.empty(cure.cure_prompt_attn_workspace_size(x["q"].shape[0], 3, 28, x["kv"]), dtype=torch.uint8, device=DEV)
    _run(cure, x, workspace=ws)
    torch.cuda.synchronize()
    outs, graphs = [torch.zeros_like(x["q"]) for _ in range(2)], []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _run(cure, x, out=o, workspace=ws)
        graphs.append(g)
    for turn in range(3):
        x["q"].normal_(0.0, 1.0 + turn)
        x["cache_len"].copy_(_i32([600 - 100 * turn, 4000 - 1000 * turn, 3 + turn]))
        for o in outs:
            o.zero_()
        graphs[0].replay()
        graphs[1].replay()
        graphs[0].replay()
        want = _run(cure, x, out=torch.zeros_like(x["q"]))
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = cure.cure_prompt_attn(x["q"], x["kc"], x["vc"], x["kv"], x["row_start"], x["cache_len"], SCALE, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    assert cure.cure_device_error() == 0


def test_prompt_agrees_with_the_tree_attention(cure):
    """A chain of rows is the in-place tree whose node j has the ancestors 0 .. j."""
    B, n, Hq, Hkv = 4, 17, 28, 4
    x = _case(cure, [1000, 0, 64, 3000], [n] * B, Hq, Hkv, 16, 31)
    got = _run(cure, x)
    anc = torch.tensor([[(1 << (j + 1)) - 1] for j in range(n)], dtype=torch.int64, device=DEV).expand(B, n, 1).contiguous()
    tree = cure.cure_tree_attn(x["q"].view(B, n, Hq, D), None, None, x["kc"], x["vc"], x["kv"], x["cache_len"],
                               _i32([n] * B), anc, SCALE)
    # the same sums in other groups of keys: both within the bound of the exact value
    _check(x, got)
    _check(x, tree.view(B * n, Hq, D))


def test_prompt_output_aligned_to_16_bytes_only(cure):
    """32-byte stores need 32-byte alignment; an output that is aligned to 16 bytes gets the same bits."""
    x = _case(cure, [0, 300], [150, 40], 8, 2, 16, 41)
    want = _run(cure, x)
    buf = torch.full((want.numel() + 8,), 3.5, dtype=torch.bfloat16, device=DEV)
    got = _run(cure, x, out=buf[8:].view(want.shape))
    assert got.data_ptr() % 32 == 16 and torch.equal(got, want) and torch.all(buf[:8] == 3.5)


def test_prompt_whole_and_cut_units(cure):
    """Shapes on both sides of the choice: many short units, few long ones, one CTA's worth, long and short together."""
    for n, lens, Hq, Hkv in (([300] * 40, [0] * 40, 28, 4), ([900] * 3, [5000, 0, 20000], 7, 1), ([5], [0], 1, 1),
                             ([1500, 1, 3, 700], [0, 40000, 9000, 10], 32, 8), ([33] * 200, [100] * 200, 4, 4)):
        x = _case(cure, lens, n, Hq, Hkv, 16, sum(n))
        _check(x, _run(cure, x), rows=[0, 1, 31, 200, 299, 650, 899, 1499, -1])
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("B,lo,hi,past,Hq,Hkv,ps", [(12, 300, 2500, 0, 28, 4, 16), (32, 1, 1500, 900, 4, 4, 0),
                                                    (33, 700, 1400, 500, 2, 2, 0), (64, 0, 1100, 2000, 28, 4, 32),
                                                    (255, 130, 520, 700, 8, 1, 16), (256, 128, 128, 1000, 16, 2, 8)])
def test_prompt_ragged_batches_of_whole_units(cure, B, lo, hi, past, Hq, Hkv, ps):
    """Units that are dealt out by length, for batches that the scheduler keeps in registers and larger ones; with
    sequences of no rows among them and equal lengths."""
    rng = np.random.default_rng(B)
    n = [int(v) for v in rng.integers(lo, hi + 1, B)]
    n[B // 2] = n[B // 3] = 0
    n[B // 4] = n[0]
    lens = [int(v) for v in rng.integers(0, past + 1, B)]
    x = _case(cure, lens, n, Hq, Hkv, ps, B)
    got = _run(cure, x)
    _check(x, got, rows=[0, 17, 35, 36, 255, 256, 511, 899, -1])
    assert torch.equal(got, _run(cure, x))  # and every row is written, the same way
    assert torch.all((got != 3.5).any(-1)) and cure.cure_device_error() == 0


def test_prompt_binding_refusals(cure):
    x = _case(cure, [0, 5], [4, 3], 8, 2, 16, 37)
    args = [x["q"], x["kc"], x["vc"], x["kv"], x["row_start"], x["cache_len"], SCALE]

    def call(i, v, **kw):
        a = list(args)
        a[i] = v
        return lambda: cure.cure_prompt_attn(*a, **kw)
    for kind, f in ((TypeError, call(0, x["q"].float())), (ValueError, call(0, x["q"][:, :, :64])),
                    (ValueError, call(0, x["q"].transpose(0, 1).contiguous().transpose(0, 1))),
                    (TypeError, call(4, x["row_start"].long())), (ValueError, call(4, x["row_start"][:2])),
                    (ValueError, call(5, x["cache_len"].cpu())), (ValueError, call(1, x["kc"][:1])),
                    (ValueError, call(0, x["q"], out=x["q"][:3].clone())),
                    (ValueError, call(3, cure.kv_desc(2, D, 4, block_table=x["kv"]._keep[:1], page_size=16, num_pages=4)))):
        with pytest.raises(kind):
            f()
    from paper_2608_00531_gb300._lib import CureError
    for f in (call(6, 0.0), call(6, math.inf), call(6, math.nan), call(0, x["q"][:, :7].contiguous()),
              call(6, SCALE, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))):
        with pytest.raises(CureError):
            f()
    assert cure.cure_device_error() == 0
