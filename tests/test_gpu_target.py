"""The target's attention layers as a serving program runs them: prompts (whole and in chunks) into the caches, a
repair-verify step from the projections of its tree, and the next rows behind what the step committed.

Every stage is compared in 64 bits with what it was given: the rotated rows from the projections (the bound of
cure_rope_qkv: 2^-8 |y| + 2^-18 (|a| + |b|)), the attention from the cache's rows (2^-8 |o| + (2^-8 + 2^-10)
sum_j w_j |v_j|)."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2608_00531_gb300 import workload as W

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
D = 128
HQ, HKV, LAYERS, PS = 28, 4, 2, 16
BASE, EPS = 1.0e6, 1e-6


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2608_00531_gb300 import cure, step
    torch.cuda.set_device(DEV)
    return cure, step


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _rotated(x, w, pos):
    """x [rows][heads][D] -> (value in 64 bits, |a| + |b|), half layout."""
    x = x.double()
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w.double()
    f = torch.tensor([BASE ** (-2.0 * i / D) for i in range(D // 2)], dtype=torch.float64, device=DEV)
    ang = pos.double()[:, None, None] * f
    a, b = x[..., :D // 2], x[..., D // 2:]
    size = (a.abs() + b.abs()).repeat(1, 1, 2)
    return torch.cat([a * torch.cos(ang) - b * torch.sin(ang), b * torch.cos(ang) + a * torch.sin(ang)], -1), size


def _near(got, want, size):
    err = (got.double() - want).abs()
    assert torch.all(err <= 2.0 ** -8 * want.abs() + 2.0 ** -18 * size), float(err.max())


def _attention(q, k, v, first):
    """q [n][Hq][D] at positions first .., k, v [keys][Hkv][D], in 64 bits: (output, sum_j w_j |v_j|)."""
    o, s = torch.zeros(2, *q.shape, dtype=torch.float64, device=DEV)
    G = HQ // HKV
    for h in range(HKV):
        x = (q[:, h * G:(h + 1) * G].double() @ k[:, h].double().T) / math.sqrt(D)
        later = torch.arange(k.shape[0], device=DEV)[None] > first + torch.arange(q.shape[0], device=DEV)[:, None]
        w = torch.softmax(x.masked_fill(later[:, None], -math.inf), -1)
        o[:, h * G:(h + 1) * G], s[:, h * G:(h + 1) * G] = w @ v[:, h].double(), w @ v[:, h].double().abs()
    return o, s


class _Caches:
    def __init__(self, cure, cap):
        B = len(cap)
        per = [-(-c // PS) for c in cap]
        pages = sum(per)
        perm = np.random.default_rng(3).permutation(pages).astype(np.int32)
        self.table = np.full((B, max(per)), -1, dtype=np.int32)
        o = 0
        for b, n in enumerate(per):
            self.table[b, :n] = perm[o:o + n]
            o += n
        self.k, self.v = (list(torch.full((LAYERS, pages, PS, HKV, D), math.nan, dtype=torch.bfloat16, device=DEV))
                          for _ in range(2))
        self.kv = cure.kv_desc(HKV, D, self.table.shape[1], block_table=torch.from_numpy(self.table).to(DEV),
                               page_size=PS, num_pages=pages)

    def rows(self, t, b, n):
        at = torch.from_numpy(self.table[b][np.arange(n) // PS].astype(np.int64) * PS + np.arange(n) % PS).to(DEV)
        return t.view(-1, HKV, D)[at]


def _check_pass(c, p, l, qkv, start, lens, out, norms):
    x = qkv.unflatten(-1, (-1, D))
    for b in range(len(lens)):
        n = start[b + 1] - start[b]
        if n == 0:
            continue
        r = slice(start[b], start[b + 1])
        pos = torch.arange(lens[b], lens[b] + n, device=DEV)
        _near(p.q[r], *_rotated(x[r, :HQ], norms[0][l], pos))
        k, v = (c.rows(t[l], b, lens[b] + n) for t in (c.k, c.v))
        _near(k[lens[b]:], *_rotated(x[r, HQ:HQ + HKV], norms[1][l], pos))
        assert torch.equal(v[lens[b]:], x[r, HQ + HKV:])
        o, s = _attention(p.q[r], k, v, lens[b])
        err = (out[r].double() - o).abs()
        assert torch.all(err <= 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -10) * s), (l, b, float(err.max()))


def test_prompts_step_and_the_next_rows(mods):
    cure, step = mods
    g = torch.Generator(device=DEV).manual_seed(5)
    rnd = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(generator=g)  # noqa: E731
    F = (HQ + 2 * HKV) * D
    norms = [[1.0 + 0.1 * rnd(D) for _ in range(LAYERS)] for _ in range(2)]
    rope = cure.rope_desc(D, BASE)
    n = [200, 0, 37, 90]
    B, K, R, V = len(n), 8, 6, 2000
    cap = [x + 80 for x in n]

    # the prompts in one pass, and in two chunks: the same caches bit for bit
    start = [0] + [int(x) for x in np.cumsum(n)]
    one, two = _Caches(cure, cap), _Caches(cure, cap)
    p = step.PromptPass(start[-1], B, HQ, one.kv, rope, DEV, norms[0], norms[1], EPS)
    prompts = [rnd(start[-1], F) for _ in range(LAYERS)]
    lens = _i32([0] * B)
    for l in range(LAYERS):
        out = p.layer(l, prompts[l], _i32(start), lens, one.k[l], one.v[l])
        _check_pass(one, p, l, prompts[l], start, [0] * B, out, norms)
    cut = [x // 3 for x in n]
    at = [0] * B
    for part in ([0] * B, cut), (cut, n):
        m = [b - a for a, b in zip(*part)]
        s2 = [0] + [int(x) for x in np.cumsum(m)]
        for l in range(LAYERS):
            rows = torch.cat([prompts[l][start[b] + part[0][b]:start[b] + part[1][b]] for b in range(B)])
            out = p.layer(l, rows, _i32(s2), _i32(at), two.k[l], two.v[l])
            _check_pass(two, p, l, rows, s2, at, out, norms)
        at = [a + x for a, x in zip(at, m)]
    for a, b in zip(one.k + one.v, two.k + two.v):
        for i in range(B):
            assert torch.equal(one.rows(a, i, n[i]), two.rows(b, i, n[i]))
    lens = p.advance(_i32(start), lens)
    assert lens.tolist() == n

    # a step from the tree's projections
    N = 1 + K + R
    st = step.RepairVerifyStep(B, K, V, 2, 1.0, R, 2, 1, LAYERS, HQ, one.kv, DEV, rope=rope, q_norm=norms[0],
                               k_norm=norms[1], eps=EPS)
    root = torch.randint(0, V, (B,), dtype=torch.int32, device=DEV, generator=g)
    qkv = rnd(LAYERS, B, N, F)
    target = rnd(B, N, V)
    x = step.StepInputs(rnd(B, K, V), root, lens, None, None, None, None, target, qkv=qkv)
    r = st.run(x, one.k, one.v)
    tree = r["tree"]
    nodes = tree["n_nodes"].tolist()
    y = qkv.unflatten(-1, (-1, D))
    for l in range(LAYERS):
        q, tk, tv = (t[l] for t in st._rows)
        for b in range(B):
            j = nodes[b]
            pos = tree["pos"][b, :j]
            assert pos.min() >= n[b]
            _near(q[b, :j], *_rotated(y[l, b, :j, :HQ], norms[0][l], pos))
            _near(tk[b, :j], *_rotated(y[l, b, :j, HQ:HQ + HKV], norms[1][l], pos))
            assert torch.equal(tv[b, :j], y[l, b, :j, HQ + HKV:])
            kc, vc = (c.rows(t[l], b, n[b]).unsqueeze(0) for c, t in ((one, one.k), (one, one.v)))
            ref = oracle.tree_attn(*(W.bf16_to_f64(t[b:b + 1].cpu()) for t in (q, tk, tv)), W.bf16_to_f64(kc.cpu()),
                                   W.bf16_to_f64(vc.cpu()), np.array([n[b]]), np.array([j]),
                                   tree["anc"][b:b + 1].cpu().numpy().view(np.uint64), 1.0 / math.sqrt(D))
            # the probabilities' and the output's rounding, |v| below 5
            assert np.abs(r["attn"][l, b, :j].double().cpu().numpy() - ref[0, :j]).max() <= 2 * 2.0 ** -8 * 5
    # what the step committed lies behind the prompts
    lens2 = r["resync"]["cache_len"]
    path = r["acc"]["path_nodes"].tolist()
    for b in range(B):
        a = lens2.tolist()[b] - n[b]
        assert a == r["acc"]["accept_len"].tolist()[b] + 1
        for l in range(LAYERS):
            k, v = (one.rows(t[l], b, n[b] + a)[n[b]:] for t in (one.k, one.v))
            assert torch.equal(k, st._rows[1][l][b, path[b][:a]]) and torch.equal(v, st._rows[2][l][b, path[b][:a]])

    # single rows and short chunks behind it
    m = [1, 3, 1, 0]
    s3 = [0] + [int(x) for x in np.cumsum(m)]
    for l in range(LAYERS):
        rows = rnd(s3[-1], F)
        out = p.layer(l, rows, _i32(s3), lens2, one.k[l], one.v[l])
        _check_pass(one, p, l, rows, s3, lens2.tolist(), out, norms)
    assert cure.cure_device_error() == 0


def test_step_from_projections_captured(mods):
    """Not before it has run once; then replays give what a run gives, also after other inputs."""
    cure, step = mods
    g = torch.Generator(device=DEV).manual_seed(9)
    rnd = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(generator=g)  # noqa: E731
    B, K, R, V = 2, 4, 3, 500
    c = _Caches(cure, [60, 40])
    for t in c.k + c.v:
        t.normal_(generator=g)
    rope = cure.rope_desc(D, BASE)
    x, y = (step.StepInputs(rnd(B, K, V), torch.randint(0, V, (B,), dtype=torch.int32, device=DEV, generator=g),
                            _i32([20, 7]), None, None, None, None, rnd(B, 1 + K + R, V),
                            qkv=rnd(LAYERS, B, 1 + K + R, (HQ + 2 * HKV) * D)) for _ in range(2))
    make = lambda: step.RepairVerifyStep(B, K, V, 2, 1.0, R, 2, 1, LAYERS, HQ, c.kv, DEV, rope=rope)  # noqa: E731
    st, graph = make(), torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    k0, v0 = ([t.clone() for t in ts] for ts in (c.k, c.v))

    def fresh():
        for a, b in zip(c.k + c.v, k0 + v0):
            a.copy_(b)

    def result(r):
        return [t.clone() for t in (r["attn"], r["tree"]["n_nodes"], r["acc"]["accept_len"], *c.k, *c.v)]
    inputs = [[t.clone() for t in (z.draft_logits, z.root_tok, z.target_logits, z.qkv)] for z in (x, y)]
    want = []
    for z in (x, y):
        fresh()
        want.append(result(make().run(z, c.k, c.v)))
    fresh()
    with pytest.raises(RuntimeError):
        with torch.cuda.graph(graph):
            st.run(x, c.k, c.v)
    st, graph = make(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    st.run(y, c.k, c.v, stream=stream)
    torch.cuda.synchronize()
    fresh()
    with torch.cuda.graph(graph):
        r = st.run(x, c.k, c.v)
    for i in (0, 1, 0):
        for a, b in zip((x.draft_logits, x.root_tok, x.target_logits, x.qkv), inputs[i]):
            a.copy_(b)
        fresh()
        graph.replay()
        nodes = r["tree"]["n_nodes"].tolist()
        for a, b in zip(result(r), want[i]):
            if a.dim() == 5 and a.shape[:2] == (LAYERS, B):  # rows of nodes
                assert all(torch.equal(a[:, j, :n], b[:, j, :n]) for j, n in enumerate(nodes))
            else:
                assert torch.equal(a, b)
    assert cure.cure_device_error() == 0


@pytest.mark.parametrize("ps", [0, 16])
def test_cache_offsets_past_32_bits(mods, ps):
    """Rows appended and read more than 2^31 values into a cache."""
    cure, step = mods
    g = torch.Generator(device=DEV).manual_seed(21)
    n = [3, 0, 150]
    if ps == 0:
        cap = 2_100_000  # sequence 2 starts at value 2.15e9
        kv = cure.kv_desc(HKV, D, cap)
        shape = (3, cap, HKV, D)
        at = [torch.arange(b * cap, b * cap + m, device=DEV) for b, m in enumerate(n)]
    else:
        pages = 270_000
        table = torch.full((3, 10), -1, dtype=torch.int32)
        table[0, 0], table[2] = 5, torch.arange(pages - 1, pages - 11, -1)
        kv = cure.kv_desc(HKV, D, 10, block_table=table.to(DEV), page_size=ps, num_pages=pages)
        shape = (pages, ps, HKV, D)
        at = [(table[b, np.arange(m) // ps].long() * ps + torch.arange(m) % ps).to(DEV) for b, m in enumerate(n)]
    kc, vc = (torch.empty(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    assert kc.numel() > 2 ** 31 and int(at[2].max()) * HKV * D > 2 ** 31
    x = torch.empty(sum(n), (HQ + 2 * HKV) * D, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    p = step.PromptPass(sum(n), 3, HQ, kv, cure.rope_desc(D, BASE), DEV)
    out = p.layer(0, x, _i32([0, 3, 3, 153]), _i32([0, 0, 0]), kc, vc)
    y = x.unflatten(-1, (-1, D))
    for b, r in ((0, slice(0, 3)), (2, slice(3, 153))):
        k, v = (t.view(-1, HKV, D)[at[b]] for t in (kc, vc))
        assert torch.equal(v, y[r, HQ + HKV:])
        plain = cure.cure_rope_qkv(None, y[r, HQ:HQ + HKV], None, torch.arange(n[b], dtype=torch.int32, device=DEV),
                                        p.rope)[1]
        assert torch.equal(k, plain)
        o, size = _attention(p.q[r], k, v, 0)
        assert torch.all((out[r].double() - o).abs() <= 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -10) * size)
    assert cure.cure_device_error() == 0


def test_prompt_pass_captured_and_two_at_once(mods):
    """Two layers over some thousand rows, captured and replayed on other inputs; two passes on two streams."""
    cure, step = mods
    g = torch.Generator(device=DEV).manual_seed(23)
    n = [2500, 1, 1800, 0, 1700]
    start = _i32([0] + [int(v) for v in np.cumsum(n)])
    lens = _i32([0, 300, 40, 7, 0])
    a, b = (_Caches(cure, [2500, 400, 2000, 100, 1800]) for _ in range(2))
    for t in a.k + a.v:
        t.normal_(generator=g)
    for t, u in zip(b.k + b.v, a.k + a.v):
        t.copy_(u)
    make = lambda c: step.PromptPass(sum(n), 5, HQ, c.kv, cure.rope_desc(D, BASE), DEV)  # noqa: E731
    x = torch.empty(2, LAYERS, sum(n), (HQ + 2 * HKV) * D, dtype=torch.bfloat16, device=DEV).normal_(generator=g)

    def run(p, c, qkv, stream=None):
        return [p.layer(l, qkv[l], start, lens, c.k[l], c.v[l], stream=stream) for l in range(LAYERS)]
    p, q = make(a), make(b)
    want = [[t.clone() for t in run(p, a, x[i])] for i in range(2)]
    graph, qkv = torch.cuda.CUDAGraph(), x[0].clone()
    with torch.cuda.graph(graph):
        outs = run(p, a, qkv)
    for i in (0, 1, 0):
        qkv.copy_(x[i])
        graph.replay()
        assert all(torch.equal(s, t) for s, t in zip(outs, want[i]))
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        got = run(p, a, x[0], s), run(q, b, x[1], t)
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(u, w) for u, w in zip(got[i], want[i]))
    assert cure.cure_device_error() == 0


def test_refusals(mods):
    cure, step = mods
    c = _Caches(cure, [32])
    p = step.PromptPass(4, 1, HQ, c.kv, cure.rope_desc(D, BASE), DEV)
    row = torch.zeros(4, (HQ + 2 * HKV) * D, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        p.layer(0, torch.cat([row, row]), _i32([0, 8]), _i32([0]), c.k[0], c.v[0])
    with pytest.raises(ValueError):
        p.layer(0, row[:, :-D].contiguous(), _i32([0, 4]), _i32([0]), c.k[0], c.v[0])
    st = step.RepairVerifyStep(1, 4, 100, 2, 1.0, 2, 2, 1, 1, HQ, c.kv, DEV)
    x = step.StepInputs(torch.zeros(1, 4, 100, dtype=torch.bfloat16, device=DEV), _i32([1]), _i32([0]), None, None, None,
                        None, torch.zeros(1, 7, 100, dtype=torch.bfloat16, device=DEV),
                        qkv=torch.zeros(1, 1, 5, (HQ + 2 * HKV) * D, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(ValueError):
        st.run(x, c.k, c.v)
    with pytest.raises(ValueError):
        st.run_from_host(x, c.k, c.v)
