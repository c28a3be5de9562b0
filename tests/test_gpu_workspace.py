"""What the attention operators' workspaces hold on entry does not matter: the counters of units that several CTAs
share are told from anything that an earlier user of the memory left there, small integers (token ids, positions)
among them.

A captured call keeps what it counts by, so one graph is replayed behind every filling that a counter of few bits
could take for its own: (t << 9) | count for t = 1, 2, .., in 32-bit and in 64-bit words.  The rest of the workspace
and the output hold NaN, so that a unit that is joined before its parts are there (count 1, where the parts end far
enough apart), or never (a count above any number of parts), shows.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
D = 128
SCALE = 1.0 / math.sqrt(D)
TAGS = 6000
FRONT = 4096  # bytes that hold the counters, at least


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


def _rnd(g, *s):
    return torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(generator=g)


def _replay_on_all_fillings(call, ws, out, good):
    """call() writes `out` by way of `ws`; good(out): a truth value on the device."""
    ws.zero_()
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    rest = ws[FRONT:].view(torch.float32)
    bad = torch.zeros((), dtype=torch.int64, device=DEV)
    for words in (ws[:FRONT].view(torch.int32), ws[:FRONT].view(torch.int64)):
        for count in (1, 300):
            for t in range(1, TAGS + 1):
                words.fill_((t << 9) | count)
                rest.fill_(math.nan)
                out.fill_(math.nan)
                graph.replay()
                bad += ~good(out)
    assert int(bad) == 0


def test_prompt_attention_counts_no_stale_words(cure):
    g = torch.Generator(device=DEV).manual_seed(3)
    lens, Hq, Hkv = [20000, 500], 28, 4  # two rows whose keys all CTAs share
    kc, vc = (_rnd(g, 2, 20001, Hkv, D) for _ in range(2))
    kv, q = cure.kv_desc(Hkv, D, 20001), _rnd(g, 2, Hq, D)
    start, held = _i32([0, 1, 2]), _i32(lens)
    ws = torch.empty(cure.cure_prompt_attn_workspace_size(2, 2, Hq, kv), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    call = lambda: cure.cure_prompt_attn(q, kc, vc, kv, start, held, SCALE, out=out, workspace=ws)  # noqa: E731
    ws.zero_()
    want = call().clone()
    assert torch.isfinite(want).all()
    _replay_on_all_fillings(call, ws, out, lambda o: (o == want).all())
    assert cure.cure_device_error() == 0


def test_tree_attention_counts_no_stale_words(cure):
    g = torch.Generator(device=DEV).manual_seed(4)
    lens, n, Hq, Hkv = [900, 37, 1500, 64, 300, 0, 1100, 700, 129, 2000, 511, 1024], 9, 32, 8
    B = len(lens)
    kc, vc = (_rnd(g, B, max(lens), Hkv, D) for _ in range(2))
    kv = cure.kv_desc(Hkv, D, max(lens))
    assert cure.cure_selftest_attn_route(B, n, Hq, kv, False)[0] == 0  # units are cut, not given to clusters
    q, tk, tv = (_rnd(g, B, n, h, D) for h in (Hq, Hkv, Hkv))
    anc = _i32([[(1 << (j + 1)) - 1] for j in range(n)]).long().expand(B, n, 1).contiguous()
    held, nodes = _i32(lens), _i32([n] * B)
    ws = torch.empty(cure.cure_tree_attn_workspace_size(B, n, Hq, kv), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    call = lambda: cure.cure_tree_attn(q, tk, tv, kc, vc, kv, held, nodes, anc, SCALE, out=out,  # noqa: E731
                                       workspace=ws)
    ws.zero_()
    want = call().float().clone()
    # which part of a unit comes last may move a value by a rounding to bf16 and float32's own
    _replay_on_all_fillings(call, ws, out, lambda o: ((o.float() - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -16).all())
    assert cure.cure_device_error() == 0


def test_a_call_holds_its_own_workspace_until_it_is_launched(cure, monkeypatch):
    """Without a workspace of the caller's, the call's own must not be free for another thread's tensors before the
    kernel that uses it is queued."""
    kv = cure.kv_desc(2, D, 64)
    q = torch.zeros(4, 8, D, dtype=torch.bfloat16, device=DEV)
    kc, vc = (torch.zeros(1, 64, 2, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    size = cure.cure_prompt_attn_workspace_size(4, 1, 8, kv)
    lib, held = cure._lib.load(), []

    class Library:
        def __getattr__(self, name):
            f = getattr(lib, name)
            if name not in ("cure_prompt_attn", "cure_selftest_prompt_timeout"):
                return f
            return lambda *a: held.append(torch.cuda.memory_allocated()) or f(*a)
    start, lens = _i32([0, 4]), _i32([0])
    monkeypatch.setattr(cure._lib, "load", lambda: Library())
    for call in (lambda: cure.cure_prompt_attn(q, kc, vc, kv, start, lens, SCALE),
                 lambda: cure.cure_selftest_prompt_timeout(q, kc, vc, kv, start, lens, SCALE, 11, 1000)):
        before = torch.cuda.memory_allocated()
        call()
        assert held.pop() >= before + size
    torch.cuda.synchronize()
    assert cure.cure_device_error() == 0
