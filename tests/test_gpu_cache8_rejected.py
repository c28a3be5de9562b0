"""Rows of a tree that are rejected, over caches in 8 bits: whatever they hold, the tokens that a sequence has keep their
values.  (In place the tree shares a block of 16 slots, and its scale, with a sequence's last tokens.)"""
import math

import pytest
import torch

from test_gpu_cache8 import DEV, E4M3, SCALE, Cache, _i32, _run_tree, _tree, cure  # noqa: F401

pytestmark = pytest.mark.gpu

HUGE = [("larger", 2.0 ** 10), ("much larger", 2.0 ** 14), ("infinite", math.inf)]


class _Case:
    """A step whose targets reject every node but the root, and whose rejected rows are `factor` times larger."""

    def __init__(self, cure, ps, factor, lens, layers=2):  # noqa: F811
        from paper_2608_00531_gb300.step import RepairVerifyStep, StepInputs
        B, K, V, R, Hq, Hkv = len(lens), 8, 512, 6, 8, 2
        n_max = 1 + K + R
        self.lens, self.layers = list(lens), layers
        g = torch.Generator(device=DEV).manual_seed(ps + B)
        rnd = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)  # noqa: E731
        # (one seed: the layers' pages are the same)
        self.caches = [Cache(cure, [x + 2 * n_max for x in lens], Hkv, ps, 31) for _ in range(layers)]
        self.step = RepairVerifyStep(B, K, V, 3, 1.0, R, 2, 1, layers, Hq, self.caches[0].kv, DEV)
        draft, target = rnd(B, K, V), rnd(B, n_max, V)
        draft[..., 300:], target[..., 400] = -20.0, 20.0  # tokens of the draft, and one that it never gives
        tk, tv = rnd(layers, B, n_max, Hkv, 128), rnd(layers, B, n_max, Hkv, 128)
        for t in (tk, tv):
            if math.isinf(factor):
                t[:, :, 1, 0, 7], t[:, :, 4, 1, 99] = factor, -factor
            else:
                t[:, :, 1:] *= factor
            t[:, :, 0] = 0  # (the root, which is accepted, raises no scale)
        self.x = StepInputs(draft, _i32([0] * B), _i32(lens), None, rnd(layers, B, n_max, Hq, 128), tk, tv, target)
        self.args = ([c.codes[0] for c in self.caches], [c.codes[1] for c in self.caches])
        self.scales = ([c.scales[0] for c in self.caches], [c.scales[1] for c in self.caches])

    def held(self):
        return [c.values(w, b, n)[0] for c in self.caches for w in (0, 1) for b, n in enumerate(self.lens)]


@pytest.mark.parametrize("ps", [0, 16, 32, 64])
@pytest.mark.parametrize("name,factor", HUGE)
def test_a_step_keeps_what_is_held(cure, ps, name, factor):  # noqa: F811
    case = _Case(cure, ps, factor, [0, 1, 15, 16, 17, 39, 64, 111])
    for _ in range(2):
        before = case.held()
        r = case.step.run(case.x, *case.args, scales=case.scales)
        assert r["acc"]["accept_len"].tolist() == [0] * len(case.lens)
        assert min(r["tree"]["n_nodes"].tolist()) > 4
        assert all(torch.equal(a, b) for a, b in zip(before, case.held())), name
        # .. and the root's row is behind it
        case.lens = r["resync"]["cache_len"].tolist()
        case.x.cache_len.copy_(r["resync"]["cache_len"])
        for c in case.caches:
            for b, n in enumerate(case.lens):
                assert torch.all(c.values(0, b, n)[0][n - 1] == 0) and torch.all(c.values(1, b, n)[0][n - 1] == 0)
    assert cure.cure_device_error() == 0


def test_a_captured_step_keeps_what_is_held(cure):  # noqa: F811
    case = _Case(cure, 16, math.inf, [3, 40, 16])
    before = case.held()
    case.step.run(case.x, *case.args, scales=case.scales)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        case.step.run(case.x, *case.args, scales=case.scales)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(before, case.held()))
    assert cure.cure_device_error() == 0


def test_a_step_that_is_refused_keeps_what_is_held(cure):  # noqa: F811
    """The attention refuses its arguments when the tree's rows are in the cache already."""
    import dataclasses
    case = _Case(cure, 16, 2.0 ** 14, [3, 40, 16])
    before = case.held()
    with pytest.raises(ValueError):
        case.step.run(dataclasses.replace(case.x, q=case.x.q[..., :64]), *case.args, scales=case.scales)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, case.held()))


def _bytes(c):
    return [t.view(torch.uint8).clone() for t in (*c.codes, *c.scales)]


@pytest.mark.parametrize("ps", [0, 16, 32, 64])
@pytest.mark.parametrize("Hkv,layers", [(2, 1), (5, 3), (1, 128)])
def test_save_and_restore(cure, ps, Hkv, layers):  # noqa: F811
    """Rows appended for a time: every bit of what the caches hold is back, the slots behind it aside."""
    lens, n = [0, 1, 15, 16, 17, 100, 31, 64], [9, 40, 1, 9, 16, 0, 1, 3]
    cs = [Cache(cure, [a + b for a, b in zip(lens, n)], Hkv, ps, 70, slack=1) for _ in range(layers)]
    if ps:  # a sequence whose last block has no page: it cannot be appended to either
        for c in cs:
            c.table[4, 17 // ps] = -1
            c.kv._keep.copy_(torch.from_numpy(c.table))
    start = [0]
    for m in n:
        start.append(start[-1] + m)
    before = [_bytes(c) for c in cs]
    values = [c.values(w, b, m)[0] for c in cs for w in (0, 1) for b, m in enumerate(lens) if not (ps and b == 4)]
    all_of = ([c.codes[0] for c in cs], [c.codes[1] for c in cs], [c.scales[0] for c in cs], [c.scales[1] for c in cs],
              cs[0].kv)
    saved = cure.cure_save_kv8(*all_of, _i32(lens))
    assert saved.numel() == cure.cure_save_kv8_size(layers, len(lens), cs[0].kv)
    assert all(torch.equal(a, b) for x, c in zip(before, cs) for a, b in zip(x, _bytes(c)))
    x = torch.randn(start[-1], Hkv, 128, device=DEV).bfloat16() * 2.0 ** 13
    for c in cs:
        cure.cure_append_kv8(x, -x, *c.args(), _i32(start), _i32(lens), None)
    assert cure.cure_device_error() == (cure.DEVERR_PAGE if ps else 0)
    cure.cure_restore_kv8(*all_of, _i32(lens), saved)
    now = [c.values(w, b, m)[0] for c in cs for w in (0, 1) for b, m in enumerate(lens) if not (ps and b == 4)]
    assert all(torch.equal(a, b) for a, b in zip(values, now))
    for c, old in zip(cs, before):  # the blocks' codes and scales, and nothing but the appended rows' slots differs
        for w in (0, 1):
            codes = old[w].view(-1, Hkv, 128)
            scales = old[2 + w].view(torch.float32).view(-1, Hkv)
            got, gs = c.codes[w].view(torch.uint8).view(-1, Hkv, 128), c.scales[w].view(-1, Hkv)
            for b, (L, m) in enumerate(zip(lens, n)):
                new = [t for t in range(L, L + m) if ps == 0 or c.table[b, t // ps] >= 0]
                if new:
                    codes[c.rows(b, new)] = got[c.rows(b, new)]
                blocks = sorted({t // 16 for t in new if t // 16 * 16 >= L})  # of the appended rows alone
                if blocks:
                    scales[c.places(b, blocks)] = gs[c.places(b, blocks)]
            assert torch.equal(got, codes)
            assert torch.equal(gs.view(torch.int32), scales.view(torch.int32))
    assert cure.cure_device_error() == 0


def test_lengths_out_of_range(cure):  # noqa: F811
    """Nothing is begun below no length, at a whole block, at or past the capacity: nothing is touched."""
    for ps in (0, 16):
        c = Cache(cure, [40, 40, 40, 40, 40], 2, ps, 5)
        cap = c.kv.max_len * max(ps, 1)
        lens = _i32([-7, 32, cap + 1, 2 ** 31 - 1, -2 ** 31])
        one = ([c.codes[0]], [c.codes[1]], [c.scales[0]], [c.scales[1]], c.kv)
        before = _bytes(c)
        saved = torch.full((cure.cure_save_kv8_size(1, 5, c.kv),), 9, dtype=torch.uint8, device=DEV)
        cure.cure_save_kv8(*one, lens, out=saved)
        assert torch.all(saved == 9)
        cure.cure_restore_kv8(*one, lens, saved)
        assert all(torch.equal(a, b) for a, b in zip(before, _bytes(c)))
    assert cure.cure_device_error() == 0


def test_a_tree_in_place_by_the_calls_themselves(cure):  # noqa: F811
    """Save, append, attend, restore, commit, as the step does it, on a stream of its own."""
    lens, n_max = [100, 33, 5], 20
    x = _tree(cure, lens, [n_max] * 3, n_max, 8, 2, 16, 3)
    c = x["cache"]
    one = ([c.codes[0]], [c.codes[1]], [c.scales[0]], [c.scales[1]], c.kv)
    before = [c.values(w, b, n)[0] for w in (0, 1) for b, n in enumerate(lens)]
    t = torch.randn(1, 3, n_max, 2, 128, device=DEV).bfloat16()
    t[:, :, 1:] *= 2.0 ** 12
    t[:, :, 0] = 0
    acc = dict(path_nodes=_i32([[0] + [-1] * 5] * 3), accept_len=_i32([0] * 3), diverge_depth=_i32([-1] * 3),
               out_tokens=_i32([[1] * 6] * 3))
    start, cache_len = _i32([0, n_max, 2 * n_max, 3 * n_max]), _i32(lens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        saved = cure.cure_save_kv8(*one, cache_len)
        cure.cure_append_kv8(t[0], t[0], *c.args(), start, cache_len, None)
        _run_tree(cure, x)
        cure.cure_restore_kv8(*one, cache_len, saved)
        r = cure.cure_resync_kv8(*one, t, t, acc, cache_len, 4)
    s.synchronize()
    assert r["cache_len"].tolist() == [n + 1 for n in lens]
    assert all(torch.equal(a, b) for a, b in zip(before, [c.values(w, b, n)[0] for w in (0, 1) for b, n in enumerate(lens)]))
    assert cure.cure_device_error() == 0
