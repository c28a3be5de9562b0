"""Steps whose next tokens do not stand at their slots, as behind a prompt with images: the tree's rows turn by the positions
that ``StepInputs.next_pos`` gives, on one axis as well as on several that are the same."""
import dataclasses

import pytest
import torch

from test_gpu_cache8 import DEV, Cache, _i32, _packed, _rotated, cure  # noqa: F401

pytestmark = pytest.mark.gpu

B, K, V, R, LAYERS, HQ, HKV = 3, 8, 512, 6, 2, 8, 2
N_MAX = 1 + K + R


@pytest.fixture(params=[False, True], ids=["bf16", "8 bits"])
def chain(request, cure):  # noqa: F811
    """A prompt with images through PromptPass; then what a step behind it takes, and where its next tokens stand."""
    from paper_2608_00531_gb300.step import PromptPass, RepairVerifyStep, StepInputs
    n, held = [40, 7, 129], request.param
    g = torch.Generator(device=DEV).manual_seed(5)
    rnd = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)  # noqa: E731
    base = [Cache(cure, [x + 3 * N_MAX for x in n], HKV, 16, 8) for _ in range(LAYERS)]
    kv, start = base[0].kv, _packed(n, 0)
    codes = [[c.codes[w] for c in base] for w in (0, 1)]
    scales = [[c.scales[w] for c in base] for w in (0, 1)]
    if not held:
        codes, scales = [[torch.zeros(c.codes[0].shape, dtype=torch.bfloat16, device=DEV) for c in base] for _ in (0, 1)], None
    rope, axes = cure.rope_desc(128, 1e6), cure.rope_axes([0] * 16 + [1] * 24 + [2] * 24)
    # text, an image of 4 rows of 5 from position 3 on (20 tokens that move the text on by 5), text
    pos, at = [[], [], []], []
    for m in n:
        p = [(j, j, j) if j < 3 else (3, 3 + (j - 3) // 5, 3 + (j - 3) % 5) if j < 23 else (j - 15,) * 3 for j in range(m)]
        for a in range(3):
            pos[a].extend(x[a] for x in p)
        at.append(max(max(x) for x in p) + 1)
    p = PromptPass(start[-1], B, HQ, kv, rope, DEV)
    row_start, none = _i32(start), _i32([0] * B)
    for l in range(LAYERS):
        p.layer(l, rnd(start[-1], (HQ + 2 * HKV) * 128), row_start, none, codes[0][l], codes[1][l], pos=_i32(pos), axes=axes,
                scales=None if scales is None else (scales[0][l], scales[1][l]))
    step = RepairVerifyStep(B, K, V, 3, 1.0, R, 2, 1, LAYERS, HQ, kv, DEV, rope=rope)
    x = StepInputs(rnd(B, K, V), _i32([0] * B), p.advance(row_start, none), None, None, None, None, rnd(B, N_MAX, V),
                   rnd(LAYERS, B, N_MAX, (HQ + 2 * HKV) * 128))
    kw = {} if scales is None else dict(scales=scales)
    return dict(step=step, x=x, at=at, n=n, rope=rope, axes=axes, run=lambda x: step.run(x, codes[0], codes[1], **kw),
                caches=codes, rnd=rnd)


def _check_rows(cure, c, x, tree, at):  # noqa: F811
    """The rows that the step made of its projections: those of positions at[b] + depth, on every axis."""
    nn, depth = tree["n_nodes"].tolist(), tree["depth"].long()
    for b in range(B):
        want = torch.tensor(at[b], device=DEV) + depth[b, :nn[b]]
        assert torch.equal(tree["pos"][b, :nn[b]].long(), want) and torch.all(tree["pos"][b, nn[b]:] < 0)
    for l in range(LAYERS):
        qkv = x.qkv[l].unflatten(-1, (-1, 128))
        parts = qkv[..., :HQ, :], qkv[..., HQ:HQ + HKV, :], qkv[..., HQ + HKV:, :]
        pos = tree["pos"].flatten()
        outs = [torch.zeros(t.shape, dtype=torch.bfloat16, device=DEV) for t in parts]
        cure.cure_rope_qkv(*parts, pos.expand(3, -1).contiguous(), c["rope"], axes=c["axes"], out=tuple(outs))
        for got, three, raw, turned in zip(c["step"]._rows, outs, parts, (True, True, False)):
            for b in range(B):
                assert torch.equal(got[l, b, :nn[b]], three[b, :nn[b]])
                ref = raw[b, :nn[b]].double()
                if turned:
                    ref = _rotated(ref, tree["pos"][None, b, :nn[b]], 128, 1e6, "half", [0] * 64)
                tol = 2.0 ** -8 * ref.abs() + 2.0 ** -17 * ref.abs().amax(-1, keepdim=True)
                assert torch.all((got[l, b, :nn[b]].double() - ref).abs() <= tol)


def test_steps_behind_images(cure, chain):  # noqa: F811
    c, at = chain, list(chain["at"])
    assert at != c["n"]
    x = dataclasses.replace(c["x"], next_pos=_i32(at))
    for _ in range(2):
        lens = x.cache_len.tolist()
        r = c["run"](x)
        _check_rows(cure, c, x, r["tree"], at)
        new = r["resync"]["cache_len"]
        assert new.tolist() == [n + a + 1 for n, a in zip(lens, r["acc"]["accept_len"].tolist())]
        next_pos = x.next_pos + (new - x.cache_len)  # the accepted tokens are text
        at = [p + m - n for p, m, n in zip(at, new.tolist(), lens)]
        x = dataclasses.replace(x, cache_len=new.clone(), next_pos=next_pos)
    assert cure.cure_device_error() == 0


def test_without_next_pos_tokens_stand_at_their_slots(cure, chain):  # noqa: F811
    r = chain["run"](chain["x"])
    _check_rows(cure, chain, chain["x"], r["tree"], chain["n"])
    assert cure.cure_device_error() == 0


def test_next_pos_is_checked(cure, chain):  # noqa: F811
    x = chain["x"]
    for bad, error in ((torch.zeros(B, dtype=torch.int64, device=DEV), TypeError), (_i32([1] * (B + 1)), ValueError),
                       (torch.zeros(B, dtype=torch.int32), ValueError)):
        with pytest.raises(error):
            chain["run"](dataclasses.replace(x, next_pos=bad))


def test_from_host(cure, chain):  # noqa: F811
    """run_from_host takes rows that are rotated already; its tree has the positions that it is given.  It refuses caches in
    8 bits."""
    from paper_2608_00531_gb300.step import StepInputs
    x, rnd = chain["x"], chain["rnd"]
    xh = StepInputs(*(t.cpu() for t in (x.draft_logits, x.root_tok, x.cache_len)), None,
                    *(rnd(LAYERS, B, N_MAX, h, 128).cpu() for h in (HQ, HKV, HKV)), x.target_logits.cpu(),
                    next_pos=torch.tensor(chain["at"], dtype=torch.int32))
    if chain["caches"][0][0].dtype is not torch.bfloat16:
        with pytest.raises(TypeError):
            chain["step"].run_from_host(xh, *chain["caches"])
        torch.cuda.synchronize()
        return
    for want, xh in ((chain["at"], xh), (chain["n"], dataclasses.replace(xh, next_pos=None))):
        r = chain["step"].run_from_host(xh, *chain["caches"])
        tree = r["tree"]
        for b, m in enumerate(tree["n_nodes"].tolist()):
            assert torch.equal(tree["pos"][b, :m] - tree["depth"][b, :m], torch.full_like(tree["pos"][b, :m], want[b]))
    assert cure.cure_device_error() == 0
