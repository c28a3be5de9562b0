"""Prompt attention's own way out when a wait of one of its roles runs out: the call ends, CURE_DEVERR_TIMEOUT comes
back through cure_device_error, what was written is right, and the next call on the same workspace is too.  The wait is
for a barrier that nothing completes, with a limit of 2^20 cycles; nothing faults, traps or hangs."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
D = 128
SCALE = 1.0 / math.sqrt(D)
# warps 0-3, 4-7: softmax of each M tile; 8: copies; 9, 10: products; 11: scheduler; 12-15: epilogue
SOFTMAX, COPIES, S, PV, SCHEDULER, EPILOGUE = (0, 5), 8, 9, 10, 11, (12, 15)


@pytest.fixture(scope="module")
def cure():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2608_00531_gb300 import cure as c
    torch.cuda.set_device(DEV)
    return c


@pytest.fixture(scope="module")
def cases(cure):
    """A unit that all CTAs share (6 to 8 tiles each), and units of one tile, ten to a CTA."""
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    g = torch.Generator(device=DEV).manual_seed(7)
    rnd = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV).normal_(generator=g)  # noqa: E731
    made = {}
    for name, lens, n, Hq, Hkv in (("cut", [150000], [32], 8, 1), ("whole", [0] * 200, [60] * 200, 28, 4)):
        cap, start = max(a + b for a, b in zip(lens, n)), [0]
        for x in n:
            start.append(start[-1] + x)
        args = [rnd(start[-1], Hq, D), rnd(len(n), cap, Hkv, D), rnd(len(n), cap, Hkv, D), cure.kv_desc(Hkv, D, cap),
                i32(start), i32(lens), SCALE]
        ws = torch.empty(cure.cure_prompt_attn_workspace_size(start[-1], len(n), Hq, args[3]), dtype=torch.uint8,
                         device=DEV)
        want = cure.cure_prompt_attn(*args, workspace=ws).clone()
        assert cure.cure_device_error() == 0 and torch.isfinite(want).all()
        made[name] = (args, ws, want)
    return made


def _check(cure, case, warp, wait):
    args, ws, want = case
    out = torch.full_like(want, 3.5)
    cure.cure_selftest_prompt_timeout(*args, warp, wait, out=out, workspace=ws)
    from paper_2608_00531_gb300 import _lib
    assert cure.cure_device_error() == _lib.DEVERR_TIMEOUT
    assert torch.all((out == want) | (out == 3.5))
    for _ in range(2):
        out.fill_(3.5)
        cure.cure_prompt_attn(*args, out=out, workspace=ws)
        assert cure.cure_device_error() == 0
        assert torch.equal(out, want)


@pytest.mark.parametrize("warp,waits", [(SOFTMAX[0], (1, 2, 3, 9)), (SOFTMAX[1], (1, 2, 8)), (COPIES, (1, 2, 3, 4, 11)),
                                        (S, (1, 2, 3, 4, 13)), (PV, (1, 2, 3, 4, 5, 12)), (SCHEDULER, (1, 2)),
                                        (EPILOGUE[0], (1, 2, 3, 4, 6)), (EPILOGUE[1], (1, 5, 6))])
def test_a_wait_runs_out_in_a_cut_unit(cure, cases, warp, waits):
    for wait in waits:
        _check(cure, cases["cut"], warp, wait)


@pytest.mark.parametrize("warp,waits", [(SOFTMAX[0], (2, 7)), (SOFTMAX[1], (2, 7)), (COPIES, (2, 9)), (S, (3, 10)),
                                        (PV, (3, 10)), (SCHEDULER, (1, 7)), (EPILOGUE[0], (2, 8)), (EPILOGUE[1], (3, 8))])
def test_a_wait_runs_out_among_whole_units(cure, cases, warp, waits):
    for wait in waits:
        _check(cure, cases["whole"], warp, wait)


def test_a_wait_that_is_not_reached(cure, cases):
    args, ws, want = cases["cut"]
    assert torch.equal(cure.cure_selftest_prompt_timeout(*args, 11, 1000, workspace=ws), want)
    assert cure.cure_device_error() == 0


def test_refusals(cure, cases):
    from paper_2608_00531_gb300._lib import CureError
    args, ws, _ = cases["cut"]
    for warp, wait in ((-1, 1), (16, 1), (0, 0)):
        with pytest.raises(CureError):
            cure.cure_selftest_prompt_timeout(*args, warp, wait, workspace=ws)
    assert cure.cure_device_error() == 0
