"""The way out of the attention kernels over caches in 8 bits when a wait of one of their roles runs out: the call ends,
CURE_DEVERR_TIMEOUT comes back through cure_device_error, what was written is right, and the next call on the same workspace
is too.  The wait is for a barrier that nothing completes, with a limit of 2^20 cycles; nothing faults, traps or hangs."""
import pytest
import torch

from test_gpu_cache8 import SCALE, _prompt, _tree, cure  # noqa: F401

pytestmark = pytest.mark.gpu

# packed rows and trees, of warps: 0-3, 4-7 softmax of each M tile, or in turn; 8 copies; 9, 10 products; 11 scheduler;
# 12-15 V tiles and the epilogue.  Single tokens: 0-10 attend, 11 the scheduler
FORMS = ("cut", "whole", "tree", "trees", "clusters", "small clusters", "tokens cut", "tokens whole", "tokens alone")


@pytest.fixture(scope="module")
def cases(cure):  # noqa: F811
    """Each form's call: its function, the self-test's, arguments, workspace and the right outputs."""
    made = {}
    for name, x in (
            ("cut", _prompt(cure, [150000], [32], 8, 1, 0, 1)),  # a unit that all CTAs share, 6 tiles of it in the first
            ("whole", _prompt(cure, [0] * 200, [60] * 200, 28, 4, 16, 2)),  # units of a tile
            ("tokens cut", _prompt(cure, [150000] * 3, [1] * 3, 7, 1, 16, 3)),  # 60 steps of keys a CTA
            ("tokens whole", _prompt(cure, [3000] * 64, [1] * 64, 28, 4, 16, 4)),
            ("tokens alone", _prompt(cure, [300] * 200, [1] * 200, 32, 8, 16, 5)),  # 10 steps, a warp each
            ("tree", _tree(cure, [20000], [200], 200, 128, 1, 16, 6)),  # 100 units, cut
            ("trees", _tree(cure, [1000] * 32, [33] * 32, 33, 28, 4, 16, 7)),
            ("clusters", _tree(cure, [4096], [25], 25, 32, 8, 16, 8)),
            ("small clusters", _tree(cure, [2000], [100], 100, 28, 4, 0, 9))):
        if "anc" in x:
            calls = cure.cure_tree_attn8, cure.cure_selftest_tree8_timeout
            args = (x["q"], *x["cache"].args(), x["cache_len"], x["n_nodes"], x["anc"], SCALE)
            size = cure.cure_tree_attn8_workspace_size(len(x["lens"]), x["q"].shape[1], x["q"].shape[2], x["cache"].kv)
        else:
            calls = cure.cure_prompt_attn8, cure.cure_selftest_prompt8_timeout
            args = (x["q"], *x["cache"].args(), x["row_start"], x["cache_len"], SCALE)
            size = cure.cure_prompt_attn8_workspace_size(x["q"].shape[0], len(x["lens"]), x["q"].shape[1], x["cache"].kv)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        want = calls[0](*args, workspace=ws).clone()
        assert cure.cure_device_error() == 0 and torch.isfinite(want).all()
        made[name] = (*calls, args, ws, want)
    return made


def _check(cure, case, warp, wait):  # noqa: F811
    from paper_2608_00531_gb300 import _lib
    call, selftest, args, ws, want = case
    out = torch.full_like(want, 3.5)
    selftest(*args, warp, wait, out=out, workspace=ws)
    assert cure.cure_device_error() == _lib.DEVERR_TIMEOUT, (warp, wait)
    assert torch.all((out == want) | (out == 3.5)), (warp, wait)
    for _ in range(2):
        out.fill_(3.5)
        call(*args, out=out, workspace=ws)
        assert cure.cure_device_error() == 0
        assert torch.equal(out, want), (warp, wait)


def _run(cure, case, waits):  # noqa: F811
    for warp, numbers in waits.items():
        for wait in numbers:
            _check(cure, case, warp, wait)


def test_a_cut_unit(cure, cases):  # noqa: F811
    _run(cure, cases["cut"], {0: (1, 2, 3, 4, 9), 5: (1, 2, 3, 8), 8: (1, 2, 3, 4, 5, 6, 12), 9: (1, 2, 3, 4, 5, 6, 7, 13),
                              10: (1, 2, 3, 4, 5, 6, 13), 11: (1, 2), 12: (1, 2, 3, 8, 14, 15, 16, 17, 18, 19), 15: (1, 9, 15, 17)})


def test_whole_units(cure, cases):  # noqa: F811
    _run(cure, cases["whole"], {0: (1, 2, 3, 7), 5: (1, 2, 7), 8: (1, 2, 3, 4, 9), 9: (1, 3, 10), 10: (1, 3, 10), 11: (1, 7),
                                12: (1, 2, 3, 8), 15: (3, 8)})


def test_trees(cure, cases):  # noqa: F811
    _run(cure, cases["tree"], {0: (1, 2, 3, 4, 9), 5: (1, 2, 3, 8), 8: (1, 2, 4, 5, 12), 9: (1, 2, 3, 4, 5, 13),
                               10: (1, 2, 3, 4, 13), 11: (1, 2), 12: (1, 2, 3, 8)})
    _run(cure, cases["trees"], {0: (2, 6), 5: (2, 5), 8: (3, 9), 9: (3, 9), 10: (3, 9), 11: (1,), 12: (2, 7), 15: (3, 8)})


@pytest.mark.parametrize("name", ["clusters", "small clusters"])
def test_clusters(cure, cases, name):  # noqa: F811
    """The unit whose cluster has a CTA that gave up is left unwritten by all of them."""
    _run(cure, cases[name], {0: (1, 2, 3, 4), 5: (1, 2, 3), 8: (1, 2, 3, 4, 5, 6, 7), 9: (1, 2, 3, 4, 5, 6, 7, 8),
                             10: (1, 2, 3, 4, 5, 6, 7, 8), 12: (1, 2, 3, 4, 5, 6, 7, 8, 9, 10), 15: (1, 5, 8)})


def test_single_tokens(cure, cases):  # noqa: F811
    _run(cure, cases["tokens cut"], {0: (1, 2, 3, 5, 8, 9, 10, 11), 4: (2, 3, 7), 10: (1, 2, 3, 4), 11: (1, 2)})
    _run(cure, cases["tokens whole"], {0: (1, 2, 3, 8, 11, 12, 13), 9: (3, 7), 11: (1, 2)})
    _run(cure, cases["tokens alone"], {0: (1, 2, 3, 8), 3: (2, 4), 11: (1, 2)})


def test_a_wait_that_is_not_reached(cure, cases):  # noqa: F811
    for name in FORMS:
        call, selftest, args, ws, want = cases[name]
        assert torch.equal(selftest(*args, 11, 100000, workspace=ws), want)
    assert cure.cure_device_error() == 0


def test_refusals(cure, cases):  # noqa: F811
    from paper_2608_00531_gb300._lib import CureError
    for name in ("cut", "tree", "tokens cut"):
        call, selftest, args, ws, _ = cases[name]
        for warp, wait in ((-1, 1), (16, 1), (0, 0), (0, -3)):
            with pytest.raises(CureError):
                selftest(*args, warp, wait, workspace=ws)
    assert cure.cure_device_error() == 0
