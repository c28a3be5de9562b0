"""Appends into a contiguous cache in 8 bits whose rows run past its capacity, which need not be a multiple of the scales'
16 slots: what fits is written, what does not is left out and reported, whichever CTA comes upon it."""
import pytest
import torch

from test_gpu_cache8 import D, DEV, Cache, _check_append, _i32, _packed, cure  # noqa: F401

pytestmark = pytest.mark.gpu


def _append_past(cure, cap, lens, n, fits):  # noqa: F811
    """n rows of each sequence, of which `fits` lie below the capacity."""
    Hq, Hkv = 4, 2
    c = Cache(cure, [cap] * len(lens), Hkv, 0, cap + sum(n))
    assert c.cap == cap
    start = _packed(n, 0)
    g = torch.Generator(device=DEV).manual_seed(cap)
    k, v, q = (torch.empty(start[-1], h, D, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)
               for h in (Hkv, Hkv, Hq))
    before, out = c.copy(), torch.full_like(q, 3.5)
    cure.cure_append_kv8(k, v, *c.args(), _i32(start), _i32(lens), None, q=q, out=out)
    assert cure.cure_device_error() == (cure.DEVERR_SLOT if fits != n else 0), (cap, lens, n)
    _check_append(c, before, lens, fits, start, (k, v))
    for b, m in enumerate(fits):
        at = start[b] + m
        assert torch.equal(out[start[b]:at], q[start[b]:at]) and torch.all(out[at:start[b + 1]] == 3.5)


@pytest.mark.parametrize("over", [0, 1, 2, 5, 8, 15, 16, 33])
@pytest.mark.parametrize("cap", [18, 31, 32, 33, 47, 100])
def test_one_sequence(cure, cap, over):  # noqa: F811
    for L in sorted({0, 1, 3, 15, 16, 17, cap - 17, cap - 16, cap - 3, cap - 1, cap}):
        m = cap - L
        if L >= 0 and m + over > 0:
            _append_past(cure, cap, [L], [m + over], [m])


@pytest.mark.parametrize("cap", [18, 45, 100])
def test_several_sequences(cure, cap):  # noqa: F811
    """The one that runs past its capacity first, last and between others, few rows and many on average."""
    for over in (1, 6, 14):
        for others in ([1], [1, 4, 2], [cap] * 3):
            for at in range(len(others) + 1):
                for L in (1, cap - 9):
                    lens, n, fits = [0] * len(others), list(others), list(others)
                    lens.insert(at, L)
                    n.insert(at, cap - L + over)
                    fits.insert(at, cap - L)
                    _append_past(cure, cap, lens, n, fits)
