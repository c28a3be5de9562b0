"""A row's rotation does not depend on how many rows a call has, in whatever parts its heads are then dealt out."""
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


@pytest.mark.parametrize("Hq,Hkv", [(28, 4), (32, 4), (35, 2), (64, 8), (1, 1)])
def test_same_rows_in_calls_of_all_sizes(cure, Hq, Hkv):
    g = torch.Generator(device=DEV).manual_seed(Hq)
    n = 8001
    qkv = torch.empty(n, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    pos = torch.randint(0, 100000, (n,), dtype=torch.int32, device=DEV, generator=g)
    w = (1.0 + 0.1 * torch.randn(D, device=DEV, generator=g)).to(torch.bfloat16)
    rope = cure.rope_desc(128, 1e6)
    parts = lambda m: (qkv[:m, :Hq], qkv[:m, Hq:Hq + Hkv], qkv[:m, Hq + Hkv:])  # noqa: E731
    want = cure.cure_rope_qkv(*parts(n), pos, rope, q_norm=w, k_norm=w)
    for m in (1, 100, 700, 1500, 3647, 3648, 3649, 4500, 5015, 5016, 5017, 7295, 7296, 8000):
        got = cure.cure_rope_qkv(*parts(m), pos[:m], rope, q_norm=w, k_norm=w)
        assert all(torch.equal(a, b[:m]) for a, b in zip(got, want)), m
    assert cure.cure_device_error() == 0
