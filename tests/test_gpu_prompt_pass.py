"""A layer of a PromptPass that its attention refuses leaves the cache as it was: nothing is appended before the whole
call is known to run."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
D, HQ, HKV = 128, 4, 2


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


def _outputs():
    good = torch.zeros(3, HQ, D, dtype=torch.bfloat16, device=DEV)
    odd = torch.zeros(good.numel() + 1, dtype=torch.bfloat16, device=DEV)[1:].view(good.shape)  # aligned to 2 bytes
    return dict(rows=good[:2], heads=good[:, :2].contiguous(), type=good.float(), strides=good.transpose(0, 1).contiguous()
                .transpose(0, 1), device=good.cpu(), alignment=odd)


@pytest.mark.parametrize("kind", ["rows", "heads", "type", "strides", "device", "alignment"])
def test_a_refused_output_leaves_the_cache(mods, kind):
    cure, step = mods
    kc, vc = (torch.full((1, 8, HKV, D), 2.25, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    p = step.PromptPass(3, 1, HQ, cure.kv_desc(HKV, D, 8), cure.rope_desc(D, 1e4), DEV)
    x = torch.ones(3, (HQ + 2 * HKV) * D, dtype=torch.bfloat16, device=DEV)
    with pytest.raises((ValueError, TypeError)):
        p.layer(0, x, _i32([0, 3]), _i32([0]), kc, vc, out=_outputs()[kind])
    torch.cuda.synchronize()
    assert torch.all(kc == 2.25) and torch.all(vc == 2.25) and cure.cure_device_error() == 0


def test_more_sequences_than_the_attention_takes_leave_the_cache(mods):
    cure, step = mods
    B = 257
    kc, vc = (torch.full((B, 2, HKV, D), 2.25, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    p = step.PromptPass(B, 4, HQ, cure.kv_desc(HKV, D, 2), cure.rope_desc(D, 1e4), DEV)
    x = torch.ones(B, (HQ + 2 * HKV) * D, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        p.layer(0, x, _i32(list(range(B + 1))), _i32([0] * B), kc, vc)
    torch.cuda.synchronize()
    assert torch.all(kc == 2.25) and torch.all(vc == 2.25)
    # as many as it takes, more than the pass was made for
    n = 256
    p.layer(0, x[:n], _i32(list(range(n + 1))), _i32([0] * n), kc, vc)
    torch.cuda.synchronize()
    assert torch.all(kc[:n, 0] != 2.25) and torch.all(kc[n:] == 2.25) and cure.cure_device_error() == 0
