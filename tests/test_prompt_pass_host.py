"""PromptPass refuses in its constructor what its attention cannot take, without a GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def mods():
    import __graft_entry__
    try:
        __graft_entry__.build()
    except RuntimeError as e:  # no toolkit on this machine
        pytest.skip(f"cannot build libcure: {e}")
    from paper_2608_00531_gb300 import cure, step
    return cure, step


def _make(mods, rows=4, batch=2, heads_q=4, heads_kv=2, max_len=64):
    cure, step = mods
    kv = cure.kv_desc(heads_kv, 128, max_len)
    return step.PromptPass(rows, batch, heads_q, kv, cure.rope_desc(128, 1e4), torch.device("cpu"))


@pytest.mark.parametrize("bad", [dict(batch=257), dict(rows=(1 << 22) + 1, heads_q=2), dict(heads_q=5), dict(heads_q=0),
                                 dict(heads_q=258), dict(rows=-1), dict(batch=-1)])
def test_shapes_that_the_attention_refuses(mods, bad):
    with pytest.raises(ValueError):
        _make(mods, **bad)


def test_the_largest_shapes(mods):
    for ok in (dict(batch=256), dict(rows=1 << 22, heads_q=2), dict(heads_q=256), dict(rows=0), dict(batch=0)):
        cure, _ = mods
        p = _make(mods, **ok)
        assert p.workspace.numel() == cure.cure_prompt_attn_workspace_size(4, 2, 4, p.kv)
