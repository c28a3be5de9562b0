"""Calls over every layer's cache in 8 bits refuse a block table with fewer rows than the batch has sequences, before
anything is launched."""
import pytest
import torch

from test_gpu_cache8 import DEV, Cache, _i32, cure  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_table_of_too_few_rows_is_refused(cure):  # noqa: F811
    c = Cache(cure, [40, 20], 2, 16, 1)  # a table of two rows
    one = ([c.codes[0]], [c.codes[1]], [c.scales[0]], [c.scales[1]], c.kv)
    before = [t.view(torch.uint8).clone() for t in (*c.codes, *c.scales)]
    for B in (3, 9):
        lens = _i32([3] * B)
        tree = torch.randn(1, B, 9, 2, 128, device=DEV).bfloat16()
        acc = dict(path_nodes=_i32([[0, 1, -1, -1, -1, -1]] * B), accept_len=_i32([1] * B), diverge_depth=_i32([-1] * B),
                   out_tokens=_i32([[1] * 6] * B))
        saved = torch.zeros(cure.cure_save_kv8_size(1, B, c.kv), dtype=torch.uint8, device=DEV)
        for call in (lambda: cure.cure_resync_kv8(*one, tree, tree, acc, lens, 4),
                     lambda: cure.cure_save_kv8(*one, lens), lambda: cure.cure_restore_kv8(*one, lens, saved)):
            with pytest.raises(ValueError, match="block_table"):
                call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, t.view(torch.uint8)) for a, t in zip(before, (*c.codes, *c.scales)))
    assert cure.cure_device_error() == 0
