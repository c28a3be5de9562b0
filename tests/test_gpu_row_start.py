"""A row_start that does not ascend: which rows cure_append_kv writes, and what it and cure_prompt_attn report."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
D, HKV, ROWS, PS = 128, 2, 12, 8
NODES, PAGE = 0x4, 0x1


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


# row_start; contiguous: {row: (sequence, slot)} and bits; the same in pages, where sequences 1 and 2 have one good page
CASES = [
    ([0, 9, 3, 12, 12], {0: (0, 0), 1: (0, 1), 2: (0, 2), 9: (2, 6), 10: (2, 7), 11: (2, 8)}, NODES),
    ([0, 12, 4, 4, 4], {r: (0, r) for r in range(4)}, NODES),        # rows 4 .. 11 lie before the end 12
    ([-3, 4, 4, 4, 12], {r: (3, r - 4) for r in range(4, 12)}, NODES),
    ([11, 2, 2, 2, 2], {}, 0),                                       # before the first start or behind every end
    ([0, 0, 0, 11, 12], {**{r: (2, r) for r in range(11)}, 11: (3, 0)}, 0),
]


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("start,rows,bits", CASES)
def test_append(cure, start, rows, bits, paged):
    table = np.array([[0, 1], [2, -1], [3, 99], [4, 5]], dtype=np.int32)
    if paged:
        kv = cure.kv_desc(HKV, D, 2, block_table=torch.from_numpy(table).to(DEV), page_size=PS, num_pages=6)
        kc, vc = (torch.full((6, PS, HKV, D), 2.25, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    else:
        kv = cure.kv_desc(HKV, D, 16)
        kc, vc = (torch.full((4, 16, HKV, D), 2.25, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    want = vc.clone()
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.empty(ROWS, HKV, D, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    for r, (b, slot) in rows.items():
        if paged:
            page = table[b, slot // PS]
            if not 0 <= page < 6:
                bits |= PAGE
                continue
            want[page, slot % PS] = v[r]
        else:
            want[b, slot] = v[r]
    cure.cure_append_kv(k, v, kc, vc, kv, _i32(start), _i32([0] * 4), cure.rope_desc(D, 1e4))
    assert cure.cure_device_error() == bits
    assert torch.equal(vc, want)


@pytest.mark.parametrize("start,rows,bits", CASES)
def test_prompt_attention_reports_each(cure, start, rows, bits):
    kv = cure.kv_desc(HKV, D, 16)
    kc, vc = (torch.zeros(4, 16, HKV, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.zeros(ROWS, HKV, D, dtype=torch.bfloat16, device=DEV)
    cure.cure_prompt_attn(q, kc, vc, kv, _i32(start), _i32([0] * 4), 1.0)
    ascends = start[0] >= 0 and all(a <= b for a, b in zip(start, start[1:]))
    assert cure.cure_device_error() == (0 if ascends else NODES)
