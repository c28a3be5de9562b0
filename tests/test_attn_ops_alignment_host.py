"""Integer arrays that are not aligned to their type are refused before anything is launched, without a GPU: a kernel
that read them would fault.  The pointers are stand-ins that are never dereferenced; the tests run only where no GPU can
be reached, so that a missing check cannot launch a kernel on them."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("runs only without a reachable GPU")
    import __graft_entry__
    try:
        __graft_entry__.build()
    except RuntimeError as e:  # no toolkit on this machine
        pytest.skip(f"cannot build libcure: {e}")
    from paper_2608_00531_gb300 import _lib
    return _lib.load()


DEV, ODD = C.c_void_p(1 << 20), C.c_void_p((1 << 20) + 2)
INVALID, CUDA = 1, 3


def _kv(table=None):
    from paper_2608_00531_gb300._lib import KVDesc
    return KVDesc(layout=0 if table is None else 1, heads_kv=2, head_dim=128, page_size=16, max_len=8, num_pages=4,
                  block_table=table)


def test_positions(lib):
    call = lambda pos: lib.cure_rope_qkv(DEV, DEV, DEV, 1024, 256, 256, 4, 8, 2, 128, pos, None, None, None, 1e-6, DEV,  # noqa: E731
                                         DEV, DEV, 1024, 256, 256, None)
    assert call(ODD) == INVALID and call(DEV) == CUDA  # the launch, without a device


@pytest.mark.parametrize("which", ["row_start", "cache_len", "pos", "block_table"])
def test_append(lib, which):
    def call(**kw):
        a = dict(dict(row_start=DEV, cache_len=DEV, pos=DEV, block_table=1 << 20), **kw)
        kv = _kv(a["block_table"])
        return lib.cure_append_kv(DEV, DEV, DEV, 1024, 256, 256, 4, 8, 1, a["row_start"], a["cache_len"], a["pos"],
                                  C.byref(kv), DEV, DEV, None, None, None, 1e-6, DEV, 1024, None)
    assert call(**{which: ODD if which != "block_table" else (1 << 20) + 2}) == INVALID
    assert call() == CUDA and call(pos=None) == CUDA


@pytest.mark.parametrize("which", ["row_start", "cache_len", "block_table"])
def test_prompt_attention(lib, which):
    def call(**kw):
        a = dict(dict(row_start=DEV, cache_len=DEV, block_table=1 << 20), **kw)
        kv = _kv(a["block_table"])
        return lib.cure_prompt_attn(DEV, DEV, DEV, C.byref(kv), a["row_start"], a["cache_len"], 4, 1, 8, 0.1, DEV, DEV,
                                    1 << 30, None)
    assert call(**{which: ODD if which != "block_table" else (1 << 20) + 2}) == INVALID
    assert call() == CUDA
