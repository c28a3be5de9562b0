"""cure_resync_kv8 refuses integer arrays that are not aligned to their type, as the other calls over caches in 8 bits do."""
import ctypes as C

import pytest

from test_cache8_host import DEV, UNALIGNED, _kv, lib  # noqa: F401

ARRAYS = ("path_nodes", "accept_len", "diverge_depth", "out_tokens", "cache_len_in", "cache_len_out", "draft_valid_len",
          "replay_tokens", "n_replay")


@pytest.mark.parametrize("layers", [0, 2])
@pytest.mark.parametrize("name", ARRAYS)
def test_refused(lib, name, layers):  # noqa: F811
    kc, vc, ks, vs = ((C.c_void_p * 2)(i << 20, (i + 1) << 20) for i in (1, 3, 5, 7))
    arrays = {n: DEV for n in ARRAYS}
    for at in (UNALIGNED, C.c_void_p((1 << 20) + 1), None):
        assert lib.cure_resync_kv8(layers, kc, vc, ks, vs, _kv(), DEV, DEV, 1, 9, 8,
                                   *dict(arrays, **{name: at}).values(), None) == 1
