"""The calls over a paged cache on a machine without a GPU: the binding's packed arguments against the header's structs, null handles
and arguments, the room they take."""
import ctypes as C
import os
import sys

import pytest

import paper_2605_24786_amd as pkg
from paper_2605_24786_amd import binding as b

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_operators_abi import _fields  # noqa: E402


@pytest.mark.parametrize("name,packed", [("conf_kv_pages", b._PAGES), ("conf_kv_chunk", b._CHUNK)])
def test_packed_arguments_match_the_header(name, packed):
    fields = _fields(name)
    struct = type(name, (C.Structure,), {"_fields_": fields})
    assert packed.size == C.sizeof(struct)
    values = list(range(1, len(fields) + 1))
    got = struct.from_buffer_copy(packed.pack(*values))
    assert [getattr(got, n) for n, _ in fields] == values


def test_null_arguments_are_refused():
    lib = pkg.load_library()
    pages, chunk = bytes(b._PAGES.size), bytes(b._CHUNK.size)
    for args in ((None, None), (pages, None), (None, chunk), (pages, chunk)):
        assert lib.conf_kv_attend_pages(None, *args, None) == b.ERR_INVALID_ARG
    assert lib.conf_kv_load_pages(None, 0, None, 0, None, None) == b.ERR_INVALID_ARG
    assert lib.conf_kv_load_pages(None, 0, pages, 0, None, None) == b.ERR_INVALID_ARG


@pytest.mark.parametrize("D", [64, 128])
def test_scratch_of_a_paged_cache(D):
    """max_paged adds the parts' partial results, 256 blocks of 256 rows, and a counter for 512
    where a cache is long enough to be cut, and no state."""
    def sizes(**kw):
        cfg, *_ = pkg.make_config(n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=D, vocab=1000, capacity=256, fp16_window=16,
                                  protected_window=8, n_tight=[64, 64], n_loose=[128, 128], **kw)
        lib = pkg.load_library()
        return lib.conf_kv_state_bytes(C.byref(cfg)), lib.conf_kv_scratch_bytes(C.byref(cfg))
    none, short, long, longest = sizes(), sizes(max_paged=128), sizes(max_paged=129), sizes(max_paged=1 << 30)
    assert none == short and long == longest and none[0] == long[0]
    assert 0 <= long[1] - none[1] - 256 * 256 * (D + 2) * 4 - 2048 <= 512
    assert sizes(max_paged=-1) == (0, 0) and sizes(max_paged=(1 << 30) + 1) == (0, 0)
