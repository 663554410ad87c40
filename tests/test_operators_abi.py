"""The calls around the attention on a machine without a GPU: the binding's packed arguments against the header's structs, null
handles and arguments, and the plans of the shared prefix's kernel."""
import ctypes as C
import os
import re

import pytest

import paper_2605_24786_amd as pkg
from paper_2605_24786_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def clib():
    return pkg.load_library()


def _fields(name):
    """(name, ctypes type) of a struct in the header, in order."""
    header = open(os.path.join(ROOT, "include", "conf_kv.h")).read()
    block = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), header, re.S).group(1)
    out = []
    for decl in re.sub(r"/\*.*?\*/", "", block, flags=re.S).split(";"):
        decl = re.sub(r"^const\s+", "", decl.strip())
        if not decl:
            continue
        base, names = re.match(r"(\w+)\s+(.*)", decl, re.S).groups()
        for n in names.split(","):
            n = n.strip()
            kind = C.c_void_p if n.startswith("*") else dict(int32_t=C.c_int32, int64_t=C.c_int64, float=C.c_float)[base]
            out.append((n.lstrip("* "), kind))
    return out


@pytest.mark.parametrize("name,packed", [("conf_kv_prefix", b._PREFIX), ("conf_kv_qkv", b._QKV), ("conf_kv_constraints", b._CONSTRAINTS)])
def test_packed_arguments_match_the_header(name, packed):
    fields = _fields(name)
    struct = type(name, (C.Structure,), {"_fields_": fields})
    assert packed.size == C.sizeof(struct)
    values = [float(i + 1) if k is C.c_float else i + 1 for i, (_, k) in enumerate(fields)]
    got = struct.from_buffer_copy(packed.pack(*values))
    assert [getattr(got, n) for n, _ in fields] == values


def test_null_arguments_are_refused(clib):
    assert clib.conf_kv_prepare_qkv(None, 0, None, None) == b.ERR_INVALID_ARG
    assert clib.conf_kv_prepare_qkv(None, 0, bytes(b._QKV.size), None) == b.ERR_INVALID_ARG
    assert clib.conf_kv_constrain(None, None, None) == b.ERR_INVALID_ARG
    assert clib.conf_kv_constrain(None, bytes(b._CONSTRAINTS.size), None) == b.ERR_INVALID_ARG
    assert clib.conf_kv_attend_shared(None, 0, 1, None, None, None, None, None, None) == b.ERR_INVALID_ARG
    assert clib.conf_kv_attend_shared(None, 0, 1, bytes(b._PREFIX.size), None, None, None, None, None) == b.ERR_INVALID_ARG


def test_scratch_of_a_shared_prefix(clib):
    """max_shared adds up to 64 partial results per query row of a unit, and nothing to the state."""
    def sizes(**kw):
        cfg, *_ = pkg.make_config(n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=128, vocab=1000, capacity=256, fp16_window=16,
                                  protected_window=8, n_tight=[64, 64], n_loose=[128, 128], **kw)
        return clib.conf_kv_state_bytes(C.byref(cfg)), clib.conf_kv_scratch_bytes(C.byref(cfg))
    none, small, large = sizes(), sizes(max_shared=100), sizes(max_shared=1 << 30)
    row = 128 * 4 + 8
    assert none[0] == small[0] == large[0]
    assert 6 * 4 * row <= small[1] - none[1] <= 6 * 4 * row + 1024
    assert 6 * 4 * 64 * row <= large[1] - none[1] <= 6 * 4 * 64 * row + 1024
    chunk = sizes(max_chunk=4)
    assert sizes(max_chunk=4, max_shared=128)[1] - chunk[1] >= 6 * 16 * row        # sixteen rows per unit
    assert sizes(max_shared=-1) == (0, 0) and sizes(max_shared=(1 << 30) + 1) == (0, 0)


class _Plan(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("row_waves", "blocks", "parts", "part_keys")]


def test_plans_of_the_prefix_kernel(clib):
    """Every key lies in one part, no part is empty, all parts fit the scratch, one workgroup per CU where the rows allow it."""
    plan = getattr(clib, "_ZN6confkv11shared_planEiiiiiiPNS_10SharedPlanE")
    most = getattr(clib, "_ZN6confkv17shared_parts_mostEi")
    plan.argtypes, plan.restype, most.restype = [C.c_int] * 6 + [C.POINTER(_Plan)], None, C.c_size_t
    seen = set()
    for rows in (1, 4, 32, 33, 64, 65, 128, 129, 500, 4096):
        for heads in (1, 2, 8, 12, 64, 300):
            for D in (64, 128):
                for T in (1, 31, 32, 33, 255, 256, 257, 1000, 4096, 32001, 200000, 1 << 27):
                    for forced in (0, 1, 2, 4, 3):
                        p = _Plan()
                        plan(rows, heads, D, T, 256, forced, C.byref(p))
                        assert p.row_waves in (1, 2, 4) and (forced not in (1, 2, 4) or p.row_waves == forced)
                        assert p.blocks == -(-rows // (32 * p.row_waves))
                        assert 1 <= p.parts <= most(T) <= 64 and p.part_keys % 32 == 0
                        assert (p.parts - 1) * p.part_keys < T <= p.parts * p.part_keys
                        assert p.parts == 1 or p.parts * p.blocks * heads <= 256
                        if not forced:
                            seen.add(p.row_waves)
    assert seen == {1, 2, 4}
