"""``fetch_lds`` in ``csrc/attn_kv.hip`` writes m0 in inline asm.  The compiler keeps that register for itself and takes no declaration of it, so the
built code is checked: in kernels with such fetches nothing else reads or writes m0, neither by name nor by what it does."""
import os

import pytest

from paper_2512_04939_amd import build
from test_isa_lds_waits import LLVM, _code, _disassembly, _kernels

IMPLICIT = ("global_load_lds", "ds_gws", "ds_ordered", "ds_append", "ds_consume", "ds_add_gs", "ds_sub_gs", "s_movrel", "v_movrel", "s_sendmsg", "s_ttrace")


def _fetch(op, args):
    return op.startswith("buffer_load") and args.split()[-1:] == ["lds"]


def strangers(code):
    """Addresses of instructions that have to do with m0 and are no part of a fetch: s_mov to m0, s_nop, load into LDS."""
    bad, i = [], 0
    while i < len(code):
        addr, op, args, _ = code[i]
        if op == "s_mov_b32" and args.startswith("m0,") and i + 2 < len(code) and code[i + 1][1] == "s_nop" and _fetch(*code[i + 2][1:3]):
            i += 3
            continue
        if "m0" in args.replace(",", " ").split() or op.startswith(IMPLICIT) or _fetch(op, args):
            bad.append(addr)
        i += 1
    return bad


def test_m0_belongs_to_the_fetches(tmp_path):
    if not os.path.exists(build.LIB):
        pytest.skip("library not built")
    if not os.path.exists(os.path.join(LLVM, "llvm-objdump")):
        pytest.skip("no disassembler")
    kernels = fetches = 0
    for text in _disassembly(tmp_path):
        for name, code in _kernels(text).items():
            if "k_kv_attn" not in name:      # (the others' fetches are the compiler's own)
                continue
            kernels += 1
            fetches += sum(_fetch(op, args) for _, op, args, _ in code)
            assert strangers(code) == [], name
    assert kernels > 12 and fetches > 50


FETCH = ("s_mov_b32 m0, s3", "s_nop 4", "buffer_load_dwordx4 v0, s[4:7], 0 offen lds")


@pytest.mark.parametrize("lines,bad", [
    (FETCH + FETCH + ("s_endpgm",), []),
    (FETCH[:1] + FETCH[2:] + ("s_endpgm",), [0, 1]),
    (FETCH + FETCH[2:] + ("s_endpgm",), [3]),
    (FETCH + ("s_mov_b32 s9, m0", "s_endpgm"), [3]),
    (("s_mov_b32 m0, s3", "global_load_lds_dwordx4 v[0:1], off") + FETCH, [0, 1]),
    (FETCH + ("v_movrels_b32_e32 v1, v2", "buffer_load_dwordx4 v[0:3], v4, s[4:7], 0 offen", "s_endpgm"), [3]),
])
def test_strangers(lines, bad):
    assert strangers(_code(*lines)) == bad
