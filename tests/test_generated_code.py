"""CPU tests: what the compiler made of the kernels (see generated_code.py)."""
import os

import pytest

import generated_code as gen
from paper_2211_00839_amd import binding

LISTING = """
0000000000001000 <k>:
\ts_and_saveexec_b64 s[2:3], vcc                             // 000000001000: BE82206A
\ts_cbranch_execz 4                                          // 000000001004: BF880004 <k+0x18>
\tv_add_u32_e32 v2, 64, v2                                   // 000000001008: 680404C0
\ts_andn2_b64 exec, exec, s[36:37]                           // 00000000100C: 89FE247E
\ts_cbranch_execnz 65533                                     // 000000001010: BF89FFFD <k+0x8>
\ts_nop 0                                                    // 000000001014: BF800000
%s\ts_or_b64 exec, exec, s[2:3]                               // 000000001020: 87FE027E
%s\tglobal_load_lds_dwordx4 v6, s[26:27]                      // 00000000102C: DDF48000 001A0006
\ts_endpgm                                                   // 000000001034: BF810000
"""
COPY = "\tv_accvgpr_write_b32 a118, v6                               // 000000001018: D3D94076 18000106\n"
SPILL = "\tv_writelane_b32 v254, s47, 4                               // 000000001018: D28A00FE 0001082F\n"
SHORT = "\ts_nop 0                                                    // 000000001028: BF800000\n"
LONG = "\ts_nop 4                                                    // 000000001028: BF800004\n"


def test_what_is_found():
    def both(*a):
        (name, code), = gen.functions((LISTING % a).splitlines())
        assert name == "k"
        return [text for _, text in gen.moved_before_exec(code)], [text for _, text in gen.short_waits(code)[0]]

    load, copy = "global_load_lds_dwordx4 v6, s[26:27]", "v_accvgpr_write_b32 a118, v6"
    assert both("", LONG) == ([], [])
    assert both(SPILL, LONG) == ([], [])
    assert both("", "") == ([], [load])
    assert both("", SHORT) == ([], [load])
    # (once from the branch and once from the loop's end)
    assert set(both(COPY, LONG)[0]) == {copy}
    assert set(both(SPILL + COPY, LONG)[0]) == {copy}


def test_the_library(tmp_path):
    if not os.path.exists(gen.OBJDUMP):
        pytest.skip("no llvm-objdump")
    if not os.path.exists(binding.lib_path()):
        from paper_2211_00839_amd import build
        build.build()
    loads = kernels = 0
    wrong = []
    objects = gen.code_objects(binding.lib_path())
    assert len(objects) >= 4
    for i, data in enumerate(objects):
        path = str(tmp_path / ("%d.co" % i))
        with open(path, "wb") as f:
            f.write(data)
        for name, code in gen.disassembled(path):
            short, count = gen.short_waits(code)
            wrong += [(name, "%x" % at, text) for at, text in short + gen.moved_before_exec(code)]
            loads += count
            kernels += 1
    assert kernels > 200 and loads > 6000, (kernels, loads)
    assert not wrong, (len(wrong), wrong[:10])
