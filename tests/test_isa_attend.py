"""Attention's loads into LDS take their address there from m0, which an instruction sequence of the source's own sets.  The compiler has no way to be told (m0 in a
list of clobbers is reserved, and not looked at), so nothing else in these kernels may use it."""
import concurrent.futures
import os
import re

import pytest

#: instructions that read or write m0 without naming it (those that load into LDS are looked at one by one)
SILENT = r"\b(?:s_movrel\w*|v_movrel\w*|s_sendmsg\w*|ds_gws\w*|ds_append|ds_consume|ds_ordered_count|v_interp\w*|buffer_load\w*\s[^\n]*\blds\b)"


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    from paper_2512_11920_amd import build

    d = tmp_path_factory.mktemp("asm")
    units = [u for u in build.UNITS if u[0] == "kvc_attend.hip"]
    assert len(units) == 8
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        return {obj: open(f.result()).read() for obj, f in [(obj, ex.submit(build.compile_unit, src, defs, str(d / (obj + ".s")), (), True)) for src, defs, obj in units]}


def test_m0_is_set_for_every_load_into_lds_and_used_by_nothing_else(asm):
    for name, text in asm.items():
        lines = [l.split(";")[0].strip() for l in text.splitlines()]
        lines = [l for l in lines if l and not l.startswith((";", "."))]
        loads = [i for i, l in enumerate(lines) if l.startswith("global_load_lds")]
        assert len(loads) > 20, name
        for i in loads:
            assert re.fullmatch(r"s_mov_b32 m0, s\d+", lines[i - 2]) and lines[i - 1] == "s_nop 0", (name, lines[i - 2:i + 1])
        named = [i for i, l in enumerate(lines) if re.search(r"\bm0\b", l)]
        assert named == [i - 2 for i in loads], (name, [lines[i] for i in set(named) - {i - 2 for i in loads}][:3])
        assert not re.search(SILENT, "\n".join(lines)), name
