"""Direct global-to-LDS loads read m0, which needs one wait state behind the
instruction that writes it.  The compiler adds none inside a statement of inline
assembly, so the machine code of the files that hold such statements is checked:
between a write of m0 and a direct load stands at least one other instruction."""
import glob
import os
import re
import subprocess

import pytest

from paper_2606_08635_amd import build as B


def _too_close(asm):
    """Direct loads of an assembly listing whose previous instruction writes m0, and how many there are in all."""
    last, close, loads = "", [], 0
    for line in asm.splitlines():
        line = line.split(";")[0].strip()
        if not line or line.endswith(":") or line.startswith((".", "//")):
            continue
        if re.match(r"(global|buffer)_load\S*", line) and ("_lds_" in line or re.search(r"\blds\b", line)):
            loads += 1
            if re.match(r"s_\w+ m0\b", last):
                close.append(line)
        last = line
    return close, loads


def test_the_check_sees_a_missing_wait():
    bad = "\ts_mov_b32 m0, s4\n; note\n\tglobal_load_lds_dwordx4 v[2:3], off\n"
    assert _too_close(bad) == (["global_load_lds_dwordx4 v[2:3], off"], 1)
    assert _too_close(bad.replace("; note", "\ts_nop 0")) == ([], 1)


@pytest.mark.parametrize("source", ["attn.hip", "ceiling.hip"])
def test_machine_code_waits_between_m0_and_the_load(source, tmp_path):
    if not os.path.exists(B.HIPCC):
        pytest.skip("hipcc not found")
    out = str(tmp_path / "listing.s")
    subprocess.run([B.HIPCC, *B.FLAGS, "--offload-device-only", "-S", os.path.join(B.CSRC, source), "-o", out],
                   check=True, capture_output=True, timeout=300)
    with open(out) as f:
        close, loads = _too_close(f.read())
    assert loads > 0 and close == []


def test_every_statement_waits_between_m0_and_the_load():
    """The same in the sources' own assembly text, the files included that take long to compile."""
    found = 0
    for path in sorted(glob.glob(os.path.join(B.CSRC, "**", "*.h*"), recursive=True)):
        with open(path) as f:
            for text in re.findall(r'"(s_mov_b32 m0[^"]*)"', f.read()):
                close, loads = _too_close(text.replace(r"\n\t", "\n"))
                found += loads
                assert close == [], path
    assert found >= 5
