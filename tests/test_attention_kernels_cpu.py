"""The attention kernels' loads to LDS take their place from m0, which the compiler does not know of: nothing else in those kernels may use it."""
import os
import re
import subprocess

import pytest

import __graft_entry__ as entry
from test_shift_amounts_cpu import TOOLS


def other_uses(listing):
    """(loads to LDS, lines that set or use m0 in another way than right before one)."""
    lines = [m.group(1) for m in re.finditer(r"^\t(\S.*?)\s*(?://.*)?$", listing, re.M)]
    loads, other, ready = 0, [], False
    for i, line in enumerate(lines):
        if line.startswith("global_load_lds_dwordx4"):
            loads += 1
            if lines[i - 1] != "s_nop 0" or not re.match(r"s_mov_b32 m0, s\d+$", lines[i - 2]):
                other.append(line)
        elif "m0" in re.findall(r"\w+", line):
            if not (line.startswith("s_mov_b32 m0,") and lines[i + 1:i + 2] == ["s_nop 0"] and lines[i + 2].startswith("global_load_lds_dwordx4")):
                other.append(line)
        elif re.match(r"s_movrel|v_movrel|s_sendmsg|ds_\w*(addtid|gws)|buffer_load\S* .*\blds\b|v_interp", line):
            other.append(line)
    return loads, other


def test_the_reader_of_listings():
    good = "\ts_mov_b32 m0, s3 // 00\n\ts_nop 0 // 00\n\tglobal_load_lds_dwordx4 v1, s[2:3] // 00\n"
    assert other_uses(good) == (1, [])
    assert other_uses("\ts_mov_b32 m0, s3 // 00\n\tv_add_f32 v0, v1, v2 // 00\n" + good)[1]
    assert other_uses("\ts_add_u32 s1, s2, m0 // 00\n" + good)[1]


@pytest.mark.skipif(not all(os.path.exists(t) for t in TOOLS), reason="needs the ROCm LLVM tools")
@pytest.mark.parametrize("source", sorted(s for s in entry.SOURCES if re.match(r"lba_attn\w*_(bf16|f32)\.hip$", os.path.basename(s))))
def test_nothing_else_uses_m0(source, tmp_path):
    obj = os.path.join(entry.BUILD_DIR, os.path.splitext(source)[0] + ".o")
    if not os.path.exists(obj):
        pytest.skip("no object of a build here")
    objcopy, bundler, _, objdump = TOOLS
    fat, code = str(tmp_path / "fat"), str(tmp_path / "code.co")
    subprocess.run([objcopy, "--dump-section", ".hip_fatbin=" + fat, obj, code + ".o"], check=True)
    subprocess.run([bundler, "--type=o", "--unbundle", "--input=" + fat, "--output=" + code, "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True)
    loads, other = other_uses(subprocess.run([objdump, "-d", "--mcpu=gfx950", code], check=True, capture_output=True, text=True).stdout)
    assert other == [] and (loads > 0) == ("bf16" in source)
