"""No kernel takes the amount of a 64-bit shift from the last vector register of its allocation: gfx950 reads such an amount wrong now and
then (tests/test_gpu_dropout.py::test_masks_of_many_rows_that_end_inside_a_word failed so), and the compiler does not avoid it."""
import glob
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

import __graft_entry__ as entry

LLVM = os.environ.get("ROCM_LLVM", "/opt/rocm/llvm/bin")
TOOLS = [os.path.join(LLVM, t) for t in ("llvm-objcopy", "clang-offload-bundler", "llvm-readelf", "llvm-objdump")]


def last_register_shifts(notes, listing):
    """(64-bit shifts by a vector register, those whose register is the last of the kernel's allocation, in blocks of 8)."""
    counts = {}
    for block in notes.split("- .agpr_count:")[1:]:
        counts[re.search(r"\.name:\s+(\S+)", block).group(1)] = int(re.search(r"\.vgpr_count:\s+(\d+)", block).group(1))
    kernel, seen, last = None, 0, []
    for line in listing.split("\n"):
        m = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
        if m:
            kernel = m.group(1)
            continue
        m = re.search(r"v_(?:lshlrev_b64|lshrrev_b64|ashrrev_i64)\S* v\[\d+:\d+\], v(\d+),", line)
        if m:
            seen += 1
            if kernel not in counts or int(m.group(1)) + 1 >= (counts[kernel] + 7) // 8 * 8:
                last.append((kernel, line.strip()[:60]))
    return seen, last


def test_the_reader_of_listings():
    notes = "- .agpr_count: 0\n .name: k\n .vgpr_count: 47\n"
    line = "\tv_lshlrev_b64 v[2:3], v%d, v[4:5] // 00"
    assert last_register_shifts(notes, "00 <k>:\n" + line % 46) == (1, [])
    assert last_register_shifts(notes, "00 <k>:\n" + line % 47)[1]
    assert last_register_shifts(notes, "00 <k>:\n\tv_lshlrev_b64 v[2:3], s4, v[4:5]") == (0, [])


@pytest.mark.skipif(not all(os.path.exists(t) for t in TOOLS), reason="needs the ROCm LLVM tools")
def test_no_shift_by_the_last_register(tmp_path):
    objects = [os.path.join(entry.BUILD_DIR, os.path.splitext(s)[0] + ".o") for s in entry.SOURCES if s.endswith(".hip")]
    objects = [o for o in objects if os.path.exists(o)]
    if not objects:
        pytest.skip("no objects of a build here")
    objcopy, bundler, readelf, objdump = TOOLS

    def read(obj):
        fat, code = (str(tmp_path / (os.path.basename(obj) + e)) for e in (".fat", ".co"))
        subprocess.run([objcopy, "--dump-section", ".hip_fatbin=" + fat, obj, code + ".o"], check=True)
        subprocess.run([bundler, "--type=o", "--unbundle", "--input=" + fat, "--output=" + code,
                        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True)
        run = lambda *a: subprocess.run(a, check=True, capture_output=True, text=True).stdout  # noqa: E731
        return last_register_shifts(run(readelf, "--notes", code), run(objdump, "-d", "--mcpu=gfx950", code))

    with ThreadPoolExecutor(4) as pool:
        found = list(pool.map(read, objects))
    assert [f for _, last in found for f in last] == []
    assert glob.glob(str(tmp_path / "*.co"))
