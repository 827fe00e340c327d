"""What the kernels of the 8-bit cache and their launches count on: the compiler, the chip, registers and LDS."""
import ctypes
import glob
import os
import re
import shutil
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2506_14107_amd", "csrc")


def test_no_instruction_hides_from_the_compiler():
    """A vector instruction that reads a matrix instruction's result has to stand 8 or 12 wait states behind it,
    which the compiler sees to for its own instructions and not for those of inline assembly: such statements pin
    values to registers and hold no instruction."""
    held = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        with open(path) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        held += [(os.path.basename(path), m.group(1)) for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(\s*((?:\"[^\"]*\"\s*)+)", text)
                 if m.group(1).replace('"', "").strip()]
    assert not held


def test_heads_of_a_writes_blocks_follow_the_chip(tmp_path):
    """Blocks take as many heads as leave two of them a compute unit of whatever device there is."""
    src, so = tmp_path / "heads.cpp", str(tmp_path / "heads.so")
    src.write_text('#include "cache_plan.h"\n'
                   'extern "C" int heads(long long slots, int kv_heads, int cus) { return dv::write_heads(slots, kv_heads, cus); }\n')
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run([shutil.which("g++") or "c++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I",
                    os.path.join(rocm, "include"), "-I", CSRC, str(src), "-o", so], check=True)
    heads = ctypes.CDLL(so).heads
    for cus in (32, 64, 256, 304):
        for kv_heads in (1, 3, 8, 16, 40):
            for slots in (1, 5, 64, 150, 1000, 100000):
                n = heads(ctypes.c_longlong(slots), kv_heads, cus)
                blocks = [slots * 2 * -(-kv_heads // k) for k in range(1, min(16, kv_heads) + 1)]
                assert 1 <= n <= min(16, kv_heads)
                assert blocks[n - 1] >= 2 * cus or n == 1
                assert 2 * n > min(16, kv_heads) or blocks[min(2 * n, len(blocks)) - 1] < 2 * cus
    assert heads(ctypes.c_longlong(150), 16, 0) == heads(ctypes.c_longlong(150), 16, 256) != heads(ctypes.c_longlong(150), 16, 32)
