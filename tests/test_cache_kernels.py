"""What the kernels of the 8-bit cache and their launches count on: the compiler, the chip, registers and LDS."""
import ctypes
import glob
import os
import re
import shutil
import subprocess

from .test_kernel_resources import kernels, of  # noqa: F401 (a fixture)

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


def test_resident_blocks_of_the_attention_kernels(kernels):
    """Blocks of four wavefronts, one a SIMD of 512 registers a lane (in steps of 8), 160 KB of LDS a compute unit: small
    bf16 tiles have at least the blocks there that the choice of tiles counts, every kernel the two that splits count."""
    def resident(name, lds=None):
        k, = of(kernels, name)
        return min(512 // (-(-k["vgpr_count"] // 8) * 8), (160 << 10) // (lds or k["group_segment_fixed_size"]))

    with open(os.path.join(CSRC, "cache_plan.h")) as f:
        rule = re.search(r"small_resident\(int head_dim\) \{ return head_dim > (\d+) \? (\d) : head_dim > (\d+) \? (\d) : (\d); \}", f.read())
    a, few, b, some, many = (int(x) for x in rule.groups())
    for dh in range(16, 129, 16):
        assert resident(f"cache_attn_kILi{dh}ELb1E") >= (few if dh > a else some if dh > b else many), dh
        assert resident(f"cache_attn_kILi{dh}ELb0E") >= 2
        lds = 2 * 64 * (2 * dh + 16) + 2 * dh * (2 * 64 + 16) + 16
        for one in (0, 1):
            assert resident(f"cache_attn_tile_kILi{dh}ELb{one}E", lds) >= 2
