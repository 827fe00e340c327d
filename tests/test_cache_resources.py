"""What the kernels around the 8-bit cache spill, and which calls take which: of the library as it is built."""
import ctypes
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_14107_amd import dejavu as dj

from .test_kernel_resources import LLVM

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2506_14107_amd", "csrc")


@pytest.fixture(scope="module")
def scratch(tmp_path_factory):
    """Mangled name -> bytes of scratch a lane of every kernel in the library."""
    dj.load()
    d = str(tmp_path_factory.mktemp("lib"))
    so = shutil.copy(dj.LIB_PATH, d)
    subprocess.run([os.path.join(LLVM, "llvm-objdump"), "--offloading", so], check=True, capture_output=True, cwd=d)
    out = {}
    for obj in glob.glob(os.path.join(d, "*gfx950")):
        notes = subprocess.run([os.path.join(LLVM, "llvm-readelf"), "--notes", obj], check=True, capture_output=True, text=True).stdout
        for k in re.split(r"\n  - (?=\.agpr)", notes)[1:]:
            out[re.search(r"\n    \.name: +(\S+)", k).group(1)] = int(re.search(r"\.private_segment_fixed_size: +(\d+)", k).group(1))
    return out


def host(tmp_path, code):
    src, so = tmp_path / "host.cpp", str(tmp_path / "host.so")
    src.write_text('#include <cstddef>\n#include "cache_plan.h"\nusing namespace dv;\n' + code)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run([shutil.which("g++") or "c++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I",
                    os.path.join(rocm, "include"), "-I", CSRC, str(src), "-o", so], check=True)
    return ctypes.CDLL(so)


@pytest.mark.parametrize("threads", [256, 512])
def test_writes_of_one_pass_spill_nothing(scratch, threads):
    """bf16, eight channels at once, without norms."""
    found = [v for k, v in scratch.items() if f"cache_write_kILb1ELi8ELi{threads}ELb0ELb0E" in k]
    assert found == [0]


def test_steps_of_single_tokens_take_one_pass(tmp_path):
    """... whatever the heads, as far as a pass's items go; prompts and long writes do not."""
    one = host(tmp_path, 'extern "C" int one(int pt, int dh, int heads, int n, int rows) '
               '{ return write_in_one_pass(pt, dh, heads, n, rows); }\n').one
    for pt in (16, 32, 64, 128):
        for dh in range(16, 129, 16):
            threads = 512 if pt * (dh // 16) > 512 else 256
            for n in (1, 48, 1000):
                for heads in (1, 3, 16):
                    assert one(pt, dh, heads, n, n)
                    for tokens in (2, 5, 40, 200):
                        assert bool(one(pt, dh, heads, n, tokens * n)) == (min(tokens, pt) * (dh // 16) * heads <= 2 * threads)
    assert not one(64, 80, 16, 6, 9232) and not one(64, 128, 8, 4, 60000) and not one(128, 128, 8, 4, (1 << 31) - 1)


def test_arguments_that_every_call_reads_come_first(tmp_path):
    """A block waits for each 64 bytes of its arguments that it reads: what only windows, shared prefixes and norms need lies
    behind what every call does, and sequences hold nothing of groups."""
    at = host(tmp_path, """extern "C" void at(long long* o) {
    const size_t x[] = {sizeof(SeqArgs), offsetof(CacheAttnArgs, many) + sizeof(CacheAttnCut), offsetof(CacheAttnArgs, window),
                        offsetof(CacheAttnArgs, front), offsetof(CacheAttnArgs, groups), offsetof(WriteArgs, by_tok), offsetof(WriteArgs, k_norm)};
    for (size_t i = 0; i < sizeof x / sizeof x[0]; ++i) o[i] = (long long)x[i];
}
""").at
    o = (ctypes.c_longlong * 7)()
    at(o)
    seq, plain, window, front, groups, tok, norm = o
    assert seq == 48 and plain <= min(window, front, groups) and tok < norm
    assert plain <= 4 * 64
