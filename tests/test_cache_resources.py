"""What the kernels around the 8-bit cache spill, and which calls take which: of the library as it is built."""
import ctypes
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_14107_amd import dejavu as dj

from .test_kernel_resources import LLVM, kernels, of  # noqa: F401 (a fixture)

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


@pytest.mark.parametrize("kind", ["window", "behind", "shared"])
def test_resident_blocks_of_windows_and_shared_prefixes(kernels, kind):
    """As of attention over all keys: what the choice of tiles and splits counts on, of registers and LDS."""
    def resident(name, lds=None):
        k, = of(kernels, name)
        return min(512 // (-(-k["vgpr_count"] // 8) * 8), (160 << 10) // (lds or k["group_segment_fixed_size"]))

    small, large = (f"cache_{kind}_k", f"cache_{kind}_tile_k") if kind != "shared" else ("cache_shared_small_k", "cache_shared_k")
    for dh in range(16, 129, 16):
        count = 2 if dh > 85 else 3 if dh > 64 else 4
        assert resident(f"{small}ILi{dh}ELb1E") >= count and resident(f"{small}ILi{dh}ELb0E") >= 2, dh
        lds = max(2 * 64 * (2 * dh + 16) + 2 * dh * (2 * 64 + 16) + 16, 4 * 4 * 16 * (dh + 6))   # (large tiles', or small ones' partial results)
        for one in (0, 1):
            assert resident(f"{large}ILi{dh}ELb{one}E", lds) >= 2, dh


def test_what_spills(scratch):
    """Attention and norms of rows spill nothing; writes do where a lane takes one channel, and a little in bf16 without norms with rows
    ahead and with norms by fours."""
    for k, v in scratch.items():
        if re.search(r"cache_(attn|window|behind|shared|join|read|extend)|norm_rotary_k", k):
            assert v == 0, k
    most = {"Lb1ELi8": 20, "Lb0ELi8": 0, "Lb1ELi4": 28, "Lb0ELi4": 0}
    writes = {k: v for k, v in scratch.items() if "cache_write_k" in k and "Li1E" not in k}
    assert len(writes) == 14
    for k, v in writes.items():
        assert v <= most[re.search(r"cache_write_kI(Lb[01]ELi[48])", k).group(1)], k
        assert v == 0 or "Li4E" in k or "ELb0ELb1E" in k, k
