"""Registers of the kernels of attention under a score rule and of the eviction, as the compiler reports them (no GPU needed)."""
import re
import struct
import subprocess

import pytest

from paper_2510_21270_amd import binding

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def _code_objects(data):
    """The gfx950 code objects of a library's bundles: a count, then offset, size and target of each entry."""
    for at in (m.start() for m in re.finditer(MAGIC, data)):
        n, = struct.unpack_from("<Q", data, at + len(MAGIC))
        place = at + len(MAGIC) + 8
        for _ in range(n):
            offset, size, length = struct.unpack_from("<3Q", data, place)
            if b"gfx950" in data[place + 24:place + 24 + length]:
                yield data[at + offset:at + offset + size]
            place += 24 + length


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """name -> what the notes of the built library say."""
    with open(binding.LIB_PATH, "rb") as f:
        data = f.read()
    path, found = str(tmp_path_factory.mktemp("code") / "x.co"), {}
    for code in _code_objects(data):
        with open(path, "wb") as f:
            f.write(code)
        text = subprocess.run(["/opt/rocm/llvm/bin/llvm-readelf", "--notes", path], check=True, stdout=subprocess.PIPE, text=True).stdout
        for entry in text.split("  - .agpr_count:")[1:]:
            name = re.search(r"\.name:\s+(\S+)", entry).group(1)
            found[name] = {k: int(v) for k, v in re.findall(r"\.(\w+):\s+(\d+)\n", entry.split(".name:", 1)[1])}
            found[name]["lds"] = int(re.search(r"\.group_segment_fixed_size:\s+(\d+)", entry).group(1))
    return found


def _of(kernels, pattern, n):
    some = {k: v for k, v in kernels.items() if re.search(pattern, k)}
    assert len(some) == n, sorted(some)
    return some.items()


def _spilled(info):
    return info["vgpr_spill_count"], info["private_segment_fixed_size"]


def test_prompts(kernels):
    for name, info in _of(kernels, "prompt_rule_kernel", 20):
        # two waves to a SIMD; LDS is two rings of 128 keys
        assert info["vgpr_count"] <= 256 and info["lds"] < 160 * 1024, name
        if "ILi64E" in name:
            assert _spilled(info) == (0, 0), (name, info)
        else:                                              # in the pass over values that are not finite
            assert info["vgpr_spill_count"] <= 18 and info["private_segment_fixed_size"] <= 80, (name, info)


@pytest.mark.parametrize("held", ["bf16", "e4m3", "i8"])
def test_new_tokens(kernels, held):
    code = {"bf16": binding.PBS_BF16, "e4m3": binding.PBS_E4M3, "i8": binding.PBS_I8}[held]
    for name, info in _of(kernels, "decode_own_kernelILi%dE.*FormArgs" % code, 68):
        _, d, nt, several, _, form = re.search(r"ILi(\d)ELi(\d+)ELi(\d)ELb(\d)ELb(\d)ENS_8FormArgsILi(\d+)E", name).groups()
        assert info["vgpr_count"] <= (256 if nt == "1" else 512), (name, info)
        # one wave's tile of 128 features in bf16 leaves no room for a window: some are kept over its loop, none within it
        full = held == "bf16" and d == "128" and nt == "1"
        assert info["vgpr_spill_count"] <= (25 if full else 0) and info["private_segment_fixed_size"] <= (96 if full else 0), (name, info)
        # forms without positions hold none
        assert info["lds"] <= (64 if int(form) & 15 in (0, 1) else 16448), (name, info)


@pytest.mark.parametrize("pattern,n", [("evict_(select|phase|move)_kernel", 10), ("join_weigh_kernel", 4), ("cache_mark_kernel", 1)])
def test_the_others(kernels, pattern, n):
    for name, info in _of(kernels, pattern, n):
        assert info["vgpr_count"] <= 128 and _spilled(info) == (0, 0) and info["sgpr_spill_count"] == 0, (name, info)
