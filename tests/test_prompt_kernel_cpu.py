"""What the assembly statements of the kernels on key_pipeline.h rely on, as the compiler emits it (no GPU needed).

The compiler does not see that these statements are matrix instructions.  It therefore keeps none of the distances that the
hardware asks for: two wait states from a vector instruction's write to a matrix instruction's read of A, B or C, and, after a
32x32x16 product, about a dozen instructions before its result is read."""
import os
import re
import subprocess

import pytest

from paper_2510_21270_amd import build


def _registers(text):
    out = set()
    for kind, lo, hi, one, n in re.findall(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", text):
        out |= {(kind, k) for k in range(int(lo), int(hi) + 1)} if kind else {(one, int(n))}
    return out


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    found = {}
    for source in ("prompt_attn.hip", "prefix_attn.hip"):
        out = str(tmp_path_factory.mktemp("asm") / "kernels.s")
        flags = [f for f in build.FLAGS if f != "-fPIC"]
        subprocess.run(["hipcc"] + flags + ["-S", "--cuda-device-only", os.path.join(build.CSRC, source), "-o", out],
                       check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
        with open(out) as f:
            text = f.read()
        for name in set(re.findall(r"^(_ZN\S*(?:prompt|prefix)_kernel\S*):", text, re.M)):
            body = text[text.index("\n%s:" % name):]
            body = body[:body.index(".Lfunc_end")]
            found[name] = [l.split(";")[0].rstrip() for l in body.split("\n") if re.match(r"\t[a-z]", l) or re.match(r"\.LBB", l)]
    return found


def _wait_states(line):
    return int(line.split()[1]) + 1 if "s_nop" in line else 1


def test_operands_are_in_place_and_results_are_left_alone(kernels):
    assert len(kernels) == 8
    for name, lines in kernels.items():
        seen = 0
        for k, line in enumerate(lines):
            m = re.match(r"\tv_mfma_f32_32x32x16_bf16 (v\S+), (\S+), (\S+), (\S+)", line)
            if not m:
                continue
            seen += 1
            result, operands = _registers(m.group(1)), _registers(" ".join(m.groups()[1:]))
            states = 0
            for before in reversed(lines[max(0, k - 2):k]):
                if states >= 2:
                    break
                if before.startswith("\tv_") and "mfma" not in before and "cmp" not in before:
                    assert not _registers(before.split(None, 1)[1].split(",")[0]) & operands, (name, before, line)
                states += _wait_states(before)
            states = 0
            for after in lines[k + 1:k + 20]:
                if states >= 18 or after.startswith(".LBB"):
                    break
                if "mfma" in after:
                    ops = [o.strip() for o in after.split(None, 1)[1].split(",")]
                    assert not _registers(" ".join(ops[1:3])) & result, (name, line, after)
                    states += 8
                elif not after.startswith("\ts_") and len(after.split(None, 1)) > 1:
                    assert not _registers(after.split(None, 1)[1]) & result, (name, line, after)
                    states += 1
                else:
                    states += _wait_states(after)
        assert seen >= 40, name                            # five times the scores of a tile


def test_the_loop_moves_nothing_between_register_files(kernels):
    # four iterations to a turn of the loop, each with all its matrix instructions in one block
    for name, lines in kernels.items():
        blocks, now = [], []
        for l in lines:
            if l.startswith(".LBB"):
                blocks.append(now)
                now = []
            else:
                now.append(l)
        per = 32 if "128" in name else 16
        loop = [b for b in blocks if sum("mfma" in l for l in b) == per and sum("v_exp_f32" in l for l in b) == 32]
        assert len(loop) == 4, (name, len(loop))
        for b in loop:
            # a prefix with factors beside its values keeps nine load offsets and a few more there, each read once to a tile
            assert sum("accvgpr" in l for l in b) <= (2 if "prompt_kernel" in name else 12), name
            assert not any("scratch" in l for l in b), name
            # a prefix's tiles have an address each, or factors
            most = (210 if per == 32 else 170) + (0 if "prompt_kernel" in name else 60)
            assert sum(not l.startswith("\ts_nop") for l in b) <= most, (name, len(b))
