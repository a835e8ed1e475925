"""Matrix products that add to each other's results are of one length along the contraction, in the listings of all kernels.

On this target a product that takes the result of one of another length as its sum a few instructions later gets a part of it, and the compiler puts no wait
between the two; of one length they may follow each other directly."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2107_01460_amd import build

WINDOW = 16   # instructions


def mixed_chains(listing):
    """[(kernel, the later product)] whose sum is a result, at most WINDOW instructions old, of a product of another shape"""
    found = []
    for m in re.finditer(r"^(_Z\S+):\s", listing, re.M):
        end = listing.find(".Lfunc_end", m.end())
        if end < 0:
            continue
        recent = {}   # registers: (instructions ago, shape)
        for line in listing[m.end():end].split("\n"):
            line = re.sub(r"\s*;.*", "", line.strip())
            if not line or line.startswith(".") or line.endswith(":"):
                continue
            recent = {r: (n + 1, s) for r, (n, s) in recent.items() if n < WINDOW}
            p = re.match(r"v_mfma_\w+?_(\d+x\d+x\d+)\w*\s+(.*)", line)
            if p is None:
                continue
            registers = [x.strip() for x in p.group(2).split(",")]
            if registers[3] in recent and recent[registers[3]][1] != p.group(1):
                found.append((m.group(1), line))
            recent[registers[0]] = (0, p.group(1))
    return found


def test_a_mixed_chain_is_seen():
    text = "_Z1kv: ; @_Z1kv\n%s\ts_endpgm\n.Lfunc_end0:\n"
    first, nop = "\tv_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0\n", "\ts_nop 0\n"
    assert len(mixed_chains(text % (first + nop + "\tv_mfma_f32_16x16x16_bf16 v[12:15], v[4:5], v[8:9], v[0:3]\n"))) == 1
    assert mixed_chains(text % (first + nop + "\tv_mfma_f32_16x16x32_bf16 v[12:15], v[4:7], v[8:11], v[0:3]\n")) == []
    assert mixed_chains(text % (first + nop * (WINDOW + 1) + "\tv_mfma_f32_16x16x16_bf16 v[12:15], v[4:5], v[8:9], v[0:3]\n")) == []


@pytest.mark.parametrize("src", build.SOURCES)
def test_kernels(listings, src):
    assert mixed_chains(listings[src]) == []


def test_linear_attention_in_bf16(tmp_path):
    if shutil.which("hipcc") is None:
        pytest.skip("needs hipcc")
    out = str(tmp_path / "linear_attention_bf16.s")
    subprocess.check_call(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "linear_attention_bf16.hip"), "-o", out])
    with open(out) as f:
        listing = f.read()
    assert mixed_chains(listing) == []
    assert set(re.findall(r"v_mfma_\w+?_(\d+x\d+x\d+)", listing)) == {"16x16x32"}
