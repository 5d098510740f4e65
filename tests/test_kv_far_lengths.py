"""Requests near 2^31 tokens: the largest length that the caches' kernels take leaves room for the keys they look ahead, in 31 bits."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_17698_b200", "csrc")


def _constant(name, *files):
    for f in files:
        m = re.search(rf"constexpr int {name} = (\d+);", open(os.path.join(CSRC, f)).read())
        if m:
            return int(m.group(1))
    raise AssertionError(name)


@pytest.mark.parametrize("kind", ["kv4", "kv8"])
def test_no_key_that_is_looked_at_passes_31_bits(tmp_path, kind):
    src, exe = tmp_path / "most.cpp", tmp_path / "most"
    pages = [(16, (1 << 31) // 16 - 1), (16, ((1 << 31) - 65536) // 16), (16, 100), (1 << 20, 2047), (4096, 524287)]
    src.write_text(f'#include "{kind}.cuh"\n#include <stdio.h>\nint main() {{\n' + "".join(
        f"  {{ sb_{kind}_cache c{{}}; c.page_tokens = {p}; c.table_pages = {n}; c.dim = 16; c.heads = 1; c.requests = 1;\n"
        f"    printf(\"%d \", {kind}_geom(&c, 1, nullptr, nullptr, 1).most); }}\n" for p, n in pages) + "}\n")
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", "/usr/local/cuda/include", "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    step, warps, batch = (_constant(n, "kv_rows.cuh") for n in ("AT_STEP", "AT_WARPS", "AT_BATCH"))
    tile = _constant("PR_KEYS", "kv8_prompt.cu")
    for (p, n), most in zip(pages, got):
        assert most == min(p * n, (1 << 31) - 65536)
        # few rows: at a batch's first step the entries of the batch two on are fetched, by lanes of up to 16 steps of 4 warps
        ahead = most + (warps * (batch * 2 + batch - 1) + warps - 1) * step + step
        # prompts: two tiles on, by 32 lanes of 16 keys; quotients by a step round up
        assert max(ahead, most + 2 * tile + 32 * 16, most + tile - 1) < 1 << 31
