"""Kernels that are launched before the one ahead of them has ended may not read by .nc what that one writes (sources only, on the CPU)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_17698_b200", "csrc")


def _code(path):
    return re.sub(r"//[^\n]*", "", open(path).read())


def _kernels(code):
    """Every kernel's body."""
    for m in re.finditer(r"__global__[^{;]*\{", code):
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(code[i], 0)
            i += 1
        yield code[m.end():i]


def test_no_read_only_loads_where_a_kernel_starts_early():
    early = [p for p in sorted(glob.glob(os.path.join(CSRC, "*.cu"))) if re.search(r"\b(sb|at)_after_previous\(\)", _code(p))]
    assert {"kv4_attention.cu", "kv4_cache.cu", "kv8_prompt.cu", "lora.cu", "rotary.cu"} <= {os.path.basename(p) for p in early}
    shared = [os.path.join(CSRC, h) for h in ("kv_rows.cuh", "kv8_attention.cuh", "kv8.cuh", "kv4.cuh", "fp4.cuh")]
    for path in early + shared:
        found = re.findall(r"__ldg|\.nc\b|ld_stream\d+", _code(path))
        assert not found, (os.path.basename(path), found)


def test_every_early_kernel_waits():
    for name in ("kv4_attention.cu", "kv4_cache.cu", "rotary.cu"):
        bodies = list(_kernels(_code(os.path.join(CSRC, name))))
        assert bodies
        for body in bodies:
            let, wait = body.find("sb_let_next()"), body.find("sb_after_previous()")
            assert 0 <= wait and body[:wait].count("return") == 0 and 0 <= let


def test_who_lets_a_kernel_in_that_reads_before_its_wait_has_waited_itself():
    down, up = (next(b for b in _kernels(_code(os.path.join(CSRC, "lora.cu"))) if mark in b) for mark in ("a.h + tile.row0 * RP + i", "a.h + (k * a.total"))
    assert 0 <= down.find("sb_after_previous()") < down.find("sb_let_next()")
    assert 0 <= up.find("if (wide < 16) sb_after_previous();") < up.find("lo_tile<")
