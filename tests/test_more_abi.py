"""The argument structs of the 4-bit cache, rotary positions and adapters as a C compiler lays them out, against the binding's; and what the binding
refuses or passes on, on the CPU."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2602_17698_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("c_name,struct", [("sb_kv4_cache", binding.Kv4CacheStruct), ("sb_rotary_table", binding.RotaryTableStruct),
                                           ("sb_rotary_part", binding.RotaryPartStruct), ("sb_lora_adapters", binding.LoraAdaptersStruct)])
def test_structs_of_the_binding_match_the_header(tmp_path, c_name, struct):
    names = [f for f, _ in struct._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "scalebits.h"\nint main(void) {\n  printf("%zu", sizeof(' + c_name + '));\n' +
                   "".join(f'  printf(" %zu", offsetof({c_name}, {f.rstrip("_")}));\n' for f in names) + "  return 0;\n}\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got[0] == ctypes.sizeof(struct)
    assert got[1:] == [getattr(struct, f).offset for f in names]


@pytest.fixture
def on_cpu(monkeypatch):
    """Structs around tensors of the host (nothing is called)."""
    monkeypatch.setattr(binding, "_dev", lambda t: None if t is None else t.data_ptr())


def _parts(dim=80, pages=8, heads=2, page=16):
    row, scales = (dim + 31) // 32 * 16, (dim + 63) // 64 * 4
    k, s = torch.zeros(pages, heads, page, row, dtype=torch.uint8), torch.zeros(pages, heads, page, scales, dtype=torch.uint8)
    return [k, k.clone(), s, s.clone(), torch.zeros(3, 10, dtype=torch.int32), dim]


def test_the_4_bit_cache(on_cpu):
    parts = _parts()
    head = torch.ones(2)
    c = binding.Kv4Cache(*parts, head, None).struct
    assert (c.pages, c.requests, c.heads, c.page_tokens, c.dim, c.table_stride, c.table_pages) == (8, 3, 2, 16, 80, 10, 10)
    assert c.k_head == head.data_ptr() and c.v_head is None
    table = parts[4]
    for view, stride, pages in [(table[:, :4], 10, 4), (table[::2, :4], 20, 4), (table[:1, :4].expand(5, 4), 0, 4)]:
        s = binding.Kv4Cache(*parts[:4], view, 80).struct
        assert (s.table_stride, s.table_pages, s.requests) == (stride, pages, view.shape[0])
    assert binding.Kv4Cache(*parts[:2], *(t.view(torch.float8_e4m3fn) for t in parts[2:4]), *parts[4:]).struct.dim == 80
    for dim, row, scales in [(16, 16, 4), (64, 32, 4), (80, 48, 8), (96, 48, 8), (128, 64, 8), (144, 80, 12), (256, 128, 16)]:
        e = binding.Kv4Cache.empty(4, 2, 16, dim, table)
        assert e.k.shape == (4, 2, 16, row) and e.v_scale.shape == (4, 2, 16, scales)


def test_what_the_4_bit_cache_refuses(on_cpu):
    def but(i, what):
        parts = _parts()
        parts[i] = what(parts[i])
        return parts
    for error, parts in [(TypeError, but(0, lambda t: t.view(torch.int8))), (TypeError, but(2, lambda t: t.float())), (TypeError, but(4, lambda t: t.long())),
                         (ValueError, but(1, lambda t: t[:, :, :8])), (ValueError, but(2, lambda t: t[..., :4].contiguous())), (ValueError, but(5, lambda d: 128)),
                         (ValueError, but(0, lambda t: t.transpose(1, 2).contiguous().transpose(1, 2))), (ValueError, but(4, lambda t: t[:, ::2])),
                         (ValueError, but(4, lambda t: t[:, :0])), (ValueError, _parts() + [torch.ones(3)]), (ValueError, _parts() + [None, torch.ones(2).double()])]:
        with pytest.raises(error):
            binding.Kv4Cache(*parts)


def test_rotary_tables_and_adapters(on_cpu):
    t = binding.RotaryTable(torch.ones(20), True, 1.5)
    assert (t.rotated, t.struct().rotated, t.struct().interleaved, t.struct().inverse, t.struct(True).inverse, t.struct(True).factor) == (40, 40, 1, 0, 1, 1.5)
    assert binding._ROTARY_PART.size == ctypes.sizeof(binding.RotaryPartStruct)
    got = binding.RotaryPartStruct.from_buffer_copy(binding._ROTARY_PART.pack(1, 2, 3, 4, 5, 6, 7, 8))
    assert [getattr(got, f) for f, _ in got._fields_] == [1, 2, 3, 4, 5, 6, 7, 8]
    for bad in (torch.ones(20).double(), torch.ones(2, 10), torch.ones(40)[::2], torch.ones(0)):
        with pytest.raises(ValueError):
            binding.RotaryTable(bad)
    a, b = torch.zeros(3, 16, 64, dtype=torch.bfloat16), torch.zeros(3, 40, 16, dtype=torch.bfloat16)
    s = binding.LoraAdapters(a, b, torch.ones(3)).struct
    assert (s.adapters, s.rank, s.in_, s.out) == (3, 16, 64, 40)
    for error, args in [(TypeError, (a.float(), b)), (TypeError, (a, b.transpose(1, 2))), (ValueError, (a[:2], b)), (ValueError, (a, b, torch.ones(2)))]:
        with pytest.raises(error):
            binding.LoraAdapters(*args)


def test_frequencies():
    """Each scaling against its formula, pair by pair."""
    f = binding.rotary_frequencies(64, 500.0)
    assert f.dtype == torch.float32 and f.shape == (32,) and f[0] == 1
    for i in range(32):
        plain = 500.0 ** (-2 * i / 64)
        turns = plain * 1000 / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 2) / (8 - 2)))
        want = {None: plain, "linear": plain / 8, "base": (500.0 * 8 ** (64 / 62)) ** (-2 * i / 64), "parts": plain * (keep + (1 - keep) / 8)}
        for scaling, w in want.items():
            got = binding.rotary_frequencies(64, 500.0, scaling, 8.0, trained=1000, low=2.0, high=8.0)[i]
            assert abs(float(got) - w) <= 2.0 ** -23 * w, (scaling, i)
    base = binding.rotary_frequencies(64, 500.0, "base", 8.0)
    assert abs(float(base[-1]) * 8 / float(f[-1]) - 1) < 1e-6 and base[0] == 1
    for bad in [dict(rotated=63), dict(rotated=0), dict(rotated=64, scaling="other"), dict(rotated=64, stretch=0), dict(rotated=64, scaling="parts", low=4, high=4)]:
        with pytest.raises(ValueError):
            binding.rotary_frequencies(**bad)
