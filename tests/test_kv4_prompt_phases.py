"""The order of waits and arrivals in the prompt kernel where it reads the 4-bit cache (csrc/kv8_prompt.cu), in every interleaving on the CPU:
no scales beside the tiles, and for heads of more than 128 shorter rings and one row tile."""
import pytest

import test_kv8_prompt_phases as phases


def _programs(monkeypatch, pieces, ring, raw_ring, rescale):
    monkeypatch.setattr(phases, "RING", ring)
    programs, counts = phases._programs(pieces, idle_rows_wait_for_scales=False, scores_first=False)
    for role, steps in programs.items():
        programs[role] = [s for s in steps if s[0] not in ("read", "write") and not s[1].startswith("scfull")]
    # raw tiles: copied, then converted
    copy, convert, n = [], [], 0
    for step in programs["convert"]:
        convert.append(step)
        if step[0] == "wait":
            copy += [("wait", f"raw_empty{n % raw_ring}", n // raw_ring - 1), ("arrive", f"raw_full{n % raw_ring}", 0)]
            convert.append(("wait", f"raw_full{n % raw_ring}", n // raw_ring))
        else:
            convert.append(("arrive", f"raw_empty{n % raw_ring}", 0))
            n += 1
    programs["copy"], programs["convert"] = copy, convert
    if rescale:
        # a row's reference may move in any half but a piece's first: the products of the half before have to be done then
        for q in (0, 1):
            steps, half, first = [], 0, True
            for s in programs[f"softmax{q}"]:
                if s[1].startswith("qready"):
                    first = True
                if s[1].startswith("pfull"):
                    if not first:
                        steps.append(("wait", f"odone{q}", half - 1))
                    half, first = half + 1, False
                steps.append(s)
            programs[f"softmax{q}"] = steps
    return programs, counts


@pytest.mark.parametrize("rescale", [False, True])
@pytest.mark.parametrize("ring,raw_ring,pieces", [
    (3, 4, [(4, False)]), (3, 4, [(2, False), (1, True)]), (3, 4, [(1, True), (3, False), (1, True)]), (3, 4, [(3, True)]),
    (2, 1, [(6, False)]), (2, 1, [(1, False), (3, False), (1, False)])])
def test_every_interleaving_ends(monkeypatch, ring, raw_ring, pieces, rescale):
    stuck, wrong = phases._explore(*_programs(monkeypatch, pieces, ring, raw_ring, rescale))
    assert stuck is None and not wrong
