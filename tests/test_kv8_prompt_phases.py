"""The order of waits and arrivals in the prompt kernel of the 8-bit cache's attention (csrc/kv8_prompt.cu), played through in
every interleaving on the CPU.

A wait on an mbarrier sees one bit of its phase number, so a role that falls two phases behind waits for a phase that may never
come, and one that runs ahead passes too early. The roles are restated here as straight lists of steps, with the kernel's
names; a group of warps that arrive together is one role, products end as soon as they are issued, and the raw copies (a chain
of their own) are left out. `pieces`: (key tiles, whether the second row tile has rows) of a share's pieces."""
import pytest

RING, SLOTS = 3, 4


def _programs(pieces, idle_rows_wait_for_scales, scores_first):
    """Steps of every role, and how many arrivals end a phase of a barrier. A step is (what, name, number): a wait for that
    phase, an arrival, a write of a scale slot or a read of what it should hold."""
    def wait(name, phase): return ("wait", name, phase)
    def arrive(name): return ("arrive", name, 0)
    tiles = sum(n for n, _ in pieces)
    convert = []
    for n in range(2 * tiles):
        convert.append(wait(f"empty{n % RING}", n // RING - 1))
        if n % 2 == 0:
            j = n // 2
            convert += [("write", f"slot{j % SLOTS}", j), arrive(f"scfull{j % SLOTS}")]
        convert.append(arrive(f"full{n % RING}"))
    programs = {"convert": convert}
    for q in (0, 1):
        # products of row tile q
        p, t, mine, piece = [], 0, 0, 0
        def there(n): p.append(wait(f"full{n % RING}", n // RING))
        def done(n): p.append(arrive(f"empty{n % RING}"))
        for count, both in pieces:
            if q == 1 and not both:
                for n in range(t, t + 2 * count):
                    there(n)
                    done(n)
            else:
                p.append(wait(f"qready{q}", piece))
                piece += 1
                there(t)
                p += [arrive(f"sfull{q}0"), arrive(f"sfull{q}1")]
                done(t)
                for h in range(2 * count):
                    tile = t + (h & ~1)
                    if h % 2 == 0:
                        there(tile + 1)
                    p += [wait(f"pfull{q}{h & 1}", (mine + h) >> 1), arrive(f"odone{q}")]
                    if h & 1:
                        done(tile + 1)
                    if h + 2 < 2 * count:
                        if h % 2 == 0:
                            there(tile + 2)
                        p += [wait(f"odone{q}", mine + h), arrive(f"sfull{q}{h & 1}")]
                        if h & 1:
                            done(tile + 2)
                p.append(arrive(f"fin{q}"))
                mine += 2 * count
            t += 2 * count
        programs[f"products{q}"] = p
        # softmax of row tile q
        s, tiles_all, tiles_mine, piece, skipped = [], 0, 0, 0, False
        for count, both in pieces:
            if q == 1 and not both:
                skipped = True
                if idle_rows_wait_for_scales:
                    s += [wait(f"scfull{(tiles_all + j) % SLOTS}", (tiles_all + j) // SLOTS) for j in range(count)]
            else:
                s.append(arrive(f"qready{q}"))
                for j in range(count):
                    slot, phase = (tiles_all + j) % SLOTS, (tiles_all + j) // SLOTS
                    scales = [wait(f"scfull{slot}", phase)]
                    scores = [wait(f"sfull{q}0", tiles_mine + j)]
                    s += scores + scales if j == 0 and skipped and scores_first else scales + scores
                    s += [("read", f"slot{slot}", tiles_all + j), arrive(f"pfull{q}0"), wait(f"sfull{q}1", tiles_mine + j),
                          ("read", f"slot{slot}", tiles_all + j), arrive(f"pfull{q}1")]
                s.append(wait(f"fin{q}", piece))
                piece += 1
                tiles_mine += count
                skipped = False
            tiles_all += count
        programs[f"softmax{q}"] = s
    return programs, {f"empty{i}": 2 for i in range(RING)}


def _explore(programs, counts):
    """(a state in which nobody can go on and somebody has not ended, or None; whether a wait passed before its phase had ended or
    a read found another tile's scales)."""
    names = list(programs)
    # how often a barrier was arrived on, and what a slot holds, follow from how far each role is
    arrived = {r: [{}] for r in names}
    for r in names:
        for what, name, _ in programs[r]:
            d = arrived[r][-1]
            if what == "arrive":
                d = dict(d)
                d[name] = d.get(name, 0) + 1
            arrived[r].append(d)
    wrong = False
    seen, todo = set(), [tuple(0 for _ in names)]
    while todo:
        at = todo.pop()
        if at in seen:
            continue
        seen.add(at)
        moves = 0
        for i, r in enumerate(names):
            if at[i] == len(programs[r]):
                continue
            what, name, number = programs[r][at[i]]
            if what == "wait":
                phase = sum(arrived[q][at[k]].get(name, 0) for k, q in enumerate(names)) // counts.get(name, 1)
                if (phase ^ number) & 1 == 0:               # the phase of that parity is the one that has not ended
                    continue
                wrong |= phase <= number
            elif what == "read":
                puts = [n for w, s, n in programs["convert"][:at[names.index("convert")]] if w == "write" and s == name]
                wrong |= not puts or puts[-1] != number
            moves += 1
            todo.append(at[:i] + (at[i] + 1,) + at[i + 1:])
        if moves == 0 and any(at[i] < len(programs[r]) for i, r in enumerate(names)):
            return {r: at[i] for i, r in enumerate(names)}, wrong
    return None, wrong


@pytest.mark.parametrize("pieces", [[(9, False)], [(5, False), (2, True)], [(1, True), (9, False), (2, True)], [(2, True), (1, False), (1, True), (6, False)],
                                    [(5, True)], [(4, False), (5, False), (1, True)]])
def test_every_interleaving_ends_with_the_right_scales(pieces):
    stuck, wrong = _explore(*_programs(pieces, idle_rows_wait_for_scales=False, scores_first=True))
    assert stuck is None and not wrong


def test_what_the_model_finds():
    """Row tiles without rows that wait for the scales like the others, but that nobody waits for, can be left behind; and where
    they do not wait, a wait for the scales of the next piece before its scores passes too early."""
    stuck, _ = _explore(*_programs([(9, False)], idle_rows_wait_for_scales=True, scores_first=False))
    assert stuck is not None and stuck["softmax1"] < 9
    _, wrong = _explore(*_programs([(9, False), (2, True)], idle_rows_wait_for_scales=False, scores_first=False))
    assert wrong
