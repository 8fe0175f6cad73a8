"""The exchange at a group's end in the 128-row form of tree attention, as a model: every order in which its barriers let two partner warps
and the issuing warp run is walked through, and no warp may write what its partner has still to read."""
import itertools
import re
from pathlib import Path

import pytest

SOURCE = Path(__file__).resolve().parent.parent / "paper_2509_22951_b200" / "csrc" / "tq_tree.cu"


def sets_in_the_kernel():
    m = re.search(r"constexpr uint32_t kMlSets = (\d+);", SOURCE.read_text())
    return int(m.group(1)) if m else 1


def program(tiles):
    """What a softmax warp does for groups of so many tiles each."""
    steps, last = [], -1
    for g, n in enumerate(tiles):
        for t in range(last + 1, last + 1 + n):
            steps += [("scores", t), ("p", t)]  # waits for the tile's scores; announces its p
        last += n
        steps += [("write", g), ("arrive", g), ("product", last), ("both", g), ("read", g)]
    return steps, last + 1


def meets(tiles, sets):
    """Whether some order has a warp write a set that its partner has not read."""
    steps, total = program(tiles)
    wrote = [sum(1 for s in steps[:i] if s[0] == "write") for i in range(len(steps) + 1)]
    read = [sum(1 for s in steps[:i] if s[0] == "read") for i in range(len(steps) + 1)]
    arrived = [sum(1 for s in steps[:i] if s[0] == "arrive") for i in range(len(steps) + 1)]
    given = [sum(1 for s in steps[:i] if s[0] == "p") for i in range(len(steps) + 1)]
    todo, known = [(0, 0, 0, 0)], {(0, 0, 0, 0)}  # place of the two warps, tiles with scores, tiles with products
    while todo:
        at = todo.pop()
        a, b, asked, done = at
        after = []
        if asked < total and asked - done < 2:
            after.append((a, b, asked + 1, done))
        if done < asked and min(given[a], given[b]) > done:
            after.append((a, b, asked, done + 1))
        for me, other in ((0, 1), (1, 0)):
            i, j = at[me], at[other]
            if i == len(steps):
                continue
            what, n = steps[i]
            if what == "scores" and asked <= n or what == "product" and done <= n or what == "both" and min(arrived[i], arrived[j]) <= n:
                continue
            if what == "write" and read[j] <= n - sets:  # the set was last written for group n - sets
                return True
            if what in ("both", "scores"):  # the barriers tell phases apart by a parity: nobody is a whole turn behind
                assert abs(arrived[i] - arrived[j]) <= 1
            after.append((i + 1, j, asked, done) if me == 0 else (j, i + 1, asked, done))
        for s in after:
            if s not in known:
                known.add(s)
                todo.append(s)
    return False


@pytest.mark.parametrize("groups", [2, 3, 4, 5])
def test_no_warp_writes_what_its_partner_has_to_read(groups):
    sets = sets_in_the_kernel()
    for tiles in itertools.product((1, 2, 3, 4), repeat=groups):
        assert not meets(tiles, sets), (tiles, sets)


def test_the_model_sees_the_fault():
    assert meets((1, 1), 1) and meets((3, 2), 1) and not meets((3, 3), 1)
