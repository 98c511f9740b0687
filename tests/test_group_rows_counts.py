"""CPU: the 16-bit counts of lq_group_rows, two groups in a word, as group_rows.hip adds them up.  A workgroup counts the rows of a round per
wavefront and group, turns the counts into those of the earlier wavefronts, and adds every placed row to its own; nothing tells it
when a count passes 65,535, so the rows of a round must stay below that.  The rounds are read from the source."""
import os
import re

import numpy as np
import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2306_08367_amd", "csrc", "group_rows.hip")
WAVES, MOST = 16, 1 << 19        # MOST: keys of a workgroup at most


def _rounds():
    """Most rows that a workgroup counts at a time: in one launch, sorting, not sorting."""
    text, known = open(SOURCE).read(), {}
    for line in re.findall(r"^constexpr int(?:64_t)? (.+?);", text, re.M):
        for name, value in re.findall(r"(\w+) = ([\w* /]+)", line):
            known[name] = int(eval(value.replace("/", "//"), {}, dict(known)))
    assert known["THREADS"] == 64 * WAVES
    return known["ONE_GROUP_KEYS"], known["SORTED"], known.get("UNSORTED", MOST)


def _places(keys, G, rows):
    """Places of the rows of one workgroup with `rows` rows in a round: packed words that wrap around and carry like the hardware's."""
    words, of = (G + 2) // 2, np.where((keys >= 0) & (keys < G), keys, G)
    total = np.bincount(of, minlength=G + 1)
    base, places = np.cumsum(total) - total, np.empty(len(keys), dtype=np.int64)
    for at in range(0, len(keys), rows):
        g = of[at:at + rows]
        per = -(-len(g) // WAVES)
        counts = np.zeros((WAVES, words), dtype=np.uint32)
        for w in range(WAVES):
            np.add.at(counts[w], g[w * per:(w + 1) * per] >> 1, (1 << 16 * (g[w * per:(w + 1) * per] & 1)).astype(np.uint32))
        counts = np.cumsum(counts, axis=0, dtype=np.uint32) - counts
        for w in range(WAVES):
            for step in range(w * per, min((w + 1) * per, len(g)), 64):
                i = np.arange(step, min(step + 64, (w + 1) * per, len(g)))
                word, half = g[i] >> 1, 16 * (g[i] & 1)
                earlier = (counts[w, word] >> half) & 0xffff
                np.add.at(counts[w], word, (1 << half).astype(np.uint32))
                shared = ((counts[w, word] >> half) & 0xffff).astype(np.int64) - earlier > 1
                before = np.array([np.count_nonzero(shared[:j] & (g[i[:j]] == g[i[j]])) if shared[j] else 0 for j in range(len(i))])
                places[at + i] = base[g[i]] + earlier + before
        every = np.arange(G + 1)
        base = base + ((counts[WAVES - 1, every >> 1] >> (16 * (every & 1))) & 0xffff)
    return places


def _keys(how, n, G):
    if how == "one":
        return np.full(n, 6)
    if how == "odd":
        return np.full(n, 7)
    if how == "none":
        return np.full(n, -1)
    rng = np.random.default_rng(n)
    return np.where(rng.random(n) < 0.97, 4 + (rng.random(n) < 0.01), rng.integers(-1, G, n))


@pytest.mark.parametrize("how", ["one", "odd", "none", "mixed"])
@pytest.mark.parametrize("form", [0, 1, 2], ids=["one-launch", "sorting", "not-sorting"])
def test_every_row_gets_its_place(form, how):
    rows, G = _rounds()[form], 8
    n = rows if form == 0 else min(2 * rows + 100, MOST)
    keys = _keys(how, n, G)
    want = np.empty(n, dtype=np.int64)
    want[np.argsort(np.where(keys < 0, G, keys), kind="stable")] = np.arange(n)
    np.testing.assert_array_equal(_places(keys, G, rows), want)


def test_more_rows_than_a_count_holds_are_told():
    """The same check with a round of 70,000 rows fails: it sees what it is there for."""
    keys = _keys("one", 70_000, 8)
    assert (_places(keys, 8, 70_000) != np.arange(70_000)).any()
