"""Where the scoring kernel keeps things in shared memory, worked out from the constants in its source: what is read and written at one time with no barrier in between has
bytes of its own.  (A read that only timing keeps ahead of a write is not shown on a GPU: the late reader would take what was written for a sequence's number.)"""
import os
import re

import pytest

from paper_2509_25224_b200 import build

SOURCE = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, "amla_select.cu")).read())
KERNEL = SOURCE[SOURCE.index("page_scores_kernel(const ScoreParams p"):SOURCE.index("pages_select_kernel(const SelectParams p)")]


def constants(text):
    """The whole numbers that `constexpr` lines and the list of barriers give."""
    known = {"kDqk": 576, "kDv": 512, "kPage": 64}
    for line in re.findall(r"\bconstexpr (?:int|uint32_t) ([^;]*);", text):
        for name, value in re.findall(r"(k\w+) = ([^,]*(?:\([^)]*\)[^,]*)*)", line):
            if re.fullmatch(r"[\w\s+*/()-]*", value) and "sizeof" not in value:
                try:
                    known[name] = eval(value.replace("/", "//"), {}, known)
                except NameError:
                    pass                                          # (of a template, say)
    at = 0
    for item in re.search(r"enum \{ (X_FULL[^}]*) \}", text)[1].split(","):
        name, _, value = item.partition("=")
        at = eval(value, {}, known) if value else at
        known[name.strip()] = at
        at += 1
    return known


def regions(text):
    """name -> (first byte, byte behind the last) of what the summing warps, the barriers and the peers write, and of the word that says which sequence a block has."""
    k = constants(text)
    kernel = text[text.index("page_scores_kernel(const ScoreParams p"):text.index("pages_select_kernel(const SelectParams p)")]
    found = re.search(r"found = reinterpret_cast<int\*>\(smem \+ ([\w\s+-]*)\)", kernel)[1]
    late = re.search(r"late = reinterpret_cast<int\*>\(smem \+ ([\w\s+-]*)\)", kernel)
    slot = re.search(r"tmem_slot = bars \+ ([\w\s+-]*);", kernel)[1]
    rows, at = k["kTileRows"], k["kOffBars"]
    return {"sequence": (eval(found, {}, k), eval(found, {}, k) + 4), "lengths": (0, 4 * k["kThreads"]), "ring and shares": (0, k["kWorkBytes"]), "known": (k["kOffKnown"], k["kOffKnown"] + 8 * rows),
            "lse": (k["kOffLse"], k["kOffLse"] + 4 * rows), "halves": (k["kOffHalves"], k["kOffHalves"] + 4 * (k["kTilePages"] // 2)), "barriers": (at, at + 8 * k["X_NUM"]),
            "tensor memory": (at + eval(slot, {}, k), at + eval(slot, {}, k) + 4)} | ({"late": (eval(late[1], {}, k), eval(late[1], {}, k) + 4)} if late else {})


def overlapping(found, name):
    a, b = found[name]
    return [other for other, (x, y) in found.items() if other != name and a < y and x < b]


def test_the_constants_are_read():
    k = constants(SOURCE)
    assert (k["kThreads"], k["kTileRows"], k["kTilePages"], k["kWorkBytes"], k["kMostStages"], k["X_EMPTY"], k["X_NUM"]) == (416, 128, 256, 227328, 9, 9, 24)
    assert k["kOffKnown"] < k["kOffLse"] < k["kOffHalves"] < k["kOffBars"] < k["kScoreSmem"] <= 232448


def test_the_word_that_says_which_sequence_a_block_has_is_nobody_elses():
    """Warps read it behind a barrier, and no further one stands between that and what the quickest of them write next."""
    found = regions(SOURCE)
    assert overlapping(found, "sequence") == []
    a, b = found["sequence"]
    assert a % 4 == 0 and b <= constants(SOURCE)["kScoreSmem"]
    # (written once, by the thread that has the sequence)
    assert len(re.findall(r"\*found = ", KERNEL)) == 1


@pytest.mark.parametrize("place", ["kOffLse", "kOffKnown", "kOffBars", "kOffBars + 256 - 8", "kOffHalves + 8", "kOffStats"])
def test_a_word_that_is_somebody_elses_would_be_seen(place):
    moved = re.sub(r"(found = reinterpret_cast<int\*>\(smem \+ )[\w\s+-]*\)", r"\g<1>%s)" % place, SOURCE)
    assert overlapping(regions(moved), "sequence") != []


def test_all_that_lives_beside_the_ring_is_apart():
    found = regions(SOURCE)
    for name in ("known", "lse", "halves", "barriers", "tensor memory", "late"):
        assert overlapping(found, name) == [], name
