"""Kernels of tokens, means, scores and selection that are placed while the kernel in front still writes read nothing of what it brings up to date ahead of the wait:
neither by a pointer, with or without a subscript, nor by a helper that reads one.  Each such reading is shown to be seen."""
import os
import re

import pytest

from paper_2509_25224_b200 import build

WAIT = "behind_the_kernel_in_front();"
POINTERS = ("p.seqlens", "p.block_table", "p.scores", "p.tokens", "p.positions", "p.cos_sin", "p.weight", "p.kv", "p.q", "p.q_pe", "p.means", "p.cache", "select.scores", "select.block_table", "select.seqlens",
            "tokens.", "cache,", "means[", "means +")
HELPERS = ("seen_by", "ldg_here", "place_of_token", "select_row", "load_key", "load8", "key8", "store_key", "cp_async_16", "Angles")


def sources(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, name)).read())
    return [k[k.index("{"):] for k in text.split("__global__")[1:]]


def ahead(body):
    """What of the above stands in front of the wait (of the lines that do so, a dimension or the address of a row is no reading)."""
    front = body[:body.index(WAIT)]
    names = [p for p in POINTERS if re.search(r"(?<![\w.])" + re.escape(p) + (r"\b" if p[-1].isalnum() else ""), front)]
    return names + [h for h in HELPERS if re.search(r"\b" + h + r"\b(<[^;{}]*>)?\s*(\w+)?\(", front)]


KERNELS = [(name, i) for name in ("amla_append.cu", "amla_select.cu") for i in range(2)]


def test_they_are_all_there():
    assert [len(sources(name)) for name in ("amla_append.cu", "amla_select.cu")] == [2, 2]
    assert all(body.count(WAIT) == 1 for name, i in KERNELS for body in [sources(name)[i]])


@pytest.mark.parametrize("name,i", KERNELS)
def test_nothing_is_read_ahead_of_the_wait(name, i):
    assert ahead(sources(name)[i]) == []


# what each kernel reads behind the wait, moved in front of it
MOVED = [("amla_append.cu", 0, "const Place at = place_of_token(p.tokens, token, lane);"), ("amla_append.cu", 0, "key = load_key<kWide>(p, token, lane);"),
         ("amla_append.cu", 0, "const int position = p.positions ? p.positions[token] : at.position;"), ("amla_append.cu", 1, "const Place at = place_of_token(tokens, token, lane);"),
         ("amla_append.cu", 1, "key8<kFormat>(cache, pages[k], r * kRowGroups + group, col8, x);"), ("amla_select.cu", 0, "const int mine = tid < p.B ? ldg_here(p.seqlens + tid) : INT_MIN;"),
         ("amla_select.cu", 0, "const int seen = seen_by(p.seqlens, b, p.Sq, t0 + tokens - 1, p.width);"), ("amla_select.cu", 1, "const int seen = seen_by(p.seqlens, row / p.Sq, p.Sq, row % p.Sq, p.width);"),
         ("amla_select.cu", 1, "const float* scores = p.scores + static_cast<size_t>(row) * p.width;"), ("amla_select.cu", 1, "select_row<kSelectThreads, kHeld>(p, row, seen, held_keys, scratch);")]


@pytest.mark.parametrize("name,i,line", MOVED)
def test_what_is_moved_ahead_of_the_wait_is_seen(name, i, line):
    body = sources(name)[i]
    at = body.index(WAIT)
    assert line in body[at:]
    assert ahead(body[:at] + line + body[at:]) != []
