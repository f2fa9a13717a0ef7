"""The beam search on a 4-bit cache: its own checks, and its last attention against the FP64 oracle on what the cache then holds."""
import numpy as np
import pytest
import torch

import _fp4_util as F
from _gpu_util import compare
from oracle import reference as R
from paper_2509_25224_b200 import beam_search
from paper_2509_25224_b200.binding import AmlaError

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups,beams,heads,prompt,steps", [(1, 2, 16, 1, 1), (2, 3, 16, 63, 5), (3, 4, 128, 64, 70), (2, 8, 32, 200, 20)])
def test_search(groups, beams, heads, prompt, steps):
    r = beam_search.search(groups, beams, heads, prompt, steps, kv_scale=0.25)
    assert beam_search.faults(r) == []
    cache = r["cache"].cpu().numpy()
    v = F.values(*F.unpack(cache))
    lens = r["lens"].cpu().numpy()
    held = np.zeros(v.shape[0], bool)
    table = r["table"].cpu().numpy()
    held[table[table >= 0]] = True
    v[~held] = 0.0
    # (what a page holds beyond its sequence is whatever was there)
    v[np.isnan(v)] = 0.0
    q = r["q"].view(torch.int16).cpu().numpy().view(np.uint16)
    o, l = R.decode(q, F.bf16_bits(v), np.maximum(table, 0), lens, r["scale"] * 0.25)
    compare(r["out"].float().cpu().numpy(), r["lse"].cpu().numpy(), o * 0.25, l)


def test_prompts_and_full_pages_are_shared():
    r = beam_search.search(2, 8, 16, 640, 3, kv_scale=0.25)
    assert beam_search.faults(r) == []
    # ten full pages a group, and at most a page a row
    assert r["live"] <= 2 * 10 + 16
    assert (r["table"][:, :10].view(2, 8, 10) == r["table"][:, :10].view(2, 8, 10)[:, :1]).all()


def test_a_cache_that_is_too_small_is_reported():
    r = beam_search.search(1, 4, 16, 60, 8, kv_scale=0.25, num_blocks=3)
    assert r["failed"] > 0 and "found no page" in beam_search.faults(r)[0]
    with pytest.raises((AmlaError, ValueError, RuntimeError)):
        beam_search.search(1, 4, 16, 60, 8, num_blocks=0)


# (a shared full page with two pages left for four rows; a prompt whose last page is not full; two groups over many pages; a group without a prompt)
@pytest.mark.parametrize("groups,beams,prompt,steps,num_blocks", [(1, 4, 64, 8, 3), (1, 4, 60, 8, 3), (2, 4, 128, 70, 9), (2, 3, 63, 5, 1)])
def test_rows_that_find_no_page_leave_the_others_alone(groups, beams, prompt, steps, num_blocks):
    r = beam_search.search(groups, beams, 16, prompt, steps, kv_scale=0.25, num_blocks=num_blocks)
    assert r["failed"] > 0
    # every row, refused ones too, still reads back as the tokens that it was granted
    assert beam_search.faults(r) == ["%d requests found no page" % r["failed"], "a row has the wrong length"]
    lens = r["lens"].cpu().numpy()
    assert lens.max() > 0 and (r["read"].abs().sum(-1) > 0).sum(1).tolist() == lens.tolist()
