"""Decoding over long contexts with a part of their pages: the example's own checks, for every cache."""
import pytest
import torch

from paper_2509_25224_b200 import long_context

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "fp4"])
@pytest.mark.parametrize("sequences,heads,prompt,steps,keep", [(1, 16, 700, 3, 7), (3, 128, 4096, 70, 12), (5, 33, 2500, 66, 20)])
def test_runs(cache, sequences, heads, prompt, steps, keep):
    r = long_context.serve(sequences, heads, prompt, steps, keep, cache)
    assert long_context.faults(r) == []
    assert r["chosen"].shape == (sequences, keep) and int(r["lens"][0]) == prompt + steps


def test_what_no_page_is_left_out_of_is_the_plain_attention():
    r = long_context.serve(2, 16, 640, 5, 11, "bf16")
    assert long_context.faults(r) == [] and torch.equal(r["out"], r["whole"][0]) and torch.equal(r["lse"], r["whole"][1])
