"""What the beam search refuses, and that its checks find what they look for (no GPU)."""
import pytest
import torch

from paper_2509_25224_b200 import beam_search


@pytest.mark.parametrize("bad", [dict(beams=1), dict(groups=0), dict(prompt=0), dict(steps=0)])
def test_refusals(bad):
    with pytest.raises(ValueError):
        beam_search.search(**bad)


def result():
    """Two rows of 65 tokens that share a page."""
    history = torch.randn((2, 65, 576), generator=torch.Generator().manual_seed(1)).bfloat16()
    history[1, :64] = history[0, :64]
    out, lse = torch.randn(2, 1, 16, 512), torch.randn(2, 1, 16)
    i = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return dict(out=out, lse=lse, before=(out.clone(), lse.clone()), table=i([[0, 1, -1], [0, 2, -1]]), lens=i([65, 65]), refs=i([2, 1, 1, 0]), history=history, read=history.clone(),
                live=3, failed=0)


def test_a_sound_search_has_no_faults():
    assert beam_search.faults(result()) == []


@pytest.mark.parametrize("key,at,value", [("out", (0, 0, 0, 0), 9.0), ("lse", (1, 0, 3), 9.0), ("lens", (1,), 64), ("refs", (0,), 1), ("refs", (3,), 1), ("table", (1, 1), 3), ("read", (1, 64, 7), 99.0)])
def test_faults_are_found(key, at, value):
    r = result()
    r[key][at] = value
    assert len(beam_search.faults(r)) == 1


def test_requests_without_a_page_are_counted():
    assert beam_search.faults(dict(result(), failed=2)) == ["2 requests found no page"]
