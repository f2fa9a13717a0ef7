"""Scores of pages, their selection and sparse decode: more sequences than a block has threads, tables far wider than their sequences."""
import numpy as np
import pytest
import torch

import _fp4_util as F
import _sparse_util as S
from _gpu_util import compare
from oracle import reference as R
from paper_2509_25224_b200 import binding, sparse
from test_gpu_sparse import SCALE, check_scores, dev, dev_bf16, workload

pytestmark = pytest.mark.gpu

WIDE = 2100                              # more pages than eight blocks have tiles for: clusters of eight, which do not all have room


@pytest.mark.parametrize("B", [100, 415, 416, 417, 1000])
def test_scores_of_many_sequences_in_a_wide_table(B):
    """The longest sequences come first where there are at most as many as a block has threads; most blocks have no page at all."""
    rng = np.random.default_rng(B)
    lens = [int(n) for n in rng.choice([0, 1, 63, 64, 65, 128, 129, 700, 5000], B)]
    lens[B // 2] = 64 * WIDE - 5
    check_scores(lens, 1, 5, width=WIDE)


@pytest.mark.parametrize("B,Sq,H", [(40, 1, 16), (24, 3, 40), (20, 8, 128)])
def test_sparse_decode_of_short_sequences_in_a_wide_table(B, Sq, H):
    rng, keep = np.random.default_rng(B), 5
    lens = [int(n) for n in rng.choice([0, 1, 64, 65, 64 * 5, 64 * 5 + 1, 700], B - 1)] + [3000]
    q, cache, values, kv_scale, means, table, lens = workload("bf16", lens, Sq, H, width=WIDE)
    q_d, table_d, lens_d = dev_bf16(q), dev(table), dev(lens)
    ws = torch.full((sparse.sparse_workspace_size(B, Sq, H, WIDE, keep),), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = sparse.mla_decode_sparse(q_d, cache, kv_scale, means, table_d, lens_d, SCALE, keep, 1, 2, workspace=ws)
    sparse.check_status(ws)
    scores = sparse.page_scores(q_d, means, table_d, lens_d, SCALE)
    sub, sub_lens, chosen = sparse.pages_select(scores, table_d, lens_d, keep, 1, 2)
    o, l = binding.mla_decode(q_d.view(B * Sq, 1, H, 576), cache, sub, sub_lens, SCALE)
    assert torch.equal(o.view_as(out), out) and torch.equal(l.view_as(lse), lse)
    for r, (pages, n) in enumerate(S.select(scores.cpu().numpy(), lens, keep, 1, 2, Sq, WIDE)):
        assert chosen[r].tolist() == pages + [-1] * (keep - len(pages)) and int(sub_lens[r]) == n
    ro, rl = R.decode(q.reshape(B * Sq, 1, H, 576), F.bf16_bits(values), np.maximum(sub.cpu().numpy(), 0), sub_lens.cpu().numpy(), SCALE)
    # An output is rounded to bf16, off by at most 2^-8 of itself; each of its weights is, so that their sum with the values is off by at most 2^-8 of the largest value
    # besides.  (Largest here: 4.8 and 6.3.  Where the two add up they pass the 2e-2 that outputs below 2 are held to elsewhere: -4.417 lies 0.0047 from the middle between two bf16 numbers 2^-5 apart.)
    v = abs(values[..., :512]).max()
    compare(out.double().cpu().numpy().reshape(ro.shape), lse.double().cpu().numpy().reshape(rl.shape), ro, rl, tol_abs=2.0 ** -8 * (abs(ro).max() + v))


def softmax(x):
    """By its definition, of numbers and infinities: a logit of -infinity has no share, one of +infinity or nothing but -infinity leaves no numbers."""
    with np.errstate(invalid="ignore"):
        e = np.exp(x - x.max())
        return e / e.sum()


@pytest.mark.parametrize("H", [1, 2, 16, 128])
@pytest.mark.parametrize("signs", [(1, 1), (1, -1), (-1, 1), (-1, -1)])
@pytest.mark.parametrize("pages", [2, 70, 700])
def test_infinite_means_follow_the_softmax(H, signs, pages):
    """(the sign of the queries in the column that is infinite, that of the infinity): what is +infinity makes its head's shares NaN, what is -infinity is no share."""
    rng = np.random.default_rng(pages)
    q, m = rng.standard_normal((1, 1, H, 576)), 0.5 * rng.standard_normal((pages + 1, 576))
    q[..., 7] = abs(q[..., 7]) * signs[0] + signs[0]
    q, m = S.values(S.bf16(q)), S.values(S.bf16(m))
    m[pages // 2, 7] = signs[1] * np.inf
    bits = lambda x: (np.ascontiguousarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)  # noqa: E731  (of numbers that bf16 has)
    table, lens = np.arange(pages + 1, dtype=np.int32)[None], np.array([64 * pages + 1], np.int32)
    got = sparse.page_scores(dev_bf16(bits(q)), dev_bf16(bits(m)), dev(table), dev(lens), SCALE).double().cpu().numpy()[0, 0]
    want = sum(softmax(q[0, 0, h] @ m[:pages].T * SCALE) for h in range(H))
    assert (np.isnan(got[:pages]) == np.isnan(want)).all() and got[pages] == 0
    if signs[0] != signs[1]:
        clean = np.delete(m, pages // 2, 0)
        _, bound = S.scores(q, clean, table[:, :pages], lens - 64, SCALE)
        assert got[pages // 2] == 0 and (abs(got[:pages] - want) <= bound[0, 0] * want).all()
    else:
        assert np.isnan(got[:pages]).all()


def test_queries_and_pages_that_are_infinite_throughout():
    """A head's logits that are -infinity for every page leave no numbers, for its token alone; a sequence's pages that all are so, too."""
    q, means = torch.ones(1, 2, 4, 576, device="cuda").bfloat16(), torch.ones(6, 576, device="cuda").bfloat16()
    table, lens = torch.arange(6, device="cuda").int().view(1, 6), torch.tensor([64 * 5 + 2], dtype=torch.int32, device="cuda")
    q[0, 0, 2] = -float("inf")
    got = sparse.page_scores(q, means, table, lens, SCALE)[0]
    assert torch.isnan(got[0, :5]).all() and not torch.isnan(got[1]).any() and not got[:, 5].any()
    q.fill_(1)
    means.fill_(-float("inf"))
    assert torch.isnan(sparse.page_scores(q, means, table, lens, SCALE)[0, :, :5]).all()
