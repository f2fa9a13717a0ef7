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
