"""What is not a number stays in its row, in calls that split their sequences and merge them as in those that do not, for every cache and kernel."""
import math

import numpy as np
import pytest
import torch

from _gpu_util import compare, to_device, wide_table
from paper_2509_25224_b200 import binding, synth
from test_gpu_fp4 import bf16, dev, expected, run, workload
from test_gpu_merge import merge_alone  # noqa: F401  (a fixture: the merge kernel by itself)

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def test_the_merge_takes_over_a_nan_and_leaves_out_what_saw_nothing(merge_alone):  # noqa: F811
    # four partials of 16 rows in items of 32, of which partial s is s + 1 everywhere
    cuda = torch.device("cuda", 0)
    info = torch.tensor([[0, 0, 4, 0]], dtype=torch.int32, device=cuda)
    slots = [0, 2, 4, 6]                                      # a part has two
    part_lse = torch.full((8, 32), 50.0, device=cuda)         # (slots that are not named must not matter)
    part_o = torch.full((8, 32, 512), -9.0, device=cuda)
    for s, slot in enumerate(slots):
        part_lse[slot], part_o[slot] = 0.0, s + 1.0
    part_lse[4, 3] = NAN                                      # row 3: one partial is not a number
    part_lse[0, 5], part_o[0, 5] = -INF, 0.0                  # row 5: one saw nothing
    part_lse[slots, 7] = -INF                                 # row 7: none saw anything
    part_o[slots, 7] = 0.0
    word = torch.zeros(1, dtype=torch.int32, device=cuda)
    out, lse = torch.full((16, 512), -7.0, dtype=torch.bfloat16, device=cuda), torch.full((16,), -7.0, device=cuda)
    stream = torch.cuda.current_stream().cuda_stream
    assert merge_alone(word.data_ptr(), info.data_ptr(), part_lse.data_ptr(), part_o.data_ptr(), out.data_ptr(), lse.data_ptr(), stream) == 0
    out, lse = out.float().cpu().numpy(), lse.cpu().numpy()
    assert np.isnan(out[3]).all() and math.isnan(lse[3])
    assert (out[5] == 3.0).all() and abs(lse[5] - math.log(3)) < 1e-6
    assert (out[7] == 0.0).all() and lse[7] == -INF
    rest = [r for r in range(16) if r not in (3, 5, 7)]
    assert (out[rest] == 2.5).all() and np.abs(lse[rest] - math.log(4)).max() < 1e-6


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("Sq,H,kernel", [(1, 16, 32), (1, 128, 128), (2, 128, 256)])
def test_rows_of_a_bf16_call(Sq, H, kernel, split, bad):
    # sequences of two keys a part and of thousands in few parts; a row whose Q holds such a thing has no row sum
    lens = [4000, 2500] if split else [128, 90] * 80
    w = synth.make_workload("nan", len(lens), Sq, H, lens, seed=2700 + H)
    if kernel == 256:
        wide_table(w)
    q, kv, bt, sl = to_device(w)
    want, lse = binding.mla_decode(q, kv, bt, sl, w.scale)
    assert binding.last_item_rows() == kernel
    q[1, Sq - 1, H - 3, 123] = bad
    got, bad_lse = binding.mla_decode(q, kv, bt, sl, w.scale)
    at = (1, Sq - 1, H - 3)
    row = got[at].clone()
    assert bad_lse[at] == -INF and (torch.isnan(row).all() or (row == 0).all())
    got[at], bad_lse[at] = want[at], lse[at]
    assert torch.equal(got.view(torch.int16), want.view(torch.int16)) and torch.equal(bad_lse, lse)


@pytest.mark.parametrize("bits", [0x7FC0, 0x7F80, 0xFF80])
@pytest.mark.parametrize("lens", [[4000, 900], [200, 100]])
@pytest.mark.parametrize("H", [16, 32, 128])
def test_rows_of_a_4_bit_call(H, lens, bits):
    q, cache, table, n = workload(lens, 1, H)
    q = q.copy()
    ref_out, ref_lse = expected(q, cache, table, n, 0.25)
    q[1, 0, H - 3, 123] = bits
    out, lse = run(q, cache, table, n, 0.25)
    at = (1, 0, H - 3)
    assert np.isnan(out[at]).all() and math.isnan(lse[at])
    out[at], lse[at] = ref_out[at], ref_lse[at]
    compare(out, lse, ref_out, ref_lse)
