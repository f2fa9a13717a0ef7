"""Waits that are bounded by a number of tries: they run out, say so, do not wait again, and cost nothing where there is nothing to wait for."""
import ctypes

import pytest

from paper_2509_25224_b200 import binding, build


def test_bad_arguments_are_refused_without_a_device():
    build.build()
    f, z, p = binding.lib().amla_wait_tries_selftest, ctypes.c_void_p(0), ctypes.c_void_p(256)
    for args in [(z, 10, p), (p, 10, z), (p, 0, p), (p, -1, p), (p, 4097, p), (ctypes.c_void_p(258), 10, p), (p, 10, ctypes.c_void_p(258))]:
        assert f(*args, z) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("tries", [1, 16, 1024])
def test_a_wait_runs_out_of_tries(tries):
    import torch
    ws, report = torch.zeros(256, dtype=torch.uint8, device="cuda"), torch.full((5,), -7, dtype=torch.int32, device="cuda")
    binding.wait_tries_selftest(ws, report, tries)
    with pytest.raises(binding.AmlaError) as e:
        binding.check_status(ws)
    assert e.value.code == -5
    after, second, complete, ns, ns_second = report.tolist()
    print("%d tries: %.1f us, %.2f a try" % (tries, ns / 1e3, ns / 1e3 / tries))
    assert after == 0 and complete == tries
    assert second == -1                                       # one look, no loop
    # the decode kernel has 2^18 of them: that is a bound (below ten seconds) and not the first hiccup (above a millisecond)
    if tries == 1024:
        assert 1e6 < ns / tries * 2 ** 18 < 10e9


@pytest.mark.gpu
def test_the_context_decodes_on_afterwards():
    import torch
    ws, report = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    binding.wait_tries_selftest(ws, report, 16)
    q, cache = torch.zeros((1, 1, 16, 576), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 20736), dtype=torch.uint8, device="cuda")
    ws = torch.cat([ws, torch.zeros(binding.fp4_workspace_size(1, 1, 16, 1, 0), dtype=torch.uint8, device="cuda")])
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    out, lse = binding.mla_decode_fp4(q, cache, 1.0, i(0).view(1, 1), i(5), 0.1, workspace=ws)
    binding.check_status(ws)
    assert not out.any() and torch.allclose(lse, torch.full_like(lse, 1.6094379))
