"""paging.cache_format, also as the first call of a process (without a device, and without the library)."""
import subprocess
import sys

import pytest
import torch

from conftest import ROOT
from paper_2509_25224_b200 import paging


@pytest.mark.parametrize("make,want", [("torch.zeros(2, 64, 576, dtype=torch.bfloat16)", paging.CACHE_BF16), ("torch.zeros(2, 64, 576, dtype=torch.uint8)", paging.CACHE_E4M3),
                                       ("torch.zeros(2, 20736, dtype=torch.uint8)", paging.CACHE_FP4), ("torch.zeros(2, 64, 576)", None)])
def test_as_the_first_call_of_a_process(make, want):
    program = ("import torch\nfrom paper_2509_25224_b200 import binding, paging\nbinding.lib = None\n"
               "try:\n    print('format', paging.cache_format(%s))\nexcept ValueError:\n    print('format', None)\n" % make)
    r = subprocess.run([sys.executable, "-c", program], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert r.stdout.split() == ["format", str(want)]


@pytest.mark.parametrize("shape,dtype", [((2, 64, 576), torch.float16), ((2, 64, 512), torch.uint8), ((64, 576), torch.bfloat16), ((2, 20736), torch.bfloat16), ((2, 20735), torch.uint8), ((0,), torch.uint8)])
def test_what_is_no_cache_is_refused(shape, dtype):
    with pytest.raises(ValueError):
        paging.cache_format(torch.zeros(shape, dtype=dtype))
