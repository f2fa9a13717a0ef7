"""What the kernel for a 4-bit cache does when a wait runs out, read from its source (no role of a real kernel is starved on a GPU): products that were
issued behind such a wait are waited for before tensor memory is given back, and it is given back wherever the kernel returns."""
import os
import re

from paper_2509_25224_b200 import build

SOURCE = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, "amla_decode_fp4.cu")).read())
KERNEL = SOURCE[SOURCE.index("decode_fp4_kernel(const DecodeParams prm)"):SOURCE.index("int fp4_item_rows")]


def test_roles_that_issue_products_wait_for_them_when_they_give_up():
    roles = [r for r in re.split(r"if \((?=wid )", KERNEL) if "mma_ts(" in r]
    assert len(roles) == 2
    barriers = []
    for r in roles:
        end = r[r.rindex("mma_ts("):]
        barriers += re.findall(r"if \(!ok\) give_up\(bar\((C::X_\w+)\)\);", end)
        assert "report_timeout(" not in end.split("give_up(")[0]
    assert len(set(barriers)) == 2                            # each has its own, and nobody else arrives there
    for b in barriers:
        assert "mbar_init(bar(%s), 1)" % b in KERNEL and KERNEL.count(b) == 2
    body = re.search(r"auto give_up = \[&\]\(uint32_t (\w+)\) \{(.*?)\};", KERNEL, re.S)
    assert re.search(r"mma_commit\(%s\);\s*mbar_wait_inline\(%s, 0\);" % (body[1], body[1]), body[2])


def test_tensor_memory_is_given_back_wherever_the_kernel_returns():
    # (from the barrier behind which all warps know the address to the end, in the kernel itself: the roles' helpers return too)
    behind = KERNEL[KERNEL.index("tmem_alloc("):]
    setup = behind[:behind.index("setmaxnreg")]
    returns = [m.start() for m in re.finditer(r"\breturn;", setup)]
    assert len(returns) == 1 and "tmem_dealloc(" in setup[setup.index("if (ld_shared_b32(tmem_slot) != 0)"):returns[0]]
    last = behind[behind.rindex("__syncthreads();"):]
    assert "tmem_dealloc(" in last
