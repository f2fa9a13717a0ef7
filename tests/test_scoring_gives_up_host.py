"""What the scoring kernel leaves behind when a wait runs out, read from its source (no role of a real kernel is starved on a GPU)."""
import os
import re

from paper_2509_25224_b200 import build

SOURCE = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, "amla_select.cu")).read())
KERNEL = SOURCE[SOURCE.index("page_scores_kernel(const ScoreParams p"):SOURCE.index("pages_select_kernel(const SelectParams p)")]


def issuer(kernel):
    """What the thread that issues products does behind its last one."""
    role = kernel[kernel.index("if (elect_one())"):]
    return role[role.rindex("mma_ss(", 0, role.index("__syncwarp();")):role.index("__syncwarp();")]


def waits_for_all_products(kernel):
    """Whether it gave up or not: those who add the products up may have given up on them, and then nobody else waits before tensor memory goes back."""
    end = issuer(kernel)
    gave_up = re.search(r"if \(!ok\) \{\s*mma_commit\(bar\(X_GIVE_UP\)\);\s*mbar_wait\(bar\(X_GIVE_UP\), 0\);", end)
    went_on = re.search(r"for \(int (\w+) = 0; \1 < 2; \+\+\1\)\s*if \(ok && used\[\1\] > 0\) ok = mbar_wait\(bar\(X_DONE \+ \1\), \(used\[\1\] - 1\) & 1\);", end)
    return gave_up is not None and went_on is not None


def test_the_issuer_waits_for_its_products_whoever_gave_up():
    assert waits_for_all_products(KERNEL)
    # every product is committed to the barrier that is waited for, and both uses of a buffer are counted in one place
    assert len(re.findall(r"mma_ss\(", KERNEL)) == 1 and len(re.findall(r"\+\+used\[buf\]", KERNEL)) == 1
    assert re.search(r"if \(ok\) mma_commit\(bar\(X_DONE \+ buf\)\);", KERNEL)


def test_an_issuer_that_does_not_wait_would_be_seen():
    assert not waits_for_all_products(KERNEL.replace("ok = mbar_wait(bar(X_DONE + i), (used[i] - 1) & 1)", ""))
    assert not waits_for_all_products(KERNEL.replace("mbar_wait(bar(X_GIVE_UP), 0);", ""))


def keeps_its_place(kernel):
    """A peer may send a row's statistics when this block has given up on them: it sends them before it comes to the cluster's barrier, so that behind this and a wait
    (with a limit) they are in, and the block may end or use the memory for something else."""
    exchange = kernel[kernel.index("st_async_v2("):]
    noted = re.search(r"const bool told = mbar_wait<true>\(bar\(X_STATS\), 0\);\s*ok = __all_sync\(0xffffffffu, told && ok\);\s*if \(!told\) \*late = 1;", exchange)
    end = kernel[kernel.rindex("tc_fence_before_sync();"):]
    behind = re.search(r"if \(\*late\) \{\s*cluster_arrive\(\);\s*cluster_wait\(\);\s*mbar_wait<true>\(bar\(X_STATS\), 0\);\s*(if \(select\.table == nullptr\) return;)\s*scratch\.clear\(\);", end)
    return noted is not None and behind is not None and end.index("__syncthreads();") < end.index("tmem_dealloc(") < behind.start() and len(re.findall(r"\*late = ", kernel)) == 2


def test_statistics_that_come_late_find_their_place():
    assert keeps_its_place(KERNEL)
    # each block sends to all of its cluster, whatever it has given up on, and only in one place
    assert len(re.findall(r"st_async_v2\(", KERNEL)) == 1 and re.search(r"for \(int i = 0; i < blocks; \+\+i\) st_async_v2\(", KERNEL)
    assert not re.search(r"if \([^\n]*ok[^\n]*\)[^\n]*st_async_v2\(", KERNEL)


def test_a_block_that_does_not_wait_for_them_would_be_seen():
    end = KERNEL.rindex("mbar_wait<true>(bar(X_STATS), 0);")
    assert not keeps_its_place(KERNEL[:end] + KERNEL[end + len("mbar_wait<true>(bar(X_STATS), 0);"):])
    assert not keeps_its_place(KERNEL.replace("if (!told) *late = 1;", ""))
