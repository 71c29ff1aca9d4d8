"""Waits of the attention over the 8-bit cache after one of them has run out, on the host: nobody is left behind."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2402_11809_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = tmp_path_factory.mktemp("waits") / "kvb_waits.so"
    cmd = [build._nvcc(), "-gencode", "arch=compute_100a,code=compute_100a", "-O0", "-std=c++17", "-shared", "-Xcompiler", "-fPIC",
           "-cudart", "static", "-Xlinker", "--unresolved-symbols=ignore-all", os.path.join(HERE, "kvb_waits_host.cu"), "-o", str(so)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    return C.CDLL(str(so), os.RTLD_LAZY)


def bring(lib, answers, alone):
    a, brought = np.ascontiguousarray(answers, np.int32), np.zeros(2, np.int32)
    p = lambda x: x.ctypes.data_as(C.c_void_p)  # noqa: E731
    return lib.host_bring_own(p(a), len(a), int(alone), p(brought)), brought.tolist()


ANSWERS = [[[1, 1]] * 5, [[1, 1], [0, 1], [1, 1]], [[1, 1], [1, 0], [1, 1]], [[0, 1]], [[1, 0]], [[0, 0], [1, 1]], [[1, 1], [1, 1], [1, 0], [0, 1]]]


@pytest.mark.parametrize("answers", ANSWERS)
def test_both_warps_go_by_both_answers(lib, answers):
    stuck, brought = bring(lib, answers, False)
    n = next((i for i, a in enumerate(answers) if not all(a)), len(answers))
    assert not stuck and brought == [n, n]


def test_answers_of_their_own_leave_a_warp_behind(lib):
    assert bring(lib, [[1, 1], [1, 0], [1, 1]], True)[0] and not bring(lib, [[1, 1]] * 3, True)[0]


def test_the_kernel_leaves_with_both_warps_only():
    text = open(os.path.join(build.CSRC, "kvb_attn_tc.cu")).read()
    role = text[text.index("// ---- the block's own rows, an item ahead"):text.index("bring_own<DH>(p, wk.b")]
    assert role.count("break") == 1 and "if (!all_told(place, pair_all)) break;" in role


@pytest.mark.parametrize("src", ["kvb_attn.cu", "kvq_attn.cu"])
def test_a_warp_goes_by_one_answer(src):
    """What a whole warp goes by, how a wait ended and whether one has run out, is voted on by its lanes."""
    text = open(os.path.join(build.CSRC, src)).read()
    kernel = text[text.index("__global__"):]
    assert not re.search(r"(?<!warp_)wait\(bar", kernel) and "if (!warp_wait(bar" in kernel
    assert "const bool over = __any_sync(0xFFFFFFFFu, *abort_flag);" in kernel and kernel.count("*abort_flag") == 2      # (the other: cleared)
    header = open(os.path.join(build.CSRC, "kvq_attn.cuh")).read()
    assert "return __all_sync(0xFFFFFFFFu, wait(" in header[header.index("bool warp_wait("):]


def test_the_softmax_goes_by_announcements_together():
    text = open(os.path.join(build.CSRC, "kvb_attn_tc.cu")).read()
    look = text[text.index("auto look = [&]"):text.index("next_page = desc[m")]
    assert "__all_sync(0xFFFFFFFFu, hold(SAID" in look


def test_products_are_done_before_tensor_memory_is_released():
    """Whatever has run out: the thread that asked for the products waits for a barrier of its own, without a look at the flag."""
    text = open(os.path.join(build.CSRC, "kvb_attn_tc.cu")).read()
    role = text[text.index("// ---- products: scores of page q"):text.index("} else if (warp >= 10) {")]
    assert role.rstrip().endswith("mbar_drain_bounded(BAR(OVER), 0, WAIT_NS);")
    assert role.index("tc_commit(BAR(OVER));") > max(role.rindex("mma8_ts("), role.rindex("++m;"))
    assert text.count("BAR(OVER)") == 3 and "mbar_init(BAR(OVER), 1);" in text
    drain = open(os.path.join(build.CSRC, "tc_common.cuh")).read()
    drain = drain[drain.index("void mbar_drain_bounded("):]
    assert "abort_flag" not in drain[:drain.index("\n}")]


def test_scores_are_read_before_weights_take_their_place():
    """Where both halves of a row have the same 32 columns, tensor memory changes hands with their largest scores."""
    text = open(os.path.join(build.CSRC, "kvb_attn_tc.cu")).read()
    meet = text[text.index("auto meet = [&]"):text.index("auto put = [&]")]
    at = [meet.index(x) for x in ("if (REP == 4) tc_fence_before();", "mbar_arrive(BAR(XCH + w4))", "hold(XCH + w4, m, 16)", "if (REP == 4) tc_fence_after();", "xch[threadIdx.x ^ GROUP]")]
    assert at == sorted(at)
    read = text.index("tmem_ld16(TM_SM + key0, v)")
    assert read < text.index("tmem_wait_ld();", read) < text.index("auto meet = [&]")
