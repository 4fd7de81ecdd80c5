"""Bounded waits that run out, read from the sources (on a GPU none may be made to): the
kernels of the orthogonalised updates record them in the call's status word, and no
kernel adds up a split tile whose parts are not all there."""
import re

import pytest

from tests.test_kernel_waits import _clean, _read


def test_waits_of_the_updates_are_recorded():
    """Every wait that runs out ends in one of the accumulator's, which the epilogue's warps make: the producers' and the issuer's
    ones keep the accumulator from being committed."""
    text = _clean(_read("orth_product.cu"))
    epilogue = text[text.index("} else if (warp >= 4) {"):]
    assert re.search(r"auto give_up = \[&\] \{\s*if \(lane == 0\) atomicCAS\(a\.status, kDevOk, kDevTimeoutAccum\);", epilogue)
    waits = re.findall(r"mbar_wait_warp\(&bars->accf\[b\][^;]*kDevTimeoutAccum\)\)\)?[^;]*;", epilogue)
    assert len(waits) == 2 and len(re.findall(r"\bmbar_wait", epilogue)) == 2 and len(re.findall(r"\bgive_up\(\);\s*break;", epilogue)) == 2
    for f in ("orth_small.cu", "orthogonal.cu"):
        assert "mbar_wait" not in _clean(_read(f))


def test_the_last_kernel_looks_at_the_status_before_it_writes():
    text = _clean(_read("orth_product.cu"))
    assert re.search(r"before = EPI == kNsLast && warp >= 4 \? \*static_cast<const volatile int\*>\(a\.status\) : 0;", text)
    assert re.search(r"rows = col < a\.N && before == 0 \?", text)
    # read behind the wait for the launch before, whose status it is
    assert text.index("pdl_wait();") < text.index("before = EPI == kNsLast")


@pytest.mark.parametrize("f,give_up", [("orth_product.cu", r"if \(kSplit && lane < a\.split\) st_dsmem_at\(cluster_addr\(&bars->failed, lane\), 1u\);"),
                                       ("gemm_i8.cu", r"if \(kSplit && lane < a\.split\) st_peer\(&bars->failed, lane, 1\);")])
def test_parts_that_are_missing_are_not_added_up(f, give_up):
    text = _clean(_read(f))
    start, told = re.search(r"bars->failed = 0;", text), re.search(give_up, text)
    read = re.search(r"missing = bars->failed;[^}]*?for \([^;]*;[^;]*missing == 0[^;]*;", text)
    syncs = [m.start() for m in re.finditer(r"if \(CL > 1 \|\| kSplit\) cluster_sync\(\);", text)]
    assert start and told and read and len(syncs) == 2
    # initialised before the peers start, told before the barrier, read behind it
    assert start.start() < syncs[0] < told.start() < syncs[1] < read.start()
