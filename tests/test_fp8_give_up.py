"""What the 8-bit kernels do once a bounded wait has expired, checked by reading their sources (CPU): a role that issues copies or
products waits for them before the CTA's memory goes, whether its own waits expired or another's, and every wait is bounded."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2405_03594_gb300", "csrc")
FILES = ("sp_fp8_few.cu", "sp_fp8_linear.cu")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"/\*.*?\*/|//[^\n]*", "", f.read(), flags=re.S)


def role(s, first, last):
    """From the last of `first`'s uses on to the first of `last` behind it."""
    i = s.rindex(first)
    return s[i:s.index(last, i)]


def test_the_copies_of_few_tokens_are_waited_for_by_whoever_issued_them():
    text = role(source("sp_fp8_few.cu"), "tma_load_2d(", "warp == 5")
    # behind the loop, under no condition on the role's own waits
    assert re.search(r"for \(int i = max\(0, issued - S\); i < issued; \+\+i\) mbar_wait\(&w_full", text)
    assert not re.search(r"if \(dead\) \{", text)


def test_the_copies_of_many_tokens_are_waited_for_by_whoever_issued_them():
    text = role(source("sp_fp8_linear.cu"), "tma_load_2d_pair(", "warp == 1")
    # every stage's products are waited for; where one does not come, the copies get the time of another wait
    assert re.search(r"for \(int j = 0; j < P::kStages && !dead; \+\+j\)\s*\{\s*dead = !mbar_wait_short\(&done", text)
    assert re.search(r"if \(dead\) \{[^}]*mbar_wait\(never", text)


@pytest.mark.parametrize("name", FILES)
def test_products_are_drained(name):
    s = source(name)
    text = s[s.rindex("mma_commit"):]
    assert re.search(r"mma_commit2?\(drain\)", s) and re.match(r"mma_commit2?\(drain\);\s*__syncwarp\(\);\s*if \(!mbar_wait_short\(drain, 0", text)


@pytest.mark.parametrize("name", FILES)
def test_waits_are_bounded_and_barriers_are_not_left_out(name):
    s = source(name)
    assert not re.search(r"while \(!mbar|while \(true\)|for \(;;\)", s)
    for m in re.finditer(r"mbar_wait\w*\(([^;]*?)\)\)?[;)&|]", s):
        assert "timeout_ns" in m.group(1), m.group(0)
    # no barrier of several warps or CTAs under a condition on a wait that expired
    for barrier in ("named_bar_sync(", "cluster_sync_all(", "__syncthreads("):
        for m in re.finditer(re.escape(barrier), s):
            assert not re.search(r"if \([^)]*(dead|ok)\)\s*\{?\s*$", s[:m.start()]), barrier
