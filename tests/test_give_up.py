"""What the attention kernels do once a bounded wait has expired, checked by reading their sources (CPU).  Such
a path is not run where it could hang or leave a copy behind, so its rules are held here; the launches
of tests/test_gpu_serve_failure.py take it where they hold."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2405_03594_gb300", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"/\*.*?\*/|//[^\n]*", "", f.read(), flags=re.S)


def closing(s, i):
    """Index of the brace that closes s[i]."""
    depth = 0
    for j in range(i, len(s)):
        depth += (s[j] == "{") - (s[j] == "}")
        if depth == 0:
            return j
    raise AssertionError("unbalanced source")


def body(s, name):
    """The body of the function `name`."""
    m = re.search(r"\b%s\s*\(" % name, s)
    i = s.index("{", s.index(")", m.end()))
    return s[i:closing(s, i) + 1]


def leaves_with_work_behind(text):
    """Whether a role leaves, once any warp has given up, without waiting for what it has issued."""
    m = re.search(r"if\s*\(!end_item\(wait\)\)\s*", text)
    if text[m.end()] != "{":
        return True
    left = text[m.end():closing(text, m.end())]
    return not re.search(r"\bmbar_wait\w*\s*\(", left)


def barriers_that_one_warp_can_miss(text):
    """Where a warp leaves a loop with a barrier of several warps because of its own expired wait."""
    loops = text[:text.index("end_item(")]
    assert re.search(r"\bnamed_bar_sync\(2\b", loops)
    return re.findall(r"\bif\s*\([^)]*\bdead\s*\)\s*\{?\s*(?:break|continue|return)", loops)


def test_no_warp_misses_a_barrier_that_others_wait_at():
    """A warp judges its waits alone: the one that expires and the one that completes at the same moment must
    meet at the same barriers until the item's end, or the others wait there without a bound."""
    s = source("sp_attend_rows.cu")
    assert barriers_that_one_warp_can_miss(body(s, "fill_role")) == []
    assert not re.search(r"\bsh\.dead\b", s)  # and at its end all get the same verdict, a barrier's, not a flag's


def test_the_check_of_barriers_finds_one_that_can_be_missed():
    loop = "{ for (int j = 0; j < n; ++j) { wait(a); %s named_bar_sync(2, 128); } alive = end_item(wait); if (!alive) break; }"
    assert barriers_that_one_warp_can_miss(loop % "if (wait.dead) break; fill();")
    assert barriers_that_one_warp_can_miss(loop % "if (wait.dead) { return; } fill();")
    assert not barriers_that_one_warp_can_miss(loop % "if (!wait.dead) { fill(); }")


def test_roles_that_issue_copies_and_products_wait_for_them_before_the_cta_ends():
    s = source("sp_attend_rows.cu")
    for role, issues in (("copy_role", "bulk_g2s"), ("product_role", "mma_commit")):
        text = body(s, role)
        assert issues in text
        assert not leaves_with_work_behind(text), role


def test_the_check_of_roles_finds_one_that_leaves():
    assert leaves_with_work_behind("{ bulk_g2s(a); if (!end_item(wait)) break; }")
    assert leaves_with_work_behind("{ if (!end_item(wait)) { x = 1; break; } }")
    assert not leaves_with_work_behind("{ if (!end_item(wait)) { mbar_wait_sleep(b, 0, t); break; } }")
