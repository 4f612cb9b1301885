"""What the kernels do when a wait runs out, as far as reading shows it: no run makes a wait run out at a given place."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_05534_b200", "csrc")


def _text(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def _body(text, at):
    """The braces' content that begins at the first '{' from `at` on."""
    start = i = text.index("{", at) + 1
    depth = 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
    return text[start:i - 1]


def test_warps_that_meet_in_a_loop_leave_it_together():
    """Where a warp's loop ends by what it has waited for (a task), and not by a number that all its warps know, one warp may give up where
    another one does not.  A barrier of theirs inside must then decide for all of them: it counts the warps in and says whether all go on."""
    text = _text("paged_attention_tc.cuh")
    kernel = _body(text, text.index("cache_attention_tc_kernel(const __grid_constant__"))
    loops = [kernel[m.start():m.end()] + _body(kernel, m.end() - 1) for m in re.finditer(r"\b(?:for|while) \([^;{]*(?:;[^;{]*;)?[^;{]*\{", kernel)
             if re.search(r"(wait|take)_task\(", m.group())]
    meeting = [body for body in loops if "epi_" in body or "bar.sync" in body]
    assert len(meeting) == 1, [body[:80] for body in loops]
    assert "bar.sync" not in text and "bar.red.and.pred" in text
    calls = re.findall(r"[^\n]*\bepi_all\([^\n]*", kernel)
    assert len(calls) == 3 and all(re.search(r"if \(!?epi_all\(ok\)|= epi_all\(ok\)", c) for c in calls), calls
    # left at once, and with no other barrier behind
    assert re.search(r"if \(!epi_all\(ok\)\) \{\s*together = false;\s*break;", meeting[0])
    assert re.search(r"if \(together && group > 0\)", kernel)


def test_a_tensor_memory_read_on_its_way_is_waited_for_also_after_a_give_up():
    """Its registers would be written when they already hold something else."""
    text = _text("paged_attention_tc.cuh")
    kernel = _body(text, text.index("cache_attention_tc_kernel(const __grid_constant__"))
    assert kernel.count("tmem_ld_wait(s);") == 2 and len(re.findall(r"tmem_ld_wait\(s\);\s*if \(!ok\) continue;", kernel)) == 2
