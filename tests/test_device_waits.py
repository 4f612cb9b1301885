"""What the kernels do when a wait runs out, as far as reading shows it: no run makes a wait run out at a given place."""
import os
import re
import subprocess

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


RING = r"""
#include <stdio.h>
#include "ring.cuh"
int main() {
    int i, st, phase;
    while (scanf("%d %d %d", &i, &st, &phase) == 3) printf("%d\n", flowmm::last_copy_parity(i, st, phase));
}
"""


def test_the_wait_for_a_rings_last_copies_ends_when_they_have_landed(tmp_path):
    """A barrier model: a stage's copies complete its phases 0, 1, 2, ...; a wait for a parity passes unless the phase with that parity is the one
    under way.  Whatever number of copies a ring of n stages has had: a stage lets the wait pass when, and only when, its last copy has landed."""
    (tmp_path / "r.cpp").write_text(RING)
    subprocess.check_call(["g++", "-std=c++17", "-I", CSRC, "-o", str(tmp_path / "r"), str(tmp_path / "r.cpp")])
    cases = [(i, n, copies) for n in range(1, 11) for copies in range(4 * n + 1) for i in range(n)]
    text = "".join("%d %d %d\n" % (i, copies % n, copies // n & 1) for i, n, copies in cases)
    out = subprocess.run([str(tmp_path / "r")], input=text, capture_output=True, text=True, check=True).stdout.split()
    for (i, n, copies), parity in zip(cases, map(int, out)):
        fills = len(range(i, copies, n))
        passes = lambda completed: completed & 1 != parity          # the phase under way is number `completed`
        assert passes(fills), (i, n, copies)
        assert fills == 0 or not passes(fills - 1), (i, n, copies)


def test_no_wait_takes_either_parity():
    """One of the two always lets it pass: such a wait waits for nothing.  Warps that issue a ring's copies see them land."""
    loaders = {}
    for name in sorted(os.listdir(CSRC)):
        text = _text(name)
        assert not re.search(r"mbar_try_wait\(([^;]*), 0\) && !(?:tc::)?mbar_try_wait\(\1, 1\)", text), name
        n = len(re.findall(r"tc::copies_land\(", text))
        if n:
            loaders[name] = n                                       # rings
    assert loaders == {"decode_tc.cuh": 1, "match_merge_tc.cuh": 3, "match_small_tc.cuh": 2, "merge_tc.cuh": 1, "paged_attention_tc.cuh": 1,
                       "score_fused_tc.cuh": 2, "tc_stream.cuh": 3}, loaders
