"""Barriers between warps that each wait, with a limit, for something else, read from the sources (on a GPU no wait may be made to
run out): a wait may run out in one warp and not in another, and a warp that leaves a loop on its own lets the others wait for
it at the loop's barrier for ever.  Such a loop's first barrier therefore carries the warps' answers (bar_and) and all
leave on it together; a warp whose wait ran out comes back to it."""
import re

import pytest

from tests.test_kernel_waits import _calls, _clean, _functions, _loops, _read, _sources

BARRIERS = ("bar_named", "bar_and")


def left_alone(text):
    """Kernels with a loop that has a barrier of several warps, and in which a warp that gave up a wait leaves by itself."""
    bad = []
    for name, (kernel, body) in _functions(_clean(text)).items():
        if not kernel:
            continue
        for lo, hi in _loops(body):
            loop = body[lo:hi]
            flags = set(re.findall(r"\b(\w+) = mbar_wait(?:_warp)?\(", loop))
            at = _calls(loop, BARRIERS)
            if not flags or not at:
                continue
            head = body[body.rindex("for (", 0, lo):lo]
            for f in flags:
                if not re.search(r";[^;]*\b%s\b[^;]*;" % f, head) and not re.search(r"if \(!%s\)" % f, loop):
                    continue   # never left on it
                vote = re.match(r"bar_and\([^;]*,\s*%s\)\) break;" % f, loop[at[0]:]) and loop[:at[0]].endswith("if (!")
                # left, or not entered again, by this warp's answer alone: not in the form that has the barriers
                alone = re.search(r";[^;]*\b%s\b[^;]*;" % f, head) and not re.search(r"\(kTokens \|\| %s\) && " % f, head)
                after = loop[_calls(loop, ("mbar_wait_warp", "mbar_wait"))[-1]:]
                out = re.search(r"if \(!%s\)" % f, after)
                alone = alone or (out and not re.match(r"if \(!%s\) \{\s*if constexpr \(kTokens\) continue;\s*else break;\s*\}" % f, after[out.start():]))
                if not vote or alone:
                    bad.append(name)
    return bad


@pytest.mark.parametrize("f", _sources())
def test_warps_leave_a_barrier_together(f):
    assert left_alone(_read(f)) == []


def test_the_loop_is_found_and_each_way_out_is_caught():
    text = _read("gemm_fp4.cu")
    assert left_alone(text) == []
    for now, then in (("if (!bar_and(1 + group, 128, ok)) break;", "bar_named(1 + group, 128);"), ("(kTokens || ok) && u", "ok && u"),
                      ("if constexpr (kTokens) continue;", "if constexpr (kTokens) break;")):
        assert text.count(now) == 1
        assert left_alone(text.replace(now, then)) == ["gemm_fp4_kernel"]


class Warp:
    """A warp of the four that have the same columns: what it does at each step of its loop over tiles, as the kernel's source has it."""

    def __init__(self, tiles, fails_at):
        self.tiles, self.fails_at, self.ok, self.t, self.done = tiles, fails_at, True, 0, False

    def arrive(self):
        """Its answer at the tile's first barrier, None once it is past its last tile."""
        return self.ok if self.t < self.tiles and not self.done else None

    def leave(self):
        self.done = True

    def wait(self):
        self.ok = self.t != self.fails_at   # every later wait is the limit's again, or not reached
        self.t += 1


@pytest.mark.parametrize("tiles", [1, 2, 3, 7])
def test_four_warps_come_to_an_end_whichever_waits_run_out(tiles):
    for fails in [(f, None, None, None) for f in range(tiles)] + [(f, g, None, 0) for f in range(tiles) for g in range(tiles)] + [(None,) * 4]:
        warps = [Warp(tiles, f) for f in fails]
        for _ in range(tiles + 1):
            answers = [w.arrive() for w in warps]
            assert len({a is None for a in answers}) == 1   # all four come to the barrier, or none does
            if answers[0] is None:
                break
            for w in warps:
                w.wait() if all(answers) else w.leave()
        assert all(w.arrive() is None for w in warps)
