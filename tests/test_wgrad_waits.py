"""The weight gradient kernel's bounded waits.  One that runs out would need a GPU whose
copies or products never come, so what happens then is looked for in the source."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2609_06086_gb300", "csrc")


def kernel():
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "wgrad.cu")).read())
    body = text[text.index("    wgrad_kernel(const __grid_constant__"):]
    return text, body[:body.index("\n}\n")]


def test_a_warp_gives_up_as_a_whole():
    """Lanes of a warp may differ in whether a wait gave up, and one that left its loop
    would be waited for by the others' next vote.  So a wait belongs to a single lane, or
    its outcome is voted on at once, and nothing but a vote's result ends a loop."""
    text, body = kernel()
    wait = r"\bbar_wait\("
    alone = re.findall(r"if \(warp == \d[^{]*lane == 0\) \{(.*?)(?=\n        \} else if)", body,
                       re.S)
    assert sum(len(re.findall(wait, a)) for a in alone) == 3
    decode = body[body.index("group <= kDecodeGroups"):body.index("take_registers<kSumRegs>")]
    assert len(re.findall(wait, decode)) == 2
    assert len(re.findall(wait, body)) == 5 and len(re.findall(r"\bbar_wait_warp\(", body)) == 2
    vote = text[text.index("bool bar_wait_warp("):]
    assert "__all_sync(0xffffffffu, bar_wait(" in vote[:vote.index("}")]
    assert re.findall(r"if \(([^;{]*)\) break;", decode) == ["!ok"]
    votes = re.findall(r"ok = __all_sync\(0xffffffffu, (\w+)\([^;]*&&\s*(\w+)\([^;]*;", decode)
    assert votes == [("bar_try", "bar_try"), ("bar_wait", "bar_wait")]
    assert len(re.findall(r"\bok = ", decode)) == 3  # true, and the votes


def test_only_a_waits_own_time_counts(tmp_path):
    """The limit against a clock of the test's: two seconds of tries a millisecond or a
    microsecond apart run out, and not before; gaps of ten seconds, in which the GPU ran
    something else, do not use them up."""
    src = tmp_path / "limit.cpp"
    src.write_text("""
#include <cstdio>
#include "%s"
// tries until the limit, the clock moving by `step`, at every `every`-th try by `jump`
static long tries(uint64_t step, long every, uint64_t jump) {
    uint64_t now = 12345;
    pos::WaitLimit limit(now);
    for (long i = 1;; ++i) {
        now += every && i %% every == 0 ? jump : step;
        if (limit.reached(now)) return i;
        if (i > 100000000) return -1;
    }
}
int main() {
    const uint64_t us = 1000, ms = 1000000, s = 1000000000;
    std::printf("%%ld %%ld %%ld %%ld\\n", tries(ms, 0, 0), tries(us, 0, 0), tries(ms, 100, 10 * s),
                tries(10 * s, 0, 0));
}
""" % os.path.join(CSRC, "wait_limit.h"))
    subprocess.run(["g++", "-std=c++17", "-O2", "-o", str(tmp_path / "limit"), str(src)], check=True)
    out = subprocess.run([str(tmp_path / "limit")], capture_output=True, text=True, check=True).stdout
    each_ms, each_us, jumps, all_jumps = map(int, out.split())
    assert each_ms == 2001 and each_us == 2000001
    assert 1900 <= jumps <= 2000   # 19 gaps of four milliseconds among them
    assert all_jumps == 501
