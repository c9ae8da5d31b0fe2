"""The chunk kernel's waits, by their rules and their source: a wait that runs out must end the kernel, not leave
a part of a block waiting for warps that have gone."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_14256_b200", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def outcomes(warps, agree):
    """Every way in which `warps` warps can meet when any wait may run out at any time: the set of (how many go
    on to the hardware barrier, how many came).  A warp comes or has left already; one that came waits until all have
    come or its wait runs out; with `agree`, whoever is first settles the answer for all."""
    seen, ends = set(), set()

    def step(state):
        if state in seen:
            return
        seen.add(state)
        where, settled = state
        came = sum(w in ("waits", "full", "empty", "goes", "stops") for w in where)
        moved = False
        for i, w in enumerate(where):
            nexts = []
            if w == "before":
                nexts = [("waits", settled), ("left", settled)]
            elif w == "waits":
                nexts = [("empty", settled)] + ([("full", settled)] if came == warps else [])
            elif w in ("full", "empty"):
                answer = (settled or w) if agree else w
                nexts = [("goes" if answer == "full" else "stops", answer if agree else None)]
            for to, s in nexts:
                moved = True
                step((where[:i] + (to,) + where[i + 1:], s))
        if not moved:
            ends.add((sum(w == "goes" for w in where), came))

    step((("before",) * warps, None))
    return ends


def test_the_groups_agree_before_they_meet():
    """All of the warps go to the barrier that cannot be given up, or none does; without the agreement some orders of
    events leave a few of them there."""
    for warps in (2, 3, 4):
        ends = outcomes(warps, agree=True)
        assert {n for n, _ in ends} == {0, warps}
        assert all(came == warps for n, came in ends if n)
        assert any(0 < n < warps for n, _ in outcomes(warps, agree=False))


def test_the_barrier_of_the_groups_comes_behind_the_agreement():
    text = source("zc_paged_chunk.cu")
    bars = [m.start() for m in re.finditer(r"\bbar(?:rier)?\.(?:cta\.)?(?:sync|arrive|red)\b", text)]
    assert len(bars) == 1                          # the one that the groups share, in groups_sync
    agreement = text.index("if (meet) meet = all_here();")
    calls = [m.start() for m in re.finditer(r"groups_sync\(\);", text)]
    assert len(calls) == 2 and min(calls) > agreement
    assert "const bool other = meet &&" in text[agreement:calls[0]]
    settle = text.index("atomicCAS(meet_slot")
    assert text.index("bar_wait(meet_bar") < settle < agreement
    assert "bar.sync" not in source("zc_paged_decode.cu") and "bar.sync" not in source("zc_paged.cuh")


def test_the_warps_that_issue_leave_where_a_wait_runs_out():
    """Copies and products: every wait's answer is used before anything more is issued, and what is in flight is
    waited for at the end."""
    text = source("zc_paged_chunk.cu")
    roles = text[text.index("setmaxnreg.dec"):text.index("setmaxnreg.inc")]
    calls = list(re.finditer(r"\b(?:bar_wait|warp_wait)\(", roles))
    assert len(calls) > 8
    for m in calls:
        before = roles[:m.start()].rstrip()
        assert re.search(r"(=|!|\|\||&&|\?|:)$", before), roles[m.start() - 30:m.start() + 60]
    assert roles.count("landed(") == 2 and "drain(q_last, q_last_phase)" in roles and "drain(&drained[g], 0)" in roles
