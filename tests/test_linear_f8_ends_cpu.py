"""CPU: the end of the loading warps of the products of 8-bit floating point numbers.  Their waits, as an event model that may stop any warp at any step, and the
places in the source that the model stands for."""
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(__file__), "..", "paper_2208_00763_b200", "csrc", "hikonv_linear_f8.cu")


def passes(phases, parity):
    """Whether a wait for the phase of this parity passes at a barrier of which so many phases have completed."""
    return (phases - 1) & 1 == parity


@pytest.mark.parametrize("stages", range(2, 13))
def test_a_free_stage_is_one_whose_last_multiply_has_arrived(stages):
    for loads in range(5 * stages):
        stage, phase = loads % stages, loads // stages & 1                 # the ring behind so many loads
        arrived = [len(range(s, loads, stages)) for s in range(stages)]    # phases of `empty` when all multiplies have arrived
        for _ in range(stages):
            assert passes(arrived[stage], phase ^ 1)
            # with the last one missing the wait does not pass
            assert arrived[stage] == 0 or not passes(arrived[stage] - 1, phase ^ 1)
            stage += 1
            if stage == stages:
                stage, phase = 0, phase ^ 1


def pair(stages, steps, stop, rng, mend=True):
    """Two loading warps and the multiplying ones, which stop where their wait runs out (`stop`: steps of each); then the end's work on the first
    CTA.  Returns copies that are in flight when its last wait passes."""
    pending, bytes_due, full = [1] * stages, [0] * stages, [0] * stages
    flight, loads, multiplied = [], [0, 0], 0

    def settle(s):
        if pending[s] == 0 and bytes_due[s] == 0:
            full[s] += 1
            pending[s] = 1

    def expect(s, n):
        pending[s] -= 1
        bytes_due[s] += n
        assert pending[s] >= 0
        settle(s)

    def land(i):
        s = flight.pop(i)
        bytes_due[s] -= 1
        settle(s)

    while True:
        acts = [("load", r) for r in (0, 1) if loads[r] < min(steps, stop[r]) and loads[r] - multiplied < stages]
        if multiplied < min(steps, stop[2]) and full[multiplied % stages] > multiplied // stages:
            acts.append(("multiply", 0))
        acts += [("land", i) for i in range(len(flight))]
        if not acts or all(a[0] == "land" for a in acts) and rng.random() < 0.5:
            break
        what, i = rng.choice(acts)
        if what == "land":
            land(i)
        elif what == "multiply":
            multiplied += 1
        else:
            if i == 0:
                expect(loads[0] % stages, 2)
            flight.append(loads[i] % stages)
            loads[i] += 1
    if loads == [steps, steps] and multiplied == steps:
        return len(flight)                                                 # every stage is free again
    mine, theirs = loads
    most = max(loads) if mend else mine
    assert abs(mine - theirs) <= stages
    if mend:
        for u in range(min(loads), most):
            if u >= mine:
                expect(u % stages, 1)
            else:
                flight.append(u % stages)
    last = range(max(0, most - stages), most)
    while flight and not all(passes(full[u % stages], u // stages & 1) for u in last):
        land(rng.randrange(len(flight)))
    return len(flight)


def test_no_copy_is_in_flight_behind_the_last_wait_of_a_pair():
    rng = random.Random(1)
    for _ in range(20000):
        assert pair(rng.randrange(2, 7), rng.randrange(0, 25), [rng.randrange(0, 30) for _ in range(3)], rng) == 0
    # the model shows the fault of waiting for the first CTA's loads alone
    assert any(pair(4, 20, [rng.randrange(0, 30) for _ in range(3)], rng, mend=False) for _ in range(2000))


def test_the_source_has_these_waits():
    text = open(SOURCE).read()
    # in the kernel of pairs, whose multiplies arrive at both CTAs' barriers, each loading warp waits for free stages behind its last load
    pairs = text[text.index("linear_f8_pair_kernel(const"):]
    assert len(re.findall(r"fine = fine && f8_stages_free\(q, ring, HIKONV_BAR\(empty, 0\)\);", pairs)) == 1
    # ... in the one of single CTAs the stages' arrivals are committed in front of the accumulators', which the adding warps wait for
    single = text[text.index("linear_f8_kernel(const"):text.index("linear_f8_pair_kernel(const")]
    assert single.index("tc_commit(HIKONV_BAR(empty, ring.stage));") < single.index("tc_commit(HIKONV_BAR(acc_full, acc.stage));")
    # the scales' copies are in no group: the wait behind them is the one that counts those
    scales = text[text.index("fine = bring_scales("):]
    assert scales.index('"cp.async.wait_all;"') < scales.index("if (q.splits > 1)")
    assert text.count("store_then_arrive_at(") == 2 and "HIKONV_BAR(peer, 0), 0)" in text
