"""A row that a cluster of CTAs shares while its gradient replaces its logits (``k_class_ring``, csrc/lrgd_class.cuh), replayed on the CPU under
random schedules.  Every CTA reads the target's logit, whichever CTA's stage holds it; a CTA that has the sums of all writes the gradient over its
stages.  A load takes its value some time after it was issued, and what needs the value waits for it: a sum that depends on the logit
goes out after the logit has been read, one that does not may go out before."""
import random

import pytest

LOGIT, GRADIENT = "logit", "gradient"


def cta(rank, C, world, depends):
    """Reads the target, sends its sum to all, waits for all sums, writes its part of the row, uses the target's logit."""
    load = {"value": None}
    world["loads"].append(load)
    yield
    if depends:
        while load["value"] is None:
            yield
    for peer in range(C):
        world["sums"][peer].add(rank)
        yield
    while len(world["sums"][rank]) < C:
        yield
    if world["owner"] == rank:
        world["memory"] = GRADIENT
    yield
    while load["value"] is None:
        yield
    world["used"].append(load["value"])


def replay(seed, depends):
    rng = random.Random(seed)
    C = rng.choice([2, 4, 8])
    world = {"loads": [], "sums": [set() for _ in range(C)], "owner": rng.randrange(C), "memory": LOGIT, "used": []}
    alive = [cta(r, C, world, depends) for r in range(C)]
    slow = rng.choice([0.02, 0.3])
    while alive:
        agent = rng.choice(alive)
        try:
            next(agent)
        except StopIteration:
            alive.remove(agent)
        for load in world["loads"]:
            if load["value"] is None and rng.random() < slow:
                load["value"] = world["memory"]
    assert len(world["used"]) == C
    return all(v == LOGIT for v in world["used"])


@pytest.mark.parametrize("seed", range(200))
def test_the_logit_is_read_before_it_is_replaced(seed):
    assert replay(seed, depends=True)


def test_the_replay_sees_a_sum_that_does_not_wait():
    assert not all(replay(seed, depends=False) for seed in range(200))
