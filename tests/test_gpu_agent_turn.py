"""The example of an agent's turns: prompt attention, draft verification and 8-bit images together."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# Logits have a deviation of sqrt(512) = 22.6. Two ways of computing one differ by the roundings to
# bf16 of a few products and of the cached rows, about 1% of that each way; four deviations of the
# difference of two such logits are 1.3.
MARGIN = 2.0


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import agent_turn
    return agent_turn


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("cold_int8", [True, False])
def test_drafts_and_single_tokens_answer_alike(cuda_dev, example, cold_int8, bt):
    size = dict(sessions=5, turns=3, context=150, tokens=40, seed=3, vocab=200, block_tokens=bt, cold_int8=cold_int8)
    drafted, single = example.run(drafts=True, **size), example.run(drafts=False, **size)
    assert single.steps == single.generated
    assert drafted.generated == single.generated and drafted.steps < drafted.generated
    for a, b in zip(drafted.sessions, single.sessions):
        assert len(a.history) == len(b.history) and a.cached == b.cached == len(a.history) - 1
        given = [i for i, (x, y) in enumerate(zip(a.history, b.history)) if x != y]
        if given:   # the first token that differs: a tie of the logits
            n = generated_before(a, size, given[0])
            assert a.gaps[n] < MARGIN and b.gaps[n] < MARGIN
    for agent in (drafted, single):
        stats = agent.pool.stats()
        token = agent.model.L * 2 * agent.model.Hkv * (129 if cold_int8 else 256)
        assert stats["bytes_packed"] == token * sum(s.cached for s in agent.sessions)
        agent.pool.close()


def generated_before(session, size, at):
    """How many generated tokens come before place `at`: each turn ends with `tokens` of them."""
    ends, place = [], 0
    for n in session.contexts:
        ends.append((place + n, place + n + size["tokens"]))
        place += n + size["tokens"]
    return sum(max(0, min(at, hi) - lo) for lo, hi in ends)
