"""The draft trees of the example of an agent's turn, without a GPU."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import __graft_entry__
    __graft_entry__.build()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import agent_turn
    return agent_turn


def test_tree_of_a_history(example):
    # after 7 came 1 2 (latest) and, before that, 3 4 5 6; 7 1 again earlier is no branch of its own
    history = [7, 1, 9, 7, 3, 4, 5, 6, 7, 1, 2, 7]
    tokens, parents = example.draft_tree(history)
    assert tokens == [7, 1, 2, 7, 3, 4, 5, 6]
    assert parents == [-1, 0, 1, 2, 0, 4, 5, 6]
    assert example.ancestor_masks(parents) == [1, 0b11, 0b111, 0b1111, 0b10001, 0b110001, 0b1110001, 0b11110001]


def test_a_token_seen_for_the_first_time_is_alone(example):
    assert example.draft_tree([5, 6, 7]) == ([7], [-1])
    assert example.ancestor_masks([-1]) == [1]


@pytest.mark.parametrize("answers,most,path", [
    ([1, 2, 7, 0, 0, 0, 0, 0], 9, [0, 1, 2, 3]),      # the first branch to its end
    ([3, 9, 9, 9, 4, 8, 0, 0], 9, [0, 4, 5]),         # the second one, for two tokens
    ([8, 2, 7, 0, 4, 5, 6, 0], 9, [0]),               # neither, whatever goes on below
    ([1, 2, 7, 0, 0, 0, 0, 0], 2, [0, 1]),
    ([1, 2, 7, 0, 0, 0, 0, 0], 1, [0]),
])
def test_accepted_path(example, answers, most, path):
    tokens, parents = [7, 1, 2, 7, 3, 4, 5, 6], [-1, 0, 1, 2, 0, 4, 5, 6]
    assert example.accepted(tokens, parents, answers, most) == path


def test_offsets(example):
    assert example.offsets([3, 0, 2]) == [0, 3, 3, 5]
