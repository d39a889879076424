"""The example's comparison covers what it says: every step up to the first half of the decode steps, replayed ones too."""
import pytest

from tests.test_paged_serving import example  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("graph", [False, True])
def test_all_compared_steps_are_near_plain_attention(example, graph):  # noqa: F811
    """Half a step of a group's largest over 127 for keys and values, 0.7 % together (as in test_paged_serving), twice that for a draw.  24 decode
    steps fill a page of 16 at least once in every sequence."""
    lines = []
    worst = example.run(layers=2, bits=8, prompts=(150, 37, 1, 90), steps=50, chunk=64, graph=graph, say=lines.append)
    assert len(lines) == 4 and 0.0 < worst < 2 * 0.007


def test_a_replay_that_does_nothing_is_seen(example, monkeypatch):  # noqa: F811
    import torch
    replay, made = torch.cuda.CUDAGraph.replay, []

    def first_only(graph):
        made.append(graph)
        if len(made) == 1:
            replay(graph)
    monkeypatch.setattr(torch.cuda.CUDAGraph, "replay", first_only)
    worst = example.run(layers=2, bits=8, prompts=(150, 37, 1, 90), steps=12, chunk=64, graph=True, say=lambda line: None)
    assert len(made) > 2 and worst > 2 * 0.007
