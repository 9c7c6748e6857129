"""The decoding example with less room than its tokens need: an error, where the loop would otherwise go on for good (a history that is full takes no
token, so no sequence ever has enough).  A batch that stands for a real one, on the CPU."""
import types

import pytest
import torch

from paper_2604_02047_b200 import shared_prompt


def _batch(own, room, nodes, positions=10000, shared=20):
    hist = torch.zeros(len(own), shared + room + nodes, dtype=torch.int32)
    steps = []

    def step(*args):
        steps.append(args)
        raise StopIteration                                    # (far enough: a step was made)

    return types.SimpleNamespace(S=len(own), B=nodes, shared=shared, room=room, hist=hist, step=step,
                                 hist_len=torch.tensor([shared + n - 1 for n in own], dtype=torch.int32),
                                 m=types.SimpleNamespace(vocab=50, rope=torch.zeros(positions, 128)))


@pytest.fixture(autouse=True)
def no_gpu(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self, *a, **k: self)


@pytest.mark.parametrize("own,room,nodes,tokens,positions", [([5, 9], 20, 4, 14, 10000), ([100], 50, 8, 1, 10000), ([5], 100, 8, 60, 90)])
def test_what_does_not_fit_is_an_error(own, room, nodes, tokens, positions):
    with pytest.raises(ValueError):
        shared_prompt.decode(_batch(own, room, nodes, positions), tokens)


def test_what_just_fits_is_decoded():
    with pytest.raises(StopIteration):
        shared_prompt.decode(_batch([5, 9], 20, 4), 13)
    with pytest.raises(StopIteration):
        shared_prompt.decode(_batch([5], 100, 8, positions=91), 60)


@pytest.mark.parametrize("sequences", [[], [[1, 2], []]])
def test_every_sequence_has_an_anchor(sequences):
    with pytest.raises(ValueError):
        shared_prompt.Batch(None, types.SimpleNamespace(), [1, 2, 3], sequences, 10, 4)
