"""The example's task and its arguments, without a GPU."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import train_block


def test_a_sequence_asks_for_nothing_that_it_has_not_seen():
    tokens = torch.tensor([[3, 1, 4, 1], [5, 9, 2, 6]])
    assert train_block.labels(tokens, 11).tolist() == [[-100, 18 % 11, 8, 23 % 11], [-100, 28 % 11, 48 % 11, 13 % 11]]
    assert train_block.labels(tokens[0], 11).tolist() == [18 % 11, 8, 23 % 11, 8]           # without sequences: of the token itself


@pytest.mark.parametrize("sequence", [1, 7, 1024, -32])
def test_sequences_that_do_not_fill_the_batch_are_refused(sequence):
    with pytest.raises(ValueError, match="sequence"):
        train_block.train(steps=1, batch=512, sequence=sequence)
