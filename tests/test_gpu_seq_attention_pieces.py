"""Gradients of the first tokens' keys over batches in which few of many sequences
are longer than the window: only those have partial sums."""
import random

import pytest
import torch

import test_gpu_seq_attention_bwd as backward

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _starts(seed, short, count, long):
    """Lengths up to `short`, empty ones among them, and the long ones between them."""
    r = random.Random(seed)
    n = [r.choice([0, 0, 1, short, r.randint(0, short)]) for _ in range(count)]
    for length in long:
        n[r.randrange(count)] = length
    starts = [r.randint(0, 3)]
    for v in n:
        starts.append(starts[-1] + v)
    return starts


CASES = [
    (F32, 2, 1, 16, 5, 3, _starts(1, 5, 200, [6, 7, 140, 300, 129, 6]), None, 0), (BF16, 4, 2, 64, 20, 4, _starts(2, 20, 90, [21, 150, 149, 400]), None, 1),
    (F32, 1, 1, 32, 1, 2, _starts(3, 1, 300, [2, 3, 2, 260, 128, 127]), None, 0), (BF16, 2, 2, 128, 100, 32, _starts(4, 90, 8, [101, 700]), None, 0),
    (F32, 2, 1, 16, 4, 1, [0] + [5 * i for i in range(70)], None, 0),                       # all of them one token longer
    (BF16, 64, 64, 64, 30, 2, _starts(5, 30, 40, [31, 200, 60]), None, 0),                  # tiles of 128 keys
]


@pytest.mark.parametrize("case", CASES, ids=range(len(CASES)))
def test_backward(case):
    backward.test_backward(case)
