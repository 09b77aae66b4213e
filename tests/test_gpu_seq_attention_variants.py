"""Window attention at the smallest sizes that reach the variants for large
problems: tiles of 128 keys for the keys' gradients (256 of them and more),
several tiles ahead on wide heads, many shares of a request's rows."""
import pytest
import torch

import paper_2306_14320_amd as P
import test_gpu_seq_attention as forward
import test_gpu_seq_attention_bwd as backward

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# tiles of 128 keys x key heads: at least 256
MANY = [
    (BF16, 128, 128, 64, 100, 3, (130, 1), None, 0), (F32, 86, 86, 32, 50, 2, [0, 100, 101, 300], None, 1), (BF16, 128, 64, 128, 150, 4, (512, 2), None, 0),
    (BF16, 128, 128, 80, 1000, 0, (256, 1), None, 0), (F32, 64, 64, 104, 33, 1, (512, 1), None, 0), (BF16, 64, 64, 184, 90, 5, (385, 1), None, 0),
    (F32, 64, 64, 160, 20, 0, (400, 1), None, 0), (BF16, 64, 64, 256, 129, 2, (400, 1), None, 0), (F32, 64, 64, 256, 64, 1, (390, 1), None, 0), (BF16, 130, 130, 32, 1, 0, (200, 1), None, 0),
]
LONG = [
    (F32, 2, 1, 128, 150, 2, (400, 1), None, 0), (BF16, 2, 1, 256, 200, 3, (500, 1), None, 0), (F32, 2, 2, 192, 100, 0, (300, 1), None, 0), (F32, 1, 1, 256, 250, 5, [0, 3, 420], None, 0),
    (BF16, 4, 1, 192, 300, 4, [0, 200, 520], [700, 20], 0), (F32, 3, 1, 128, 90, 3, [0, 150, 160], [200, 91], 0), (BF16, 3, 1, 128, 500, 1, (900, 1), None, 0), (BF16, 3, 1, 64, 400, 1, (900, 1), None, 0),
]


def _ids(cases):
    return ["%s-%dq%dk%d-w%d-s%d" % ((str(c[0])[6:],) + c[1:6]) for c in cases]


@pytest.mark.parametrize("case", MANY, ids=_ids(MANY))
def test_keys_in_tiles_of_128(case):
    rows = case[6][0] // case[6][1] if isinstance(case[6], tuple) else 0
    tiles = case[6][1] * -(-rows // 128) if rows else case[6][-1] // 128 + len(case[6]) - 1
    assert tiles * case[2] >= 256
    backward.test_backward(case)


@pytest.mark.parametrize("case", LONG + MANY[:2], ids=_ids(LONG + MANY[:2]))
def test_forward(case):
    forward.test_forward(case)


@pytest.mark.parametrize("case", [c for c in LONG if c[7] is None], ids=_ids([c for c in LONG if c[7] is None]))
def test_backward(case):
    backward.test_backward(case)


def test_step_of_many_shares():
    """More shares of a request's rows than a wave has lanes."""
    case = (BF16, 2, 1, 16, 9000, 4, [9003, 20000])
    q = torch.empty(2, 2, 16)
    need = P.im2win_window_attention_step_workspace_bytes(P.im2win_window_desc(2, 1, 2, 1, 16, 9000, 4, 32, 16, 16, P.IM2WIN_BF16, 0.25))
    assert need >= 2 * 2 * 65 * (q.shape[2] + 2) * 4
    forward.test_step(case)
