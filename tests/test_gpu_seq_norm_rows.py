"""The norm's gradients of more rows than workgroups (1024), at every number of
waves that share a row: each workgroup walks two or three rows, its waves'
partial sums change places from one to the next, and dw adds up over them.
Bounds and checks are those of test_gpu_seq_norm.py."""
import pytest
import torch

import test_gpu_seq_norm as norm

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# up to 512 channels a wave holds a row, up to 8192 four waves, then sixteen
CASES = [(BF16, BF16, 3001, 200, 0, 0), (BF16, F32, 2500, 520, 0, 0), (F32, F32, 2311, 2049, 0, 0), (F32, BF16, 2100, 2500, 0, 0),
         (BF16, BF16, 2100, 4100, 0, 0), (F32, F32, 1100, 6001, 0, 0), (BF16, F32, 2060, 8200, 0, 0), (F32, F32, 2060, 8196, 0, 0), (BF16, BF16, 2060, 9001, 0, 0)]


@pytest.mark.parametrize("case", CASES, ids=["%s-%s-%dx%d" % (str(c[0])[6:], str(c[1])[6:], c[2], c[3]) for c in CASES])
def test_backward(case):
    norm.test_backward(case)
