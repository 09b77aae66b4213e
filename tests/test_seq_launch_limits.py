"""Host-side: sizes whose launch would have 2^32 threads or more are refused
before anything is launched (pointers that are never dereferenced)."""
import pytest

import paper_2306_14320_amd as P
from test_seq_host import FAKE, _code, conv_desc, scan_desc

HUGE = 1 << 60


def conv(**kw):
    kw.setdefault("sequences", 1)
    return conv_desc(**dict(dict(channels=8, ld_x=8), **kw))


def test_conv1d():
    # one wave for four rows, four a workgroup of 256 threads
    d = conv(tokens=1 << 28)
    assert _code(P.im2win_causal_conv1d, d, FAKE, FAKE, FAKE, 0, FAKE, FAKE, FAKE, 0) == P.IM2WIN_EOVERFLOW
    # final states of many sequences
    d = conv(tokens=64, sequences=1 << 27)
    assert _code(P.im2win_causal_conv1d, d, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0) == P.IM2WIN_EOVERFLOW


@pytest.mark.parametrize("d,starts", [
    (conv(tokens=1 << 30, channels=2049, ld_x=2049), 0),      # 2^22 stripes of 256 rows for each of 5 groups of channels
    (conv(tokens=64, sequences=1 << 22), FAKE),               # gradients of 3 * 2^22 rows of initial states, 512 threads each
], ids=["rows", "states"])
def test_conv1d_backward(d, starts):
    assert _code(P.im2win_causal_conv1d_backward, d, FAKE, FAKE, FAKE, FAKE, starts, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, HUGE, 0) == P.IM2WIN_EOVERFLOW


def test_single_tokens():
    assert _code(P.im2win_causal_conv1d_step, conv(tokens=1 << 26), FAKE, FAKE, FAKE, 0, FAKE, 4, FAKE, 0) == P.IM2WIN_EOVERFLOW
    assert _code(P.im2win_selective_scan_step, scan_desc(tokens=1 << 25), *[FAKE] * 8, 0, FAKE, 4, FAKE, 0) == P.IM2WIN_EOVERFLOW


@pytest.mark.parametrize("kw", [
    dict(tokens=1 << 30, states=16, groups=2),                # 2^24 chunks of 64 rows and more
    dict(tokens=1 << 28, states=16, groups=1, ld_b=16, ld_c=16),      # 2^32 values of dB
], ids=["chunks", "values"])
def test_scan_backward(kw):
    d = scan_desc(sequences=1, **kw)
    assert _code(P.im2win_selective_scan_backward, d, *[FAKE] * 9, 0, *[FAKE] * 12, HUGE, 0) == P.IM2WIN_EOVERFLOW
