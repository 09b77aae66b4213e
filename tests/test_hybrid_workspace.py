"""Workspaces of the operators of hybrid layers and the names in their refusals
(host only)."""
import pytest

import paper_2306_14320_amd as P
from test_seq_host import FAKE


def test_first_tokens_sums_of_short_sequences():
    """Only sequences longer than the window leave sums for the first tokens' keys:
    4096 of 16 tokens have none with a window of 1024, and tokens / 1025 of them at most."""
    def need(sequences, window, sinks):
        return P.im2win_window_attention_backward_workspace_bytes(
            P.im2win_window_desc(65536, sequences, 8, 8, 128, window, sinks, 1024, 1024, 1024, P.IM2WIN_BF16, 0.1))

    piece = 2 * 32 * 128 * 4 * 8          # dk and dv of 32 first tokens, in fp32, of all key heads
    delta = 65536 * 8 * 4
    assert need(4096, 1024, 0) == delta
    assert need(4096, 1024, 32) <= delta + (65536 // 128 + 65536 // 1025) * piece
    assert need(1, 1024, 32) >= delta + piece
    assert need(4096, 65536, 32) == delta


def test_refusals_name_the_argument():
    d = P.im2win_qk_desc(6, 2, 1, 8, 8, 16, 8, P.IM2WIN_BF16, 0, 1e-6)
    forward = ["q", "k", "wq", "wk", "positions", "freqs", "yq", "yk"]
    back = ["dyq", "dyk", "q", "k", "wq", "wk", "positions", "freqs", "dq", "dk", "dwq", "dwk", "workspace"]
    for names, call in ((forward, lambda a: P.im2win_qk_norm_rope(d, *a, 0)), (back, lambda a: P.im2win_qk_norm_rope_backward(d, *a, 1 << 40, 0))):
        for missing in names:
            with pytest.raises(P.Im2winError, match=r"\b%s is NULL" % missing):
                call([0 if n == missing else FAKE for n in names])
