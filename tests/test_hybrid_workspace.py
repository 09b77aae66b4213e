"""Workspaces of the operators of hybrid layers: what the queries ask for (host only)."""
import paper_2306_14320_amd as P


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
