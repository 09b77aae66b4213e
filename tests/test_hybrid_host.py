"""Host-side tests of the operators of hybrid layers (no GPU needed): arguments
that the kernels could not run on are refused before any HIP call, by the C
entry points and by the tensor helpers."""
import pytest
import torch

import paper_2306_14320_amd as P
from test_seq_host import FAKE, _code

HUGE = 1 << 60


def rec_desc(**kw):
    d = dict(tokens=600, channels=8, sequences=3, ld_x=8, ld_r=8, ld_i=8, dtype=P.IM2WIN_BF16, c=8.0)
    d.update(kw)
    return P.im2win_recurrence_desc(**d)


# x r i lam starts init y final chunk_states workspace; dy x r i lam starts init d_final chunk_states dx dr di dlam d_init workspace
REC, REC_BWD, REC_STEP = [FAKE] * 4 + [0] + [FAKE] * 5, [FAKE] * 5 + [0] + [FAKE] * 9, [FAKE] * 4 + [0, FAKE, 4, FAKE]


def rec_calls(d):
    return [lambda: P.im2win_gated_recurrence(d, *REC, HUGE, 0), lambda: P.im2win_gated_recurrence_backward(d, *REC_BWD, HUGE, 0),
            lambda: P.im2win_gated_recurrence_step(d, *REC_STEP, 0)]


@pytest.mark.parametrize("field,value,code", [
    ("tokens", -1, "EINVAL"), ("channels", 0, "EINVAL"), ("ld_x", 7, "EINVAL"), ("ld_r", 7, "EINVAL"), ("ld_i", 0, "EINVAL"), ("dtype", 2, "EINVAL"),
    ("c", 0.0, "EINVAL"), ("c", -1.0, "EINVAL"), ("c", float("nan"), "EINVAL"), ("c", float("inf"), "EINVAL"), ("tokens", 1 << 31, "EOVERFLOW"),
    ("channels", 1 << 21, "EOVERFLOW"), ("ld_r", 1 << 29, "EOVERFLOW"),
])
def test_recurrence_bad_descriptor(field, value, code):
    d = rec_desc(**{field: value})
    for call in rec_calls(d) + [lambda: P.im2win_gated_recurrence_chunks(d), lambda: P.im2win_gated_recurrence_workspace_bytes(d),
                                lambda: P.im2win_gated_recurrence_backward_workspace_bytes(d)]:
        assert _code(call) == getattr(P, "IM2WIN_" + code)


def test_recurrence_pointers_sequences_and_workspace():
    d = rec_desc()
    need, back = P.im2win_gated_recurrence_workspace_bytes(d), P.im2win_gated_recurrence_backward_workspace_bytes(d)
    assert need > 0 and back > need and P.im2win_gated_recurrence_workspace_bytes(rec_desc(tokens=60)) == 0
    for sequences in (0, -1, 7):
        for call in rec_calls(rec_desc(sequences=sequences))[:2]:
            assert _code(call) == P.IM2WIN_EINVAL
    for i in (0, 1, 2, 3, 6, 9):
        assert _code(P.im2win_gated_recurrence, d, *[0 if j == i else v for j, v in enumerate(REC)], need, 0) == P.IM2WIN_ENULL
    for i in (0, 1, 2, 3, 5, 6, 7, 8, 9):
        assert _code(P.im2win_gated_recurrence, d, *[v + 1 if j == i else v for j, v in enumerate(REC)], need, 0) == P.IM2WIN_EALIGN
    assert _code(P.im2win_gated_recurrence, d, *REC, need - 1, 0) == P.IM2WIN_EWORKSPACE
    for i in (0, 1, 2, 3, 4, 9, 10, 11, 12, 14):
        assert _code(P.im2win_gated_recurrence_backward, d, *[0 if j == i else v for j, v in enumerate(REC_BWD)], back, 0) == P.IM2WIN_ENULL
    for i in set(range(15)) - {5}:
        assert _code(P.im2win_gated_recurrence_backward, d, *[v + 1 if j == i else v for j, v in enumerate(REC_BWD)], back, 0) == P.IM2WIN_EALIGN
    assert _code(P.im2win_gated_recurrence_backward, d, *REC_BWD, back - 1, 0) == P.IM2WIN_EWORKSPACE
    for i in (0, 1, 2, 3, 5, 7):
        assert _code(P.im2win_gated_recurrence_step, d, *[0 if j == i else v for j, v in enumerate(REC_STEP)], 0) == P.IM2WIN_ENULL
    assert _code(P.im2win_gated_recurrence_step, d, *REC_STEP[:6], -1, FAKE, 0) == P.IM2WIN_EINVAL


def test_recurrence_launches():
    """2^32 threads and more are refused before anything is launched."""
    d = rec_desc(tokens=1 << 30, channels=256, ld_x=256, ld_r=256, ld_i=256, sequences=1)
    for call in rec_calls(d):
        assert _code(call) == P.IM2WIN_EOVERFLOW
    d = rec_desc(tokens=0, sequences=1 << 30)
    assert _code(P.im2win_gated_recurrence, d, *REC, HUGE, 0) == P.IM2WIN_EOVERFLOW


def test_recurrence_helpers_refuse():
    x = torch.zeros(12, 8)
    with pytest.raises(ValueError):
        P.gated_recurrence_desc_for(x.t(), x.t(), x.t())
    with pytest.raises(ValueError):
        P.gated_recurrence_desc_for(x.half(), x.half(), x.half())
    with pytest.raises(ValueError):
        P.gated_recurrence_desc_for(x[0], x, x)
    wide = torch.zeros(12, 20)
    d = P.gated_recurrence_desc_for(x, wide[:, 1:9], wide[:, 10:18], 3, c=4.0)
    assert (d.tokens, d.channels, d.sequences, d.ld_x, d.ld_r, d.ld_i, d.dtype, d.c) == (12, 8, 3, 8, 20, 20, P.IM2WIN_F32, 4.0)
    for call in (lambda: P.gated_recurrence(x, x, x, x[0], d), lambda: P.gated_recurrence_backward(x, x, x, x, x[0], d), lambda: P.gated_recurrence_step(x, x, x, x[0], x, d)):
        with pytest.raises(ValueError):
            call()                           # no device tensors


def qk_desc(**kw):
    d = dict(tokens=5, q_heads=4, k_heads=2, head_dim=64, rot_dim=64, ld_q=256, ld_k=128, dtype=P.IM2WIN_BF16, interleaved=0, eps=1e-6)
    d.update(kw)
    return P.im2win_qk_desc(**d)


@pytest.mark.parametrize("field,value,code", [
    ("tokens", -1, "EINVAL"), ("q_heads", -1, "EINVAL"), ("k_heads", 1 << 20, "EINVAL"), ("head_dim", 0, "EINVAL"), ("head_dim", 63, "EINVAL"), ("head_dim", 514, "EINVAL"),
    ("rot_dim", 66, "EINVAL"), ("rot_dim", 31, "EINVAL"), ("rot_dim", -2, "EINVAL"), ("ld_q", 255, "EINVAL"), ("ld_k", 127, "EINVAL"), ("dtype", 7, "EINVAL"),
    ("eps", -1.0, "EINVAL"), ("eps", float("nan"), "EINVAL"), ("tokens", 1 << 31, "EOVERFLOW"), ("ld_q", 1 << 28, "EOVERFLOW"),
])
def test_qk_bad_descriptor(field, value, code):
    d = qk_desc(**{field: value})
    for call in (lambda: P.im2win_qk_norm_rope(d, *[FAKE] * 8, 0), lambda: P.im2win_qk_norm_rope_backward(d, *[FAKE] * 13, HUGE, 0),
                 lambda: P.im2win_qk_norm_rope_backward_workspace_bytes(d)):
        assert _code(call) == getattr(P, "IM2WIN_" + code)
    assert _code(P.im2win_qk_norm_rope, qk_desc(q_heads=0, k_heads=0), *[FAKE] * 8, 0) == P.IM2WIN_EINVAL


def test_qk_pointers_and_workspace():
    d = qk_desc()
    for i in range(8):
        assert _code(P.im2win_qk_norm_rope, d, *[0 if j == i else FAKE for j in range(8)], 0) == P.IM2WIN_ENULL
        assert _code(P.im2win_qk_norm_rope, d, *[FAKE + 1 if j == i else FAKE for j in range(8)], 0) == P.IM2WIN_EALIGN
    need = P.im2win_qk_norm_rope_backward_workspace_bytes(d)
    assert need >= 2 * 64 * 4
    for i in range(13):
        assert _code(P.im2win_qk_norm_rope_backward, d, *[0 if j == i else FAKE for j in range(13)], need, 0) == P.IM2WIN_ENULL
        assert _code(P.im2win_qk_norm_rope_backward, d, *[FAKE + 1 if j == i else FAKE for j in range(13)], need, 0) == P.IM2WIN_EALIGN
    assert _code(P.im2win_qk_norm_rope_backward, d, *[FAKE] * 13, need - 1, 0) == P.IM2WIN_EWORKSPACE
    assert _code(P.im2win_qk_norm_rope, qk_desc(tokens=1 << 30, ld_q=256), *[FAKE] * 8, 0) == P.IM2WIN_EOVERFLOW


def test_qk_helpers_refuse():
    q, k = torch.zeros(5, 4, 64), torch.zeros(5, 2, 64)
    for bad in ((q, k[:4]), (q, k[..., :32]), (q, k.bfloat16()), (q[:, 0], k[:, 0]), (q.transpose(1, 2), k.transpose(1, 2)), (q.half(), k.half())):
        with pytest.raises(ValueError):
            P.qk_norm_rope_desc_for(*bad)
    rows = torch.zeros(5, 600)
    d = P.qk_norm_rope_desc_for(rows[:, 3:259].unflatten(1, (4, 64)), k, rot_dim=32, interleaved=True)
    assert (d.tokens, d.q_heads, d.k_heads, d.head_dim, d.rot_dim, d.ld_q, d.ld_k, d.interleaved) == (5, 4, 2, 64, 32, 600, 128, 1)
    with pytest.raises(ValueError):
        P.qk_norm_rope(q, k, q[0, 0], q[0, 0], P.qk_norm_rope_desc_for(q, k))
    with pytest.raises(ValueError):
        P.qk_norm_rope_backward(q, k, q, k, q[0, 0], q[0, 0], P.qk_norm_rope_desc_for(q, k))


def win_desc(**kw):
    d = dict(tokens=600, sequences=3, q_heads=4, kv_heads=2, head_dim=64, window=100, sinks=4, ld_q=256, ld_k=128, ld_v=128, dtype=P.IM2WIN_BF16, scale=0.125)
    d.update(kw)
    return P.im2win_window_desc(**d)


# q k v starts k_cache v_cache slots(count) past slots y lse; q k v k_cache v_cache count past slots y workspace; dy q k v y lse starts dq dk dv workspace
ATT, ATT_STEP, ATT_BWD = [FAKE] * 3 + [0, FAKE, FAKE, 4] + [FAKE] * 4, [FAKE] * 5 + [4] + [FAKE] * 4, [FAKE] * 6 + [0] + [FAKE] * 4


def att_calls(d):
    return [lambda: P.im2win_window_attention(d, *ATT, 0), lambda: P.im2win_window_attention_step(d, *ATT_STEP, HUGE, 0),
            lambda: P.im2win_window_attention_backward(d, *ATT_BWD, HUGE, 0)]


@pytest.mark.parametrize("field,value,code", [
    ("tokens", -1, "EINVAL"), ("q_heads", 0, "EINVAL"), ("q_heads", 3, "EINVAL"), ("kv_heads", 0, "EINVAL"), ("kv_heads", 3, "EINVAL"), ("q_heads", 1 << 17, "EINVAL"),
    ("head_dim", 60, "EINVAL"), ("head_dim", 0, "EINVAL"), ("head_dim", 264, "EINVAL"), ("window", 0, "EINVAL"), ("sinks", -1, "EINVAL"), ("sinks", 33, "EINVAL"),
    ("ld_q", 255, "EINVAL"), ("ld_k", 127, "EINVAL"), ("ld_v", 1, "EINVAL"), ("dtype", 3, "EINVAL"), ("scale", 0.0, "EINVAL"), ("scale", -1.0, "EINVAL"), ("scale", float("nan"), "EINVAL"),
    ("tokens", 1 << 30, "EOVERFLOW"), ("window", 1 << 31, "EOVERFLOW"), ("ld_v", 1 << 24, "EOVERFLOW"), ("ld_q", 1 << 29, "EOVERFLOW"),
])
def test_attention_bad_descriptor(field, value, code):
    d = win_desc(**{field: value})
    for call in att_calls(d) + [lambda: P.im2win_window_attention_step_workspace_bytes(d), lambda: P.im2win_window_attention_backward_workspace_bytes(d)]:
        assert _code(call) == getattr(P, "IM2WIN_" + code)


def test_attention_pointers_sequences_and_workspace():
    d = win_desc()
    for sequences in (0, -1, 7):
        for call in (att_calls(win_desc(sequences=sequences))[0], att_calls(win_desc(sequences=sequences))[2]):
            assert _code(call) == P.IM2WIN_EINVAL
    for i in (0, 1, 2, 4, 5, 9):
        assert _code(P.im2win_window_attention, d, *[0 if j == i else v for j, v in enumerate(ATT)], 0) == P.IM2WIN_ENULL
    for i in (0, 1, 2, 4, 5, 7, 8, 9, 10):
        assert _code(P.im2win_window_attention, d, *[v + 1 if j == i else v for j, v in enumerate(ATT)], 0) == P.IM2WIN_EALIGN
    assert _code(P.im2win_window_attention, d, *ATT[:6], -1, *ATT[7:], 0) == P.IM2WIN_EINVAL
    for past, slots in ((FAKE, 0), (0, FAKE)):        # of a cache that is not there
        assert _code(P.im2win_window_attention, d, *ATT[:4], 0, 0, 0, past, slots, FAKE, FAKE, 0) == P.IM2WIN_EINVAL
    few = win_desc(tokens=2, window=4000)
    need = P.im2win_window_attention_step_workspace_bytes(few)
    assert need > 0 and P.im2win_window_attention_step_workspace_bytes(win_desc()) == 0
    for i in (0, 1, 2, 3, 4, 6, 8, 9):
        assert _code(P.im2win_window_attention_step, few, *[0 if j == i else v for j, v in enumerate(ATT_STEP)], need, 0) == P.IM2WIN_ENULL
    for i in (0, 1, 2, 3, 4, 6, 7, 8, 9):
        assert _code(P.im2win_window_attention_step, few, *[v + 1 if j == i else v for j, v in enumerate(ATT_STEP)], need, 0) == P.IM2WIN_EALIGN
    assert _code(P.im2win_window_attention_step, few, *ATT_STEP, need - 1, 0) == P.IM2WIN_EWORKSPACE
    assert _code(P.im2win_window_attention_step, few, *ATT_STEP[:5], -1, *ATT_STEP[6:], need, 0) == P.IM2WIN_EINVAL
    back = P.im2win_window_attention_backward_workspace_bytes(d)
    assert back >= 600 * 4 * 4
    for i in set(range(11)) - {6}:
        assert _code(P.im2win_window_attention_backward, d, *[0 if j == i else v for j, v in enumerate(ATT_BWD)], back, 0) == P.IM2WIN_ENULL
        assert _code(P.im2win_window_attention_backward, d, *[v + 1 if j == i else v for j, v in enumerate(ATT_BWD)], back, 0) == P.IM2WIN_EALIGN
    assert _code(P.im2win_window_attention_backward, d, *ATT_BWD, back - 1, 0) == P.IM2WIN_EWORKSPACE


def test_attention_launches():
    """2^32 threads and more are refused before anything is launched."""
    d = win_desc(tokens=1 << 29, sequences=1, kv_heads=4, ld_k=256, ld_v=256)
    for call in att_calls(d):
        assert _code(call) == P.IM2WIN_EOVERFLOW


def test_attention_helpers_refuse():
    q, k = torch.zeros(5, 4, 64), torch.zeros(5, 2, 64)
    for bad in ((q, k, k[:4]), (q, k[..., :32], k[..., :32]), (q, k.bfloat16(), k), (q.half(), k.half(), k.half()), (q.transpose(0, 2), k.transpose(0, 2), k.transpose(0, 2))):
        with pytest.raises(ValueError):
            P.window_attention_desc_for(*bad, 8)
    d = P.window_attention_desc_for(q, k, k, 8, 2)
    assert (d.tokens, d.sequences, d.q_heads, d.kv_heads, d.head_dim, d.window, d.sinks, d.ld_q, d.ld_k, d.ld_v, d.scale) == (5, 1, 4, 2, 64, 8, 2, 256, 128, 128, 0.125)
    lse = torch.zeros(5, 4)
    for call in (lambda: P.window_attention(q, k, k, d), lambda: P.window_attention_backward(q, q, k, k, q, lse, d),
                 lambda: P.window_attention_step(q, k, k, torch.zeros(5, 10, 2, 64), torch.zeros(5, 10, 2, 64), torch.zeros(5, dtype=torch.int32), d)):
        with pytest.raises(ValueError):
            call()                           # no device tensors
