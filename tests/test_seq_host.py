"""Host-side tests of the sequence operators (no GPU needed): arguments that
the kernels could not run on are refused before any HIP call, by the C entry
points and by the tensor helpers."""
import pytest
import torch

import paper_2306_14320_amd as P

FAKE = 0x10000   # never dereferenced: every call below is rejected before any HIP call


def _code(fn, *args):
    with pytest.raises(P.Im2winError) as ei:
        fn(*args)
    assert P.im2win_last_error() != ""
    return ei.value.code


def conv_desc(**kw):
    d = dict(tokens=12, channels=8, width=4, sequences=3, ld_x=8, dtype=P.IM2WIN_BF16, silu=1)
    d.update(kw)
    return P.im2win_conv1d_desc(**d)


def conv_calls(d):
    ok = 1 << 40
    return [lambda: P.im2win_causal_conv1d(d, FAKE, FAKE, FAKE, 0, FAKE, FAKE, FAKE, 0),
            lambda: P.im2win_causal_conv1d_backward(d, FAKE, FAKE, FAKE, FAKE, 0, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, ok, 0),
            lambda: P.im2win_causal_conv1d_step(d, FAKE, FAKE, FAKE, 0, FAKE, 4, FAKE, 0)]


@pytest.mark.parametrize("field,value,code", [
    ("tokens", -1, "EINVAL"), ("channels", 0, "EINVAL"), ("width", 0, "EINVAL"), ("width", 9, "EINVAL"), ("ld_x", 7, "EINVAL"),
    ("dtype", 5, "EINVAL"), ("tokens", 1 << 31, "EOVERFLOW"), ("channels", 1 << 21, "EOVERFLOW"), ("ld_x", 1 << 31, "EOVERFLOW"),
])
def test_conv1d_bad_descriptor(field, value, code):
    d = conv_desc(**{field: value})
    for call in conv_calls(d):
        assert _code(call) == getattr(P, "IM2WIN_" + code)
    assert _code(P.im2win_causal_conv1d_backward_workspace_bytes, d) == getattr(P, "IM2WIN_" + code)


@pytest.mark.parametrize("sequences", [0, -1, 5])   # 12 tokens are not 5 equal sequences
def test_conv1d_bad_sequences(sequences):
    for call in conv_calls(conv_desc(sequences=sequences))[:2]:
        assert _code(call) == P.IM2WIN_EINVAL


def test_conv1d_null_misaligned_and_short_workspace():
    d = conv_desc()
    fwd = [FAKE, FAKE, FAKE, 0, FAKE, FAKE, FAKE]
    for i in (0, 1, 5):
        assert _code(P.im2win_causal_conv1d, d, *[0 if j == i else v for j, v in enumerate(fwd)], 0) == P.IM2WIN_ENULL
    for i in (0, 1, 2, 4, 5, 6):
        assert _code(P.im2win_causal_conv1d, d, *[v + 1 if j == i else v for j, v in enumerate(fwd)], 0) == P.IM2WIN_EALIGN
    assert _code(P.im2win_causal_conv1d, d, FAKE, FAKE, FAKE, FAKE + 2, FAKE, FAKE, FAKE, 0) == P.IM2WIN_EALIGN
    need = P.im2win_causal_conv1d_backward_workspace_bytes(d)
    assert need >= 5 * 8 * 4
    bwd = [FAKE, FAKE, FAKE, FAKE, 0, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE]
    for i in (0, 1, 2, 7, 8, 11):
        assert _code(P.im2win_causal_conv1d_backward, d, *[0 if j == i else v for j, v in enumerate(bwd)], need, 0) == P.IM2WIN_ENULL
    assert _code(P.im2win_causal_conv1d_backward, d, *bwd, need - 1, 0) == P.IM2WIN_EWORKSPACE
    assert _code(P.im2win_causal_conv1d_backward, d, *bwd[:11], FAKE + 8, need, 0) == P.IM2WIN_EALIGN
    for i in (0, 1, 4, 6):
        step = [FAKE, FAKE, FAKE, 0, FAKE, 4, FAKE]
        step[i] = 0
        assert _code(P.im2win_causal_conv1d_step, d, *step, 0) == P.IM2WIN_ENULL
    assert _code(P.im2win_causal_conv1d_step, d, FAKE, FAKE, FAKE, 0, FAKE, -1, FAKE, 0) == P.IM2WIN_EINVAL


def test_conv1d_helpers_refuse():
    x, w = torch.zeros(12, 8), torch.zeros(8, 4)
    with pytest.raises(ValueError):
        P.causal_conv1d_desc_for(x, torch.zeros(9, 4))
    with pytest.raises(ValueError):
        P.causal_conv1d_desc_for(x.half(), w)
    with pytest.raises(ValueError):
        P.causal_conv1d_desc_for(x.t(), torch.zeros(12, 4))        # channels are not contiguous
    d = P.causal_conv1d_desc_for(torch.zeros(12, 20)[:, 3:11], w, 3, silu=False)
    assert (d.tokens, d.channels, d.width, d.sequences, d.ld_x, d.dtype, d.silu) == (12, 8, 4, 3, 20, P.IM2WIN_F32, 0)
    with pytest.raises(ValueError):
        P.causal_conv1d(x, w, P.causal_conv1d_desc_for(x, w))      # not a device tensor


def norm_desc(**kw):
    d = dict(tokens=4, channels=256, ld_x=256, block=0, dtype=P.IM2WIN_BF16, residual_dtype=P.IM2WIN_F32, eps=1e-5)
    d.update(kw)
    return P.im2win_norm_desc(**d)


@pytest.mark.parametrize("field,value,code", [
    ("tokens", -1, "EINVAL"), ("channels", 0, "EINVAL"), ("ld_x", 255, "EINVAL"), ("dtype", 2, "EINVAL"), ("residual_dtype", 2, "EINVAL"),
    ("eps", -1.0, "EINVAL"), ("eps", float("nan"), "EINVAL"), ("block", 8, "EINVAL"), ("block", 48, "EINVAL"), ("block", 1024, "EINVAL"),
    ("block", -64, "EINVAL"), ("tokens", 1 << 31, "EOVERFLOW"), ("channels", 16385, "EOVERFLOW"),
])
def test_norm_bad_descriptor(field, value, code):
    d = norm_desc(**{field: value})
    for call in (lambda: P.im2win_add_rms_norm(d, FAKE, FAKE, FAKE, FAKE, FAKE, 0),
                 lambda: P.im2win_add_rms_norm_fp8(d, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0),
                 lambda: P.im2win_add_rms_norm_backward(d, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, 0)):
        assert _code(call) == getattr(P, "IM2WIN_" + code)


def test_norm_null_misaligned_and_short_workspace():
    d = norm_desc()
    assert _code(P.im2win_add_rms_norm, norm_desc(block=128), FAKE, FAKE, FAKE, FAKE, FAKE, 0) == P.IM2WIN_EINVAL
    assert _code(P.im2win_add_rms_norm_fp8, norm_desc(channels=320, ld_x=320, block=128), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0) == P.IM2WIN_EINVAL
    for i in (0, 2, 3, 4):     # h is needed beside a residual
        assert _code(P.im2win_add_rms_norm, d, *[0 if j == i else FAKE for j in range(5)], 0) == P.IM2WIN_ENULL
    for i in (0, 2, 3, 4, 5):
        assert _code(P.im2win_add_rms_norm_fp8, d, *[0 if j == i else FAKE for j in range(6)], 0) == P.IM2WIN_ENULL
    for i in range(5):
        assert _code(P.im2win_add_rms_norm, d, *[FAKE + 1 if j == i else FAKE for j in range(5)], 0) == P.IM2WIN_EALIGN
    need = P.im2win_add_rms_norm_backward_workspace_bytes(d)
    assert need == 4 * 256 * 4
    for i in (0, 1, 2, 4, 5, 6):
        assert _code(P.im2win_add_rms_norm_backward, d, *[0 if j == i else FAKE for j in range(7)], need, 0) == P.IM2WIN_ENULL
    assert _code(P.im2win_add_rms_norm_backward, d, *[FAKE] * 7, need - 1, 0) == P.IM2WIN_EWORKSPACE
    with pytest.raises(ValueError):
        P.rms_norm_desc_for(4, 8, torch.float16)
    with pytest.raises(ValueError):
        P.add_rms_norm(torch.zeros(4, 8), torch.zeros(8), P.rms_norm_desc_for(4, 8, torch.float32))


def scan_desc(**kw):
    d = dict(tokens=12, channels=8, states=16, groups=2, sequences=3, ld_x=8, ld_dt=8, ld_z=8, ld_b=32, ld_c=32, dtype=P.IM2WIN_F32, softplus=1)
    d.update(kw)
    return P.im2win_scan_desc(**d)


def scan_calls(d):
    ok = 1 << 50
    return [lambda: P.im2win_selective_scan(d, *[FAKE] * 8, 0, FAKE, FAKE, FAKE, FAKE, ok, 0),
            lambda: P.im2win_selective_scan_step(d, *[FAKE] * 8, 0, FAKE, 4, FAKE, 0)]


@pytest.mark.parametrize("field,value,code", [
    ("tokens", -1, "EINVAL"), ("channels", 0, "EINVAL"), ("states", 0, "EINVAL"), ("states", 129, "EINVAL"), ("groups", 0, "EINVAL"),
    ("groups", 3, "EINVAL"), ("ld_x", 7, "EINVAL"), ("ld_dt", 7, "EINVAL"), ("ld_z", 0, "EINVAL"), ("ld_b", 31, "EINVAL"), ("ld_c", 16, "EINVAL"),
    ("dtype", 3, "EINVAL"), ("tokens", 1 << 31, "EOVERFLOW"), ("channels", 1 << 21, "EOVERFLOW"), ("ld_b", 1 << 31, "EOVERFLOW"),
])
def test_scan_bad_descriptor(field, value, code):
    d = scan_desc(**{field: value})
    for call in scan_calls(d):
        assert _code(call) == getattr(P, "IM2WIN_" + code)
    assert _code(P.im2win_selective_scan_workspace_bytes, d) == getattr(P, "IM2WIN_" + code)


def test_scan_null_misaligned_and_short_workspace():
    d = scan_desc(tokens=600, channels=16)
    d.ld_x = d.ld_dt = d.ld_z = 16
    need = P.im2win_selective_scan_workspace_bytes(d)
    assert need > 0
    good = [FAKE] * 8 + [0, FAKE, FAKE, FAKE, FAKE]
    for i in (0, 1, 2, 3, 4, 10, 12):
        assert _code(P.im2win_selective_scan, d, *[0 if j == i else v for j, v in enumerate(good)], need, 0) == P.IM2WIN_ENULL
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 9, 10, 11, 12):
        assert _code(P.im2win_selective_scan, d, *[v + 2 if j == i else v for j, v in enumerate(good)], need, 0) == P.IM2WIN_EALIGN
    assert _code(P.im2win_selective_scan, d, *good, need - 1, 0) == P.IM2WIN_EWORKSPACE
    for bad in (0, -2, 7):
        d.sequences = bad
        assert _code(P.im2win_selective_scan, d, *good, need, 0) == P.IM2WIN_EINVAL
    step = [FAKE] * 8 + [0, FAKE, 4, FAKE]
    for i in (0, 1, 2, 3, 4, 9, 11):
        assert _code(P.im2win_selective_scan_step, d, *[0 if j == i else v for j, v in enumerate(step)], 0) == P.IM2WIN_ENULL
    assert _code(P.im2win_selective_scan_step, d, *step[:10], -1, FAKE, 0) == P.IM2WIN_EINVAL
    with pytest.raises(ValueError):
        P.selective_scan_desc_for(torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros(8, 3), torch.zeros(4, 1, 4), torch.zeros(4, 1, 4))


def test_scan_workspace_covers_every_plan():
    """No workspace where one chunk holds all rows; otherwise a state for each
    chunk, channel and padded state, at chunks of 16 rows or more."""
    for tokens, seqs, channels, n, groups in [(64, 1, 2048, 16, 1), (1, 1, 1, 1, 1), (8192, 1, 2048, 16, 1), (16384, 8, 2048, 16, 1), (3001, 17, 777, 24, 3), (100000, 7, 33, 128, 1)]:
        d = scan_desc(tokens=tokens, channels=channels, states=n, groups=groups, sequences=seqs, ld_x=channels, ld_dt=channels, ld_z=channels, ld_b=groups * n, ld_c=groups * n)
        need = P.im2win_selective_scan_workspace_bytes(d)
        assert (need == 0) == (tokens <= 64)
        assert need <= (tokens / 16 + 1) * channels * (4 * 132) + tokens + 4096


def test_scan_backward_refuses():
    d = scan_desc(tokens=600, channels=16, ld_x=16, ld_dt=16, ld_z=16)
    need = P.im2win_selective_scan_backward_workspace_bytes(d)
    # dy x dt A B C D z dt_bias starts init d_final dx ddt dA dB dC dD dz ddt_bias d_init workspace
    good = [FAKE] * 9 + [0] + [FAKE] * 12
    for i in (0, 1, 2, 3, 4, 5, 12, 13, 14, 15, 16, 18, 21):
        assert _code(P.im2win_selective_scan_backward, d, *[0 if j == i else v for j, v in enumerate(good)], need, 0) == P.IM2WIN_ENULL
    for i in set(range(22)) - {9}:
        assert _code(P.im2win_selective_scan_backward, d, *[v + 2 if j == i else v for j, v in enumerate(good)], need, 0) == P.IM2WIN_EALIGN
    assert _code(P.im2win_selective_scan_backward, d, *good, need - 1, 0) == P.IM2WIN_EWORKSPACE
    for field, value in (("states", 129), ("groups", 5), ("sequences", 7), ("dtype", 9), ("tokens", -4)):
        bad = scan_desc(tokens=600, channels=16, ld_x=16, ld_dt=16, ld_z=16)
        setattr(bad, field, value)
        assert _code(P.im2win_selective_scan_backward, bad, *good, need, 0) == P.IM2WIN_EINVAL
        if field != "sequences":     # with seq_starts 7 sequences may share 600 rows
            assert _code(P.im2win_selective_scan_backward_workspace_bytes, bad) == P.IM2WIN_EINVAL
