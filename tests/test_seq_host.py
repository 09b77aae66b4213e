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
