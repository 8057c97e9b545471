"""Argument checks of the fused gate + residual + norm + modulation step (no GPU: nothing gets past them here), and the
64-bit statement that the GPU tests compare with, pinned by hand and by differences."""
import ctypes

import pytest
import torch

from tests import adaln_ref

A, STEP = 0x7F0000000000, 1 << 32        # fake, aligned, well separated addresses


@pytest.fixture(scope="module")
def aj():
    from paper_2510_08431_b200 import build
    build.build_library()
    import paper_2510_08431_b200 as aj
    aj.load()
    return aj


def args(aj, **kw):
    a = dict(x=A, h=A + STEP, gate=A + 2 * STEP, scale=A + 3 * STEP, shift=A + 4 * STEP, weight=A + 5 * STEP,
             post_weight=A + 6 * STEP, tx=A + 7 * STEP, th=A + 8 * STEP, tgate=A + 9 * STEP, tscale=A + 10 * STEP,
             tshift=A + 11 * STEP, gate_stride=512, scale_stride=512, shift_stride=512, tgate_stride=512,
             tscale_stride=512, tshift_stride=512, B=2, L=10, C=512, x_dtype=0, norm=1, post_norm=0, eps=1e-6)
    a.update(kw)
    return aj.AdaLNArgs(**a)


OUT = [A + 20 * STEP, A + 21 * STEP, A + 22 * STEP, A + 23 * STEP]

BAD_COMMON = [
    (dict(B=0), 2), (dict(L=0), 2), (dict(C=0), 2), (dict(C=12), 2), (dict(C=8200), 2), (dict(B=1 << 30, L=1 << 30), 2),
    (dict(x_dtype=2), 5), (dict(norm=3), 5), (dict(post_norm=-1), 5), (dict(eps=-1.0), 6), (dict(eps=float("nan")), 6),
    (dict(x=None), 1), (dict(x=A + 8), 4), (dict(h=A + STEP + 2), 4), (dict(gate=A + 2 * STEP + 2), 4),
    (dict(gate_stride=-1), 2),
]


@pytest.mark.parametrize("kw,code", BAD_COMMON)
def test_both_directions_refuse(aj, kw, code):
    assert aj.attn_jvp_adaln_fwd(args(aj, **kw), *OUT, None) == code
    assert aj.attn_jvp_adaln_bwd(args(aj, **kw), A + 24 * STEP, A + 25 * STEP, *OUT, None, None, None, A + 30 * STEP,
                                 1 << 30, None) == code


def test_forward_refuses(aj):
    f = aj.attn_jvp_adaln_fwd
    o = OUT
    assert f(args(aj), None, o[1], None, None, None) == 1              # h without x_new
    assert f(args(aj, h=None), o[0], o[1], None, None, None) == 1      # x_new without h
    assert f(args(aj), o[0], None, None, None, None) == 1              # a norm without y
    assert f(args(aj, norm=0), o[0], o[1], None, None, None) == 1      # y without a norm
    assert f(args(aj), o[0], o[1], o[2], None, None) == 1              # one of the two tangents
    assert f(args(aj, tx=None), *o, None) == 1
    assert f(args(aj, th=None), *o, None) == 1
    assert f(args(aj, h=None, norm=0), None, None, None, None, None) == 1
    assert f(args(aj), o[0], A + 16, o[2], o[3], None) == 7            # y over x
    assert f(args(aj), o[0], o[0] + 64, o[2], o[3], None) == 7         # y over x_new
    assert f(args(aj), o[0], o[1], o[2], A + 3 * STEP, None) == 7      # ty over the modulation
    assert f(args(aj), o[0] + 2, o[1], o[2], o[3], None) == 4
    assert _null(aj) == 1


def _null(aj):
    lib = aj.load()
    return lib.attn_jvp_adaln_fwd(None, None, None, None, None, None)


def test_backward_refuses(aj):
    def f(a, dxn=A + 24 * STEP, dy=A + 25 * STEP, dx=OUT[0], dh=OUT[1], ws=A + 30 * STEP, n=1 << 30):
        return aj.attn_jvp_adaln_bwd(a, dxn, dy, dx, dh, OUT[2], OUT[3], None, None, None, ws, n, None)

    need = aj.attn_jvp_adaln_bwd_workspace_bytes(2, 10, 512)
    assert need > 0 and need % 16 == 0
    assert f(args(aj), dx=None) == 1
    assert f(args(aj), dh=None) == 1
    assert f(args(aj, h=None)) == 1
    assert f(args(aj, norm=0)) == 1                                     # dy without a y
    assert f(args(aj), ws=None) == 1
    assert f(args(aj), n=need - 1) == 12
    assert f(args(aj), ws=A + 30 * STEP + 4) == 4
    assert f(args(aj), ws=OUT[0]) == 7
    assert f(args(aj), dx=A + 25 * STEP) == 7                           # dx over dy


def test_good_arguments_stop_at_the_device(aj):
    if torch.cuda.is_available():
        pytest.skip("would enqueue work on fake addresses")
    assert aj.attn_jvp_adaln_fwd(args(aj), *OUT, None) in (8, 9)
    assert aj.attn_jvp_adaln_fwd(args(aj, gate_stride=0, gate=None, tgate=None), OUT[0], OUT[1], None, None, None) in (8, 9)
    need = aj.attn_jvp_adaln_bwd_workspace_bytes(2, 10, 512)
    assert aj.attn_jvp_adaln_bwd(args(aj), None, A + 25 * STEP, OUT[0], OUT[1], None, None, None, None, None, A + 30 * STEP,
                                 need, None) in (8, 9)


def test_workspace_sizes(aj):
    size = aj.attn_jvp_adaln_bwd_workspace_bytes
    for B, L, C in ((1, 1, 8), (1, 32760, 5120), (3, 1000, 1536), (500, 3, 64), (1, 7, 8192)):
        n = size(B, L, C)
        assert n % (12 * C) == 0 and B <= n // (12 * C) <= B * L        # three sums per CTA, at least one CTA per batch
    assert size(0, 1, 8) == size(1, 1, 12) == size(1, 1, 9000) == 0


def test_python_layer_refuses_cpu_and_mismatched_tensors(aj):
    x = torch.zeros(1, 4, 64)
    with pytest.raises(ValueError):
        aj.adaln_jvp(x)
    with pytest.raises(ValueError):
        aj.adaln_backward(x, None, x)


def test_argument_struct_matches_the_header(aj):
    """Twelve pointers, six strides, six ints, one float, padded to 8 bytes."""
    assert ctypes.sizeof(aj.AdaLNArgs) == 12 * 8 + 6 * 8 + 6 * 4 + 4 + 4


def test_statement_by_hand():
    x = torch.tensor([[[1.0, 3.0]]], dtype=torch.float64)
    h = torch.tensor([[[3.0, 4.0]]], dtype=torch.float64)
    gate = torch.tensor([[2.0, 0.0]], dtype=torch.float64)
    # rms of (3, 4) is sqrt(12.5); x' = (1 + 6 / sqrt(12.5), 3); layer norm of two values a < b is (-1, 1) at eps = 0
    xn, y = adaln_ref.step(x, h, gate, None, None, None, None, "layer", "rms", 0.0)
    a = 1 + 6 / 12.5 ** 0.5
    assert torch.allclose(xn, torch.tensor([[[a, 3.0]]], dtype=torch.float64), atol=1e-14)
    assert torch.allclose(y, torch.tensor([[[-1.0, 1.0]]], dtype=torch.float64), atol=1e-12)
    scale, shift = torch.tensor([[1.0, -1.0]], dtype=torch.float64), torch.tensor([[0.5, 0.25]], dtype=torch.float64)
    w = torch.tensor([3.0, 5.0], dtype=torch.float64)
    _, y = adaln_ref.step(x, None, None, scale, shift, w, None, "layer", None, 0.0)
    assert torch.allclose(y, torch.tensor([[[-5.5, 0.25]]], dtype=torch.float64), atol=1e-12)
