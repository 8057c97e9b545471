"""Refused sizes of attention are the library's error, with its code, whichever way a call takes."""
import pytest
import torch

from tests.test_gpu_attention import aj  # noqa: F401

pytestmark = pytest.mark.gpu

EMPTY, UNSUPPORTED_D = (1, 2), (3,)         # (an empty tensor has no address: a null pointer or a size that is refused, whichever is looked at first)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape,code", [((2, 30, 3, 20), UNSUPPORTED_D), ((2, 30, 3, 96), UNSUPPORTED_D), ((1, 1, 1, 7), UNSUPPORTED_D), ((2, 30, 0, 64), EMPTY), ((2, 0, 3, 64), EMPTY),
                                        ((0, 30, 3, 64), EMPTY)])
def test_sizes(aj, shape, code, causal):
    t = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    B, L, H, _ = shape
    for kw in (dict(fwd_only=True), dict(tq=t), dict(tq=t, tk=t, tv=t, return_mu=True)):
        with pytest.raises(aj.AttnJvpError) as e:
            aj.attention_jvp(t, t, t, causal=causal, **kw)
        assert e.value.code in code
    with pytest.raises(aj.AttnJvpError) as e:
        aj.attention_backward(t, t, t, t, t, torch.zeros(B, H, L, device="cuda"), causal=causal)
    assert e.value.code in code


def test_strides(aj):
    t = torch.zeros(2, 30, 3, 68, dtype=torch.bfloat16, device="cuda")[..., :64]
    for kw in (dict(), dict(causal=True)):
        with pytest.raises(ValueError, match="multiples of 8"):
            aj.attention_jvp(t, t, t, fwd_only=True, **kw)
