"""What the layers hand to the library as an output's gradient (no GPU): contiguous and 16-byte aligned, copied only where it is not."""
import torch

from paper_2510_08431_b200.layers import _whole


def test_gradients_are_made_whole():
    base = torch.randn(4000).bfloat16()
    assert base.data_ptr() % 16 == 0
    assert _whole(None) is None
    aligned = base[8:8 + 1024].view(2, 4, 2, 64)
    assert _whole(aligned).data_ptr() == aligned.data_ptr()
    for start in (1, 3, 7):
        g = base[start:start + 1024].view(2, 4, 2, 64)
        assert g.is_contiguous() and g.data_ptr() % 16 != 0
        got = _whole(g)
        assert got.data_ptr() % 16 == 0 and got.is_contiguous() and torch.equal(got, g)
    for g in (base[:1].expand(2, 4, 2, 64), base[:1024].view(2, 2, 4, 64).transpose(1, 2)):
        got = _whole(g)
        assert got.is_contiguous() and got.data_ptr() % 16 == 0 and torch.equal(got, g)
