"""Arguments of the binding's gated delta rule that need no GPU: which inputs are
read in place, and
numbers that the parameter block cannot hold."""
import pytest
import torch

from paper_2512_23068_amd import binding


def inputs(L=3, d=64):
    q, k, v = (torch.randn(1, 2, L, d) for _ in range(3))
    return q, k, v, -torch.rand(1, 2, L), torch.rand(1, 2, L)


def test_far_steps_are_copied():
    """Steps 2^24 bytes apart and more, which the kernels do not take."""
    q, k, v, g, beta = inputs()
    big = torch.zeros(3, 1 << 22)                       # 2^24 bytes a step
    near = torch.zeros(3, (1 << 22) - 4)
    for src, copied in ((big, True), (near, False)):
        far = src[:, :128].unflatten(1, (1, 2, 64)).permute(1, 2, 0, 3)
        far.copy_(q)
        c = binding._Gdr(far, k, v, g, beta, None, 0)
        assert (c.q.data_ptr() != far.data_ptr()) == copied and torch.equal(c.q, q)
        assert c.qs[2] * 4 < 1 << 24
        gate = src[:, :2].unflatten(1, (1, 2)).permute(1, 2, 0)
        gate.copy_(g)
        c = binding._Gdr(q, k, v, gate, beta, None, 0)
        assert (c.g.data_ptr() != gate.data_ptr()) == copied and torch.equal(c.g, g)


def test_segments_beyond_the_parameter_block():
    x = inputs()
    for seg in (1 << 31, -1 << 40):
        with pytest.raises(ValueError, match="seg_len"):
            binding._Gdr(*x, None, seg)
