"""The query/key preparation on the GPU in place, at sizes of one, where a tensor's
strides of the indexes that do not move say nothing.  In place it gives what it
gives elsewhere, bit for bit."""
import pytest
import torch

from paper_2512_23068_amd import binding
from tests.test_gdr_gpu import BF16, DEV, F32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hk,L", [(1, 4, 2, 9), (3, 4, 1, 1), (2, 1, 1, 9), (1, 1, 1, 9), (1, 4, 2, 1), (1, 1, 1, 1),
                                       (2, 3, 2, 5)])
def test_in_place(dtype, B, Hq, Hk, L):
    print(f"case {dtype} {B} {Hq} {Hk} {L}", flush=True)
    gen = torch.Generator().manual_seed(1)
    rand = lambda h: torch.randn(B, h, L, 64, generator=gen).to(DEV, dtype)  # noqa: E731
    q, k, dq, dk = rand(Hq), rand(Hk), rand(Hq), rand(Hk)
    w = torch.rand(64, device=DEV)
    kw = dict(wq=w, wk=w, inv_freq=torch.rand(16, device=DEV))
    want, back = binding.qk_norm(q, k, **kw), binding.qk_norm_grads(q, k, dq, dk, **kw)
    x, y = dq.clone(), dk.clone()
    got = binding.qk_norm_grads(q, k, x, y, out=(x, y), **kw)
    assert got[0] is x and all(torch.equal(a, b) for a, b in zip(got, back))
    x, y = q.clone(), k.clone()
    got = binding.qk_norm_grads(x, y, dq, dk, out=(x, y), **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, back))
    x, y = q.clone(), k.clone()
    got = binding.qk_norm(x, y, out=(x, y), **kw)
    assert got[0] is x and all(torch.equal(a, b) for a, b in zip(got, want))
    # a slice of one index of a larger array
    x, y = (torch.stack([t, t], 2) for t in (q, k))
    got = binding.qk_norm(x[:, :, 1], y[:, :, 1], out=(x[:, :, 1], y[:, :, 1]), **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(x[:, :, 0], q)
