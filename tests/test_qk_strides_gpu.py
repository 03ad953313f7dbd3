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


def test_many_short_rows():
    """More steps than a launch has blocks for: of 2^24 + 1 blocks of 256 threads, eight
    steps each, one would run (20 s; in as many blocks as fit it is 40 ms).  Of each of 2^27 + 5 rows of eight bf16, against the rule on a sample and
    on the last rows (one rounding, 2^-8; the sums of eight are far below it)."""
    L = (1 << 27) + 5
    q = torch.empty(1, 1, L, 8, device=DEV, dtype=BF16).uniform_(0.5, 2.0)
    k = torch.empty(1, 1, 1, 8, device=DEV, dtype=BF16).uniform_(0.5, 2.0).expand(1, 1, L, 8)
    out = torch.zeros(2, 1, 1, L, 8, device=DEV, dtype=BF16)
    k = k.clone(memory_format=torch.contiguous_format)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    binding.qk_norm(q, k, norm="l2", eps=0.0, out=(out[0], out[1]))
    end.record()
    torch.cuda.synchronize()
    print(f"{begin.elapsed_time(end):.1f} ms", flush=True)
    assert begin.elapsed_time(end) < 1000.0
    at = torch.cat([torch.randint(0, L, (100000,), device=DEV), torch.arange(L - 2000, L, device=DEV)])
    for x, y in ((q, out[0]), (k, out[1])):
        x, y = x[0, 0, at].double(), y[0, 0, at].double()
        want = x / x.norm(dim=-1, keepdim=True)
        assert bool(((y - want).abs() <= 2.0 ** -8 * want).all())
    assert int((out == 0).sum()) == 0
