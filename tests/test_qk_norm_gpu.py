"""The query/key preparation and its adjoint on the GPU against float64.

Tolerances (relative L2): f32 1e-6 (a sum of at most 512 squares, an inverse
root, three products and a rotation: about ten roundings of 2^-24, and the
sine and cosine a few more); weight gradients 1e-5 (long sums of f32); bf16 one
rounding of at most 2^-8."""
import pytest
import torch

from paper_2512_23068_amd import binding
from tests import gdr_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 1e-6, BF16: 2.0 ** -8 + 1e-6}
DEV = "cuda:0"


def inv(rot):
    return torch.pow(10000.0, -torch.arange(rot // 2) / (rot // 2)).float() if rot else None


CASES = [(1, 1, 1, 1, 8, 0, "l2", False, False), (2, 3, 1, 5, 64, 64, "rms", True, False),
         (2, 4, 2, 37, 72, 48, "rms", True, True), (1, 2, 2, 130, 128, 64, "l2", False, False),
         (3, 8, 8, 3, 256, 256, "rms", True, True), (1, 1, 5, 9, 512, 496, "rms", True, False),
         (64, 2, 1, 1, 96, 32, "none", False, False), (1, 16, 16, 700, 32, 16, "l2", True, True)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hk,L,d,rot,norm,weight,il", CASES)
def test_qk_norm_and_adjoint(dtype, B, Hq, Hk, L, d, rot, norm, weight, il):
    print(f"case {dtype} {B} {Hq} {Hk} {L} {d} {rot} {norm} {weight} {il}", flush=True)
    gen = torch.Generator().manual_seed(1)
    big = (torch.randn(B, L, (Hq + Hk) * d, generator=gen) * 2).to(dtype)
    q = big[..., :Hq * d].unflatten(-1, (Hq, d)).transpose(1, 2)
    k = big[..., Hq * d:].unflatten(-1, (Hk, d)).transpose(1, 2)
    bd = big.to(DEV)
    qd = bd[..., :Hq * d].unflatten(-1, (Hq, d)).transpose(1, 2)
    kd = bd[..., Hq * d:].unflatten(-1, (Hk, d)).transpose(1, 2)
    wq, wk = (1 + 0.3 * torch.randn(d, generator=gen), 1 + 0.3 * torch.randn(d, generator=gen)) if weight else (None,) * 2
    pos = torch.randint(0, 1 << 22, (B, 1), generator=gen) + torch.arange(L)
    f = inv(rot)
    kw = dict(wq=None if wq is None else wq.to(DEV), wk=None if wk is None else wk.to(DEV), norm=norm, eps=1e-5,
              positions=pos.to(DEV), inv_freq=None if f is None else f.to(DEV), interleaved=il)
    dq, dk = torch.randn(q.shape, generator=gen).to(dtype), torch.randn(k.shape, generator=gen).to(dtype)
    got = binding.qk_norm(qd, kd, **kw)
    back = binding.qk_norm_grads(qd, kd, dq.to(DEV), dk.to(DEV), **kw)
    torch.cuda.synchronize()
    ins = [x.double().clone().requires_grad_(True) for x in (q, k)]
    ws = [None if w is None else w.double().clone().requires_grad_(True) for w in (wq, wk)]
    want = [ref.qk_prep(x, w, norm, 1e-5, pos, f, il) for x, w in zip(ins, ws)]
    for g, w in zip(got, want):
        assert g.dtype == dtype and g.shape == w.shape
        e = ref.rel(g, w)
        print(f"out rel {e:.2e}", flush=True)
        assert e <= TOL[dtype]
    loss = sum((y * g.double()).sum() for y, g in zip(want, (dq, dk)))
    grads = torch.autograd.grad(loss, ins + [w for w in ws if w is not None])
    assert len(back) == len(grads)
    for i, (g, w) in enumerate(zip(back, grads)):
        e = ref.rel(g, w)
        print(f"grad {i} rel {e:.2e}", flush=True)
        assert e <= (TOL[dtype] if i < 2 else 1e-5)
    again = binding.qk_norm_grads(qd, kd, dq.to(DEV), dk.to(DEV), **kw)
    assert all(torch.equal(a, b) for a, b in zip(again, back))
    # positions as int32, in place
    kw["positions"] = kw["positions"].to(torch.int32)
    binding.qk_norm(qd, kd, out=(qd, kd), **kw)
    assert torch.equal(qd, got[0]) and torch.equal(kd, got[1])


def test_default_positions_and_rows():
    q, k = torch.randn(2, 2, 9, 32, device=DEV), torch.randn(2, 1, 9, 32, device=DEV)
    f = inv(32).to(DEV)
    a = binding.qk_norm(q, k, inv_freq=f)
    b = binding.qk_norm(q, k, inv_freq=f, positions=torch.arange(9, device=DEV))
    c = binding.qk_norm(q, k, inv_freq=f, positions=torch.arange(18, device=DEV)[::2].sub(torch.arange(9, device=DEV)))
    assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(a, b, c))


def test_empty():
    q, k = torch.randn(2, 2, 0, 32, device=DEV), torch.randn(2, 1, 0, 32, device=DEV)
    a = binding.qk_norm(q, k)
    assert a[0].shape == q.shape
    w = torch.ones(32, device=DEV)
    g = binding.qk_norm_grads(q, k, q, k, wq=w, wk=w)
    assert not g[2].any() and not g[3].any()
