"""Roundings on the GPU: bf16 outputs of the gated delta rule, its gradients under
strong decays, and the rotation of queries and keys.

A bf16 input is the first of its f32 value's three parts and the other two are
zero, so the scan of bf16 inputs and that of the same values in f32 add the same
products in the same order: the bf16 output is the f32 output rounded once, bit
for bit, and the states are the same."""
import pytest
import torch

from paper_2512_23068_amd import binding
from tests.test_gdr_gpu import BF16, DEV, F32, TOL, check, make
from tests.test_gdr_grads_gpu import compare, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Hk,Hv,L,dk,dv,seg", [
    (1, 1, 2, 100, 64, 64, -1), (2, 2, 4, 333, 128, 128, -1), (1, 2, 2, 500, 128, 72, 128), (20, 4, 16, 65, 64, 32, -1),
    (12, 2, 6, 70, 128, 128, -1), (1, 1, 1, 64, 24, 40, -1)])
def test_scan_rounds_its_output_once(B, Hk, Hv, L, dk, dv, seg):
    print(f"case {B} {Hk} {Hv} {L} {dk} {dv} {seg}", flush=True)
    _, d = make(B, Hk, Hv, L, dk, dv, BF16, seed=71)
    S0 = torch.randn(B, Hv, dk, dv, generator=torch.Generator().manual_seed(9)).to(DEV)
    o, S = binding.gdr_scan(*d, S_in=S0, return_state=True, seg_len=seg)
    o32, S32 = binding.gdr_scan(*[x.float() for x in d], S_in=S0, return_state=True, seg_len=seg)
    differ = int((o != o32.to(BF16)).sum())
    print(f"{differ} of {o.numel()} outputs differ", flush=True)
    assert torch.equal(S, S32)
    assert differ == 0


@pytest.mark.parametrize("il", [False, True])
def test_rotation_is_rounded_once(il):
    """Pairs (1, 0) and (0, 1) without a norm: f32 outputs are the cosine and sine of
    position * inv_freq.  That product is exact in f64 here (20 and 24 bits); its turn
    has two roundings of 2^-53 relative, and sine and cosine one more of an angle up to
    2 pi.  Rounded to f32 once they are off by 2^-24 relative beside that."""
    d, L = 64, 4096
    half = d // 2
    gen = torch.Generator().manual_seed(3)
    pos = torch.randint(0, 1 << 20, (L,), generator=gen)
    freq = torch.exp(-6 * torch.rand(half, generator=gen)).float()
    q, k = torch.zeros(1, 1, L, d), torch.zeros(1, 1, L, d)
    a, b = (slice(0, d, 2), slice(1, d, 2)) if il else (slice(0, half), slice(half, d))
    q[..., a], k[..., b] = 1.0, 1.0
    y, z = binding.qk_norm(q.to(DEV), k.to(DEV), norm="none", inv_freq=freq.to(DEV), positions=pos.to(DEV), interleaved=il)
    ang = pos.double()[:, None] * freq.double()
    for got, want in ((y[..., a], ang.cos()), (y[..., b], ang.sin()), (z[..., a], -ang.sin()), (z[..., b], ang.cos())):
        err = (got[0, 0].double().cpu() - want).abs()
        worst = float((err / want.abs()).max())
        print(f"worst {worst * 2 ** 24:.3f} x 2^-24", flush=True)
        assert bool((err <= 2.0 ** -24 * want.abs() + 3 * 2.0 ** -53 * (ang + 2 * torch.pi)).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("strength", [0.5, 3.0, 10.0, 30.0])
@pytest.mark.parametrize("Hk,Hv,L,dk,dv", [(2, 4, 130, 64, 64), (1, 1, 200, 128, 40), (1, 2, 33, 24, 200)])
def test_gradient_of_strong_decays(dtype, strength, Hk, Hv, L, dk, dv):
    """dl/dg falls with the decays: what one step leaves to the next, e^g of it.  Its
    terms do as well, so its error stays that of sums of some hundred f32 terms of its
    own size, 1e-5 as for every f32 output, head by head.  (The decays of a head are
    within 10 % of each other, e^3 at the strongest.)"""
    print(f"case {dtype} {strength} {Hk} {Hv} {L} {dk} {dv}", flush=True)
    c, d = make(1, Hk, Hv, L, dk, dv, dtype, seed=72)
    gen = torch.Generator().manual_seed(4)
    g = -strength * (1 + 0.1 * torch.rand(1, Hv, L, generator=gen))
    c, d = (*c[:3], g, c[4]), (*d[:3], g.to(DEV), d[4])
    S0, dS1 = (torch.randn(1, Hv, dk, dv, generator=gen) for _ in range(2))
    do = torch.randn(1, Hv, L, dv, generator=gen).to(dtype)
    got = binding.gdr_grads(*d, do.to(DEV), S_in=S0.to(DEV), dS_out=dS1.to(DEV))
    want = reference(c, do, dk ** -0.5, S0, dS1)
    compare(got, want, dtype)
    for h in range(Hv):
        check(f"dg of head {h}", got[3][:, h], want[3][:, h], TOL[F32])
