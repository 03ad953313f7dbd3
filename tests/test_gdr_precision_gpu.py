"""Roundings on the GPU: bf16 outputs of the gated delta rule, and the rotation of
queries and keys.

A bf16 input is the first of its f32 value's three parts and the other two are
zero, so the scan of bf16 inputs and that of the same values in f32 add the same
products in the same order: the bf16 output is the f32 output rounded once, bit
for bit, and the states are the same."""
import pytest
import torch

from paper_2512_23068_amd import binding
from tests.test_gdr_gpu import BF16, DEV, make

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
