"""Roundings of the gated delta rule's bf16 outputs on the GPU.

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
