"""The gated delta rule on the GPU with the strides that single steps, broadcasts
and windows have, against float64.  Tolerances as in test_gdr_gpu."""
import pytest
import torch

from paper_2512_23068_amd import binding
from tests import gdr_ref as ref
from tests.test_gdr_gpu import BF16, DEV, F32, TOL, check, make
from tests.test_gdr_grads_gpu import compare, reference

pytestmark = pytest.mark.gpu


def one_step(dtype, B, Hk, Hv, dk, dv, seed):
    """Five steps of inputs, the adjoint signal and states; step 2 is the call's."""
    c, d = make(B, Hk, Hv, 5, dk, dv, dtype, seed=seed)
    gen = torch.Generator().manual_seed(seed)
    do = torch.randn(B, Hv, 5, dv, generator=gen).to(dtype)
    S0, dS1 = (torch.randn(B, Hv, dk, dv, generator=gen) * 0.5 for _ in range(2))
    return c, d, do, S0, dS1


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hk,Hv,dk,dv", [(2, 2, 4, 64, 64), (1, 2, 2, 128, 40), (3, 1, 1, 24, 136)])
def test_one_step_of_longer_inputs(dtype, B, Hk, Hv, dk, dv):
    """All inputs and the adjoint signal are one step of longer arrays."""
    print(f"case {dtype} {B} {Hk} {Hv} {dk} {dv}", flush=True)
    c, d, do, S0, dS1 = one_step(dtype, B, Hk, Hv, dk, dv, 81)
    cut = lambda xs: [x[:, :, 2:3] for x in xs]  # noqa: E731
    o, S = binding.gdr_scan(*cut(d), S_in=S0.to(DEV), return_state=True)
    ro, rS = ref.scan(*cut(c), dk ** -0.5, S0)
    check("o", o, ro, TOL[dtype])
    check("S", S, rS, TOL[F32])
    got = binding.gdr_grads(*cut(d), do.to(DEV)[:, :, 2:3], S_in=S0.to(DEV), dS_out=dS1.to(DEV))
    compare(got, reference(cut(c), do[:, :, 2:3], dk ** -0.5, S0, dS1), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hk,Hv,dk,dv", [(2, 2, 4, 64, 64), (1, 2, 2, 128, 40), (3, 1, 1, 24, 136)])
@pytest.mark.parametrize("sliced", [False, True])
def test_one_step_into_given_outputs(dtype, B, Hk, Hv, dk, dv, sliced):
    """Outputs of one step: contiguous ones, and one step of longer arrays, whose
    other steps stay as they were."""
    print(f"case {dtype} {B} {Hk} {Hv} {dk} {dv} {sliced}", flush=True)
    c, d, do, S0, dS1 = one_step(dtype, B, Hk, Hv, dk, dv, 82)
    c, d = ([x[:, :, 2:3].contiguous() for x in xs] for xs in (c, d))
    whole = [torch.full((B, h, 5 if sliced else 1, n), 7.0, device=DEV, dtype=dtype)
             for h, n in ((Hv, dv), (Hk, dk), (Hk, dk), (Hv, dv))]
    at = slice(3, 4) if sliced else slice(0, 1)
    out = [x[:, :, at] for x in whole]
    o, S = binding.gdr_scan(*d, S_in=S0.to(DEV), return_state=True, out=out[0])
    ro, rS = ref.scan(*c, dk ** -0.5, S0)
    check("o", o, ro, TOL[dtype])
    check("S", S, rS, TOL[F32])
    do = do[:, :, 2:3].contiguous()
    got = binding.gdr_grads(*d, do.to(DEV), S_in=S0.to(DEV), dS_out=dS1.to(DEV), out=out[1:])
    compare(got, reference(c, do, dk ** -0.5, S0, dS1), dtype)
    if sliced:
        assert all(bool((x[:, :, [0, 1, 2, 4]] == 7).all()) for x in whole)
