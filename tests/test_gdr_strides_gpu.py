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


def spread(x, kind):
    """x [B,H,L,d] with one row for all steps, or with rows that begin 16 bytes after
    each other, on the CPU and on the GPU."""
    B, H, L, d = x.shape
    if kind == "broadcast":
        return x[:, :, :1].expand(B, H, L, d), x[:, :, :1].to(DEV).expand(B, H, L, d)
    unit = 16 // x.element_size()
    n = d + unit * (L - 1)
    flat = x.flatten(2)[..., :n].contiguous()
    return tuple(f.as_strided(x.shape, (H * n, n, unit, 1)) for f in (flat, flat.to(DEV)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["broadcast", "window"])
@pytest.mark.parametrize("which", ["q do", "q k v do"])
@pytest.mark.parametrize("B,Hk,Hv,L,dk,dv,cu", [
    (2, 2, 4, 33, 64, 64, None), (1, 2, 2, 70, 128, 40, None), (2, 1, 2, 65, 24, 136, None),
    (1, 2, 4, 100, 64, 64, [0, 33, 34, 100])])
def test_broadcast_and_window_inputs(dtype, kind, which, B, Hk, Hv, L, dk, dv, cu):
    """Step strides below a row: what follows a sequence's last row in memory is the
    array's own, and does not count."""
    print(f"case {dtype} {kind} {which} {B} {Hk} {Hv} {L} {dk} {dv}", flush=True)
    c, d = (list(x) for x in make(B, Hk, Hv, L, dk, dv, dtype, seed=83))
    gen = torch.Generator().manual_seed(84)
    do = torch.randn(B, Hv, L, dv, generator=gen).to(dtype)
    dod = do.to(DEV)
    for i, n in enumerate("qkv"):
        if n in which.split():
            c[i], d[i] = spread(c[i], kind)
    if kind == "window" and "k" in which.split():      # (keys stay near norm 1: a window of normalised keys)
        c[1], d[1] = spread(make(B, Hk, Hv, L, dk, dv, dtype, seed=85)[0][1], kind)
    do, dod = spread(do, kind)
    n = B if cu is None else len(cu) - 1
    S0, dS1 = (torch.randn(n, Hv, dk, dv, generator=gen) * 0.5 for _ in range(2))
    kw = {} if cu is None else dict(cu_seqlens=torch.tensor(cu, device=DEV, dtype=torch.int32))
    o, S = binding.gdr_scan(*d, S_in=S0.to(DEV), return_state=True, **kw)
    got = binding.gdr_grads(*d, dod, S_in=S0.to(DEV), dS_out=dS1.to(DEV), **kw)
    if cu is None:
        ro, rS = ref.scan(*c, dk ** -0.5, S0)
        want = reference(c, do, dk ** -0.5, S0, dS1)
    else:
        parts = ref.packed(lambda *a: ref.scan(*a[:5], dk ** -0.5, a[5]), cu, c, [S0])
        ro, rS = torch.cat([p[0] for p in parts], 2), torch.cat([p[1] for p in parts])
        parts = ref.packed(lambda *a: reference(a[:5], a[5], dk ** -0.5, a[6], a[7]), cu, (*c, do), [S0, dS1])
        want = [torch.cat([p[i] for p in parts], 2) for i in range(5)] + [torch.cat([p[5] for p in parts])]
    check("o", o, ro, TOL[dtype])
    check("S", S, rS, TOL[F32])
    compare(got, want, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_grads_into_rows_of_heads(dtype):
    """dq, dk and dv as parts of each head's rows [B, H, L, 3 d]."""
    c, d = make(2, 3, 3, 70, 64, 64, dtype, seed=86)
    do = torch.randn(2, 3, 70, 64, device=DEV).to(dtype)
    want = binding.gdr_grads(*d, do)
    big = torch.empty(2, 3, 70, 192, device=DEV, dtype=dtype)
    got = binding.gdr_grads(*d, do, out=big.split(64, -1))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert torch.equal(big, torch.cat(want[:3], -1))


def test_steps_far_apart():
    """Inputs whose steps lie 2^24 bytes apart, as documented: any strides."""
    c, d = make(1, 2, 2, 5, 64, 64, F32, seed=87)
    big = torch.empty(5, 1 << 22, device=DEV)
    far = []
    for i, x in enumerate(d[:3]):
        v = big[:, 128 * i:128 * (i + 1)].unflatten(1, (1, 2, 64)).permute(1, 2, 0, 3)
        v.copy_(x)
        far.append(v)
    do = torch.randn(1, 2, 5, 64, device=DEV)
    assert torch.equal(binding.gdr_scan(*far, *d[3:]), binding.gdr_scan(*d))
    for x, y in zip(binding.gdr_grads(*far, *d[3:], do), binding.gdr_grads(*d, do)):
        assert torch.equal(x, y)
    S = [torch.zeros(1, 2, 64, 64, device=DEV) for _ in range(2)]
    assert torch.equal(binding.gdr_step(*far, *d[3:], S[0]), binding.gdr_step(*d, S[1])) and torch.equal(*S)
