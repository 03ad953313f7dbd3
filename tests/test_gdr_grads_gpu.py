"""Gradients of the gated delta rule on the GPU against float64 (autograd of the
recurrence, and differences of it), at the lengths, sizes, types and layouts
where they can go wrong.

Tolerances (relative L2): 1e-5 for f32 outputs (dg, dbeta and dS_in also of bf16
inputs; the repository's bound for f32), one rounding of at most 2^-8 on top for
bf16 ones."""
import pytest
import torch

from paper_2512_23068_amd import binding
from tests import gdr_ref as ref
from tests.test_gdr_gpu import BF16, DEV, F32, TOL, check, make

pytestmark = pytest.mark.gpu
NAMES = ("dq", "dk", "dv", "dg", "dbeta", "dS_in")


def reference(c, do, scale, S0=None, dS1=None):
    ins = [x.double().clone().requires_grad_(True) for x in c]
    B, H = c[2].shape[:2]
    S0 = torch.zeros(B, H, c[0].shape[3], c[2].shape[3]) if S0 is None else S0
    S0 = S0.double().clone().requires_grad_(True)
    o, S = ref.scan(*ins, scale, S0)
    loss = (o * do.double()).sum() + (0 if dS1 is None else (S * dS1.double()).sum())
    grads = torch.autograd.grad(loss, ins + [S0], allow_unused=True)
    return [torch.zeros_like(x) if g is None else g for g, x in zip(grads, ins + [S0])]


def compare(got, want, dtype):
    for n, g, w in zip(NAMES, got, want):
        assert g.dtype == (dtype if n in ("dq", "dk", "dv") else F32)
        check(n, g, w, TOL[dtype] if n in ("dq", "dk", "dv") else TOL[F32])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hk,Hv,L,dk,dv", [
    (1, 1, 1, 1, 8, 8), (2, 1, 2, 31, 16, 16), (1, 2, 2, 32, 64, 64), (1, 2, 4, 33, 64, 72), (2, 2, 2, 65, 24, 40),
    (1, 1, 3, 257, 72, 200), (2, 2, 4, 128, 128, 128), (1, 1, 1, 96, 128, 8), (3, 1, 1, 63, 120, 136)])
def test_grads(dtype, B, Hk, Hv, L, dk, dv):
    print(f"case {dtype} {B} {Hk} {Hv} {L} {dk} {dv}", flush=True)
    c, d = make(B, Hk, Hv, L, dk, dv, dtype, fused=L % 2 == 1)
    gen = torch.Generator().manual_seed(4)
    S0, dS1 = (torch.randn(B, Hv, dk, dv, generator=gen) * 0.5 for _ in range(2))
    do = torch.randn(B, Hv, L, dv, generator=gen).to(dtype)
    got = binding.gdr_grads(*d, do.to(DEV), S_in=S0.to(DEV), dS_out=dS1.to(DEV))
    torch.cuda.synchronize()
    assert len(got) == 6
    compare(got, reference(c, do, dk ** -0.5, S0, dS1), dtype)
    got = binding.gdr_grads(*d, do.to(DEV), scale=0.25)
    assert len(got) == 5
    compare(got, reference(c, do, 0.25), dtype)
    again = binding.gdr_grads(*d, do.to(DEV), scale=0.25)
    assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Hk,Hv,L,dk,dv", [(1, 4, 130, 128, 24), (2, 6, 65, 40, 32), (1, 2, 100, 104, 96), (1, 3, 64, 64, 104)])
def test_grads_shared_heads(dtype, Hk, Hv, L, dk, dv):
    """Value heads of one key head follow each other through one to four rounds of 32 value columns."""
    print(f"case {dtype} {Hk} {Hv} {L} {dk} {dv}", flush=True)
    c, d = make(1, Hk, Hv, L, dk, dv, dtype, seed=11)
    do = torch.randn(1, Hv, L, dv, generator=torch.Generator().manual_seed(12)).to(dtype)
    compare(binding.gdr_grads(*d, do.to(DEV)), reference(c, do, dk ** -0.5), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_grads_widest(dtype):
    """The largest head: 128 keys, 4096 value columns; the scan and the steps of the same."""
    c, d = make(1, 1, 1, 70, 128, 4096, dtype, seed=13)
    gen = torch.Generator().manual_seed(14)
    S0, dS1 = (torch.randn(1, 1, 128, 4096, generator=gen) * 0.5 for _ in range(2))
    do = torch.randn(1, 1, 70, 4096, generator=gen).to(dtype)
    got = binding.gdr_grads(*d, do.to(DEV), S_in=S0.to(DEV), dS_out=dS1.to(DEV))
    compare(got, reference(c, do, 128 ** -0.5, S0, dS1), dtype)
    want, wS = ref.scan(*c, 128 ** -0.5, S0)
    o, S = binding.gdr_scan(*d, S_in=S0.to(DEV), return_state=True)
    check("o", o, want, TOL[dtype])
    check("S", S, wS, TOL[F32])
    S = S0.to(DEV)
    check("o of steps", binding.gdr_step(*d, S), want, TOL[dtype])
    check("S of steps", S, wS, TOL[F32])


def test_grads_empty():
    _, d = make(2, 1, 2, 0, 64, 64, F32)
    dS = torch.randn(2, 2, 64, 64, device=DEV)
    got = binding.gdr_grads(*d, torch.empty_like(d[2]), dS_out=dS)
    assert torch.equal(got[5], dS) and got[0].shape == d[0].shape


@pytest.mark.parametrize("dtype,dk,dv", [(F32, 64, 64), (BF16, 128, 72)])
def test_grads_packed(dtype, dk, dv):
    """Empty sequences, ones of a single step, and rows of no sequence that hold
    NaN: their gradients are zero in new outputs and stay as they were in given ones."""
    cu = [3, 3, 70, 71, 71, 135, 230]
    T, n = 240, 6
    c, d = make(1, 2, 4, T, dk, dv, dtype, seed=3)
    gen = torch.Generator().manual_seed(4)
    S0, dS1 = (torch.randn(n, 4, dk, dv, generator=gen) * 0.5 for _ in range(2))
    do = torch.randn(1, 4, T, dv, generator=gen).to(dtype)
    dod = do.to(DEV)
    for x in (*d, dod):
        x[:, :, :3] = float("nan")
        x[:, :, 230:] = float("nan")
    cud = torch.tensor(cu, device=DEV, dtype=torch.int32)
    got = binding.gdr_grads(*d, dod, S_in=S0.to(DEV), dS_out=dS1.to(DEV), cu_seqlens=cud)
    torch.cuda.synchronize()
    parts = ref.packed(lambda *a: reference(a[:5], a[5], dk ** -0.5, a[6], a[7]), cu, (*c, do), [S0, dS1])
    want = [torch.cat([p[i] for p in parts], 2) for i in range(5)] + [torch.cat([p[5] for p in parts])]
    compare([g[:, :, 3:230] for g in got[:5]] + [got[5]], want, dtype)
    for g in got[:5]:
        assert not g[:, :, :3].any() and not g[:, :, 230:].any()
    out = [torch.full_like(x, 7.0) for x in d[:3]]
    got = binding.gdr_grads(*d, dod, cu_seqlens=cud, out=out)
    assert not any(bool(x[:, :, :3].any() or x[:, :, 230:].any()) for x in got[3:5])
    assert all(bool((x[:, :, :3] == 7).all() and (x[:, :, 230:] == 7).all()) for x in out)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_grads_decays(dtype):
    """No decay, -inf in the middle (nothing reaches back over it, and its own
    gradient is zero), and beta of zero and one."""
    c, d = make(1, 2, 2, 100, 64, 64, dtype, seed=5)
    for g in (c[3], d[3]):
        g[:, 0] = 0.0
        g[:, 1, 41:60] = -1000.0
        g[:, 1, 60:] = -0.001
    d[3][:, 1, 40] = float("-inf")
    c[3][:, 1, 40] = -800.0            # (e^-800 is zero in float64's products with f32 data; autograd of e^-inf is not defined)
    for b in (c[4], d[4]):
        b[:, :, 10:20] = 0.0
        b[:, :, 20:30] = 1.0
    do = torch.randn(1, 2, 100, 64, generator=torch.Generator().manual_seed(4)).to(dtype)
    got = binding.gdr_grads(*d, do.to(DEV))
    want = reference(c, do, 0.125)
    for h in range(2):
        compare([g[:, h:h + 1] for g in got], [w[:, h:h + 1] for w in want[:5]], dtype)


def test_grads_against_differences():
    """dl along a random direction of every input against a central difference of
    the GPU's own scan, in float32 with a step that balances rounding (2^-24 of the
    loss's terms over the step) and curvature: 1e-3 of the sum."""
    c, d = make(1, 2, 4, 150, 64, 64, F32, seed=21)
    gen = torch.Generator(device=DEV).manual_seed(4)
    do = torch.randn(1, 4, 150, 64, generator=gen, device=DEV)
    got = binding.gdr_grads(*d, do)
    dirs = [torch.randn(x.shape, generator=gen, device=DEV) * s for x, s in zip(d, (1, 0.1, 1, 0.01, 0.1))]
    eps = 1e-3
    for i, n in enumerate(NAMES[:5]):
        loss = []
        for sign in (1, -1):
            x = list(d)
            x[i] = d[i] + sign * eps * dirs[i]
            loss.append(float((binding.gdr_scan(*x).double() * do.double()).sum()))
        want = (loss[0] - loss[1]) / (2 * eps)
        have = float((got[i].double() * dirs[i].double()).sum())
        size = float((got[i].double().abs() * dirs[i].double().abs()).sum())
        print(n, have, want, size, flush=True)
        assert abs(have - want) <= 1e-3 * size, n


def test_grads_into_one_array():
    """dq, dk and dv as views of one fused array, other strides than the inputs'."""
    c, d = make(2, 2, 4, 70, 64, 64, BF16, seed=22)
    do = torch.randn(2, 4, 70, 64, device=DEV).bfloat16()
    want = binding.gdr_grads(*d, do)
    big = torch.empty(2, 70, 2 * 64 + 2 * 64 + 4 * 64, device=DEV, dtype=BF16)
    parts = [big[..., :128].unflatten(-1, (2, 64)).transpose(1, 2), big[..., 128:256].unflatten(-1, (2, 64)).transpose(1, 2),
             big[..., 256:].unflatten(-1, (4, 64)).transpose(1, 2)]
    got = binding.gdr_grads(*d, do, out=parts)
    assert all(g is p for g, p in zip(got, parts))
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype,dk,dv", [(F32, 64, 72), (BF16, 128, 40), (F32, 104, 128)])
def test_grads_segments(dtype, dk, dv):
    """Segments, the last one short, dense and packed with empty sequences."""
    c, d = make(2, 1, 2, 330, dk, dv, dtype, seed=14, g_scale=0.02)
    gen = torch.Generator().manual_seed(4)
    S0, dS1 = (torch.randn(2, 2, dk, dv, generator=gen) * 0.5 for _ in range(2))
    do = torch.randn(2, 2, 330, dv, generator=gen).to(dtype)
    want = reference(c, do, dk ** -0.5, S0, dS1)
    for seg in (-1, 64, 128):
        print("segments of", seg, flush=True)
        compare(binding.gdr_grads(*d, do.to(DEV), S_in=S0.to(DEV), dS_out=dS1.to(DEV), seg_len=seg), want, dtype)
    cu = [0, 200, 200, 231, 329, 330]
    c, d = make(1, 1, 2, 330, dk, dv, dtype, seed=15, g_scale=0.02)
    S0, dS1 = (torch.randn(5, 2, dk, dv, generator=gen) * 0.5 for _ in range(2))
    do = torch.randn(1, 2, 330, dv, generator=gen).to(dtype)
    got = binding.gdr_grads(*d, do.to(DEV), S_in=S0.to(DEV), dS_out=dS1.to(DEV), seg_len=64,
                            cu_seqlens=torch.tensor(cu, device=DEV, dtype=torch.int32))
    parts = ref.packed(lambda *a: reference(a[:5], a[5], dk ** -0.5, a[6], a[7]), cu, (*c, do), [S0, dS1])
    compare(got, [torch.cat([p[i] for p in parts], 2) for i in range(5)] + [torch.cat([p[5] for p in parts])], dtype)
