"""Sizes from which the gated delta rule and the query/key preparation take other
blocks: a column tile to one wave (more than 512 tiles), 128 value columns a block
of steps (256 blocks of them), several steps a block and several turns of a block
in the preparation and its adjoint.  Against float64, tolerances as in
test_gdr_gpu and test_qk_norm_gpu."""
import pytest
import torch

from paper_2512_23068_amd import binding
from tests import gdr_ref as ref
from tests.test_gdr_gpu import BF16, DEV, F32, TOL, check, make
from tests.test_gdr_grads_gpu import compare, reference
from tests.test_qk_norm_gpu import TOL as QK_TOL
from tests.test_qk_norm_gpu import inv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dk", [64, 128])
@pytest.mark.parametrize("B,Hk,Hv,L,dv,seg", [(20, 8, 32, 33, 16, -1), (5, 4, 12, 70, 168, -1), (3, 4, 8, 330, 80, 64)])
def test_scan_of_many_tiles(dtype, dk, B, Hk, Hv, L, dv, seg):
    print(f"case {dtype} {dk} {B} {Hk} {Hv} {L} {dv} {seg}", flush=True)
    assert B * (1 if seg < 0 else -(-L // seg)) * Hv * -(-dv // 16) > 512
    c, d = make(B, Hk, Hv, L, dk, dv, dtype, seed=91, fused=True)
    S0 = torch.randn(B, Hv, dk, dv, generator=torch.Generator().manual_seed(9)) * 0.5
    o, S = binding.gdr_scan(*d, S_in=S0.to(DEV), return_state=True, seg_len=seg)
    ro, rS = ref.scan(*c, dk ** -0.5, S0)
    check("o", o, ro, TOL[dtype])
    check("S", S, rS, TOL[F32])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_scan_of_many_tiles(dtype):
    """Packed prompts, one of them empty, at a tile a wave; gradients of the same."""
    cu = [2, 40, 40, 41, 105, 238]
    c, d = make(1, 8, 32, 240, 64, 72, dtype, seed=92, fused=True)
    n = len(cu) - 1
    gen = torch.Generator().manual_seed(9)
    S0, dS1 = (torch.randn(n, 32, 64, 72, generator=gen) * 0.5 for _ in range(2))
    do = torch.randn(1, 32, 240, 72, generator=gen).to(dtype)
    kw = dict(S_in=S0.to(DEV), cu_seqlens=torch.tensor(cu, device=DEV, dtype=torch.int32))
    o, S = binding.gdr_scan(*d, return_state=True, **kw)
    parts = ref.packed(lambda *a: ref.scan(*a[:5], 0.125, a[5]), cu, c, [S0])
    check("o", o[:, :, 2:238], torch.cat([p[0] for p in parts], 2), TOL[dtype])
    check("S", S, torch.cat([p[1] for p in parts]), TOL[F32])
    got = binding.gdr_grads(*d, do.to(DEV), dS_out=dS1.to(DEV), **kw)
    parts = ref.packed(lambda *a: reference(a[:5], a[5], 0.125, a[6], a[7]), cu, (*c, do), [S0, dS1])
    want = [torch.cat([p[i] for p in parts], 2) for i in range(5)] + [torch.cat([p[5] for p in parts])]
    compare([g[:, :, 2:238] for g in got[:5]] + [got[5]], want, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dk", [64, 104])
@pytest.mark.parametrize("B,Hk,Hv,L,dv", [(64, 2, 4, 4, 128), (43, 1, 3, 3, 200), (90, 3, 3, 17, 40)])
def test_steps_of_many_states(dtype, dk, B, Hk, Hv, L, dv):
    print(f"case {dtype} {dk} {B} {Hk} {Hv} {L} {dv}", flush=True)
    assert L > 2 and B * Hv * -(-dv // 128) >= 256
    c, d = make(B, Hk, Hv, L, dk, dv, dtype, seed=93, fused=True)
    gen = torch.Generator().manual_seed(2)
    S = torch.randn(B + 5, Hv, dk, dv, generator=gen)
    slots = torch.randperm(B + 5, generator=gen)[:B].to(torch.int32)
    slots[3], slots[7] = -1, slots[6]               # padding, and a state named twice
    live = [b for b in range(B) if b not in (3, 7)]
    Sd = S.to(DEV)
    o = binding.gdr_step(*d, Sd, slots=slots.to(DEV))
    at = slots[live].long()
    ro, rS = ref.scan(*[x[live] for x in c], dk ** -0.5, S[at])
    check("o", o[live], ro, TOL[dtype])
    check("S", Sd[at.to(DEV)], rS, TOL[F32])
    assert not o[[3, 7]].any()
    rest = sorted(set(range(B + 5)) - set(at.tolist()))
    assert torch.equal(Sd[rest].cpu(), S[rest])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hk,L,d,rot,il", [(3, 2, 1, 6001, 32, 32, False), (3, 2, 1, 6001, 32, 16, True),
                                                (1, 1, 1, 2049, 256, 128, False), (5, 1, 2, 821, 72, 64, True)])
def test_preparation_of_many_steps(dtype, B, Hq, Hk, L, d, rot, il):
    print(f"case {dtype} {B} {Hq} {Hk} {L} {d} {rot} {il}", flush=True)
    assert B * L >= 2048
    gen = torch.Generator().manual_seed(1)
    q, k, dq, dk = (torch.randn(B, h, L, d, generator=gen).to(dtype) for h in (Hq, Hk, Hq, Hk))
    w = [1 + 0.3 * torch.randn(d, generator=gen) for _ in range(2)]
    pos = torch.randint(0, 1 << 22, (B, 1), generator=gen) + torch.arange(L)
    f = inv(rot)
    kw = dict(wq=w[0].to(DEV), wk=w[1].to(DEV), eps=1e-5, positions=pos.to(DEV), inv_freq=f.to(DEV), interleaved=il)
    got = binding.qk_norm(q.to(DEV), k.to(DEV), **kw)
    back = binding.qk_norm_grads(q.to(DEV), k.to(DEV), dq.to(DEV), dk.to(DEV), **kw)
    ins = [x.double().clone().requires_grad_(True) for x in (q, k, *w)]
    want = [ref.qk_prep(x, wt, "rms", 1e-5, pos, f, il) for x, wt in ((ins[0], ins[2]), (ins[1], ins[3]))]
    for n, g, x in zip("qk", got, want):
        check(n, g, x, QK_TOL[dtype])
    grads = torch.autograd.grad(sum((y * g.double()).sum() for y, g in zip(want, (dq, dk))), ins)
    for n, g, x in zip(("dq", "dk", "dwq", "dwk"), back, grads):
        check(n, g, x, QK_TOL[dtype] if n in ("dq", "dk") else 1e-5)
