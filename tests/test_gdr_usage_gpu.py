"""The gated delta rule and the query/key preparation as programs use them:
prompt, then tokens, behind the preparation; a training step through both
adjoints; captured calls; several streams; arrays beyond 2^32 bytes; refusals of
the binding.  Tolerances as in test_gdr_gpu."""
import pytest
import torch

from paper_2512_23068_amd import binding
from tests import gdr_ref as ref
from tests.test_gdr_gpu import BF16, DEV, F32, TOL, check, make

pytestmark = pytest.mark.gpu


def prep_of(d, dtype, L, start=0):
    gen = torch.Generator().manual_seed(5)
    w = [1 + 0.2 * torch.randn(d, generator=gen) for _ in range(2)]
    inv = torch.pow(10000.0, -torch.arange(d // 4) / (d // 4)).float()
    pos = start + torch.arange(L)
    kw = dict(wq=w[0].to(DEV), wk=w[1].to(DEV), norm="l2", eps=1e-6, positions=pos.to(DEV), inv_freq=inv.to(DEV))
    return w, inv, pos, kw


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompt_and_tokens_with_preparation(dtype):
    """Preparation and prompt in one call, then tokens in one call each, against
    float64 on the q and k that the preparation gives (its rounding is its own)."""
    c, d = make(2, 2, 4, 75, 64, 64, dtype, seed=31, fused=True)
    w, inv, pos, kw = prep_of(64, dtype, 75)
    qp, kp = binding.qk_norm(d[0], d[1], **kw)
    for got, x, wt in ((qp, c[0], w[0]), (kp, c[1], w[1])):
        check("prepared", got, ref.qk_prep(x, wt, "l2", 1e-6, pos, inv, False), 1e-6 if dtype == F32 else 2.0 ** -8 + 1e-6)
    kw70 = {**kw, "positions": kw["positions"][:70]}
    o, S = binding.gdr_scan(*[x[:, :, :70] for x in d], return_state=True, qk_prep=kw70)
    outs = [o]
    for t in range(70, 75):
        one = {**kw, "positions": kw["positions"][t:t + 1]}
        outs.append(binding.gdr_step(*[x[:, :, t:t + 1] for x in d], S, qk_prep=one))
    ro, rS = ref.scan(qp.cpu(), kp.cpu(), *c[2:], 0.125)
    check("o", torch.cat(outs, 2), ro, TOL[dtype])
    check("S", S, rS, TOL[F32])


def test_training_step():
    """dl/d(inputs of the preparation) and dl/d(weights) through both adjoints
    against autograd of both maps (f32; tolerance 1e-5, as for every f32 output)."""
    c, d = make(2, 1, 2, 100, 64, 48, F32, seed=32)
    w, inv, pos, kw = prep_of(64, F32, 100)
    do = torch.randn(2, 2, 100, 48, generator=torch.Generator().manual_seed(4))
    qp, kp = binding.qk_norm(d[0], d[1], **kw)
    dq, dk, dv, dg, db = binding.gdr_grads(qp, kp, *d[2:], do.to(DEV))
    gq, gk, gwq, gwk = binding.qk_norm_grads(d[0], d[1], dq, dk, **kw)
    ins = [x.double().clone().requires_grad_(True) for x in (*c, *w)]
    q2, k2 = (ref.qk_prep(x, wt, "l2", 1e-6, pos, inv, False) for x, wt in ((ins[0], ins[5]), (ins[1], ins[6])))
    loss = (ref.scan(q2, k2, *ins[2:5], 0.125)[0] * do.double()).sum()
    want = torch.autograd.grad(loss, ins)
    for n, g, x in zip(("dq", "dk", "dv", "dg", "dbeta", "dwq", "dwk"), (gq, gk, dv, dg, db, gwq, gwk), want):
        check(n, g, x, TOL[F32])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_captured_calls(dtype):
    """A captured chain (preparation, scan of packed sequences in segments,
    gradients, steps) replayed with new inputs between eager work of its own,
    every replay equal to the eager calls."""
    cu = torch.tensor([0, 150, 150, 260], device=DEV, dtype=torch.int32)
    _, d = make(1, 2, 4, 260, 64, 64, dtype, seed=33)
    do = torch.randn(1, 4, 260, 64, device=DEV).to(dtype)
    _, _, _, kw = prep_of(64, dtype, 260)
    pool = torch.zeros(3, 4, 64, 64, device=DEV)
    slots = torch.tensor([2], device=DEV, dtype=torch.int32)

    def chain():
        q, k = binding.qk_norm(d[0], d[1], **kw)
        o, S = binding.gdr_scan(q, k, *d[2:], cu_seqlens=cu, return_state=True, seg_len=64)
        grads = binding.gdr_grads(q, k, *d[2:], do, cu_seqlens=cu, dS_out=S, seg_len=64)
        gq = binding.qk_norm_grads(d[0], d[1], grads[0], grads[1], **kw)
        t = binding.gdr_step(*[x[:, :, :1] for x in (q, k, *d[2:])], pool, slots=slots)
        return (o, S, *grads, *gq, t)

    chain()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = chain()
    gen = torch.Generator(device=DEV).manual_seed(6)
    for i in range(4):
        print("replay", i, flush=True)
        d[2].copy_(torch.randn(d[2].shape, generator=gen, device=DEV))
        d[4].copy_(torch.rand(d[4].shape, generator=gen, device=DEV))
        pool.zero_()
        eager = [x.clone() for x in chain()]
        keep = pool.clone()
        pool.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(captured, eager)) and torch.equal(pool, keep)


def test_streams():
    """Calls on streams of their own at the same time, with workspaces of their own."""
    cases = [make(1, 2, 2, 500, 64, 64, F32, seed=40 + i)[1] for i in range(4)]
    dos = [torch.randn(1, 2, 500, 64, device=DEV) for _ in cases]
    want = [(binding.gdr_scan(*d), *binding.gdr_grads(*d, do)) for d, do in zip(cases, dos)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [None] * 4
    for r in range(3):
        for i, (d, do, s) in enumerate(zip(cases, dos, streams)):
            got[i] = (binding.gdr_scan(*d, stream=s), *binding.gdr_grads(*d, do, stream=s))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(g, w))
    qs = [binding.qk_norm(d[0], d[1], norm="l2", stream=s) for d, s in zip(cases, streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(x[0], binding.qk_norm(d[0], d[1], norm="l2")[0]) for x, d in zip(qs, cases))


def test_far_offsets():
    """A pool of states and strided batches that span more than 2^32 bytes."""
    c, d = make(2, 1, 1, 3, 128, 128, F32, seed=50)
    S = torch.empty(70000, 1, 128, 128, device=DEV)             # 4.6 GB
    S0 = torch.randn(2, 1, 128, 128)
    slots = torch.tensor([69999, 0], device=DEV, dtype=torch.int32)
    S[69999], S[0] = S0[0].to(DEV), S0[1].to(DEV)
    o = binding.gdr_step(*d, S, slots=slots)
    ro, rS = ref.scan(*c, 128 ** -0.5, S0)
    check("o", o, ro, TOL[F32])
    check("S", S[slots.long()], rS, TOL[F32])
    del S
    c, d = make(2, 1, 2, 100, 64, 64, BF16, seed=51)
    far = []
    buf = torch.empty((1 << 31) + (1 << 20), device=DEV, dtype=BF16)      # batch entries 2^31 elements apart
    at = 0
    for x in d[:3]:
        H, L, n = x.shape[1:]
        v = buf.as_strided((2, H, L, n), (1 << 31, L * n, n, 1), at)
        v.copy_(x)
        far.append(v)
        at += H * L * n
    out = buf.as_strided((2, 2, 100, 64), (1 << 31, 6400, 64, 1), at)
    o = binding.gdr_scan(*far, *d[3:], out=out)
    check("o", o, ref.scan(*c, 0.125)[0], TOL[BF16])
    do = torch.randn(2, 2, 100, 64, device=DEV).to(BF16)
    for x, y in zip(binding.gdr_grads(*far, *d[3:], do), binding.gdr_grads(*d, do)):
        assert torch.equal(x, y)
    for x, y in zip(binding.qk_norm(far[0], far[1]), binding.qk_norm(d[0], d[1])):
        assert torch.equal(x, y)


def test_binding_refusals():
    _, d = make(2, 1, 2, 40, 64, 64, F32, seed=60)
    q, k, v, g, beta = d
    S = torch.zeros(2, 2, 64, 64, device=DEV)
    cu = torch.tensor([0, 40], device=DEV, dtype=torch.int32)
    bad = [
        lambda: binding.gdr_scan(q.cpu(), k, v, g, beta), lambda: binding.gdr_scan(q.double(), k, v, g, beta),
        lambda: binding.gdr_scan(q.bfloat16(), k, v, g, beta), lambda: binding.gdr_scan(q, k[..., :32], v, g, beta),
        lambda: binding.gdr_scan(q, k, v[:, :, :39], g, beta), lambda: binding.gdr_scan(q, k, v, g.double(), beta),
        lambda: binding.gdr_scan(q, k, v, g, beta[:1]), lambda: binding.gdr_scan(q, k, v, g, beta, S_in=S[:1]),
        lambda: binding.gdr_scan(q, k, v, g, beta, S_in=S.transpose(2, 3)),
        lambda: binding.gdr_scan(q, k, v, g, beta, cu_seqlens=cu),           # batch of 2
        lambda: binding.gdr_scan(q[:1], k[:1], v[:1], g[:1], beta[:1], cu_seqlens=cu.long()),
        lambda: binding.gdr_scan(q, k, v, g, beta, out=torch.empty_like(v).bfloat16()),
        lambda: binding.gdr_scan(q, k, v, g, beta, out=v[:, :1].expand(2, 2, 40, 64)),
        lambda: binding.gdr_scan(q, k, v, g, beta, workspace=torch.empty(16, device=DEV, dtype=torch.uint8)),
        lambda: binding.gdr_scan(q, k, v, g, beta, stream=3),
        lambda: binding.gdr_grads(q, k, v, g, beta, v[:, :1]), lambda: binding.gdr_grads(q, k, v, g, beta, v, out=(q,)),
        lambda: binding.gdr_step(q, k, v, g, beta, S[:1]), lambda: binding.gdr_step(q, k, v, g, beta, S[0]),
        lambda: binding.gdr_step(q, k, v, g, beta, S, slots=torch.zeros(2, device=DEV)),
        lambda: binding.qk_norm(q, k, norm="layer"), lambda: binding.qk_norm(q, k.bfloat16()),
        lambda: binding.qk_norm(q, k, wq=torch.ones(32)), lambda: binding.qk_norm(q, k, inv_freq=3.0),
        lambda: binding.qk_norm(q, k, inv_freq=torch.ones(16, device=DEV), positions=torch.arange(39, device=DEV)),
        lambda: binding.qk_norm_grads(q, k, q[:, :, :39], k)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("case", i)
    odd = [lambda: binding.gdr_scan(*make(1, 2, 3, 8, 64, 64, F32)[1]), lambda: binding.gdr_scan(q, k, v, g, beta, seg_len=32),
           lambda: binding.gdr_scan(q, k, v, g, beta, out=v), lambda: binding.gdr_scan(*make(1, 1, 1, 8, 136, 64, F32)[1]),
           lambda: binding.gdr_step(q, k, v, g, beta, S, out=v), lambda: binding.qk_norm(q, k, inv_freq=torch.ones(4, device=DEV))]
    for f in odd:
        with pytest.raises(RuntimeError, match="PGF_ERR"):
            f()
    torch.cuda.synchronize()
