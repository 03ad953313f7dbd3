"""The gated delta rule on the GPU against the float64 recurrence: lengths
around the chunk of 32 steps, odd head sizes, shared key heads, both types,
strided and broadcast inputs, packed sequences with empty ones and foreign
rows, entry and final states, full forgetting, and single steps on a pool.

Tolerances (relative L2).  f32 outputs and states: 1e-5, the repository's bound
for f32 (sums of some hundred f32 roundings of 2^-24 each stay below 1e-6).
bf16 outputs: one rounding of at most 2^-8 relative on top of that."""
import pytest
import torch

from paper_2512_23068_amd import binding
from tests import gdr_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 1e-5, BF16: 2.0 ** -8 + 1e-5}
DEV = "cuda:0"


def make(B, Hk, Hv, L, dk, dv, dtype, seed=0, g_scale=0.1, fused=False):
    gen = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    q, k = rn(B, Hk, L, dk) + 0.3, rn(B, Hk, L, dk) + 0.3
    q, k = q / q.norm(dim=-1, keepdim=True), k / k.norm(dim=-1, keepdim=True)
    v = rn(B, Hv, L, dv)
    g = -g_scale * torch.exp(rn(B, Hv, L))
    beta = torch.sigmoid(rn(B, Hv, L))
    q, k, v = (x.to(dtype) for x in (q, k, v))
    if fused:      # views of one array [B, L, all heads]
        big = torch.cat([x.transpose(1, 2).flatten(2) for x in (q, k, v)], -1).to(DEV)
        parts, at = [], 0
        for h, d in ((Hk, dk), (Hk, dk), (Hv, dv)):
            parts.append(big[..., at:at + h * d].unflatten(-1, (h, d)).transpose(1, 2))
            at += h * d
        return (q, k, v, g, beta), (*parts, g.to(DEV), beta.to(DEV))
    return (q, k, v, g, beta), tuple(x.to(DEV) for x in (q, k, v, g, beta))


def check(what, got, want, tol):
    e = ref.rel(got, want)
    print(f"{what}: rel {e:.2e}", flush=True)
    assert bool(torch.isfinite(got).all()) and e <= tol, (what, e, tol)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hk,Hv,L,dk,dv", [
    (1, 1, 1, 1, 8, 8), (2, 1, 2, 31, 16, 16), (1, 2, 2, 32, 64, 64), (1, 2, 4, 33, 64, 72), (2, 2, 2, 65, 24, 40),
    (1, 1, 3, 257, 72, 200), (2, 2, 4, 200, 128, 128), (1, 1, 1, 96, 128, 8), (3, 1, 1, 63, 120, 136)])
def test_scan(dtype, B, Hk, Hv, L, dk, dv):
    print(f"case {dtype} {B} {Hk} {Hv} {L} {dk} {dv}", flush=True)
    c, d = make(B, Hk, Hv, L, dk, dv, dtype, fused=L % 2 == 1)
    S0 = torch.randn(B, Hv, dk, dv, generator=torch.Generator().manual_seed(9)) * 0.5
    o, S = binding.gdr_scan(*d, S_in=S0.to(DEV), return_state=True)
    torch.cuda.synchronize()
    ro, rS = ref.scan(*c, dk ** -0.5, S0)
    assert o.dtype == dtype and o.shape == d[2].shape
    check("o", o, ro, TOL[dtype])
    check("S", S, rS, TOL[F32])
    o2 = binding.gdr_scan(*d, S_in=S0.to(DEV))
    assert torch.equal(o2, o)
    o3 = binding.gdr_scan(*d, scale=0.25)
    check("o without an entry state", o3, ref.scan(*c, 0.25)[0], TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_empty(dtype):
    _, d = make(2, 1, 2, 0, 64, 64, dtype)
    S0 = torch.randn(2, 2, 64, 64, device=DEV)
    o, S = binding.gdr_scan(*d, S_in=S0, return_state=True)
    torch.cuda.synchronize()
    assert o.shape == (2, 2, 0, 64) and torch.equal(S, S0)
    S = binding.gdr_scan(*d, return_state=True)[1]
    assert not S.any()


@pytest.mark.parametrize("dtype,dk,dv", [(F32, 64, 64), (BF16, 128, 72)])
def test_scan_packed(dtype, dk, dv):
    """Empty sequences, ones of a single step, rows before the first and behind
    the last sequence that hold NaN and stay as they were."""
    cu = [3, 3, 70, 71, 71, 135, 230]
    T = 240
    c, d = make(1, 2, 4, T, dk, dv, dtype, seed=3)
    for x in d:
        x[:, :, :3] = float("nan")
        x[:, :, 230:] = float("nan")
    n = len(cu) - 1
    S0 = torch.randn(n, 4, dk, dv, generator=torch.Generator().manual_seed(9))
    out = torch.full((1, 4, T, dv), 7.0, device=DEV, dtype=dtype)
    cud = torch.tensor(cu, device=DEV, dtype=torch.int32)
    o, S = binding.gdr_scan(*d, S_in=S0.to(DEV), return_state=True, cu_seqlens=cud, out=out)
    torch.cuda.synchronize()
    assert bool((o[:, :, :3] == 7).all()) and bool((o[:, :, 230:] == 7).all())
    want = ref.packed(lambda *a: ref.scan(*a[:5], dk ** -0.5, a[5]), cu, c, [S0])
    check("o", o[:, :, 3:230], torch.cat([w[0] for w in want], 2), TOL[dtype])
    check("S", S, torch.cat([w[1] for w in want]), TOL[F32])
    fresh = binding.gdr_scan(*d, cu_seqlens=cud)
    assert not fresh[:, :, :3].any() and not fresh[:, :, 230:].any()
    # clipped and descending bounds stay within the arrays
    bad = torch.tensor([-5, 100, 50, 1 << 30], device=DEV, dtype=torch.int32)
    binding.gdr_scan(*d, cu_seqlens=bad)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_decays(dtype):
    """No decay, -inf in the middle of a chunk (all that came before is gone),
    strong decay beside a weak one, and beta of zero and one."""
    c, d = make(1, 2, 2, 100, 64, 64, dtype, seed=5)
    for g in (c[3], d[3]):
        g[:, 0] = 0.0
        g[:, 1, 40] = float("-inf")
        g[:, 1, 41:60] = -1000.0
        g[:, 1, 60:] = -0.001
    for b in (c[4], d[4]):
        b[:, :, 10:20] = 0.0
        b[:, :, 20:30] = 1.0
    o, S = binding.gdr_scan(*d, return_state=True)
    ro, rS = ref.scan(*c, 64 ** -0.5)
    for h in range(2):
        check(f"o head {h}", o[:, h], ro[:, h], TOL[dtype])
        check(f"S head {h}", S[:, h], rS[:, h], TOL[F32])


def test_scan_repeated_keys():
    """The same key at every step with beta 1: each write replaces the last one."""
    c, d = make(1, 1, 1, 90, 64, 64, F32, seed=6)
    for k in (c[1], d[1]):
        k[:] = k[:, :, :1].clone()
    for x, val in ((3, 0.0), (4, 1.0)):
        c[x][:] = val
        d[x][:] = val
    o, S = binding.gdr_scan(*d, return_state=True)
    ro, rS = ref.scan(*c, 64 ** -0.5)
    check("o", o, ro, TOL[F32])
    check("S", S, rS, TOL[F32])


def test_scan_views_and_broadcasts():
    """Transposed, offset and broadcast inputs, and an output of other strides."""
    c, d = make(2, 2, 4, 70, 32, 48, F32, seed=7)
    ro, _ = ref.scan(*c, 32 ** -0.5)
    q = torch.randn(2 * 2 * 70 * 32 + 1, device=DEV)[1:].view(2, 2, 70, 32)      # address off by one element
    q.copy_(d[0])
    k = d[1].transpose(2, 3).contiguous().transpose(2, 3)                        # d_key not dense
    out = torch.empty(2, 70, 4, 48, device=DEV).transpose(1, 2)
    o = binding.gdr_scan(q, k, *d[2:], out=out)
    assert o.data_ptr() == out.data_ptr()
    check("o", o, ro, TOL[F32])
    g = torch.full((), -0.25, device=DEV).expand(2, 4, 70)
    beta = torch.rand(1, 4, 1, device=DEV).expand(2, 4, 70)
    v = d[2][:, :1].expand(2, 4, 70, 48)
    o = binding.gdr_scan(d[0], d[1], v, g, beta)
    ro, _ = ref.scan(c[0], c[1], c[2][:, :1].expand(2, 4, 70, 48), g.cpu(), beta.cpu(), 32 ** -0.5)
    check("broadcast", o, ro, TOL[F32])


def test_scan_later_chunks_do_not_reach_back():
    c, d = make(1, 1, 1, 128, 64, 64, F32, seed=8)
    o = binding.gdr_scan(*d)
    d[2][:, :, 64] = float("nan")
    d[1][:, :, 70] = float("inf")
    o2 = binding.gdr_scan(*d)
    assert torch.equal(o2[:, :, :64], o[:, :, :64])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hk,Hv,L,dk,dv", [(1, 1, 1, 1, 8, 8), (3, 2, 4, 1, 64, 64), (2, 1, 3, 5, 128, 200),
                                             (2, 2, 2, 2, 72, 40), (70, 4, 8, 1, 128, 128)])
def test_step(dtype, B, Hk, Hv, L, dk, dv):
    c, d = make(B, Hk, Hv, L, dk, dv, dtype, seed=11, fused=True)
    S = torch.randn(B, Hv, dk, dv, generator=torch.Generator().manual_seed(2))
    Sd = S.to(DEV)
    o = binding.gdr_step(*d, Sd)
    ro, rS = ref.scan(*c, dk ** -0.5, S)
    check("o", o, ro, TOL[dtype])
    check("S", Sd, rS, TOL[F32])


def test_step_slots():
    """A pool larger than the batch; padding (-1 and beyond the pool), and a state named twice."""
    B, H, dk, dv, pool = 7, 2, 64, 64, 9
    c, d = make(B, H, H, 3, dk, dv, F32, seed=12)
    S = torch.randn(pool, H, dk, dv, generator=torch.Generator().manual_seed(2))
    slots = torch.tensor([4, -1, 8, 9, 0, 4, 3], dtype=torch.int32)
    Sd = S.to(DEV)
    o = binding.gdr_step(*d, Sd, slots=slots.to(DEV))
    live = [0, 2, 4, 6]
    ro, rS = ref.scan(*[x[live] for x in c], dk ** -0.5, S[slots[live].long()])
    check("o", o[live], ro, TOL[F32])
    assert not o[[1, 3, 5]].any()
    check("S", Sd[slots[live].long()], rS, TOL[F32])
    rest = [i for i in range(pool) if i not in slots[live].tolist()]
    assert torch.equal(Sd[rest].cpu(), S[rest])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompt_then_tokens(dtype):
    """A prompt with the scan, then tokens one by one from its state: as one scan over all."""
    c, d = make(2, 1, 2, 77, 128, 64, dtype, seed=13)
    whole, S1 = binding.gdr_scan(*d, return_state=True)
    o, S = binding.gdr_scan(*[x[:, :, :70] for x in d], return_state=True)
    outs = [o]
    for t in range(70, 77):
        outs.append(binding.gdr_step(*[x[:, :, t:t + 1] for x in d], S))
    got = torch.cat(outs, 2)
    ro, rS = ref.scan(*c, 128 ** -0.5)
    check("o", got, ro, TOL[dtype])
    check("S", S, rS, TOL[F32])
    check("whole", whole, ro, TOL[dtype])


@pytest.mark.parametrize("dtype,dk,dv", [(F32, 64, 72), (BF16, 128, 40), (F32, 104, 128), (BF16, 24, 64)])
def test_segments(dtype, dk, dv):
    """Sequences cut into segments, the last one short, dense and packed, with
    sequences shorter than a segment and empty ones."""
    c, d = make(2, 1, 2, 330, dk, dv, dtype, seed=14, g_scale=0.02)
    S0 = torch.randn(2, 2, dk, dv, generator=torch.Generator().manual_seed(9))
    ro, rS = ref.scan(*c, dk ** -0.5, S0)
    for seg in (-1, 64, 128):
        o, S = binding.gdr_scan(*d, S_in=S0.to(DEV), return_state=True, seg_len=seg)
        check(f"o seg {seg}", o, ro, TOL[dtype])
        check(f"S seg {seg}", S, rS, TOL[F32])
    cu = [0, 200, 200, 231, 329, 330]
    c, d = make(1, 1, 2, 330, dk, dv, dtype, seed=15, g_scale=0.02)
    S0 = torch.randn(5, 2, dk, dv, generator=torch.Generator().manual_seed(9))
    want = ref.packed(lambda *a: ref.scan(*a[:5], dk ** -0.5, a[5]), cu, c, [S0])
    o, S = binding.gdr_scan(*d, S_in=S0.to(DEV), return_state=True, seg_len=64,
                            cu_seqlens=torch.tensor(cu, device=DEV, dtype=torch.int32))
    check("packed o", o, torch.cat([w[0] for w in want], 2), TOL[dtype])
    check("packed S", S, torch.cat([w[1] for w in want]), TOL[F32])


def test_default_segments():
    """A long sequence of one head is cut by default."""
    c, d = make(1, 1, 1, 3000, 64, 16, F32, seed=16, g_scale=0.01)
    o, S = binding.gdr_scan(*d, return_state=True)
    ro, rS = ref.scan(*c, 0.125)
    check("o", o, ro, TOL[F32])
    check("S", S, rS, TOL[F32])
