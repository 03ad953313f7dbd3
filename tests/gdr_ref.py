"""The gated delta rule and the query/key preparation in float64 on the CPU,
one step after the other, from their definitions (gradients by autograd)."""
import torch


def scan(q, k, v, g, beta, scale, S0=None):
    """q, k [B,Hk,L,dk], v [B,Hv,L,dv], g, beta [B,Hv,L] -> o [B,Hv,L,dv], S [B,Hv,dk,dv]."""
    q, k, v, g, beta = (x.double() for x in (q, k, v, g, beta))
    r = v.shape[1] // q.shape[1]
    q, k = q.repeat_interleave(r, 1), k.repeat_interleave(r, 1)
    B, H, L, dk = q.shape
    S = torch.zeros(B, H, dk, v.shape[3], dtype=torch.float64) if S0 is None else S0.double()
    o = []
    for t in range(L):
        S = torch.exp(g[:, :, t])[..., None, None] * S
        u = beta[:, :, t, None] * (v[:, :, t] - torch.einsum("bhij,bhi->bhj", S, k[:, :, t]))
        S = S + k[:, :, t, :, None] * u[:, :, None]
        o.append(scale * torch.einsum("bhij,bhi->bhj", S, q[:, :, t]))
    o = torch.stack(o, 2) if L else torch.zeros(v.shape, dtype=torch.float64)
    return o, S


def packed(fn, cu, args, states):
    """fn on each packed sequence: args [1,H,T,..] cut by cu, states [n,..] one each."""
    outs = []
    for i, (a, b) in enumerate(zip(cu, cu[1:])):
        outs.append(fn(*[x[:, :, a:b] for x in args], *[None if s is None else s[i:i + 1] for s in states]))
    return outs


def qk_prep(x, w, norm, eps, positions, inv_freq, interleaved):
    """x [B,H,L,d] -> prepared, in float64."""
    x = x.double()
    d = x.shape[-1]
    n = x.square().sum(-1, keepdim=True)
    if norm != "none":
        x = x / torch.sqrt((n / d if norm == "rms" else n) + eps)
    if w is not None:
        x = x * w.double()
    if inv_freq is None:
        return x
    half = inv_freq.numel()
    ang = positions.double().reshape(-1, 1, x.shape[2], 1) * inv_freq.double()
    cos, sin = torch.cos(ang), torch.sin(ang)
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., 2 * half:]], -1)


def rel(got, ref):
    """||got - ref|| / ||ref|| in float64."""
    got, ref = got.detach().double().cpu(), ref.detach().double()
    assert got.shape == ref.shape, (got.shape, ref.shape)
    den = float(ref.norm())
    return float((got - ref).norm()) / (den if den > 0 else 1.0)
