"""Timed cases of the gated delta rule and of the query/key preparation.

The gated delta rule keeps one d_key x d_value state S per sequence and value
head.  A step with query q, key k, value v, log-decay g and write strength
beta does

    S <- e^g S;   u = beta (v - S^T k);   S <- S + k u^T;   o = scale S^T q

``scan`` runs it over whole sequences, ``grads`` is its adjoint, ``step``
advances a pool of states by a few tokens in place.  ``norm`` normalises the
queries and keys of every head and rotates them by their position, and
``norm_grads`` is the adjoint of that.

With ``own`` false, ``run`` evaluates the same maps with elementary torch
operations in float32: the recurrence in chunks of 64 steps (the products of
one chunk for all chunks at once, then one pass over the chunks that carries
the state).  ``exact`` takes one step at a time in float64.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
CHUNK = 64
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _seq(op, name=None, **kw):
    c = dict(op=op, dtype="bf16", B=1, L=1024, seqs=0, Hk=16, Hv=16, dk=128, dv=128, fused=False, state=True)
    if op == "step":
        c = dict(op=op, dtype="bf16", B=1, L=1, pool=0, Hk=16, Hv=16, dk=128, dv=128)
    c.update(kw)
    return c if name is None else {"name": name, **c}


def _norm(op, name=None, **kw):
    c = dict(op=op, dtype="bf16", B=1, L=1024, Hq=16, Hk=16, d=128, rot=64, kind="rms", interleaved=False, fused=True)
    c.update(kw)
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # One token of one conversation: the latency of a call.
        _seq("step", "step_one", B=1, Hk=16, Hv=32),
        # One token of a serving batch: a shuffled pool of states, a few rows of padding.
        _seq("step", "step_batch", B=128, pool=160, Hk=16, Hv=32),
        # Four drafted tokens at a time, everything in float32.
        _seq("step", "step_draft", B=24, L=4, pool=24, Hk=8, Hv=8, dk=64, dtype="f32"),
        # Prompts of very different lengths packed into one row, read from the fused projection's output.
        _seq("scan", "scan_prompts", L=6011, seqs=9, Hk=16, Hv=32, fused=True),
        # One layer of a training step.
        _seq("scan", "scan_train", B=4, L=4096, Hk=16, Hv=16, state=False),
        # The repository's long linear-attention workload (32 heads of 64 x 64, 131072 steps, float32).
        _seq("scan", "scan_rwkv128k", L=131072, Hk=32, Hv=32, dk=64, dv=64, dtype="f32"),
        # One long document on few heads (a model that is split over GPUs).
        _seq("scan", "scan_few_heads", L=32768, Hk=2, Hv=4),
        # The gradients of a training step with shared key heads.
        _seq("grads", "grads_train", B=2, L=4096, Hk=8, Hv=16, state=False),
        # Gradients of a ragged packed batch in float32, through the entry and final states.
        _seq("grads", "grads_ragged_f32", L=2777, seqs=5, Hk=3, Hv=6, dk=72, dv=104, dtype="f32"),
        # Queries and keys of a prompt, from the fused projection's output.
        _norm("norm", "norm_prefill", L=16384),
        # Queries and keys of one token of a serving batch.
        _norm("norm", "norm_step", B=64, L=1, kind="l2", rot=128),
        # Training: the gradients of the same, with those of the learned weights.
        _norm("norm_grads", "norm_grads_train", B=4, L=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["step", "scan", "scan", "grads", "norm", "norm_grads"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op in ("norm", "norm_grads"):
        d = rng.choice([32, 64, 72, 96, 128, 192, 256])
        H = _log(rng, 1, 32)
        B, L = _log(rng, 1, 64), _log(rng, 1, 16384)
        L = max(1, min(L, (1 << 25) // (B * H * d)))
        return _norm(op, B=B, L=L, Hq=H, Hk=rng.choice([H, max(1, H // 4)]), d=d, dtype=dtype,
                     rot=rng.choice([0, d // 2 // 16 * 16, d // 16 * 16]), kind=rng.choice(["rms", "l2"]),
                     interleaved=rng.random() < 0.4, fused=rng.random() < 0.5)
    Hk, r = _log(rng, 1, 24), rng.choice([1, 1, 2, 3])
    dk, dv = rng.choice([32, 64, 80, 128]), rng.choice([32, 64, 72, 128, 192])
    if op == "step":
        B = min(_log(rng, 1, 256), max(1, (1 << 26) // (Hk * r * dk * dv)))
        return _seq("step", B=B, L=rng.choice([1, 1, 2, 5]), pool=rng.choice([0, B + 3]), Hk=Hk, Hv=Hk * r, dk=dk,
                    dv=dv, dtype=dtype)
    most = (1 << 24) if op == "grads" else (1 << 26)        # elements of one of the large arrays
    seqs = rng.choice([0, 0, _log(rng, 1, 24)])
    B = 1 if seqs else _log(rng, 1, 8)
    L = max(1, min(_log(rng, 16, 32768 if op == "scan" else 8192), most // (B * Hk * r * max(dk, dv))))
    return _seq(op, B=B, L=L, seqs=seqs, Hk=Hk, Hv=Hk * r, dk=dk, dv=dv, dtype=dtype, fused=rng.random() < 0.5,
                state=rng.random() < 0.5)


def _lengths(case, seed):
    """Lengths of the packed sequences: log-spread, one of them empty or of one step where there are several."""
    n, L = case["seqs"], case["L"]
    gen = torch.Generator().manual_seed(seed * 7 + 1)
    w = torch.exp(3.0 * torch.rand(n, generator=gen))
    cuts = torch.floor(torch.cumsum(w, 0) / w.sum() * L + 0.5).long()
    cuts[-1] = L
    if n > 2:
        cuts[1] = min(int(cuts[0]) + seed % 2, L)
    return [0] + torch.cummax(cuts, 0).values.tolist()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device=DEV)

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device=DEV)

    def rows(B, L, *widths):
        """Parts [B, H, L, d] of one projection's output [B, L, sum H d] (or of arrays of their own)."""
        if not case.get("fused"):
            return [randn(B, h, L, d).to(dt) for h, d in widths]
        big = randn(B, L, sum(h * d for h, d in widths)).to(dt)
        out, at = [], 0
        for h, d in widths:
            out.append(big[..., at:at + h * d].unflatten(-1, (h, d)).transpose(1, 2))
            at += h * d
        return out

    B, L = case["B"], case["L"]
    s = {"case": case}
    if case["op"] in ("norm", "norm_grads"):
        d = case["d"]
        s["q"], s["k"] = rows(B, L, (case["Hq"], d), (case["Hk"], d))
        s["wq"], s["wk"] = (1 + 0.2 * randn(d), 1 + 0.2 * randn(d)) if case["kind"] == "rms" else (None, None)
        # a prompt starts anywhere in a long context; the largest position is beyond 2^17
        s["pos"] = (torch.randint(0, 1 << 18, (B, 1), generator=gen, device=DEV)
                    + torch.arange(L, device=DEV)).to(torch.int32)
        half = case["rot"] // 2
        s["inv"] = (torch.pow(10000.0, -torch.arange(half, device=DEV, dtype=torch.float64) / max(half, 1))
                    .to(torch.float32) if half else None)
        if case["op"] == "norm_grads":
            s["dq"], s["dk"] = randn(B, case["Hq"], L, d).to(dt), randn(B, case["Hk"], L, d).to(dt)
        return s
    Hk, Hv, dk, dv = (case[n] for n in ("Hk", "Hv", "dk", "dv"))
    q, k, v = rows(B, L, (Hk, dk), (Hk, dk), (Hv, dv))
    # What a short convolution and a SiLU leave: keys with a common part, then normalised per head.
    for x in (q, k):
        y = x.float() + 0.3
        x.copy_(y * torch.rsqrt(y.square().sum(-1, keepdim=True) + 1e-6))
    s["q"], s["k"], s["v"] = q, k, v
    c = math.log(1e-3) + rand(1, Hv, 1) * math.log(1e3)
    s["g"] = -torch.exp(c + 0.5 * randn(B, Hv, L))
    s["beta"] = torch.sigmoid(randn(B, Hv, L))
    if case["op"] == "step":
        pool = case["pool"]
        s["S"] = randn(pool or B, Hv, dk, dv) * 0.3
        if pool:
            slots = torch.randperm(pool, generator=gen, device=DEV)[:B].to(torch.int32)
            if B > 8:
                slots[B // 2::B // 4] = -1           # rows of padding
            s["slots"] = slots
        return s
    n = case["seqs"] or B
    if case["seqs"]:
        s["cu"] = _lengths(case, seed)
        s["cu_dev"] = torch.tensor(s["cu"], device=DEV, dtype=torch.int32)
    if case["state"]:
        s["S0"] = randn(n, Hv, dk, dv) * 0.3
    if case["op"] == "grads":
        s["do"] = randn(B, Hv, L, dv).to(dt)
        if case["state"]:
            s["dS1"] = randn(n, Hv, dk, dv) * 0.3
    return s


# ------------------------------------------------------------------ plain forms
def _pad_index(s, multiple):
    """Row of each (sequence, step) in a batch of equal length, and which of them exist."""
    cu = s["cu_dev"].long()
    most = max(b - a for a, b in zip(s["cu"], s["cu"][1:]))
    most = max(1, -(-most // multiple)) * multiple
    at = cu[:-1, None] + torch.arange(most, device=DEV)
    live = at < cu[1:, None]
    return at.clamp(max=max(s["cu"][-1] - 1, 0)), live


def _batched(s, names, dtype, multiple):
    """The inputs as [sequence, head, step, ..] in `dtype`, every row that is not there zero, heads of their own."""
    case, out = s["case"], {}
    r = case["Hv"] // case["Hk"]
    if case.get("seqs"):
        at, live = _pad_index(s, multiple)
    for n in names:
        x = s[n].to(dtype)
        if case.get("seqs"):
            x = x[0][:, at]                                        # [H, sequence, step, ..]
            x = (x * live.view(live.shape + (1,) * (x.dim() - 3))).transpose(0, 1)
        elif x.shape[2] % multiple:
            pad = multiple - x.shape[2] % multiple
            x = torch.nn.functional.pad(x, (0, 0) * (x.dim() - 3) + (0, pad))
        out[n] = x.repeat_interleave(r, 1) if n in ("q", "k") and r > 1 else x
    return out


def _unbatched(s, x):
    """[sequence, head, step, ..] back to the layout of the inputs."""
    case = s["case"]
    if not case.get("seqs"):
        return x[:, :, :case["L"]]
    at, live = _pad_index(s, x.shape[2])
    live = live[:, :x.shape[2]]
    return x.transpose(1, 2)[live].transpose(0, 1).unsqueeze(0)    # the sequences follow one another


def _chunks(b):
    """The products within all chunks at once: keys' products, decays, inverse of the unit triangle."""
    C = CHUNK
    c = {n: x.unflatten(2, (-1, C)) for n, x in b.items()}
    G = torch.cumsum(c["g"].double(), -1)
    dec = torch.exp((G[..., :, None] - G[..., None, :]).clamp(max=0).float()).tril()
    c["eG"], c["end"], c["out"] = torch.exp(G).float(), torch.exp(G[..., -1]).float(), torch.exp(G[..., -1:] - G).float()
    c["dec"], c["kk"] = dec, c["k"] @ c["k"].transpose(-1, -2)
    low = (c["beta"][..., None] * dec * c["kk"]).tril(-1)
    T = torch.eye(C, device=DEV).expand(low.shape).clone()
    for i in range(1, C):
        T[..., i, :i] = -(low[..., i, None, :i] @ T[..., :i, :i])[..., 0, :]
    c["T"], c["low"] = T, low
    return c


def _entry(s, name, b):
    return (s[name].clone() if s.get(name) is not None else
            torch.zeros(b["k"].shape[0], b["k"].shape[1], b["k"].shape[3], s["case"]["dv"], device=DEV))


def _plain_scan(s, keep=None):
    case = s["case"]
    b = _batched(s, ("q", "k", "v", "g", "beta"), torch.float32, CHUNK)
    c = _chunks(b)
    scale = case["dk"] ** -0.5
    W = c["T"] @ (c["beta"] * c["eG"])[..., None].mul(c["k"])
    U = c["T"] @ (c["beta"][..., None] * c["v"])
    A = c["dec"] * (c["q"] @ c["k"].transpose(-1, -2))
    qe, ko = c["q"] * c["eG"][..., None], (c["k"] * c["out"][..., None]).transpose(-1, -2)
    S, o, entry, vs = _entry(s, "S0", b), [], [], []
    for i in range(U.shape[2]):
        v2 = U[:, :, i] - W[:, :, i] @ S
        o.append(qe[:, :, i] @ S + A[:, :, i] @ v2)
        if keep is not None:
            entry.append(S)
            vs.append(v2)
        S = c["end"][:, :, i, None, None] * S + ko[:, :, i] @ v2
    if keep is not None:
        keep.update(c=c, A=A, entry=torch.stack(entry, 2), v2=torch.stack(vs, 2), b=b, S=S)
    return _unbatched(s, scale * torch.cat(o, 2)).to(DTYPES[case["dtype"]]), S


def _grouped(x, r):
    return x.unflatten(1, (-1, r)).sum(2) if r > 1 else x


def _plain_grads(s):
    case, f = s["case"], {}
    dt, scale, r = DTYPES[case["dtype"]], case["dk"] ** -0.5, case["Hv"] // case["Hk"]
    _plain_scan(s, f)
    c, v2, S0 = f["c"], f["v2"], f["entry"]
    do = _batched(s, ("do",), torch.float32, CHUNK)["do"].unflatten(2, (-1, CHUNK)) * scale
    t = lambda x: x.transpose(-1, -2)  # noqa: E731
    local = t(f["A"]) @ do
    TT = t(c["T"])
    be = c["beta"] * c["eG"]
    qd = t(c["q"] * c["eG"][..., None]) @ do
    kr, kw = t(c["k"] * be[..., None]), c["k"] * c["out"][..., None]
    dS, dS1, dR = _entry(s, "dS1", f["b"]), [], []
    for i in reversed(range(do.shape[2])):
        x = TT[:, :, i] @ (local[:, :, i] + kw[:, :, i] @ dS)
        dS1.append(dS)
        dR.append(x)
        dS = c["end"][:, :, i, None, None] * dS + qd[:, :, i] - kr[:, :, i] @ x
    dS1, dR = torch.stack(dS1[::-1], 2), torch.stack(dR[::-1], 2)
    S1 = torch.cat([S0[:, :, 1:], f["S"][:, :, None]], 2)
    dA = (do @ t(v2)).tril() * c["dec"]
    dL = -(dR @ t(v2)).tril(-1) * c["dec"]
    u = c["v"] - c["eG"][..., None] * (c["k"] @ S0)
    dbeta = (dR * u).sum(-1) + (dL * c["kk"]).sum(-1)
    dLb = dL * c["beta"][..., None]
    dq = c["eG"][..., None] * (do @ t(S0)) + dA @ c["k"]
    read = dLb @ c["k"] - be[..., None] * (dR @ t(S0))
    write = c["out"][..., None] * (v2 @ t(dS1)) + t(dA) @ c["q"] + t(dLb) @ c["k"]
    dG = (c["q"] * dq).sum(-1) + (c["k"] * read).sum(-1) - (c["k"] * write).sum(-1)
    dG[..., -1] += (dS1 * S1).sum((-1, -2))
    dg = torch.flip(torch.cumsum(torch.flip(dG, (-1,)), -1), (-1,))
    back = lambda x: _unbatched(s, x.flatten(2, 3))  # noqa: E731
    out = [_grouped(back(dq), r).to(dt), _grouped(back(read + write), r).to(dt),
           back(c["beta"][..., None] * dR).to(dt), back(dg), back(dbeta)]
    return out + [dS] if case["state"] else out


def _plain_step(s):
    case = s["case"]
    B, r, scale = case["B"], case["Hv"] // case["Hk"], case["dk"] ** -0.5
    q, k = (s[n].float().repeat_interleave(r, 1) for n in ("q", "k"))
    v, o = s["v"].float(), []
    slots = s["slots"].long() if case["pool"] else torch.arange(B, device=DEV)
    S, live = s["S"][slots.clamp(min=0)], (slots >= 0)[:, None, None]
    for t in range(case["L"]):
        S = torch.exp(s["g"][:, :, t])[..., None, None] * S
        kt = k[:, :, t, :, None]
        u = s["beta"][:, :, t, None] * (v[:, :, t] - (S * kt).sum(2))
        S = S + kt * u[:, :, None]
        o.append(torch.where(live, scale * (S * q[:, :, t, :, None]).sum(2), 0.0))
    keep = slots >= 0
    s["S"][slots[keep]] = S[keep]
    return torch.stack(o, 2).to(DTYPES[case["dtype"]]), s["S"]


def _rotation(s, dtype):
    ang = s["pos"].double()[..., None] * s["inv"].double()
    return torch.cos(ang).to(dtype)[:, None], torch.sin(ang).to(dtype)[:, None]


def _rotate(case, x, cos, sin, sign=1):
    rot = case["rot"]
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - sign * b * sin, b * cos + sign * a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - sign * b * sin, b * cos + sign * a * sin], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _norm_of(s, dtype, grads):
    """The preparation (or its adjoint) of q and k in `dtype`."""
    case, d, out, dws = s["case"], s["case"]["d"], [], []
    cs = _rotation(s, dtype) if case["rot"] else None
    for n, wn in (("q", "wq"), ("k", "wk")):
        x, w = s[n].to(dtype), s[wn]
        c = 1.0 / d if case["kind"] == "rms" else 1.0
        r = torch.rsqrt(x.square().sum(-1, keepdim=True) * c + 1e-6)
        if not grads:
            y = x * r if w is None else x * r * w.to(dtype)
            out.append(_rotate(case, y, *cs) if cs else y)
            continue
        du = s["d" + n].to(dtype)
        du = _rotate(case, du, *cs, sign=-1) if cs else du
        if w is not None:
            dws.append((du * x * r).sum((0, 1, 2)))
            du = du * w.to(dtype)
        out.append(r * (du - x * (r * r * c) * (x * du).sum(-1, keepdim=True)))
    return out, dws


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        from paper_2512_23068_amd import binding
        if op in ("norm", "norm_grads"):
            kw = dict(wq=s["wq"], wk=s["wk"], norm=case["kind"], positions=s["pos"], inv_freq=s["inv"],
                      interleaved=case["interleaved"])
            if op == "norm":
                return binding.qk_norm(s["q"], s["k"], **kw)
            return binding.qk_norm_grads(s["q"], s["k"], s["dq"], s["dk"], **kw)
        if op == "step":
            o = binding.gdr_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["S"], slots=s.get("slots"))
            return o, s["S"]
        kw = dict(S_in=s.get("S0"), cu_seqlens=s.get("cu_dev"))
        if op == "scan":
            return binding.gdr_scan(s["q"], s["k"], s["v"], s["g"], s["beta"], return_state=case["state"], **kw)
        return binding.gdr_grads(s["q"], s["k"], s["v"], s["g"], s["beta"], s["do"], dS_out=s.get("dS1"), **kw)
    if op == "step":
        return _plain_step(s)
    if op == "scan":
        o, S = _plain_scan(s)
        return (o, S) if case["state"] else o
    if op == "grads":
        return _plain_grads(s)
    out, dws = _norm_of(s, torch.float32, op == "norm_grads")
    return [x.to(DTYPES[case["dtype"]]) for x in out] + dws


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    B, L = case["B"], case["L"]
    if case["op"] in ("norm", "norm_grads"):
        n = B * L * (case["Hq"] + case["Hk"]) * case["d"]
        return {"bytes": n * e * (3 if case["op"] == "norm_grads" else 2) + 4 * B * L, "flops": n * 10}
    Hk, Hv, dk, dv = (case[n] for n in ("Hk", "Hv", "dk", "dv"))
    rows = B * L
    qk, vo, gates, cell = 2 * rows * Hk * dk * e, rows * Hv * dv * e, 2 * rows * Hv * 4, Hv * dk * dv * 4
    if case["op"] == "step":
        live = B - (len(range(B // 2, B, B // 4)) if case["pool"] and B > 8 else 0)
        return {"bytes": 2 * live * cell + qk + 2 * vo + gates, "flops": 8 * live * L * Hv * dk * dv}
    states = 2 * (case["seqs"] or B) * cell if case["state"] else 0
    if case["op"] == "scan":
        return {"bytes": qk + 2 * vo + gates + states, "flops": 8 * rows * Hv * dk * dv}
    return {"bytes": 2 * qk + 3 * vo + 2 * gates + 2 * states, "flops": 26 * rows * Hv * dk * dv}


# ------------------------------------------------------------------ float64
def _matvec(S, x):
    """S^T x per sequence and head."""
    return (x.unsqueeze(-2) @ S).squeeze(-2)


def exact(case, seed):
    """The definition, one step after the other in float64."""
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "norm_grads"):
        out, dws = _exact_norm(s)
        return out + dws
    scale = case["dk"] ** -0.5
    if op == "step":
        r = case["Hv"] // case["Hk"]
        b = {n: s[n].double() for n in ("v", "g", "beta")}
        b.update({n: s[n].double().repeat_interleave(r, 1) for n in ("q", "k")})
        slots = s["slots"].long() if case["pool"] else torch.arange(case["B"], device=DEV)
        rows = torch.nonzero(slots >= 0)[:, 0]
        b = {n: x[rows] for n, x in b.items()}
        pool = s["S"].double()
        S = pool[slots[rows]]
        o = torch.zeros(case["B"], case["Hv"], case["L"], case["dv"], device=DEV, dtype=torch.float64)
        for t in range(case["L"]):
            S, o[rows, :, t] = _exact_step(b, t, S, scale)
        pool[slots[rows]] = S
        return o, pool
    if s.get("cu"):
        r = case["Hv"] // case["Hk"]
        n, most = case["seqs"], max(b - a for a, b in zip(s["cu"], s["cu"][1:]))
        names = ("q", "k", "v", "g", "beta") + (("do",) if op == "grads" else ())
        b = {}
        for m in names:
            x = s[m][0].double()
            x = x.repeat_interleave(r, 0) if m in ("q", "k") else x
            y = torch.zeros((n, x.shape[0], max(most, 1)) + x.shape[2:], device=DEV, dtype=torch.float64)
            for i, (lo, hi) in enumerate(zip(s["cu"], s["cu"][1:])):
                y[i, :, :hi - lo] = x[:, lo:hi]
            b[m] = y
    else:
        r = case["Hv"] // case["Hk"]
        b = {m: s[m].double() for m in ("v", "g", "beta") + (("do",) if op == "grads" else ())}
        b.update({m: s[m].double().repeat_interleave(r, 1) for m in ("q", "k")})

    def back(x):
        if not s.get("cu"):
            return x
        return torch.cat([x[i, :, :hi - lo] for i, (lo, hi) in enumerate(zip(s["cu"], s["cu"][1:]))], 1)[None]

    N, H, L = b["g"].shape
    S = (s["S0"].double() if case["state"] else
         torch.zeros(N, H, case["dk"], case["dv"], device=DEV, dtype=torch.float64))
    if op == "scan":
        o = torch.empty(N, H, L, case["dv"], device=DEV, dtype=torch.float64)
        for t in range(L):
            S, o[:, :, t] = _exact_step(b, t, S, scale)
        return (back(o), S) if case["state"] else back(o)
    if N * H * L * case["dk"] * case["dv"] * 8 > 150e9:
        return None
    before = []
    for t in range(L):
        before.append(S)
        S, _ = _exact_step(b, t, S, scale)
    before.append(S)
    dS = s["dS1"].double() if case["state"] else torch.zeros_like(S)
    d = {m: torch.empty_like(b[m]) for m in ("q", "k", "v", "g", "beta")}
    for t in reversed(range(L)):
        k, q, beta = b["k"][:, :, t], b["q"][:, :, t], b["beta"][:, :, t, None]
        dec = torch.exp(b["g"][:, :, t])[..., None, None] * before[t]
        err = b["v"][:, :, t] - _matvec(dec, k)
        do = scale * b["do"][:, :, t]
        d["q"][:, :, t] = (before[t + 1] @ do.unsqueeze(-1)).squeeze(-1)
        dS = dS + q.unsqueeze(-1) * do.unsqueeze(-2)
        du = _matvec(dS, k)
        derr = beta * du
        d["beta"][:, :, t] = (du * err).sum(-1)
        d["v"][:, :, t] = derr
        d["k"][:, :, t] = (dS @ (beta * err).unsqueeze(-1) - dec @ derr.unsqueeze(-1)).squeeze(-1)
        dS = dS - k.unsqueeze(-1) * derr.unsqueeze(-2)
        d["g"][:, :, t] = (dS * dec).sum((-1, -2))
        dS = torch.exp(b["g"][:, :, t])[..., None, None] * dS
    r = case["Hv"] // case["Hk"]
    d = {m: back(x) for m, x in d.items()}
    out = [d["q"].unflatten(1, (-1, r)).sum(2), d["k"].unflatten(1, (-1, r)).sum(2), d["v"], d["g"], d["beta"]]
    return out + [dS] if case["state"] else out


def _exact_step(b, t, S, scale):
    k = b["k"][:, :, t]
    S = torch.exp(b["g"][:, :, t])[..., None, None] * S
    u = b["beta"][:, :, t, None] * (b["v"][:, :, t] - _matvec(S, k))
    S = S + k.unsqueeze(-1) * u.unsqueeze(-2)
    return S, scale * _matvec(S, b["q"][:, :, t])


def _exact_norm(s):
    """Pairs as complex numbers: a rotation is a product with e^{i angle}; gradients by differentiation of the map."""
    case, d, half = s["case"], s["case"]["d"], s["case"]["rot"] // 2
    if half:
        turn = torch.polar(torch.ones((), device=DEV, dtype=torch.float64),
                           s["pos"].double()[:, None, :, None] * s["inv"].double())

    def prep(x, w):
        n = x.square().sum(-1, keepdim=True)
        y = x / torch.sqrt((n / d if case["kind"] == "rms" else n) + 1e-6)
        y = y if w is None else y * w
        if not half:
            return y
        p, rest = y[..., :2 * half], y[..., 2 * half:]
        p = p.unflatten(-1, (half, 2)) if case["interleaved"] else p.unflatten(-1, (2, half)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(p.contiguous()) * turn)
        z = z if case["interleaved"] else z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), rest], -1)

    out, dws = [], []
    for n, wn in (("q", "wq"), ("k", "wk")):
        x, w = s[n].double(), None if s[wn] is None else s[wn].double()
        if case["op"] == "norm":
            out.append(prep(x, w))
            continue
        x.requires_grad_(True)
        if w is not None:
            w.requires_grad_(True)
        got = torch.autograd.grad(prep(x, w), [x] if w is None else [x, w], s["d" + n].double())
        out.append(got[0])
        dws += list(got[1:])
    return out, dws
