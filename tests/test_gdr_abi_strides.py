"""Strides, overlaps and sizes of the gated delta rule and the query/key preparation
that the host takes or refuses (no GPU needed)."""
import ctypes

import pytest

from paper_2512_23068_amd import binding
from tests.test_gdr_abi import A, GB, INVALID, OK, UNSUPPORTED, gdr, plan, qk


@pytest.mark.parametrize("kw,code", [
    (dict(), OK), (dict(o_strides=(6400 * 4, 6400, 64)), OK),                   # [B, H, L, d]
    (dict(o_strides=(64 * 4 * 100, 64, 64 * 4)), OK),                           # [B, L, H, d]
    (dict(o_strides=(64 * 4, 64, 64 * 8)), OK),                                 # [L, B, H, d]
    (dict(o_strides=(51200, 72, 512)), OK),                                     # padded rows
    (dict(o_strides=(25600, 72, 512)), INVALID),                                # (99 steps of 512 reach beyond 25600)
    (dict(o_strides=(25600, 6400, 56)), INVALID), (dict(o_strides=(25600, 6400, 8)), INVALID),       # rows over each other
    (dict(o_strides=(25600, 32, 256)), INVALID), (dict(o_strides=(25600, 64, 200)), INVALID),        # heads over steps
    (dict(o_strides=(6400, 6400, 64)), INVALID), (dict(o_strides=(512, 64, 256)), INVALID),          # batch entries
    (dict(batch=1, o_strides=(8, 6400, 64)), OK), (dict(seqlen=1, o_strides=(256, 64, 8)), OK),      # (do not move)
    (dict(v_strides=(25600, 6400, 8), q_strides=(0, 0, 8)), OK)])               # inputs may
def test_rows_of_outputs(kw, code):
    assert plan(gdr(**kw))[0] == code
    if "o_strides" in kw:
        p = gdr(grads=1, dv_strides=kw["o_strides"], **{n: x for n, x in kw.items() if n != "o_strides"})
        assert plan(p)[0] == code


@pytest.mark.parametrize("strides", [(2560, 640, 56), (2560, 32, 256), (512, 64, 256)])
def test_rows_of_prepared_queries(strides):
    good = [A + i * GB for i in range(4)]
    p = qk(q_out_strides=strides)
    assert binding.lib().pgf_qk_norm(good[0], good[1], ctypes.byref(p), good[2], good[3], None) == INVALID


def test_overlaps_of_preparation():
    """Outputs (the weights' gradients and the workspace among them) over any input,
    or over each other."""
    lib = binding.lib()
    at = {n: A + i * GB for i, n in enumerate(("q", "k", "dq", "dk", "q_out", "k_out", "w_q", "w_k", "inv_freq", "positions",
                                              "grad_w_q", "grad_w_k", "workspace"))}
    n = lib.pgf_qk_norm_workspace_bytes(ctypes.byref(qk(w_q=A, w_k=A)))

    def call(fn="pgf_qk_norm_grads", **move):
        x = {**at, **move}
        p = qk(pos_bits=64, pos_stride=10, workspace_bytes=n, **{k: x[k] for k in (
            "w_q", "w_k", "inv_freq", "positions", "grad_w_q", "grad_w_k", "workspace")})
        if fn == "pgf_qk_norm":
            return lib.pgf_qk_norm(x["q"], x["k"], ctypes.byref(p), x["q_out"], x["k_out"], None)
        return lib.pgf_qk_norm_grads(x["q"], x["k"], x["dq"], x["dk"], ctypes.byref(p), x["q_out"], x["k_out"], None)

    small = {"w_q": 256, "w_k": 256, "inv_freq": 128, "positions": 2 * 10 * 8, "grad_w_q": 256, "grad_w_k": 256}
    ins = ("q", "k", "dq", "dk", "w_q", "w_k", "inv_freq", "positions")
    for o in ("grad_w_q", "grad_w_k", "workspace", "q_out", "k_out"):
        for i in ins:
            # the output's first bytes on the input's last ones
            last = at[i] + (small[i] - 4 if i in small else 256)
            if o not in small:
                last = last // 256 * 256 if last % 256 else last
            if (o, i) in (("q_out", "q"), ("k_out", "k"), ("q_out", "dq"), ("k_out", "dk")):
                last = at[i] + 256                 # (on its own input it may lie, not beside)
            assert call(**{o: last}) == INVALID, (o, i)
    for o, i in (("grad_w_q", "grad_w_k"), ("grad_w_q", "q_out"), ("grad_w_k", "k_out"), ("grad_w_q", "workspace"),
                 ("workspace", "q_out"), ("workspace", "k_out")):
        assert call(**{o: at[i]}) == INVALID, (o, i)
    for i in ("w_q", "w_k", "inv_freq", "positions"):
        assert call("pgf_qk_norm", q_out=at[i]) == INVALID, i


def _packed(fn, **kw):
    """A packed call of made-up addresses that is refused for what kw says (or for its workspace)."""
    p = gdr(batch=1, n_seqs=3, **kw)
    x = [A + i * GB for i in range(11)]
    lib = binding.lib()
    if fn == "pgf_gdr_scan":
        return lib.pgf_gdr_scan(*x[:5], ctypes.byref(p), x[5], None)
    return lib.pgf_gdr_grads(*x[:6], ctypes.byref(p), *x[6:], None)


@pytest.mark.parametrize("fn", ["pgf_gdr_scan", "pgf_gdr_grads"])
def test_bounds_of_packed_sequences_are_inputs(fn):
    """cu_seqlens under an output, a state that is written, or the workspace."""
    n = binding.lib().pgf_gdr_workspace_bytes(ctypes.byref(gdr(batch=1, n_seqs=3, grads=1)))
    ws = dict(workspace=A + 20 * GB, workspace_bytes=n)
    for o in range(5, 6) if fn == "pgf_gdr_scan" else range(6, 11):
        assert _packed(fn, cu_seqlens=A + o * GB, **ws) == INVALID, o
    assert _packed(fn, cu_seqlens=A + 20 * GB + 64, **ws) == INVALID
    state = "S_out" if fn == "pgf_gdr_scan" else "dS_in"
    assert _packed(fn, cu_seqlens=A + 30 * GB + 4, **{state: A + 30 * GB}, **ws) == INVALID


def test_addresses_of_small_arrays():
    """States, bounds, slots and f32 gradients at addresses that are no multiple of
    their element."""
    n = binding.lib().pgf_gdr_workspace_bytes(ctypes.byref(gdr(batch=1, n_seqs=3, grads=1)))
    ws = dict(workspace=A + 20 * GB, workspace_bytes=n, cu_seqlens=A + 40 * GB)
    x = [A + i * GB for i in range(11)]
    lib = binding.lib()
    for kw in (dict(S_in=A + 30 * GB + 2), dict(S_out=A + 30 * GB + 1), dict(cu_seqlens=A + 30 * GB + 2)):
        p = gdr(batch=1, n_seqs=3, **{**ws, **kw})
        assert lib.pgf_gdr_scan(*x[:5], ctypes.byref(p), x[5], None) == INVALID, kw
    for kw in (dict(S_in=A + 30 * GB + 2), dict(dS_out=A + 30 * GB + 1), dict(dS_in=A + 30 * GB + 2),
               dict(cu_seqlens=A + 30 * GB + 2)):
        p = gdr(batch=1, n_seqs=3, **{**ws, **kw})
        assert lib.pgf_gdr_grads(*x[:6], ctypes.byref(p), *x[6:], None) == INVALID, kw
    for o in (9, 10):
        y = [a + 2 * (i == o) for i, a in enumerate(x)]
        p = gdr(batch=1, n_seqs=3, **ws)
        assert lib.pgf_gdr_grads(*y[:6], ctypes.byref(p), *y[6:], None) == INVALID, o
    p = gdr(seqlen=1, S_pool=A + 20 * GB, pool=2, slots=A + 30 * GB + 2)
    assert lib.pgf_gdr_step(*x[:5], ctypes.byref(p), x[5], None) == INVALID
    m = lib.pgf_qk_norm_workspace_bytes(ctypes.byref(qk(w_q=A, w_k=A)))
    good = dict(w_q=A + 10 * GB, w_k=A + 11 * GB, inv_freq=A + 12 * GB, positions=A + 13 * GB, grad_w_q=A + 14 * GB,
                grad_w_k=A + 15 * GB)
    for bits in (32, 64):
        for name in good:
            p = qk(**{**good, name: good[name] + (4 if name == "positions" and bits == 64 else 2)}, pos_bits=bits, pos_stride=10,
                   workspace=A + 20 * GB, workspace_bytes=m)
            assert lib.pgf_qk_norm_grads(*x[:4], ctypes.byref(p), x[4], x[5], None) == INVALID, (name, bits)


@pytest.mark.parametrize("name", ["g_strides", "beta_strides"])
def test_steps_of_gates(name):
    """A step's stride is below 2^24 bytes: 2^22 elements of f32."""
    for step, code in (((1 << 22) - 1, OK), (1 << 21, OK), (1 << 22, UNSUPPORTED)):
        assert plan(gdr(**{name: (0, 0, step)}))[0] == code, step


@pytest.mark.parametrize("Hk,Hv", [(4, 4), (2, 4), (1, 1)])
def test_workspace_of_gradients(Hk, Hv):
    """Records, states and errors with their adjoints; sums over value heads only
    where a key head has several."""
    B, L, dk, dv = 3, 150, 72, 40
    p = gdr(batch=B, key_heads=Hk, value_heads=Hv, seqlen=L, d_key=dk, d_value=dv, grads=1, seg_len=-1)
    chunks, runs = B * -(-L // 32), B * -(-L // 64)
    parts = [chunks * Hv * (9 * 1024 + 256)] + 2 * [runs * Hv * dk * dv * 4] + 2 * [chunks * Hv * 32 * dv * 4]
    parts += [runs * Hk * 2 * 64 * dk * 4] if Hv > Hk else []
    assert binding.lib().pgf_gdr_workspace_bytes(ctypes.byref(p)) == sum(-(-x // 256) * 256 for x in parts)
