"""Host-side checks of the gated delta rule and the query/key preparation (no GPU
needed): the parameter blocks' layout, sizes and strides that are refused before
anything is launched, and the plans."""
import ctypes
import random

import pytest

from paper_2512_23068_amd import binding

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
A = 1 << 40          # addresses that are never touched: every call below is refused first
GB = 1 << 30


def gdr(**kw):
    p = binding.PgfGdrParams()
    v = dict(batch=2, key_heads=2, value_heads=4, seqlen=100, d_key=64, d_value=64, in_dtype=1, scale=1.0)
    v.update(kw)
    for n, x in v.items():
        if n.endswith("strides"):
            getattr(p, n)[:] = x
        else:
            setattr(p, n, x)
    return p


def plan(p):
    seg = ctypes.c_int32(-7)
    return binding.lib().pgf_gdr_plan(ctypes.byref(p), ctypes.byref(seg)), seg.value


def test_packed_blocks_are_the_structs():
    for pack, struct in ((binding._GDR_PACK, binding.PgfGdrParams), (binding._QK_PACK, binding.PgfQkParams)):
        assert pack.size == ctypes.sizeof(struct)
    p = binding.PgfGdrParams.from_buffer_copy(binding._GDR_PACK.pack(
        *range(1, 7), 7, 8, 9, 10, 0.5, 12, 22, *range(100, 127), 13, 14, 15, 16, 17, 18, 19, 20, 21))
    assert (p.batch, p.d_value, p.n_seqs, p.cu_seqlens, p.in_dtype, p.seg_len, p.scale, p.grads,
            p.clear_rest) == (1, 6, 7, 8, 9, 10, 0.5, 12, 22)
    assert list(p.q_strides) == [100, 101, 102] and list(p.dv_strides) == [124, 125, 126]
    assert (p.S_in, p.dS_in, p.S_pool, p.pool, p.slots, p.workspace, p.workspace_bytes) == (13, 16, 17, 18, 19, 20, 21)
    p = binding.PgfQkParams.from_buffer_copy(binding._QK_PACK.pack(
        *range(1, 7), 7, 2, 1, 0.5, *range(100, 118), 20, 21, 22, 23, 64, 25, 26, 27, 28, 29))
    assert (p.batch, p.rot, p.in_dtype, p.norm, p.interleaved, p.eps) == (1, 6, 7, 2, 1, 0.5)
    assert list(p.dk_strides) == [115, 116, 117]
    assert (p.w_q, p.positions, p.pos_bits, p.pos_stride, p.grad_w_k, p.workspace_bytes) == (20, 23, 64, 25, 27, 29)


@pytest.mark.parametrize("kw,code", [
    (dict(), OK), (dict(seqlen=0), OK), (dict(d_key=8, d_value=8), OK), (dict(d_key=128, d_value=4096), OK),
    (dict(batch=0), INVALID), (dict(key_heads=0), INVALID), (dict(value_heads=3), INVALID), (dict(seqlen=-1), INVALID),
    (dict(d_key=0), INVALID), (dict(in_dtype=2), INVALID), (dict(n_seqs=-1), INVALID), (dict(n_seqs=2), INVALID),
    (dict(clear_rest=2), OK), (dict(clear_rest=3), INVALID), (dict(clear_rest=-1), INVALID),
    (dict(n_seqs=2, batch=1), OK), (dict(seg_len=-2), INVALID), (dict(seg_len=32), INVALID), (dict(seg_len=64), OK),
    (dict(d_key=12), UNSUPPORTED), (dict(d_key=136), UNSUPPORTED), (dict(d_value=4), UNSUPPORTED),
    (dict(d_value=4104), UNSUPPORTED), (dict(batch=1 << 25), UNSUPPORTED), (dict(seqlen=1 << 33), UNSUPPORTED),
    (dict(batch=1 << 24, value_heads=1 << 16, key_heads=1), UNSUPPORTED),
    (dict(q_strides=(-8, 8, 8)), INVALID), (dict(q_strides=(0, 4, 8)), INVALID), (dict(q_strides=(0, 8, 64)), OK),
    (dict(in_dtype=0, v_strides=(0, 4, 64)), OK), (dict(o_strides=(0, 64, 256)), INVALID), (dict(g_strides=(0, 0, 1)), OK),
    (dict(k_strides=(8, 8, 1 << 23)), UNSUPPORTED), (dict(k_strides=(1 << 45, 8, 64)), INVALID)])
def test_sizes_and_strides(kw, code):
    p = gdr(**kw)
    rc, seg = plan(p)
    assert rc == code
    n = binding.lib().pgf_gdr_workspace_bytes(ctypes.byref(p))
    assert (n > 0) == (code == OK)
    if code == OK:
        assert seg >= 0 and seg % 64 == 0
        p.grads = 1
        assert binding.lib().pgf_gdr_workspace_bytes(ctypes.byref(p)) >= n


def test_null_arguments():
    lib = binding.lib()
    assert lib.pgf_gdr_workspace_bytes(None) == 0 and lib.pgf_qk_norm_workspace_bytes(None) == 0
    assert lib.pgf_gdr_plan(None, ctypes.byref(ctypes.c_int32())) == INVALID
    assert lib.pgf_gdr_plan(ctypes.byref(gdr()), None) == INVALID
    assert lib.pgf_gdr_scan(*[None] * 5, None, None, None) == INVALID


def _call(p, ptrs, fn="pgf_gdr_scan"):
    """A call with made-up addresses: q, k, v, g, beta, o (and do, gradients)."""
    lib = binding.lib()
    if fn == "pgf_gdr_grads":
        q, k, v, g, b, do, dq, dk, dv, dg, db = ptrs
        return lib.pgf_gdr_grads(q, k, v, g, b, do, ctypes.byref(p), dq, dk, dv, dg, db, None)
    q, k, v, g, b, o = ptrs
    return getattr(lib, fn)(q, k, v, g, b, ctypes.byref(p), o, None)


def test_scan_refusals():
    n = binding.lib().pgf_gdr_workspace_bytes(ctypes.byref(gdr()))
    good = [A + i * GB for i in range(6)]
    assert _call(gdr(), good) == WORKSPACE
    assert _call(gdr(workspace=A + 9 * GB, workspace_bytes=n - 1), good) == WORKSPACE
    assert _call(gdr(workspace=A + 9 * GB + 16, workspace_bytes=n), good) == WORKSPACE
    ws = dict(workspace=A + 9 * GB, workspace_bytes=n)
    for i in range(6):
        bad = list(good)
        bad[i] = None
        assert _call(gdr(**ws), bad) == INVALID, i
        bad[i] = good[i] + 2                                   # not aligned
        assert _call(gdr(**ws), bad) == INVALID, i
    for i in range(5):                                         # o over an input, the workspace over anything
        assert _call(gdr(**ws), good[:5] + [good[i] + 16]) == INVALID, i
        assert _call(gdr(workspace=good[i], workspace_bytes=n), good) == INVALID, i
    assert _call(gdr(workspace=good[5], workspace_bytes=n), good) == INVALID
    assert _call(gdr(n_seqs=3, batch=1, **ws), good) == INVALID          # no cu_seqlens
    assert _call(gdr(S_out=good[0], **ws), good) == INVALID
    assert _call(gdr(S_out=good[5], **ws), good) == INVALID
    assert _call(gdr(S_in=A + 20 * GB, S_out=A + 20 * GB + 256, **ws), good) == INVALID


def test_step_refusals():
    good = [A + i * GB for i in range(6)]
    ok = dict(S_pool=A + 20 * GB, pool=2, seqlen=1)
    for kw in (dict(pool=1), dict(pool=-1), dict(S_pool=None), dict(S_pool=A + 20 * GB + 4), dict(S_pool=good[0]),
               dict(S_pool=good[5]), dict(n_seqs=1, batch=1)):
        assert _call(gdr(**{**ok, **kw}), good, "pgf_gdr_step") == INVALID, kw
    assert _call(gdr(**ok), good[:5] + [good[2]], "pgf_gdr_step") == INVALID
    assert _call(gdr(pool=1, S_pool=A + 20 * GB, seqlen=1, slots=good[5]), good, "pgf_gdr_step") == INVALID
    assert _call(gdr(**{**ok, "d_key": 12}), good, "pgf_gdr_step") == UNSUPPORTED


def test_grads_refusals():
    n = binding.lib().pgf_gdr_workspace_bytes(ctypes.byref(gdr(grads=1)))
    good = [A + i * GB for i in range(11)]
    fn = "pgf_gdr_grads"
    assert _call(gdr(), good, fn) == WORKSPACE
    ws = dict(workspace=A + 20 * GB, workspace_bytes=n)
    for i in range(11):
        bad = list(good)
        bad[i] = None
        assert _call(gdr(**ws), bad, fn) == INVALID, i
    for o in range(6, 11):
        for i in range(6):
            bad = list(good)
            bad[o] = good[i]
            assert _call(gdr(**ws), bad, fn) == INVALID, (o, i)
        assert _call(gdr(workspace=good[o], workspace_bytes=n), good, fn) == INVALID
        assert _call(gdr(dS_in=good[o], **ws), good, fn) == (INVALID if o > 8 else INVALID), o
    for o, i in ((6, 7), (7, 8), (6, 8), (9, 10), (9, 6)):
        bad = list(good)
        bad[o] = good[i]
        assert _call(gdr(**ws), bad, fn) == INVALID, (o, i)
    assert _call(gdr(dq_strides=(0, 64, 128), **ws), good, fn) == INVALID       # rows on each other


def qk(**kw):
    p = binding.PgfQkParams()
    v = dict(batch=2, q_heads=4, k_heads=2, seqlen=10, d_head=64, rot=64, in_dtype=1, norm=2, eps=1e-6, inv_freq=A)
    v.update(kw)
    for n, x in v.items():
        if n.endswith("strides"):
            getattr(p, n)[:] = x
        else:
            setattr(p, n, x)
    return p


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), INVALID), (dict(q_heads=0, k_heads=0), INVALID), (dict(q_heads=-1), INVALID), (dict(d_head=0), INVALID),
    (dict(seqlen=-1), INVALID), (dict(rot=-16), INVALID), (dict(rot=80), INVALID), (dict(inv_freq=None), INVALID),
    (dict(norm=3), INVALID), (dict(norm=-1), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(in_dtype=5), INVALID), (dict(positions=A, pos_bits=16), INVALID), (dict(pos_stride=-1), INVALID),
    (dict(d_head=20, rot=16), UNSUPPORTED), (dict(d_head=520), UNSUPPORTED), (dict(rot=24), UNSUPPORTED),
    (dict(batch=1 << 20, seqlen=1 << 20), UNSUPPORTED), (dict(q_strides=(8, 8, 4)), INVALID),
    (dict(q_out_strides=(0, 64, 64)), INVALID)])
def test_qk_refusals(kw, code):
    good = [A + i * GB for i in range(2)], [A + i * GB for i in range(2, 4)]
    lib = binding.lib()
    assert lib.pgf_qk_norm(*good[0], ctypes.byref(qk(**kw)), *good[1], None) == code


def test_qk_pointers():
    lib = binding.lib()
    q, k, qo, ko, dq, dk = [A + i * GB for i in range(6)]

    def call(a, b, c, d, **kw):
        return lib.pgf_qk_norm(a, b, ctypes.byref(qk(**kw)), c, d, None)

    assert call(None, k, qo, ko) == INVALID and call(q, k, qo, None) == INVALID
    assert call(q + 2, k, qo, ko) == INVALID and call(q, k, qo, ko + 8) == INVALID
    assert call(q, k, q + 16, ko) == INVALID          # over an input, not on it
    assert call(q, k, k, ko) == INVALID and call(q, k, qo, qo) == INVALID
    g = lambda **kw: lib.pgf_qk_norm_grads(q, k, dq, dk, ctypes.byref(qk(**kw)), qo, ko, None)  # noqa: E731
    assert g(w_q=A + 7 * GB) == INVALID               # no place for its gradient
    assert g(w_q=A + 7 * GB, grad_w_q=A + 8 * GB) == WORKSPACE
    n = lib.pgf_qk_norm_workspace_bytes(ctypes.byref(qk(w_q=A + 7 * GB)))
    assert n > 0 and lib.pgf_qk_norm_workspace_bytes(ctypes.byref(qk())) == 0
    assert g(w_q=A + 7 * GB, grad_w_q=A + 8 * GB, workspace=qo, workspace_bytes=n) == INVALID
    assert lib.pgf_qk_norm_grads(q, k, None, dk, ctypes.byref(qk()), qo, ko, None) == INVALID


def test_random_plans():
    """Any sizes are refused with a status or give a workspace that holds at least the records, and whole segments."""
    rng = random.Random(3)
    for _ in range(2000):
        r = rng.choice([1, 2, 3, 8])
        kw = dict(batch=rng.randint(1, 300), key_heads=rng.randint(1, 64), seqlen=int(2 ** rng.uniform(0, 21)),
                  d_key=8 * rng.randint(1, 17), d_value=8 * rng.randint(1, 520), in_dtype=rng.randint(0, 1),
                  grads=rng.randint(0, 1), seg_len=rng.choice([0, 0, -1, 64, 128, 4096, 100]))
        kw["value_heads"] = kw["key_heads"] * r
        if rng.random() < 0.3:
            kw.update(batch=1, n_seqs=rng.randint(1, 1000))
        p = gdr(**kw)
        rc, seg = plan(p)
        n = binding.lib().pgf_gdr_workspace_bytes(ctypes.byref(p))
        assert rc in (OK, INVALID, UNSUPPORTED) and (n > 0) == (rc == OK)
        if rc == OK:
            assert seg == 0 or (seg % 64 == 0 and seg < kw["seqlen"])
            chunks = kw["batch"] * -(-kw["seqlen"] // 32)
            assert n >= chunks * kw["value_heads"] * 6400 or kw.get("n_seqs")
