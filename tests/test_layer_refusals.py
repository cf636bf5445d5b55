"""Arguments that the operators between a layer's products refuse, on the host, before anything is enqueued (no GPU)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2504_12984_amd import binding
    return binding


def _norm(B, **o):
    a = dict(x=16, residual=None, weight=16, eps=1e-5, act=B.QG_F16, M=1, N=64, xs=64, rs=0, A8=16, scale=16, sum=None, ss=0)
    a.update(o)
    return B._lib.qg_rmsnorm_a8(a["x"], a["residual"], a["weight"], a["eps"], a["act"], a["M"], a["N"], a["xs"], a["rs"], a["A8"],
                                a["scale"], a["sum"], a["ss"], None)


def test_norm_refusals(B):
    assert _norm(B, M=0) == B.QG_OK
    for bad in (dict(x=None), dict(weight=None), dict(A8=None), dict(scale=None), dict(eps=-1.0), dict(eps=float("nan")), dict(act=2),
                dict(M=-1), dict(N=0), dict(N=1 << 25), dict(xs=63), dict(residual=16, rs=63), dict(sum=16, ss=10), dict(x=17),
                dict(scale=18)):
        assert _norm(B, **bad) == B.QG_EINVAL, bad


def _silu(B, **o):
    a = dict(gate=16, up=32, act=B.QG_BF16, M=1, N=64, gs=128, us=128, A8=16, scale=16)
    a.update(o)
    return B._lib.qg_silu_a8(a["gate"], a["up"], a["act"], a["M"], a["N"], a["gs"], a["us"], a["A8"], a["scale"], None)


def test_gate_refusals(B):
    assert _silu(B, M=0) == B.QG_OK
    for bad in (dict(gate=None), dict(up=None), dict(A8=None), dict(scale=None), dict(act=-1), dict(M=-1), dict(N=0), dict(gs=63),
                dict(us=63), dict(up=33), dict(scale=2)):
        assert _silu(B, **bad) == B.QG_EINVAL, bad


def _kv(B, fn, **o):
    """All pointers are small integers: a call that is not refused would have to be one with nothing to do."""
    a = dict(q=16, k=16, v=16, act=B.QG_F16, qs=1024, ks=128, vs=128, cos=None, sin=None, positions=0, rot=0, neighbours=0,
             start=4, length=4, table=4, width=4, batch=1, rows=1, max_rows=1, Hq=8, H=1, D=128, t=B.WType(B.QG_INT, 8), blocks=4,
             kc=16, vc=16, ksc=4, vsc=4, out=16, out2=16, scale=0.1, causal=1, window=0, max_kv=0, stream=None)
    a.update(o)
    t = a["t"].c()
    if fn == "append":
        return B._lib.qg_kv_append(a["q"], a["k"], a["v"], a["act"], a["qs"], a["ks"], a["vs"], a["cos"], a["sin"], a["positions"],
                                   a["rot"], a["neighbours"], a["start"], a["length"], a["table"], a["width"], a["batch"], a["rows"],
                                   a["max_rows"], a["Hq"], a["H"], a["D"], t, a["blocks"], a["kc"], a["vc"], a["ksc"], a["vsc"],
                                   a["out"], a["stream"])
    if fn == "attention":
        return B._lib.qg_kv_attention(a["q"], a["act"], a["qs"], a["kc"], a["vc"], a["ksc"], a["vsc"], t, a["blocks"], a["start"],
                                      a["length"], a["table"], a["width"], a["batch"], a["rows"], a["max_rows"], a["max_kv"], a["Hq"],
                                      a["H"], a["D"], a["scale"], a["causal"], a["window"], a["out"], a["stream"])
    return B._lib.qg_kv_dequant(a["kc"], a["vc"], a["ksc"], a["vsc"], t, a["blocks"], a["start"], a["length"], a["table"], a["width"],
                                a["batch"], a["rows"], a["max_rows"], a["H"], a["D"], a["act"], a["out"], a["out2"], a["stream"])


@pytest.mark.parametrize("fn", ["append", "attention", "dequant"])
def test_cache_refusals(B, fn):
    for nothing in (dict(batch=0), dict(rows=0), dict(max_rows=0)):
        assert _kv(B, fn, **nothing) == B.QG_OK, nothing
    for bad in (dict(act=2), dict(H=0), dict(D=0), dict(batch=-1), dict(rows=-1), dict(max_rows=-1), dict(blocks=0), dict(width=0),
                dict(start=None), dict(length=None), dict(table=None), dict(kc=None), dict(vc=None), dict(ksc=None), dict(vsc=None),
                dict(kc=8), dict(vc=24), dict(ksc=2), dict(table=6), dict(out=None), dict(out=8), dict(t=B.WType(B.QG_INT, 9)),
                dict(t=B.WType(B.QG_FLOAT, 8, 4, 4))):
        assert _kv(B, fn, **bad) == B.QG_EINVAL, bad
    for none in (dict(D=32), dict(D=256), dict(t=B.WType(B.QG_INT, 4)), dict(t=B.WType(B.QG_UINT, 8)), dict(t=B.WType(B.QG_FLOAT, 6, 3, 2)),
                 dict(t=B.WType(B.QG_FLOAT, 8, 5, 2))):
        assert _kv(B, fn, **none) == B.QG_EUNSUPPORTED, none


def test_append_refusals(B):
    for bad in (dict(k=None), dict(v=None), dict(ks=127), dict(vs=0), dict(qs=1023), dict(Hq=0), dict(cos=16), dict(sin=16),
                dict(cos=16, sin=16, positions=0, rot=64), dict(cos=16, sin=16, positions=9, rot=63), dict(rot=130), dict(k=17),
                dict(cos=18, sin=16, positions=9, rot=64)):
        assert _kv(B, "append", **bad) == B.QG_EINVAL, bad


def test_attention_refusals(B):
    for bad in (dict(q=None), dict(Hq=7, H=2, qs=4096), dict(qs=1000), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
                dict(scale=float("nan")), dict(window=-1), dict(max_kv=-1), dict(q=17)):
        assert _kv(B, "attention", **bad) == B.QG_EINVAL, bad
    # the handle that names another stream in every thread
    assert _kv(B, "attention", stream=ctypes.c_void_p(2)) == B.QG_EINVAL
    assert b"hipStreamPerThread" in B._lib.qg_last_error()
