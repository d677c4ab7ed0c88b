"""Refusals of sd_rope and sd_kv_append (CPU: nothing is launched)."""

import ctypes

import pytest

import paper_2505_12728_amd as sd
from tests.test_abi import _fake, lib  # noqa: F401


def _sections(*n):
    return (ctypes.c_int32 * len(n))(*n)


@pytest.fixture
def rope(lib):
    keep, (x, pos, y) = _fake(3)
    # x and y 16 rows of 16 elements each, apart
    y = ctypes.c_void_p(x.value + 1024)

    def call(x=x, xs=16, pos=pos, y=y, ys=16, T=4, H=2, D=8, axes=1, secs=None, theta=1e4, freq=0, inv=0, dt=1):
        return lib.sd_rope(x, xs, pos, y, ys, T, H, D, axes, secs, theta, freq, inv, dt, None)
    call.x, call.keep = x, keep
    return call


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(pos=None), dict(y=None), dict(T=-1), dict(H=0), dict(D=0), dict(axes=0), dict(axes=-1),
    dict(dt=2), dict(freq=2), dict(theta=0.0), dict(theta=-1.0), dict(theta=float("nan")), dict(theta=float("inf")),
    dict(axes=2), dict(D=7, xs=64, ys=64), dict(xs=15), dict(ys=15), dict(xs=(1 << 32) + 1),
    dict(axes=2, secs=_sections(2, 0)), dict(axes=2, secs=_sections(2, 3)), dict(secs=_sections(5)),
    dict(axes=2, secs=_sections(2, -1)), dict(axes=2, secs=_sections(2147483647, 2147483647))])
def test_rope_invalid(rope, bad):
    assert rope(**bad) == sd.SD_ERR_INVALID_ARG


def test_rope_unsupported_and_misaligned(rope):
    assert rope(D=258, xs=1024, ys=1024) == sd.SD_ERR_UNSUPPORTED
    assert rope(axes=5, secs=_sections(*[1] * 5), D=16, xs=32, ys=32) == sd.SD_ERR_UNSUPPORTED
    assert rope(T=(1 << 30) + 1) == sd.SD_ERR_UNSUPPORTED
    assert rope(H=(1 << 20) + 1, xs=1 << 24, ys=1 << 24) == sd.SD_ERR_UNSUPPORTED
    assert rope(x=ctypes.c_void_p(rope.x.value + 1)) == sd.SD_ERR_INVALID_ARG
    assert rope(dt=0, y=ctypes.c_void_p(rope.x.value + 1026)) == sd.SD_ERR_INVALID_ARG


def test_rope_overlap_refused(rope):
    at = lambda n: ctypes.c_void_p(rope.x.value + n)          # noqa: E731
    assert rope(y=at(2)) == sd.SD_ERR_INVALID_ARG              # one element on
    assert rope(y=at(32)) == sd.SD_ERR_INVALID_ARG             # one row on
    assert rope(y=at(0), ys=32) == sd.SD_ERR_INVALID_ARG       # other stride
    assert rope(xs=40, ys=40, y=at(30)) == sd.SD_ERR_INVALID_ARG
    assert rope(xs=40, ys=40, y=at(50)) == sd.SD_ERR_INVALID_ARG   # reaches the next row of x
    assert rope(xs=40, ys=40, x=at(80 + 50), y=at(0)) == sd.SD_ERR_INVALID_ARG


def test_no_rows_launch_nothing(rope, lib):
    assert rope(T=0, x=None, pos=None, y=None) == sd.SD_OK
    assert lib.sd_kv_append(None, 0, None, 0, None, 0, None, None, None, None, None, None, 0, 0, 8, None, 0, 2, 4, 2,
                            8, 1, None, 1e4, 0, 1, 1, None) == sd.SD_OK


@pytest.fixture
def append(lib):
    keep, (q, k, v, qo, kc, vc, rs, kl, pt, pos) = _fake(10)
    base = dict(q=q, qs=32, k=k, ks=16, v=v, vs=16, qo=qo, kc=kc, vc=vc, rs=None, kl=kl, pt=None, mp=0, npg=0, lmax=64,
                pos=None, T=4, B=2, Hq=4, Hkv=2, D=8, axes=1, secs=None, theta=1e4, freq=0, sdt=1, dt=1)

    def call(**kw):
        a = dict(base, **kw)
        return lib.sd_kv_append(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["qo"], a["kc"], a["vc"], a["rs"],
                                a["kl"], a["pt"], a["mp"], a["npg"], a["lmax"], a["pos"], a["T"], a["B"], a["Hq"],
                                a["Hkv"], a["D"], a["axes"], a["secs"], a["theta"], a["freq"], a["sdt"], a["dt"], None)
    call.base, call.keep = base, keep
    return call


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(k=None), dict(v=None), dict(qo=None), dict(kc=None), dict(vc=None), dict(kl=None), dict(T=-1),
    dict(T=5), dict(B=0), dict(Hq=-1), dict(Hkv=0), dict(D=0), dict(axes=-1), dict(axes=2), dict(theta=0.0),
    dict(dt=3), dict(sdt=-1), dict(lmax=0), dict(qs=31), dict(ks=15), dict(vs=15), dict(ks=(1 << 32) + 1)])
def test_append_invalid(append, bad):
    assert append(**bad) == sd.SD_ERR_INVALID_ARG


def test_append_pages_and_types(append):
    pt = append.base["kl"]
    assert append(pt=pt, mp=0, npg=4) == sd.SD_ERR_INVALID_ARG
    assert append(pt=pt, mp=4, npg=0) == sd.SD_ERR_INVALID_ARG
    assert append(pt=pt, mp=(1 << 26) + 1, npg=4) == sd.SD_ERR_INVALID_ARG
    assert append(pt=ctypes.c_void_p(pt.value + 2), mp=4, npg=4) == sd.SD_ERR_INVALID_ARG
    assert append(sdt=1, dt=0) == sd.SD_ERR_UNSUPPORTED
    assert append(D=258, qs=2048, ks=2048, vs=2048) == sd.SD_ERR_UNSUPPORTED
    assert append(T=(1 << 30) + 2) == sd.SD_ERR_UNSUPPORTED
    assert append(Hkv=(1 << 20) + 1, ks=1 << 24, vs=1 << 24) == sd.SD_ERR_UNSUPPORTED


def test_append_overlapping_queries_refused(append):
    q, k = append.base["q"], append.base["k"]
    assert append(qo=ctypes.c_void_p(q.value + 2)) == sd.SD_ERR_INVALID_ARG
    assert append(qo=q, qs=40) == sd.SD_ERR_INVALID_ARG          # q strided, its output dense
    assert append(qo=q, sdt=0) == sd.SD_ERR_INVALID_ARG          # fp32 rows, bf16 output in their place
    assert append(qo=k) == sd.SD_ERR_INVALID_ARG
    assert append(qo=append.base["v"]) == sd.SD_ERR_INVALID_ARG


@pytest.fixture
def shared(lib):
    keep, (q, kc, vc, kl, pt, kp, vp, pl, ppt, gs, out, lse, ws) = _fake(13)
    base = dict(q=q, kc=kc, vc=vc, kl=kl, pt=None, mp=0, npg=0, lmax=64, kp=kp, vp=vp, pl=pl, ppt=None, pp=0, pn=0,
                plm=96, gs=None, out=out, lse=lse, B=4, k=4, Hq=8, Hkv=2, D=128, G=2, scale=0.1, dt=1, odt=0, ws=ws,
                wsb=1 << 34)
    order = list(base)

    def call(**kw):
        a = dict(base, **kw)
        return lib.sd_verify_shared(*[a[n] for n in order], None)
    call.base, call.keep = base, keep
    return call


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(kc=None), dict(vc=None), dict(kl=None), dict(kp=None), dict(vp=None), dict(pl=None),
    dict(out=None), dict(B=0), dict(k=0), dict(Hq=6, Hkv=4), dict(G=0), dict(G=3), dict(lmax=0), dict(plm=0),
    dict(dt=2), dict(odt=2), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_shared_invalid(shared, bad):
    assert shared(**bad) == sd.SD_ERR_INVALID_ARG


def test_shared_unsupported(shared, lib):
    for bad in (dict(k=17), dict(D=96), dict(Hq=512, Hkv=1), dict(dt=0, Hq=32, Hkv=1), dict(G=5), dict(dt=0, odt=1),
                dict(B=1 << 20, G=1 << 20, lmax=1 << 20), dict(B=1 << 28, Hq=8, Hkv=8, G=1),
                dict(Hq=1 << 17, Hkv=1 << 17)):
        assert shared(**bad) == sd.SD_ERR_UNSUPPORTED, bad
    assert shared(B=(1 << 16) + 1, k=1, Hq=1, Hkv=1, G=1) == sd.SD_ERR_UNSUPPORTED
    assert lib.sd_verify_shared_workspace_size((1 << 16) + 1, 1, 1, 1, 64, 1, 1, 1, 1) == 0
    assert lib.sd_verify_shared_workspace_size(1 << 16, 1, 1, 1, 64, 1, 1, 1, 1) > 0
    assert lib.sd_verify_shared_workspace_size(1 << 20, 4, 8, 2, 128, 1, 64, 1 << 20, 1) == 0
    assert lib.sd_verify_shared_workspace_size(4, 4, 8, 2, 128, 5, 64, 64, 1) == 0
    assert lib.sd_verify_shared_workspace_size(4, 4, 8, 2, 128, 4, 64, 64, 1) > 0


def test_shared_tables_alignment_and_workspace(shared):
    t = shared.base["kl"]
    assert shared(pt=t, mp=0, npg=1) == sd.SD_ERR_INVALID_ARG
    assert shared(pt=t, mp=1, npg=0) == sd.SD_ERR_INVALID_ARG
    assert shared(ppt=t, pp=0, pn=1) == sd.SD_ERR_INVALID_ARG
    assert shared(ppt=t, pp=1, pn=0) == sd.SD_ERR_INVALID_ARG
    assert shared(ppt=t, pp=(1 << 26) + 1, pn=1) == sd.SD_ERR_INVALID_ARG
    for name in ("q", "kc", "vc", "kp", "vp"):
        assert shared(**{name: ctypes.c_void_p(shared.base[name].value + 8)}) == sd.SD_ERR_INVALID_ARG, name
    for name in ("kl", "pl", "lse"):
        assert shared(**{name: ctypes.c_void_p(shared.base[name].value + 2)}) == sd.SD_ERR_INVALID_ARG, name
    assert shared(out=ctypes.c_void_p(shared.base["out"].value + 8)) == sd.SD_ERR_INVALID_ARG
    assert shared(gs=ctypes.c_void_p(t.value + 2)) == sd.SD_ERR_INVALID_ARG
    assert shared(ws=None) == sd.SD_ERR_WORKSPACE
    assert shared(wsb=64) == sd.SD_ERR_WORKSPACE
    assert shared(ws=ctypes.c_void_p(shared.base["ws"].value + 8)) == sd.SD_ERR_WORKSPACE
