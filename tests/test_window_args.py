"""Refusals of uc_rotary, uc_window_append, uc_window_attend and uc_verify_draft:
every bad argument is turned down before anything is launched (CPU)."""
import ctypes as C

import pytest
import torch

from paper_2609_32831_gb300 import _lib, api

FAKE = 1 << 30
LIB = _lib.lib


@pytest.fixture(autouse=True)
def nothing_launched():
    n0 = LIB().uc_launch_count()
    yield
    assert LIB().uc_launch_count() == n0


def _rows(i, sb=64 * 128 * 4, sh=64 * 128, st=128, off=0):
    return C.byref(_lib.UcRows(i * FAKE + off, sb, sh, st))


def _table(n=64, inter=0, scale=1.0, f=1.0):
    t = _lib.UcRotaryTable(n, inter, scale)
    for i in range(64):
        t.freq[i] = f
    return C.byref(t)


def _rotary(**kw):
    a = dict(table=_table(), pos=9 * FAKE, per=1, dtype=_lib.BF16, B=2, T=10, q=_rows(1), qo=_rows(2), hq=4, k=_rows(3),
             ko=_rows(4), hkv=2)
    a.update(kw)
    return LIB().uc_rotary(a["table"], a["pos"], a["per"], a["dtype"], a["B"], a["T"], a["q"], a["qo"], a["hq"], a["k"],
                           a["ko"], a["hkv"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), "ARG"), (dict(dtype=-1), "ARG"), (dict(table=None), "ARG"), (dict(table=_table(0)), "ARG"),
    (dict(table=_table(65)), "ARG"), (dict(table=_table(inter=2)), "ARG"), (dict(table=_table(scale=float("inf"))), "ARG"),
    (dict(table=_table(f=float("nan"))), "ARG"), (dict(table=_table(f=2.0 ** 31)), "ARG"), (dict(pos=None), "ARG"),
    (dict(pos=9 * FAKE + 2), "ARG"), (dict(B=0), "SHAPE"), (dict(T=0), "SHAPE"), (dict(hq=0), "SHAPE"),
    (dict(hkv=0), "SHAPE"), (dict(B=65535, T=1 << 28), "SHAPE"), (dict(B=1 << 30, T=1 << 30, hq=14), "SHAPE"), (dict(q=None), "ARG"), (dict(qo=None), "ARG"),
    (dict(ko=None), "ARG"), (dict(k=None), "ARG"), (dict(q=_rows(1, off=8)), "ARG"), (dict(q=_rows(1, st=64)), "SHAPE"),
    (dict(qo=_rows(2, sb=0)), "SHAPE"), (dict(k=_rows(3, st=132)), "SHAPE"), (dict(qo=_rows(1, off=256)), "ARG"),
    (dict(ko=_rows(2)), "ARG"), (dict(ko=_rows(1)), "ARG"), (dict(qo=_rows(9)), "ARG"),
    (dict(qo=_rows(2, st=64 * 128)), "ARG")])
def test_rotary(kw, code):
    assert _rotary(**kw) == getattr(_lib, "UC_ERR_" + code)
    assert b"uc_rotary" in LIB().uc_last_error()


def _cache(k=1, v=2, B=2, hkv=2, rows=64, window=16, sinks=4, sb=2 * 64 * 128, koff=0):
    c = _lib.UcWindowCache(_lib.UcRows(k * FAKE + koff, sb, 64 * 128, 128), _lib.UcRows(v * FAKE, sb, 64 * 128, 128), B,
                           hkv, rows, window, sinks)
    return C.byref(c)


CACHES = [(dict(cache=None), "ARG"), (dict(cache=_cache(B=0)), "SHAPE"), (dict(cache=_cache(hkv=0)), "SHAPE"),
          (dict(cache=_cache(rows=0)), "SHAPE"), (dict(cache=_cache(window=0)), "SHAPE"),
          (dict(cache=_cache(sinks=-1)), "SHAPE"),
          (dict(cache=_cache(sb=0)), "SHAPE"), (dict(cache=_cache(koff=8)), "ARG"),
          (dict(cache=_cache(rows=(1 << 30) + 1)), "SHAPE")]


def _append(**kw):
    a = dict(cache=_cache(), k=_rows(3), v=_rows(4), T=10, held=5 * FAKE, n_new=None, table=_table(), q=_rows(6),
             qo=_rows(7), hq=4, total=8 * FAKE, ws=9 * FAKE, wn=256)
    a.update(kw)
    return LIB().uc_window_append(a["cache"], a["k"], a["v"], a["T"], a["held"], a["n_new"], a["table"], a["q"], a["qo"],
                                  a["hq"], a["total"], a["ws"], a["wn"], None)


@pytest.mark.parametrize("kw,code", CACHES + [
    (dict(cache=_cache(v=1)), "ARG"), (dict(k=None), "ARG"), (dict(v=_rows(0)), "ARG"), (dict(T=0), "SHAPE"),
    (dict(held=None), "ARG"), (dict(held=5 * FAKE + 1), "ARG"), (dict(total=None), "ARG"), (dict(total=5 * FAKE), "ARG"),
    (dict(total=5 * FAKE + 4), "ARG"), (dict(n_new=8 * FAKE), "ARG"), (dict(table=None), "ARG"), (dict(table=_table(65)), "ARG"),
    (dict(q=None), "ARG"), (dict(qo=None), "ARG"), (dict(hq=0), "SHAPE"), (dict(k=_rows(1)), "ARG"), (dict(v=_rows(1)), "ARG"),
    (dict(q=_rows(2), qo=_rows(2)), "ARG"), (dict(qo=_rows(3)), "ARG"), (dict(total=FAKE + 64), "ARG"),
    (dict(total=3 * FAKE), "ARG"), (dict(ws=None), "ARG"), (dict(ws=9 * FAKE + 8), "ARG"), (dict(wn=16), "OOM")])
def test_window_append(kw, code):
    assert _append(**kw) == getattr(_lib, "UC_ERR_" + code)
    assert b"uc_window_append" in LIB().uc_last_error()


def _attend(**kw):
    a = dict(cache=_cache(), q=_rows(3), hq=4, T=10, lengths=5 * FAKE, n_query=None, out=_rows(6), lse=7 * FAKE,
             ws=9 * FAKE, wn=1 << 28)
    a.update(kw)
    return LIB().uc_window_attend(a["cache"], a["q"], a["hq"], a["T"], a["lengths"], a["n_query"], a["out"], a["lse"],
                                  a["ws"], a["wn"], None)


@pytest.mark.parametrize("kw,code", CACHES + [
    (dict(q=None), "ARG"), (dict(out=None), "ARG"), (dict(hq=3), "SHAPE"), (dict(hq=1), "SHAPE"), (dict(T=0), "SHAPE"),
    (dict(T=1 << 29), "SHAPE"), (dict(lengths=None), "ARG"), (dict(lengths=5 * FAKE + 2), "ARG"), (dict(lse=7 * FAKE + 1), "ARG"),
    (dict(out=_rows(3)), "ARG"), (dict(out=_rows(1)), "ARG"), (dict(out=_rows(2, off=128 * 128)), "ARG"),
    (dict(out=_rows(5)), "ARG"), (dict(out=_rows(7)), "ARG"), (dict(lse=5 * FAKE), "ARG"), (dict(lse=3 * FAKE), "ARG"),
    (dict(n_query=7 * FAKE), "ARG"), (dict(out=_rows(6, st=64)), "SHAPE"), (dict(ws=None), "ARG"), (dict(wn=64), "OOM")])
def test_window_attend(kw, code):
    assert _attend(**kw) == getattr(_lib, "UC_ERR_" + code)
    assert b"uc_window_attend" in LIB().uc_last_error()


def _verify(**kw):
    a = dict(x=FAKE, xb=6000, xt=1000, y=2 * FAKE, yb=5000, yt=1000, dtype=_lib.BF16, B=2, T=5, V=1000, tok=3 * FAKE, n=None,
             u=4 * FAKE, e=5 * FAKE, tau=1.0, acc=6 * FAKE, out=7 * FAKE, lp=8 * FAKE, ws=9 * FAKE, wn=1 << 24)
    a.update(kw)
    return LIB().uc_verify_draft(a["x"], a["xb"], a["xt"], a["y"], a["yb"], a["yt"], a["dtype"], a["B"], a["T"], a["V"],
                                 a["tok"], a["n"], a["u"], a["e"], a["tau"], a["acc"], a["out"], a["lp"], a["ws"], a["wn"],
                                 None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), "ARG"), (dict(B=0), "SHAPE"), (dict(T=0), "SHAPE"), (dict(T=65), "SHAPE"), (dict(V=0), "SHAPE"),
    (dict(B=30000), "SHAPE"), (dict(xt=999), "SHAPE"), (dict(xb=0), "SHAPE"), (dict(yt=0), "SHAPE"), (dict(yb=0), "SHAPE"),
    (dict(x=None), "ARG"), (dict(x=FAKE + 1), "ARG"), (dict(y=2 * FAKE + 1), "ARG"), (dict(tok=None), "ARG"),
    (dict(u=None), "ARG"), (dict(e=None), "ARG"), (dict(e=5 * FAKE + 2), "ARG"), (dict(tau=-1.0), "ARG"),
    (dict(tau=float("nan")), "ARG"), (dict(tau=float("inf")), "ARG"), (dict(tau=1e-9), "ARG"), (dict(acc=None), "ARG"),
    (dict(out=None), "ARG"), (dict(lp=8 * FAKE + 2), "ARG"), (dict(acc=3 * FAKE), "ARG"), (dict(out=FAKE + 64), "ARG"),
    (dict(lp=7 * FAKE), "ARG"), (dict(n=6 * FAKE), "ARG"), (dict(ws=None), "ARG"), (dict(ws=9 * FAKE + 8), "ARG"),
    (dict(wn=256), "OOM")])
def test_verify_draft(kw, code):
    assert _verify(**kw) == getattr(_lib, "UC_ERR_" + code)
    assert b"uc_verify_draft" in LIB().uc_last_error()


def test_workspace_sizes():
    assert LIB().uc_window_workspace_size(None, 4, 1) == 0
    assert LIB().uc_window_workspace_size(_cache(), 3, 1) == 0
    assert LIB().uc_window_workspace_size(_cache(), 4, 0) == 0
    assert LIB().uc_window_workspace_size(_cache(), 4, 1) >= 256
    assert LIB().uc_verify_workspace_size(0, 1, 1) == 0
    assert LIB().uc_verify_workspace_size(1, 1, 1) >= 256


def test_binding_refuses_what_the_library_cannot_see():
    bf = torch.zeros((2, 2, 4, 128), dtype=torch.bfloat16)
    n = torch.zeros(2, dtype=torch.int32)
    p = torch.zeros((2, 4), dtype=torch.int32)
    ws = api.Workspace("cpu")
    turn = api.Rotary([1.0, 0.5])
    for f in ([], [1.0] * 65):
        with pytest.raises(ValueError):
            api.Rotary(f)
    cut = bf.transpose(2, 3).contiguous().transpose(2, 3)
    for q, k, at in ((bf.double(), bf, p), (bf[..., :64], bf, p), (bf, bf.float(), p), (bf, bf[:, :, :3], p), (bf, bf, p.long()),
                     (bf, bf, p[:, :3]), (cut, bf, p), (bf, cut, p), (bf, bf, p)):      # (the last: not on a GPU)
        with pytest.raises(ValueError):
            api.rotary(turn, at, q, k)
    for bad in (dict(k=bf.float()), dict(v=bf[:, :1]), dict(k=cut), dict(window=0), dict(n_sink=-1)):
        with pytest.raises(ValueError):
            api.WindowCache(**{**dict(k=bf, v=bf.clone(), window=2, n_sink=1), **bad})
    c = api.WindowCache(bf, bf.clone(), 2, 1)
    for bad in (dict(k=bf.float()), dict(v=bf[:1]), dict(held=n.long()), dict(held=n[:1]), dict(n_new=n[:1]), dict(q=bf),
                dict(q=bf[:1], rotary=turn), dict(out_q=bf), dict(held=None), dict(total=n[:1]), dict()):
        with pytest.raises(ValueError):
            api.window_append(**{**dict(cache=c, k=bf.clone(), v=bf.clone(), held=n, ws=ws), **bad})
    for bad in (dict(q=bf.float()), dict(q=bf[:1]), dict(q=cut), dict(lengths=n.long()), dict(n_query=n[:1]),
                dict(lse=torch.zeros(2, 2, 3)), dict()):
        with pytest.raises(ValueError):
            api.window_attend(**{**dict(q=bf.clone(), cache=c, lengths=n, ws=ws), **bad})
    x, t = torch.zeros((2, 3, 10)), torch.zeros((2, 2), dtype=torch.int32)
    u, e = torch.zeros((2, 2)), torch.ones((2, 10))
    for bad in (dict(logits=x.double()), dict(logits=x[..., ::2]), dict(tokens=t.long()), dict(tokens=t[:, :1]), dict(u=None),
                dict(noise=None), dict(u=u.double()), dict(noise=e[:, :9]), dict(draft_logits=x), dict(n_draft=n.long()),
                dict(draft_logits=x[:, :2].half()), dict()):
        with pytest.raises(ValueError):
            api.verify_draft(**{**dict(logits=x, tokens=t, u=u, noise=e, ws=ws), **bad})
