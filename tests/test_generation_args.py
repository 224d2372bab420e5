"""Refusals of uc_linear_attend, uc_beam_select and uc_reorder: every bad
argument is turned down before anything is launched (CPU)."""
import ctypes as C

import pytest
import torch

from paper_2609_32831_gb300 import _lib, api

FAKE = 1 << 20
LIB = _lib.lib


@pytest.fixture(autouse=True)
def nothing_launched():
    n0 = LIB().uc_launch_count()
    yield
    assert LIB().uc_launch_count() == n0


def _rows(ptr=FAKE, sb=4096 * 128, sh=128 * 64, st=128):
    return C.byref(_lib.UcRows(ptr, sb, sh, st))


def _linear(**kw):
    a = dict(q=_rows(FAKE), k=_rows(2 * FAKE), v=_rows(3 * FAKE), B=2, hq=4, hkv=2, T=10, lengths=None,
             decay=(C.c_float * 2)(-0.1, -0.2), s_in=None, s_out=5 * FAKE, out=_rows(4 * FAKE), ws=8 * FAKE, wn=256)
    a.update(kw)
    if kw.get("wn") is None:
        a["wn"] = max(256, LIB().uc_linear_workspace_size(a["B"], a["hq"], a["hkv"], a["T"]))
    return LIB().uc_linear_attend(a["q"], a["k"], a["v"], a["B"], a["hq"], a["hkv"], a["T"], a["lengths"], a["decay"],
                                  a["s_in"], a["s_out"], a["out"], a["ws"], a["wn"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), "SHAPE"), (dict(B=65), "SHAPE"), (dict(hq=5), "SHAPE"), (dict(hq=1), "SHAPE"), (dict(hkv=0), "SHAPE"),
    (dict(T=0), "SHAPE"), (dict(q=None), "ARG"), (dict(k=_rows(0)), "ARG"), (dict(v=_rows(FAKE + 8)), "ARG"),
    (dict(out=_rows(0)), "ARG"), (dict(q=_rows(st=64)), "SHAPE"), (dict(k=_rows(st=132)), "SHAPE"),
    (dict(v=_rows(sh=-128)), "SHAPE"), (dict(q=_rows(sb=0)), "SHAPE"), (dict(decay=None), "ARG"),
    (dict(decay=(C.c_float * 2)(-0.1, 0.1)), "ARG"), (dict(decay=(C.c_float * 2)(float("nan"), -1)), "ARG"),
    (dict(decay=(C.c_float * 2)(-1, float("-inf"))), "ARG"), (dict(s_out=None), "ARG"), (dict(s_out=FAKE + 4), "ARG"),
    (dict(s_in=5 * FAKE + 4096), "ARG"), (dict(lengths=(C.c_int32 * 2)(3, 11)), "SHAPE"),
    (dict(lengths=(C.c_int32 * 2)(-1, 3)), "SHAPE"), (dict(out=_rows(FAKE)), "ARG"), (dict(ws=None), "ARG"),
    (dict(ws=8 * FAKE + 8), "ARG"), (dict(wn=16), "OOM")])
def test_linear_attend(kw, code):
    assert _linear(**kw) == getattr(_lib, "UC_ERR_" + code)
    assert b"linear_attend" in LIB().uc_last_error()


def _beam(**kw):
    a = dict(x=FAKE, dtype=_lib.BF16, sb=4000, sk=1000, B=2, K=4, V=1000, scores=2 * FAKE, fin=None, eos=-1, n=4,
             os=3 * FAKE, op=4 * FAKE, ot=5 * FAKE, of=None, ws=8 * FAKE, wn=1 << 20)
    a.update(kw)
    return LIB().uc_beam_select(a["x"], a["dtype"], a["sb"], a["sk"], a["B"], a["K"], a["V"], a["scores"], a["fin"],
                                a["eos"], a["n"], a["os"], a["op"], a["ot"], a["of"], a["ws"], a["wn"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), "ARG"), (dict(B=0), "SHAPE"), (dict(K=0), "SHAPE"), (dict(K=33), "SHAPE"), (dict(V=0), "SHAPE"),
    (dict(n=0), "SHAPE"), (dict(n=33), "SHAPE"), (dict(K=1, V=3, n=4), "SHAPE"), (dict(B=20000), "SHAPE"),
    (dict(sk=999), "SHAPE"), (dict(sb=0), "SHAPE"), (dict(x=None), "ARG"), (dict(x=FAKE + 1), "ARG"),
    (dict(scores=None), "ARG"), (dict(os=None), "ARG"), (dict(op=None), "ARG"), (dict(ot=FAKE + 2), "ARG"),
    (dict(eos=1000), "ARG"), (dict(eos=-2), "ARG"), (dict(fin=FAKE), "ARG"), (dict(ws=None), "ARG"),
    (dict(wn=300), "OOM")])
def test_beam_select(kw, code):
    assert _beam(**kw) == getattr(_lib, "UC_ERR_" + code)
    assert b"beam_select" in LIB().uc_last_error()


def _segs(kind=_lib.KIND_EVICT, bits=16, S=4, hkv=2, cap=64, base=1):
    """A segment whose arrays are made-up addresses far apart."""
    c = _lib.UcSegment()
    c.kind, c.bits, c.batch, c.n_kv_heads, c.head_dim, c.n_src, c.cap = kind, bits, S, hkv, 128, 100, cap
    for i, name in enumerate(("n_kept", "kept_idx", "k", "v", "k_codes", "k_params", "v_codes", "v_params")):
        setattr(c, name, (base * 16 + i) << 30)
    packed = kind in (_lib.KIND_QUANT, _lib.KIND_EVICT_QUANT)
    c.row_stride = 32 if packed else cap
    c.rows_total = S * hkv * c.row_stride
    return c


def _reorder(src, dst, parent=FAKE, G=2, n_from=2, n_to=2, ws=2 * FAKE, wn=256, state=(None, None, 0)):
    item = _lib.UcReorderItem(None if src is None else C.addressof(src), None if dst is None else C.addressof(dst), *state)
    return LIB().uc_reorder(C.byref(item), 1, parent, G, n_from, n_to, ws, wn, None)


def test_reorder_segments():
    a, b = _segs(), _segs(base=2)
    for kw in (dict(parent=None), dict(parent=FAKE + 1), dict(ws=None)):
        assert _reorder(a, b, **kw) == _lib.UC_ERR_ARG
    assert _reorder(a, b, wn=128) == _lib.UC_ERR_OOM
    for kw in (dict(G=0), dict(n_from=0), dict(n_to=0), dict(G=4), dict(n_from=4), dict(n_to=3), dict(G=70000)):
        assert _reorder(a, b, **kw) == _lib.UC_ERR_SHAPE
    assert _reorder(a, None) == _lib.UC_ERR_ARG
    assert _reorder(None, None) == _lib.UC_ERR_ARG
    assert _reorder(a, b, state=(FAKE, 2 * FAKE, 4)) == _lib.UC_ERR_ARG
    assert _reorder(a, a) == _lib.UC_ERR_ARG                       # itself
    c = _segs(base=2)
    c.v = a.v + 1024
    assert _reorder(a, c) == _lib.UC_ERR_ARG                       # shared rows
    assert _reorder(a, _segs(cap=32, base=2)) == _lib.UC_ERR_SHAPE
    assert _reorder(a, _segs(hkv=1, base=2)) == _lib.UC_ERR_SHAPE
    assert _reorder(a, _segs(_lib.KIND_EVICT_QUANT, 4, base=2)) == _lib.UC_ERR_SHAPE
    assert _reorder(_segs(_lib.KIND_QUANT, 4), _segs(_lib.KIND_QUANT, 2, base=2)) == _lib.UC_ERR_SHAPE
    c = _segs(base=2)
    c.n_src = 99
    assert _reorder(a, c) == _lib.UC_ERR_SHAPE
    c = _segs()
    c.n_kept_host[1] = 5                                           # beams of one group differ
    assert _reorder(c, b) == _lib.UC_ERR_SHAPE
    c = _segs(base=2)
    c.rows_total -= 1
    assert _reorder(a, c) == _lib.UC_ERR_SHAPE
    c = _segs(base=2)
    c.kept_idx = None
    assert _reorder(a, c) == _lib.UC_ERR_ARG
    assert b"uc_reorder" in LIB().uc_last_error()


def test_reorder_states():
    for state, code in (((FAKE, 2 * FAKE, 0), "SHAPE"), ((FAKE, 2 * FAKE, 6), "SHAPE"),
                        ((FAKE + 2, 2 * FAKE, 8), "SHAPE"), ((FAKE, 2 * FAKE, 1 << 33), "SHAPE"),
                        ((FAKE, None, 8), "ARG"), ((FAKE, FAKE, 64), "ARG"), ((FAKE, FAKE + 192, 64), "ARG")):
        assert _reorder(None, None, state=state) == getattr(_lib, "UC_ERR_" + code)


def test_binding_refuses_what_the_library_cannot_see():
    bf = torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16)
    ws = api.Workspace("cpu")
    for q, k, ld in ((bf.float(), bf, [-1, -1]), (bf, bf[..., :64], [-1, -1]), (bf, bf[:, :, :3], [-1, -1]),
                     (bf, bf, [-1]), (bf, bf.transpose(2, 3).contiguous().transpose(2, 3), [-1, -1])):
        with pytest.raises(ValueError):
            api.linear_attend(q, k, k, ld, ws=ws)
    with pytest.raises(ValueError):
        api.linear_attend(bf, bf, bf, [-1, -1], state=torch.zeros((1, 2, 128, 64)), ws=ws)
    with pytest.raises(ValueError):
        api.linear_attend(bf, bf, bf, [-1, -1], lengths=[4, 4], ws=ws)
    x, s = torch.zeros((2, 3, 10)), torch.zeros((2, 3))
    for bad in ((x.double(), s, None), (x, s.double(), None), (x, s[:, :2], None), (x[:, :, ::2], s, None),
                (x, s, torch.zeros((2, 3)))):
        with pytest.raises(ValueError):
            api.beam_select(bad[0], bad[1], 2, finished=bad[2], eos=0, ws=ws)
    p = torch.zeros((2, 3), dtype=torch.int32)
    for pairs, parent in (([(x, x[:1])], p), ([(torch.zeros(6, 2), torch.zeros(6, 3))], p), ([], p),
                          ([(torch.zeros(6, 2), torch.zeros(6, 2))], p.long()),
                          ([(torch.zeros(5, 2), torch.zeros(6, 2))], p),
                          ([(torch.zeros(6, 2), torch.zeros(6, 2)), (torch.zeros(4, 2), torch.zeros(6, 2))], p)):
        with pytest.raises(ValueError):
            api.reorder(pairs, parent, ws=ws)
