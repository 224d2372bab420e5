"""The cache of a layer with a sliding window, and attention over it, against fp64:
rings, first tokens, windows of one token, lengths from none on, ragged
prompts, groups of heads, strides; what is masked does not reach a query."""
import numpy as np
import pytest
import torch

from oracle import rotary as orot
from oracle import window as owin
from tests.test_gpu_rotary import bound as rotary_bound
from tests.test_gpu_rotary import freqs_of, rows

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")
from paper_2609_32831_gb300 import _lib  # noqa: E402

DEV = "cuda"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make_cache(g, B, hkv, n_rows, lengths, sinks, strided=False):
    """Rows that hold no token are NaN."""
    k, v = (rows(g, B, hkv, n_rows, "cut" if strided else "bhtd") for _ in range(2))
    for b in range(B):
        free = sorted(set(range(n_rows)) - set(owin.held_tokens(lengths[b], sinks, n_rows)))
        k[b, :, free] = v[b, :, free] = float("nan")
    return k, v


def check(out, lse, want, steps):
    """A logit is within 2^-20 of sum |q k| / sqrt(128) (128 products, summed in fp32 and cut), so its
    exponential is within d = 2^-19 reach + 2^-20; p enters the product with v with 16 bits (up to 8 query rows of a KV
    head) or rounded to bf16, at most 2^-8 off; the output is rounded once more. lse: its logits' error, the sum's and its own."""
    o, l, spread, reach = want
    d = 2.0 ** -19 * reach + 2.0 ** -20
    err = (2 * d[..., None] + (2.0 ** -16 if steps else 2.0 ** -8)) * spread
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    far = np.abs(got - o) - (err + 2.0 ** -8 * (np.abs(o) + err) + 1e-30)
    assert (far <= 0).all(), float(far.max())
    if lse is not None:
        ls = lse.double().cpu().numpy()
        none = np.isneginf(l)
        assert np.isneginf(ls[none]).all() and (got[none] == 0).all()
        some = ~none
        assert (np.abs(ls[some] - l[some]) <= d[some] + 2.0 ** -19 + 2.0 ** -22 * np.abs(l[some])).all()


# B, hq, hkv, T, window, sinks, rows, lengths, n_query
RINGS = [
    (1, 28, 4, 1, 16, 4, 24, [100], None),
    (3, 4, 4, 1, 1, 0, 1, [1, 5, 77], None),                    # the query's own token alone
    (3, 7, 1, 1, 10, 3, 13, [0, 1, 12], None),                  # none, one, not yet full
    (2, 16, 2, 5, 1000, 3, 1011, [3333, 1009], None),           # drafts; one ring about to wrap
    (4, 8, 2, 3, 7, 4, 13, [3, 6, 13, 14], None),
    (2, 12, 4, 8, 33, 0, 40, [41, 500], [8, 3]),
    (5, 6, 2, 4, 20, 100, 123, [0, 4, 99, 105, 1000], [4, 4, 0, 2, 1]),
    (2, 28, 4, 8, 200, 17, 300, [90, 2000], None),              # 56 rows
    (2, 65, 1, 1, 50, 4, 64, [64, 65], None),                   # more heads of a group than a CTA's rows
    (1, 4, 2, 2, 64, 5, 6, [50], None),                         # a ring of one row: the last token alone is left
    (3, 4, 2, 4, 8, 2, 64, [2, 3, 1], [4, 4, 4]),               # more queries than tokens
    (2, 4, 1, 2, 1 << 30, 0, 700, [700, 333], None),            # a window that nothing leaves
]


@pytest.mark.parametrize("B,hq,hkv,T,window,sinks,n_rows,lengths,n_query", RINGS)
@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_steps(B, hq, hkv, T, window, sinks, n_rows, lengths, n_query, layout):
    g = torch.Generator(device=DEV).manual_seed(window + T)
    k, v = make_cache(g, B, hkv, n_rows, lengths, sinks, layout == "bthd")
    q = rows(g, B, hq, T, layout)
    ws = uc.Workspace(DEV)
    out, lse = uc.window_attend(q, uc.WindowCache(k, v, window, sinks), ints(lengths),
                                None if n_query is None else ints(n_query), ws=ws)
    want = owin.attend(q.float().cpu().numpy(), k.float().cpu().numpy(), v.float().cpu().numpy(), lengths,
                       [T] * B if n_query is None else n_query, window, sinks)
    assert ws.status() == _lib.UC_OK and out.stride() == q.stride()
    check(out, lse, want, hq // hkv * T <= 8)


PROMPTS = [
    (1, 4, 4, 9, 4, 0, 9, [9], None),
    (2, 28, 4, 33, 1 << 30, 0, 40, [33, 40], None),
    (3, 4, 2, 129, 16, 4, 130, [129, 0, 1], [129, 0, 1]),
    (2, 16, 16, 300, 64, 20, 301, [300, 150], [300, 150]),
    (2, 7, 1, 100, 50, 3, 200, [200, 163], [100, 63]),
    (1, 4, 1, 257, 128, 130, 700, [700], None),                  # more first tokens than a tile
    (2, 6, 2, 70, 130, 5, 5 + 130 + 70, [1000, 205], None),      # a ring
    (1, 2, 2, 400, 1, 1, 400, [400], None),
    (2, 4, 1, 513, 300, 9, 1100, [1000, 1100], None),
    (1, 40, 1, 260, 200, 8, 600, [555], None),
    (1, 8, 1, 70, 1 << 30, 5, 3000, [2999], None),               # few queries over many keys: split over keys
    (2, 130, 1, 2, 700, 5, 1200, [900, 1150], [2, 1]),           # more heads of a group than a tile's rows
    (2, 16, 1, 9, 600, 200, 900, [5000, 870], [9, 4]),           # a ring whose end and start lie in reach, first tokens too
]


@pytest.mark.parametrize("B,hq,hkv,T,window,sinks,n_rows,lengths,n_query", PROMPTS)
@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_prompts(B, hq, hkv, T, window, sinks, n_rows, lengths, n_query, layout):
    g = torch.Generator(device=DEV).manual_seed(window + T)
    k, v = make_cache(g, B, hkv, n_rows, lengths, sinks, layout == "bthd")
    q = rows(g, B, hq, T, layout)
    ws = uc.Workspace(DEV)
    out, lse = uc.window_attend(q, uc.WindowCache(k, v, window, sinks), ints(lengths),
                                None if n_query is None else ints(n_query), ws=ws)
    want = owin.attend(q.float().cpu().numpy(), k.float().cpu().numpy(), v.float().cpu().numpy(), lengths,
                       [T] * B if n_query is None else n_query, window, sinks)
    assert ws.status() == _lib.UC_OK and out.stride() == q.stride()
    check(out, lse, want, False)


@pytest.mark.parametrize("T,hq,hkv", [(5, 4, 2), (300, 4, 2), (300, 3, 3)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_nonfinite_tokens_reach_only_who_sees_them(T, hq, hkv, bad):
    """A token's k and v (one channel) turn bad: queries before it and past its window keep their outputs."""
    g = torch.Generator(device=DEV).manual_seed(3)
    window, sinks, n = 20, 2, 400
    k, v = make_cache(g, 1, hkv, n, [n], sinks)
    q = rows(g, 1, hq, T, "bhtd")
    cache = uc.WindowCache(k, v, window, sinks)
    want, lse = uc.window_attend(q, cache, ints([n]))
    at = n - T + T // 2
    pos = torch.arange(n - T, n, device=DEV)
    sees = (pos >= at) & (pos - at < window)
    old = v[0, 1, at, 77].clone()
    v[0, 1, at, 77] = bad
    got, l2 = uc.window_attend(q, cache, ints([n]))
    grp = hq // hkv
    assert torch.equal(got[:, :grp], want[:, :grp]) and torch.equal(l2, lse)
    assert not torch.isfinite(got[0, grp:2 * grp, sees, 77]).any()
    same = torch.ones(128, dtype=torch.bool, device=DEV)
    same[77] = False
    # (a row taken alone differs by roundings: two bf16 steps of its largest output)
    step = 2.0 ** -6 * float(want.abs().max())
    assert float((got[0, grp:2 * grp][:, sees][..., same] - want[0, grp:2 * grp][:, sees][..., same]).abs().max()) <= step
    assert float((got[0, :, ~sees] - want[0, :, ~sees]).abs().max()) <= step
    v[0, 1, at, 77] = old
    k[0, 1, at, 5] = bad
    got, l2 = uc.window_attend(q, cache, ints([n]))
    assert torch.equal(got[0, :, ~sees], want[0, :, ~sees]) and torch.equal(l2[0, :, ~sees], lse[0, :, ~sees])


def test_no_lse_and_given_outputs():
    g = torch.Generator(device=DEV).manual_seed(4)
    for T in (2, 140):
        k, v = make_cache(g, 2, 2, 200, [150, 200], 3)
        q = rows(g, 2, 4, T, "bhtd")
        cache = uc.WindowCache(k, v, 50, 3)
        want, lse = uc.window_attend(q, cache, ints([150, 200]))
        out = torch.full((2, T, 4, 128), 7.0, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
        got, none = uc.window_attend(q, cache, ints([150, 200]), out=out, want_lse=False)
        assert got is out and none is None and torch.equal(out, want)
        l2 = torch.zeros_like(lse)
        assert uc.window_attend(q, cache, ints([150, 200]), lse=l2)[1] is l2 and torch.equal(l2, lse)


def test_counts_out_of_range_are_reported():
    g = torch.Generator(device=DEV).manual_seed(5)
    k, v = make_cache(g, 2, 2, 64, [64, 64], 3)
    q = rows(g, 2, 4, 3, "bhtd")
    cache = uc.WindowCache(k, v, 50, 3)
    ws = uc.Workspace(DEV)
    want, _ = uc.window_attend(q, cache, ints([64, 0]), ints([3, 0]), ws=ws)
    assert ws.status() == _lib.UC_OK
    got, _ = uc.window_attend(q, cache, ints([64, -5]), ints([4, -1]), ws=ws)
    assert ws.status() == _lib.UC_ERR_RANGE and torch.equal(got, want)
    before = k.clone(), v.clone()
    for held, new in (([-1, 5], [3, 3]), ([5, 5], [4, 3]), ([5, 5], [-1, 3]), ([2 ** 31 - 2, 5], [3, 3])):
        total, _ = uc.window_append(cache, rows(g, 2, 2, 3, "bhtd"), rows(g, 2, 2, 3, "bhtd"), ints(held), ints(new), ws=ws)
        assert ws.status() == _lib.UC_ERR_RANGE
        assert total.tolist() == [held[0], 8]
        assert torch.equal(k[0], before[0][0]) and torch.equal(v[0], before[1][0])
        assert not torch.equal(k[1], before[0][1])


@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
@pytest.mark.parametrize("pairs,inter", [(64, False), (17, False), (20, True), (0, False)])
@pytest.mark.parametrize("B,hq,hkv,T,sinks,n_rows,held,new", [
    (1, 4, 1, 1, 0, 1, [9], None), (2, 28, 4, 5, 4, 60, [57, 1000], None), (3, 6, 2, 40, 3, 20, [0, 2, 17], [40, 0, 1]),
    (2, 4, 4, 130, 0, 200, [0, 190], [130, 77]), (2, 5, 5, 9, 7, 8, [3, 100], None)])
def test_append(B, hq, hkv, T, sinks, n_rows, held, new, pairs, inter, layout):
    g = torch.Generator(device=DEV).manual_seed(T)
    k, v = (rows(g, B, hkv, n_rows, "cut" if layout == "bthd" else "bhtd") for _ in range(2))
    kn, vn, q = (rows(g, B, h, T, layout) for h in (hkv, hkv, hq))
    table = uc.Rotary(freqs_of(pairs), interleaved=inter, scale=1.5) if pairs else None
    before = [x.float().cpu().numpy() for x in (k, v)]
    ws = uc.Workspace(DEV)
    total, oq = uc.window_append(uc.WindowCache(k, v, 3, sinks), kn, vn, ints(held), None if new is None else ints(new),
                                 rotary=table, q=q if pairs else None, ws=ws)
    assert ws.status() == _lib.UC_OK
    n = [T] * B if new is None else new
    assert total.tolist() == [h + x for h, x in zip(held, n)]
    kt = kn.double().cpu().numpy()
    p = np.array(held)[:, None] + np.arange(T)
    err = np.zeros_like(kt)
    if pairs:
        turned = orot.rotary(kt, p, freqs_of(pairs), inter, 1.5)
        err = rotary_bound(kt, pairs, inter, 1.5, torch.bfloat16, turned)
        kt = turned
        qs = q.double().cpu().numpy()
        want = orot.rotary(qs, p, freqs_of(pairs), inter, 1.5)
        assert (np.abs(oq.double().cpu().numpy() - want) <= rotary_bound(qs, pairs, inter, 1.5, torch.bfloat16, want)).all()
    else:
        assert oq is None
    wk, wv = owin.append(before[0].astype(np.float64), before[1], kt, vn.float().cpu().numpy(), held, n, sinks)
    ek, _ = owin.append(np.zeros_like(wk), np.zeros_like(wk), err, err, held, n, sinks)
    assert (np.abs(k.double().cpu().numpy() - wk) <= ek).all()
    assert np.array_equal(v.float().cpu().numpy(), wv)


def test_append_in_place_and_without_rotation():
    g = torch.Generator(device=DEV).manual_seed(9)
    table = uc.Rotary(freqs_of(64))
    k, v = (rows(g, 2, 2, 30, "bhtd") for _ in range(2))
    kn, vn, q = rows(g, 2, 2, 4, "bhtd"), rows(g, 2, 2, 4, "bhtd"), rows(g, 2, 6, 4, "bhtd")
    cache = uc.WindowCache(k, v, 10, 2)
    total, oq = uc.window_append(cache, kn, vn, ints([3, 50]), rotary=table, q=q)
    total2 = torch.zeros_like(total)
    got = uc.window_append(cache, kn, vn, ints([3, 50]), rotary=table, q=q, out_q=q, total=total2)
    assert got[0] is total2 and got[1] is q and torch.equal(total, total2) and torch.equal(q, oq)


@pytest.mark.parametrize("hq,hkv,T,held", [(4, 4, 300, 0), (14, 2, 200, 700), (2, 2, 40, 3000), (8, 1, 20, 3000)])
@pytest.mark.parametrize("size", [30.0, 1000.0, 1e8])
def test_logits_that_jump(hq, hkv, T, held, size):
    """Logits that rise by any amount from tile to tile, within tiles and at their ends."""
    g = torch.Generator(device=DEV).manual_seed(8)
    n = held + T
    k, v = make_cache(g, 1, hkv, n, [n], 3)
    q = rows(g, 1, hq, T, "bhtd")
    rise = torch.ones(n, device=DEV)
    for at in (70, 127, 128, 200, 255, 300, 650, 2100, 2999):
        rise[at:at + 1] *= size ** ((at % 7 + 1) / 7)
    k = (k.float() * rise[:, None]).bfloat16()
    for window in (1 << 30, 150):
        ws = uc.Workspace(DEV)
        out, lse = uc.window_attend(q, uc.WindowCache(k, v, window, 3), ints([n]), ws=ws)
        o, l, spread, reach = owin.attend(q.float().cpu().numpy(), k.float().cpu().numpy(), v.float().cpu().numpy(), [n], [T],
                                          window, 3)
        assert ws.status() == _lib.UC_OK
        # as check(); where the logits' own rounding, 2^-19 of sum |q k|, is no small share of 1 the weights say
        # nothing: those rows' outputs are only within what they are made of
        d = 2.0 ** -19 * reach + 2.0 ** -20
        err = np.where(d[..., None] < 0.1, (2.5 * d[..., None] + 2.0 ** -8) * spread, 2 * np.abs(v.float().cpu().numpy()).max())
        got = out.double().cpu().numpy()
        assert np.isfinite(got).all()
        assert (np.abs(got - o) <= err + 2.0 ** -8 * (np.abs(o) + err)).all()
        assert (np.abs(lse.double().cpu().numpy() - l) <= d + 2.0 ** -19 + 2.0 ** -22 * np.abs(l)).all()


@pytest.mark.parametrize("T", [1, 5, 100])
def test_a_cache_of_more_than_2_31_elements(T):
    """The same tokens far out in a long cache and in a short one."""
    g = torch.Generator(device=DEV).manual_seed(11)
    n, window, sinks = 9_000_000, 700, 6                  # rows x 128 x 2 heads: 2.3e9 elements
    near = sinks + window + T - 1
    short = [rows(g, 1, 2, near, "bhtd") for _ in range(2)]
    long = [torch.full((1, 2, n, 128), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for x, y in zip(long, short):
        x[:, :, :sinks] = y[:, :, :sinks]
        x[:, :, n - (near - sinks):] = y[:, :, sinks:]
    q = rows(g, 1, 14, T, "bhtd")
    want = uc.window_attend(q, uc.WindowCache(*short, window, sinks), ints([near]))
    got = uc.window_attend(q, uc.WindowCache(*long, window, sinks), ints([n]))
    # (keys lie in other tiles: sums in another order, and in prompts p is rounded from another reference: twice
    # 2^-8 of p and of the output, |v| below 6 here)
    assert float((got[0].float() - want[0].float()).abs().max()) <= 2 * 2.0 ** -8 * 6
    assert float((got[1] - want[1]).abs().max()) <= 2.0 ** -16
    kn, vn = rows(g, 1, 2, 3, "bhtd"), rows(g, 1, 2, 3, "bhtd")
    total, _ = uc.window_append(uc.WindowCache(*long, window, sinks), kn, vn, ints([n - 3]))
    assert total.tolist() == [n] and torch.equal(long[0][:, :, n - 3:], kn) and torch.equal(long[1][:, :, n - 3:], vn)


@pytest.mark.parametrize("T", [3, 200])
def test_a_call_in_a_graph(T):
    """Captured once; lengths, queries and the cache change between replays; a batch of more items than SMs too."""
    g = torch.Generator(device=DEV).manual_seed(12)
    B, n = 6, 900
    k, v = (rows(g, B, 8, n, "bhtd") for _ in range(2))
    q = rows(g, B, 16, T, "bhtd")
    lengths, nq = ints([n] * B), ints([T] * B)
    cache = uc.WindowCache(k, v, 300, 4)
    ws = uc.Workspace(DEV)
    uc.window_attend(q, cache, lengths, n_query=nq, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = uc.window_attend(q, cache, lengths, n_query=nq, ws=ws)
    for step in range(4):
        q.copy_(rows(g, B, 16, T, "bhtd"))
        k.copy_(rows(g, B, 8, n, "bhtd"))
        lengths.copy_(ints([max(0, n - 150 * b - step) for b in range(B)]))
        nq.copy_(ints([min(T, 1 + b * T // 5) for b in range(B)]))
        graph.replay()
        want, l2 = uc.window_attend(q, cache, lengths, n_query=nq)
        assert torch.equal(out, want) and torch.equal(lse, l2)
    assert ws.status() == _lib.UC_OK


def test_the_same_call_gives_the_same_bits():
    """Items are taken as CTAs come to them; no result depends on which one does."""
    g = torch.Generator(device=DEV).manual_seed(13)
    k, v = (rows(g, 4, 8, 1500, "bhtd") for _ in range(2))
    for T in (1, 8, 1500):
        q = rows(g, 4, 16, T, "bhtd")
        cache = uc.WindowCache(k, v, 400, 4)
        first = uc.window_attend(q, cache, ints([1500] * 4))
        for _ in range(5):
            again = uc.window_attend(q, cache, ints([1500] * 4))
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
