"""CPU-only checks of the calls for several tokens a step: what the host refuses before any launch, and calls of nothing.
The addresses are never dereferenced."""
import ctypes as C
import math

import pytest
import torch

from test_kv_cpu import BAD_POOLS, BAD_SEQS, P, oqm, pool_of, seqs_of  # noqa: F401


def tree(oqm, pool=None, seqs=None, **kw):  # noqa: F811
    a = dict(layer=0, n=9, first=P, parent=P, hq=28, q=P, qt=28 * 128, qh=128, scale=0.1, cap=0.0, window=0, out=P, ot=28 * 128,
             oh=128, lse=None, ws=P, nb=1 << 40)
    a.update(kw)
    return oqm.lib().stom_kv_attend_tree(
        C.byref(pool or pool_of(oqm)), C.byref(seqs or seqs_of(oqm)), a["layer"], a["n"], a["first"], a["parent"], a["hq"], a["q"],
        a["qt"], a["qh"], a["scale"], a["cap"], a["window"], a["out"], a["ot"], a["oh"], a["lse"], a["ws"], a["nb"], None, None)


def accept(oqm, pool=None, seqs=None, **kw):  # noqa: F811
    a = dict(n=9, first=P, parent=P, draft=P, chosen=P, path=P, count=P, following=P)
    a.update(kw)
    return oqm.lib().stom_kv_accept(C.byref(pool or pool_of(oqm)), C.byref(seqs or seqs_of(oqm)), a["n"], a["first"], a["parent"],
                                    a["draft"], a["chosen"], a["path"], a["count"], a["following"], None, None)


@pytest.mark.parametrize("kw,code", BAD_POOLS)
def test_bad_pools(oqm, kw, code):  # noqa: F811
    assert tree(oqm, pool=pool_of(oqm, **kw)) == code and accept(oqm, pool=pool_of(oqm, **kw)) == code
    need = oqm.lib().stom_kv_attend_tree_workspace_bytes
    assert need(C.byref(pool_of(oqm, **kw)), C.byref(seqs_of(oqm)), 9, 28) == code


@pytest.mark.parametrize("kw,code", BAD_SEQS)
def test_bad_sequences(oqm, kw, code):  # noqa: F811
    assert tree(oqm, seqs=seqs_of(oqm, **kw)) == code and accept(oqm, seqs=seqs_of(oqm, **kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(layer=2), -1), (dict(layer=-1), -1), (dict(n=-1), -1), (dict(hq=0), -1), (dict(hq=30), -2), (dict(hq=260), -2),
    (dict(window=-1), -1), (dict(cap=-1.0), -1), (dict(cap=math.nan), -1), (dict(cap=math.inf), -1), (dict(scale=math.nan), -1),
    (dict(scale=math.inf), -1), (dict(scale=3e38, cap=0.5), -1), (dict(scale=0.1, cap=1e-40), -1), (dict(first=None), -1),
    (dict(q=None), -1), (dict(out=None), -1), (dict(q=P + 2), -3), (dict(out=P + 8), -3), (dict(first=P + 2), -3),
    (dict(parent=P + 1), -3), (dict(lse=P + 2), -3), (dict(qh=100), -3), (dict(qt=4), -3), (dict(ot=28 * 128 + 4), -3),
    (dict(oh=64), -1), (dict(ot=64), -1), (dict(qt=-128), -1), (dict(qh=-128), -1), (dict(ws=None), -8), (dict(ws=P + 4), -8),
    (dict(nb=100), -8), (dict(n=1 << 27), -2),
])
def test_tree_refuses(oqm, kw, code):  # noqa: F811
    assert tree(oqm, **kw) == code


def test_tree_refuses_more_sequences_or_longer_rows_than_it_counts(oqm):  # noqa: F811
    assert tree(oqm, seqs=seqs_of(oqm, n_seqs=8193)) == -2 and accept(oqm, seqs=seqs_of(oqm, n_seqs=8193)) == -2
    long = seqs_of(oqm, n_seqs=1, max_pages=1 << 30, table_stride=1 << 30)
    assert tree(oqm, seqs=long) == -2 and accept(oqm, seqs=long) == -2


def test_tree_refuses_rows_whose_last_tile_would_pass_32_bits(oqm):  # noqa: F811
    """Token numbers of a tile are 32 bits wide, also behind a row's end."""
    pages = (2 ** 31 - 64) // pool_of(oqm).page_tokens
    assert tree(oqm, seqs=seqs_of(oqm, n_seqs=1, max_pages=pages, table_stride=pages)) == -2


def test_calls_of_nothing_need_no_arrays(oqm):  # noqa: F811
    none = seqs_of(oqm, table=None, len=None, n_seqs=0)
    assert tree(oqm, seqs=none, n=0, first=None, parent=None, q=None, out=None) == 0
    assert tree(oqm, n=0, q=None, out=None, parent=None) == 0
    assert accept(oqm, seqs=none, n=0, first=None, parent=None, draft=None, chosen=None, path=None, count=None, following=None) == 0
    need = oqm.lib().stom_kv_attend_tree_workspace_bytes
    assert need(C.byref(pool_of(oqm)), C.byref(none), 0, 28) >= 0
    assert need(C.byref(pool_of(oqm)), C.byref(none), -1, 28) == -1 and need(C.byref(pool_of(oqm)), C.byref(none), 5, 30) == -2


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), -1), (dict(first=None), -1), (dict(draft=None), -1), (dict(chosen=None), -1), (dict(first=P + 1), -3),
    (dict(parent=P + 2), -3), (dict(draft=P + 2), -3), (dict(chosen=P + 3), -3), (dict(path=P + 2), -3), (dict(count=P + 2), -3),
    (dict(following=P + 1), -3),
])
def test_accept_refuses(oqm, kw, code):  # noqa: F811
    assert accept(oqm, **kw) == code


def test_accept_needs_counts(oqm):  # noqa: F811
    assert accept(oqm, seqs=seqs_of(oqm, refs=None)) == -1


def linear(oqm, w=None, **kw):  # noqa: F811
    m = dict(codes=P, scale=P, zero=P, n=70, k=512, group=64, meta_dtype=0, code_stride=256, meta_stride=8)
    m.update(w or {})
    a = dict(dt=0, rows=5, x=P, xs=512, bias=P, add=P, adds=70, y=P, ys=70, ws=P, nb=1 << 30)
    a.update(kw)
    desc = oqm.W4Desc(*[m[n] for n, _ in oqm.W4Desc._fields_])
    return oqm.lib().stom_w4_linear(C.byref(desc), a["dt"], a["rows"], a["x"], a["xs"], a["bias"], a["add"], a["adds"], a["y"],
                                    a["ys"], a["ws"], a["nb"], None, None)


@pytest.mark.parametrize("w,code", [
    (dict(codes=None), -1), (dict(scale=None), -1), (dict(n=0), -1), (dict(k=0), -1), (dict(k=96, group=64), -2), (dict(group=16), -2),
    (dict(group=256), -2), (dict(group=0), -2), (dict(meta_dtype=3), -6), (dict(codes=P + 8), -3), (dict(code_stride=264), -3),
    (dict(code_stride=240), -1), (dict(meta_stride=7), -1), (dict(scale=P + 1), -3), (dict(zero=P + 2, meta_dtype=2), -3),
    (dict(n=1 << 23), -2), (dict(k=(1 << 24) + 64, code_stride=1 << 24, meta_stride=1 << 20), -2),
])
def test_linear_refuses_bad_matrices(oqm, w, code):  # noqa: F811
    assert linear(oqm, w) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dt=2), -6), (dict(dt=5), -6), (dict(rows=-1), -1), (dict(x=None), -1), (dict(y=None), -1), (dict(x=P + 8), -3),
    (dict(xs=516), -3), (dict(xs=-512), -1), (dict(ys=69), -1), (dict(adds=-70), -1), (dict(y=P + 1), -3), (dict(bias=P + 1), -3),
    (dict(add=P + 1), -3), (dict(rows=65535 * 8 + 1), -2), (dict(rows=40, ws=None), -8), (dict(rows=40, ws=P + 64), -8),
    (dict(rows=40, nb=1000), -8),
])
def test_linear_refuses(oqm, kw, code):  # noqa: F811
    assert linear(oqm, **kw) == code


def test_linear_of_no_token_is_nothing(oqm):  # noqa: F811
    assert linear(oqm, rows=0) == 0 and linear(oqm, rows=0, x=None, y=None, bias=None, add=None) == 0


def test_bindings_refuse_tensors_that_do_not_fit(oqm):  # noqa: F811
    i32 = dict(dtype=torch.int32)
    k = torch.zeros(1, 4, 16, 2, 64, dtype=torch.bfloat16)
    pool = oqm.KvPool(k, k.clone())
    seqs = oqm.KvSeqs(torch.zeros(3, 2, **i32), torch.zeros(3, **i32), torch.zeros(4, **i32))
    ws = torch.empty(1 << 20, dtype=torch.uint8)
    good = dict(q=torch.zeros(7, 4, 64, dtype=torch.bfloat16), out=torch.zeros(7, 4, 64, dtype=torch.bfloat16),
                first=torch.zeros(4, **i32), parent=torch.zeros(7, **i32), lse=torch.zeros(7, 4))
    for bad in (dict(q=good["q"].half()), dict(out=good["out"][:6]), dict(first=torch.zeros(3, **i32)), dict(first=None),
                dict(parent=torch.zeros(6, **i32)), dict(lse=good["lse"].double()), {}):       # the last: on the CPU
        a = {**good, **bad}
        with pytest.raises(ValueError):
            oqm.stom_kv_attend_tree(pool, seqs, 0, a["first"], a["q"], a["out"], 0.1, ws, parent=a["parent"], lse=a["lse"])
    rows = torch.zeros(7, **i32)
    for bad in (dict(draft=rows.long()), dict(chosen=rows[:6]), dict(first=None), dict(chosen=None), dict(path=rows[:3]),
                dict(next=rows), {}):
        a = {**dict(first=good["first"], draft=rows, chosen=rows, path=None, next=None), **bad}
        with pytest.raises(ValueError):
            oqm.stom_kv_accept(pool, seqs, a["first"], a["draft"], a["chosen"], a["path"], None, a["next"])
    with pytest.raises(ValueError):                                                            # no counts
        oqm.stom_kv_accept(pool, oqm.KvSeqs(seqs.table, seqs.len), good["first"], rows, rows)
    codes, scale = torch.zeros(10, 64, dtype=torch.uint8), torch.zeros(10, 2)
    for bad in (dict(codes=codes.int()), dict(codes=codes[0]), dict(codes=torch.zeros(10, 128, dtype=torch.uint8)[:, ::2]),
                dict(scale=scale[:9]), dict(scale=torch.zeros(10, 3)), dict(scale=scale.double()), dict(zero=scale.half()),
                dict(zero=torch.zeros(10, 4)[:, :2])):
        a = {**dict(codes=codes, scale=scale, zero=None), **bad}
        with pytest.raises(ValueError):
            oqm.W4Matrix(a["codes"], a["scale"], a["zero"])
    w = oqm.W4Matrix(codes, scale, scale.clone())
    x, y = torch.zeros(3, 128, dtype=torch.bfloat16), torch.zeros(3, 10, dtype=torch.bfloat16)
    for bad in (dict(x=x[:, :64]), dict(y=y.half()), dict(y=y[:2]), dict(bias=y[0, :9]), dict(add=y[:, :9]), dict(x=x.float()), {}):
        a = {**dict(x=x, y=y, bias=None, add=None), **bad}
        with pytest.raises(ValueError):
            oqm.stom_w4_linear(w, a["x"], a["y"], bias=a["bias"], add=a["add"])
