"""CPU-only checks of the paged cache and of the token choice: what the host refuses before any launch, the workspace
sizes, the rotation frequencies, and the arithmetic identity the page lookup relies on.  No kernel is launched here:
the addresses are never dereferenced."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

P = 0x7f1000000000


@pytest.fixture(scope="module")
def oqm():
    from paper_2510_18269_b200 import build, oqm as m
    build.build()
    m.lib()
    return m


def pool_of(oqm, **kw):
    a = dict(k=P, v=P + (1 << 30), dtype=oqm.BF16, n_layers=2, n_pages=10, page_tokens=50, n_kv_heads=4, head_dim=128,
             stride_layer=10 * 50 * 512, stride_page=50 * 512, stride_token=512, stride_head=128)
    a.update(kw)
    return oqm.KvPoolDesc(*[a[n] for n, _ in oqm.KvPoolDesc._fields_])


def seqs_of(oqm, **kw):
    a = dict(table=P, len=P, refs=P, n_seqs=3, max_pages=5, table_stride=5)
    a.update(kw)
    return oqm.KvSeqsDesc(*[a[n] for n, _ in oqm.KvSeqsDesc._fields_])


BAD_POOLS = [(dict(k=None), -1), (dict(v=None), -1), (dict(k=P + 8), -3), (dict(dtype=2), -6), (dict(dtype=9), -6),
             (dict(head_dim=96), -2), (dict(n_layers=0), -1), (dict(n_pages=0), -1), (dict(page_tokens=0), -1),
             (dict(n_kv_heads=0), -1), (dict(stride_token=516), -3), (dict(stride_head=64), -1),
             (dict(stride_page=-512), -1), (dict(stride_layer=0), -1)]
BAD_SEQS = [(dict(table=None), -1), (dict(len=None), -1), (dict(n_seqs=-1), -1), (dict(max_pages=0), -1),
            (dict(table_stride=4), -1), (dict(len=P + 2), -3)]


def attend(oqm, pool=None, seqs=None, **kw):
    pool, seqs = pool or pool_of(oqm), seqs or seqs_of(oqm)
    a = dict(layer=0, hq=28, q=P, qs=28 * 128, qh=128, scale=0.1, cap=0.0, window=0, out=P, os=28 * 128, oh=128, lse=None,
             ws=P, nb=1 << 40)
    a.update(kw)
    return oqm.lib().stom_kv_attend(C.byref(pool), C.byref(seqs), a["layer"], a["hq"], a["q"], a["qs"], a["qh"],
                                    a["scale"], a["cap"], a["window"], a["out"], a["os"], a["oh"], a["lse"], a["ws"],
                                    a["nb"], None, None)


@pytest.mark.parametrize("kw,code", BAD_POOLS)
def test_attend_refuses_bad_pools(oqm, kw, code):
    assert attend(oqm, pool=pool_of(oqm, **kw)) == code
    assert oqm.lib().stom_kv_attend_workspace_bytes(C.byref(pool_of(oqm, **kw)), C.byref(seqs_of(oqm)), 28) == code


@pytest.mark.parametrize("kw,code", BAD_SEQS)
def test_attend_refuses_bad_sequences(oqm, kw, code):
    assert attend(oqm, seqs=seqs_of(oqm, **kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(layer=2), -1), (dict(layer=-1), -1), (dict(hq=0), -1), (dict(hq=30), -2), (dict(hq=260), -2),
    (dict(window=-1), -1), (dict(cap=-1.0), -1), (dict(cap=math.nan), -1), (dict(cap=math.inf), -1),
    (dict(scale=math.nan), -1), (dict(scale=math.inf), -1), (dict(q=None), -1), (dict(out=None), -1), (dict(q=P + 2), -3),
    (dict(qh=100), -3), (dict(os=28 * 128 + 4), -3), (dict(oh=64), -1), (dict(ws=None), -8), (dict(ws=P + 4), -8),
    (dict(nb=1000), -8),
])
def test_attend_refuses(oqm, kw, code):
    assert attend(oqm, **kw) == code


def test_attend_refuses_more_sequences_or_longer_rows_than_it_counts(oqm):
    assert attend(oqm, seqs=seqs_of(oqm, n_seqs=8193)) == -2
    assert attend(oqm, seqs=seqs_of(oqm, n_seqs=8192, max_pages=1 << 24, table_stride=1 << 24)) == -2
    assert attend(oqm, seqs=seqs_of(oqm, n_seqs=1, max_pages=1 << 30, table_stride=1 << 30)) == -2


def test_attend_of_no_sequence_is_nothing(oqm):
    assert attend(oqm, seqs=seqs_of(oqm, n_seqs=0)) == 0
    assert attend(oqm, seqs=seqs_of(oqm, refs=None, n_seqs=0)) == 0            # counts are not needed here


def test_attend_workspace_is_enough_for_two_rows_of_partial_results_per_block(oqm):
    for hq, d, per in ((28, 128, 8), (40, 64, 16), (128, 256, 8)):
        pool = pool_of(oqm, head_dim=d, stride_head=d, stride_token=4 * d, stride_page=200 * d, stride_layer=2000 * d)
        n = oqm.lib().stom_kv_attend_workspace_bytes(C.byref(pool), C.byref(seqs_of(oqm)), hq)
        assert n >= 148 * 2 * per * (d + 2) * 4 + 148 * 8


def rope_of(oqm, **kw):
    a = dict(freq=P, rot_dim=64, layout=0, magnitude=1.0)
    a.update(kw)
    return oqm.RopeDesc(*[a[n] for n, _ in oqm.RopeDesc._fields_])


def rotate(oqm, rope=None, **kw):
    a = dict(dt=0, d=128, n=5, pos=P, q=P, hq=4, qt=512, qh=128, qo=P, qot=512, qoh=128, qw=P, k=P, hk=2, kt=256, kh=128,
             ko=P, kot=256, koh=128, kw=P, eps=1e-6)
    a.update(kw)
    return oqm.lib().stom_kv_rotate(
        C.byref(rope or rope_of(oqm)), a["dt"], a["d"], a["n"], a["pos"], a["q"], a["hq"], a["qt"], a["qh"], a["qo"], a["qot"],
        a["qoh"], a["qw"], a["k"], a["hk"], a["kt"], a["kh"], a["ko"], a["kot"], a["koh"], a["kw"], a["eps"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), -1), (dict(dt=3), -6), (dict(d=96), -2), (dict(pos=None), -1), (dict(pos=P + 2), -3), (dict(q=None, k=None), -1),
    (dict(qo=None), -1), (dict(ko=None), -1), (dict(hq=0), -1), (dict(hk=-1), -1), (dict(hq=70000), -2), (dict(q=P + 8), -3),
    (dict(qo=P + 4), -3), (dict(ko=P + 4), -3), (dict(qw=P + 4), -3), (dict(kw=P + 8), -3), (dict(qt=516), -3),
    (dict(koh=124), -3), (dict(qot=64), -1), (dict(kot=120), -1), (dict(koh=64), -1), (dict(qt=-512), -1), (dict(eps=-1.0), -1),
    (dict(eps=math.nan), -1), (dict(eps=math.inf), -1),
])
def test_rotate_refuses(oqm, kw, code):
    assert rotate(oqm, **kw) == code


@pytest.mark.parametrize("kw,code", [(dict(freq=None), -1), (dict(freq=P + 4), -3), (dict(rot_dim=24), -2), (dict(rot_dim=-16), -2),
                                     (dict(rot_dim=144), -2), (dict(layout=2), -6), (dict(magnitude=math.nan), -1)])
def test_rotate_refuses_bad_ropes(oqm, kw, code):
    assert rotate(oqm, rope=rope_of(oqm, **kw)) == code
    assert append(oqm, rope=rope_of(oqm, **kw)) == code


def test_rotate_of_nothing_is_nothing(oqm):
    assert rotate(oqm, n=0) == 0
    assert rotate(oqm, n=0, q=None, hq=0, qo=None) == 0 and rotate(oqm, n=0, k=None, hk=0, ko=None) == 0
    assert rotate(oqm, rope=rope_of(oqm, rot_dim=0, freq=None), n=0, pos=None) == 0


def append(oqm, pool=None, seqs=None, rope=None, **kw):
    a = dict(layer=1, n=3, pos=P, slot=P, seq=None, q=P, hq=28, qt=28 * 128, qh=128, qo=P, qot=28 * 128, qoh=128, qw=None, k=P,
             kt=512, kh=128, kw=None, v=P, vt=512, vh=128, eps=1e-6)
    a.update(kw)
    return oqm.lib().stom_kv_append(
        C.byref(pool or pool_of(oqm)), C.byref(seqs or seqs_of(oqm)), a["layer"], C.byref(rope or rope_of(oqm)), a["n"],
        a["pos"], a["slot"], a["seq"], a["q"], a["hq"], a["qt"], a["qh"], a["qo"], a["qot"], a["qoh"], a["qw"], a["k"], a["kt"],
        a["kh"], a["kw"], a["v"], a["vt"], a["vh"], a["eps"], None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(layer=2), -1), (dict(layer=-1), -1), (dict(n=-1), -1), (dict(slot=None), -1), (dict(slot=P + 1), -3), (dict(k=None), -1),
    (dict(v=None), -1), (dict(v=P + 8), -3), (dict(vt=516), -3), (dict(vh=-128), -1), (dict(n=4), -1), (dict(seq=P + 2, n=4), -3),
    (dict(pos=None), -1), (dict(qo=None), -1),
])
def test_append_refuses(oqm, kw, code):
    assert append(oqm, **kw) == code


def test_append_and_pages_refuse_bad_pools_and_sequences(oqm):
    for kw, code in BAD_POOLS:
        assert append(oqm, pool=pool_of(oqm, **kw)) == code
        for call in (reserve, fork, free, compact):
            assert call(oqm, pool=pool_of(oqm, **kw)) == code
    for kw, code in BAD_SEQS:
        assert append(oqm, seqs=seqs_of(oqm, **kw)) == code
        for call in (reserve, fork, free, compact):
            assert call(oqm, seqs=seqs_of(oqm, **kw)) == code
    assert append(oqm, n=0) == 0


def test_calls_of_nothing_need_no_arrays(oqm):
    """Tensors without an element have no address."""
    none = seqs_of(oqm, table=None, len=None, n_seqs=0)
    assert attend(oqm, seqs=none, q=None, out=None) == 0
    assert oqm.lib().stom_kv_attend_workspace_bytes(C.byref(pool_of(oqm)), C.byref(none), 28) > 0
    assert rotate(oqm, n=0, pos=None, q=None, qo=None, k=None, ko=None) == 0
    assert rotate(oqm, n=0, pos=None, qo=None, ko=None) == 0
    assert append(oqm, n=0, pos=None, slot=None, q=None, qo=None, k=None, v=None) == 0
    assert append(oqm, seqs=none, n=0, pos=None, slot=None, k=None, v=None) == 0
    assert reserve(oqm, seqs=none, want=None) == 0 and fork(oqm, seqs=none, wish=None) == 0 and free(oqm, seqs=none, wish=None) == 0
    # tokens without a sequence to go to, and pages without their counts
    assert append(oqm, seqs=none) == -1 and append(oqm, seqs=none, seq=P) == -1
    assert compact(oqm, seqs=none, r=None) == -1 and compact(oqm, t=None) == -1


def _pages(oqm, name, pool, seqs, *args):
    return getattr(oqm.lib(), name)(C.byref(pool or pool_of(oqm)), C.byref(seqs or seqs_of(oqm)), *args)


def reserve(oqm, pool=None, seqs=None, want=P, ws=P, nb=1 << 30):
    return _pages(oqm, "stom_kv_reserve", pool, seqs, want, ws, nb, None, None)


def fork(oqm, pool=None, seqs=None, wish=P):
    return _pages(oqm, "stom_kv_fork", pool, seqs, wish, None, None)


def free(oqm, pool=None, seqs=None, wish=P):
    return _pages(oqm, "stom_kv_free", pool, seqs, wish, None, None)


def compact(oqm, pool=None, seqs=None, t=P, r=P, n=None, ws=P, nb=1 << 30):
    return _pages(oqm, "stom_kv_compact", pool, seqs, t, r, n, ws, nb, None, None)


def test_pages_refuse(oqm):
    for call in (reserve, fork, free, compact):
        assert call(oqm, seqs=seqs_of(oqm, refs=None)) == -1
    assert reserve(oqm, want=None) == -1 and fork(oqm, wish=None) == -1 and free(oqm, wish=None) == -1
    assert reserve(oqm, want=P + 1) == -3 and fork(oqm, wish=P + 2) == -3 and free(oqm, wish=P + 2) == -3
    need = oqm.lib().stom_kv_pages_workspace_bytes(C.byref(pool_of(oqm)), C.byref(seqs_of(oqm)))
    assert need >= 256 + 10 * 4 + 10 * 16
    for call in (reserve, compact):
        assert call(oqm, ws=None) == -8 and call(oqm, ws=P + 8) == -8 and call(oqm, nb=need - 1) == -8
    assert reserve(oqm, seqs=seqs_of(oqm, n_seqs=8193)) == -2                      # more rows than a plan holds
    assert compact(oqm, t=None) == -1 and compact(oqm, r=None) == -1 and compact(oqm, r=P + 2) == -3 and compact(oqm, n=P + 1) == -3
    for call in (reserve, fork, free):
        assert call(oqm, seqs=seqs_of(oqm, n_seqs=0)) == 0
    assert reserve(oqm, pool=pool_of(oqm, page_tokens=1 << 25)) == -2              # a page's 16-byte chunks pass 2^30


def sample(oqm, **kw):
    a = dict(x=P, dt=0, rows=4, n=100, stride=100, t=P, k=P, p=P, m=P, u=P, token=P, kept=P, lp=P)
    a.update(kw)
    return oqm.lib().stom_sample_tokens(a["x"], a["dt"], a["rows"], a["n"], a["stride"], a["t"], a["k"], a["p"], a["m"], a["u"],
                                        a["token"], a["kept"], a["lp"], None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), -1), (dict(n=0), -1), (dict(dt=3), -6), (dict(n=500001, stride=500001), -2), (dict(x=None), -1),
    (dict(token=None), -1), (dict(u=None, t=None), -1), (dict(stride=99), -1), (dict(stride=-100), -1), (dict(x=P + 1), -3),
    (dict(x=P + 2, dt=2), -3), (dict(t=P + 2), -3), (dict(k=P + 1), -3), (dict(p=P + 2), -3), (dict(m=P + 2), -3),
    (dict(u=P + 2), -3), (dict(token=P + 2), -3), (dict(kept=P + 2), -3), (dict(lp=P + 2), -3),
])
def test_sample_refuses(oqm, kw, code):
    assert sample(oqm, **kw) == code


def test_sample_of_no_row_is_nothing(oqm):
    assert sample(oqm, rows=0) == 0 and sample(oqm, rows=0, x=None, token=None) == 0


def test_page_of_a_token_by_multiplication_equals_the_division():
    """floor(x / d) = (mulhi(x, m) + x) >> s with s = ceil(log2 d), m = floor(2^32 (2^s - d) / d) + 1, for x < 2^31."""
    rng = np.random.default_rng(1)
    for d in list(range(1, 260)) + [1000, 4095, 4096, 4097, 65535, 10 ** 6, 2 ** 30, 2 ** 31 - 1]:
        s = (d - 1).bit_length()
        m = ((1 << 32) * ((1 << s) - d)) // d + 1
        assert m < 1 << 32
        x = np.concatenate([rng.integers(0, 1 << 31, 2000), np.arange(64), (1 << 31) - 1 - np.arange(64),
                            np.minimum(d * rng.integers(0, max(1, (1 << 31) // d), 500), (1 << 31) - 1)])
        x = np.concatenate([x, np.maximum(x - 1, 0)]).astype(np.uint64)
        total = ((x * np.uint64(m)) >> np.uint64(32)) + x
        assert (total < 1 << 32).all()
        assert np.array_equal(total >> np.uint64(s), x // np.uint64(d)), d


def test_frequencies(oqm):
    i = np.arange(64)
    plain = 1.0e6 ** (-2 * i / 128.0)
    near = lambda a, b: np.allclose(a.numpy(), b, rtol=1e-14, atol=0)  # noqa: E731
    assert near(oqm.stom_kv_frequencies(128), plain)
    assert near(oqm.stom_kv_frequencies(128, scaling=oqm.ROPE_LINEAR, factor=4.0), plain / 4)
    assert near(oqm.stom_kv_frequencies(128, scaling=oqm.ROPE_BASE, factor=8.0),
                (1.0e6 * 8.0 ** (128 / 126)) ** (-2 * i / 128.0))
    # the slowest pair of a raised base covers `factor` times the positions
    assert math.isclose(oqm.stom_kv_frequencies(128, scaling=oqm.ROPE_BASE, factor=8.0)[-1], plain[-1] / 8, rel_tol=1e-12)
    waves = oqm.stom_kv_frequencies(128, scaling=oqm.ROPE_WAVES, factor=8.0, trained=8192.0, low=1.0, high=4.0).numpy()
    turns = 8192.0 * plain / (2 * math.pi)
    assert np.allclose(waves[turns > 4], plain[turns > 4], rtol=1e-14)
    assert np.allclose(waves[turns < 1], plain[turns < 1] / 8, rtol=1e-14)
    between = (turns >= 1) & (turns <= 4)
    assert between.any() and (waves[between] <= plain[between]).all() and (waves[between] >= plain[between] / 8).all()
    assert oqm.stom_kv_frequencies(0).numel() == 0


@pytest.mark.parametrize("kw", [dict(rot_dim=24), dict(rot_dim=-16), dict(rot_dim=64, theta=0.0),
                                dict(rot_dim=64, scaling=7), dict(rot_dim=64, scaling=1, factor=0.0),
                                dict(rot_dim=64, scaling=3, factor=2.0, trained=0.0),
                                dict(rot_dim=64, scaling=3, factor=2.0, trained=9.0, low=4.0, high=4.0),
                                dict(rot_dim=64, theta=math.nan), dict(rot_dim=64, scaling=2, factor=math.inf)])
def test_frequencies_refuse(oqm, kw):
    with pytest.raises(oqm.StomError):
        oqm.stom_kv_frequencies(**kw)


def test_bindings_refuse_tensors_that_do_not_fit(oqm):
    k = torch.zeros(1, 4, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        oqm.KvPool(k, k.half())
    with pytest.raises(ValueError):
        oqm.KvPool(k, torch.zeros(1, 4, 16, 4, 64, dtype=torch.bfloat16)[:, :, :, ::2])   # other strides
    with pytest.raises(ValueError):
        oqm.KvPool(k[..., ::2], k[..., ::2])
    table, n = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for bad in (dict(table=table.long(), len=n), dict(table=table, len=n[:2]), dict(table=table, len=n.long()),
                dict(table=torch.zeros(3, 4, dtype=torch.int32)[:, ::2], len=n), dict(table=table, len=n, refs=n.float())):
        with pytest.raises(ValueError):
            oqm.KvSeqs(**bad)
    pool, seqs = oqm.KvPool(k, k.clone()), oqm.KvSeqs(table, n)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    ws = torch.empty(1 << 20, dtype=torch.uint8)
    for bad in (dict(q=q.half()), dict(q=q[:2]), dict(out=q[:, :2]), dict(q=torch.zeros(3, 4, 128, dtype=q.dtype)[..., ::2]),
                dict(lse=torch.zeros(3, 4, dtype=torch.float64)), dict()):                  # the last: on the CPU
        a = dict(q=q, out=q.clone(), lse=None)
        a.update(bad)
        with pytest.raises(ValueError):
            oqm.stom_kv_attend(pool, seqs, 0, a["q"], a["out"], 0.1, ws, lse=a["lse"])
    with pytest.raises(ValueError):
        oqm.Rope(torch.zeros(8))


def test_the_library_needs_no_binding_but_for_the_calls_that_use_it():
    """A Python whose torch the binding does not fit, or without it, has all that is called through ctypes."""
    import subprocess
    import sys
    from pathlib import Path

    code = """
import sys
sys.modules["paper_2510_18269_b200._stom_bind"] = None        # importing it fails
import torch
from paper_2510_18269_b200 import oqm
assert oqm.lib().stom_oqm_budget_to_k(12000, 50, 8) == 8
assert oqm.stom_kv_frequencies(64).numel() == 32
x = torch.zeros(1, 2, 64)
for call in (lambda: oqm.stom_kv_rotate(oqm.Rope(), torch.zeros(1, dtype=torch.int32), q=x, q_out=x),
             lambda: oqm.stom_sample_tokens(x[0], None, None)):
    try:
        call()
    except ImportError as e:
        assert "paper_2510_18269_b200.build" in str(e)
    else:
        raise SystemExit("no ImportError")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=Path(__file__).resolve().parent.parent, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


def test_the_binding_is_built_again_for_another_torch(oqm, monkeypatch, tmp_path):
    from paper_2510_18269_b200 import build

    built = []
    monkeypatch.setattr(build, "_build_library", lambda verbose: built.append("library"))
    monkeypatch.setattr(build, "_build_binding", lambda: built.append("binding"))
    build.build()
    assert built == []                                                       # both are there
    monkeypatch.setattr(build, "BUILT_FOR", tmp_path / "other.txt")
    build.build()
    assert built == ["binding"]                                              # not known what for
    (tmp_path / "other.txt").write_text(build._installed())
    build.build()
    (tmp_path / "other.txt").write_text(build._installed().replace("torch ", "torch 0."))
    build.build()
    assert built == ["binding"] * 2

    def broken():
        raise RuntimeError("no compiler")

    monkeypatch.setattr(build, "_build_binding", broken)
    monkeypatch.setattr(build, "LIB", tmp_path / "lib.so")
    with pytest.raises(RuntimeError, match="no compiler"):
        build.build()
    assert built[-1] == "library"                                            # it was built all the same


@pytest.mark.parametrize("scale,cap", [(0.1, 2.5e38), (0.0, 2.5e38), (2.5e38, 0.0), (-2.5e38, 0.0), (0.1, 1e-40), (-0.1, 1e-40),
                                       (0.05, 1.9e38), (3e38, 0.5)])
def test_attend_refuses_factors_that_are_no_numbers_of_32_bits(oqm, scale, cap):
    """softcap * log2(e), softmax_scale / softcap or softmax_scale * log2(e) would overflow, or be a subnormal number."""
    assert attend(oqm, scale=scale, cap=cap) == -1


@pytest.mark.parametrize("scale,cap", [(0.0, 30.0), (2e38, 0.0), (0.1, 1e30), (0.1, 1e-30), (-0.5, 50.0), (0.0, 0.0)])
def test_attend_takes_all_other_factors(oqm, scale, cap):
    assert attend(oqm, scale=scale, cap=cap, seqs=seqs_of(oqm, n_seqs=0)) == 0
