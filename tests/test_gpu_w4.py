"""Products with 4-bit weights (stom_w4_linear) against products in 64 bits.

Tolerance of y, element by element, with u the type's half step (2^-8 bf16, 2^-11 fp16) and k columns:
    u |y|                                  the one rounding of the result
  + 2^-24 * 1000 * sum over groups of M_g (16 s + |z|) / 16, M_g = sum of the group's |x|
                                           the sums of a group: products of codes and tokens are exact; sums of codes times
                                            x, at most 15 M, and of x, at most M, are off by 2^-24 of their size for each of at
                                            most 128 additions.  The worst case, 130 * (15 s + |z|) M, is twice the bound;
                                            random signs come nowhere near it (a root: sqrt(128) ~ 11.3 for 128 additions)
  + 2^-23 |y|                              the sums over groups and over warps
  + 2^-24 (fp16)                           where the result is subnormal"""
import numpy as np
import pytest
import torch

import _kv as K
import _tree as T

pytestmark = pytest.mark.gpu
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


def _lib():
    from paper_2510_18269_b200 import oqm
    oqm.lib()
    return oqm


def _make(rows, n, k, group, dtype=BF, meta=BF, zero=True, seed=0, offset=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    s = dict(codes=torch.randint(0, 256, (n, k // 2), generator=g, device="cuda", dtype=torch.uint8),
             scale=(0.02 * (0.5 + torch.rand(n, k // group, generator=g, device="cuda"))).to(meta), zero=None, group=group,
             x=(r(rows, k) + offset).to(dtype), bias=r(n).to(dtype), add=r(rows, n).to(dtype))
    if zero:
        s["zero"] = (-0.02 * (6.5 + 2 * torch.rand(n, k // group, generator=g, device="cuda"))).to(meta)
    return s


def _check(s, y, bias=True, add=True, x=None, added=None):
    x = (s["x"] if x is None else x).double().cpu().numpy()
    group, dtype = s["group"], y.dtype
    scale, zero = s["scale"].cpu(), None if s["zero"] is None else s["zero"].cpu()
    w = T.weights(s["codes"].cpu(), scale, zero, group)
    want = x @ w.T
    if bias:
        want = want + s["bias"].double().cpu().numpy()
    if add:
        want = want + (s["add"] if added is None else added).double().cpu().numpy()
    sd = scale.double().numpy()
    zd = 8 * sd if zero is None else np.abs(zero.double().numpy())
    m = np.abs(x).reshape(x.shape[0], -1, group).sum(-1)
    u = K.HALF_STEP[dtype]
    lim = u * np.abs(want) + 2.0 ** -24 * 1000 * (m @ (sd + zd / 16).T) + 2.0 ** -23 * np.abs(want) + (2.0 ** -24 if dtype is HF else 0)
    got = y.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= lim)
    assert not bad.any(), (int(bad.sum()), float(np.nanmax(np.abs(got - want) / lim)))


def _call(s, bias=True, add=True):
    oqm = _lib()
    n = s["codes"].shape[0]
    y = torch.full((s["x"].shape[0], n), 7.0, dtype=s["x"].dtype, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    oqm.stom_w4_linear(oqm.W4Matrix(s["codes"], s["scale"], s["zero"]), s["x"], y, bias=s["bias"] if bias else None,
                       add=s["add"] if add else None, dev_flags=flags)
    torch.cuda.synchronize()
    assert flags.item() == 0
    return y


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype,meta,zero", [(BF, BF, True), (HF, HF, True), (BF, FP, False), (HF, BF, False), (HF, FP, True),
                                             (BF, HF, True)])
def test_types_and_groups(group, dtype, meta, zero):
    for rows in (1, 5, 40):
        s = _make(rows, 197, 1280, group, dtype, meta, zero, seed=rows)
        _check(s, _call(s))


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 200, 256, 257, 700])
def test_token_counts(rows):
    s = _make(rows, 131, 640, 128, seed=rows)
    _check(s, _call(s))


@pytest.mark.parametrize("n,k,group", [(1, 32, 32), (1, 128, 128), (2, 64, 64), (15, 96, 32), (16, 128, 64), (17, 384, 128), (127, 256, 128),
                                       (128, 256, 32), (129, 2048, 64), (4608, 3584, 128), (1000, 14336, 128), (300, 8192, 32),
                                       (33, 32768, 64)])
@pytest.mark.parametrize("rows", [1, 6, 20, 64])
def test_sizes(n, k, group, rows):
    s = _make(rows, n, k, group, seed=n + k)
    _check(s, _call(s))


@pytest.mark.parametrize("n,k,group", [(9472, 512, 32), (9473, 640, 128), (12001, 3584, 64), (30011, 384, 128)])
@pytest.mark.parametrize("rows", [1, 3, 8, 13, 16])
def test_matrices_of_many_rows(n, k, group, rows):
    s = _make(rows, n, k, group, seed=rows + n)
    _check(s, _call(s))


@pytest.mark.parametrize("n", [1184, 1185])
@pytest.mark.parametrize("rows", [8, 9, 16, 17])
def test_where_one_kernel_takes_over_from_the_other(n, rows):
    s = _make(rows, n, 1152, 64, seed=rows)
    _check(s, _call(s))


@pytest.mark.parametrize("rows", [1, 12, 50, 130])
def test_with_and_without_bias_and_addend(rows):
    s = _make(rows, 77, 512, 64)
    for bias in (False, True):
        for add in (False, True):
            _check(s, _call(s, bias, add), bias, add)


@pytest.mark.parametrize("rows", [1, 9, 40, 150])
def test_strides_and_the_addend_in_place(rows):
    """Rows of wider matrices, odd addresses of outputs; y is the addend; nothing is written beside it."""
    oqm = _lib()
    s = _make(rows, 101, 512, 128)
    wide = torch.zeros(101, 300, dtype=torch.uint8, device="cuda").new_zeros(101, 320)
    codes = wide[:, 16:16 + 256]
    codes.copy_(s["codes"])
    meta = torch.zeros(101, 9, dtype=BF, device="cuda")
    meta2 = torch.zeros(101, 9, dtype=BF, device="cuda")
    scale, zero = meta[:, 3:7], meta2[:, 3:7]
    scale.copy_(s["scale"]), zero.copy_(s["zero"])
    xw = torch.full((rows, 528), 9.0, dtype=BF, device="cuda")
    x = xw[:, 8:520]
    x.copy_(s["x"])
    flat = torch.full((rows * 107 + 5,), 7.0, dtype=BF, device="cuda")
    y = flat[3:3 + rows * 107].view(rows, 107)[:, 1:102]
    y.copy_(s["add"])
    before = flat.clone()
    oqm.stom_w4_linear(oqm.W4Matrix(codes, scale, zero), x, y, bias=s["bias"], add=y)
    torch.cuda.synchronize()
    _check(s, y, x=x)
    keep = torch.ones_like(flat, dtype=torch.bool)
    keep[3:3 + rows * 107].view(rows, 107)[:, 1:102] = False
    assert torch.equal(flat[keep], before[keep])


@pytest.mark.parametrize("rows", [1, 24, 70])
def test_tokens_that_are_not_centred_and_large_ones(rows):
    """Sums of tokens far from zero are where sums with an offset lose most."""
    for offset in (3.0, -20.0):
        s = _make(rows, 64, 2048, 128, offset=offset)
        _check(s, _call(s))
    s = _make(rows, 64, 512, 32, HF, HF)
    s["x"].mul_(3000.0).clamp_(-60000, 60000)
    s["scale"].mul_(0.01), s["zero"].mul_(0.01)
    y = _call(s, False, False)
    assert torch.isfinite(y).all()
    _check(s, y, False, False)


@pytest.mark.parametrize("rows", [2, 33, 90])
def test_every_code_and_every_column_counts(rows):
    """A weight matrix that picks columns: one code 1 in each row, all others 0, offsets 0."""
    n = k = 256
    for group in (32, 64, 128):
        s = _make(rows, n, k, group)
        at = torch.randperm(k, generator=torch.Generator().manual_seed(group))
        codes = torch.zeros(n, k // 2, dtype=torch.uint8)
        codes[torch.arange(n), at // 2] = torch.where(at % 2 == 0, 1, 16).to(torch.uint8)
        s["codes"], s["scale"], s["zero"] = codes.cuda(), torch.ones_like(s["scale"]), torch.zeros_like(s["zero"])
        s["x"] = torch.randint(-100, 101, s["x"].shape, device="cuda").to(BF)       # sums of these are exact
        assert torch.equal(_call(s, False, False), s["x"][:, at.cuda()])
        for code in range(16):
            s["codes"] = torch.full((n, k // 2), code * 17, dtype=torch.uint8, device="cuda")
            s["x"] = torch.ones_like(s["x"])
            assert (_call(s, False, False) == code * k).all()


@pytest.mark.parametrize("rows", [3, 40])
def test_a_token_that_is_no_number_stays_alone(rows):
    s = _make(rows, 70, 512, 64)
    want = _call(s)
    s["x"][1, 100] = float("nan")
    s["x"][2, 7] = float("inf")
    got = _call(s)
    others = [i for i in range(rows) if i not in (1, 2)]
    assert torch.equal(got[others], want[others])
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[2]).any()


@pytest.mark.parametrize("rows", [1, 20, 64, 140])
def test_captured_replayed_and_repeated(rows):
    oqm = _lib()
    s = _make(rows, 500, 3584, 128)
    w = oqm.W4Matrix(s["codes"], s["scale"], s["zero"])
    y = torch.zeros(rows, 500, dtype=BF, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    oqm.stom_w4_linear(w, s["x"], y, stream=side)
    torch.cuda.synchronize()
    want = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        oqm.stom_w4_linear(w, s["x"], y)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    s["x"].copy_(torch.randn(rows, 3584, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    _check(s, y, False, False)


def test_workspaces_given_and_not_given_on_any_stream():
    oqm = _lib()
    s = _make(40, 300, 1024, 128)
    w = oqm.W4Matrix(s["codes"], s["scale"], s["zero"])
    assert oqm.stom_w4_workspace_bytes(w, 3) == 0 and oqm.stom_w4_workspace_bytes(w, 0) == 0
    need = oqm.stom_w4_workspace_bytes(w, 40)
    want = _call(s, False, False)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    ys = [torch.zeros_like(want) for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    oqm.stom_w4_linear(w, s["x"], ys[0], workspace=ws[:need])
    for i, st in enumerate(streams):                               # two calls at once, each with a workspace of torch's
        oqm.stom_w4_linear(w, s["x"], ys[1 + i], stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in ys) and (ws[need:] == 255).all()
    with pytest.raises(oqm.StomError):
        oqm.stom_w4_linear(w, s["x"], ys[0], workspace=ws[:need - 1])


def test_no_token():
    s = _make(0, 70, 512, 64)
    assert _call(s).shape == (0, 70)
