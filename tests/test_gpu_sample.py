"""The choice of the next token (stom_sample_tokens) against sorting every row in 64 bits.  Tokens and counts are equal
(but where a mass comes within 1e-10 of a border, see _kv.choose); logprob within 2^-20 + 2^-23 |.| (binary32 result of
binary64 sums that are within 1e-10)."""
import math

import numpy as np
import pytest
import torch

import _kv as K

pytestmark = pytest.mark.gpu
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def _lib():
    from paper_2510_18269_b200 import oqm
    oqm.lib()
    return oqm


def _f(v, rows):
    return None if v is None else torch.as_tensor(np.broadcast_to(np.asarray(v, np.float32), (rows,)).copy()).cuda()


def _check(x, u, temperature=None, top_k=None, top_p=None, min_p=None, flags=0, ambiguous=0.02):
    oqm = _lib()
    rows, n = x.shape
    token = torch.full((rows + 2,), -9, dtype=torch.int32, device="cuda")
    kept, lp = torch.full_like(token, -9), torch.full((rows + 2,), 9.0, device="cuda")
    f = torch.zeros(1, dtype=torch.int32, device="cuda")
    k = None if top_k is None else torch.as_tensor(np.broadcast_to(np.asarray(top_k, np.int32), (rows,)).copy()).cuda()
    args = [_f(v, rows) for v in (u, temperature, top_p, min_p)]
    oqm.stom_sample_tokens(x, args[0], token[:rows], temperature=args[1], top_k=k, top_p=args[2], min_p=args[3],
                           logprob=lp[:rows], kept=kept[:rows], dev_flags=f)
    torch.cuda.synchronize()
    assert f.item() == flags
    assert (token[rows:] == -9).all() and (kept[rows:] == -9).all() and (lp[rows:] == 9).all()
    host = x.double().cpu().numpy()
    pick = lambda a, d, i: d if a is None else float(a[i])  # noqa: E731
    unsure = 0
    for i in range(rows):
        tokens, counts, logs = K.choose(host[i], pick(args[0], 0.0, i), pick(args[1], 1.0, i), int(pick(k, 0, i)),
                                        pick(args[2], 1.0, i), pick(args[3], 0.0, i))
        unsure += len(tokens) > 1 or len(counts) > 1
        t = int(token[i])
        assert t in tokens and int(kept[i]) in counts, (i, t, tokens, int(kept[i]), counts)
        want = logs[t]
        assert float(lp[i]) == want or abs(float(lp[i]) - want) <= 2.0 ** -20 + 2.0 ** -23 * abs(want), (i, float(lp[i]), want)
    assert unsure <= max(1, ambiguous * rows)
    return token[:rows].clone(), kept[:rows].clone()


def _logits(rows, n, dtype, seed, spread=2.5, odd=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(rows, n + (3 if odd else 0), generator=g, device="cuda") * spread).to(dtype)
    return x[:, 1:n + 1] if odd else x


def _u(rows, seed):
    return np.random.default_rng(seed).random(rows).astype(np.float32)


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.7, top_k=40), dict(top_p=0.9), dict(min_p=0.05),
            dict(temperature=1.3, top_k=50, top_p=0.95, min_p=0.01), dict(top_k=1), dict(top_p=0.0), dict(min_p=1.0),
            dict(temperature=0.01), dict(temperature=50.0, top_p=0.5)]


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("n", [1, 2, 17, 1000, 50257])
def test_settings(dtype, n):
    rows = len(SETTINGS) * 3
    x = _logits(rows, n, dtype, seed=n, odd=n % 2 == 1)
    get = lambda key, d: [s.get(key, d) for s in SETTINGS] * 3  # noqa: E731
    _check(x, _u(rows, n), get("temperature", 1.0), get("top_k", 0), get("top_p", 1.0), get("min_p", 0.0))


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("rows,n", [(1, 151001), (3, 128000), (40, 70001), (1, 300007), (200, 3001)])
def test_sizes_and_clusters(dtype, rows, n):
    x = _logits(rows, n, dtype, seed=rows + n, odd=True)
    x[:, ::1000] += 6
    _check(x, _u(rows, 1), temperature=0.9)
    _check(x, _u(rows, 2), temperature=0.8, top_k=33, top_p=0.9)
    _check(x, _u(rows, 3), temperature=1.1, top_p=0.7, min_p=0.001)


@pytest.mark.parametrize("dtype", [BF, FL])
def test_many_draws_of_one_row_follow_the_order(dtype):
    """Every border of a small row, from both sides: u just below and just above each cumulated share."""
    x = _logits(1, 40, dtype, seed=4, spread=1.0)
    host = np.sort(x.double().cpu().numpy()[0])[::-1]
    share = np.cumsum(np.exp(host - host[0]))
    share = (share / share[-1])[:-1]
    u = np.concatenate([share * (1 - 1e-6), share * (1 + 1e-6), [0.0, 1.0, 2.0, -1.0, 0.99999994]]).astype(np.float32)
    u = np.clip(u, -1, 2)
    rows = len(u)
    oqm = _lib()
    token = torch.empty(rows, dtype=torch.int32, device="cuda")
    oqm.stom_sample_tokens(x.expand(rows, 40).contiguous(), torch.from_numpy(u).cuda(), token)
    for i in range(rows):
        tokens, _, _ = K.choose(x.double().cpu().numpy()[0], min(max(float(u[i]), 0.0), 0.99999994))
        assert int(token[i]) in tokens


@pytest.mark.parametrize("dtype", [BF, HF, FL])
def test_equal_logits(dtype):
    """Ties go to the lower index, also at the borders of top-k and top-p; all of a row equal; +0 and -0 are equal."""
    n = 70000
    x = torch.zeros(6, n, dtype=dtype, device="cuda")
    x[1, ::2] = -0.0
    x[2, 5:n:7] = 1.0
    x[3, :] = -3.0
    x[4, n - 1] = 2.0
    u = [0.5, 0.25, 0.75, 0.9999, 0.3, 0.6]
    t, _ = _check(x, u)
    assert t[0] == n // 2 and t[1] == n // 4
    t, kept = _check(x, u, top_k=[4, 4, 3, 1, 2, 70000], top_p=[0.5, 1.0, 1.0, 1.0, 1.0, 0.5])
    assert kept.tolist()[:4] == [2, 4, 3, 1] and t[0] == 1 and t[1] == 1 and t[2] == 5 + 2 * 7 and t[3] == 0
    _check(x, u, temperature=0.0)


@pytest.mark.parametrize("dtype", [BF, HF, FL])
def test_masked_infinite_and_nan_logits(dtype):
    oqm = _lib()
    n = 5000
    x = _logits(8, n, dtype, seed=9)
    x[0] = -math.inf                                     # nothing allowed
    x[1] = -math.inf
    x[1, 4321] = -60000.0                                # one token, far down
    x[2, ::2] = -math.inf
    x[3, 7] = math.inf                                   # certain
    x[4, [9, 99, 999]] = math.inf                        # shared by three
    x[5] = torch.finfo(dtype).min                        # masks by the type's lowest value
    x[5, [3, 4]] = 1.0
    x[6] = torch.finfo(dtype).min
    t, kept = _check(x, [0.1, 0.5, 0.7, 0.9, 0.5, 0.8, 0.5, 0.2], ambiguous=0.2)
    assert t[0] == -1 and t[1] == 4321 and t[3] == 7 and t[4] == 99 and t[5] == 4
    assert kept.tolist()[3:5] == [1, 3] and int(kept[6]) == n
    _check(x, [0.1] * 8, temperature=0.0)
    _check(x, [0.9] * 8, temperature=0.5, top_k=20, top_p=0.9, min_p=0.1)
    x[2, 5], x[7, 0] = math.nan, math.nan
    _check(x, [0.1, 0.5, 0.7, 0.9, 0.5, 0.8, 0.5, 0.2], flags=oqm.FLAG_BAD_VALUE, ambiguous=0.2)


def test_settings_at_the_ends_of_their_ranges():
    oqm = _lib()
    x = _logits(6, 3000, BF, seed=11)
    u = _u(6, 11)
    base, _ = _check(x, u, temperature=[1e-30, 1e38, 0.0, -5.0, 1.0, 1.0], top_k=[0, 0, 0, 0, -3, 2 ** 31 - 1],
                     top_p=[1.0, 1.0, 0.5, 1.0, 7.0, -1.0], min_p=[0.0, 0.0, 0.0, 0.0, -1.0, 9.0])
    # infinite temperature: uniform; NaN settings count as not given, and are flagged
    f = torch.zeros(1, dtype=torch.int32, device="cuda")
    token, kept = (torch.empty(6, dtype=torch.int32, device="cuda") for _ in range(2))
    oqm.stom_sample_tokens(x, _f(0.5, 6), token, temperature=_f(math.inf, 6), kept=kept, dev_flags=f)
    order = np.argsort(-x.double().cpu().numpy(), axis=1, kind="stable")
    assert f.item() == 0 and (kept == 3000).all() and token.tolist() == order[:, 1500].tolist()
    oqm.stom_sample_tokens(x, _f(math.nan, 6), token, temperature=_f(math.nan, 6), top_p=_f(math.nan, 6),
                           min_p=_f(math.nan, 6), kept=kept, dev_flags=f)
    assert f.item() == oqm.FLAG_BAD_VALUE and (kept == 3000).all() and token.tolist() == order[:, 0].tolist()
    # u may be left out where a temperature is given
    oqm.stom_sample_tokens(x, None, token, temperature=_f(0.0, 6))
    assert token.tolist() == order[:, 0].tolist()


def test_strided_rows_and_a_captured_step():
    oqm = _lib()
    big = _logits(7, 4000, FL, seed=12)
    x = big[::2, 3:3500]
    _check(x, _u(4, 5), top_p=0.8)
    token, u = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    lo = x.contiguous()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        oqm.stom_sample_tokens(lo, u, token)
    for seed in range(3):
        u.copy_(torch.from_numpy(_u(4, seed)))
        lo.copy_(_logits(4, 3497, FL, seed=seed + 50))
        g.replay()
        torch.cuda.synchronize()
        for i in range(4):
            assert int(token[i]) in K.choose(lo[i].double().cpu().numpy(), float(u[i]))[0]


def test_draws_have_the_shares_of_the_distribution():
    """4 096 evenly spread random numbers give every token its share, to one draw at each of its two borders."""
    oqm = _lib()
    n, rows = 50, 4096
    x = _logits(1, n, BF, seed=20, spread=1.0)
    token = torch.empty(rows, dtype=torch.int32, device="cuda")
    u = (torch.arange(rows, device="cuda") + 0.5) / rows
    oqm.stom_sample_tokens(x.expand(rows, n).contiguous(), u, token)
    got = torch.bincount(token.long(), minlength=n).double().cpu().numpy()
    p = torch.softmax(x[0].double(), 0).cpu().numpy()
    assert (np.abs(got - p * rows) <= 1.0 + 1e-6).all()


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("n", [2, 9, 2000])
def test_log_probability_of_a_token_that_is_nearly_certain(dtype, n):
    """ln(w / mass) = -ln(1 + rest) where all the others weigh `rest` of the token drawn: relative to itself within the
    mass's own step, 2^-51 of the largest weight for every one of n <= 2048 tokens, and 2^-22 for the rest of the way."""
    oqm = _lib()
    gaps = [2.0, 8.0, 16.0, 20.0, 24.0]
    x = torch.zeros(len(gaps), n, dtype=dtype, device="cuda")
    x[:, n // 2] = torch.tensor(gaps, device="cuda").to(dtype)
    token, lp = torch.empty(len(gaps), dtype=torch.int32, device="cuda"), torch.empty(len(gaps), device="cuda")
    oqm.stom_sample_tokens(x, torch.zeros(len(gaps), device="cuda"), token, logprob=lp)
    for i, g in enumerate(gaps):
        rest = (n - 1) * math.exp(-g)
        want = -math.log1p(rest)
        assert int(token[i]) == n // 2
        assert abs(float(lp[i]) - want) <= abs(want) * 2.0 ** -22 + n * 2.0 ** -51


@pytest.mark.parametrize("dtype", [BF, HF, FL])
def test_every_nan_pattern_is_seen_and_never_drawn(dtype):
    """All bits set, as in a buffer that was filled with 0xff, among them; also at temperatures so high that the lowest
    finite logit keeps its weight."""
    oqm = _lib()
    word, patterns = ((torch.int32, [-1, -15, 0x7fffffff, 0x7fc00000]) if dtype is FL else
                      (torch.int16, [-1, -15, 0x7fff, 0x7fc0 if dtype is BF else 0x7e00]))
    n, temps = 3000, [1.0, 0.3, 90.0, 1e4, 1e38, 2e38]
    u = [0.2, 0.9, 0.5, 0.999, 0.7, 0.9999]
    for p in patterns:
        x = _logits(len(temps), n, dtype, seed=31)
        x[:, 100] = torch.finfo(dtype).min
        for where in (slice(7, 8), slice(0, 1500), slice(2000, 3000, 2)):
            y = x.clone()
            y.view(word)[:, where] = p
            _check(y, u, temperature=temps, flags=oqm.FLAG_BAD_VALUE, ambiguous=0.4)
            _check(y, u, temperature=temps, top_k=[0, 5, 2999, 2000, 0, 2999], top_p=[0.9, 1.0, 1.0, 0.999, 0.9, 1.0],
                   flags=oqm.FLAG_BAD_VALUE, ambiguous=0.4)
        y.view(word)[:] = p                              # nothing else
        t, kept = _check(y, u, temperature=temps, flags=oqm.FLAG_BAD_VALUE)
        assert (t == -1).all() and (kept == 0).all()


def _borders(n, part, near, far, seed):
    """A peak, one other token and n - 2 equal ones that weigh `part` of 2^-(62 - ceil(log2 n)) each, and random numbers
    u: rows whose border between the first two tokens lies between `near` and `far` of u, on either side."""
    bits = (n - 1).bit_length()
    low = np.float32(math.log(part) - (62 - bits) * math.log(2.0))
    tail = (n - 2) * math.exp(float(low))
    rows = []
    for second in np.random.default_rng(seed).uniform(-1.5, -0.1, 20000).astype(np.float32):
        border = 1.0 / (1.0 + math.exp(float(second)) + tail)
        u = np.float32(border)
        if near <= abs(float(u) / border - 1.0) <= far:
            rows.append((second, u, 0 if float(u) < border else 1))
        if len(rows) == 12:
            break
    assert len(rows) == 12 and len({r[2] for r in rows}) == 2
    return low, rows


@pytest.mark.parametrize("part", [0.49, 0.51, 1.49])
@pytest.mark.parametrize("n,near,far", [(131072, 1e-10, 6e-10), (500000, 2.4e-10, 4e-9)])
def test_masses_of_many_equal_light_tokens(n, near, far, part):
    """binary32: many tokens of half a unit each (the unit of the sums of ranges, 2^-45 and 2^-43 of the largest weight
    here) count for what they weigh together, in the draw and under top-p."""
    oqm = _lib()
    low, rows = _borders(n, part, near, far, n)
    x = torch.full((len(rows), n), float(low), device="cuda")
    x[:, 17] = 0.0
    x[:, n - 5] = torch.tensor([float(r[0]) for r in rows], device="cuda")
    v = torch.tensor([float(r[1]) for r in rows], device="cuda")
    second = torch.tensor([r[2] for r in rows], device="cuda")
    token, kept = (torch.empty(len(rows), dtype=torch.int32, device="cuda") for _ in range(2))
    oqm.stom_sample_tokens(x, v, token, kept=kept)
    assert token.tolist() == torch.where(second == 1, n - 5, 17).tolist() and (kept == n).all()
    oqm.stom_sample_tokens(x, torch.zeros_like(v), token, top_p=v, kept=kept)
    assert kept.tolist() == (second + 1).tolist() and (token == 17).all()
    # all but the peak equal, and the draw among them: a token's place to within what a row of weights is off by
    x[:, n - 5] = float(low)
    total = 1.0 + (n - 1) * math.exp(float(low))
    logp = torch.empty(len(rows), device="cuda")
    oqm.stom_sample_tokens(x, torch.zeros_like(v), token, logprob=logp)
    assert (token == 17).all()
    assert (logp.double() + math.log(total)).abs().max() <= 2.4e-10 + 2.0 ** -22 * math.log(total)


@pytest.mark.parametrize("dtype", [BF, HF, FL])
def test_the_highest_temperatures(dtype):
    """At T = inf every finite logit weighs the same, the type's lowest value too; just below it the formula holds."""
    x = _logits(6, 3000, dtype, seed=33)
    x[:, 5:2000:3] = torch.finfo(dtype).min
    x[3:, 9] = torch.finfo(dtype).max
    u, temps = [0.3, 0.61, 0.97, 0.2, 0.7, 0.99], [math.inf, 3.3e38, 3.4e38, math.inf, 3.3e38, 3.4e38]
    t, kept = _check(x, u, temperature=temps, ambiguous=0.4)
    assert (kept == 3000).all()
    _check(x, u, temperature=temps, top_p=0.7, min_p=0.05, ambiguous=0.4)
    _check(x, u, temperature=temps, top_k=500, ambiguous=0.4)
    x[:, 20:23] = math.inf                               # these share the mass at any temperature
    t, kept = _check(x, u, temperature=temps, ambiguous=0.4)
    assert (kept == 3).all() and (t >= 20).all() and (t < 23).all()
