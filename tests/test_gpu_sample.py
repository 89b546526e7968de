"""jb_sample against its definition. The weights are rint(2^30 exp(y)) with exp in fp32, which torch
computes here; everything after them is whole numbers, so tokens are compared exactly. That the weights
are those of a softmax is checked against 64 bits: fp32's y is off by up to |y| 2^-23 and its exponential
by 2^-22, so a weight by less than 2^30 e^y (|y| 2^-23 + 2^-22) + 1, and so is a running sum of them."""
import math

import numpy as np
import pytest
import torch

import paper_2306_10015_gb300 as jb

pytestmark = pytest.mark.gpu


def define(logits, words, temperature, top_k, top_p, min_p):
    """Tokens and log-probabilities (the latter in 64 bits from the whole-numbered weights)."""
    n, V = logits.shape
    x = logits.float()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    top = x.amax(1, keepdim=True)
    T = temperature[:, None]
    greedy = ~(T >= 2.0**-64)
    y = (x - top) * (1.0 / torch.where(greedy, torch.ones_like(T), T))
    y = torch.where(x == top, torch.zeros_like(y), y)
    w = torch.round(torch.exp(y) * 2.0**30).long().cpu().numpy()
    x, y = x.cpu().numpy() + 0.0, y.double().cpu().numpy()
    tokens, logprobs = [], []
    for i in range(n):
        if np.isneginf(x[i]).all():
            tokens.append(-1)
            logprobs.append(-math.inf)
            continue
        order = np.argsort(-x[i].astype(np.float64), kind="stable")
        k = 1 if greedy[i, 0] else int(top_k[i])
        if 0 < k < V:
            order = order[:k]
        mass = np.cumsum(w[i][order])
        p = float(top_p[i])
        if p < 1:
            goal = max(1, math.ceil(max(p, 0.0) * float(mass[-1])))
            order = order[: int(np.searchsorted(mass, goal)) + 1]
        m = float(min_p[i])
        cut = math.ceil(min(m, 1.0) * 2.0**30) if m > 0 else 0
        keep = np.sort(order[w[i][order] >= cut])
        mass = np.cumsum(w[i][keep])
        aim = (int(words[i]) & 0xFFFFFFFF) * int(mass[-1]) >> 32
        t = int(keep[np.searchsorted(mass, aim, side="right")])
        tokens.append(t)
        logprobs.append(y[i, t] - math.log(int(mass[-1]) / 2.0**30))
    return tokens, logprobs


def settings(n, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    f = lambda v, dt: torch.as_tensor(v, dtype=dt).expand(n).contiguous().cuda()  # noqa: E731
    return f(temperature, torch.float32), f(top_k, torch.int32), f(top_p, torch.float32), f(min_p, torch.float32)


def words_of(n, seed=0):
    g = np.random.default_rng(seed)
    w = g.integers(0, 1 << 32, size=n, dtype=np.uint64).astype(np.uint32)
    w[: min(n, 2)] = [0, 0xFFFFFFFF][: min(n, 2)]
    return torch.from_numpy(w.view(np.int32)).cuda()


def check(logits, words=None, **kw):
    n = logits.shape[0]
    words = words_of(n) if words is None else words
    t, k, p, m = settings(n, **kw)
    got, lp = jb.jb_sample(logits, words, temperature=t, top_k=k, top_p=p, min_p=m)
    want, want_lp = define(logits, words.tolist(), t, k.tolist(), p.tolist(), m.tolist())
    assert got.tolist() == want
    # y, the logarithm of the sum and their difference: a few fp32 roundings of operands below 64
    for a, b in zip(lp.tolist(), want_lp):
        assert a == b or abs(a - b) <= 2.0**-21 * (1 + abs(b)) + 2.0**-19, (a, b)
    return got


def logits_of(n, V, dtype, seed=0, std=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, V, generator=g, device="cuda") * std).to(dtype)


FILTERS = [dict(), dict(temperature=0.0), dict(temperature=0.3), dict(temperature=7.0), dict(top_k=1), dict(top_k=2), dict(top_k=40),
           dict(top_p=0.9), dict(top_p=0.1), dict(top_p=0.0), dict(top_p=-1.0), dict(top_p=0.9999999), dict(top_p=math.nan), dict(min_p=0.05),
           dict(min_p=1.0), dict(min_p=3.0), dict(min_p=math.nan), dict(temperature=0.8, top_k=50, top_p=0.95, min_p=0.01),
           dict(temperature=2.0, top_k=500, top_p=0.5, min_p=0.001), dict(top_k=1 << 30), dict(top_k=-3), dict(temperature=math.nan),
           dict(temperature=1e-30), dict(temperature=1e30), dict(temperature=-1.0), dict(temperature=math.inf)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("f", FILTERS, ids=str)
def test_filters(dtype, f):
    check(logits_of(9, 5003, dtype), **f)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 3, 31, 33, 1023, 1024, 1025, 4099, 32_000, 50_272, 131_071, 262_144])
def test_vocabularies(dtype, V):
    x = logits_of(5, V, dtype, seed=V)
    check(x)
    check(x, temperature=0.9, top_k=min(V, 100), top_p=0.9)
    check(x, top_p=0.97, min_p=0.003)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", [(1, 50_272), (5, 3001), (300, 9001)])
@pytest.mark.parametrize("std", [1.0, 6.0, 30.0])
def test_few_and_many_kept(dtype, n, V, std):
    """Nuclei of a few tokens and of most of them, and top-k around what one list holds."""
    x = logits_of(n, V, dtype, seed=3, std=std)
    check(x, top_p=0.9)
    check(x, top_p=0.999, min_p=0.01)
    check(x, top_k=127, top_p=0.9)
    check(x, top_k=128, min_p=0.02)
    check(x, top_k=257, top_p=0.7)


@pytest.mark.parametrize("n", [1, 2, 7, 63, 152, 153, 300, 1000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows(n, dtype):
    g = np.random.default_rng(n)
    check(logits_of(n, 2051, dtype, seed=n), temperature=torch.from_numpy(g.choice([0.0, 0.5, 1.0, 1.7], size=n)),
          top_k=torch.from_numpy(g.choice([0, 1, 30, 5000], size=n)), top_p=torch.from_numpy(g.choice([1.0, 0.8, 0.2], size=n)),
          min_p=torch.from_numpy(g.choice([0.0, 0.1], size=n)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("f", [dict(), dict(top_k=5), dict(top_p=0.4), dict(top_k=700, top_p=0.5), dict(temperature=0.0), dict(min_p=0.5)], ids=str)
def test_ties_go_to_the_lowest_index(dtype, f):
    x = torch.zeros(6, 3001, device="cuda")
    x[1] = 2.5
    x[2, ::2] = 1.0
    x[3, 1000:] = -0.0                                     # equal to 0
    x[4] = torch.randint(0, 4, (3001,), device="cuda").float()
    x[5, 7] = 1e-30
    check(x.to(dtype), words=words_of(6, 3), **f)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("f", [dict(), dict(top_k=3), dict(top_p=0.5), dict(temperature=0.0), dict(top_k=2000, top_p=0.9, min_p=0.01)], ids=str)
def test_infinities_and_nan(dtype, f):
    x = logits_of(9, 1500, torch.float32)
    x[0] = -math.inf                                       # nothing to draw
    x[1] = math.nan
    x[2, ::3] = math.nan
    x[3, 100:1400] = -math.inf
    x[4, [5, 900]] = math.inf                              # these share the draw
    x[5] = -math.inf
    x[5, 1499] = -3e38
    x[6] = torch.finfo(dtype).min                          # a mask of the type's lowest value
    x[7] = torch.finfo(dtype).min
    x[7, 77] = 1.0
    x[8, 0], x[8, 1] = 3e38, -3e38
    got = check(x.to(dtype), words=words_of(9, 5), **f).tolist()
    assert got[0] == got[1] == -1 and got[4] in (5, 900) and got[5] == 1499 and got[7] == 77 and got[8] == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_draws_follow_the_softmax(dtype):
    """4096 evenly spaced words over one row: the token changes where the running sum of the exact
    probabilities passes the word, within the weights' error."""
    n, V = 4096, 700
    row = logits_of(1, V, dtype, std=2.0)
    words = (torch.arange(n, device="cuda") * (1 << 20)).to(torch.int32)
    got, _ = jb.jb_sample(row.expand(n, V), words, temperature=0.7)
    y = (row[0].double() - row[0].double().max()) / float(np.float32(0.7))
    e = torch.exp(y)
    run = (torch.cumsum(e, 0) / e.sum()).cpu().numpy()
    err = float(((e * (y.abs() * 2.0**-22 + 2.0**-22)).sum() + V * 2.0**-30) / e.sum()) + 2.0**-30
    u = np.arange(n) / n
    t = got.cpu().numpy()
    assert (u < run[t] + err).all() and (u >= np.concatenate([[0], run])[t] - err).all()


def test_nan_payloads_strides_and_defaults():
    x = logits_of(4, 3000, torch.bfloat16)
    wide = torch.full((4, 6001), 99.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 1501:4501] = x                                # an odd element to start from
    w = words_of(4, 9)
    a, la = jb.jb_sample(x, w)
    b, lb = jb.jb_sample(wide[:, 1501:4501], w.view(torch.uint32), temperature=1.0)
    assert torch.equal(a, b) and torch.equal(la, lb)
    tokens, lp = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    c, lc = jb.jb_sample(x, w, top_k=9, temperature=0.5, tokens=tokens, logprobs=lp, stream=s)
    s.synchronize()
    assert c is tokens and lc is lp
    assert tokens.tolist() == define(x, w.tolist(), *[v if i == 0 else v.tolist() for i, v in enumerate(settings(4, 0.5, 9))])[0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_repeat_whatever_is_beside_them(dtype):
    x, w = logits_of(400, 9001, dtype), words_of(400, 4)
    all_, lp = jb.jb_sample(x, w, top_p=0.9, top_k=300)
    for i in (0, 1, 151, 399):
        one, l1 = jb.jb_sample(x[i:i + 1], w[i:i + 1], top_p=0.9, top_k=300)
        assert one.item() == all_[i].item() and l1.item() == lp[i].item()


# For each min_p the tail's y, on both sides of where a weight reaches the least that is kept: ln((least - 1/2) / 2^30), since
# weights are rounded (least = ceil(min_p 2^30) = 1, 2, 11, 43).
SMALL_MIN_P = [(2.0**-30, -21.7, -20.6), (1.8e-9, -20.6, -19.9), (1e-8, -18.5, -18.38), (4e-8, -17.06, -17.03)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", [(1, 50_272), (40, 5003), (200, 20_001)])
@pytest.mark.parametrize("min_p,low,high", SMALL_MIN_P)
@pytest.mark.parametrize("f", [dict(), dict(top_k=3000), dict(top_k=900, top_p=1 - 2.0**-24)], ids=str)
def test_min_p_keeps_weights_that_round_up_to_the_least(dtype, n, V, min_p, low, high, f):
    """One likely token before a tail whose weights are a few units: the words are spread over the tail's share of
    the draw, so that a token which is left out, or counted in one place alone, moves the tokens after it."""
    g = torch.Generator(device="cuda").manual_seed(V)
    x = low + (high - low) * torch.rand(n, V, generator=g, device="cuda")
    x[:, 0] = 0.0
    x = x.to(dtype)
    w = torch.round(torch.exp(x[0].float()) * 2.0**30)
    w[w < math.ceil(float(np.float32(min_p)) * 2**30)] = 0
    k = min(f.get("top_k", V), V)
    share = float(w.sort(descending=True)[0][1:k].sum()) / 2.0**30
    words = [(1 << 32) - 1 - int(i / n * share * 2.0**32) for i in range(n)]
    words = torch.from_numpy(np.array(words, dtype=np.uint64).astype(np.uint32).view(np.int32)).cuda()
    got = check(x, words=words, min_p=min_p, **f)
    if k == V and share > 0:
        assert (got > 0).any()
