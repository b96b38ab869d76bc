"""Sampling on the GPU against the oracle in extended precision."""

import math

import numpy as np
import pytest
import torch

from oracle import sampling as oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    from paper_2607_14431_amd import kvg as k
    return k


def run(kvg, logits, temperature, u, top_k=None, top_p=None, min_p=None, ws=None):
    R, V = logits.shape
    dev = lambda x, t: None if x is None else torch.as_tensor(np.asarray(x), dtype=t).cuda()  # noqa: E731
    tokens = torch.full((R,), 77, dtype=torch.int32, device="cuda")
    logprobs = torch.full((R,), 77.0, device="cuda")
    kvg.kvg_sample(logits, dev(temperature, torch.float32), dev(u, torch.float64), tokens, ws if ws is not None else kvg.sample_workspace(R, V),
                   top_k=dev(top_k, torch.int32), top_p=dev(top_p, torch.float32), min_p=dev(min_p, torch.float32), logprobs=logprobs)
    return tokens.cpu().numpy(), logprobs.cpu().numpy()


def compare(logits, temperature, u, tokens, logprobs, top_k=None, top_p=None, min_p=None, most_close=0, always=()):
    """Rows against the oracle.  A weight is rounded by 2^-(bits + 1) at most, bits = 62 - ceil(log2 V), so a sum of V of them is off
    by V 2^-(bits + 1) <= 2^(2 ceil(log2 V) - 63), and fp64's exponentials and products by less than 2^-45 of a total
    of at most V; a row whose choice is closer than that (twice: both sides of a comparison) is not compared.  The
    logarithm's argument is known to that over the total (at least 1), and rounds to fp32."""
    R, V = logits.shape
    off = 2.0 ** (2 * math.ceil(math.log2(max(V, 2))) - 63) + V * 2.0 ** -45
    host = logits.cpu().numpy()
    f = lambda x, r, d: d if x is None else float(np.float32(x[r])) if d != 0 or x is not top_k else int(x[r])  # noqa: E731
    close = 0
    for r in range(R):
        token, logprob, margin = oracle.sample(host[r], float(np.float32(temperature[r])), float(u[r]), 0 if top_k is None else int(top_k[r]),
                                               f(top_p, r, 1.0), 0.0 if min_p is None else float(np.float32(min_p[r])))
        if margin <= 2 * off and r not in always:
            close += 1
            continue
        assert tokens[r] == token, (r, tokens[r], token, margin)
        if token < 0:
            assert math.isnan(logprobs[r])
        else:
            assert abs(float(logprobs[r]) - logprob) <= 2.0 ** -24 * abs(logprob) + 2 * off + 1e-30
    assert close <= most_close, close


def logits_like(gen, R, V, sigma=3.0):
    z = torch.empty((R, V), device="cuda").normal_(0.0, sigma, generator=gen)
    if V >= 48:
        z.scatter_add_(1, torch.randint(0, V, (R, 48), generator=gen, device="cuda"), torch.rand((R, 48), generator=gen, device="cuda") * 16.0)
    return torch.tanh(z / 30.0) * 30.0


FILTERS = [dict(), dict(top_k=[1, 2, 20, 50, 0, 1 << 30, -3]), dict(top_p=[0.9, 0.5, 0.01, 1.0, 2.0, 0.0, 0.999]),
           dict(min_p=[0.1, 0.0, 0.5, 1.0, 0.001, 3.0, -1.0]),
           dict(top_k=[50, 64, 5, 0, 1000, 3, 20], top_p=[0.9, 0.95, 0.3, 0.8, 0.99, 1.0, 0.5]),
           dict(top_k=[50, 64, 5, 0, 300, 3, 20], top_p=[0.9, 0.95, 0.3, 0.8, 0.999, 1.0, 0.5], min_p=[0.05, 0.02, 0.0, 0.01, 0.0, 0.3, 0.1])]


@pytest.mark.parametrize("filters", FILTERS, ids=lambda f: "-".join(f) or "none")
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 4099, 32768, 50021, 262144])
def test_tokens(kvg, filters, V):
    R = 7
    gen = torch.Generator(device="cuda").manual_seed(V)
    rng = np.random.default_rng(V)
    logits = logits_like(gen, R, V)
    for temperature in ([1.0] * R, [0.7, 0.0, 1.3, 0.05, 8.0, 0.5, 1.0]):
        u = rng.random(R)
        # a number falls within 2 off of one of V borders, in a total of 1 at least, with a chance of at most 4 off V: 0.024 at
        # 262,144 (off 2.3e-8), 0.0002 at 50,257; a row has two such numbers (u, top_p), so one row in seven may be at the largest
        compare(logits, temperature, u, *run(kvg, logits, temperature, u, **filters), **filters, most_close=int(V > 131072))


def test_many_draws_of_a_row(kvg):
    """Every token of a small row, at the ends of its interval as well."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    logits = logits_like(gen, 1, 40, 1.0)
    w = torch.softmax(logits[0].double(), 0).cpu().numpy()
    c = np.concatenate([[0], np.cumsum(w)])
    u = np.concatenate([c[:-1] + 1e-9, c[1:] - 1e-9, (c[:-1] + c[1:]) / 2])
    many = logits.repeat(len(u), 1)
    tokens, _ = run(kvg, many, [1.0] * len(u), u)
    assert np.array_equal(tokens, np.tile(np.arange(40), 3))
    tokens, _ = run(kvg, many[:6], [1.0] * 6, [0.0, -1.0, 1.0, 5.0, math.inf, -math.inf])
    assert tokens.tolist() == [0, 0, 39, 39, 39, 0]


@pytest.mark.parametrize("V", [1000, 70000])
def test_ties(kvg, V):
    """Rows of equal logits, of few values, and of both zeros: of equal ones the lowest index first."""
    rng = np.random.default_rng(2)
    rows = [np.zeros(V), np.full(V, -7.25), rng.integers(0, 3, V), np.where(rng.random(V) < 0.5, 0.0, -0.0), rng.integers(-1, 1, V) * 40.0,
            np.where(np.arange(V) % 7 == 3, 2.0, -math.inf)]
    logits = torch.from_numpy(np.stack(rows)).float().cuda()
    R = len(rows)
    for filters in (dict(), dict(top_k=[5, 500, 700, 64, 3, 90]), dict(top_p=[0.5, 0.123, 0.9, 0.25, 0.6, 0.31]),
                    dict(top_k=[5, 500, 700, 64, 999, 90], top_p=[0.5, 0.123, 0.9, 0.3, 0.6, 0.31], min_p=[0.5] * R)):
        u = rng.random(R)
        # rows 0, 1 and 3 have equal weights, which both sides sum exactly: a share that a sum meets is met
        compare(logits, [1.0] * R, u, *run(kvg, logits, [1.0] * R, u, **filters), **filters, always=(0, 1, 3))


def test_masked_and_bad_rows(kvg):
    V = 3001
    rng = np.random.default_rng(2)
    x = rng.normal(size=(12, V)).astype(np.float32)
    x[0, :] = -math.inf                                        # nothing left
    x[1, :-1] = -math.inf                                      # one token left
    x[2, 100] = math.nan
    x[3, 7] = math.inf
    x[4, rng.random(V) < 0.9] = -math.inf
    x[5, 5] = -math.nan
    x[6] = x[6] * 1e38                                         # differences past fp32's range
    temperature = [1.0, 0.3, 1.0, 0.0, 1.0, 1.0, 1.0, math.nan, -1.0, math.inf, 1e-42, 3e38]
    logits = torch.from_numpy(x).cuda()
    u = rng.random(12)
    for filters in (dict(), dict(top_k=[40] * 12, top_p=[0.9] * 12)):
        tokens, logprobs = run(kvg, logits, temperature, u, **filters)
        compare(logits, temperature, u, tokens, logprobs, **filters)
        assert tokens[[0, 2, 3, 5, 7, 8, 9]].tolist() == [-1] * 7 and tokens[1] == V - 1 and tokens[10] == x[10].argmax()
    ok = [1.0] * 12
    for kw in (dict(u=np.full(12, math.nan)), dict(top_p=[math.nan] * 12), dict(min_p=[math.nan] * 12)):
        tokens, logprobs = run(kvg, logits, ok, **{"u": u, **kw})
        assert (tokens == -1).all() and np.isnan(logprobs).all()


@pytest.mark.parametrize("V", [999, 131072])
def test_a_row_alone_and_in_a_batch(kvg, V):
    gen = torch.Generator(device="cuda").manual_seed(9)
    R = 40
    wide = logits_like(gen, R, V + 13)
    logits = wide[:, 5:5 + V]                                  # strided, not on 16 bytes
    rng = np.random.default_rng(1)
    u, t, k, p = rng.random(R), rng.choice([0.0, 0.6, 1.0], R), rng.choice([0, 10, 400], R), rng.choice([1.0, 0.9, 0.4], R)
    tokens, logprobs = run(kvg, logits, t, u, k, p)
    again = run(kvg, logits.contiguous(), t, u, k, p)
    assert np.array_equal(tokens, again[0]) and np.array_equal(logprobs.view(np.int32), again[1].view(np.int32))
    for r in (0, 7, 39):
        one = run(kvg, logits[r:r + 1], t[r:r + 1], u[r:r + 1], k[r:r + 1], p[r:r + 1])
        assert one[0][0] == tokens[r] and one[1][0] == logprobs[r]


def test_captured_replays(kvg):
    R, V = 3, 40000
    gen = torch.Generator(device="cuda").manual_seed(4)
    logits = torch.zeros((R, V), device="cuda")
    t, u = torch.ones(R, device="cuda"), torch.zeros(R, dtype=torch.float64, device="cuda")
    k, p = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.ones(R, device="cuda")
    tokens, logprobs = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, device="cuda")
    ws = kvg.sample_workspace(R, V)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kvg.kvg_sample(logits, t, u, tokens, ws, top_k=k, top_p=p, logprobs=logprobs)
    for turn in range(5):
        logits.copy_(logits_like(gen, R, V))
        u.uniform_(generator=gen)
        t.fill_(0.5 + 0.2 * turn)
        k.copy_(torch.tensor([0, 50, 9 * turn], dtype=torch.int32))
        p.fill_(0.9 if turn % 2 else 1.0)
        g.replay()
        torch.cuda.synchronize()
        want = run(kvg, logits, t.cpu(), u.cpu(), k.cpu(), p.cpu())
        assert np.array_equal(tokens.cpu().numpy(), want[0]) and np.array_equal(logprobs.cpu().numpy(), want[1])


def test_frequencies(kvg):
    """Random numbers spread evenly give every token its share: the largest gap between the counts and the shares is below two
    steps of the numbers."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    n = 4096
    logits = logits_like(gen, 1, 30, 1.5)
    u = (np.arange(n) + 0.5) / n
    tokens, _ = run(kvg, logits.expand(n, 30).contiguous(), [1.0] * n, u)
    share = torch.softmax(logits[0].double(), 0).cpu().numpy()
    assert np.abs(np.bincount(tokens, minlength=30) / n - share).max() <= 2.0 / n


@pytest.mark.parametrize("V", [4000, 50021])
def test_limits_among_many_close_logits(kvg, V):
    """Hundreds to thousands of tokens of nearly or exactly equal logits where a limit ends, side by side in a part of the row or
    all over it, fewer and more of them than are listed; a few far above them or none."""
    rng = np.random.default_rng(V)
    rows = []
    for spread in (0.0, 1e-6, 0.01, 0.3, 3.0):
        for n in (150, 700, 3000, V):
            for together in (True, False):
                x = rng.uniform(-40.0, -30.0, V)
                at = np.arange(500, 500 + n) % V if together else rng.permutation(V)[:n]
                x[at] = 2.0 + spread * rng.random(n)
                x[rng.integers(0, V, 3)] = [7.0, 6.5, 6.0]
                rows.append(x)
    R = len(rows)
    logits = torch.from_numpy(np.stack(rows).astype(np.float32)).cuda()
    pick = lambda x: np.array([x[i % len(x)] for i in range(R)])  # noqa: E731
    u, temperature = rng.random(R), pick([1.0, 0.7, 1.3])
    for limits in (dict(top_k=pick([40, 100, 600, 900, 2000])), dict(top_p=pick([0.5, 0.9, 0.1, 0.99])),
                   dict(top_k=pick([40, 100, 600, 900, 1500]), top_p=pick([0.5, 0.9, 0.99])),
                   dict(top_k=pick([1024, 1025, 3000]), top_p=pick([0.3, 0.8]), min_p=pick([0.0, 0.001]))):
        tokens, logprobs = run(kvg, logits, temperature, u, **limits)
        compare(logits, temperature, u, tokens, logprobs, **limits)


def test_logits_far_apart(kvg):
    """Finite logits at the ends of fp32's range and temperatures at its ends."""
    V = 3000
    rng = np.random.default_rng(1)
    x = rng.standard_normal((6, V)).astype(np.float32)
    x[0, 5], x[0, 6] = 3.4e38, -3.4e38
    x[1] *= np.float32(1e-38)
    x[2, 100:] = -np.inf
    x[3] *= np.float32(1e37)
    temperature = [1.0, 1e-38, 1.0, 1e38, 1e-30, 3e38]
    u = rng.random(6)
    logits = torch.from_numpy(x).cuda()
    for limits in (dict(), dict(top_k=[50] * 6), dict(top_p=[0.9] * 6), dict(top_k=[200] * 6, top_p=[0.7] * 6, min_p=[0.01] * 6)):
        limits = {k: np.array(v) for k, v in limits.items()}
        tokens, logprobs = run(kvg, logits, temperature, u, **limits)
        compare(logits, temperature, u, tokens, logprobs, **limits)


def test_a_long_vocabulary(kvg):
    """Parts of more tokens than a workgroup takes at the end.  With 41 bits after the point, 2 off is 1.1e-6 of the likeliest token's
    weight, and the broad base (logits N(0, 2), 16 and more below the likeliest) weighs e^-16 = 1e-7 a token at temperature 1: a row
    whose number or limit falls into its base cannot be compared.  Its base is 2e6 E[e^x] e^-18 = 2e6 e^2 e^-18 = 0.2 beside a
    few units of likely tokens, so a top-p of 0.999 ends there always and a number falls there now and then: two rows of four."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    R, V = 4, 2_000_003
    logits = logits_like(gen, R, V, 2.0)
    rng = np.random.default_rng(2)
    for limits in (dict(), dict(top_k=np.array([50, 1000, 5000, V])), dict(top_p=np.array([0.9, 0.3, 0.999, 0.01])),
                   dict(top_k=np.array([64, 900, 4000, 0]), top_p=np.array([0.9, 0.95, 0.5, 0.99]), min_p=np.array([0.0, 0.01, 0.0, 0.001]))):
        u = rng.random(R)
        tokens, logprobs = run(kvg, logits, [1.0, 0.8, 1.2, 0.6], u, **limits)
        compare(logits, [1.0, 0.8, 1.2, 0.6], u, tokens, logprobs, **limits, most_close=2)


def test_more_equal_logits_than_are_listed(kvg):
    """The end of a limit among 5,000 and more tokens of one logit, by index, and among their neighbours."""
    V = 70000
    rng = np.random.default_rng(3)
    x = np.full((6, V), -20.0, dtype=np.float32)
    for r in range(6):
        x[r, rng.permutation(V)[:5000 + 9000 * r]] = 1.5
        x[r, rng.integers(0, V, 20)] = 3.0
        x[r, rng.integers(0, V, 20)] = np.float32(1.5) + np.float32(2.0 ** -20)
    u = rng.random(6)
    logits = torch.from_numpy(x).cuda()
    for limits in (dict(top_k=[100, 3000, 5020, 6000, 20000, 40]), dict(top_p=[0.5, 0.1, 0.9, 0.99, 0.3, 0.7]),
                   dict(top_k=[900, 1000, 4000, 9000, 30000, 1024], top_p=[0.5, 0.9, 0.5, 0.1, 0.9, 0.3])):
        limits = {k: np.array(v) for k, v in limits.items()}
        tokens, logprobs = run(kvg, logits, [1.0] * 6, u, **limits)
        compare(logits, [1.0] * 6, u, tokens, logprobs, **limits, always=range(6))
