"""Sampling with each sequence's own options on the GPU, token for token what the definition gives in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
from tests import gpu_util as gu
from tests import sample_ref

pytestmark = pytest.mark.gpu


def _sample(x, u, **options):
    import paper_2604_12989_amd as dd
    batch, T, V = x.shape
    ws = dd.Workspace(batch, 1, V, max(1, T - 1), 1, 1, 64, 0)
    out = dd.sample(gu.to_dev(x.astype(np.float32)), gu.to_dev(u.astype(np.float32)), ws, **options)
    torch.cuda.synchronize()
    return out.cpu().numpy()


def _check(x, u, **options):
    got = _sample(x, u, **options)
    o = {"tau" if k == "temperature" else k: v for k, v in options.items()}
    want = sample_ref.tokens(x, u, **{"tau": 1.0, **o})
    assert np.array_equal(got, want), (np.argwhere(got != want)[:5].tolist(), got[got != want][:5], want[got != want][:5])
    return got


def _rows(rng, batch, T, V, kind):
    x = 2.0 * rng.standard_normal((batch, T, V))
    if kind == "peaked":
        head = min(V, 40)
        for b in range(batch):
            for i in range(T):
                x[b, i, rng.permutation(V)[:head]] += 16.0 - np.cumsum(rng.random(head)) * 0.5
    elif kind == "flat":
        x *= 0.25
    elif kind == "wide":                      # far tails: many weights near the smallest that counts
        x *= 5.0
    return x.astype(np.float32)


OPTIONS = [dict(), dict(temperature=0.0), dict(temperature=0.3), dict(temperature=2.5), dict(top_k=1), dict(top_k=40), dict(top_k=700),
           dict(top_p=0.9), dict(top_p=0.3), dict(min_p=0.05), dict(min_p=1.0), dict(top_k=50, top_p=0.95), dict(top_p=0.97, min_p=0.02),
           dict(temperature=0.7, top_k=200, top_p=0.8, min_p=0.01)]


@pytest.mark.parametrize("kind", ["peaked", "flat", "wide", "bulk"])
@pytest.mark.parametrize("V", [1, 2, 7, 130, 1000, 2045, 6141, 32003])
def test_every_option_over_sizes(kind, V):
    rng = np.random.default_rng(V)
    for options in OPTIONS:
        x = _rows(rng, 2, 3, V, kind)
        _check(x, rng.random((2, 3)), **options)


@pytest.mark.parametrize("kind", ["peaked", "flat", "wide"])
def test_full_vocabulary(kind):
    rng = np.random.default_rng(11)
    x = _rows(rng, 1, 24, 151936, kind)
    for options in (dict(), dict(top_k=50, top_p=0.95), dict(temperature=0.6, top_p=0.9), dict(min_p=0.1), dict(top_k=1000), dict(top_k=20000),
                    dict(temperature=1.5, top_p=0.99), dict(top_k=5000, top_p=0.5, min_p=0.001)):
        _check(x, rng.random((1, 24)), **options)


@pytest.mark.parametrize("top_k", [32003, 32004, 1 << 30, (1 << 31) - 1])
def test_top_k_as_long_as_the_row_and_longer(top_k):
    rng = np.random.default_rng(14)
    for kind in ("peaked", "flat"):
        x, u = _rows(rng, 2, 3, 32003, kind), rng.random((2, 3))
        for rest in (dict(), dict(top_p=0.9), dict(min_p=0.1)):
            assert np.array_equal(_check(x, u, top_k=top_k, **rest), _sample(x, u, **rest))


@pytest.mark.parametrize("V", [1 << 21, (1 << 21) + 1, 1 << 22])
def test_largest_vocabularies(V):
    rng = np.random.default_rng(V)
    for kind in ("peaked", "flat"):
        x, u = _rows(rng, 1, 2, V, kind), rng.random((1, 2))
        for options in (dict(), dict(top_k=50, top_p=0.95), dict(top_p=0.9), dict(top_k=100000), dict(min_p=0.3)):
            _check(x, u, **options)


def test_many_rows_take_long_segments():
    rng = np.random.default_rng(12)
    x = _rows(rng, 3, 33, 50021, "peaked")
    x[1] = _rows(rng, 1, 33, 50021, "flat")[0]
    _check(x, rng.random((3, 33)), temperature=[0.8, 1.0, 0.0], top_k=[0, 30, 9], top_p=[0.9, 1.0, 0.2], min_p=[0.0, 0.0, 0.5])
    _check(x, rng.random((3, 33)), temperature=[0.8, 1.0, 1.2], top_p=[0.9, 0.7, 1.0], min_p=[0.0, 0.2, 0.0])


@pytest.mark.parametrize("options", [dict(top_p=0.9), dict(top_k=1500), dict(top_k=1500, top_p=0.7), dict(min_p=0.2),
                                     dict(top_p=0.95, min_p=0.3, temperature=1.3)])
def test_more_flat_rows_than_have_room_together(options):
    """600 rows that their lists do not hold; every third value is the same in all of them."""
    rng = np.random.default_rng(13)
    x = _rows(rng, 2, 300, 3001, "flat")
    x[:, :, ::3] = 0.25
    _check(x, rng.random((2, 300)), **options)


@pytest.mark.parametrize("V", [50, 3000, 70000])
def test_ties(V):
    """Rows of equal logits and of a few values: ranks and running sums go by the ids."""
    rng = np.random.default_rng(V)
    u = np.array([[0.0, 0.25, 0.5, 0.75, 0.9999999]])
    for x in (np.zeros((1, 5, V)), rng.integers(0, 3, (1, 5, V)) * 1.0, np.where(rng.random((1, 5, V)) < 0.5, -0.0, 0.0)):
        for options in (dict(), dict(top_k=7), dict(top_k=min(V, 2500)), dict(top_p=0.5), dict(top_p=0.9), dict(min_p=1.0), dict(min_p=0.3),
                        dict(top_k=20, top_p=0.25), dict(temperature=1e-30), dict(temperature=1e30, top_p=0.125)):
            _check(x.astype(np.float32), u, **options)


@pytest.mark.parametrize("low", [-np.inf, -1e9, np.finfo(np.float32).min])
def test_masked_tokens(low):
    rng = np.random.default_rng(4)
    V = 20011
    x = _rows(rng, 1, 6, V, "bulk")
    keep = rng.random((1, 6, V)) < 0.002
    keep[0, 0] = False
    keep[0, 0, 777] = True                        # one token left
    keep[0, 1] = False
    keep[0, 1, [5, V - 1]] = True
    x = np.where(keep, x, np.float32(low)).astype(np.float32)
    for options in (dict(), dict(top_k=5), dict(top_k=3000), dict(top_p=0.9), dict(min_p=0.1), dict(temperature=0.0)):
        got = _check(x, rng.random((1, 6)), **options)
        assert keep[0, np.arange(6), got[0]].all()


def test_rows_without_a_token_and_rows_with_infinities():
    V = 5000
    rng = np.random.default_rng(6)
    x = _rows(rng, 1, 8, V, "bulk")
    x[0, 0] = -np.inf
    x[0, 1, ::2] = np.nan
    x[0, 2, [17, 4000]] = np.inf
    x[0, 3] = np.nan
    x[0, 4, 100] = np.finfo(np.float32).max
    x[0, 5] = -np.inf
    x[0, 5, 9] = -1e38
    x[0, 6] *= 1e37
    u = rng.random((1, 8))
    for options in (dict(), dict(top_k=3), dict(top_p=0.9), dict(min_p=0.5), dict(temperature=0.0)):
        got = _check(x, u, **options)
        assert got[0, 0] == got[0, 3] == -1 and got[0, 1] % 2 == 1 and got[0, 2] in (17, 4000) and got[0, 5] == 9


def test_uniforms_at_and_past_their_ends():
    rng = np.random.default_rng(8)
    u = np.array([[0.0, -0.0, -3.0, np.nan, 1.0, np.inf, 1.0 - 2.0 ** -24, 1e-30]], np.float32)
    for V in (9, 30000):
        x = np.repeat(_rows(rng, 1, 1, V, "bulk"), 8, 1)
        for options in (dict(), dict(top_k=3), dict(top_p=0.9), dict(temperature=3.0, top_p=0.999)):
            got = _check(x, u, **options)
            assert got[0, 0] == got[0, 1] == got[0, 2] == got[0, 3] and got[0, 4] == got[0, 5] == got[0, 6]


def test_likely_tokens_side_by_side():
    """Thousands of the largest in one segment: its list does not hold them."""
    rng = np.random.default_rng(9)
    x = _rows(rng, 1, 4, 60000, "bulk")
    x[0, :, 12000:13500] += 15.0
    x[0, 1] = np.sort(x[0, 1])
    x[0, 2] = -np.sort(-x[0, 2])
    for options in (dict(top_k=900), dict(top_k=1400, top_p=0.9), dict(top_p=0.95), dict(min_p=0.001), dict(top_k=10)):
        _check(x, rng.random((1, 4)), **options)


def test_frequencies_follow_the_weights():
    """20 000 draws from one row by evenly spaced uniforms: each token as often as its share, to within one draw."""
    import paper_2604_12989_amd as dd
    V, n = 300, 20000
    x = np.random.default_rng(2).standard_normal(V).astype(np.float32) * 2
    rows = 1000
    u = ((np.arange(n) + 0.5) / n).astype(np.float32).reshape(n // rows, 1, rows)
    ws = dd.Workspace(1, 1, V, rows - 1, 1, 1, 64, 0)
    dev = gu.to_dev(np.broadcast_to(x, (1, rows, V)))
    got = np.concatenate([dd.sample(dev, gu.to_dev(a), ws, temperature=0.9, top_p=0.95).cpu().numpy().reshape(-1) for a in u])
    w = sample_ref.weights(x, np.float32(0.9), top_p=np.float32(0.95))
    share = w / w.sum() * n
    assert (np.abs(np.bincount(got, minlength=V) - share) <= 1.01).all()


@pytest.mark.parametrize("batch,T,V,B", [(1, 2, 50, 1), (3, 65, 5003, 8), (2, 257, 32003, 16), (1, 1025, 700, 32)])
def test_walk_with_filtered_tokens(batch, T, V, B):
    import paper_2604_12989_amd as dd
    rng = np.random.default_rng(T)
    x = _rows(rng, batch, T, V, "peaked")
    u = rng.random((batch, T)).astype(np.float32)
    options = dict(temperature=rng.choice([0.0, 0.6, 1.1], batch), top_k=rng.choice([0, 20], batch), top_p=rng.choice([0.8, 1.0], batch),
                   min_p=rng.choice([0.0, 0.05], batch))
    n = rng.integers(max(1, T - 4), T, batch).astype(np.int32)
    post = sample_ref.tokens(x, u, **{"tau" if k == "temperature" else k: v.astype(np.float32) if k != "top_k" else v for k, v in options.items()})
    tokens, parent, depth = (np.full((batch, T), -1, np.int32) for _ in range(3))
    for s in range(batch):
        depth[s, 0] = tokens[s, 0] = 0
        deep = 0                                # a chain that the walk follows, other nodes around it
        for i in range(1, n[s] + 1):
            on_path = rng.random() < 0.5 and depth[s, deep] < min(B, 6) and not (parent[s] == deep).any()
            parent[s, i] = deep if on_path else rng.integers(0, i)
            while depth[s, parent[s, i]] >= B:
                parent[s, i] = rng.integers(0, i)
            depth[s, i] = depth[s, parent[s, i]] + 1
            tokens[s, i] = post[s, parent[s, i]] if on_path else V + i     # (ids that no row selects)
            deep = i if on_path else deep
    ws = dd.Workspace(batch, B, V, T - 1, 1, 1, 64, 0)
    x[np.arange(T)[None] > n[:, None]] = np.nan
    got = dd.accept_filtered(gu.to_dev(x), *(gu.to_dev(a) for a in (tokens, parent, depth, n)), B, gu.to_dev(u), ws, **options)
    torch.cuda.synchronize()
    for s in range(batch):
        real = np.arange(T) <= n[s]
        assert np.array_equal(got["posterior"][s].cpu().numpy(), np.where(real, post[s], -1))
        planted = np.full((T, V), -1.0, np.float32)     # the oracle's greedy walk over rows whose largest is the drawn token
        planted[np.arange(T), post[s]] = 1.0
        ref = oracle.accept(planted, tokens[s], parent[s], int(n[s]), B)
        assert int(got["n_accepted"][s]) == ref["n_accepted"] and int(got["bonus_token"][s]) == ref["bonus"]
        assert np.array_equal(got["path"][s].cpu().numpy(), ref["path"])


def test_a_row_without_a_token_ends_the_walk():
    import paper_2604_12989_amd as dd
    x = np.full((1, 3, 40), -np.inf, np.float32)
    x[0, 0, 7] = 1.0
    tokens, parent, depth = (np.array([v], np.int32) for v in ([0, 7, -1], [-1, 0, 1], [0, 1, 2]))
    ws = dd.Workspace(1, 4, 40, 2, 1, 1, 64, 0)
    got = dd.accept_filtered(gu.to_dev(x), *(gu.to_dev(a) for a in (tokens, parent, depth, np.array([1], np.int32))), 4,
                             gu.to_dev(np.full((1, 3), 0.5, np.float32)), ws, top_p=0.9)
    assert got["path"].tolist() == [[0, 1, -1, -1, -1]] and got["bonus_token"].tolist() == [-1] and got["posterior"].tolist() == [[7, -1, -1]]


def test_repeated_calls_give_the_same_tokens():
    rng = np.random.default_rng(5)
    x = np.concatenate([_rows(rng, 1, 8, 40000, k) for k in ("peaked", "flat", "wide")])
    u = rng.random((3, 8))
    first = _sample(x, u, top_p=0.95, temperature=0.8)
    for _ in range(10):
        assert np.array_equal(_sample(x, u, top_p=0.95, temperature=0.8), first)
