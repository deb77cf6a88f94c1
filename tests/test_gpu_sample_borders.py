"""Rows that are read again, with uniforms next to a border: the sums that decide hold to what the definition says, and a row's
token does not depend on which rows share the call."""
import numpy as np
import pytest
import torch

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


@pytest.mark.parametrize("options,kept", [(dict(min_p=1e-8), 100000), (dict(top_k=90000), 89999)])
def test_a_likely_token_and_equal_others(options, kept):
    """Token 0 has weight 1, `kept` others exp(-d) each.  The uniforms lie 4e-4 to 2e-3 of one such weight (3e-10 of the sum and
    more) from a border of tokens 1 to 20000, on both sides."""
    V = 100001
    d = np.float32(14.0703125)
    w = np.exp(-np.float64(d))
    S = 1.0 + kept * w
    # every float above token 0's share: which token, how far above the border in front of it
    near = np.arange(int(np.ceil(2.0 ** 24 / S)), int(2.0 ** 24 * (1.0 + 20000 * w) / S)) * 2.0 ** -24
    place = (near * S - 1.0) / w
    off = place - np.rint(place)
    far = np.abs(off)
    near, place = near[(far > 4e-4) & (far < 2e-3)], place[(far > 4e-4) & (far < 2e-3)]
    pick = np.random.default_rng(1).choice(near.size, 64, replace=False)
    u, want = near[pick], 1 + np.floor(place[pick]).astype(np.int32)
    x = np.full((1, 64, V), -d, np.float32)
    x[:, :, 0] = 0.0
    got = _sample(x, u[None], **options)
    assert np.array_equal(got[0], want), (np.flatnonzero(got[0] != want).size, got[0][:8], want[:8])


@pytest.mark.parametrize("options", [dict(min_p=0.001), dict(top_k=1500), dict(top_k=700), dict(top_k=1500, min_p=0.001),
                                     dict(top_k=700, top_p=0.9999999)])
@pytest.mark.parametrize("half", [1501, 2750])
def test_rows_in_two_equal_halves(half, options):
    """u = 1/2 of a row whose second half repeats the first: the running sum in front of the second half is exactly half of
    all, so that the token is the first of the second half that stays.  600 times the same row, more than have room together;
    twice."""
    for seed in range(6):
        x = (0.5 * np.random.default_rng(seed).standard_normal(half)).astype(np.float32)
        order = np.lexsort((np.arange(2 * half), -np.concatenate([x, x])))
        stays = order[:options.get("top_k", 2 * half)]
        want = stays[stays >= half].min()
        rows = np.broadcast_to(np.concatenate([x, x]), (2, 300, 2 * half))
        u = np.full((2, 300), 0.5)
        first = _sample(rows, u, **options)
        assert (first == want).all(), (seed, want, np.unique(first, return_counts=True))
        assert np.array_equal(_sample(rows, u, **options), first)


@pytest.mark.parametrize("V,T,scale,higher,options", [
    (2000, 64, 2.0, 0, dict(top_k=300)), (12000, 24, 2.0, 0, dict(top_k=500)), (151936, 4, 2.0, 0, dict(top_k=700)),
    (151936, 24, 2.0, 6144, dict(top_k=50)), (151936, 24, 2.0, 6144, dict(top_k=50, top_p=0.95)),
    (151936, 6, 2.0, 0, dict(temperature=2.0, min_p=0.02)), (151936, 4, 0.5, 0, dict(top_k=20000, min_p=0.3))])
def test_rows_that_one_workgroup_reads_alone(V, T, scale, higher, options):
    """A top-k that the lists do not hold in a call without the launches for steps, likely ids side by side, a border in a step with
    thousands of elements."""
    rng = np.random.default_rng(V + T)
    x = (scale * rng.standard_normal((1, T, V))).astype(np.float32)
    x[:, :, :higher] += 2.0
    u = rng.random((1, T)).astype(np.float32)
    want = sample_ref.tokens(x, u, **{"tau": 1.0, **{"tau" if k == "temperature" else k: v for k, v in options.items()}})
    assert np.array_equal(_sample(x, u, **options), want)
