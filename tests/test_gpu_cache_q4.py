"""The 4-bit cache on the GPU: written from prompts and from accepted paths, and read back, byte for byte what the
definition gives (tests/q4_ref.py)."""
import numpy as np
import pytest
import torch

from tests import q4_ref

pytestmark = pytest.mark.gpu
TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _values(rng, shape, dtype):
    """Values of all kinds that a block can hold: ordinary, ties of the grid, outliers, zeros, far exponents."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-8, 8, shape[:-1] + (1,)))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.9, 3.49, 0.0, -0.0])
    flat = x.reshape(-1, 32)
    some = rng.permutation(len(flat))[: max(1, len(flat) // 4)]
    flat[some] = ties[rng.integers(0, len(ties), (len(some), 32))] * np.exp2(rng.integers(-20, 20, (len(some), 1)))
    flat[rng.permutation(len(flat))[: len(flat) // 20]] = 0.0
    far = rng.permutation(len(flat))[: len(flat) // 10]
    flat[far] *= np.exp2(rng.choice([-132, -126, -120, 113], (len(far), 1)).astype(np.float64))
    return torch.from_numpy(flat.reshape(shape)).to(TORCH[dtype])


def _cache(rows, Hkv, D, seed=5):
    import paper_2604_12989_amd as dd
    cache = dd.CacheQ4.empty(rows, Hkv, D)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        t.copy_(torch.randint(0, 253, t.shape, generator=gen, device="cuda", dtype=torch.uint8))
    return cache


def _host(cache):
    return [t.cpu().numpy().copy() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]


def _put(want, k, v, src, row):
    """Row `src` of k and v is written to cache row `row`."""
    for at, t in ((0, k), (2, v)):
        codes, scales = q4_ref.encode(t[src].double().numpy())
        want[at][:, row], want[at + 1][:, row] = codes, scales


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hkv,D", [(1, 32), (3, 64), (2, 96), (8, 128), (1, 160), (2, 256)])
@pytest.mark.parametrize("lengths", [(1,), (37,), (5, 0, 130), (0, 63, 1, 64)])
def test_store_writes_what_the_definition_gives(dtype, Hkv, D, lengths):
    import paper_2604_12989_amd as dd
    rng = np.random.default_rng(D * 100 + Hkv + len(lengths))
    first = 3                              # rows of k in front of the first sequence's
    off = np.concatenate([[first], first + np.cumsum(lengths)]).astype(np.int32)
    rows = sum(lengths) + 7 * len(lengths) + 5
    dst = (rows - np.cumsum([n + 7 for n in lengths])).astype(np.int32)   # in descending order, with gaps
    k, v = (_values(rng, (int(off[-1]), Hkv, D), dtype) for _ in range(2))
    cache = _cache(rows, Hkv, D)
    want = _host(cache)
    for s, n in enumerate(lengths):
        for j in range(n):
            _put(want, k, v, off[s] + j, dst[s] + j)
    dd.q4_store(k.cuda(), v.cuda(), off, dst, cache)
    torch.cuda.synchronize()
    for got, ref in zip(_host(cache), want):
        assert np.array_equal(got, ref)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hkv,D", [(1, 32), (8, 128), (2, 224)])
def test_load_reads_what_the_bytes_stand_for(dtype, Hkv, D):
    import paper_2604_12989_amd as dd
    rows, src, off = 400, [300, 7, 9, 0], np.array([2, 90, 90, 91, 222], np.int32)
    cache = _cache(rows, Hkv, D)           # every byte that a scale can be but 255 occurs
    cache.v_scales[0, 300, 0] = 255
    guard = torch.full((off[-1] + 3, Hkv, D), 7.0, dtype=TORCH[dtype], device="cuda")
    k, v = dd.q4_load(cache, src, off, out=(guard.clone(), guard.clone()))
    torch.cuda.synchronize()
    host = _host(cache)
    for got, codes, scales in ((k, *host[:2]), (v, *host[2:])):
        want = np.full(got.shape, 7.0)
        for s in range(4):
            n = off[s + 1] - off[s]
            want[off[s]:off[s + 1]] = q4_ref.decode(codes, scales)[:, src[s]:src[s] + n].transpose(1, 0, 2)
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    assert np.isnan(v[2, 0, :32].float().cpu().numpy()).all()
    again = dd.q4_load(cache, src, off, TORCH[dtype])
    assert torch.equal(again[0][2:].nan_to_num(), k[2:off[-1]].nan_to_num())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_element_is_off_by_more_than_half_a_step(dtype):
    """The grid's steps, in units of the block's power of two: 0.5 below 2, 1 below 4, 2 above."""
    import paper_2604_12989_amd as dd
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((500, 2, 128)) * np.exp2(rng.integers(-30, 30, (500, 2, 1)))).to(TORCH[dtype])
    cache = dd.CacheQ4.empty(500, 2, 128)
    dd.q4_store(x.cuda(), x.cuda(), [0, 500], [0], cache)
    back = dd.q4_load(cache, [0], [0, 500], TORCH[dtype])[1].double().cpu().numpy()
    unit = np.repeat(np.ldexp(1.0, cache.v_scales.cpu().numpy().astype(int) - 127).transpose(1, 0, 2), 32, -1)
    x = x.double().numpy()
    step = np.where(np.abs(x) < 2 * unit, 0.5, np.where(np.abs(x) < 4 * unit, 1.0, 2.0)) * unit
    assert (np.abs(back - x) <= step / 2).all()
    assert (np.abs(x) < 7 * unit).all()


def test_blocks_with_infinities_read_back_as_nan_and_others_are_untouched():
    import paper_2604_12989_amd as dd
    for bad in (np.inf, -np.inf, np.nan):
        x = torch.ones((3, 1, 96))
        x[1, 0, 40] = bad
        cache = dd.CacheQ4.empty(3, 1, 96)
        dd.q4_store(x.cuda(), x.bfloat16().float().cuda(), [0, 3], [0], cache)
        k, v = dd.q4_load(cache, [0], [0, 3], torch.float32)
        for got in (k, v):
            nan = np.isnan(got.cpu().numpy())
            assert nan[1, 0, 32:64].all() and nan.sum() == 32
            assert (got.cpu().numpy()[~nan] == 1.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hkv,D,T,B", [(1, 32, 2, 1), (8, 128, 65, 16), (3, 96, 17, 32), (2, 64, 1, 4)])
def test_append_takes_the_accepted_rows_and_no_others(dtype, Hkv, D, T, B):
    import paper_2604_12989_amd as dd
    rng = np.random.default_rng(T * 7 + B)
    batch, rows = 4, 4 * (B + 6)
    k, v = (_values(rng, (batch * T, Hkv, D), dtype) for _ in range(2))
    took = np.array([0, min(B, T - 1), min(1, T - 1), min(B, T - 1) // 2], np.int32)
    path = np.full((batch, B + 1), -1, np.int32)
    for s in range(batch):
        path[s, 0] = 0
        path[s, 1:took[s] + 1] = 1 + np.sort(rng.permutation(max(T - 1, 0))[:took[s]])
    if took[3] >= 1:
        path[3, 1] = T                     # no such row: passed over
    path[1, took[1] + 1:] = 0              # behind the path: not looked at
    dst = np.array([s * (B + 6) + s for s in range(batch)], np.int32)
    cache = _cache(rows, Hkv, D)
    want = _host(cache)
    for s in range(batch):
        for j in range(took[s] + 1):
            if 0 <= path[s, j] < T:
                _put(want, k, v, s * T + path[s, j], dst[s] + j)
    dd.q4_append(k.cuda(), v.cuda(), torch.tensor(path, device="cuda"), torch.tensor(took, device="cuda"), dst, batch, T, B, cache)
    torch.cuda.synchronize()
    for got, ref in zip(_host(cache), want):
        assert np.array_equal(got, ref)


def test_counts_outside_the_path_stay_inside_it():
    """n_accepted from elsewhere: more than B counts as B, a negative one as nothing."""
    import paper_2604_12989_amd as dd
    rng = np.random.default_rng(1)
    T, B = 9, 4
    k = _values(rng, (2 * T, 1, 32), "bf16")
    path = torch.arange(B + 1, dtype=torch.int32, device="cuda").repeat(2, 1)
    cache = _cache(20, 1, 32)
    want = _host(cache)
    for j in range(B + 1):
        _put(want, k, k, j, 2 + j)
    dd.q4_append(k.cuda(), k.cuda(), path, torch.tensor([1000, -3], dtype=torch.int32, device="cuda"), [2, 12], 2, T, B, cache)
    torch.cuda.synchronize()
    for got, ref in zip(_host(cache), want):
        assert np.array_equal(got, ref)


def test_rows_far_into_a_long_cache():
    """Offsets past 2^31 bytes: the last rows of a cache of 2.3 GB of codes."""
    import paper_2604_12989_amd as dd
    Hkv, D, rows = 8, 128, 4_500_000
    rng = np.random.default_rng(9)
    x = _values(rng, (70, Hkv, D), "bf16").cuda()
    cache = dd.CacheQ4.empty(rows, Hkv, D)
    dd.q4_store(x, x, [0, 70], [rows - 70], cache)
    k, v = dd.q4_load(cache, [rows - 70], [0, 70])
    codes, scales = q4_ref.encode(x.double().cpu().numpy())
    want = q4_ref.decode(codes, scales)
    for got in (k, v):                     # (some magnitudes are past the type's range: their blocks are NaN)
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    assert np.array_equal(cache.v_codes[:, rows - 70:].cpu().numpy(), codes.transpose(1, 0, 2))
