"""Attention over a 4-bit cache against the oracle's attention in 64 bits over the values that the codes stand for.

The bound of an element of the result, A being the softmax-weighted sum of |v| (the oracle's attention with |v|):
  bf16, D = 128   weights rounded to bf16 (2^-8 relative at most, the same rounded weights in the sum they are divided by):
                  2^-8 (A + |o|); partial results in fp16 relative to their row's largest magnitude: 2^-11 max_d A;
                  the result's rounding 2^-8 |o|
  bf16, others    the result's rounding alone
  all             scores, exponentials and sums in fp32: 1e-4 A (scores of magnitude s are off by some (D + s) 2^-24 |q||k|
                  scale, with |q||k| scale < 60 here under 7e-4 / 7; sums of n terms by n 2^-24)"""
import numpy as np
import pytest
import torch

import oracle
from tests import gpu_util as gu
from tests import q4_ref

pytestmark = pytest.mark.gpu
TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _tree(rng, T, n):
    par = np.full(T, -1, np.int32)
    for i in range(1, n + 1):
        par[i] = i - 1 if rng.random() < 0.5 else rng.integers(0, i)
    return oracle.ancestor_mask(par, n, T=T)


def _rounded(x, dtype):
    return torch.from_numpy(np.asarray(x, np.float32)).to(TORCH[dtype])


class Case:
    """Caches, tree rows, queries and masks of a batch; sequence s has lens[s] cache rows."""

    def __init__(self, seed, T, lens, Hq, Hkv, D, dtype="bf16", nodes=None, gap=5, q_scale=1.0):
        import paper_2604_12989_amd as dd
        rng = np.random.default_rng(seed)
        self.T, self.lens, self.Hq, self.Hkv, self.D, self.dtype = T, np.array(lens, np.int32), Hq, Hkv, D, dtype
        batch = len(lens)
        order = rng.permutation(batch)          # spans in any order, with room between them
        self.start = np.zeros(batch, np.int32)
        at = 2
        for s in order:
            self.start[s] = at
            at += lens[s] + gap
        rows = at + 3
        spread = np.exp2(rng.integers(-2, 2, (rows, Hkv, 1)))
        kv = [q4_ref.encode(rng.standard_normal((rows, Hkv, D)) * spread) for _ in range(2)]
        self.k, self.v = (q4_ref.decode(*c) for c in kv)
        # what no sequence owns reads as NaN
        owned = np.zeros(rows, bool)
        for s in range(batch):
            owned[self.start[s]:self.start[s] + lens[s]] = True
        for codes, scales in kv:
            scales[~owned] = 255
        self.cache = dd.CacheQ4(*(torch.from_numpy(np.ascontiguousarray(a.transpose(1, 0, 2))).cuda() for c in kv for a in c))
        self.q = _rounded(rng.standard_normal((batch * T, Hq, D)) * q_scale, dtype)
        self.kt, self.vt = (_rounded(rng.standard_normal((batch * T, Hkv, D)), dtype) for _ in range(2))
        self.mask = np.stack([_tree(rng, T, T - 1 if nodes is None else nodes) for _ in range(batch)])

    def run(self, ws=None, out=None, scratch=None):
        import paper_2604_12989_amd as dd
        batch = len(self.lens)
        if ws is None:
            ws = dd.Workspace(batch, 1, 8, max(1, self.T - 1), self.Hq, self.Hkv, self.D, int(self.lens.sum()))
        if scratch is not None:
            ws.nbytes = scratch
        return dd.verify_attn_q4(self.q.cuda(), self.cache, self.kt.cuda(), self.vt.cuda(),
                                 torch.from_numpy(self.mask.view(np.int64)).cuda(), self.start, self.lens, batch, self.T, self.Hq,
                                 self.Hkv, self.D, self.D ** -0.5, dd.DTYPE_BF16 if self.dtype == "bf16" else dd.DTYPE_FP32, ws, out=out)

    def check(self, got, n_pairs=40, seed=0):
        rng = np.random.default_rng(seed)
        got = got.double().cpu().numpy()
        T, Hq = self.T, self.Hq
        for s in range(len(self.lens)):
            pairs = np.stack([rng.integers(0, T, n_pairs), rng.integers(0, Hq, n_pairs)], 1).astype(np.int32)
            pairs[:4] = [[0, 0], [T - 1, Hq - 1], [0, Hq - 1], [T - 1, 0]]
            own, tree = slice(self.start[s], self.start[s] + self.lens[s]), slice(s * T, (s + 1) * T)
            q, kt, vt = (t[tree].float().numpy() for t in (self.q, self.kt, self.vt))
            k, v = (x[own].astype(np.float32) for x in (self.k, self.v))
            ref = oracle.verify_attn(q, k, v, kt, vt, self.mask[s], pairs=pairs)
            A = oracle.verify_attn(q, k, np.abs(v), kt, np.abs(vt), self.mask[s], pairs=pairs)
            tol = 1e-4 * A + (2.0 ** -8 * np.abs(ref) if self.dtype == "bf16" else 0.0)
            if self.dtype == "bf16" and self.D == 128:
                tol = tol + 2.0 ** -8 * (A + np.abs(ref)) + 2.0 ** -11 * A.max(-1, keepdims=True)
            off = np.abs(got[tree][pairs[:, 0], pairs[:, 1]] - ref)
            assert (off <= tol).all(), (s, float((off - tol).max()), float((off / np.maximum(tol, 1e-30)).max()))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,lens,Hq,Hkv", [
    (1, [0], 1, 1), (1, [1], 2, 2), (1, [31, 4097, 0], 8, 2), (2, [32], 3, 1), (8, [33], 4, 1), (17, [255], 5, 1), (33, [257], 1, 1),
    (65, [63, 1000], 8, 4), (5, [4000], 32, 8), (31, [64], 8, 8), (66, [1], 6, 2), (16, [511, 512, 513, 3], 16, 2)])
def test_few_rows(T, lens, Hq, Hkv, D):
    c = Case(T * 10 + D, T, lens, Hq, Hkv, D)
    c.check(c.run())


@pytest.mark.parametrize("T,lens,Hq,Hkv", [
    (257, [2000], 8, 2), (257, [0], 32, 8), (300, [63], 32, 8), (129, [64, 65, 127, 1], 32, 8), (513, [700], 16, 2), (257, [4100], 32, 8),
    (1025, [130], 16, 4), (101, [37, 3001, 900], 24, 8), (64, [20000], 64, 8), (200, [128, 192], 32, 4), (400, [1023, 449], 32, 8)])
def test_many_rows(T, lens, Hq, Hkv):
    c = Case(T + len(lens), T, lens, Hq, Hkv, 128)
    c.check(c.run())


@pytest.mark.parametrize("T,lens", [(70, [30, 500]), (300, [100, 900]), (9, [33])])
@pytest.mark.parametrize("D", [64, 128])
def test_padding_rows_give_zeros(T, lens, D):
    nodes = T // 2
    c = Case(T, T, lens, 16, 4, D, nodes=nodes)
    got = c.run(out=torch.full((len(lens) * T, 16, D), 7.0, dtype=torch.bfloat16, device="cuda"))
    assert (got.view(len(lens), T, 16, D)[:, nodes + 1:] == 0).all()
    c.check(got)


@pytest.mark.parametrize("D,T,lens,Hq,Hkv,dtype", [
    (32, 5, [40], 4, 2, "bf16"), (96, 17, [300, 0], 6, 3, "bf16"), (160, 3, [33], 2, 1, "bf16"), (256, 9, [257], 4, 1, "bf16"),
    (32, 9, [1], 1, 1, "fp32"), (64, 17, [128], 2, 1, "fp32"), (128, 33, [500, 77], 8, 2, "fp32"), (224, 1, [64], 2, 2, "fp32"),
    (128, 1, [0], 1, 1, "fp32"), (64, 130, [255], 4, 4, "fp32")])
def test_other_heads_and_fp32(D, T, lens, Hq, Hkv, dtype):
    c = Case(D + T, T, lens, Hq, Hkv, D, dtype)
    c.check(c.run())


@pytest.mark.parametrize("T,lens,D", [(33, [600], 128), (33, [600], 64), (257, [1500], 128)])
def test_scores_far_apart(T, lens, D):
    """Queries forty times as long: a row's reference is outgrown again and again, most weights vanish.  (The bound's 1e-4 is
    for scores under 60; here they reach 40 times that, with exponents off by up to 40 * 1e-4.)"""
    c = Case(T, T, lens, 8, 2, D, q_scale=40.0)
    got = c.run().double().cpu().numpy()
    ref = oracle.verify_attn(c.q.float().numpy(), c.k[c.start[0]:c.start[0] + c.lens[0]].astype(np.float32),
                             c.v[c.start[0]:c.start[0] + c.lens[0]].astype(np.float32), c.kt.float().numpy(), c.vt.float().numpy(), c.mask[0])
    top = np.abs(np.concatenate([c.v[c.start[0]:c.start[0] + c.lens[0]].reshape(-1), c.vt.double().numpy().reshape(-1)])).max()
    assert np.isfinite(got).all()
    assert np.abs(got - ref).max() <= (2.0 ** -7 + 2.0 ** -8 + 2.0 ** -11 + 4e-3) * top


def test_rows_of_the_largest_cache_offsets():
    """A span behind 2^31 bytes of codes."""
    import paper_2604_12989_amd as dd
    rows, Hkv, D, T, L = 4_500_000, 8, 128, 4, 700
    c = Case(3, T, [L], 32, Hkv, D, gap=0)
    big = dd.CacheQ4.empty(rows, Hkv, D)
    for n in ("k_codes", "k_scales", "v_codes", "v_scales"):
        getattr(big, n)[:, rows - L:] = getattr(c.cache, n)[:, c.start[0]:c.start[0] + L]
    small = c.run()
    c.cache, at = big, c.start[0]
    c.start = np.array([rows - L], np.int32)
    got = c.run()
    assert torch.equal(got, small)
    c.start = np.array([at], np.int32)
    c.check(got)


@pytest.mark.parametrize("T,lens,Hq,Hkv,D", [(257, [4100], 32, 8, 128), (17, [9000], 32, 8, 128), (33, [4000], 8, 4, 64)])
def test_a_workspace_of_the_advertised_size_is_enough(T, lens, Hq, Hkv, D):
    import paper_2604_12989_amd as dd
    c = Case(T, T, lens, Hq, Hkv, D)
    need = dd.verify_attn_q4_workspace_bytes(1, T, Hq, Hkv, D, dd.DTYPE_BF16, lens[0])
    full = c.run()
    assert torch.equal(c.run(scratch=need), full)
    c.check(full)


def test_it_agrees_with_the_attention_over_the_values_read_back():
    import paper_2604_12989_amd as dd
    for T, lens, Hq, Hkv, D in ((257, [2100], 32, 8, 128), (17, [700, 33], 32, 8, 128), (65, [500], 8, 2, 64)):
        c = Case(T, T, lens, Hq, Hkv, D, gap=0)
        for n in ("k_scales", "v_scales"):
            t = getattr(c.cache, n)
            t.masked_fill_(t == 255, 100)
        k, v = dd.q4_load(c.cache, [0], [0, c.cache.rows])
        ws = dd.Workspace(len(lens), 1, 8, T - 1, Hq, Hkv, D, int(c.lens.sum()))
        ref = dd.verify_attn_spans(c.q.cuda(), k, v, c.kt.cuda(), c.vt.cuda(), torch.from_numpy(c.mask.view(np.int64)).cuda(),
                                   c.start, c.lens, len(lens), T, Hq, Hkv, D, D ** -0.5, dd.DTYPE_BF16, ws)
        got = c.run()
        c.check(got)
        c.check(ref)
        print("bits equal:", torch.equal(got, ref))
