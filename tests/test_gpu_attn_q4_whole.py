"""Attention over a 4-bit cache, every row, head and element of a call against the definition in 64 bits (on the device; the bounds
are those of test_gpu_attn_q4), and against the attention over the values read back."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_attn_q4 import Case

pytestmark = pytest.mark.gpu

SHAPES = [  # T, lens, Hq, Hkv, D, dtype
    (257, [2100], 32, 8, 128, "bf16"), (257, [4100], 32, 8, 128, "bf16"), (129, [64, 65, 127, 1], 32, 8, 128, "bf16"),
    (101, [37, 3001, 900], 24, 8, 128, "bf16"), (300, [63], 32, 8, 128, "bf16"), (1025, [130], 16, 4, 128, "bf16"),
    (17, [700, 33], 32, 8, 128, "bf16"), (1, [900, 1, 0, 513], 32, 8, 128, "bf16"), (33, [257], 1, 1, 128, "bf16"),
    (65, [500], 8, 2, 64, "bf16"), (257, [1500], 16, 4, 64, "bf16"), (1, [900, 1, 0, 513], 32, 8, 64, "bf16"),
    (9, [200, 31], 6, 3, 96, "bf16"), (17, [128], 2, 1, 64, "fp32")]


def _definition(c, k, v, mask):
    """(softmax-weighted sums of v, and of |v|) in 64 bits, [batch*T, Hq, D]; k, v [rows, Hkv, D] as the codes stand for."""
    T, Hq, Hkv, D = c.T, c.Hq, c.Hkv, c.D
    q, kt, vt = (t.cuda().double() for t in (c.q, c.kt, c.vt))
    o, A = torch.zeros_like(q), torch.zeros_like(q)
    for s in range(len(c.lens)):
        own, tree = slice(int(c.start[s]), int(c.start[s] + c.lens[s])), slice(s * T, (s + 1) * T)
        sees = np.unpackbits(mask[s].view(np.uint8), axis=1, bitorder="little")[:, :T].astype(bool)
        real = torch.tensor(sees.diagonal().copy(), device="cuda")[:, None]
        sees = torch.tensor(np.concatenate([np.ones((T, int(c.lens[s])), bool), sees], 1), device="cuda")
        for h in range(Hq):
            g = h // (Hq // Hkv)
            K, V = torch.cat([k[own, g], kt[tree, g]]), torch.cat([v[own, g], vt[tree, g]])
            z = torch.where(sees, (q[tree, h].contiguous() @ K.T.contiguous()) * D ** -0.5, -math.inf)
            p = torch.where(real, torch.softmax(torch.where(real, z, 0.0), 1), 0.0)
            o[tree, h], A[tree, h] = p @ V, p @ V.abs()
    return o, A


def _bound(c, ref, A):
    tol = 1e-4 * A
    if c.dtype == "bf16":
        tol = tol + 2.0 ** -8 * ref.abs()
        if c.D == 128:
            tol = tol + 2.0 ** -8 * (A + ref.abs()) + 2.0 ** -11 * A.max(-1, keepdim=True).values
    return tol


@pytest.mark.parametrize("q_scale", [1.0, 6.0])
@pytest.mark.parametrize("T,lens,Hq,Hkv,D,dtype", SHAPES)
def test_every_element(T, lens, Hq, Hkv, D, dtype, q_scale):
    c = Case(3 * T + D, T, lens, Hq, Hkv, D, dtype, nodes=max(0, T - 1 - T // 9), q_scale=q_scale)
    got = c.run(out=torch.full((len(lens) * T, Hq, D), 7.0, dtype=c.q.dtype, device="cuda")).double()
    k, v = (torch.from_numpy(np.nan_to_num(x)).cuda() for x in (c.k, c.v))
    ref, A = _definition(c, k, v, c.mask)
    over = (got - ref).abs() - _bound(c, ref, A)
    assert bool((over <= 0).all()), (float(over.max()), (over > 0).nonzero()[:4].tolist())


@pytest.mark.parametrize("T,lens,Hq,Hkv,D,dtype", SHAPES)
def test_against_the_values_read_back(T, lens, Hq, Hkv, D, dtype):
    """Bit for bit: for these shapes both calls are cut into the same workgroups and key ranges."""
    import paper_2604_12989_amd as dd
    c = Case(T + D, T, lens, Hq, Hkv, D, dtype, gap=0)
    for n in ("k_scales", "v_scales"):
        t = getattr(c.cache, n)
        t.masked_fill_(t == 255, 100)
    k, v = dd.q4_load(c.cache, [0], [0, c.cache.rows], dtype=c.q.dtype)
    ws = dd.Workspace(len(lens), 1, 8, max(1, T - 1), Hq, Hkv, D, int(c.lens.sum()))
    ref = dd.verify_attn_spans(c.q.cuda(), k, v, c.kt.cuda(), c.vt.cuda(), torch.from_numpy(c.mask.view(np.int64)).cuda(), c.start,
                               c.lens, len(lens), T, Hq, Hkv, D, D ** -0.5, dd.DTYPE_BF16 if dtype == "bf16" else dd.DTYPE_FP32, ws)
    assert torch.equal(c.run(), ref)
