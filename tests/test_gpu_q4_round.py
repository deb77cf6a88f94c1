"""Decoding rounds over a 4-bit cache with each request's own sampling options: prompts stored, then round after round
top-K, tree, attention of two layers, filtered walk and append, against the same round put together from the references; and the
round recorded into a HIP graph and replayed over changing inputs."""
import numpy as np
import pytest
import torch

import oracle
from tests import gpu_util as gu
from tests import q4_ref, sample_ref

pytestmark = pytest.mark.gpu

BATCH, B, V, N, HQ, HKV, D, LAYERS = 2, 8, 4096, 40, 8, 2, 128, 2
T = N + 1
ROOM = 160
OPTIONS = dict(temperature=[0.9, 0.7], top_k=[0, 30], top_p=[0.9, 0.95], min_p=[0.0, 0.02])


def _bf16(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)


def _round_inputs(seed):
    """Draft and target logits, queries and tree rows of a round; the target mostly agrees with the draft's top tokens."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((BATCH, B, V)).astype(np.float32)
    x[np.arange(BATCH)[:, None], np.arange(B)[None], rng.integers(0, V, (BATCH, B))] += 9.0
    target = rng.standard_normal((BATCH, T, V)).astype(np.float32)
    trees = []
    for s in range(BATCH):
        tok, lp = oracle.topk(x[s], N)
        trees.append(oracle.build_tree(tok, lp, N, 5 + s))
        for i in range(T):
            if trees[s]["depth"][i] < B and rng.random() < 0.9:
                target[s, i, tok[trees[s]["depth"][i], 0]] += 12.0
    layers = [[_bf16(rng, BATCH * T, h, D) for h in (HQ, HKV, HKV)] for _ in range(LAYERS)]
    return x, target, rng.random((BATCH, T)).astype(np.float32), layers, trees


def test_rounds_against_the_references():
    import paper_2604_12989_amd as dd
    rng = np.random.default_rng(1)
    lens = np.array([37, 66], np.int32)
    start = (np.arange(BATCH) * ROOM).astype(np.int32)
    caches = [dd.CacheQ4.empty(ROOM * BATCH, HKV, D) for _ in range(LAYERS)]
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    kept = []                                 # per layer and sequence: the keys and values that the cache stands for
    for cache in caches:
        k, v = _bf16(rng, int(off[-1]), HKV, D), _bf16(rng, int(off[-1]), HKV, D)
        dd.q4_store(k.cuda(), v.cuda(), off, start, cache)
        held = [q4_ref.decode(*q4_ref.encode(t.double().numpy())) for t in (k, v)]
        kept.append([[h[off[s]:off[s + 1]] for h in held] for s in range(BATCH)])
    ws = dd.Workspace(BATCH, B, V, N, HQ, HKV, D, ROOM * BATCH)
    accepted = 0
    for step in range(4):
        x, target, u, layers, trees = _round_inputs(50 + step)
        tok, lp = dd.topk(gu.to_dev(x), N, ws)
        tree = dd.build(tok, lp, N, torch.tensor([5, 6], dtype=torch.int32, device="cuda"), ws)
        mask = [oracle.ancestor_mask(t["parent"], t["n_nodes"], T=T) for t in trees]
        for layer, (q, kt, vt) in enumerate(layers):
            out = dd.verify_attn_q4(q.cuda(), caches[layer], kt.cuda(), vt.cuda(), tree["ancestor_mask"], start, lens, BATCH, T, HQ, HKV, D,
                                    D ** -0.5, dd.DTYPE_BF16, ws).double().cpu().numpy()
            for s in range(BATCH):
                rows = slice(s * T, (s + 1) * T)
                k, v = (a.astype(np.float32) for a in kept[layer][s])
                args = [t[rows].float().numpy() for t in (q, kt, vt)]
                ref = oracle.verify_attn(args[0], k, v, args[1], args[2], mask[s])
                A = oracle.verify_attn(args[0], k, np.abs(v), args[1], np.abs(args[2]), mask[s])
                # (the bound of tests/test_gpu_attn_q4.py)
                tol = 1e-4 * A + 2.0 ** -8 * (A + 2 * np.abs(ref)) + 2.0 ** -11 * A.max(-1, keepdims=True)
                assert (np.abs(out[rows] - ref) <= tol).all(), (step, layer, s)
        walk = dd.accept_filtered(gu.to_dev(target), tree["tokens"], tree["parent"], tree["depth"], tree["n_nodes"], B, gu.to_dev(u), ws,
                                  **OPTIONS)
        for layer, (q, kt, vt) in enumerate(layers):
            dd.q4_append(kt.cuda(), vt.cuda(), walk["path"], walk["n_accepted"], start + lens, BATCH, T, B, caches[layer])
        post = sample_ref.tokens(target, u, *(np.array(OPTIONS[k]) for k in ("temperature", "top_k", "top_p", "min_p")))
        for s in range(BATCH):
            assert np.array_equal(tree["tokens"][s].cpu().numpy(), trees[s]["tokens"])
            planted = np.full((T, V), -1.0, np.float32)
            planted[np.arange(T), post[s]] = 1.0
            ref = oracle.accept(planted, trees[s]["tokens"], trees[s]["parent"], trees[s]["n_nodes"], B)
            n = int(walk["n_accepted"][s])
            assert np.array_equal(walk["path"][s].cpu().numpy(), ref["path"]) and int(walk["bonus_token"][s]) == ref["bonus"]
            for layer in range(LAYERS):
                new = [q4_ref.decode(*q4_ref.encode(t[s * T + ref["path"][:n + 1]].double().numpy())) for t in layers[layer][1:]]
                kept[layer][s] = [np.concatenate([a, b]) for a, b in zip(kept[layer][s], new)]
            lens[s] += n + 1
            accepted += n
    assert accepted >= 4
    for layer in range(LAYERS):
        k, v = dd.q4_load(caches[layer], start, np.concatenate([[0], np.cumsum(lens)]))
        for got, i in ((k, 0), (v, 1)):
            assert np.array_equal(got.double().cpu().numpy(), np.concatenate([kept[layer][s][i] for s in range(BATCH)]))


def test_a_round_replays_from_a_captured_graph():
    import paper_2604_12989_amd as dd
    sets = [_round_inputs(80 + i) for i in range(3)]
    lens, start = np.array([100, 33], np.int32), (np.arange(BATCH) * ROOM).astype(np.int32)
    rng = np.random.default_rng(3)
    fresh = dd.CacheQ4.empty(ROOM * BATCH, HKV, D)
    prompt = _bf16(rng, ROOM * BATCH, HKV, D).cuda()
    dd.q4_store(prompt, prompt, [0, ROOM * BATCH], [0], fresh)
    cache = dd.CacheQ4.empty(ROOM * BATCH, HKV, D)
    ws = dd.Workspace(BATCH, B, V, N, HQ, HKV, D, ROOM * BATCH)
    root = torch.tensor([5, 6], dtype=torch.int32, device="cuda")
    x, target, u, layers, _ = sets[0]
    cur = dict(x=gu.to_dev(x), target=gu.to_dev(target), u=gu.to_dev(u), q=layers[0][0].cuda(), kt=layers[0][1].cuda(), vt=layers[0][2].cuda())
    names = ("k_codes", "k_scales", "v_codes", "v_scales")
    # flat rows too: half of the last set's target rows need to be read again
    sets[2][1][:, ::2] = np.random.default_rng(4).standard_normal((BATCH, (T + 1) // 2, V)).astype(np.float32) * 0.3
    tok, lp = dd.topk(cur["x"], N, ws)
    tree = dd.build(tok, lp, N, root, ws)
    out = torch.empty_like(cur["q"])
    walk = dd.accept_filtered(cur["target"], tree["tokens"], tree["parent"], tree["depth"], tree["n_nodes"], B, cur["u"], ws, **OPTIONS)
    nxt = torch.empty((BATCH,), dtype=torch.int32, device="cuda")
    back = tuple(torch.empty((BATCH * (B + 1), HKV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def load(i):
        x, target, u, layers, _ = sets[i]
        for k, v in dict(x=torch.from_numpy(x), target=torch.from_numpy(target), u=torch.from_numpy(u), q=layers[0][0], kt=layers[0][1],
                         vt=layers[0][2]).items():
            cur[k].copy_(v)
        for n in names:
            getattr(cache, n).copy_(getattr(fresh, n))

    def step():
        dd.topk(cur["x"], N, ws, tok, lp)
        dd.build(tok, lp, N, root, out=tree)
        dd.verify_attn_q4(cur["q"], cache, cur["kt"], cur["vt"], tree["ancestor_mask"], start, lens, BATCH, T, HQ, HKV, D, D ** -0.5,
                          dd.DTYPE_BF16, ws, out=out)
        dd.accept_filtered(cur["target"], tree["tokens"], tree["parent"], tree["depth"], tree["n_nodes"], B, cur["u"], ws, out=walk, **OPTIONS)
        dd.q4_append(cur["kt"], cur["vt"], walk["path"], walk["n_accepted"], start + lens, BATCH, T, B, cache)
        dd.q4_load(cache, start + lens, [0, B + 1, 2 * (B + 1)], out=back)
        dd.sample(first, cur["u0"], ws, out=nxt, **OPTIONS)

    first = torch.empty((BATCH, V), device="cuda")
    cur["u0"] = torch.empty((BATCH,), device="cuda")

    def load_all(i):
        load(i)
        first.copy_(cur["target"][:, 0])
        cur["u0"].copy_(cur["u"][:, 0])

    def snapshot():
        torch.cuda.synchronize()
        got = dict(out=out, nxt=nxt, k=back[0], v=back[1], **{n: getattr(cache, n) for n in names}, **walk)
        return {k: v.clone() for k, v in got.items()}

    eager = []
    for i in range(3):
        load_all(i)
        step()
        eager.append(snapshot())
        assert torch.equal(eager[i]["nxt"], eager[i]["posterior"][:, 0])
    assert not torch.equal(eager[0]["posterior"], eager[1]["posterior"])
    load_all(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n_replay, i in enumerate((1, 2, 0, 2, 1)):
        load_all(i)                           # eager work between the replays
        torch.cuda.synchronize()
        graph.replay()
        for k, v in snapshot().items():
            same = v.view(torch.int16) if v.dtype == torch.bfloat16 else v
            want = eager[i][k].view(torch.int16) if v.dtype == torch.bfloat16 else eager[i][k]
            assert torch.equal(same, want), (n_replay, i, k)


def test_two_streams_with_workspaces_of_their_own():
    """The same call on two streams at once: nothing is shared but the inputs."""
    import paper_2604_12989_amd as dd
    x, target, u, layers, trees = _round_inputs(7)
    dev, ud = gu.to_dev(target), gu.to_dev(u)
    f = [gu.to_dev(np.stack([t[k] for t in trees])) for k in ("tokens", "parent", "depth")]
    n = gu.to_dev(np.array([t["n_nodes"] for t in trees], np.int32))
    ws = [dd.Workspace(BATCH, B, V, N, HQ, HKV, D, 0) for _ in range(2)]
    want = dd.accept_filtered(dev, *f, n, B, ud, ws[0], **OPTIONS)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(5):
        for s, w in zip(streams, ws):
            with torch.cuda.stream(s):
                got.append(dd.accept_filtered(dev, *f, n, B, ud, w, **OPTIONS))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(g[k], want[k]) for k in want)
