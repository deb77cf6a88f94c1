"""The operators of a decoding round that keeps its cache in 4 bits and samples with each request's own options:
their plain forms, and the calls that a user makes of the library's.

Kinds of case (field "op"):

  store      prompts' K and V rows of `rows` to `rows_hi` tokens a sequence go into the cache and are read back
  append     the accepted path of a round goes behind each sequence, and the rows there are read back
  attn       one layer of tree attention over the cache (T = 1: a single token)
  sample     one token from each row of logits
  accept     the verifier's walk with sampled tokens

A cache holds blocks of 32 values along the head dim: 4-bit codes for 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, two
a byte, and a byte with the block's power of two (2^(byte - 127); 255: not a number).  Arrays are head-major: codes
[Hkv, rows, D / 2], scales [Hkv, rows, D / 32].
"""
import math

import numpy as np
import torch

own = False  # False: plain forms; True: the library's kernels

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_FAR = 40.0 * math.log(2.0)  # a token this far below the best, in units of the temperature, has weight zero


def _case(name, op, **kw):
    return dict(name=name, op=op, **kw)


def _attn(name, batch, T, Hq, Hkv, D, L_lo, L_hi, dtype="bf16"):
    return _case(name, "attn", batch=batch, T=T, Hq=Hq, Hkv=Hkv, D=D, L_lo=L_lo, L_hi=L_hi, dtype=dtype)


def _sampling(name, op, batch, T, V, temperature, top_k, top_p, min_p, open_rows):
    return _case(name, op, batch=batch, T=T, V=V, temperature=temperature, top_k=top_k, top_p=top_p,
                 min_p=min_p, open_rows=open_rows)


def listed():
    return [
        # The end of a round for four chat requests: a few rows each, all latency.
        _case("append_batch4", "append", batch=4, T=65, B=16, Hkv=8, D=128, dtype="bf16"),
        # Prompts of a batch enter the cache.
        _case("store_prompts_batch4", "store", batch=4, rows_lo=2000, rows_hi=16384, Hkv=8, D=128, dtype="bf16"),
        # A small fp32 model with heads of 64, odd length.
        _case("store_prompt_fp32", "store", batch=1, rows_lo=2047, rows_hi=2047, Hkv=4, D=64, dtype="fp32"),
        # The fp32 model of a few million weights: kernels at their latency.
        _attn("tiny_fp32", 1, 17, 2, 1, 64, 128, 128, "fp32"),
        # Plain decoding of a batch, one token a sequence.
        _attn("token_batch8_8k", 8, 1, 32, 8, 128, 1000, 8192),
        # The smallest budget on a long document: the cache is all there is to read.
        _attn("n16_l32k", 1, 17, 32, 8, 128, 32768, 32768),
        # The headline shape of bench.py.
        _attn("n256_l8k", 1, 257, 32, 8, 128, 8192, 8192),
        # Its batch of ragged sequences.
        _attn("batch16_ragged", 16, 129, 64, 8, 128, 1024, 8192),
        # Heads of 64, odd length.
        _attn("head64_n64_l2k", 1, 65, 16, 4, 64, 2047, 2047),
        # The next token of 16 requests with the usual options.
        _sampling("sample_batch16", "sample", 16, 1, 151936, 0.7, 0, 0.9, 0.0, 0.1),
        # The walk at the headline shape, top-k and top-p.
        _sampling("walk_n256", "accept", 1, 257, 151936, 1.0, 50, 0.95, 0.0, 0.0),
        # A few requests, a vocabulary that no vector width divides, nothing but min-p and top-p, some open rows.
        _sampling("walk_batch4_odd", "accept", 4, 101, 50021, 1.2, 0, 0.98, 0.02, 0.2),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _cost(c):
    w = work(c)
    return w["bytes"] / 1e12 + w["flops"] / ((2e14 if c.get("dtype") != "fp32" else 2e12) if c["op"] == "attn" else 1e13)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choices(["append", "store", "attn", "sample", "accept"], [1, 2, 5, 2, 3])[0]
        batch = rng.choice([1, 1, 2, 3, 5, 16])
        fp32 = rng.random() < 0.2
        head = dict(Hkv=rng.choice([1, 2, 4, 8, 8]), D=rng.choice([64, 128, 128]), dtype="fp32" if fp32 else "bf16")
        if op == "append":
            B = rng.randint(4, 24)
            c = _case("", op, batch=batch, T=_log_int(rng, 8, 1025), B=B, **head)
        elif op == "store":
            a, b = _log_int(rng, 1, 16384), _log_int(rng, 1, 16384)
            c = _case("", op, batch=batch, rows_lo=min(a, b), rows_hi=max(a, b), **head)
        elif op == "attn":
            Hkv = head["Hkv"]
            a, b = _log_int(rng, 16, 512 if fp32 else 32768), _log_int(rng, 16, 512 if fp32 else 32768)
            T = 1 if rng.random() < 0.25 else _log_int(rng, 2, 64 if fp32 else 1025)
            c = _attn("", batch, T, Hkv * rng.choice([1, 2, 3, 4, 4, 5, 8]), Hkv, head["D"], min(a, b), max(a, b), head["dtype"])
        else:
            T = _log_int(rng, 2, 513) if op == "accept" else rng.choice([1, 1, 2, 7])
            c = _sampling("", op, batch, T, rng.choice([151936, _log_int(rng, 500, 160000)]),
                          rng.choice([0.0, round(rng.uniform(0.3, 1.5), 2), round(rng.uniform(0.3, 1.5), 2)]),
                          rng.choice([0, 0, _log_int(rng, 1, 1000)]), rng.choice([1.0, round(rng.uniform(0.5, 0.99), 2)]),
                          rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.3), 3)]), rng.choice([0.0, 0.0, 0.1, 1.0]))
        del c["name"]
        if _cost(c) <= most and (op not in ("sample", "accept") or c["batch"] * c["T"] * c["V"] <= 80_000_000):
            return c


# ---- inputs ----

class State:
    pass


def _tdt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _lengths(seed, n, lo, hi):
    return np.random.RandomState(seed % (1 << 31)).randint(lo, hi + 1, n).astype(np.int32)


def _tree(seed, T, B, fewest):
    """A random tree of T rows, the last few of them padding: parent, depth, nodes and mask words."""
    r = np.random.RandomState((seed + 77) % (1 << 31))
    n = int(r.randint(min(fewest, T), T + 1))  # rows in use
    parent, depth = np.full(T, -1, np.int32), np.full(T, -1, np.int32)
    bits = [0] * T
    for i in range(n):
        if i:
            while True:
                p = int(r.randint(0, i)) if r.rand() < 0.6 else max(0, i - 1 - int(r.randint(0, 3)))
                if depth[p] < B:
                    break
            parent[i], depth[i], bits[i] = p, depth[p] + 1, bits[p] | 1 << i
        else:
            depth[0], bits[0] = 0, 1
    words = [[(b >> (64 * w)) & 0xFFFFFFFFFFFFFFFF for w in range((T + 63) // 64)] for b in bits]
    return parent, depth, n, np.array(words, np.uint64).view(np.int64)


def _kv(c, gen, *shape):
    """Keys or values: unit scale, a few head dims that are larger throughout, as projections give them."""
    x = torch.randn(shape, generator=gen, device="cuda")
    big = torch.rand((1,) * (len(shape) - 2) + shape[-2:], generator=gen, device="cuda") < 0.03
    return torch.where(big, 4.0 * x, x).to(_tdt(c))


def _cache(c, gen, rows):
    """Codes and scales as a cache of such values holds them."""
    codes, scales = _encode(_kv(c, gen, rows, c["Hkv"], c["D"]).float())
    return codes.transpose(0, 1).contiguous(), scales.transpose(0, 1).contiguous()


def _logits(c, gen):
    """Rows of a target: a bulk of N(0, 2^2); but for the open ones, 60 tokens above it that fall off
    by rank, the first of them holding a probability between 0.2 and 0.98 of what it shares with the bulk."""
    batch, T, V = c["batch"], c["T"], c["V"]
    x = 2.0 * torch.randn((batch, T, V), generator=gen, device="cuda")
    head = min(60, V)
    at = torch.rand((batch, T, V), generator=gen, device="cuda").topk(head, 2).indices
    top = x.logsumexp(2, keepdim=True) + torch.logit(torch.rand((batch, T, 1), generator=gen, device="cuda") * 0.78 + 0.2)
    fall = torch.rand((batch, T, head), generator=gen, device="cuda").cumsum(2) * 0.6
    fall[:, :, 0] = 0.0
    closed = torch.rand((batch, T, 1), generator=gen, device="cuda") >= c["open_rows"]
    at_x = x.gather(2, at)
    return x.scatter(2, at, torch.where(closed, torch.maximum(at_x, top - fall), at_x)), at


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = State()
    s.c, s.kept = c, None
    batch = c["batch"]
    if c["op"] in ("store", "append"):
        if c["op"] == "store":  # (the same prompts' lengths in another order: as many rows come back for every seed)
            n = np.linspace(c["rows_lo"], c["rows_hi"], batch + 1)[1:].astype(np.int32)
            n = np.random.RandomState(seed % (1 << 31)).permutation(n)
        else:
            n = _lengths(seed, batch, 40, 400)
        room = int(n.max()) + 40
        s.dst_row = (np.arange(batch) * room + _lengths(seed + 1, batch, 0, 9)).astype(np.int32)
        s.rows = room * batch + 16
        s.k_codes, s.k_scales = _cache(c, gen, s.rows)
        s.v_codes, s.v_scales = _cache(c, gen, s.rows)
        if c["op"] == "store":
            s.offset = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
            s.k, s.v = (_kv(c, gen, int(s.offset[-1]), c["Hkv"], c["D"]) for _ in range(2))
        else:
            s.dst_row += n  # behind each sequence
            s.dst_row = np.minimum(s.dst_row, np.arange(1, batch + 1) * room - c["B"] - 1).astype(np.int32)
            s.offset = ((c["B"] + 1) * np.arange(batch + 1)).astype(np.int32)
            s.k, s.v = (_kv(c, gen, batch * c["T"], c["Hkv"], c["D"]) for _ in range(2))
            most = min(c["B"], c["T"] - 1)
            took = np.random.RandomState(seed % (1 << 31)).randint(0, most + 1, batch)
            path = np.full((batch, c["B"] + 1), -1, np.int32)
            for b in range(batch):
                inner = np.random.RandomState((seed + b) % (1 << 31)).permutation(c["T"] - 1)[:took[b]]
                path[b, :took[b] + 1] = np.concatenate([[0], 1 + np.sort(inner)])
            s.path, s.n_accepted = torch.tensor(path, device="cuda"), torch.tensor(took, dtype=torch.int32, device="cuda")
        # rows of the cache that are read back, in order
        s.at = torch.tensor(np.concatenate([np.arange(d, d + m) for d, m in zip(s.dst_row, np.diff(s.offset))]), device="cuda")
    elif c["op"] == "attn":
        s.kv_len = _lengths(seed, batch, c["L_lo"], c["L_hi"])
        room = c["L_hi"] + 25
        s.kv_start = (np.arange(batch) * room).astype(np.int32)
        s.rows = room * batch
        s.k_codes, s.k_scales = _cache(c, gen, s.rows)
        s.v_codes, s.v_scales = _cache(c, gen, s.rows)
        s.q = torch.randn((batch * c["T"], c["Hq"], c["D"]), generator=gen, device="cuda").to(_tdt(c))
        s.k_tree, s.v_tree = (_kv(c, gen, batch * c["T"], c["Hkv"], c["D"]) for _ in range(2))
        s.mask = torch.tensor(np.stack([_tree(seed + b, c["T"], 32, max(1, c["T"] - 3))[3] for b in range(batch)]), device="cuda")
        s.start_dev, s.len_dev = (torch.tensor(a, dtype=torch.int64, device="cuda") for a in (s.kv_start, s.kv_len))
    else:
        s.logits, likely = _logits(c, gen)
        s.uniforms = torch.rand((batch, c["T"]), generator=gen, device="cuda")
        # options of the requests: those of the case, every third one greedy with the others' options off
        greedy = np.arange(batch) % 3 == 2
        s.temperature = np.where(greedy, 0.0, c["temperature"]).astype(np.float32)
        s.top_k = np.where(greedy, 0, c["top_k"]).astype(np.int32)
        s.top_p = np.where(greedy, 1.0, c["top_p"]).astype(np.float32)
        s.min_p = np.where(greedy, 0.0, c["min_p"]).astype(np.float32)
        s.options = [torch.tensor(a, device="cuda") for a in (s.temperature, s.top_k, s.top_p, s.min_p)]
        if c["op"] == "accept":
            s.B = 16
            trees = [_tree(seed + b, c["T"], s.B, max(2, c["T"] - 5)) for b in range(batch)]
            parent = np.stack([t[0] for t in trees])
            # a node's children carry its most likely tokens
            rank, seen = np.zeros_like(parent), {}
            for b in range(batch):
                for i in range(1, trees[b][2]):
                    k = (b, int(parent[b, i]))
                    rank[b, i] = seen.get(k, 0)
                    seen[k] = rank[b, i] + 1
            s.parent, s.depth = torch.tensor(parent, device="cuda"), torch.tensor(np.stack([t[1] for t in trees]), device="cuda")
            s.n_nodes = torch.tensor([t[2] - 1 for t in trees], dtype=torch.int32, device="cuda")
            by_value = likely.gather(2, s.logits.gather(2, likely).argsort(2, descending=True))
            rows = by_value.gather(1, s.parent.clamp(min=0).long()[:, :, None].expand(-1, -1, likely.shape[2]))
            rank = torch.tensor(rank, dtype=torch.int64, device="cuda")
            token = rows.gather(2, rank.clamp(max=likely.shape[2] - 1)[:, :, None])[:, :, 0]
            # (a node with more children than likely tokens: the others carry a token that no row selects)
            s.tokens = torch.where((s.parent >= 0) & (rank < likely.shape[2]), token, -1).to(torch.int32)
            s.tokens[:, 0] = 1
    return s


# ---- the 4-bit format, plainly ----

def _decode(codes, scales):
    """[..., D / 2] codes and [..., D / 32] scales to fp32 values [..., D]."""
    grid = torch.tensor(_GRID + tuple(-g for g in _GRID), device=codes.device)
    x = torch.stack([grid[(codes & 15).long()], grid[(codes >> 4).long()]], -1).flatten(-2)
    unit = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)
    unit = torch.where(scales == 255, math.nan, unit)
    return (x.unflatten(-1, (-1, 32)) * unit[..., None]).flatten(-2)


def _rounded(x):
    """fp32 values [..., D] as (multiples of their block's power of two [..., D / 32, 32], its exponent)."""
    b = x.unflatten(-1, (-1, 32))
    mant, ex = torch.frexp(b.abs().amax(-1, keepdim=True))
    # the exponent of the largest magnitude, rounded to two significant bits, less that of the grid's top
    ex = (ex - 1 + (mant >= 0.875).int() - 2).clamp(min=-124)
    ex = torch.where(mant == 0, -124, ex)
    y = torch.ldexp(torch.ldexp(b, -(ex // 2)), -(ex - ex // 2))
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return torch.round(y / step) * step, ex


def _encode(x):
    y, ex = _rounded(x)
    grid = torch.tensor(_GRID, device=x.device)
    code = torch.searchsorted(grid, y.abs().contiguous()) + torch.where(torch.signbit(y), 8, 0)
    code = code.flatten(-2).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), (ex[..., 0] + 127).to(torch.uint8)


def _as_held(x):
    y, ex = _rounded(x.float())
    return torch.ldexp(y, ex.expand_as(y)).flatten(-2).to(x.dtype)


# ---- plain forms ----

def _plain_store(s):
    return _as_held(s.k), _as_held(s.v)


def _plain_append(s):
    c = s.c
    old = [_decode(codes[:, s.at], scales[:, s.at]).transpose(0, 1).to(_tdt(c))
           for codes, scales in ((s.k_codes, s.k_scales), (s.v_codes, s.v_scales))]
    j = torch.arange(c["B"] + 1, device="cuda")
    takes = (j[None] <= s.n_accepted[:, None]).flatten()[:, None, None]
    src = (s.path.clamp(min=0).long() + c["T"] * torch.arange(c["batch"], device="cuda")[:, None]).flatten()
    return tuple(torch.where(takes, _as_held(new[src]), was) for new, was in zip((s.k, s.v), old))


def _plain_attn(s):
    c = s.c
    batch, T, Hq, Hkv, D = (c[k] for k in ("batch", "T", "Hq", "Hkv", "D"))
    G, L = Hq // Hkv, int(s.kv_len.max())
    j = torch.arange(L, device="cuda")
    on = j[None] < s.len_dev[:, None]
    at = torch.where(on, s.start_dev[:, None] + j[None], s.start_dev[:, None])

    def keys(codes, scales, tree):  # [batch, Hkv, L + T, D]
        cached = _decode(codes[:, at], scales[:, at]).transpose(0, 1)
        return torch.cat([cached, tree.view(batch, T, Hkv, D).transpose(1, 2).float()], 2)

    q = s.q.view(batch, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(batch, Hkv, T * G, D).float()
    t = torch.arange(T, device="cuda")
    tree_on = ((s.mask[:, :, t // 64] >> (t % 64)) & 1).bool()
    seen = torch.cat([on[:, None].expand(-1, T, -1), tree_on], 2)
    real = tree_on[:, t, t]
    score = torch.matmul(q, keys(s.k_codes, s.k_scales, s.k_tree).transpose(2, 3)) / math.sqrt(D)
    score = score.view(batch, Hkv, T, G, L + T).masked_fill(~seen[:, None, :, None], -math.inf)
    score = score.masked_fill(~real[:, None, :, None, None], 0.0)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    p = (p / p.sum(-1, keepdim=True)).view(batch, Hkv, T * G, L + T)
    o = torch.matmul(p, keys(s.v_codes, s.v_scales, s.v_tree)).view(batch, Hkv, T, G, D)
    o = torch.where(real[:, None, :, None, None], o, 0.0)
    return o.permute(0, 2, 1, 3, 4).reshape(batch * T, Hq, D).to(s.q.dtype)


def _plain_sample(s):
    """Tokens [batch, T], all in 64 bits: a token's place against a border has to be exact."""
    V = s.c["V"]
    tau, k, top_p, min_p = (o[:, None, None] for o in s.options)
    x, order = s.logits.sort(dim=2, descending=True, stable=True)
    d = (x[..., :1].double() - x.double()) / tau.double().clamp(min=1e-300)
    w = torch.where(d <= _FAR, torch.exp(-d), 0.0)
    rank = torch.arange(V, device="cuda")
    w = torch.where((tau == 0) & (rank > 0) | (k > 0) & (rank >= k), 0.0, w)
    before = w.cumsum(2) - w
    stays = (before < top_p.double() * w.sum(2, keepdim=True)) & (w >= min_p.double())
    w = torch.zeros_like(w).scatter_(2, order, torch.where(stays, w, 0.0))  # by id
    total = w.cumsum(2)
    return (total <= s.uniforms.double()[..., None] * total[..., -1:]).sum(2).to(torch.int32)


def _plain_accept(s):
    T, batch = s.c["T"], s.c["batch"]
    i = torch.arange(T, device="cuda")
    post = torch.where(i[None] <= s.n_nodes[:, None], _plain_sample(s), -1)
    path = torch.full((batch, s.B + 1), -1, dtype=torch.int32, device="cuda")
    path[:, 0] = 0
    cur, going, n = torch.zeros((batch, 1), dtype=torch.int64, device="cuda"), True, 0
    for depth in range(1, s.B + 1):
        fits = (s.parent == cur) & (s.tokens == post.gather(1, cur)) & (i[None] <= s.n_nodes[:, None])
        going = fits.any(1) & going
        cur = torch.where(going[:, None], fits.int().argmax(1, keepdim=True), cur)
        path[:, depth] = torch.where(going, cur[:, 0], -1)
        n = n + going.int()
    return dict(path=path, n_accepted=n.to(torch.int32), bonus_token=post.gather(1, cur)[:, 0], posterior=post)


# ---- the library's calls ----

def _own(s):
    import paper_2604_12989_amd as dd
    c = s.c
    if s.kept is None:  # what a program keeps from call to call: its cache and its workspace
        if c["op"] in ("sample", "accept"):
            s.kept = dd.Workspace(c["batch"], 16, c["V"], max(1, c["T"] - 1), 1, 1, 64, 0)
        else:
            cache = dd.CacheQ4(s.k_codes, s.k_scales, s.v_codes, s.v_scales)
            ws = dd.Workspace(c["batch"], 1, 8, max(1, c["T"] - 1), c["Hq"], c["Hkv"], c["D"], int(s.kv_len.sum())) if c["op"] == "attn" else None
            s.kept = cache, ws
    if c["op"] == "sample":
        return dd.sample(s.logits, s.uniforms, s.kept, s.temperature, s.top_k, s.top_p, s.min_p)
    if c["op"] == "accept":
        return dd.accept_filtered(s.logits, s.tokens, s.parent, s.depth, s.n_nodes, s.B, s.uniforms, s.kept,
                                  s.temperature, s.top_k, s.top_p, s.min_p)
    cache, ws = s.kept
    if c["op"] == "attn":
        dtype = dd.DTYPE_BF16 if c["dtype"] == "bf16" else dd.DTYPE_FP32
        return dd.verify_attn_q4(s.q, cache, s.k_tree, s.v_tree, s.mask, s.kv_start, s.kv_len, c["batch"], c["T"], c["Hq"],
                                 c["Hkv"], c["D"], 1.0 / math.sqrt(c["D"]), dtype, ws)
    if c["op"] == "store":
        dd.q4_store(s.k, s.v, s.offset, s.dst_row, cache)
    else:
        dd.q4_append(s.k, s.v, s.path, s.n_accepted, s.dst_row, c["batch"], c["T"], c["B"], cache)
    return dd.q4_load(cache, s.dst_row, s.offset, s.k.dtype)


_PLAIN = {"store": _plain_store, "append": _plain_append, "attn": _plain_attn, "sample": _plain_sample, "accept": _plain_accept}


def run(s):
    return _own(s) if own else _PLAIN[s.c["op"]](s)


# ---- the same from the definitions, in 64 bits ----

def _exact_values(codes, scales):
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    e, m = (code & 7) >> 1, (code & 1).double()
    mag = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.pow(2.0, (e - 1).double()))
    return torch.where(code >= 8, -mag, mag) * torch.pow(2.0, scales.double() - 127).repeat_interleave(32, -1)


def _exact_held(x):
    """Nearest of the 15 values of each element's block: every candidate tried, of two equally near the one whose code is even."""
    b = x.double().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    e = torch.where(top >= 1.75 * torch.pow(2.0, e), e + 1, e) - 2
    unit = torch.pow(2.0, torch.where(top > 0, e.clamp(min=-124), -124.0))
    best, off = torch.zeros_like(b), torch.full_like(b, math.inf)
    for k in (0, 2, 4, 6, 1, 3, 5, 7):
        d = (b.abs() - _GRID[k] * unit).abs()
        best, off = torch.where(d < off, _GRID[k] * unit, best), torch.minimum(d, off)
    return torch.copysign(best, b).reshape(x.shape)


def exact(case, seed):
    c = case
    if c["op"] in ("sample", "accept"):
        return None  # whole numbers
    s = prepare(case, seed)
    if c["op"] == "store":
        return _exact_held(s.k), _exact_held(s.v)
    held_in = {n: (getattr(s, n + "_codes"), getattr(s, n + "_scales")) for n in "kv"}
    if c["op"] == "append":
        out = []
        for new, n in ((s.k, "k"), (s.v, "v")):
            held, (codes, scales) = _exact_held(new), held_in[n]
            rows = _exact_values(codes[:, s.at], scales[:, s.at]).transpose(0, 1).contiguous()
            for b in range(c["batch"]):
                for j in range(int(s.n_accepted[b]) + 1):
                    rows[b * (c["B"] + 1) + j] = held[b * c["T"] + int(s.path[b, j])]
            out.append(rows)
        return tuple(out)
    if work(c)["flops"] > 3e12:
        return None
    batch, T, Hq, Hkv, D = (c[k] for k in ("batch", "T", "Hq", "Hkv", "D"))
    o = torch.zeros((batch * T, Hq, D), dtype=torch.float64, device="cuda")
    words = s.mask.cpu().numpy().view(np.uint64)
    for b in range(batch):
        lo, hi = int(s.kv_start[b]), int(s.kv_start[b] + s.kv_len[b])
        sees = np.unpackbits(words[b].view(np.uint8), axis=1, bitorder="little")[:, :T].astype(bool)
        real = torch.tensor(sees.diagonal().copy(), device="cuda")
        sees = torch.tensor(np.concatenate([np.ones((T, hi - lo), bool), sees], 1), device="cuda")
        for h in range(Hkv):
            K, V = (torch.cat([_exact_values(held_in[n][0][h, lo:hi], held_in[n][1][h, lo:hi]), tree[b * T:(b + 1) * T, h].double()])
                    for n, tree in (("k", s.k_tree), ("v", s.v_tree)))
            for g in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                z = (s.q[b * T:(b + 1) * T, g].double() @ K.T) * (1.0 / math.sqrt(D))
                z = torch.where(sees, z, -math.inf)
                p = torch.where(real[:, None], torch.softmax(torch.where(real[:, None], z, 0.0), 1), 0.0)
                o[b * T:(b + 1) * T, g] = p @ V
    return o


def work(case):
    """Bytes that go in and out once, and the products' operations.  Sampling: an exponential's dozen operations an element."""
    c = case
    batch = c["batch"]
    if c["op"] in ("sample", "accept"):
        rows = batch * c["T"]
        return {"bytes": rows * (4 * c["V"] + 24), "flops": 12 * rows * c["V"]}
    e = 2 if c["dtype"] == "bf16" else 4
    row, packed = 2 * c["Hkv"] * c["D"] * e, 2 * c["Hkv"] * (c["D"] // 2 + c["D"] // 32)
    if c["op"] in ("store", "append"):
        rows = batch * ((c["rows_lo"] + c["rows_hi"]) / 2 if c["op"] == "store" else (min(c["B"], c["T"] - 1) / 2 + 1))
        return {"bytes": rows * (2 * row + 2 * packed), "flops": rows * 2 * c["Hkv"] * c["D"] * 6}
    L = (c["L_lo"] + c["L_hi"]) / 2
    return {"bytes": batch * (L * packed + c["T"] * (row + 2 * c["Hq"] * c["D"] * e + 8 * ((c["T"] + 63) // 64))),
            "flops": batch * 4 * c["D"] * c["Hq"] * c["T"] * (L + 3)}
