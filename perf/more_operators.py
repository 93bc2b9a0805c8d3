"""Operators of a serving program whose tree cache is held in microscaled 4-bit floating point (kv_dtype "mxfp4").

  write   one step of a search: children forked below a node, per call tokens of every child rotated by their positions and
          appended, quantised on the way (append_rotated), then the children's tokens read back as values (read_back) and the
          children pruned.  Outputs: the rotated queries, the rotated keys where the program wants them, the values of the cache.
  read    tokens of many nodes read back from the cache as values (read_back).
  attend  decode attention of many branches over the paths of their trees (decode_attention); branches share the prefix above
          them.  Outputs: the heads' outputs and the log-sum-exp of every row.

The format: 32 consecutive dims of a token's head share a power of two 2^E, E = floor(log2 of the largest magnitude) - 2, and hold e2m1
values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), to nearest, ties to the even code, at most 6; E is -126 .. 125 for keys, -23 .. 13 for values.

Keys and values are N(0, 1), queries of `attend` N(0, 4): scores have a spread of about 2, so that a softmax has a few
dominant tokens and a long tail, as in trained models.
"""

import math

import numpy as np
import torch

own = False

_DEV = "cuda"
_TINY, _HUGE = {"k": -126, "v": -23}, {"k": 125, "v": 13}  # exponents of blocks
_MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


# ---- cases -------------------------------------------------------------------------------------
def _write(nodes, count, *, iters=1, ragged=False, prompt=0, heads=(32, 8, 128), rotary=0, base=10000.0, interleaved=False,
           positions="path", fused=False, want_k=False, shape_seed=1, name=None):
    """`nodes` children get up to `count` tokens in each of `iters` calls.  rotary 0: the whole head; positions: "path" (the
    tree's own), "depth" (drafts of a token tree, by depth) or "far" (anywhere up to 2^20); fused: q, k and v are slices of one
    projection."""
    c = dict(op="write", nodes=nodes, count=count, iters=iters, ragged=ragged, prompt=prompt, q_heads=heads[0], kv_heads=heads[1],
             head_dim=heads[2], rotary=rotary or heads[2], base=base, interleaved=interleaved, positions=positions, fused=fused,
             want_k=want_k, shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def _read(nodes, count, *, ragged=False, heads=(32, 8, 128), shape_seed=1, name=None):
    c = dict(op="read", nodes=nodes, count=count, ragged=ragged, q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2], shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def _attend(queries, prompt, *, mids=0, step=0, leaves=1, tail=1, q_len=1, drafts=False, ragged=False, heads=(32, 8, 128), shape_seed=1, name=None):
    """`queries` trees: a prompt; `mids` steps below it (0: none); `leaves` branches of up to `tail` tokens below each of those.  Every branch has
    q_len query tokens, its last ones; drafts: they are a token tree, else a chain."""
    c = dict(op="attend", queries=queries, prompt=prompt, mids=mids, step=step, leaves=leaves, tail=tail, q_len=q_len, drafts=drafts,
             ragged=ragged, q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2], shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a step of one user's search, token by token: 16 branches, launches and latency count
        _write(16, 1, iters=16, prompt=1152, name="write_one_query"),
        # the same for a batch of searches: 1024 branches, the ordinary decode load, projections in one tensor
        _write(1024, 1, iters=8, prompt=512, heads=(28, 4, 128), base=1e6, fused=True, shape_seed=2, name="write_branches"),
        # prompts of many lengths behind their prefill projections, keys wanted back for attention over the prompt
        _write(8, 2048, ragged=True, fused=True, want_k=True, shape_seed=3, name="write_prompts"),
        # the steps of a search handed to a reward model's own cache
        _read(256, 128, ragged=True, shape_seed=4, name="read_steps"),
        # one document moved to another process
        _read(1, 48000, name="read_document"),
        # one user's search: 16 branches on one prompt, latency counts
        _attend(1, 512, leaves=16, tail=48, name="attend_one_query"),
        # breadth-first search for a batch of users: 16 branches each below four steps
        _attend(32, 512, mids=4, step=256, leaves=4, tail=128, shape_seed=5, name="attend_bfs"),
        # speculative branches at scale: 32 on one chain of steps
        _attend(64, 2000, mids=1, step=500, leaves=32, tail=256, ragged=True, shape_seed=6, name="attend_speculative"),
        # token trees of six drafts verified on every branch
        _attend(96, 1024, mids=2, step=128, leaves=4, tail=64, q_len=6, drafts=True, ragged=True, heads=(40, 8, 128), shape_seed=7,
                name="attend_drafts"),
        # a document and a few branches on it
        _attend(1, 64000, leaves=8, tail=100, shape_seed=8, name="attend_document"),
        # queries of any length that share nothing, smaller heads
        _attend(48, 16000, ragged=True, heads=(16, 2, 64), shape_seed=9, name="attend_alone_heads64"),
        # steps of 100 tokens scored at once: matrix products
        _attend(16, 1024, leaves=4, tail=100, q_len=100, shape_seed=10, name="attend_steps_scored"),
    ]


_HEADS = [(32, 8, 128), (28, 4, 128), (64, 8, 128), (40, 8, 128), (16, 4, 128), (8, 2, 128), (16, 2, 64), (8, 2, 64), (12, 4, 96), (16, 4, 256), (6, 3, 32)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        seed, ragged, heads, kind = rng.randrange(1 << 30), rng.random() < 0.7, rng.choice(_HEADS), rng.random()
        if kind < 0.3:
            if rng.random() < 0.5:
                nodes, count, iters = _log(rng, 1, 4096), 1, rng.choice([1, rng.randint(2, 16)])
            else:
                nodes, count, iters = _log(rng, 1, 64), _log(rng, 2, 8192), 1
            c = _write(nodes, count, iters=iters, ragged=ragged and count > 1, prompt=_log(rng, 1, 2048), heads=heads,
                       rotary=rng.choice([heads[2], heads[2], heads[2] // 2, heads[2] // 4 * 2 - 2]), base=rng.choice([1e4, 5e5, 1e6]),
                       interleaved=rng.random() < 0.4, positions=rng.choice(["path", "path", "depth", "far"]), fused=rng.random() < 0.5,
                       want_k=rng.random() < 0.5, shape_seed=seed)
        elif kind < 0.45:
            c = _read(_log(rng, 1, 2048), _log(rng, 1, 48000), ragged=ragged, heads=heads, shape_seed=seed)
        else:
            q_len = rng.choice([1, 1, 1, rng.randint(2, 16), rng.randint(17, 128)])
            mids = rng.choice([0, 0, rng.randint(1, 6)])
            c = _attend(_log(rng, 1, 128), _log(rng, 1, 64000), mids=mids, step=_log(rng, 1, 500) if mids else 0, leaves=_log(rng, 1, 40),
                        tail=q_len - 1 + _log(rng, 1, 400), q_len=q_len, drafts=2 <= q_len <= 32 and rng.random() < 0.5, ragged=ragged,
                        heads=heads, shape_seed=seed)
        w = work(c)
        if w["bytes"] < 4.7e8 and w["flops"] < 1.1e11 and (c["op"] != "attend" or _path_numbers(c) < 1.2e7):
            return c


# ---- shapes ------------------------------------------------------------------------------------
def _lengths(r, ragged, n, longest):
    return [int(x) for x in r.integers(max(1, longest // 8), longest + 1, n)] if ragged else [longest] * n


def _counts(case):
    return _lengths(np.random.default_rng(case["shape_seed"]), case["ragged"], case["nodes"], case["count"])


def _positions(case, counts):
    """[iters][tokens of a call] path positions."""
    r = np.random.default_rng(case["shape_seed"] + 1)
    within = np.concatenate([np.arange(c) for c in counts])
    if case["positions"] == "far":
        return r.integers(0, 1 << 20, (case["iters"], len(within))).astype(np.int32)
    if case["positions"] == "depth":  # a binary token tree in level order
        within = np.floor(np.log2(within + 1)).astype(np.int64)
    step = np.asarray(counts)[np.repeat(np.arange(len(counts)), counts)]
    return np.stack([case["prompt"] + within + i * step for i in range(case["iters"])]).astype(np.int32)


def _inv_freq(case):
    r = case["rotary"]
    return case["base"] ** (-np.arange(0, r, 2, dtype=np.float64) / r)


def _trees(case):
    """(parent, first token, tokens) of every node, parents first, and the requested nodes."""
    r = np.random.default_rng(case["shape_seed"])
    parent, size, leaves = [], [], []
    for prompt in _lengths(r, case["ragged"], case["queries"], case["prompt"]):
        root = len(parent)
        parent.append(-1)
        size.append(prompt)
        above = [root]
        if case["mids"]:
            above = list(range(root + 1, root + 1 + case["mids"]))
            parent += [root] * case["mids"]
            size += _lengths(r, case["ragged"], case["mids"], case["step"])
        for u in above:
            leaves += range(len(parent), len(parent) + case["leaves"])
            parent += [u] * case["leaves"]
            size += [max(case["q_len"], n) for n in _lengths(r, case["ragged"], case["leaves"], case["tail"])]
    first = np.concatenate([[0], np.cumsum(size)[:-1]]).astype(np.int64)
    return np.asarray(parent), first, np.asarray(size), np.asarray(leaves, dtype=np.int32)


def _path_lengths(parent, size, leaves):
    total = size.copy()
    for u in range(len(parent)):  # parents come first
        if parent[u] >= 0:
            total[u] += total[parent[u]]
    return total[leaves]


def _path_numbers(case):
    """Branches times the longest path."""
    parent, _, size, leaves = _trees(case)
    return len(leaves) * int(_path_lengths(parent, size, leaves).max())


def _sees(case):
    """[q_len, q_len]: whether a query sees a draft."""
    n = case["q_len"]
    if not case["drafts"]:
        return np.tril(np.ones((n, n), dtype=bool))
    see = np.eye(n, dtype=bool)
    for j in range(1, n):  # a binary tree in level order
        see[j] |= see[(j - 1) // 2]
    return see


def work(case):
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    held = 2 * hkv * d * 17 // 32  # bytes of a token in the cache
    if case["op"] == "attend":
        parent, _, size, leaves = _trees(case)
        rows, before = len(leaves) * case["q_len"] * hq, _path_lengths(parent, size, leaves) - case["q_len"]
        seen = int(before.sum()) * case["q_len"] + len(leaves) * int(_sees(case).sum())
        return {"bytes": int(size.sum()) * held + rows * (2 * d + 4 * d + 4), "flops": 4 * d * hq * seen}
    counts = _counts(case)
    if case["op"] == "read":
        return {"bytes": sum(counts) * (held + 4 * hkv * d), "flops": 2 * sum(counts) * hkv * d}
    t = sum(counts) * case["iters"]
    return {"bytes": t * (2 * d * (2 * hq + 2 * hkv + (hkv if case["want_k"] else 0)) + 2 * held + 4 * hkv * d),
            "flops": 3 * t * (hq + hkv) * case["rotary"]}


# ---- inputs ------------------------------------------------------------------------------------
def _normal(shape, gen, spread=1.0):
    return (torch.randn(shape, generator=gen, device=_DEV) * spread).to(torch.bfloat16)


def _inputs(case, seed):
    gen = torch.Generator(device=_DEV).manual_seed(seed)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "attend":
        parent, first, size, leaves = _trees(case)
        n, per = int(size.sum()), 1 << 17
        k, v = (torch.cat([_normal((min(per, n - a), hkv, d), gen) for a in range(0, n, per)]) for _ in range(2))
        q = _normal((len(leaves) * case["q_len"], hq, d), gen, 2.0)
        return dict(k=k, v=v, q=q, parent=parent, first=first, size=size, leaves=leaves, sm_scale=d ** -0.5)
    counts = _counts(case)
    if case["op"] == "read":
        return dict(k=_normal((sum(counts), hkv, d), gen), v=_normal((sum(counts), hkv, d), gen), counts=counts)
    x = torch.randn((case["iters"], sum(counts), hq + 2 * hkv, d), generator=gen, device=_DEV).to(torch.bfloat16)
    parts = x[..., :hq, :], x[..., hq:hq + hkv, :], x[..., hq + hkv:, :]
    q, k, v = parts if case["fused"] else (p.contiguous() for p in parts)
    pos = _positions(case, counts)
    # where a token of (call, token of the call) lies among the tokens read back, which are in the order of the nodes
    start = np.cumsum([0] + counts[:-1]) * case["iters"]
    node, within = np.repeat(np.arange(len(counts)), counts), np.concatenate([np.arange(c) for c in counts])
    rows = np.stack([start[node] + i * np.asarray(counts)[node] + within for i in range(case["iters"])])
    return dict(q=q, k=k, v=v, counts=counts, host_positions=pos, positions=torch.as_tensor(pos.astype(np.int64), device=_DEV),
                rows=torch.as_tensor(rows, device=_DEV), inv_freq=_inv_freq(case))


def _pages(tokens):
    return -(-int(tokens) // 16)


def _new_tree(case, pages):
    import paper_2605_10195_amd as spex
    return spex.SpexTree(case["q_heads"], case["kv_heads"], case["head_dim"], 16, "bf16", "mxfp4", num_pages=pages, device=_DEV)


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if case["op"] == "write":
        if own:
            tree = _new_tree(case, _pages(case["prompt"]) + sum(_pages(c * case["iters"]) for c in s["counts"]))
            (root,) = tree.fork(-1, 1)
            tree.append_step(root, None, None, n_tokens=case["prompt"])
            tree.set_rotation(case["rotary"], s["inv_freq"], interleaved=case["interleaved"])
            s.update(tree=tree, root=root)
        return s
    # a program that reads or attends has the cache, not what it was made of
    k, v = s.pop("k"), s.pop("v")
    if case["op"] == "read":
        size = np.asarray(s["counts"])
        parent, first = np.full(len(size), -1), np.concatenate([[0], np.cumsum(size)[:-1]])
    else:
        parent, first, size = s["parent"], s["first"], s["size"]
        _paths(s)
    if own:
        s["tree"] = tree = _new_tree(case, sum(_pages(n) for n in size))
        ids = []
        for u in range(len(size)):
            ids += tree.fork(int(ids[parent[u]]) if parent[u] >= 0 else -1, 1)
            a = int(first[u])
            tree.append_step(ids[u], k[a:a + int(size[u])], v[a:a + int(size[u])], quantize=True)
        s["nodes"] = np.asarray([ids[u] for u in s["leaves"]] if case["op"] == "attend" else ids, dtype=np.int32)
    else:
        s["k"], s["v"] = _held(k, "k"), _held(v, "v")
    return s


def _paths(s):
    """What a request for every branch needs: host lists for the framework, and on the device the tokens of every path."""
    case, leaves = s["case"], s["leaves"]
    see = _sees(case)
    s["q_lens"] = np.full(len(leaves), case["q_len"], dtype=np.int32) if case["q_len"] > 1 else None
    s["masks"] = None
    if case["drafts"]:
        bits = (see.astype(np.uint64) << np.arange(case["q_len"], dtype=np.uint64)).sum(1).astype(np.uint32)
        s["masks"] = np.tile(bits, len(leaves))
    s["sees"] = torch.as_tensor(see, device=_DEV)
    lengths = _path_lengths(s["parent"], s["size"], leaves)
    path = np.full((len(leaves), int(lengths.max())), -1, dtype=np.int32)
    for i, u in enumerate(leaves):
        chain = []
        while u >= 0:
            chain.append(u)
            u = s["parent"][u]
        at = 0
        for w in reversed(chain):
            n = s["size"][w]
            path[i, at:at + n] = np.arange(s["first"][w], s["first"][w] + n)
            at += n
    s["path"], s["lengths"] = torch.as_tensor(path, device=_DEV), torch.as_tensor(lengths, device=_DEV)


def run(s):
    return {"write": _run_write, "read": _run_read, "attend": _run_attend}[s["case"]["op"]](s)


# ---- the format --------------------------------------------------------------------------------
def _power(e):
    """2^e in 32 bits, e in -126 .. 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _held(x, which):
    """(codes [.., D / 2], two to a byte, the even dim's in the low half; exponents [.., D / 32]) of the cache."""
    lead, d = x.shape[:-1], x.shape[-1]
    x = x.float().reshape(*lead, d // 32, 32)
    e = torch.frexp(x.abs().amax(-1))[1] - 3  # amax = m 2^e with m in [0.5, 1)
    e = torch.where(x.abs().amax(-1) > 0, e, torch.full_like(e, -1000)).clamp(_TINY[which], _HUGE[which])
    y = x * _power(-e)[..., None]
    a = y.abs()
    # between neighbours: the middle goes to the even code
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (code + 8 * (y < 0)).reshape(*lead, d // 2, 2)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), e.to(torch.int16)


def _values(held):
    codes, e = held
    table = torch.tensor(_MAGNITUDES + [-m for m in _MAGNITUDES], device=_DEV)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    x = table[c].reshape(*e.shape, 32)
    return (x * _power(e)[..., None]).flatten(-2)


# ---- write -------------------------------------------------------------------------------------
def _rotate(x, c, s, case):
    r = case["rotary"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    y1, y2 = a * c - b * s, b * c + a * s
    y = torch.stack([y1, y2], -1).flatten(-2) if case["interleaved"] else torch.cat([y1, y2], -1)
    return torch.cat([y, x[..., r:]], -1)


def _by_node(x, s):
    y = torch.empty_like(x).flatten(0, 1)
    y[s["rows"].reshape(-1)] = x.flatten(0, 1)
    return y


def _run_write(s):
    case = s["case"]
    if own:
        tree, iters = s["tree"], case["iters"]
        (step,) = tree.fork(s["root"], 1)
        kids = np.asarray(tree.fork(step, case["nodes"]), dtype=np.int32)
        q_out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=_DEV)
        k_out = torch.empty(s["k"].shape, dtype=s["k"].dtype, device=_DEV) if case["want_k"] else None
        counts = None if case["count"] == 1 else s["counts"]
        for i in range(iters):
            tree.append_rotated(kids, counts, s["q"][i], s["k"][i], s["v"][i], q_out=q_out[i],
                                k_out=None if k_out is None else k_out[i],
                                positions=None if case["positions"] == "path" else s["host_positions"][i])
        k, v = tree.read_back(kids)
        tree.prune(step)
        return dict(q=q_out, cache_k=k, cache_v=v, **({} if k_out is None else dict(k=k_out)))
    t = s["positions"].double()[..., None] * torch.as_tensor(s["inv_freq"], device=_DEV)
    c, w = torch.cos(t).float()[..., None, :], torch.sin(t).float()[..., None, :]
    q, k = _rotate(s["q"].float(), c, w, case), _rotate(s["k"].float(), c, w, case)
    out = dict(q=q.to(torch.bfloat16), cache_k=_values(_held(_by_node(k, s), "k")).to(torch.bfloat16),
               cache_v=_values(_held(_by_node(s["v"].float(), s), "v")).to(torch.bfloat16))
    if case["want_k"]:
        out["k"] = k.to(torch.bfloat16)
    return out


def _run_read(s):
    if own:
        k, v = s["tree"].read_back(s["nodes"])
        return dict(k=k, v=v)
    return dict(k=_values(s["k"]).to(torch.bfloat16), v=_values(s["v"]).to(torch.bfloat16))


# ---- attend ------------------------------------------------------------------------------------
def _batches(case, longest, leaves):
    """Runs of branches whose keys and scores together are at most 2^30 numbers."""
    each = longest * (case["kv_heads"] * case["head_dim"] + case["q_heads"] * case["q_len"])
    per = max(1, (1 << 30) // each)
    return [(a, min(leaves, a + per)) for a in range(0, leaves, per)]


def _visible(s, a, b):
    """[branches, q_len, positions]"""
    n, t = s["case"]["q_len"], torch.arange(s["path"].shape[1], device=_DEV)
    rel = t - (s["lengths"][a:b, None] - n)
    draft = s["sees"][:, rel.clamp(0, n - 1)].permute(1, 0, 2)
    return (rel < 0)[:, None] | (draft & ((rel >= 0) & (rel < n))[:, None])


def _run_attend(s):
    case = s["case"]
    if own:
        out, lse = s["tree"].decode_attention(s["nodes"], s["q_lens"], s["q"], s["sm_scale"], draft_masks=s["masks"])
        return dict(out=out, lse=lse)
    hq, hkv, d, n = case["q_heads"], case["kv_heads"], case["head_dim"], case["q_len"]
    g, leaves = hq // hkv, len(s["leaves"])
    keys, values = _values(s["k"]), _values(s["v"])
    out, lse = torch.empty((leaves, n, hq, d), device=_DEV), torch.empty((leaves, n, hq), device=_DEV)
    for a, b in _batches(case, s["path"].shape[1], leaves):
        at = s["path"][a:b].clamp_min(0)
        q = s["q"].view(leaves, n, hkv, g, d)[a:b].float().permute(0, 2, 3, 1, 4).reshape((b - a) * hkv, g * n, d)
        k = keys[at].permute(0, 2, 3, 1).flatten(0, 1).contiguous()
        x = torch.matmul(q, k).view(b - a, hkv, g, n, -1) * s["sm_scale"]
        x = x.masked_fill(~_visible(s, a, b)[:, None, None], float("-inf"))
        top = x.amax(-1, keepdim=True)
        w = torch.exp(x - top)
        total = w.sum(-1, keepdim=True)
        v = values[at].transpose(1, 2).flatten(0, 1).contiguous()
        o = torch.matmul(w.view((b - a) * hkv, g * n, -1), v).view(b - a, hkv, g, n, d) / total
        out[a:b] = o.permute(0, 3, 1, 2, 4).reshape(b - a, n, hq, d)
        lse[a:b] = (top + torch.log(total))[..., 0].permute(0, 3, 1, 2).reshape(b - a, n, hq)
    return dict(out=out.view(leaves * n, hq, d), lse=lse.view(leaves * n, hq))


# ---- the definition in 64 bits -----------------------------------------------------------------
def _nearest(x, which):
    """The values that the cache holds for x, in 64 bits: the nearest of the format's, in steps of the binade."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -1000)
    e = torch.floor(torch.log2(top))
    e = e + (top >= torch.exp2(e + 1)).double() - (top < torch.exp2(e)).double()  # where log2 was rounded to a whole number
    unit = torch.exp2((e - 2).clamp(_TINY[which], _HUGE[which]))
    m = (y / unit).abs().clamp_max(6.0)
    step = torch.where(m >= 4, 2.0, torch.where(m >= 2, 1.0, 0.5))
    return (torch.sign(y) * torch.round(m / step) * step * unit).flatten(-2)


def _exact_write(case, seed):
    s = dict(_inputs(case, seed), case=case)
    angle = torch.outer(s["positions"].reshape(-1).double(), torch.as_tensor(s["inv_freq"], device=_DEV))
    turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]
    half, r = case["rotary"] // 2, case["rotary"]
    at = (torch.arange(0, r, 2), torch.arange(1, r, 2)) if case["interleaved"] else (torch.arange(half), torch.arange(half, r))

    def turned(x):  # pairs as complex numbers
        x = x.flatten(0, 1).double()
        z = torch.complex(x[..., at[0].to(_DEV)], x[..., at[1].to(_DEV)]) * turn
        y = x.clone()
        y[..., at[0].to(_DEV)], y[..., at[1].to(_DEV)] = z.real, z.imag
        return y

    q, k = turned(s["q"]), turned(s["k"])
    order = torch.argsort(s["rows"].reshape(-1))
    out = dict(q=q.view(s["q"].shape), cache_k=_nearest(k[order], "k"), cache_v=_nearest(s["v"].flatten(0, 1)[order], "v"))
    if case["want_k"]:
        out["k"] = k.view(s["k"].shape)
    return out


def _exact_attend(case, seed):
    if work(case)["flops"] > 1e12:
        return None
    s = _inputs(case, seed)
    hq, hkv, d, n = case["q_heads"], case["kv_heads"], case["head_dim"], case["q_len"]
    leaves = len(s["leaves"])
    out, lse = (torch.empty(shape, dtype=torch.float64, device=_DEV) for shape in ((leaves, n, hq, d), (leaves, n, hq)))
    see = torch.as_tensor(_sees(case), device=_DEV)
    part = lambda x, u: x[int(s["first"][u]):int(s["first"][u] + s["size"][u])]  # noqa: E731
    node, above = {}, None
    for i, u in enumerate(s["leaves"]):
        if s["parent"][u] != above:  # branches of one parent follow each other
            above, chain, w = s["parent"][u], [], s["parent"][u]
            while w >= 0:
                chain.insert(0, w)
                w = s["parent"][w]
            node = {x: [_nearest(part(s[x], c), x) for c in chain] for x in ("k", "v")}
        k, v = (torch.cat(node[x] + [_nearest(part(s[x], u), x)]).transpose(0, 1).contiguous() for x in ("k", "v"))
        q = s["q"][i * n:(i + 1) * n].double().view(n, hkv, -1, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
        x = s["sm_scale"] * torch.bmm(q, k.transpose(1, 2).contiguous()).view(hkv, hq // hkv, n, -1)
        x[..., -n:] = torch.where(see, x[..., -n:], float("-inf"))
        z = torch.logsumexp(x, -1)
        o = torch.bmm((x - z[..., None]).exp().view(hkv, (hq // hkv) * n, -1), v).view(hkv, hq // hkv, n, d)
        out[i], lse[i] = o.permute(2, 0, 1, 3).reshape(n, hq, d), z.permute(2, 0, 1).reshape(n, hq)
    return dict(out=out.view(-1, hq, d), lse=lse.view(-1, hq))


def exact(case, seed):
    if case["op"] == "attend":
        return _exact_attend(case, seed)
    if case["op"] == "write":
        return _exact_write(case, seed)
    s = _inputs(case, seed)
    return dict(k=_nearest(s["k"], "k"), v=_nearest(s["v"], "v"))
