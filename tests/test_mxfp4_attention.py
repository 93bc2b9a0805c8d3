"""Decode attention over MXFP4 pools against the definition in 64 bits, on the values the format holds."""

import numpy as np
import pytest
import torch

import paper_2605_10195_amd as spex
from mxfp4_common import attention, quantised, row_error, score_error

pytestmark = pytest.mark.gpu

HEADS = [(4, 2, 64), (8, 2, 128), (28, 4, 128), (64, 8, 128), (6, 3, 32), (12, 4, 96), (5, 5, 160), (4, 1, 192), (3, 1, 224), (16, 4, 256), (40, 1, 64), (96, 2, 32)]


class Forest:
    """The same tree in the library and as arrays: nodes of (parent, tokens), values by `value(rng, shape)`."""

    def __init__(self, heads, nodes, seed=0, value=None, spare=4, **kw):
        self.hq, self.hkv, self.dim = heads
        self.rng = np.random.default_rng(seed)
        self.value = value or (lambda rng, shape: rng.standard_normal(shape))
        pages = sum(-(-n // 16) for _, n in nodes) + spare
        self.tree = spex.SpexTree(*heads, 16, "bf16", "mxfp4", num_pages=pages, free_order=self.rng.permutation(pages), pool_fill=0xFF, **kw)
        self.parent, self.ids, self.k, self.v = [], [], [], []
        for parent, n in nodes:  # parents come first: a node is filled while it has no children
            self.ids += self.tree.fork(self.ids[parent] if parent >= 0 else -1, 1)
            self.parent.append(parent)
            self.k.append(np.zeros((0, self.hkv, self.dim)))
            self.v.append(np.zeros((0, self.hkv, self.dim)))
            self.fill(len(self.ids) - 1, n)

    def fill(self, u, n):
        if n == 0:
            return
        x = [torch.as_tensor(self.value(self.rng, (n, self.hkv, self.dim))).to(torch.bfloat16) for _ in range(2)]
        self.k[u], self.v[u] = (np.concatenate([old, quantised(y.double().numpy(), w)]) for old, y, w in ((self.k[u], x[0], "k"), (self.v[u], x[1], "v")))
        self.tree.append_step(self.ids[u], x[0].cuda(), x[1].cuda(), quantize=True)

    def path(self, u):
        chain = []
        while u >= 0:
            chain.insert(0, u)
            u = self.parent[u]
        return np.concatenate([self.k[w] for w in chain]), np.concatenate([self.v[w] for w in chain])

    def check(self, leaves, q_lens=None, masks=None, scale=None, spread=2.0, static=False, loose=1e-5, q=None):
        lens = q_lens or [1] * len(leaves)
        scale = scale or self.dim ** -0.5
        if q is None:
            q = torch.as_tensor(self.rng.standard_normal((sum(lens), self.hq, self.dim)) * spread).to(torch.bfloat16)
        ids = [self.ids[u] for u in leaves]
        out = torch.full(q.shape, float("nan"), device="cuda")
        lse = torch.full(q.shape[:2], float("nan"), device="cuda")
        self.tree.decode_attention(ids, q_lens, q.cuda(), scale, out, lse, draft_masks=masks, static_scratch=static)
        torch.cuda.synchronize()
        out, lse, q = out.cpu().double().numpy(), lse.cpu().double().numpy(), q.double().numpy()
        at, ref = 0, np.zeros_like(out)
        for u, n in zip(leaves, lens):
            k, v = self.path(u)
            total = len(k)
            see = np.arange(total)[None] <= total - n + np.arange(n)[:, None]
            if masks is not None:
                for j in range(n):
                    see[j, total - n:] = [(int(masks[at + j]) >> i) & 1 for i in range(n)]
            for h in range(self.hq):
                g = h // (self.hq // self.hkv)
                o, z, mean, size = attention(q[at:at + n, h], k[:, g], v[:, g], see, scale)
                ref[at:at + n, h] = o
                tol = row_error(self.dim, total, size, mean) + 1e-30
                assert (np.abs(out[at:at + n, h] - o) <= tol).all(), (u, h, np.abs(out[at:at + n, h] - o).max(), tol.max())
                # the logarithm of a sum of weights that are off as above, and one rounding of a sum with the reference
                assert (np.abs(lse[at:at + n, h] - z) <= score_error(self.dim, size) + 2.0 ** -15 + 2.0 ** -22 * np.abs(z)).all()
            at += n
        rel = np.linalg.norm(out - ref) / np.linalg.norm(ref)
        assert rel <= loose, rel  # as fp32 pools are held to
        return out, lse


def bushy(rng, roots, depth, fan, longest):
    """Random trees: lengths from none to `longest`, every one of them somewhere."""
    nodes, leaves = [], []
    for _ in range(roots):
        level = [len(nodes)]
        nodes.append((-1, int(rng.integers(1, longest + 1))))
        for d in range(depth):
            below = []
            for u in level:
                for _ in range(int(rng.integers(1, fan + 1))):
                    below.append(len(nodes))
                    nodes.append((u, int(rng.choice([0, 1, 15, 16, 17, int(rng.integers(1, longest + 1))]))))
            level = below
        leaves += level
    return nodes, leaves


MODES = [0, 2, 3]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("heads", HEADS)
def test_trees(heads, mode):
    """Every head size and grouping, in both kernel sets: shared nodes, empty nodes, pages that end anywhere."""
    rng = np.random.default_rng(heads[0] + heads[2])
    nodes, leaves = bushy(rng, 2, 3, 3, 70)
    f = Forest(heads, nodes, seed=heads[2], kernel_mode=mode)
    f.check(leaves)
    f.check(leaves[::-1] + leaves[:1] + [0])  # another order, one twice, an interior node
    f.tree.close()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("tokens", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 500])
def test_lengths(tokens, mode):
    f = Forest((8, 2, 128), [(-1, tokens)], seed=tokens, kernel_mode=mode)
    f.check([0])
    f.check([0], [tokens if tokens < 40 else 40])
    f.tree.close()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("heads", [(8, 2, 128), (28, 4, 128), (6, 3, 96), (4, 2, 64)])
@pytest.mark.parametrize("tall", [3, 9, 40, 130])
def test_many_queries(heads, tall, mode):
    """Requests of one query and of many together: causal ends inside every page, rows of several tiles, pieces of a request."""
    f = Forest(heads, [(-1, 37), (0, 140), (0, 150), (0, 135), (1, 131)], seed=tall, kernel_mode=mode)
    f.check([4, 2, 3, 2], [tall, 1, max(1, tall - 2), 2])
    f.tree.close()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("heads", [(8, 2, 128), (40, 8, 64), (12, 4, 96)])
def test_draft_trees(heads, mode):
    """Visibility masks: trees of drafts, single tokens, drafts that see nothing of the others, 32 of them."""
    rng = np.random.default_rng(3)
    f = Forest(heads, [(-1, 50), (0, 40), (0, 33), (0, 47), (0, 6)], seed=5, kernel_mode=mode)
    lens = [6, 32, 1, 6]
    masks = []
    for n in lens:
        masks += [(1 << j) | int(rng.integers(0, 1 << n)) for j in range(n)]
    f.check([1, 2, 3, 4], lens, np.asarray(masks, np.uint32))
    chain = np.concatenate([(1 << np.arange(1, n + 1)) - 1 for n in lens]).astype(np.uint32)
    f.check([1, 2, 3, 4], lens, chain)
    f.check([1, 2, 3, 4], lens, np.concatenate([1 << np.arange(n) for n in lens]).astype(np.uint32))
    f.tree.close()


@pytest.mark.parametrize("waves", [2, 4, 8])
@pytest.mark.parametrize("tiles", [1, 2, 4])
@pytest.mark.parametrize("heads", [(8, 2, 128), (16, 1, 64), (6, 3, 96)])
def test_walk_shapes(heads, tiles, waves):
    """Every shape of the tree walk that can be asked for."""
    if waves == 2 and tiles == 4:
        pytest.skip("no such lists")
    rng = np.random.default_rng(7)
    nodes, leaves = bushy(rng, 3, 2, 5, 90)
    f = Forest(heads, nodes, seed=9, kernel_mode=3, walk_row_tiles=tiles, walk_waves=waves)
    f.check(leaves)
    f.tree.close()


@pytest.mark.parametrize("chunks", [(1, 1), (2, 3), (7, 64)])
def test_chunks(chunks):
    f = Forest((8, 2, 128), [(-1, 333), (0, 100), (0, 90), (0, 1)], seed=11, kernel_mode=2, prefix_chunk_pages=chunks[0], suffix_chunk_pages=chunks[1])
    f.check([1, 2, 3])
    f.tree.close()


@pytest.mark.parametrize("mode", MODES)
def test_a_long_prefix_of_many_branches(mode):
    """More rows on one prefix than a workgroup holds, and a prefix much longer than what hangs below it."""
    nodes = [(-1, 3000)] + [(0, 1 + i % 20) for i in range(70)]
    f = Forest((8, 2, 128), nodes, seed=13, kernel_mode=mode)
    f.check(list(range(1, 71)))
    f.tree.close()


def test_growing_branches():
    """Branches that grow a token a call: the cached lists are patched, pages started, in the launches of the appends."""
    n = 20
    f = Forest((8, 2, 128), [(-1, 60)] + [(0, 1 + i % 4) for i in range(n)], seed=15, spare=80)
    leaves = list(range(1, n + 1))
    f.tree.set_rotation(128, np.zeros(64))
    states = set()
    for step in range(24):
        x = torch.as_tensor(f.rng.standard_normal((2, n, 2, 128))).to(torch.bfloat16)
        if step % 3 == 1:
            f.tree.append_rotated([f.ids[u] for u in leaves], None, None, x[0].cuda(), x[1].cuda())  # by no angle: unchanged
        else:
            f.tree.append_tokens([f.ids[u] for u in leaves], x[0].cuda(), x[1].cuda(), quantize=True)
        for i, u in enumerate(leaves):
            f.k[u] = np.concatenate([f.k[u], quantised(x[0, i].double().numpy(), "k")[None]])
            f.v[u] = np.concatenate([f.v[u], quantised(x[1, i].double().numpy(), "v")[None]])
        f.check(leaves)
        states.add(f.tree.last_launch_info()["plan_rebuilt"])
    assert 2 in states  # some plans were patched
    f.tree.close()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("kind", ["rising", "one key", "small scale", "large scale", "wide values", "far scores"])
def test_shaped_scores(kind, mode):
    """References that move many times, one dominant key, flat and steep softmaxes, values at the ends of the format, scores of millions."""
    def value(rng, shape):
        x = rng.standard_normal(shape)
        if kind == "rising":
            x[..., 0] = 4.0 * np.arange(shape[0])[:, None] / 16
        if kind == "one key" and shape[0] > 5:
            x[5, :, 0] = 60.0
        if kind == "wide values":
            x *= np.exp2(rng.integers(-22, 12, (shape[0], 1, shape[2] // 32))).repeat(32, -1)
        if kind == "far scores":
            x[..., 0] = 2.0 ** 20 * (1 + (np.arange(shape[0]) % 2))[:, None]
        return x

    f = Forest((8, 2, 128), [(-1, 150), (0, 70), (0, 33)], seed=17, kernel_mode=mode, value=value)
    q = torch.as_tensor(np.random.default_rng(1).standard_normal((2, 8, 128))).to(torch.bfloat16)
    if kind in ("rising", "one key"):
        q[..., 0] = 8.0
    if kind == "far scores":
        q[..., 0] = 2.0 ** 16
        q[..., 1:] = 0  # the far part is exact: whole multiples of powers of two
    scale = {"small scale": 1e-4, "large scale": 3.0}.get(kind, 128 ** -0.5)
    if kind == "wide values":  # keys of many binades would drown the bound on the scores in the largest
        q = q * 2.0 ** -14
    f.check([1, 2], scale=scale, q=q, loose=1e-5 if kind not in ("large scale", "wide values") else 1e-3)
    f.tree.close()


def test_values_at_the_ends():
    """V at 49152 and at 2^-24, alone and side by side, through the weights of a softmax over few tokens."""
    def value(rng, shape):
        x = np.zeros(shape)
        x[..., :32] = 6.0 * 2.0 ** 13
        x[..., 32:64] = 0.5 * 2.0 ** -23
        x[..., 64:96] = -6.0 * 2.0 ** 13
        x[..., 96:] = rng.choice([-1.0, 1.0], x[..., 96:].shape) * 2.0 ** -24
        return x

    f = Forest((4, 1, 128), [(-1, 19), (0, 5)], seed=19, value=value)
    out, _ = f.check([1], q=torch.zeros((1, 4, 128), dtype=torch.bfloat16))
    assert np.allclose(out[..., :32], 49152.0, rtol=1e-6) and np.allclose(out[..., 32:64], 2.0 ** -24, rtol=1e-6)
    f.tree.close()


@pytest.mark.parametrize("mode", MODES)
def test_entry_points_agree(mode):
    """The call that allocates nothing gives the same bits; so does the same call again, and one recorded in a graph and replayed."""
    rng = np.random.default_rng(21)
    nodes, leaves = bushy(rng, 4, 2, 4, 80)
    f = Forest((8, 2, 128), nodes, seed=23, kernel_mode=mode)
    q = torch.as_tensor(rng.standard_normal((len(leaves), 8, 128))).to(torch.bfloat16)
    a = f.check(leaves, q=q)
    b = f.check(leaves, q=q, static=True)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    ids, qd = [f.ids[u] for u in leaves], q.cuda()
    out, lse = f.tree.decode_attention(ids, None, qd, 128 ** -0.5)
    assert np.array_equal(out.cpu().double().numpy(), a[0])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        f.tree.decode_attention(ids, None, qd, 128 ** -0.5, out, lse)
    for i in range(4):
        out.fill_(float("nan"))
        qd.copy_(q.cuda() * (1 + i % 2))
        graph.replay()
        torch.cuda.synchronize()
        eager, _ = f.tree.decode_attention(ids, None, qd, 128 ** -0.5)
        assert torch.equal(out, eager)
    f.tree.close()


def test_offsets():
    """Queries two bytes off a 16-byte boundary, outputs four; K and V of a page side by side; a pool beyond 2^31 bytes of which the last pages are used."""
    f = Forest((8, 2, 128), [(-1, 50), (0, 20), (0, 9)], seed=25, interleave_kv=True)
    ids = [f.ids[1], f.ids[2]]
    q = torch.as_tensor(f.rng.standard_normal((2, 8, 128))).to(torch.bfloat16)
    want, _ = f.check([1, 2], q=q)
    room = torch.zeros(2 * 8 * 128 + 1, dtype=torch.bfloat16, device="cuda")
    room[1:] = q.cuda().flatten()
    place = torch.zeros(2 * 8 * 128 + 1, device="cuda")
    out, _ = f.tree.decode_attention(ids, None, room[1:].view(2, 8, 128), 128 ** -0.5, place[1:].view(2, 8, 128))
    assert np.array_equal(out.cpu().double().numpy(), want)
    f.tree.close()
    pages = 260000  # of 8 x 1088 bytes
    far = spex.SpexTree(8, 8, 128, 16, "bf16", "mxfp4", num_pages=pages, free_order=list(range(pages - 1, -1, -1)))
    (root,) = far.fork(-1, 1)
    k, v = (torch.as_tensor(np.random.default_rng(i).standard_normal((70, 8, 128))).to(torch.bfloat16) for i in (1, 2))
    far.append_step(root, k.cuda(), v.cuda(), quantize=True)
    gk, gv = far.read_back([root])
    wk, wv = quantised(k.double().numpy(), "k"), quantised(v.double().numpy(), "v")
    assert np.array_equal(gk.cpu().double().numpy(), wk) and np.array_equal(gv.cpu().double().numpy(), wv)
    q = torch.as_tensor(np.random.default_rng(3).standard_normal((1, 8, 128))).to(torch.bfloat16)
    out, _ = far.decode_attention([root], None, q.cuda(), 128 ** -0.5)
    for h in range(8):
        o, _, mean, size = attention(q[:, h].double().numpy(), wk[:, h], wv[:, h], np.ones((1, 70), bool), 128 ** -0.5)
        assert (np.abs(out[:, h].cpu().double().numpy() - o) <= row_error(128, 70, size, mean)).all()
    far.close()


def test_a_search_as_it_is_used():
    """A prompt appended rotated, branches forked, tokens appended and attended step by step, a branch pruned, the rest read back."""
    hq, hkv, dim = 8, 2, 128
    tree = spex.SpexTree(hq, hkv, dim, 16, "bf16", "mxfp4", num_pages=64, pool_fill=0xFF)
    freq = 10000.0 ** (-np.arange(0, dim, 2) / dim)
    tree.set_rotation(dim, freq)
    rng = np.random.default_rng(31)
    (root,) = tree.fork(-1, 1)

    def made(n):
        return tuple(torch.as_tensor(rng.standard_normal((n, h, dim))).to(torch.bfloat16).cuda() for h in (hq, hkv, hkv))

    tree.append_rotated([root], [53], *made(53))
    branches = tree.fork(root, 5)
    for step in range(20):
        q, _ = tree.append_rotated(branches, None, *made(len(branches)))
        out, lse = tree.decode_attention(branches, None, q, dim ** -0.5)
        if step == 9:
            tree.prune(branches.pop(1))
    gk, gv = tree.read_back([root] + branches)  # what the cache holds: attention over it in 64 bits is what came out
    gk, gv, q = (x.cpu().double().numpy() for x in (gk, gv, q))
    assert len(gk) == 53 + 4 * 20
    for i in range(len(branches)):
        own = np.r_[0:53, 53 + 20 * i:73 + 20 * i]
        for h in range(hq):
            o, z, mean, size = attention(q[i:i + 1, h], gk[own, h // 4], gv[own, h // 4], np.ones((1, 73), bool), dim ** -0.5)
            assert (np.abs(out[i, h].cpu().double().numpy() - o) <= row_error(dim, 73, size, mean)).all()
    tree.close()
