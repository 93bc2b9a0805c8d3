"""MXFP4 pools: configurations and refusals on the CPU (nothing is launched, nothing changes); appends and read back on the GPU
against the format's definition in 64 bits."""

import ctypes as C

import numpy as np
import pytest
import torch

import paper_2605_10195_amd as spex
from mxfp4_common import assert_held, quantised
from paper_2605_10195_amd import binding
from test_append_rotated import append, handle, magnitude, state, turned  # noqa: F401 (handle: a fixture)

OK, INVALID, BAD_NODE, NOT_LEAF, OOM, EMPTY, UNSUPPORTED, CAPACITY = 0, 1, 2, 3, 4, 5, 6, 8


# ---- configurations and refusals -------------------------------------------------------------------
def config(heads=(4, 2, 64), page=16, pages=8, q=binding.BF16, pool=64, **fields):
    cfg = binding.Config()
    cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim = heads
    cfg.page_size, cfg.q_dtype, cfg.kv_dtype, cfg.num_pages = page, q, binding.MXFP4, pages
    cfg.k_pool = cfg.v_pool = pool
    for name, x in fields.items():
        setattr(cfg, name, x)
    return cfg


def create(cfg):
    h = C.c_void_p()
    st = binding.lib.spex_tree_create(C.byref(cfg), C.byref(h))
    if st == OK:
        binding.lib.spex_tree_destroy(h)
    return st


@pytest.mark.parametrize("want,kw", [(OK, {}), (OK, dict(pool=None)), (OK, dict(heads=(4, 2, 32))), (OK, dict(heads=(6, 3, 96))), (OK, dict(heads=(2, 1, 256))),
                                     (OK, dict(heads=(2, 1, 224))), (UNSUPPORTED, dict(heads=(4, 2, 80))), (UNSUPPORTED, dict(heads=(4, 2, 48))),
                                     (UNSUPPORTED, dict(page=32)), (UNSUPPORTED, dict(page=8)), (UNSUPPORTED, dict(q=binding.F32)),
                                     (UNSUPPORTED, dict(q=binding.MXFP4)), (UNSUPPORTED, dict(pool=72)), (INVALID, dict(k_scale=64)),
                                     (INVALID, dict(v_scale=64)), (INVALID, dict(heads=(3, 2, 64)))])
def test_configurations(want, kw):
    assert create(config(**kw)) == want


@pytest.mark.parametrize("dim,stride,want", [(32, 0, 8 * 2 * 272), (128, 0, 8 * 2 * 1088), (256, 0, 8 * 2 * 2176), (96, 4, (7 * 4 + 2) * 816)])
def test_pool_bytes(dim, stride, want):
    n = C.c_size_t()
    assert binding.lib.spex_pool_bytes(C.byref(config(heads=(4, 2, dim), page_stride_tiles=stride)), C.byref(n)) == OK
    assert n.value == want  # 17 / 32 of a byte an element
    assert binding.lib.spex_pool_bytes(C.byref(config(heads=(4, 2, 40))), C.byref(n)) == UNSUPPORTED
    assert binding.lib.spex_pool_bytes(C.byref(config(page=64)), C.byref(n)) == UNSUPPORTED


@pytest.mark.parametrize("want,nodes,kw", [
    (INVALID, [0], dict(k_scales=64, v_scales=64, n_scales=4)), (INVALID, [0, 0], {}), (BAD_NODE, [4], {}), (NOT_LEAF, [0, 2], {}),
    (OOM, [0], dict(counts=[129])), (INVALID, [0], dict(k=None)), (OK, [], {}), (OK, [0], dict(counts=[0]))])
def test_rotated_appends_are_checked(handle, want, nodes, kw):  # noqa: F811
    h = handle(kv=binding.MXFP4)
    before = state(h)
    assert append(h, nodes, **kw) == want
    assert state(h) == before


def test_other_appends_are_checked(handle):  # noqa: F811
    h = handle(kv=binding.MXFP4)
    before = state(h)
    na = np.array([0, 1], np.int32)
    lib, at = binding.lib, na.ctypes.data
    assert lib.spex_tree_append_step(h, 0, 3, 64, 64, None, None, None) == UNSUPPORTED            # no form of given codes
    assert lib.spex_tree_append_tokens(h, at, 2, 64, 64, None, None, None) == UNSUPPORTED
    assert lib.spex_tree_append_tokens_quantize(h, at, 2, 64, 64, 64, 64, None) == INVALID       # scales
    assert lib.spex_tree_append_tokens_quantize(h, at, -1, 64, 64, None, None, None) == INVALID
    assert lib.spex_tree_append_step_quantize(h, 2, 3, 64, 64, None) == NOT_LEAF
    assert lib.spex_tree_append_step_quantize(h, 0, 200, 64, 64, None) == OOM
    assert lib.spex_tree_append_step_quantize(h, 0, -1, 64, 64, None) == INVALID
    assert lib.spex_tree_append_step_quantize(h, 0, 3, 64, None, None) == INVALID
    assert lib.spex_tree_append_step_quantize(h, 0, 0, 64, 64, None) == OK
    assert state(h) == before
    assert lib.spex_tree_append_step(h, 0, 3, None, None, None, None, None) == OK                 # page table only
    assert lib.spex_tree_append_tokens(h, at, 2, None, None, None, None, None) == OK
    assert lib.spex_tree_append_step_quantize(handle(kv=binding.BF16), 0, 3, 64, 64, None) == UNSUPPORTED
    assert lib.spex_tree_append_step_quantize(handle(kv=binding.MXFP4, pools=False), 0, 3, 64, 64, None) == INVALID


def read(h, nodes, firsts=None, counts=None, k=None, v=None, count=True, n=None):
    a = [None if x is None else np.asarray(x, np.int32) for x in (nodes, firsts, counts)]
    p = [None if x is None else x.ctypes.data for x in a]
    total = C.c_int64(-1)
    st = binding.lib.spex_tree_read_back(h, *p, len(nodes) if n is None else n, k, v, C.byref(total) if count else None, None)
    return st, total.value


def test_read_back_is_checked(handle):  # noqa: F811
    h = handle(kv=binding.MXFP4)
    assert binding.lib.spex_tree_append_step(h, 0, 20, None, None, None, None, None) == OK
    assert binding.lib.spex_tree_append_step(h, 3, 5, None, None, None, None, None) == OK
    assert read(h, [0, 3, 1]) == (OK, 25)
    assert read(h, [0, 0, 3], [20, 3, 1], [0, 9, 4]) == (OK, 13)
    assert read(h, [0, 3], [1, 2]) == (OK, 22)
    assert read(h, [2]) == (OK, 0)                                  # no leaf, no tokens
    assert read(h, []) == (OK, 0)
    for nodes, firsts, counts, want in [([4], None, None, BAD_NODE), ([-1], None, None, BAD_NODE), ([0], [-1], None, INVALID), ([0], [21], None, INVALID),
                                        ([0], [0], [21], INVALID), ([0], [20], [1], INVALID), ([0], None, [-1], INVALID), ([0], [2 ** 31 - 1], [2 ** 31 - 1], INVALID)]:
        assert read(h, nodes, firsts, counts)[0] == want, (nodes, firsts, counts)
        assert read(h, nodes, firsts, counts, 64, 64)[0] == want
    assert read(h, [0], n=-1)[0] == INVALID
    assert read(h, [0], k=64)[0] == INVALID and read(h, [0], v=64)[0] == INVALID
    assert read(h, [0], count=False)[0] == INVALID                  # neither values nor their number are asked for
    assert read(None, [0])[0] == INVALID
    assert read(handle(kv=binding.BF16), [0])[0] == UNSUPPORTED
    assert read(handle(kv=binding.FP8_E4M3), [0])[0] == UNSUPPORTED
    host = handle(kv=binding.MXFP4, pools=False)
    assert binding.lib.spex_tree_append_step(host, 0, 20, None, None, None, None, None) == OK
    assert read(host, [0]) == (OK, 20) and read(host, [0], k=64, v=64)[0] == INVALID
    assert binding.lib.spex_tree_gather_kv(h, 0, 0, 1, 64, 64, 64, 64, None) == INVALID          # no scales to give


def test_kernel_modes(handle):  # noqa: F811
    h = handle(kv=binding.MXFP4)
    assert binding.lib.spex_tree_append_step(h, 0, 3, None, None, None, None, None) == OK
    la = np.zeros(1, np.int32)
    assert binding.lib.spex_tree_set_tuning(h, 0, 0, 1, 0, 0) == OK
    assert binding.lib.spex_tree_decode_attention(h, la.ctypes.data, None, 1, 64, 64, None, 1.0, None) == UNSUPPORTED
    la[0] = 1
    assert binding.lib.spex_tree_set_tuning(h, 0, 0, 0, 0, 0) == OK
    assert binding.lib.spex_tree_decode_attention(h, la.ctypes.data, None, 1, 64, 64, None, 1.0, None) == EMPTY


def test_bytes_of_a_path(handle):  # noqa: F811
    h = handle(kv=binding.MXFP4)
    assert binding.lib.spex_tree_append_step(h, 0, 20, None, None, None, None, None) == OK
    b = C.c_double()
    assert binding.lib.spex_tree_path_kv_bytes(h, 0, C.byref(b)) == OK
    assert b.value == 20 * 2 * 2 * 64 * 17 / 32


# ---- values ----------------------------------------------------------------------------------------
def new_tree(heads=(4, 2, 64), pages=64, **kw):
    return spex.SpexTree(*heads, 16, "bf16", "mxfp4", num_pages=pages, pool_fill=0xFF, **kw)


def random(shape, seed, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * spread).to(torch.bfloat16)


def f64(x):
    return x.detach().cpu().double().numpy()


def same(a, b):
    return np.array_equal(f64(a), b)  # -0 and 0 are one value


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("interleave", [False, True])
def test_steps_round_trip(dim, interleave):
    """Runs of one node, continued at every slot of a page, come back as the nearest values of the format."""
    tree = new_tree((6, 3, dim), interleave_kv=interleave)
    (root,) = tree.fork(-1, 1)
    k, v = random((70, 3, dim), 1), random((70, 3, dim), 2)
    at = 0
    for n in [1, 2, 1, 13, 16, 3, 20, 14]:
        tree.append_step(root, k[at:at + n].cuda(), v[at:at + n].cuda(), quantize=True)
        at += n
    for first, n in [(0, 70), (5, 1), (15, 3), (16, 16), (33, 30), (69, 1)]:
        gk, gv = tree.read_back([root], [first], [n])
        assert same(gk, quantised(f64(k), "k")[first:first + n]) and same(gv, quantised(f64(v), "v")[first:first + n])
        hk, hv, ks, vs = tree.gather_kv(root, first, n)
        assert torch.equal(hk, gk) and torch.equal(hv, gv) and ks is None and vs is None
    tree.close()


@pytest.mark.gpu
def test_every_bf16_value():
    """All finite bf16 magnitudes with both signs, each with a block of its own, then as the small one beside every binade: roundings, ties,
    saturation, exponents at both ends."""
    bits = torch.arange(0x7f80, dtype=torch.int32)
    x = torch.cat([bits, bits + 0x8000]).to(torch.int16).view(torch.bfloat16)
    tree = new_tree((2, 1, 128), pages=5000)
    (root,) = tree.fork(-1, 1)
    alone = torch.zeros((len(x), 32), dtype=torch.bfloat16)
    alone[:, 7] = x
    beside = torch.zeros((len(x), 32), dtype=torch.bfloat16)
    beside[:, 0] = x
    top = (x.float().abs().clamp(2.0 ** -120, 2.0 ** 120).double() * 2.0 ** (torch.arange(len(x)) % 5)).clamp_max(3e38)
    beside[:, 31] = top.to(torch.bfloat16)
    rows = torch.cat([alone, beside]).reshape(-1, 1, 128).contiguous()
    tree.append_step(root, rows.cuda(), rows.cuda(), quantize=True)
    gk, gv = tree.read_back([root])
    assert same(gk, quantised(f64(rows), "k"))
    assert same(gv, quantised(f64(rows), "v"))
    assert float(gv.abs().max()) == 49152.0
    tree.close()


@pytest.mark.gpu
@pytest.mark.parametrize("heads,n", [((4, 2, 64), 1), ((28, 4, 128), 37), ((6, 3, 96), 5), ((8, 1, 256), 300), ((64, 8, 128), 150)])
def test_tokens_of_many_nodes(heads, n):
    """One token for each of many nodes, again and again, and all of them read back, whole and in parts, in another order, twice."""
    hkv, dim = heads[1:]
    tree = new_tree(heads, pages=3 * n + 8)
    (root,) = tree.fork(-1, 1)
    kids = tree.fork(root, n)
    for i, u in enumerate(kids):
        tree.append_step(u, None, None, n_tokens=i % 17)
    steps = 20
    k, v = random((steps, n, hkv, dim), 3), random((steps, n, hkv, dim), 4)
    for i in range(steps):
        tree.append_tokens(kids, k[i].cuda(), v[i].cuda(), quantize=True)
    firsts = [i % 17 for i in range(n)]
    gk, gv = tree.read_back(kids, firsts)
    assert same(gk, quantised(f64(k.transpose(0, 1).flatten(0, 1)), "k")) and same(gv, quantised(f64(v.transpose(0, 1).flatten(0, 1)), "v"))
    order = list(reversed(kids)) + kids[:1]
    starts, counts = [x % 17 + x % 3 for x in list(reversed(range(n))) + [0]], [x % 5 for x in list(reversed(range(n))) + [3]]
    gk, gv = tree.read_back(order, starts, counts)
    want = [(kids.index(u), s - kids.index(u) % 17, c) for u, s, c in zip(order, starts, counts)]
    assert same(gk, quantised(np.concatenate([f64(k[a:a + c, i]) for i, a, c in want]), "k"))
    assert same(gv, quantised(np.concatenate([f64(v[a:a + c, i]) for i, a, c in want]), "v"))
    tree.close()


@pytest.mark.gpu
@pytest.mark.parametrize("heads,rotary,interleaved,wide", [((4, 2, 64), 64, False, True), ((28, 4, 128), 128, False, True), ((28, 4, 128), 64, True, True),
                                                           ((6, 3, 96), 48, False, True), ((6, 3, 96), 96, True, False), ((4, 2, 128), 30, False, True),
                                                           ((4, 2, 128), 6, True, False), ((2, 1, 256), 256, False, False), ((6, 3, 32), 14, False, False),
                                                           ((3, 1, 160), 160, False, True), ((2, 1, 192), 64, True, True), ((2, 2, 224), 224, False, False)])
@pytest.mark.parametrize("place", ["fresh", "in place", "given positions"])
def test_rotated_appends(heads, rotary, interleaved, wide, place):
    """Rotated on the way, from parts of one projection; wide False: rows that begin two bytes off a 16-byte boundary."""
    hq, hkv, dim = heads
    counts = [1, 16, 0, 37, 2, 15]
    total = sum(counts)
    tree = new_tree(heads)
    (root,) = tree.fork(-1, 1)
    tree.append_step(root, None, None, n_tokens=40)
    kids = tree.fork(root, len(counts))
    for i, u in enumerate(kids):
        tree.append_step(u, None, None, n_tokens=3 * i)
    freq = 10000.0 ** (-np.arange(0, rotary, 2) / rotary)
    tree.set_rotation(rotary, freq, interleaved=interleaved)
    x = random((total, hq + 2 * hkv, dim), 5).cuda()
    row = (hq + 2 * hkv) * dim
    room = torch.zeros(total * (row + 8) + 8, dtype=torch.bfloat16, device="cuda")
    parts = room[0 if wide else 1:][:total * (row + 8)].view(total, row + 8)[:, :row].view(total, hq + 2 * hkv, dim)
    parts.copy_(x)
    q, k, v = parts[:, :hq], parts[:, hq:hq + hkv], parts[:, hq + hkv:]
    pos = np.concatenate([40 + 3 * i + np.arange(c) for i, c in enumerate(counts)])
    if place == "given positions":
        pos = np.random.default_rng(1).integers(0, 1 << 20, total)
    kw = dict(q_out=q, k_out=k) if place == "in place" else dict(want_k=place == "fresh")
    got_q, got_k = tree.append_rotated(kids, counts, q, k, v, positions=pos if place == "given positions" else None, **kw)
    want, size = turned(x, pos, freq, rotary, interleaved).numpy(), magnitude(x, rotary, interleaved).numpy()
    off = 4 * 2.0 ** -24 * size  # cosine and sine, two products and a sum, half a step of fp32 each, and the angle's own
    for got, part in ((got_q, slice(0, hq)), (got_k, slice(hq, hq + hkv))):
        if got is not None:
            assert (np.abs(f64(got) - want[:, part]) <= off[:, part] + 2.0 ** -8 * np.abs(want[:, part]) + 1e-30).all()
    gk, gv = tree.read_back(kids, [3 * i for i in range(len(kids))])
    assert_held(f64(gk), want[:, hq:hq + hkv], off[:, hq:hq + hkv], "k")
    assert same(gv, quantised(f64(x[:, hq + hkv:]), "v"))
    tree.close()


@pytest.mark.gpu
def test_other_tokens_stay():
    """An append touches its own slots and the rest of pages it starts: tokens before it, other heads and nodes keep their bytes."""
    tree = new_tree((4, 2, 64), pages=12)
    (root,) = tree.fork(-1, 1)
    a, b = tree.fork(root, 2)
    k, v = random((30, 2, 64), 6).cuda(), random((30, 2, 64), 7).cuda()
    tree.append_step(a, k[:5], v[:5], quantize=True)
    tree.append_step(b, k[5:12], v[5:12], quantize=True)
    kept = tree.k_pool.clone(), tree.v_pool.clone()
    tree.append_step(a, k[12:14], v[12:14], quantize=True)
    page = tree.path_pages(a)[0][0]
    tile = 2 * 272
    for pool, old in zip((tree.k_pool, tree.v_pool), kept):
        changed = (pool != old).nonzero()[:, 0].cpu().numpy()
        assert len(changed) and (changed // (2 * tile) == page).all()
        # two tokens of two heads: 32 bytes of codes and 2 exponents each
        assert len(changed) <= 2 * 2 * 34
    gk, gv = tree.read_back([a, b])
    rows = torch.cat([k[:5], k[12:14], k[5:12]]), torch.cat([v[:5], v[12:14], v[5:12]])
    assert same(gk, quantised(f64(rows[0]), "k")) and same(gv, quantised(f64(rows[1]), "v"))
    tree.close()


@pytest.mark.gpu
def test_read_back_into_given_tensors():
    tree = new_tree()
    (root,) = tree.fork(-1, 1)
    k, v = random((33, 2, 64), 8), random((33, 2, 64), 9)
    tree.append_step(root, k.cuda(), v.cuda(), quantize=True)
    room = torch.full((2, 31 * 128 + 9), 7.0, dtype=torch.bfloat16, device="cuda")
    ko, vo = (room[i, 1:1 + 31 * 128].view(31, 2, 64) for i in range(2))  # two bytes off a boundary
    got = binding.spex_tree_read_back(tree, [root], [2], None, ko, vo)
    assert got[0] is ko and same(ko, quantised(f64(k), "k")[2:]) and same(vo, quantised(f64(v), "v")[2:])
    assert (room[:, 0] == 7).all() and (room[:, 1 + 31 * 128:] == 7).all()
    empty = tree.read_back([root, root], [33, 4], [0, 0])
    assert empty[0].shape == (0, 2, 64)
    with pytest.raises(spex.SpexError):
        tree.read_back([root], [2], [32])
    tree.close()


@pytest.mark.gpu
def test_long_lists_and_streams():
    """Lists beyond the kernel arguments go through pinned memory: many calls in flight, on a stream of the caller's."""
    tree = new_tree((4, 2, 64), pages=6000)
    (root,) = tree.fork(-1, 1)
    kids = tree.fork(root, 40)
    stream = torch.cuda.Stream()
    k, v = random((40 * 600, 2, 64), 10).cuda(), random((40 * 600, 2, 64), 11).cuda()
    torch.cuda.synchronize()
    got = []
    with torch.cuda.stream(stream):
        for i, u in enumerate(kids):
            tree.append_step(u, k[i * 600:(i + 1) * 600], v[i * 600:(i + 1) * 600], quantize=True)
        for _ in range(70):
            got.append(tree.read_back(kids[:20] if _ % 2 else kids[20:]))
    stream.synchronize()
    wk, wv = quantised(f64(k), "k"), quantised(f64(v), "v")
    for i, (gk, gv) in enumerate(got):
        half = slice(0, 12000) if i % 2 else slice(12000, 24000)
        assert same(gk, wk[half]) and same(gv, wv[half])
    tree.close()
