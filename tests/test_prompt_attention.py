"""spex_prompt_attention: refusals on the CPU (nothing is launched), values on the GPU against the definition in 64 bits."""

import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2605_10195_amd as spex
from paper_2605_10195_amd import binding

OK, INVALID, UNSUPPORTED = 0, 1, 6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- refusals, on the CPU: every call ends before a launch -----------------------------------------
def call(lens, heads=(4, 2, 64), dtype=binding.BF16, strides=(0, 0, 0, 0), scale=0.125, pointers=(64, 64, 64, 64), n=None, cfg=True):
    la = np.asarray(lens, dtype=np.int32)
    c = binding.PromptConfig(*heads, dtype, *strides)
    return binding.lib.spex_prompt_attention(C.byref(c) if cfg else None, la.ctypes.data if lens is not None else None,
                                             len(la) if n is None else n, *pointers, None, scale, None)


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(lens=[3], cfg=False)), (INVALID, dict(lens=[3], n=-1)), (INVALID, dict(lens=[3, -1])),
    (INVALID, dict(lens=[3], heads=(5, 2, 64))), (INVALID, dict(lens=[3], heads=(4, 0, 64))), (INVALID, dict(lens=[3], heads=(256, 256, 64))),
    (INVALID, dict(lens=[3], heads=(4, 2, 0))), (INVALID, dict(lens=[3], heads=(4, 2, 257))),
    (INVALID, dict(lens=[3], scale=0.0)), (INVALID, dict(lens=[3], scale=-1.0)), (INVALID, dict(lens=[3], scale=float("nan"))),
    (INVALID, dict(lens=[3], scale=float("inf"))),
    (INVALID, dict(lens=[3], strides=(255, 0, 0, 0))), (INVALID, dict(lens=[3], strides=(0, 127, 0, 0))),
    (INVALID, dict(lens=[3], strides=(0, 0, -128, 0))), (INVALID, dict(lens=[3], strides=(0, 0, 0, 255))),
    (INVALID, dict(lens=[3], pointers=(None, 64, 64, 64))), (INVALID, dict(lens=[3], pointers=(64, None, 64, 64))),
    (INVALID, dict(lens=[3], pointers=(64, 64, None, 64))), (INVALID, dict(lens=[3], pointers=(64, 64, 64, None))),
    (UNSUPPORTED, dict(lens=[3], dtype=binding.FP8_E4M3)), (UNSUPPORTED, dict(lens=[(1 << 24) + 1])),
    (UNSUPPORTED, dict(lens=[1 << 24] * 128)), (UNSUPPORTED, dict(lens=[3], strides=(1 << 31, 0, 0, 0))),
    (UNSUPPORTED, dict(lens=[1 << 24], heads=(4096, 1, 64))),
    (OK, dict(lens=[])), (OK, dict(lens=[0, 0])), (OK, dict(lens=[0], pointers=(None, None, None, None))),
])
def test_arguments_are_checked_before_anything_is_launched(want, kw):
    assert call(**kw) == want


def test_binding_refuses_tensors_that_it_cannot_describe():
    q, k = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):                   # not on a GPU
        spex.prompt_attention([3], q, k, k, 0.125)
    for bad in (dict(lens=[2], q=q, k=k, v=k), dict(lens=[3], q=q, k=k.float(), v=k), dict(lens=[3], q=q, k=k, v=k[:2]),
                dict(lens=[3], q=q[:1].expand(3, 4, 64), k=k, v=k), dict(lens=[3], q=q, k=k.transpose(1, 2), v=k),
                dict(lens=[3], q=q.half(), k=k.half(), v=k.half())):
        with pytest.raises(AssertionError):
            spex.prompt_attention(bad["lens"], bad["q"], bad["k"], bad["v"], 0.125)


# ---- values --------------------------------------------------------------------------------------
def inputs(lens, heads, dtype, seed=0, fused=False, shift=0, spread=2.0):
    hq, hkv, d = heads
    t = sum(lens)
    g = torch.Generator(device="cuda").manual_seed(seed)
    if fused:
        x = torch.randn((t, hq + 2 * hkv, d), generator=g, device="cuda")
        x[:, :hq] *= spread
        x = x.to(TYPES[dtype])
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]

    def one(h, mult):
        x = (torch.randn((t * h * d + shift,), generator=g, device="cuda") * mult).to(TYPES[dtype])
        return x[shift:].view(t, h, d)
    return one(hq, spread), one(hkv, 1.0), one(hkv, 1.0)


def reference(lens, q, k, v, scale):
    """out, lse, the weighted mean of |v|, the largest |score| and the largest sum |q_d k_d| * scale of every row, in 64 bits."""
    hq, hkv = q.shape[1], k.shape[1]
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    outs, at = [], 0
    for n in (x for x in lens if x):
        qs, ks, vs = (x[at:at + n].transpose(0, 1) for x in (q, k, v))
        ks, vs = ks.repeat_interleave(hq // hkv, 0), vs.repeat_interleave(hq // hkv, 0)
        x = scale * (qs @ ks.transpose(1, 2)).masked_fill(torch.ones(n, n).triu(1).bool(), -torch.inf)
        lse = torch.logsumexp(x, -1)
        w = torch.exp(x - lse[..., None])
        top = torch.where(torch.isinf(x), torch.zeros(()).double(), x.abs()).amax(-1)
        sums = scale * (qs.abs() @ ks.abs().transpose(1, 2)).amax(-1)
        outs.append([(w @ vs).transpose(0, 1), lse.t(), (w @ vs.abs()).transpose(0, 1), top.t(), sums.t()])
        at += n
    return [torch.cat(z).numpy() for z in zip(*outs)]


def check(lens, q, k, v, out, lse, scale):
    """Error bounds by counting roundings (half a step: bf16 2^-8, fp32 2^-24).
    A score: a sum of D products in fp32, off by at most D 2^-24 sum|q_d k_d|; scale, log2(e) and the difference to the
    reference point round it a few times more, 4 * 2^-24 of |score| + 8 (the slack of the reference point, in log2).
    A weight 2^x: that error times ln 2 each way, relative, plus 2 steps of the exponential; so out is off by at most twice
    that (numerator and denominator) plus n 2^-24 for each of the two sums, of the weighted mean of |v|.
    bf16: every weight is rounded once more by 2^-8, and the result."""
    ref, ref_lse, mean, top, sums = reference(lens, q, k, v, scale)
    d, n = q.shape[2], max(lens)
    score = (d + 2) * 2.0 ** -24 * sums + 4 * 2.0 ** -24 * (1.45 * top + 24)
    rel = 2 * (score + 4 * 2.0 ** -24 + n * 2.0 ** -24)
    got = out.double().cpu().numpy()
    assert np.all(np.isfinite(got))
    half = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24
    bound = rel[..., None] * mean + half * np.abs(ref) * 1.01 + (half * mean * 1.01 if out.dtype == torch.bfloat16 else 2 * half * mean)
    worst = float(np.max(np.abs(got - ref) / bound))
    assert worst <= 1.0, worst
    if lse is not None:
        off = np.abs(lse.double().cpu().numpy() - ref_lse) / (score + (n + 4) * 2.0 ** -24 + 4 * 2.0 ** -24 * (np.abs(ref_lse) + 8))
        assert float(np.max(off)) <= 1.0, float(np.max(off))


HEADS = [(8, 2, 64), (8, 8, 128), (7, 1, 128), (10, 2, 96), (4, 1, 256), (6, 3, 40), (32, 4, 128), (4, 2, 192), (2, 1, 8)]
LENS = [[1], [2, 1], [31, 32, 33], [64], [65, 0, 63, 1], [130, 7], [300]]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_against_the_definition(dtype, heads, lens):
    q, k, v = inputs(lens, heads, dtype, seed=len(lens) + heads[2])
    out, lse = spex.prompt_attention(lens, q, k, v, heads[2] ** -0.5)
    check(lens, q, k, v, out, lse, heads[2] ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,heads", [([700, 129, 511], (16, 4, 128)), ([1025], (4, 1, 64)), ([1500], (2, 2, 256)), ([640, 640], (5, 1, 96))], ids=str)
@pytest.mark.parametrize("fused", [False, True])
def test_longer_prompts(dtype, lens, heads, fused):
    q, k, v = inputs(lens, heads, dtype, seed=3, fused=fused)
    out, lse = spex.prompt_attention(lens, q, k, v, heads[2] ** -0.5)
    check(lens, q, k, v, out, lse, heads[2] ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,shift", [((4, 2, 64), 1), ((4, 2, 7), 0), ((3, 1, 130), 0), ((2, 2, 1), 0), ((4, 1, 250), 3)], ids=str)
def test_rows_that_are_not_made_of_16_byte_pieces(dtype, heads, shift):
    lens = [70, 1, 33]
    q, k, v = inputs(lens, heads, dtype, seed=5, shift=shift)
    out, lse = spex.prompt_attention(lens, q, k, v, heads[2] ** -0.5)
    check(lens, q, k, v, out, lse, heads[2] ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_only_the_prompts_rows_are_written_and_strides_are_kept(dtype):
    """out and the inputs are windows of larger tensors; everything around the windows stays as it was, and q, k and v around them
    hold NaN, which nothing may read into a result."""
    lens, (hq, hkv, d) = [37, 5, 64], (4, 2, 64)
    t = sum(lens)
    want = [torch.full((t + 70, h + 2, d), float("nan"), dtype=TYPES[dtype], device="cuda") for h in (hq, hkv, hkv)]
    views = [x[3:3 + t, 1:1 + h] for x, h in zip(want, (hq, hkv, hkv))]
    for view, x in zip(views, inputs(lens, (hq, hkv, d), dtype, seed=6)):
        view.copy_(x)
    big = torch.full((t + 70, hq + 2, d), 9.0, dtype=TYPES[dtype], device="cuda")
    lse = torch.full((t + 3, hq), 9.0, device="cuda")
    spex.prompt_attention(lens, *views, 0.125, out=big[3:3 + t, 1:1 + hq], lse=lse[:t])
    check(lens, *views, big[3:3 + t, 1:1 + hq], lse[:t], 0.125)
    big[3:3 + t, 1:1 + hq] = 9.0
    assert bool((big == 9.0).all()) and bool((lse[t:] == 9.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("n", [127, 128, 129, 300])
def test_many_prompts_take_several_launches(n):
    lens = [(i * 7) % 23 for i in range(n)]
    q, k, v = inputs(lens, (4, 2, 64), "bf16", seed=n)
    out, lse = spex.prompt_attention(lens, q, k, v, 0.125)
    check(lens, q, k, v, out, lse, 0.125)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["rising", "falling", "far", "flat", "huge"])
def test_scores_that_move_the_running_maximum(dtype, what):
    """Keys whose scores rise along the prompt (the maximum moves in every tile), fall, lie far below or above zero, are all equal,
    or spread so far that one key takes all the weight."""
    lens, (hq, hkv, d) = [400], (4, 2, 64)
    q, k, v = (x.float() for x in inputs(lens, (hq, hkv, d), dtype, seed=8, spread=1.0))
    if what == "flat":
        k.zero_()
    else:
        q[..., 0] = 8.0
        pos = torch.arange(400, device="cuda")[:, None].float()
        k[..., 0] += {"rising": pos * 0.25, "falling": -pos * 0.25, "far": torch.full_like(pos, -200.0), "huge": 50.0 * (pos % 7)}[what]
    q, k, v = (x.to(TYPES[dtype]) for x in (q, k, v))
    out, lse = spex.prompt_attention(lens, q, k, v, 0.5)
    check(lens, q, k, v, out, lse, 0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_replayed_and_on_another_stream(dtype):
    lens = [200, 31, 90]
    q, k, v = inputs(lens, (8, 2, 128), dtype, seed=9)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        spex.prompt_attention(lens, q, k, v, 0.1, out=out, lse=lse)
    torch.cuda.current_stream().wait_stream(side)
    check(lens, q, k, v, out, lse, 0.1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spex.prompt_attention(lens, q, k, v, 0.1, out=out, lse=lse)
    for seed in (10, 11, 12):
        for x, y in zip((q, k, v), inputs(lens, (8, 2, 128), dtype, seed=seed)):
            x.copy_(y)
        graph.replay()
        eager, eager_lse = spex.prompt_attention(lens, q, k, v, 0.1)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(lse, eager_lse)
        check(lens, q, k, v, out, lse, 0.1)


@pytest.mark.gpu
def test_same_result_every_time_and_without_lse():
    lens = [513, 70]
    q, k, v = inputs(lens, (8, 2, 128), "bf16", seed=13)
    first, lse = spex.prompt_attention(lens, q, k, v, 0.1)
    for _ in range(3):
        again, none = spex.prompt_attention(lens, q, k, v, 0.1, want_lse=False)
        assert none is None and torch.equal(first, again)


@pytest.mark.gpu
def test_equals_decode_attention_over_the_appended_prompt():
    """The same prompt through the page pool: both are within their bounds of the definition, hence of each other."""
    lens, (hq, hkv, d) = [150, 64], (8, 2, 128)
    q, k, v = inputs(lens, (hq, hkv, d), "bf16", seed=14)
    out, lse = spex.prompt_attention(lens, q, k, v, d ** -0.5)
    tree = spex.SpexTree(hq, hkv, d, num_pages=20, device="cuda")
    roots, at = tree.fork(-1, 2), 0
    for u, n in zip(roots, lens):
        tree.append_step(u, k[at:at + n].contiguous(), v[at:at + n].contiguous())
        at += n
    ref, ref_lse = tree.decode_attention(roots, lens, q, d ** -0.5)
    # 2^-8 of the weighted mean of |v| and of the result (here), 2e-3 (there)
    bound = 2.0 ** -8 * 1.01 * (torch.as_tensor(reference(lens, q, k, v, d ** -0.5)[2], device="cuda") + ref.abs().double()) + 2e-3
    assert bool(((out.double() - ref.double()).abs() <= bound).all()) and float((lse - ref_lse).abs().max()) <= 2e-3
    tree.close()


@pytest.mark.parametrize("scale,want", [(1e-38, True), (1e37, True), (1e-42, False), (3e38, False)])
def test_scales_whose_reciprocal_fp32_does_not_hold(scale, want):
    assert call([0], scale=scale) == (0 if want else INVALID)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-38, 1e4])
def test_scales_at_the_ends(dtype, scale):
    """Scores of about nothing (all weights equal) and of tens of thousands (one key takes all the weight)."""
    lens = [1, 40, 300]
    q, k, v = inputs(lens, (4, 2, 64), dtype, 31)
    out, lse = spex.prompt_attention(lens, q, k, v, scale)
    check(lens, q, k, v, out, lse, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(8, 2, 256), (8, 4, 224), (8, 2, 192), (8, 1, 160)], ids=str)
def test_wide_heads_with_rows_enough_for_whole_workgroups(heads):
    lens = [1100, 700, 333, 0, 1]
    q, k, v = inputs(lens, heads, "bf16", 32, fused=heads[1] == 2)
    out, lse = spex.prompt_attention(lens, q, k, v, heads[2] ** -0.5)
    check(lens, q, k, v, out, lse, heads[2] ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(128, 8, 128), (130, 2, 104)], ids=str)
def test_batches_of_many_row_sets(heads):
    """More than 6144 sets of 32 rows."""
    lens = [65, 1, 700, 257, 64, 33, 0, 500, 31, 96]
    q, k, v = inputs(lens, heads, "bf16", 33, fused=heads[1] == 8)
    assert heads[0] * sum(-(-n // 32) for n in lens) > 6144
    out, lse = spex.prompt_attention(lens, q, k, v, heads[2] ** -0.5)
    check(lens, q, k, v, out, lse, heads[2] ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,lens", [((8, 2, 128), [1024]), ((4, 2, 96), [2048]), ((2, 1, 64), [129, 7, 1700]), ((8, 2, 40), [255, 0, 257]), ((1, 1, 128), [289])], ids=str)
def test_few_rows_with_long_ways(dtype, heads, lens):
    """Row sets few enough to share each over eight wavefronts, or four (fp32 above 64 dims)."""
    q, k, v = inputs(lens, heads, dtype, 34)
    out, lse = spex.prompt_attention(lens, q, k, v, heads[2] ** -0.5)
    check(lens, q, k, v, out, lse, heads[2] ** -0.5)


# ---- every kernel by name ----------------------------------------------------------------------
# Kernels that spex_prompt_form tells apart, and heads whose calls with a prompt of some 400 tokens take them.
ANY, WHOLE, SHORT_TILES, FOUR, EIGHT = range(5)
KERNELS = [("bf16", (96, 2, 64), WHOLE), ("bf16", (60, 3, 96), WHOLE), ("bf16", (64, 4, 128), WHOLE), ("bf16", (480, 2, 128), SHORT_TILES),
           ("bf16", (40, 4, 192), SHORT_TILES), ("bf16", (40, 2, 256), SHORT_TILES), ("f32", (96, 2, 64), WHOLE), ("f32", (60, 3, 128), WHOLE),
           ("f32", (4, 2, 256), WHOLE), ("bf16", (64, 2, 64), FOUR), ("bf16", (24, 2, 96), FOUR), ("bf16", (24, 4, 128), FOUR),
           ("bf16", (16, 2, 192), FOUR), ("bf16", (8, 2, 256), FOUR), ("f32", (32, 2, 64), FOUR), ("f32", (8, 1, 128), FOUR),
           ("bf16", (16, 2, 64), EIGHT), ("bf16", (4, 2, 96), EIGHT), ("bf16", (4, 2, 128), EIGHT), ("f32", (4, 2, 64), EIGHT)]
ODD = [("bf16", (4, 2, 7), ANY), ("f32", (4, 2, 7), ANY)]
NAMES = [f"{d}-{h[0]}x{h[2]}" for d, h, _ in KERNELS]
SHARING = [x for x in KERNELS if x[2] in (WHOLE, SHORT_TILES)]
MIXED = [65, 0, 400, 1, 290, 32]


def form(lens, heads, dtype, strides=(0, 0, 0, 0), pointers=(64, 64, 64, 64), out=True):
    la, got = np.asarray(lens, dtype=np.int32), C.c_int32(-7)
    c = binding.PromptConfig(*heads, {"bf16": binding.BF16, "f32": binding.F32}[dtype], *strides)
    st = binding.lib.spex_prompt_form(C.byref(c), la.ctypes.data, len(la), *pointers, C.byref(got) if out else None)
    return got.value if st == OK else ("error", st)


@pytest.mark.parametrize("dtype,heads,kernel", KERNELS + ODD, ids=NAMES + ["bf16-any", "f32-any"])
def test_the_kernel_that_each_case_is_for(dtype, heads, kernel):
    """A changed rule that empties one of the tests below of the kernel it is for fails here."""
    for n in (385, 400, 401, 415, 447):
        assert form([n], heads, dtype) == kernel, n
    if kernel in (WHOLE, SHORT_TILES):
        assert form(MIXED, heads, dtype) == kernel


def test_forms_of_other_calls():
    assert form([], (4, 2, 64), "bf16") == form([0, 0], (4, 2, 64), "bf16", pointers=(None,) * 4) == -1
    assert form([3], (4, 2, 64), "bf16") == FOUR and form([3], (4, 2, 64), "bf16", pointers=(64, 66, 64, 64)) == ANY
    assert form([3], (4, 2, 64), "f32", strides=(0, 0, 129, 0)) == ANY
    assert form([3], (4, 2, 64), "bf16", pointers=(64, None, 64, 64)) == form([-3], (4, 2, 64), "bf16") == ("error", INVALID)
    assert form([3], (4, 2, 64), "bf16", strides=(1 << 31, 0, 0, 0)) == ("error", UNSUPPORTED)
    assert form([3], (4, 2, 64), "bf16", out=False) == ("error", INVALID)


def check_some_heads(lens, q, k, v, out, lse, scale):
    """`check` on the first, the middle and the last query head of every kv head."""
    hkv, g = k.shape[1], q.shape[1] // k.shape[1]
    rows = torch.tensor([kv * g + i for kv in range(hkv) for i in (0, g // 2, g - 1)], device=q.device)
    check(lens, q[:, rows], k, v, out[:, rows], lse[:, rows], scale)


@pytest.mark.gpu
@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("dtype,heads,kernel", SHARING, ids=NAMES[:len(SHARING)])
def test_tiles_shared_by_wavefronts_against_the_definition(dtype, heads, kernel, fused):
    q, k, v = inputs(MIXED, heads, dtype, seed=51, fused=fused)
    out, lse = spex.prompt_attention(MIXED, q, k, v, heads[2] ** -0.5)
    check_some_heads(MIXED, q, k, v, out, lse, heads[2] ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["rising", "falling", "far", "flat", "huge"])
@pytest.mark.parametrize("dtype,heads,kernel", KERNELS, ids=NAMES)
def test_running_maximum_of_each_kernel(dtype, heads, kernel, what):
    """As test_scores_that_move_the_running_maximum."""
    q, k, v = (x.float() for x in inputs([400], heads, dtype, seed=52, spread=1.0))
    if what == "flat":
        k.zero_()
    else:
        q[..., 0] = 8.0
        pos = torch.arange(400, device="cuda")[:, None].float()
        k[..., 0] += {"rising": pos * 0.25, "falling": -pos * 0.25, "far": torch.full_like(pos, -200.0), "huge": 50.0 * (pos % 7)}[what]
    q, k, v = (x.to(TYPES[dtype]) for x in (q, k, v))
    out, lse = spex.prompt_attention([400], q, k, v, 0.5)
    check_some_heads([400], q, k, v, out, lse, 0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [1e-38, 1e4])
@pytest.mark.parametrize("dtype,heads,kernel", SHARING, ids=NAMES[:len(SHARING)])
def test_scales_at_the_ends_of_shared_tiles(dtype, heads, kernel, scale):
    q, k, v = inputs(MIXED, heads, dtype, 53)
    out, lse = spex.prompt_attention(MIXED, q, k, v, scale)
    check_some_heads(MIXED, q, k, v, out, lse, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,heads,kernel", SHARING, ids=NAMES[:len(SHARING)])
def test_windows_captured_and_replayed_with_shared_tiles(dtype, heads, kernel):
    """out and lse are windows of larger tensors, whose other rows stay; the launch is recorded and replayed on new inputs."""
    (hq, hkv, d), t = heads, sum(MIXED)
    big, lse = torch.full((t + 7, hq + 2, d), 9.0, dtype=TYPES[dtype], device="cuda"), torch.full((t + 3, hq), 9.0, device="cuda")
    out = big[3:3 + t, 1:1 + hq]
    qkv = inputs(MIXED, heads, dtype, seed=54, fused=True)
    spex.prompt_attention(MIXED, *qkv, 0.1, out=out, lse=lse[:t])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spex.prompt_attention(MIXED, *qkv, 0.1, out=out, lse=lse[:t])
    for seed in (55, 56, 57):
        for x, y in zip(qkv, inputs(MIXED, heads, dtype, seed=seed)):
            x.copy_(y)
        graph.replay()
        eager, eager_lse = spex.prompt_attention(MIXED, *qkv, 0.1)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(lse[:t], eager_lse)
    check_some_heads(MIXED, *qkv, out, lse[:t], 0.1)
    out.fill_(9.0)
    assert bool((big == 9.0).all()) and bool((lse[t:] == 9.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("n", [385, 401, 415, 447])
@pytest.mark.parametrize("dtype,heads,kernel", KERNELS, ids=NAMES)
def test_nothing_behind_a_prompt_is_read(dtype, heads, kernel, n):
    """q, k and v are windows with NaN around them, and the prompt ends 1, 17, 31 and 63 keys into a tile."""
    (hq, hkv, d), big = heads, []
    for x, h in zip(inputs([n], heads, dtype, seed=n), (hq, hkv, hkv)):
        y = torch.full((n + 140, h, d), float("nan"), dtype=x.dtype, device="cuda")
        y[70:70 + n] = x
        big.append(y[70:70 + n])
    out, lse = spex.prompt_attention([n], *big, d ** -0.5)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    dense, dense_lse = spex.prompt_attention([n], *(x.clone() for x in big), d ** -0.5)
    assert torch.equal(out, dense) and torch.equal(lse, dense_lse)


def of_scores(levels, heads, dtype, seed):
    """q, k, v of one prompt whose scores are exact: query t, head h and key s have levels[0][t % .., h % ..] * levels[1][s]."""
    (hq, hkv, d), n = heads, len(levels[1])
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k = torch.zeros((n, hq, d), device="cuda"), torch.zeros((n, hkv, d), device="cuda")
    rows = torch.as_tensor(levels[0], dtype=torch.float64)
    q[..., 0] = rows[torch.arange(n)[:, None] % rows.shape[0], torch.arange(hq)[None] % rows.shape[1]].float().cuda()
    k[..., 0] = torch.as_tensor(levels[1], dtype=torch.float64).float().cuda()[:, None]
    v = torch.randn((n, hkv, d), generator=g, device="cuda")
    return [x.to(TYPES[dtype]) for x in (q, k, v)]


N = 400
LEVELS = {
    "flat": ([[1.0, 3e4, 1e10, 1e25]], [1.1875] * N),
    "steps": ([[2.0 ** 31, -2.0 ** 34, 2.0 ** 60]], [1.0 + (s * 5 % 7) / 64 for s in range(N)]),
    "climb": ([[1.0, 1e-3, 1e3]], [np.sign(s - 200) * 2.0 ** (abs(s - 200) / 200 * 90) for s in range(N)]),
    "fall": ([[1.0, 1e-3, 1e3]], [np.sign(200 - s) * 2.0 ** (abs(s - 200) / 200 * 90) for s in range(N)]),
    "ends": ([[8.8e29, -8.8e29, 6.9e29, -7.1e29]], [1.0 + (s % 3) / 128 for s in range(N)]),
    "border": ([[2.0 ** 23, 2.0 ** 24, -2.0 ** 24, 2.0 ** 25, -2.0 ** 23]], [1.0 + (s * 3 % 11) / 128 for s in range(N)]),
    "fine": ([[2.0 ** 22, -2.0 ** 24, 2.0 ** 25, 2.0 ** 30]], [1.0 + (s * 3 % 5) * 2.0 ** -23 for s in range(N)]),
    # the keys of one wavefront of a split launch far below zero, of others near, or near the border of the two
    "states": ([[1.0], [2.0 ** -2]], [[-2.0 ** 40, -2.0 ** 24 - 64, -2.0 ** 24 + 130, (s % 5) * 1.5, 2.0 ** 24 - 60, 2.0 ** 24 + 32, 2.0 ** 27][s // 32 % 7] * (1 if s < 300 else -1) for s in range(N)]),
    "mixed": ([[1.0, 2.0 ** 33], [-2.0 ** 80, 0.25], [2.0 ** 24, -2.0 ** 24], [0.0, 2.0 ** 10]], [(s * 7 % 13 - 6) / 8 for s in range(N)]),
}


@pytest.mark.gpu
@pytest.mark.parametrize("what,scale", [(what, scale) for what in LEVELS for scale in (1.0, 0.09) if (what, scale) != ("ends", 0.09)])
@pytest.mark.parametrize("dtype,heads,kernel", KERNELS + ODD, ids=NAMES + ["bf16-any", "f32-any"])
def test_scores_far_from_zero(dtype, heads, kernel, scale, what):
    """Scores up to the documented ends, times the scale +-1e30.  They are exact in fp32, so the definition in 64 bits knows the weights: keys
    of the largest score share a row between them, and only keys within 150 / log2(e) of it count ("ends": those of scale 1).  A weight's exponent is a difference of
    scores times the scale, rounded three times and the scale twice (5 * 2^-24 of at most 150), its power off by 2 steps; then as `check`."""
    scale = float(np.float32(scale))
    q, k, v = of_scores(LEVELS[what], heads, dtype, 41)
    out, lse = spex.prompt_attention([N], q, k, v, scale)
    hq, hkv, d = heads
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    rel = 2 * (5 * 2.0 ** -24 * 150 * 0.7 + 4 * 2.0 ** -24 + N * 2.0 ** -24)
    future = torch.ones(N, N, device="cuda").triu(1).bool()
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    for h in range(hq):
        kv = h * hkv // hq
        x = (q[:, h, 0].double()[:, None] * k[:, kv, 0].double()[None] * scale).masked_fill(future, -torch.inf)
        top = x.amax(-1, keepdim=True)
        w = torch.exp(x - top)
        total = w.sum(-1, keepdim=True)
        ref, mean = (w @ v[:, kv].double()) / total, (w @ v[:, kv].double().abs()) / total
        bound = rel * mean + half * ref.abs() * 1.01 + half * mean * (1.01 if dtype == "bf16" else 2)
        worst = float(((out[:, h].double() - ref).abs() / bound).max())
        assert worst <= 1.0, (h, worst)
        ref_lse = (top + torch.log(total))[:, 0]
        off = (lse[:, h].double() - ref_lse).abs() / (8 * 2.0 ** -24 * (ref_lse.abs() + 200) + (N + 4) * 2.0 ** -24)
        assert float(off.max()) <= 1.0, (h, float(off.max()))


# ---- launches ------------------------------------------------------------------------------------
def test_lists_of_the_launches_under_sanitizers(tmp_path):
    """Every row set exactly once, however many launches prompts and heads take."""
    include = "/opt/rocm/include"
    if shutil.which("g++") is None or not os.path.exists(os.path.join(include, "hip", "hip_runtime.h")):
        pytest.skip("needs g++ and the HIP headers")
    here = os.path.dirname(os.path.abspath(__file__))
    exe = str(tmp_path / "prompt_lists")
    build = subprocess.run(
        ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-static-libasan", "-static-libubsan",
         "-D__HIP_PLATFORM_AMD__", "-I" + include, "-D__align__(n)=__attribute__((aligned(n)))", os.path.join(here, "prompt_lists.cpp"),
         os.path.join(here, "..", "paper_2605_10195_amd", "csrc", "prompt.cpp"), "-o", exe], capture_output=True, text=True)
    if build.returncode != 0 and "cannot find" in build.stderr and any(w in build.stderr for w in ("asan", "ubsan", "sanitize")):
        pytest.skip("the sanitizer runtime is not installed")
    assert build.returncode == 0, build.stderr[-2000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert run.returncode == 0 and run.stdout == "ok\n", (run.stdout[-2000:], run.stderr[-4000:])


def test_most_row_sets_of_a_prompt():
    assert form([1 << 24], (4095, 1, 1), "bf16") == ANY and form([1 << 24], (4096, 1, 1), "bf16") == ("error", UNSUPPORTED)
    assert form([1 << 24], (1 << 20, 1 << 6, 1), "bf16") == ("error", UNSUPPORTED)


@pytest.mark.gpu
def test_a_prompt_that_takes_several_launches():
    """8.4 million query heads: two prompts in four launches.  Values are the same for all tokens of a kv head, which is then what every row
    returns; the first row's score is its log-sum-exp."""
    lens, (hq, hkv) = [40, 3], (255 * 33000, 255)
    g = torch.Generator(device="cuda").manual_seed(61)
    q = torch.randn((43, hq, 1), generator=g, device="cuda").bfloat16()
    k = torch.randn((43, hkv, 1), generator=g, device="cuda").bfloat16()
    v = (1 + torch.arange(hkv, device="cuda") / 64).bfloat16()[None, :, None].expand(43, hkv, 1).contiguous()
    out, lse = torch.full_like(q, float("nan")), torch.full((43, hq), float("nan"), device="cuda")
    spex.prompt_attention(lens, q, k, v, 1.0, out=out, lse=lse)
    # the mean is off by 2 * 41 roundings of fp32, 5e-6 of the value, far less than the 2^-9 to the next number that rounds elsewhere
    assert torch.equal(out, v.repeat_interleave(hq // hkv, 1))
    for row in (0, 40):
        score = q[row, :, 0].float() * k[row].repeat_interleave(hq // hkv, 0)[:, 0].float()
        # two products with log2(e) and ln 2 and their constants, relative 4 * 2^-24
        assert bool(((lse[row] - score).abs() <= 4 * 2.0 ** -24 * score.abs()).all())
    heads = torch.randint(0, hq, (300,), generator=g, device="cuda").sort().values
    cols = torch.cat([heads, torch.tensor([0, hq - 1], device="cuda")])
    kh, at = k[:, cols * hkv // hq, 0].double(), 0
    for n in lens:
        x = (q[at:at + n, cols, 0].double()[:, None] * kh[at:at + n][None]).masked_fill(torch.ones(n, n, device="cuda").triu(1).bool()[..., None], -torch.inf)
        ref = torch.logsumexp(x, 1)
        # scores are below 32 and off by 4 * 2^-24 of that, sums by n and the logarithm by a few steps more
        assert float((lse[at:at + n, cols].double() - ref).abs().max()) <= (4 * 32 + n + 32 * 4) * 2.0 ** -24
        assert float(x[x > -1e9].abs().max()) < 32
        at += n
