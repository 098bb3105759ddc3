"""The norm of many gradients together and their clipping (GradList, grad_norm, clip_grad_norm) against plain numpy in 64 bits.

Tolerances.  The kernels sum squares in fp64: relative error below (terms) * 2^-53, at most 2^-28 here; the norm is
rounded once to fp32: 2^-24 of it.  Outputs: the factor rounds once to fp32 and the product once more, 2 * 2^-24 of the value
(2^-149 where that is denormal); to bf16 (8 significant bits) another 2^-8."""
import math

import numpy as np
import pytest

import paper_1909_05073_amd as P

from gpu_util import say

U = 2.0 ** -24


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64).ravel()


def plain(grads, max_norm, eps=1e-6):
    norm = math.sqrt(math.fsum(float(np.dot(g, g)) for g in grads))
    return norm, [g * min(1.0, max_norm / (norm + eps)) for g in grads]


def check(norm, outs, want_norm, want):
    import torch
    assert norm.dtype == torch.float32 and norm.dim() == 0
    assert abs(float(norm) - want_norm) <= 1.01 * U * want_norm, (float(norm), want_norm)
    for i, (o, w) in enumerate(zip(outs, want)):
        tol = 2.02 * U * np.abs(w) + 2.0 ** -149
        if o.dtype == torch.bfloat16:
            tol = tol * 1.01 + 2.0 ** -8 * np.abs(w) * 1.01 + 2.0 ** -133
        err = np.abs(host(o) - w)
        assert (err <= tol).all(), f"tensor {i}: {err.max()} at {err.argmax()} of {w.size}"


def make(rng, sizes, types, scale=1.0):
    import torch
    return [torch.from_numpy((rng.standard_normal(n) * scale * np.exp(rng.uniform(-2, 2))).astype(np.float32)).cuda()
            .to(torch.bfloat16 if t == "bf16" else torch.float32) for n, t in zip(sizes, types)]


LISTS = {"one": [1], "few": [3, 1, 2], "chunk_ends": [16383, 16384, 16385, 32768, 32769, 4], "layer": [16 * 16 * 9, 16],
         "empty_ones": [0, 5, 0, 0, 70000, 0], "long": [3_000_001, 17, 250_000], "many": [(i * 37) % 91 for i in range(500)],
         "table_full": [10] * 160, "table_over": [10] * 161, "many_long": [20000 + i for i in range(330)], "small_edge": [32768], "small_over": [32769],
         "nothing": [0, 0]}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_norm_and_clipping_against_the_formula(name, dtype):
    import torch
    sizes = LISTS[name]
    say(f"[case] clip {name} {dtype}: {len(sizes)} tensors, {sum(sizes)} elements")
    rng = np.random.default_rng(len(sizes) + sum(sizes))
    types = [("f32", "bf16")[i % 2] if dtype == "mixed" else dtype for i in range(len(sizes))]
    grads = make(rng, sizes, types)
    values = [host(g) for g in grads]
    full, _ = plain(values, 1.0)
    for max_norm in (0.3 * full, 2 * full, 0.0, math.inf):
        want_norm, want = plain(values, float(np.float32(max_norm)))
        for out_type in ("same", torch.float32, torch.bfloat16):
            outs = [torch.full_like(g, float("nan"), dtype=g.dtype if out_type == "same" else out_type) for g in grads]
            norm = P.clip_grad_norm(grads, max_norm, out=outs)
            check(norm, outs, want_norm, want)
        mine = [g.clone() for g in grads]
        norm = P.clip_grad_norm(mine, max_norm)
        check(norm, mine, want_norm, want)
        if max_norm > full:
            assert all(torch.equal(a, b) for a, b in zip(mine, grads)), "gradients below the limit were changed"
    assert float(P.grad_norm(grads)) == float(norm)


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [1, 2, 3, 5])
def test_tensors_that_begin_anywhere(offset):
    import torch
    say(f"[case] clip offset={offset}")
    rng = np.random.default_rng(offset)
    for dtype in (torch.float32, torch.bfloat16):
        flat = torch.from_numpy(rng.standard_normal(100_000).astype(np.float32)).cuda().to(dtype)
        out = torch.full((100_100,), 7.0, dtype=dtype, device="cuda")
        cuts, at = [], offset
        for n in (1, 7, 40_003, 129, 30_000):
            cuts.append((at, n)); at += n + offset
        grads = [flat[a:a + n] for a, n in cuts]
        outs = [out[a + 3:a + 3 + n] for a, n in cuts]
        want_norm, want = plain([host(g) for g in grads], 1.0)
        check(P.clip_grad_norm(grads, 1.0, out=outs), outs, want_norm, want)
        for a, n in cuts:
            out[a + 3:a + 3 + n] = 7.0
        assert bool((out == 7.0).all()), "elements between the tensors were written"


@pytest.mark.gpu
def test_large_small_and_odd_values():
    import torch
    say("[case] clip odd values")
    rng = np.random.default_rng(0)
    big = make(rng, [5000, 70_000], ["f32", "f32"], 1e30)             # squares beyond fp32
    values = [host(g) for g in big]
    norm, want = plain(values, 2.0)
    outs = [torch.empty_like(g) for g in big]
    check(P.clip_grad_norm(big, 2.0, out=outs), outs, norm, want)
    small = make(rng, [5000, 9], ["f32", "f32"], 1e-30)               # squares below fp32
    values = [host(g) for g in small]
    norm, want = plain(values, 1e-30, 0.0)
    outs = [torch.empty_like(g) for g in small]
    check(P.clip_grad_norm(small, 1e-30, 0.0, out=outs), outs, float(np.float32(norm)), plain(values, float(np.float32(1e-30)), 0.0)[1])
    huge = [torch.full((2_000_000,), 3e38, device="cuda")]            # the norm is no fp32 number, the factor is
    norm = P.clip_grad_norm(huge, 1.0)
    assert math.isinf(float(norm)) and abs(float(huge[0][77]) * math.sqrt(2e6) - 1) < 1e-6
    for size in (100, 200_000):
        g = [torch.ones(size, device="cuda"), torch.ones(5, device="cuda")]
        g[0][size // 2] = float("nan")
        assert math.isnan(float(P.clip_grad_norm(g, 1.0))) and bool(torch.isnan(g[0]).all()) and bool(torch.isnan(g[1]).all())
        g = [torch.ones(size, device="cuda"), torch.ones(5, device="cuda")]
        g[0][size // 2] = float("-inf")
        assert math.isinf(float(P.clip_grad_norm(g, 1.0))) and bool((g[1] == 0).all()) and int(torch.isnan(g[0]).sum()) == 1
    z = [torch.zeros(100, device="cuda")]
    assert float(P.clip_grad_norm(z, 1.0)) == 0 and bool((z[0] == 0).all())


@pytest.mark.gpu
def test_layouts_streams_and_equal_bits():
    import torch
    say("[case] clip layouts, streams")
    rng = np.random.default_rng(1)
    w = torch.from_numpy(rng.standard_normal((64, 32, 3, 3)).astype(np.float32)).cuda()
    grads = [w.to(memory_format=torch.channels_last), w[0, 0].t(), torch.from_numpy(rng.standard_normal(300_000).astype(np.float32)).cuda()]
    want_norm, want = plain([host(g.contiguous()) for g in grads], 5.0)
    outs = [torch.empty_like(g) for g in grads]
    norm = P.clip_grad_norm(grads, 5.0, out=outs)
    check(norm, [o.contiguous() for o in outs], want_norm, want)
    plan = P.GradList(grads, outs)
    first = [o.clone() for o in outs]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        big = torch.randn(3000, 3000, device="cuda")
        for _ in range(5):
            big = big @ big * 1e-3
        grads[2].mul_(2.0)
        half = plan.clip(10.0)
        grads[2].mul_(0.5)
        again = plan.clip(5.0)
        alone = plan.norm()
    s.synchronize()
    assert float(again) == float(norm) == float(alone) and float(half) > float(norm)
    assert all(torch.equal(a, b) for a, b in zip(first, outs))


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[2304, 16], [500_000, 16, 30_001], [50] * 170])
def test_replays_of_a_captured_step(sizes):
    import torch
    say(f"[case] clip captured {len(sizes)}")
    rng = np.random.default_rng(len(sizes))
    grads = make(rng, sizes, ["f32"] * len(sizes))
    outs = [torch.empty_like(g) for g in grads]
    plan = P.GradList(grads, outs)
    plan.clip(1.0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        norm = plan.clip(1.0)
    for i in range(4):
        for t in grads:
            t.mul_(1.7)
        for o in outs:
            o.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        eager = plan.clip(1.0)
        assert float(norm) == float(eager) and all(torch.equal(a, b) for a, b in zip(got, outs)), f"replay {i}"


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    import torch
    n = (1 << 32) + 40_000
    say(f"[case] clip {n} bf16 elements")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[5], g[1 << 31], g[n - 1] = 3.0, 4.0, 12.0
    norm = P.clip_grad_norm([g], 1.3)
    assert float(norm) == 13.0
    got = [float(g[5]), float(g[1 << 31]), float(g[n - 1])]
    for a, b in zip(got, (0.3, 0.4, 1.2)):
        assert abs(a - b) <= 2.0 ** -8 * b
    assert int((g != 0).sum()) == 3


# ---- refusals ------------------------------------------------------------------------------------------------------------

def test_c_entries_refuse_what_they_cannot_run():
    import ctypes as C
    p, need = 1 << 20, P.pconv_grad_workspace(2)
    ptrs = lambda *v: (C.c_void_p * len(v))(*v)
    i64, i32 = (lambda *v: (C.c_int64 * len(v))(*v)), (lambda *v: (C.c_int32 * len(v))(*v))
    two, n, f32 = ptrs(p, p + 4096), i64(4, 4), i32(0, 0)
    bad = {
        "null": [lambda: P.pconv_grad_norm(None, n, f32, 2, p, p, need), lambda: P.pconv_grad_norm(two, None, f32, 2, p, p, need),
                 lambda: P.pconv_grad_norm(two, n, None, 2, p, p, need), lambda: P.pconv_grad_norm(two, n, f32, 2, 0, p, need),
                 lambda: P.pconv_grad_norm(two, n, f32, 2, p, 0, need), lambda: P.pconv_grad_norm(ptrs(p, None), n, f32, 2, p, p, need),
                 lambda: P.pconv_clip_grads(two, None, n, f32, f32, 2, 1.0, 0.0, p, p, need),
                 lambda: P.pconv_clip_grads(two, two, n, f32, None, 2, 1.0, 0.0, p, p, need),
                 lambda: P.pconv_clip_grads(two, ptrs(p, None), n, f32, f32, 2, 1.0, 0.0, p, p, need)],
        "num": [lambda: P.pconv_grad_norm(two, n, f32, -1, p, p, need), lambda: P.pconv_grad_norm(two, n, f32, (1 << 24) + 1, p, p, 1 << 40)],
        "counts": [lambda: P.pconv_grad_norm(two, i64(4, -1), f32, 2, p, p, need),
                   lambda: P.pconv_grad_norm(two, i64(1 << 45, 1), f32, 2, p, p, need)],
        "dtype": [lambda: P.pconv_grad_norm(two, n, i32(0, 2), 2, p, p, need),
                  lambda: P.pconv_clip_grads(two, two, n, f32, i32(0, -1), 2, 1.0, 0.0, p, p, need)],
        "aligned": [lambda: P.pconv_grad_norm(ptrs(p, p + 4098), n, f32, 2, p, p, need),
                    lambda: P.pconv_grad_norm(ptrs(p, p + 4097), n, i32(0, 1), 2, p, p, need),
                    lambda: P.pconv_grad_norm(two, n, f32, 2, p, p + 8, need),
                    lambda: P.pconv_clip_grads(two, ptrs(p, p + 4097), n, f32, i32(0, 1), 2, 1.0, 0.0, p, p, need)],
        "too small": [lambda: P.pconv_grad_norm(two, n, f32, 2, p, p, need - 1)],
        "max_norm": [lambda: P.pconv_clip_grads(two, two, n, f32, f32, 2, -1.0, 0.0, p, p, need),
                     lambda: P.pconv_clip_grads(two, two, n, f32, f32, 2, math.nan, 0.0, p, p, need)],
        "eps": [lambda: P.pconv_clip_grads(two, two, n, f32, f32, 2, 1.0, -1.0, p, p, need),
                lambda: P.pconv_clip_grads(two, two, n, f32, f32, 2, 1.0, math.inf, p, p, need),
                lambda: P.pconv_clip_grads(two, two, n, f32, f32, 2, 1.0, math.nan, p, p, need)],
        "place": [lambda: P.pconv_clip_grads(two, two, n, f32, i32(0, 1), 2, 1.0, 0.0, p, p, need)],
    }
    for what, calls in bad.items():
        for i, call in enumerate(calls):
            with pytest.raises(P.PconvError) as e:
                call()
            assert e.value.status == P.INVALID_ARG and what in str(e.value), (what, i, str(e.value))


def test_work_space_holds_the_sums_of_all_launches():
    """One sum for each workgroup: 2048 with one launch, at least 64 for each launch of 160 tensors, and the total."""
    for num in (0, 1, 160, 161, 5000, 5120, 5121, 100_000):
        tables = -(-num // 160)
        blocks = 2048 if tables <= 1 else max(64, 2048 // tables)
        assert P.pconv_grad_workspace(num) >= 8 * (1 + max(1, tables) * blocks)


def test_lists_that_cannot_be_clipped_are_refused():
    import torch
    with pytest.raises(ValueError, match="CUDA"):
        P.GradList([torch.zeros(3)])
    with pytest.raises(ValueError):
        P.grad_norm([])


@pytest.mark.gpu
def test_wrong_tensors_are_refused():
    import torch
    z = torch.zeros(4000, device="cuda")
    a, b = z[:1000], z[1000:2000]
    bad = [lambda: P.GradList([z.half()]), lambda: P.GradList([z[::2]]), lambda: P.GradList([z[:1].expand(5)]),
           lambda: P.GradList([a, z[999:1500]]), lambda: P.GradList([a, a]), lambda: P.GradList([a], out=[b, b]),
           lambda: P.GradList([a], out=[z[500:1500]]), lambda: P.GradList([a, b], out=[b, a]),
           lambda: P.GradList([a, b], out=[z[2000:3000], z[2999:3999]]), lambda: P.GradList([a], out=[z[2000:2999]]),
           lambda: P.GradList([a.view(10, 100)], out=[z[2000:3000].view(100, 10).t()]), lambda: P.GradList([a], out=[b.double()]),
           lambda: P.GradList([a], out=[a.view(torch.bfloat16)[:1000]]), lambda: P.GradList([a], out=[b.cpu()])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"list {i} was not refused")
    for call in (lambda: P.clip_grad_norm([a], -1.0), lambda: P.clip_grad_norm([a], 1.0, eps=math.nan)):
        with pytest.raises(P.PconvError):
            call()
    P.GradList([a, b], out=[a, z[2000:3000]]).clip(1.0)  # one in place, one not
    P.GradList([a, a], out=[b, z[2000:3000]]).clip(1.0)  # read twice, written once each


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
def test_more_than_the_caches_hold_in_several_launches(in_place):
    """300 tensors of 256 KiB to 2 MiB, fp32 and bf16: two tables, read and written past the caches, the last part kept there."""
    import torch
    rng = np.random.default_rng(9)
    sizes = [int(n) for n in rng.integers(1 << 16, 1 << 20, 300)]
    say(f"[case] clip {len(sizes)} tensors, {sum(sizes)} elements, in place {in_place}")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    grads = [torch.randn(n, generator=gen, device="cuda").to(torch.bfloat16 if i % 3 == 0 else torch.float32) for i, n in enumerate(sizes)]
    want_norm = math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))
    factor = 7.0 / (want_norm + 1e-6)
    want = [g.double() * factor for g in grads]
    outs = grads if in_place else [torch.full_like(g, float("nan"), dtype=torch.float32) for g in grads]
    norm = P.clip_grad_norm(grads, 7.0, out=None if in_place else outs)
    assert abs(float(norm) - want_norm) <= 1.01 * U * want_norm
    for i, (o, w) in enumerate(zip(outs, want)):
        tol = 2.02 * U * w.abs() + 2.0 ** -149
        if o.dtype == torch.bfloat16:
            tol = tol * 1.01 + 2.0 ** -8 * 1.01 * w.abs() + 2.0 ** -133
        assert bool(((o.double() - w).abs() <= tol).all()), f"tensor {i}"
    mine = [torch.ones(3, device="cuda")] + [torch.zeros(1 << 26, device="cuda") for _ in range(2)]
    mine[2][-1] = 2.0
    assert abs(float(P.clip_grad_norm(mine, 1.0)) - math.sqrt(7)) <= 3 * U and abs(float(mine[2][-1]) * math.sqrt(7) / 2 - 1) < 1e-6
