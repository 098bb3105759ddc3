"""Layers in 8-bit integers (quantize_rows, matmul_i8, linear_i8) against plain numpy: whole numbers for the sums, 64 bits
for the rest.

Tolerances.  Quantised values and scales: equal, bit for bit (each is defined as the nearest number of the exact quotient of two
fp32 numbers, which numpy's fp32 division gives).  Outputs: the sum is exact; its conversion to fp32, the product of the
scales, their product and the addition of the bias each round once, by at most 2^-24 of what they give, so that
|y - exact| <= 4 * 2^-24 * (|sum * scales| + |bias|); rounding to bf16 (8 significant bits) adds 2^-8 of the value."""
import numpy as np
import pytest

import paper_1909_05073_amd as P

from gpu_util import say

U = 2.0 ** -24


# ---- the plain implementation ----------------------------------------------------------------------------------------

def plain_quantize(x):
    """x: fp32 array [m, k] (bf16 values as fp32) -> (q int64, scale fp32)."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        most = np.abs(x).max(axis=1, initial=0.0)        # (numpy's maximum hands NaN on)
        scale = (most / np.float32(127)).astype(np.float32)
        bad = ~np.isfinite(most)
        scale[bad] = np.nan
        q = np.zeros(x.shape, np.int64)
        rows = (scale > 0) & ~bad
        q[rows] = np.clip(np.rint(x[rows] / scale[rows, None]), -127, 127).astype(np.int64)
    return q, scale


def plain_product(q, sa, w, sb, bias, relu):
    """(y, bound of the error of an fp32 y), both fp64."""
    acc = (q.astype(np.float64) @ w.astype(np.float64).T)             # whole numbers below 2^53: exact
    with np.errstate(invalid="ignore"):
        scaled = acc * sa.astype(np.float64)[:, None] * sb.astype(np.float64)[None, :]
    b = np.zeros(w.shape[0]) if bias is None else bias.astype(np.float64)
    y = scaled + b
    # (2^-140: products of scales below the normal numbers)
    bound = 4 * U * (np.abs(scaled) + np.abs(b)) + np.abs(acc) * 2.0 ** -149 + 2.0 ** -140
    if relu:
        y = np.where(y < 0, 0.0, y)
    return y, bound


def check(y, want, bound, what):
    import torch
    got = y.detach().float().cpu().numpy().astype(np.float64).reshape(want.shape)
    if y.dtype == torch.bfloat16:
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8)
    nan = np.isnan(want)
    assert np.array_equal(nan, np.isnan(got)), f"{what}: NaN elsewhere"
    err = np.abs(np.where(nan, 0, got) - np.where(nan, 0, want))
    bad = np.argwhere(err > np.where(nan, 0, bound))
    assert bad.size == 0, f"{what}: {len(bad)} of {want.size} outside; first at {tuple(bad[0])}: {got[tuple(bad[0])]} for {want[tuple(bad[0])]}"


# ---- inputs ------------------------------------------------------------------------------------------------------------

def make_x(rng, m, k):
    x = np.maximum(rng.standard_normal((m, k)), -0.3).astype(np.float32) * np.exp(rng.uniform(-3, 3, (m, 1))).astype(np.float32)
    if m > 2:
        x[1] = 0                                         # a row without any value
    return x


def make_layer8(rng, n, k, bias=True):
    w = rng.integers(-127, 128, (n, k)).astype(np.int8)
    return w, np.exp(rng.uniform(-6, 0, n)).astype(np.float32), rng.standard_normal(n).astype(np.float32) if bias else None


def dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def laid_out(a, offset, extra):
    """A CUDA copy of the matrix that begins `offset` elements into its storage, its rows `extra` elements further apart
    than they are long; around it only values that would show."""
    import torch
    m, k = a.shape
    flat = torch.full((offset + m * (k + extra) + 1,), 101 if a.dtype == np.int8 else float("nan"),
                      dtype=torch.int8 if a.dtype == np.int8 else torch.float32, device="cuda")
    t = torch.as_strided(flat, (m, k), (k + extra, 1), offset)
    t.copy_(torch.from_numpy(a))
    return t


def as_type(x, dtype):
    """(CUDA tensor, the fp32 values that it holds)."""
    import torch
    t = dev(x, torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t, t.float().cpu().numpy()


# ---- quantize_rows -------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k", [(1, 1), (3, 2), (1, 7), (5, 8), (33, 9), (7, 31), (40, 32), (3, 63), (257, 64), (9, 100), (5, 255),
                                 (6, 257), (4, 513), (65, 1000), (3, 2049), (2, 4100), (3, 8191), (2, 16385), (1, 25088), (2, 70001)])
def test_quantized_rows_are_the_definition(m, k, dtype):
    say(f"[case] quantize_rows {m}x{k} {dtype}")
    rng = np.random.default_rng(m * 100003 + k)
    x, values = as_type(make_x(rng, m, k), dtype)
    q, scale = P.quantize_rows(x)
    want, ws = plain_quantize(values)
    assert np.array_equal(scale.cpu().numpy(), ws)
    assert np.array_equal(q.cpu().numpy().astype(np.int64), want)


@pytest.mark.gpu
def test_quotients_near_ties_round_as_the_division_does():
    """Values that lie within a few units in the last place of (j + 1/2) * scale, for scales of all sizes."""
    rng = np.random.default_rng(5)
    m, k = 600, 1016
    most = np.exp2(rng.uniform(-98, 120, m)).astype(np.float32)
    most[:64] = np.exp2(rng.uniform(-60, -40, 64)).astype(np.float32)
    scale = most / np.float32(127)
    j = rng.integers(0, 127, (m, k))
    x = ((j + 0.5) * scale[:, None].astype(np.float64)).astype(np.float32)
    x = (x.view(np.int32) + rng.integers(-3, 4, (m, k), dtype=np.int32)).view(np.float32)
    x = np.minimum(x, most[:, None]) * rng.choice([-1, 1], (m, k)).astype(np.float32)
    x[:, 0] = most
    say(f"[case] quantize_rows near ties {m}x{k}")
    q, s = P.quantize_rows(dev(x))
    want, ws = plain_quantize(x)
    assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(q.cpu().numpy().astype(np.int64), want)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [5, 64, 300, 3001, 9000])
def test_rows_with_tiny_huge_infinite_and_nan_values(k):
    rng = np.random.default_rng(k)
    x = rng.standard_normal((12, k)).astype(np.float32)
    x[0] *= np.float32(1e-37)                            # scales below 2^-100
    x[1] = (x[1] * 1e-30).astype(np.float32) * np.float32(1e-12)      # denormal values
    x[2] = np.float32(2.0 ** -149)                       # a scale that rounds to zero
    x[3] = np.float32(3.4e38) * np.sign(x[3])
    x[4, k - 1] = np.inf
    x[5, 0] = -np.inf
    x[6, k // 2] = np.nan
    x[7, k - 1] = -np.nan
    x[8] = 0
    x[9] = -0.0
    x[10] = np.float32(1e-40) * rng.integers(0, 50, k)
    say(f"[case] quantize_rows odd values k={k}")
    q, scale = P.quantize_rows(dev(x))
    want, ws = plain_quantize(x)
    got = scale.cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ws)) and np.isnan(ws[4:8]).all()
    assert np.array_equal(got[~np.isnan(ws)], ws[~np.isnan(ws)])
    assert np.array_equal(q.cpu().numpy().astype(np.int64), want)


@pytest.mark.gpu
@pytest.mark.parametrize("offset,extra", [(0, 4), (1, 0), (3, 5), (2, 1)])
@pytest.mark.parametrize("k", [1, 30, 333, 5000])
def test_quantized_rows_that_lie_apart_and_begin_anywhere(k, offset, extra):
    import torch
    rng = np.random.default_rng(k + offset)
    a = make_x(rng, 6, k)
    say(f"[case] quantize_rows k={k} offset={offset} extra={extra}")
    for dtype in (torch.float32, torch.bfloat16):
        x = laid_out(a, offset, extra)
        if dtype == torch.bfloat16:
            flat = torch.empty(offset + 6 * (k + extra) + 1, dtype=dtype, device="cuda").fill_(float("inf"))
            y = torch.as_strided(flat, (6, k), (k + extra, 1), offset)
            y.copy_(x)
            x = y
        qs = torch.full((offset + 6 * (k + extra) + 8,), 77, dtype=torch.int8, device="cuda")
        scale = torch.empty(6, device="cuda")
        P.pconv_quantize_rows(x.data_ptr(), k + extra, "f32" if dtype == torch.float32 else "bf16", 6, k,
                              qs.data_ptr() + offset, k + extra, scale.data_ptr(), torch.cuda.current_stream().cuda_stream)
        want, ws = plain_quantize(x.float().cpu().numpy())
        host = qs.cpu().numpy()
        got = np.lib.stride_tricks.as_strided(host[offset:], (6, k), (k + extra, 1))
        assert np.array_equal(got.astype(np.int64), want) and np.array_equal(scale.cpu().numpy(), ws)
        keep = np.ones(host.size, bool)
        for r in range(6):
            keep[offset + r * (k + extra): offset + r * (k + extra) + k] = False
        assert (host[keep] == 77).all(), "bytes between the rows were written"


# ---- the product ---------------------------------------------------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 10, 512), (2, 3, 15), (1, 1000, 2048), (3, 17, 16), (15, 16, 17), (16, 15, 63), (17, 130, 64), (8, 33, 4097),
         (31, 257, 65), (32, 64, 1000), (33, 63, 127), (48, 100, 257), (63, 129, 128), (64, 128, 255), (65, 127, 129), (100, 1, 300),
         (127, 129, 256), (128, 128, 128), (129, 257, 383), (300, 64, 64), (1000, 40, 16), (257, 300, 1155), (513, 511, 511),
         (2000, 256, 64), (700, 520, 640), (5, 4000, 300), (4, 70, 20000), (70, 20, 9000)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product_and_layer_against_the_formula(m, n, k, dtype):
    import torch
    say(f"[case] matmul_i8 / linear_i8 {m}x{n}x{k} {dtype}")
    rng = np.random.default_rng(m * 1000003 + n * 1009 + k)
    x, values = as_type(make_x(rng, m, k), dtype)
    w, sb, bias = make_layer8(rng, n, k)
    relu = (m + n + k) % 2 == 0
    q, sa = plain_quantize(values)
    want, bound = plain_product(q, sa, w, sb, bias, relu)
    wd, sd, bd = dev(w), dev(sb), dev(bias)
    y = P.linear_i8(x, wd, sd, bd, relu=relu)
    assert y.dtype == x.dtype
    check(y, want, bound, "linear_i8")
    z = P.matmul_i8(dev(q.astype(np.int8)), dev(sa), wd, sd, bd, relu=relu, out_dtype=x.dtype)
    assert torch.equal(y, z), "the call in one gives other values than the two calls"
    # no bias, the other type of outputs, the other activation
    other = torch.bfloat16 if dtype == "f32" else torch.float32
    want, bound = plain_product(q, sa, w, sb, None, not relu)
    check(P.linear_i8(x, wd, sd, relu=not relu, out_dtype=other), want, bound, "linear_i8, no bias")


# Lengths that are whole pieces of 16 bytes but no whole stages of 128, by each kernel; few, many and odd channels; k split.
PIECES = [(20, 64, 192), (20, 24, 320), (100, 256, 448), (130, 520, 192), (70, 128, 384), (17, 8, 64), (33, 1000, 64), (64, 136, 512),
          (1, 40, 16), (3, 48, 272), (16, 16, 4112), (2, 300, 8208), (1, 9, 24992), (5, 17, 30000),
          (20, 64, 528), (65, 130, 576), (40, 256, 1104), (300, 300, 2064), (129, 512, 720), (1000, 260, 656), (24, 40, 20016),
          (2600, 2050, 592), (33, 7, 16400), (10, 100, 13120), (12, 64, 16384)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", PIECES)
def test_lengths_that_end_inside_a_stage(m, n, k, dtype):
    import torch
    say(f"[case] linear_i8 {m}x{n}x{k} {dtype}")
    rng = np.random.default_rng(m * 10007 + n * 101 + k)
    x, values = as_type(make_x(rng, m, k), dtype)
    w, sb, bias = make_layer8(rng, n, k)
    q, sa = plain_quantize(values)
    want, bound = plain_product(q, sa, w, sb, bias, True)
    # behind the weights lie bytes that would show
    wide = torch.full((n, k + 64), 101, dtype=torch.int8, device="cuda")
    wide[:, :k] = dev(w)
    for b in (dev(w), wide[:, :k]):
        check(P.linear_i8(x, b, dev(sb), dev(bias), relu=True), want, bound, "linear_i8")
        a = torch.full((m, k + 16), 99, dtype=torch.int8, device="cuda")
        a[:, :k] = dev(q.astype(np.int8))
        check(P.matmul_i8(a[:, :k], dev(sa), b, dev(sb), dev(bias), relu=True, out_dtype=x.dtype), want, bound, "matmul_i8")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(4, 40, 8192), (8, 33, 4096), (12, 20, 2704), (5, 130, 5136), (6, 7, 5440), (9, 24, 2560), (3, 20, 10000),
                                   (4, 5000, 8176), (7, 17, 4112)])
def test_a_few_long_rows(m, n, k, dtype):
    test_lengths_that_end_inside_a_stage(m, n, k, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [513, 527, 585, 641, 1023, 1155, 2050, 9001, 20013])
def test_what_lies_behind_the_rows_does_not_count(k):
    """Rows at multiples of 16 bytes whose last piece is not theirs alone; the last row ends with the memory."""
    import torch
    for m, n in ((17, 5), (32, 128), (33, 129), (64, 300), (130, 520), (1500, 700)):
        if m * k > 2_000_000:
            continue
        say(f"[case] matmul_i8 {m}x{n}x{k}")
        rng = np.random.default_rng(m * 10007 + n * 101 + k)
        _, values = as_type(make_x(rng, m, k), "f32")
        w, sb, bias = make_layer8(rng, n, k)
        q, sa = plain_quantize(values)
        want, bound = plain_product(q, sa, w, sb, bias, True)
        rows = []
        for t, byte in ((q.astype(np.int8), 99), (w, -101)):
            step = (k + 15) // 16 * 16 + 16 * (m % 2)
            flat = torch.full(((len(t) - 1) * step + k,), byte, dtype=torch.int8, device="cuda")
            rows.append(flat.as_strided((len(t), k), (step, 1)))
            rows[-1].copy_(dev(t))
        check(P.matmul_i8(rows[0], dev(sa), rows[1], dev(sb), dev(bias), relu=True), want, bound, "matmul_i8")
        x = dev(values.astype(np.float32))
        check(P.linear_i8(x, rows[1], dev(sb), dev(bias), relu=True), want, bound, "linear_i8")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [16, 32, 48, 80, 96, 112, 144, 176, 208, 240, 272, 336, 400, 432, 496])
def test_short_rows_of_whole_pieces(k, dtype):
    for m, n in ((17, 8), (64, 136), (130, 520)):
        test_lengths_that_end_inside_a_stage(m, n, k, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(7900, 4000, 592), (7900, 4000, 585), (5000, 1030, 1040), (90_000, 72, 560), (40_000, 200, 320), (20_000, 264, 448)])
def test_many_tiles(m, n, k):
    """Products whose tiles fill the card, against 64 bits on the card."""
    import torch
    say(f"[case] matmul_i8 {m}x{n}x{k}")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m + k)
    x = torch.randn(m, k, generator=gen, device="cuda") * torch.rand(m, 1, generator=gen, device="cuda")
    w = torch.randint(-127, 128, (n, k), generator=gen, device="cuda", dtype=torch.int8)
    sb, bias = torch.rand(n, generator=gen, device="cuda"), torch.randn(n, generator=gen, device="cuda")
    most = x.abs().amax(1, keepdim=True)
    scale = most / torch.full_like(most, 127.0)
    q = (x / scale).round()                              # (no row of zeros among these)
    scaled = (q.double() @ w.double().t()) * scale.double() * sb.double()
    want = scaled + bias.double()
    bound = 4 * U * (scaled.abs() + bias.double().abs())
    got, s = P.quantize_rows(x)
    assert torch.equal(got.float(), q) and torch.equal(s, scale[:, 0])
    for dtype in (torch.float32, torch.bfloat16):
        tol = bound if dtype == torch.float32 else bound * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs() * (1 + 2.0 ** -8)
        for y in (P.linear_i8(x, w, sb, bias, out_dtype=dtype), P.matmul_i8(got, s, w, sb, bias, out_dtype=dtype)):
            assert bool(((y.double() - want).abs() <= tol).all())
        assert torch.equal(P.linear_i8(x, w, sb, bias, relu=True, out_dtype=dtype), y.clamp(min=0))


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 20, 70), (5, 33, 300), (40, 50, 129), (130, 140, 200), (300, 130, 64)])
@pytest.mark.parametrize("offset,extra", [(0, 16), (0, 1), (1, 0), (3, 6), (16, 48)])
def test_operands_and_outputs_that_lie_apart_and_begin_anywhere(m, n, k, offset, extra):
    import torch
    say(f"[case] matmul_i8 {m}x{n}x{k} offset={offset} extra={extra}")
    rng = np.random.default_rng(m + n + k + offset + extra)
    w, sb, bias = make_layer8(rng, n, k)
    q = rng.integers(-128, 128, (m, k)).astype(np.int8)
    sa = np.exp(rng.uniform(-3, 3, m)).astype(np.float32)
    want, bound = plain_product(q.astype(np.int64), sa, w, sb, bias, False)
    a, b = laid_out(q, offset, extra), laid_out(w, extra, offset)
    for dtype in (torch.float32, torch.bfloat16):
        flat = torch.full((offset + m * (n + extra) + 8,), 7.0, dtype=dtype, device="cuda")
        out = torch.as_strided(flat, (m, n), (n + extra, 1), offset)
        y = P.matmul_i8(a, dev(sa), b, dev(sb), dev(bias), out=out)
        assert y is out
        check(y, want, bound, "matmul_i8")
        rest = flat.clone()
        torch.as_strided(rest, (m, n), (n + extra, 1), offset).fill_(7.0)
        assert bool((rest == 7.0).all()), "outputs outside the matrix were written"
    x = laid_out(make_x(rng, m, k), offset, extra)
    qx, sx = plain_quantize(x.cpu().numpy())
    want, bound = plain_product(qx, sx, w, sb, bias, True)
    check(P.linear_i8(x, b, dev(sb), dev(bias), relu=True), want, bound, "linear_i8")


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 3, 20, 50, 130])
@pytest.mark.parametrize("va,vb", [(-128, -128), (127, -128), (127, 127)])
def test_sums_that_fill_32_bits(m, va, vb):
    import torch
    k, n = 131071, 18
    say(f"[case] matmul_i8 extremes m={m} {va} {vb}")
    a = torch.full((m, k), va, dtype=torch.int8, device="cuda")
    b = torch.full((n, k), vb, dtype=torch.int8, device="cuda")
    one = torch.ones(max(m, n), device="cuda")
    y = P.matmul_i8(a, one[:m].clone(), b, one[:n].clone())
    exact = np.float32(k * va * vb)                      # the nearest fp32 number of the exact sum
    assert bool((y == float(exact)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(6, 20, 40), (20, 20, 40), (40, 20, 40), (100, 70, 200)])
def test_rows_of_zeros_infinities_and_nan(m, n, k):
    say(f"[case] linear_i8 odd rows {m}x{n}x{k}")
    rng = np.random.default_rng(m)
    x = make_x(rng, m, k)
    x[0] = 0; x[2, 3] = np.inf; x[3, k - 1] = np.nan; x[5] *= np.float32(1e-38)
    w, sb, bias = make_layer8(rng, n, k)
    q, sa = plain_quantize(x)
    for relu in (False, True):
        want, bound = plain_product(q, sa, w, sb, bias, relu)
        assert np.isnan(want[2:4]).all() and np.isfinite(np.delete(want, [2, 3], 0)).all()
        check(P.linear_i8(dev(x), dev(w), dev(sb), dev(bias), relu=relu), want, bound, f"linear_i8 relu={relu}")


@pytest.mark.gpu
def test_sizes_of_zero():
    import torch
    say("[case] 8-bit layers, sizes of zero")
    w, sb, bias = (dev(a) for a in make_layer8(np.random.default_rng(0), 20, 8))
    for m in (0, 3, 100):
        y = P.linear_i8(torch.zeros(m, 8, device="cuda"), w, sb, bias, relu=True)
        assert y.shape == (m, 20) and torch.equal(y, bias.clamp(min=0).expand(m, 20))
        q, s = P.quantize_rows(torch.zeros(m, 0, device="cuda"))
        assert q.shape == (m, 0) and bool((s == 0).all())
        y = P.linear_i8(torch.zeros(m, 0, device="cuda"), w[:, :0], sb, bias)
        assert torch.equal(y, bias.expand(m, 20))
        y = P.matmul_i8(torch.zeros(m, 0, dtype=torch.int8, device="cuda"), torch.ones(m, device="cuda"), w[:, :0], sb)
        assert torch.equal(y, torch.zeros(m, 20, device="cuda"))
        assert P.linear_i8(torch.zeros(m, 8, device="cuda"), w[:0], sb[:0]).shape == (m, 0)


@pytest.mark.gpu
def test_leading_dimensions_are_rows():
    import torch
    say("[case] linear_i8 on [2, 5, 7, 24]")
    rng = np.random.default_rng(3)
    x = make_x(rng, 70, 24)
    w, sb, bias = make_layer8(rng, 40, 24)
    q, sa = plain_quantize(x)
    want, bound = plain_product(q, sa, w, sb, bias, False)
    y = P.linear_i8(dev(x).view(2, 5, 7, 24), dev(w), dev(sb), dev(bias))
    assert y.shape == (2, 5, 7, 40)
    check(y, want, bound, "linear_i8")
    v, s = P.quantize_rows(dev(x).view(2, 5, 7, 24))
    assert v.shape == (2, 5, 7, 24) and s.shape == (2, 5, 7)
    check(P.matmul_i8(v, s, dev(w), dev(sb), dev(bias)), want, bound, "matmul_i8")
    one = P.linear_i8(dev(x)[4], dev(w), dev(sb), dev(bias))
    assert one.shape == (40,) and torch.equal(one, P.linear_i8(dev(x)[4:5], dev(w), dev(sb), dev(bias))[0])


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1030, 24, 48), (40, 24, 48), (3, 24, 48), (40, 24, 600), (3, 24, 600)])
def test_offsets_beyond_32_bits(m, n, k):
    """Rows of a, of x and of y that lie so far apart that the last ones are beyond 2^32 bytes; rows of b as well."""
    import torch
    say(f"[case] matmul_i8 far rows {m}x{n}x{k}")
    rng = np.random.default_rng(m)
    step = (1 << 32) // (m - 1) // 16 * 16 + 64
    w, sb, bias = make_layer8(rng, n, k)
    x = make_x(rng, m, k)
    q, sa = plain_quantize(x)
    want, bound = plain_product(q, sa, w, sb, bias, False)
    room = torch.empty((m - 1) * step + k + 64, dtype=torch.int8, device="cuda")
    a = torch.as_strided(room, (m, k), (step, 1))
    a.copy_(dev(q.astype(np.int8)))
    check(P.matmul_i8(a, dev(sa), dev(w), dev(sb), dev(bias)), want, bound, "far rows of a")
    rows = min(n, 24)
    far = (1 << 32) // (rows - 1) // 16 * 16 + 64
    room = torch.empty((rows - 1) * far + k + 64, dtype=torch.int8, device="cuda")
    b = torch.as_strided(room, (n, k), (far, 1))
    b.copy_(dev(w))
    check(P.matmul_i8(dev(q.astype(np.int8)), dev(sa), b, dev(sb), dev(bias)), want, bound, "far rows of b")
    del room, a, b
    room = torch.empty((m - 1) * (step // 4) + k + 64, dtype=torch.float32, device="cuda")
    xs = torch.as_strided(room, (m, k), (step // 4, 1))
    xs.copy_(dev(x))
    check(P.linear_i8(xs, dev(w), dev(sb), dev(bias)), want, bound, "far rows of x")
    ys = torch.as_strided(room, (m, n), (step // 4, 1))
    check(P.matmul_i8(dev(q.astype(np.int8)), dev(sa), dev(w), dev(sb), dev(bias), out=ys), want, bound, "far rows of y")


@pytest.mark.gpu
@pytest.mark.parametrize("m", [2, 40, 300])
def test_another_stream_and_equal_bits(m):
    """The call runs on torch's current stream, behind what is queued there, and gives the same bits every time."""
    import torch
    say(f"[case] linear_i8 on another stream m={m}")
    rng = np.random.default_rng(m)
    x, w, sb, bias = dev(make_x(rng, m, 3000)), *(dev(a) for a in make_layer8(rng, 200, 3000))
    want = P.linear_i8(x, w, sb, bias)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    late = torch.zeros_like(x)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        big = torch.randn(3000, 3000, device="cuda")
        for _ in range(5):
            big = big @ big * 1e-3
        late.copy_(x)
        y = P.linear_i8(late, w, sb, bias)
    s.synchronize()
    assert torch.equal(y, want)
    for _ in range(3):
        assert torch.equal(P.linear_i8(x, w, sb, bias), want)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 40, 300])
def test_replays_of_a_captured_layer(m):
    import torch
    say(f"[case] linear_i8 captured m={m}")
    rng = np.random.default_rng(m)
    w, sb, bias = (dev(a) for a in make_layer8(rng, 300, 2050))
    x = torch.zeros(m, 2050, device="cuda")
    out = torch.empty(m, 300, device="cuda")
    P.linear_i8(x, w, sb, bias, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.linear_i8(x, w, sb, bias, relu=True, out=out)
        z = P.linear_i8(out, w[:, :300], sb, bias)
    for i in range(4):
        x.copy_(dev(make_x(rng, m, 2050)))
        g.replay()
        torch.cuda.synchronize()
        want = P.linear_i8(x, w, sb, bias, relu=True)
        assert torch.equal(out, want) and torch.equal(z, P.linear_i8(want, w[:, :300], sb, bias)), f"replay {i}"


# ---- refusals ------------------------------------------------------------------------------------------------------------

def c_calls():
    """(what is wrong, call) for raw calls that return before anything is launched; no pointer is followed."""
    p = 1 << 20
    yield "rows", lambda: P.pconv_quantize_rows(p, 8, "f32", -1, 8, p, 8, p)
    yield "2^31", lambda: P.pconv_quantize_rows(p, 1 << 31, "f32", 1, 1 << 31, p, 1 << 31, p)
    yield "null", lambda: P.pconv_quantize_rows(0, 8, "f32", 2, 8, p, 8, p)
    yield "null", lambda: P.pconv_quantize_rows(p, 8, "f32", 2, 8, 0, 8, p)
    yield "null", lambda: P.pconv_quantize_rows(p, 8, "f32", 2, 8, p, 8, 0)
    yield "apart", lambda: P.pconv_quantize_rows(p, 7, "f32", 2, 8, p, 8, p)
    yield "apart", lambda: P.pconv_quantize_rows(p, 8, "f32", 2, 8, p, 7, p)
    yield "apart", lambda: P.pconv_quantize_rows(p, 1 << 60, "f32", 2, 8, p, 8, p)
    yield "m and n", lambda: P.pconv_matmul_i8(p, 16, p, p, 16, p, 0, p, 4, "f32", 4, (1 << 30) + 1, 16)
    yield "k must", lambda: P.pconv_matmul_i8(p, 1 << 18, p, p, 1 << 18, p, 0, p, 4, "f32", 4, 4, 131072)
    yield "m and n", lambda: P.pconv_matmul_i8(p, 16, p, p, 16, p, 0, p, 4, "f32", 1 << 31, 4, 16)
    yield "m and n", lambda: P.pconv_matmul_i8(p, 16, p, p, 16, p, 0, p, 4, "f32", 4, -4, 16)
    yield "apart", lambda: P.pconv_matmul_i8(p, 15, p, p, 16, p, 0, p, 4, "f32", 4, 4, 16)
    yield "apart", lambda: P.pconv_matmul_i8(p, 16, p, p, 15, p, 0, p, 4, "f32", 4, 4, 16)
    yield "apart", lambda: P.pconv_matmul_i8(p, 16, p, p, 16, p, 0, p, 3, "f32", 4, 4, 16)
    for i in range(5):
        args = [p, p, p, p, p]
        args[i] = 0
        a, sa, b, sb, y = args
        yield "null", lambda a=a, sa=sa, b=b, sb=sb, y=y: P.pconv_matmul_i8(a, 16, sa, b, 16, sb, 0, y, 4, "f32", 4, 4, 16)
    need = P.pconv_linear_i8_workspace(400, 40, 2600, True)
    assert need >= 400 * 2600
    yield "work space", lambda: P.pconv_linear_i8(p, 2600, "f32", p, 2600, p, 0, p, 40, "f32", 400, 40, 2600, False, p, need - 1)
    yield "work space", lambda: P.pconv_linear_i8(p, 2600, "f32", p, 2600, p, 0, p, 40, "f32", 400, 40, 2600, False, 0, need)
    yield "work space", lambda: P.pconv_linear_i8(p, 2600, "f32", p, 2600, p, 0, p, 40, "f32", 400, 40, 2600, False, p + 8, need)
    yield "null", lambda: P.pconv_linear_i8(0, 2600, "f32", p, 2600, p, 0, p, 40, "f32", 400, 40, 2600, False, p, need)
    yield "apart", lambda: P.pconv_linear_i8(p, 1599, "f32", p, 2600, p, 0, p, 40, "f32", 400, 40, 2600, False, p, need)


def test_c_entries_refuse_what_they_cannot_run():
    for what, call in c_calls():
        with pytest.raises(P.PconvError) as e:
            call()
        assert e.value.status == P.INVALID_ARG and what in str(e.value), (what, str(e.value))


def test_unknown_types_are_refused_at_the_c_entries():
    p = 1 << 20
    L = P.lib()
    assert L.pconv_quantize_rows(p, 8, 7, 2, 8, p, 8, p, None) == P.INVALID_ARG
    assert L.pconv_matmul_i8(p, 16, p, p, 16, p, None, p, 4, 7, 4, 4, 16, 0, None, 0, None) == P.INVALID_ARG
    assert L.pconv_linear_i8(p, 16, 7, p, 16, p, None, p, 4, 0, 4, 4, 16, 0, None, 0, None) == P.INVALID_ARG


def test_calls_on_the_host_are_refused():
    import torch
    x, w, s = torch.zeros(4, 8), torch.zeros(3, 8, dtype=torch.int8), torch.ones(3)
    for call in (lambda: P.quantize_rows(x), lambda: P.linear_i8(x, w, s), lambda: P.matmul_i8(w, s, w, s)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


@pytest.mark.gpu
def test_wrong_tensors_are_refused():
    import torch
    z = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")
    x, w, s, b, q, sa = z(4, 8), z(3, 8, dtype=torch.int8), z(3), z(3), z(4, 8, dtype=torch.int8), z(4)
    bad = [lambda: P.quantize_rows(x.half()), lambda: P.quantize_rows(x.t()), lambda: P.quantize_rows(z(1, 8).expand(4, 8)),
           lambda: P.quantize_rows(torch.zeros((), device="cuda")), lambda: P.quantize_rows(z(9)[::2]),
           lambda: P.quantize_rows(z(4, 6, 8)[:, :3].transpose(0, 1)),
           lambda: P.linear_i8(x, w.float(), s), lambda: P.linear_i8(x, w[:, :7], s), lambda: P.linear_i8(x, w.view(-1), s),
           lambda: P.linear_i8(x, w, s[:2]), lambda: P.linear_i8(x, w, s.double()), lambda: P.linear_i8(x, w, s, b[:2]),
           lambda: P.linear_i8(x, w, z(6)[::2], b), lambda: P.linear_i8(x, w, s, b, out=z(4, 4)),
           lambda: P.linear_i8(x, w, s, b, out=z(4, 3), out_dtype=torch.bfloat16), lambda: P.linear_i8(x, w, s, b.cpu()),
           lambda: P.linear_i8(x, w, s, out_dtype=torch.float16), lambda: P.linear_i8(x, w, s, out=z(3, 4).t()),
           lambda: P.matmul_i8(x, sa, w, s), lambda: P.matmul_i8(q, s, w, s), lambda: P.matmul_i8(q, sa, w, sa),
           lambda: P.matmul_i8(q, sa, w[:, :5], s), lambda: P.matmul_i8(q, sa, w, s, out=z(4, 3, dtype=torch.float64))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
