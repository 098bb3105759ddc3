"""Layers in 4-bit floats (quantize_mx4, matmul_mx4, linear_mx4) against plain numpy in 64 bits.

Tolerances.  Codes and scales: equal, bit for bit (values and powers of two are exact in 64 bits).  Products of two 4-bit values
are whole multiples of 1/4 up to 36, and scales powers of two, so every term is exact in fp32.  Where all partial sums are whole
multiples below 2^24 of one power of two (`exact_in_fp32`) the sum is exact in any order, and only the bias rounds, by 2^-24.
Elsewhere each of at most 32 * blocks + 80 additions (terms, parts of k, the bias) is off by at most 2^-23 of the sum of all
magnitudes, rounded or cut.  Rounding to bf16 adds 2^-8 of the value."""
import numpy as np
import pytest

import paper_1909_05073_amd as P

from gpu_util import say
from test_i8_layers import as_type, dev

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate([VALUES, -VALUES])
MIDDLES = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])


# ---- the plain implementation ----------------------------------------------------------------------------------------

def plain_quantize(x):
    """x: fp32 array [m, k] -> (codes uint8 [m, blocks * 32], scale bytes uint8 [m, blocks])."""
    m, k = x.shape
    blocks = -(-k // 32)
    wide = np.zeros((m, blocks * 32), np.float32)
    wide[:, :k] = x
    wide = wide.reshape(m, blocks, 32)
    most = np.abs(wide).max(2, initial=0)                # (hands NaN on)
    bad = ~np.isfinite(most)
    e = np.frexp(np.where(bad | (most == 0), 1, most).astype(np.float64))[1] - 1
    power = np.where(most == 0, -127, np.clip(e - 2, -127, 127))
    v = np.where(bad[..., None], 0, wide).astype(np.float64) / np.exp2(power.astype(np.float64))[..., None]
    a = np.abs(v)
    code = (a[..., None] > MIDDLES).sum(-1)
    tie = (a[..., None] == MIDDLES).any(-1)
    code = np.where(tie & (code % 2 == 1), code + 1, code)               # (from the odd code below the middle to the even one)
    code = code + 8 * np.signbit(np.where(bad[..., None], 0, wide))
    return code.astype(np.uint8).reshape(m, -1), np.where(bad, 255, power + 127).astype(np.uint8)


def packed(codes, scales):
    """As the library keeps them: (q [m, blocks * 16], scale [slabs, m, 8])."""
    m, blocks = scales.shape
    q = (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)
    slabs = -(-blocks // 8)
    wide = np.zeros((m, slabs * 8), np.uint8)
    wide[:, :blocks] = scales
    return q, np.ascontiguousarray(wide.reshape(m, slabs, 8).transpose(1, 0, 2))


def values(codes, scales):
    m, blocks = scales.shape
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (VALUES[codes].reshape(m, blocks, 32) * s[..., None]).reshape(m, -1)


def exact_in_fp32(a, b):
    """Whether every partial sum of a @ b.T is a whole multiple below 2^24 of one power of two; a, b: (codes, scales)."""
    sa, sb = (s[s != 255].astype(int) for _, s in (a, b))
    if not sa.size or not sb.size:
        return True
    unit = 2.0 ** (sa.min() + sb.min() - 254 - 2)
    return 36 * a[0].shape[1] * 2.0 ** (sa.max() + sb.max() - 254) < unit * 2 ** 24


def plain_product(a, b, bias, relu):
    """a, b: (codes, scales).  (y, bound of the error of an fp32 y), both fp64."""
    va, vb = values(*a), values(*b)
    y = va @ vb.T
    size = np.nan_to_num(np.abs(va)) @ np.nan_to_num(np.abs(vb)).T
    add = np.zeros(len(vb)) if bias is None else bias.astype(np.float64)
    exact = exact_in_fp32(a, b)
    y = y + add
    bound = 2.0 ** -24 * np.nan_to_num(np.abs(y)) + 2.0 ** -149 if exact else (va.shape[1] + 80) * 2.0 ** -23 * (size + np.abs(add)) + 2.0 ** -140
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

def make_x(rng, m, k, spread=0.0):
    x = rng.standard_normal((m, k)) * np.exp(rng.uniform(-spread, spread, (m, k)))
    x = np.maximum(x, -0.7).astype(np.float32)
    if m > 2:
        x[1] = 0
    return x


def make_layer4(rng, n, k, spread=0):
    """(codes, scales) of weights, with whole blocks of any codes; `spread`: of the scales' exponents."""
    blocks = -(-k // 32)
    codes = rng.integers(0, 16, (n, blocks * 32)).astype(np.uint8)
    codes[:, k:] = 0
    return codes, rng.integers(120, 121 + spread, (n, blocks)).astype(np.uint8)


def on_card(operand):
    return tuple(dev(t) for t in packed(*operand))


def check_quantized(q, scale, x):
    codes, scales = plain_quantize(x)
    want, ws = packed(codes, scales)
    assert np.array_equal(scale.cpu().numpy(), ws)
    assert np.array_equal(q.cpu().numpy().reshape(want.shape), want)


# ---- quantize_mx4 --------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k", [(1, 1), (3, 2), (1, 7), (5, 8), (33, 9), (7, 31), (40, 32), (3, 33), (257, 64), (9, 100), (5, 255), (4, 256),
                                 (6, 257), (4, 513), (65, 1000), (3, 2049), (2, 4100), (3, 8191), (2, 16385), (1, 25088), (2, 70001), (9000, 40)])
def test_quantized_rows_are_the_definition(m, k, dtype):
    say(f"[case] quantize_mx4 {m}x{k} {dtype}")
    x, v = as_type(make_x(np.random.default_rng(m * 100003 + k), m, k, 2.0), dtype)
    check_quantized(*P.quantize_mx4(x), v)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_at_and_beside_the_middles(dtype):
    """Every middle between two values, and its neighbours, at scales of all sizes and both signs."""
    rng = np.random.default_rng(5)
    rows, k = 500, 96
    power = rng.integers(-127, 126, (rows, k // 32)).repeat(32, 1)
    power[:20] = -127
    power[20:40] = 125
    a = rng.choice(np.concatenate([MIDDLES, [6.0, 7.0, 0.0, 5.0]]), (rows, k))
    a[:, ::32] = rng.choice([4.0, 5.0, 6.0, 7.5], (rows, k // 32))       # (the block's largest: its exponent is the scale's and two)
    x = np.ldexp(a, power).astype(np.float32)
    moved = x.view(np.int32) + np.where(a > 0, rng.integers(-1, 2, (rows, k)), 0).astype(np.int32)
    x = moved.astype(np.int32).view(np.float32) * rng.choice([-1, 1], (rows, k)).astype(np.float32)
    assert np.isfinite(x).all()
    say(f"[case] quantize_mx4 middles {dtype}")
    t, v = as_type(x, dtype)
    check_quantized(*P.quantize_mx4(t), v)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [5, 64, 300, 3001])
def test_blocks_with_tiny_huge_infinite_and_nan_values(k):
    rng = np.random.default_rng(k)
    x = rng.standard_normal((12, k)).astype(np.float32)
    x[0] *= np.float32(1e-37)
    x[1] = (x[1] * 1e-30).astype(np.float32) * np.float32(1e-12)
    x[2] = np.float32(2.0 ** -149)
    x[3] = np.float32(3.4e38) * np.sign(x[3])
    x[4, k - 1] = np.inf
    x[5, 0] = -np.inf
    x[6, k // 2] = np.nan
    x[7, k - 1] = -np.nan
    x[8] = 0
    x[9] = -0.0
    x[10] = np.float32(1e-40) * rng.integers(0, 50, k)
    say(f"[case] quantize_mx4 odd values k={k}")
    check_quantized(*P.quantize_mx4(dev(x)), x)


@pytest.mark.gpu
@pytest.mark.parametrize("offset,extra", [(0, 4), (1, 0), (3, 5), (2, 1)])
@pytest.mark.parametrize("k", [1, 30, 333, 5000])
def test_quantized_rows_that_lie_apart_and_begin_anywhere(k, offset, extra):
    import torch
    rng = np.random.default_rng(k + offset)
    m, blocks = 6, -(-k // 32)
    a = make_x(rng, m, k)
    say(f"[case] quantize_mx4 k={k} offset={offset} extra={extra}")
    for dtype in (torch.float32, torch.bfloat16):
        flat = torch.full((offset + m * (k + extra) + 1,), float("inf"), dtype=dtype, device="cuda")
        x = torch.as_strided(flat, (m, k), (k + extra, 1), offset)
        x.copy_(dev(a))
        step, slabs = blocks * 16 + 16 * extra, -(-blocks // 8)
        slab = 8 * (m + extra)
        q = torch.full((m * step + 16,), 77, dtype=torch.uint8, device="cuda")
        s = torch.full((slabs * slab + 8,), 78, dtype=torch.uint8, device="cuda")
        P.pconv_quantize_mx4(x.data_ptr(), k + extra, "f32" if dtype == torch.float32 else "bf16", m, k, q.data_ptr(), step, s.data_ptr(), slab,
                             torch.cuda.current_stream().cuda_stream)
        want, ws = packed(*plain_quantize(x.float().cpu().numpy()))
        expect = np.full(q.numel(), 77, np.uint8)
        for r in range(m):
            expect[r * step:r * step + blocks * 16] = want[r]
        assert np.array_equal(q.cpu().numpy(), expect)
        expect = np.full(s.numel(), 78, np.uint8)
        for i in range(slabs):
            expect[i * slab:i * slab + 8 * m] = ws[i].ravel()
        assert np.array_equal(s.cpu().numpy(), expect)


# ---- the product ---------------------------------------------------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 10, 512), (2, 3, 15), (1, 1000, 2048), (3, 17, 32), (15, 16, 33), (16, 15, 63), (17, 130, 64), (8, 33, 4097),
         (31, 257, 65), (32, 64, 1000), (33, 63, 257), (48, 100, 512), (63, 129, 128), (64, 128, 255), (65, 127, 320), (100, 1, 300),
         (127, 129, 256), (128, 128, 768), (129, 257, 383), (300, 64, 64), (1000, 40, 40), (257, 300, 1155), (513, 511, 511),
         (2000, 256, 64), (700, 520, 640), (5, 4000, 300), (4, 70, 20000), (70, 20, 9000), (16, 70, 25088), (9, 257, 12345), (2, 40, 70001)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product_and_layer_against_the_formula(m, n, k, dtype):
    import torch
    say(f"[case] matmul_mx4 / linear_mx4 {m}x{n}x{k} {dtype}")
    rng = np.random.default_rng(m * 1000003 + n * 1009 + k)
    x, v = as_type(make_x(rng, m, k), dtype)
    w, bias = make_layer4(rng, n, k, 4), rng.standard_normal(n).astype(np.float32)
    relu = (m + n + k) % 2 == 0
    a = plain_quantize(v)
    want, bound = plain_product(a, w, bias, relu)
    wd, sd = on_card(w)
    y = P.linear_mx4(x, wd, sd, dev(bias), relu=relu)
    assert y.dtype == x.dtype
    check(y, want, bound, "linear_mx4")
    z = P.matmul_mx4(*on_card(a), wd, sd, dev(bias), relu=relu, out_dtype=x.dtype)
    assert torch.equal(y, z), "the call in one gives other values than the two calls"
    other = torch.bfloat16 if dtype == "f32" else torch.float32
    want, bound = plain_product(a, w, None, not relu)
    check(P.linear_mx4(x, wd, sd, relu=not relu, out_dtype=other), want, bound, "linear_mx4, no bias")


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(17, 40, 4096), (32, 130, 4095), (31, 16, 1023), (32, 40, 1024), (32, 40, 1025), (16, 50, 8190), (4, 300, 25088), (6, 40, 25088),
                                   (7, 40, 25088), (32, 4100, 512), (20, 9000, 200), (30, 33, 4700), (2, 50, 65536), (2, 50, 65537)])
def test_few_rows(m, n, k):
    """One or two groups of 16 rows, two or three turns of weights under way, quantised by all workgroups or by a launch; the largest that fit and the
    first that do not."""
    test_product_and_layer_against_the_formula(m, n, k, "f32")
    test_product_and_layer_against_the_formula(m, n, k, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 40, 12000), (16, 33, 2048), (40, 40, 12000), (100, 200, 5000), (300, 300, 2000), (1000, 1000, 700), (600, 2100, 900)])
def test_sums_of_equal_scales_are_exact(m, n, k):
    """All scales alike: every partial sum is a whole number of quarters, so that the order of nothing counts."""
    say(f"[case] matmul_mx4 exact {m}x{n}x{k}")
    rng = np.random.default_rng(k)
    a, b = make_layer4(rng, m, k), make_layer4(rng, n, k)
    assert exact_in_fp32(a, b)
    want, _ = plain_product(a, b, None, False)
    check(P.matmul_mx4(*on_card(a), *on_card(b)), want, np.zeros_like(want), "matmul_mx4")


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 5, 20, 100, 300])
@pytest.mark.parametrize("block", [0, 1, 2, 5, 7, 8, 15, 18])
def test_each_block_meets_its_own_scales(m, block):
    """One block alone holds values; its scales differ from all others'."""
    n, k = 70, 19 * 32
    rng = np.random.default_rng(block)
    say(f"[case] matmul_mx4 block {block} of m={m}")
    ops = []
    for rows in (m, n):
        codes, scales = make_layer4(rng, rows, k, 6)
        codes.reshape(rows, 19, 32)[:, np.arange(19) != block] = 0
        scales[:, block] = rng.integers(100, 150, rows)
        ops.append((codes, scales))
    want = values(*ops[0]) @ values(*ops[1]).T           # (32 terms at one scale: exact)
    check(P.matmul_mx4(*on_card(ops[0]), *on_card(ops[1])), want, np.zeros_like(want), "matmul_mx4")


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(7900, 4000, 592), (5000, 1030, 1056), (40_000, 200, 320), (1024, 4096, 2304)])
def test_many_tiles(m, n, k):
    """Products whose tiles fill the card, against 64 bits on the card."""
    import torch
    say(f"[case] matmul_mx4 {m}x{n}x{k}")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m + k)
    table = torch.tensor(VALUES, device="cuda")
    made = []
    for rows in (m, n):
        blocks = -(-k // 32)
        q = torch.randint(0, 256, (rows, blocks * 16), generator=gen, device="cuda", dtype=torch.uint8)
        if k % 32:
            q[:, k // 2:] = 0
        s = torch.randint(124, 127, (-(-blocks // 8), rows, 8), generator=gen, device="cuda", dtype=torch.uint8)
        v = torch.stack([table[(q & 15).long()], table[(q >> 4).long()]], 2).view(rows, blocks, 32)
        power = s.permute(1, 0, 2).reshape(rows, -1)[:, :blocks].double() - 127
        made.append((q, s, (v * torch.exp2(power)[:, :, None]).view(rows, -1)))
    (a, sa, va), (b, sb, vb) = made
    assert 36 * k < 2 ** (24 - 2 - 4)                    # (exponents differ by four together: sums are exact)
    want = va @ vb.t().contiguous()
    for dtype in (torch.float32, torch.bfloat16):
        y = P.matmul_mx4(a, sa, b, sb, out_dtype=dtype)
        assert torch.equal(y, want.to(torch.float32).to(dtype)), dtype
        assert torch.equal(P.matmul_mx4(a, sa, b, sb, relu=True, out_dtype=dtype), y.clamp(min=0))


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1, 20, 70), (5, 33, 300), (40, 50, 800), (130, 140, 2600), (300, 130, 64)])
def test_parts_of_operands_and_outputs_that_lie_apart(m, n, k):
    """Rows cut out of wider and longer operands, an output between other rows."""
    import torch
    say(f"[case] matmul_mx4 views {m}x{n}x{k}")
    rng = np.random.default_rng(m + n + k)
    a, b = make_layer4(rng, m + 5, k + 64, 2), make_layer4(rng, n + 3, k + 64, 2)
    wide = -(-k // 32)
    cut = lambda op, first, rows: (op[0][first:first + rows, :wide * 32], op[1][first:first + rows, :wide])
    want, bound = plain_product(cut(a, 2, m), cut(b, 3, n), None, False)
    (ad, asd), (bd, bsd) = on_card(a), on_card(b)
    slabs = -(-wide // 8)
    if wide % 8:                                         # behind the last block lies what does not count
        asd[slabs - 1, :, wide % 8:] = 255
        bsd[slabs - 1, :, wide % 8:] = 255
    ys = torch.full((m, n + 6), 7.0, device="cuda")
    y = P.matmul_mx4(ad[2:2 + m, :wide * 16], asd[:slabs, 2:2 + m], bd[3:3 + n, :wide * 16], bsd[:slabs, 3:3 + n], out=ys[:, 1:n + 1])
    check(y, want, bound, "matmul_mx4")
    assert bool((ys[:, 0] == 7).all()) and bool((ys[:, n + 1:] == 7).all())
    x = dev(make_x(rng, m, k + 3))[:, 1:k + 1]
    av = plain_quantize(np.ascontiguousarray(x.cpu().numpy()))
    want, bound = plain_product(av, cut(b, 3, n), None, True)
    check(P.linear_mx4(x, bd[3:3 + n, :wide * 16], bsd[:slabs, 3:3 + n], relu=True), want, bound, "linear_mx4")


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(6, 20, 40), (20, 20, 40), (100, 70, 600), (16, 40, 3000)])
def test_rows_of_zeros_infinities_and_nan(m, n, k):
    say(f"[case] linear_mx4 odd rows {m}x{n}x{k}")
    rng = np.random.default_rng(m)
    x = make_x(rng, m, k)
    x[0] = 0; x[2, 3] = np.inf; x[3, k - 1] = np.nan; x[5] *= np.float32(1e-30)
    w, bias = make_layer4(rng, n, k, 2), rng.standard_normal(n).astype(np.float32)
    w[1][7, 0] = 255                                     # a weight that is none
    a = plain_quantize(x)
    for relu in (False, True):
        want, bound = plain_product(a, w, bias, relu)
        assert np.isnan(want[2:4]).all() and np.isnan(want[:, 7]).all()
        check(P.linear_mx4(dev(x), *on_card(w), dev(bias), relu=relu), want, bound, f"linear_mx4 relu={relu}")


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 20, 300])
def test_scales_of_all_sizes(m):
    """Exponents so far apart that sums are infinite, and so small that they are zero or denormal."""
    say(f"[case] matmul_mx4 scales m={m}")
    n, k = 40, 64
    one = np.zeros((m, 64), np.uint8)
    one[:, 5], one[:, 40] = 7, 2                         # 6 and 1
    two = np.zeros((n, 64), np.uint8)
    two[:, 5], two[:, 40] = 2, 7
    for ea, eb in ((0, 254), (254, 0), (0, 0), (254, 254), (60, 60), (1, 120)):
        a, b = (one, np.full((m, 2), ea, np.uint8)), (two, np.full((n, 2), eb, np.uint8))
        got = P.matmul_mx4(*on_card(a), *on_card(b)).cpu().numpy()
        with np.errstate(over="ignore"):
            want = np.float32(12 * 2.0 ** (ea + eb - 254))
        assert (got == want).all(), (ea, eb, got[0, 0], want)


@pytest.mark.gpu
def test_sizes_of_zero():
    import torch
    say("[case] 4-bit layers, sizes of zero")
    rng = np.random.default_rng(0)
    w, s = on_card(make_layer4(rng, 20, 8))
    bias = dev(rng.standard_normal(20).astype(np.float32))
    for m in (0, 3, 100):
        y = P.linear_mx4(torch.zeros(m, 8, device="cuda"), w, s, bias, relu=True)
        assert y.shape == (m, 20) and torch.equal(y, bias.clamp(min=0).expand(m, 20))
        q, sq = P.quantize_mx4(torch.zeros(m, 0, device="cuda"))
        assert q.shape == (m, 0) and sq.shape == (0, m, 8)
        y = P.linear_mx4(torch.zeros(m, 0, device="cuda"), w[:, :0], s[:0], bias)
        assert torch.equal(y, bias.expand(m, 20))
        assert torch.equal(P.matmul_mx4(q, sq, w[:, :0], s[:0]), torch.zeros(m, 20, device="cuda"))
        assert P.linear_mx4(torch.zeros(m, 8, device="cuda"), w[:0], s[:, :0]).shape == (m, 0)


@pytest.mark.gpu
def test_leading_dimensions_are_rows():
    import torch
    say("[case] linear_mx4 on [2, 5, 7, 72]")
    rng = np.random.default_rng(3)
    x = make_x(rng, 70, 72)
    w = make_layer4(rng, 40, 72, 2)
    want, bound = plain_product(plain_quantize(x), w, None, False)
    y = P.linear_mx4(dev(x).view(2, 5, 7, 72), *on_card(w))
    assert y.shape == (2, 5, 7, 40)
    check(y, want, bound, "linear_mx4")
    q, s = P.quantize_mx4(dev(x).view(2, 5, 7, 72))
    assert q.shape == (2, 5, 7, 48) and s.shape == (1, 70, 8)
    check(P.matmul_mx4(q, s, *on_card(w)), want, bound, "matmul_mx4")
    one = P.linear_mx4(dev(x)[4], *on_card(w))
    assert one.shape == (40,) and torch.equal(one, P.linear_mx4(dev(x)[4:5], *on_card(w))[0])


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(1030, 24, 48), (40, 24, 48), (600, 300, 520)])
def test_offsets_beyond_32_bits(m, n, k):
    """Rows of a, x and y, and slabs, that lie so far apart that the last ones are beyond 2^32 bytes."""
    import torch
    say(f"[case] matmul_mx4 far rows {m}x{n}x{k}")
    rng = np.random.default_rng(m)
    w, x = make_layer4(rng, n, k, 2), make_x(rng, m, k)
    a = plain_quantize(x)
    want, bound = plain_product(a, w, None, False)
    (q, s), (wd, sd) = on_card(a), on_card(w)
    step = min(1 << 23, (1 << 32) // (m - 1) // 16 * 16 + 64)
    room = torch.empty((m - 1) * step + q.shape[1], dtype=torch.uint8, device="cuda")
    far = torch.as_strided(room, q.shape, (step, 1))
    far.copy_(q)
    check(P.matmul_mx4(far, s, wd, sd), want, bound, "far rows of a")
    del room, far
    if s.shape[0] > 1:
        apart = (1 << 32) // (s.shape[0] - 1) // 8 * 8 + 64
        room = torch.empty((s.shape[0] - 1) * apart + 8 * m, dtype=torch.uint8, device="cuda")
        far = torch.as_strided(room, s.shape, (apart, 8, 1))
        far.copy_(s)
        check(P.matmul_mx4(q, far, wd, sd), want, bound, "far slabs of a")
        room = torch.empty((s.shape[0] - 1) * apart + 8 * n, dtype=torch.uint8, device="cuda")
        far = torch.as_strided(room, sd.shape, (apart, 8, 1))
        far.copy_(sd)
        check(P.matmul_mx4(q, s, wd, far), want, bound, "far slabs of b")
        del room, far
    step = (1 << 30) // (m - 1) + 16
    room = torch.empty((m - 1) * step + max(n, k), dtype=torch.float32, device="cuda")
    xs = torch.as_strided(room, (m, k), (step, 1))
    xs.copy_(dev(x))
    check(P.linear_mx4(xs, wd, sd), want, bound, "far rows of x")
    check(P.matmul_mx4(q, s, wd, sd, out=torch.as_strided(room, (m, n), (step, 1))), want, bound, "far rows of y")


@pytest.mark.gpu
@pytest.mark.parametrize("m", [2, 40, 300])
def test_another_stream_and_equal_bits(m):
    import torch
    say(f"[case] linear_mx4 on another stream m={m}")
    rng = np.random.default_rng(m)
    x, (w, s) = dev(make_x(rng, m, 5000, 2.0)), on_card(make_layer4(rng, 200, 5000, 9))
    want = P.linear_mx4(x, w, s)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    late = torch.zeros_like(x)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        big = torch.randn(3000, 3000, device="cuda")
        for _ in range(5):
            big = big @ big * 1e-3
        late.copy_(x)
        y = P.linear_mx4(late, w, s)
    stream.synchronize()
    assert torch.equal(y, want)
    for _ in range(3):
        assert torch.equal(P.linear_mx4(x, w, s), want)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 40, 300])
def test_replays_of_a_captured_layer(m):
    import torch
    say(f"[case] linear_mx4 captured m={m}")
    rng = np.random.default_rng(m)
    (w, s), (v, t) = on_card(make_layer4(rng, 320, 5000, 2)), on_card(make_layer4(rng, 100, 320, 2))
    x = torch.zeros(m, 5000, device="cuda")
    out = torch.empty(m, 320, device="cuda")
    P.linear_mx4(x, w, s, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.linear_mx4(x, w, s, relu=True, out=out)
        z = P.linear_mx4(out, v, t)
    for i in range(4):
        x.copy_(dev(make_x(rng, m, 5000)))
        g.replay()
        torch.cuda.synchronize()
        want = P.linear_mx4(x, w, s, relu=True)
        assert torch.equal(out, want) and torch.equal(z, P.linear_mx4(want, v, t)), f"replay {i}"


@pytest.mark.gpu
def test_written_outputs_count_as_changed():
    import torch
    rng = np.random.default_rng(1)
    w, s = on_card(make_layer4(rng, 8, 40))
    out = torch.zeros(3, 8, device="cuda")
    before = out._version
    P.linear_mx4(dev(make_x(rng, 3, 40)), w, s, out=out)
    assert out._version > before


@pytest.mark.gpu
def test_ordinary_calls_and_the_long_way_give_the_same():
    """Ordinary calls are made in native code; an output given, a type asked for or a step of its own go the long way."""
    import torch
    rng = np.random.default_rng(6)
    for m, n, k in ((1, 40, 200), (30, 70, 333), (300, 100, 1000)):
        say(f"[case] both ways {m}x{n}x{k}")
        (w, s), x, bias = on_card(make_layer4(rng, n, k, 3)), dev(make_x(rng, m, k)), dev(rng.standard_normal(n).astype(np.float32))
        y = P.linear_mx4(x, w, s, bias, relu=True)
        assert torch.equal(y, P.linear_mx4(x, w, s, bias, True, out=torch.empty_like(y))) and torch.equal(y, P.linear_mx4(x, w, s, bias, True, torch.float32))
        q, sq = P.quantize_mx4(x)
        q3, sq3 = P.quantize_mx4(torch.nn.functional.pad(x, (0, 3))[:, :k].unsqueeze(1).expand(m, 1, k))
        assert torch.equal(q, q3.view_as(q)) and torch.equal(sq, sq3)
        assert torch.equal(y, P.matmul_mx4(q, sq, w, s, bias, True)) and torch.equal(y, P.matmul_mx4(q, sq, w, s, bias, True, out=torch.empty_like(y)))
        wide = torch.zeros(n, w.shape[1] + 32, dtype=torch.uint8, device="cuda")
        wide[:, :w.shape[1]] = w
        assert torch.equal(y, P.linear_mx4(x, wide[:, :w.shape[1]], s, bias, relu=True))
        with pytest.raises(RuntimeError):
            P.linear_mx4(x, w, s, bias, relu=torch.ones(3))


@pytest.mark.gpu
@pytest.mark.parametrize("lead", [(7,), (3, 5), (2, 1, 20)])
def test_long_rows_lie_a_multiple_of_128_bytes_apart(lead):
    """1008 bytes of values end where the next row begins; of 1024 and more there may be room between."""
    import torch
    rng = np.random.default_rng(len(lead))
    for k in (2016, 2048, 2049, 2100):
        say(f"[case] steps of rows {lead} {k}")
        blocks, rows = -(-k // 32), int(np.prod(lead))
        x = make_x(rng, rows, k)
        q, s = P.quantize_mx4(dev(x).view(*lead, k))
        wide = 16 * blocks
        assert q.shape == (*lead, wide) and q.stride(-2) == (wide if wide < 1024 else -(-wide // 128) * 128)
        want = P.quantize_mx4(torch.nn.functional.pad(dev(x), (0, 1))[:, :k])
        assert torch.equal(q.reshape(rows, wide), want[0]) and torch.equal(s, want[1])
        (w, ws), y = on_card(make_layer4(rng, 40, k, 3)), torch.empty(*lead, 40, device="cuda")
        assert torch.equal(P.matmul_mx4(q, s, w, ws), P.matmul_mx4(q.contiguous(), s, w.contiguous(), ws, out=y))
        assert torch.equal(y, P.linear_mx4(dev(x).view(*lead, k), w, ws))


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(70, 290, 200), (300, 401, 70), (1100, 515, 600), (3000, 1101, 64), (9000, 1299, 96)])
def test_bf16_outputs_that_begin_within_a_word(m, n, k):
    """Rows an odd number of elements apart, and all of them at odd places: the same sums as in fp32, rounded, and nothing beside them."""
    import torch
    rng = np.random.default_rng(n)
    (w, ws), x, bias = on_card(make_layer4(rng, n, k, 3)), dev(make_x(rng, m, k)), dev(rng.standard_normal(n).astype(np.float32))
    q, s = P.quantize_mx4(x)
    want = P.matmul_mx4(q, s, w, ws, bias, True).bfloat16()
    for step, first in ((n | 1, 0), ((n | 1) + 1, 1), (n + 7 | 1, 1), (n + 8, 2)):
        say(f"[case] bf16 rows {m}x{n}x{k} {step} apart from {first} on")
        room = torch.full((m * step + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
        out = room[first:first + m * step].view(m, step)[:, :n]
        assert P.matmul_mx4(q, s, w, ws, bias, True, out=out) is out and torch.equal(out, want)
        out.fill_(7.0)
        assert bool((room == 7.0).all())


# ---- plans ---------------------------------------------------------------------------------------------------------------

FORMS = {(1, 0, 0, False): (9, 40, 256), (2, 32, 1, False): (129, 11206, 64), (2, 32, 1, True): (1, 9309, 22924), (2, 32, 2, False): (40, 64, 256),
         (2, 32, 2, True): (40, 33, 10096), (2, 64, 1, False): (145, 18962, 40), (2, 64, 1, True): (33, 9394, 32445), (2, 64, 2, False): (8395, 9, 562),
         (2, 64, 2, True): (2105, 20, 9403), (2, 128, 1, False): (34014, 20, 64), (2, 128, 1, True): (17908, 15, 19019),
         (2, 128, 2, False): (17004, 2, 1026), (2, 128, 2, True): (4750, 20, 19083), (2, 256, 1, False): (41430, 130, 64),
         (2, 256, 1, True): (773, 1782, 152295)}


def form_of(m, n, k):
    p = P.pconv_debug_mx4_plan(m, n, -(-k // 32))
    return p.kernel, p.tile_m, p.sets, p.splits > 1


@pytest.mark.gpu
@pytest.mark.parametrize("form", FORMS)
def test_every_form_of_the_product(form):
    """Equal scales: sums are exact, whoever adds them."""
    import torch
    m, n, k = FORMS[form]
    say(f"[case] matmul_mx4 {m}x{n}x{k}, form {form}")
    assert form_of(m, n, k) == form
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m + k)
    table = torch.tensor(VALUES, device="cuda")
    made = []
    for rows in (m, n):
        blocks = -(-k // 32)
        q = torch.randint(0, 256, (rows, blocks * 16), generator=gen, device="cuda", dtype=torch.uint8)
        q[:, (k + 1) // 2:] = 0
        if k % 2:
            q[:, k // 2] &= 15
        s = torch.full((-(-blocks // 8), rows, 8), 125, dtype=torch.uint8, device="cuda")
        made.append((q, s, torch.stack([table[(q & 15).int()], table[(q >> 4).int()]], 2).view(rows, -1) / 4))
    (a, sa, va), (b, sb, vb) = made
    bias = torch.randn(n, generator=gen, device="cuda")
    want = va @ vb.t().contiguous()
    assert torch.equal(P.matmul_mx4(a, sa, b, sb), want.float())
    want = (want.float() + bias).clamp(min=0).bfloat16()
    assert torch.equal(P.matmul_mx4(a, sa, b, sb, bias, relu=True, out_dtype=torch.bfloat16), want)


def test_plans_of_the_products():
    for form, size in FORMS.items():
        assert form_of(*size) == form
    for m, n, blocks in ((0, 1, 1), (1, 0, 1), (1, 1, -1), ((1 << 30) + 1, 1, 1), (1, 1, (1 << 19) + 1)):
        with pytest.raises(P.PconvError):
            P.pconv_debug_mx4_plan(m, n, blocks)


# ---- refusals ------------------------------------------------------------------------------------------------------------

def c_calls():
    """(what is wrong, call) for raw calls that return before anything is launched; no pointer is followed."""
    p = 1 << 20
    yield "rows must", lambda: P.pconv_quantize_mx4(p, 8, "f32", -1, 8, p, 16, p, 16)
    yield "cols", lambda: P.pconv_quantize_mx4(p, 1 << 25, "f32", 1, (1 << 24) + 1, p, 1 << 24, p, 16)
    yield "null", lambda: P.pconv_quantize_mx4(0, 8, "f32", 2, 8, p, 16, p, 16)
    yield "null", lambda: P.pconv_quantize_mx4(p, 8, "f32", 2, 8, 0, 16, p, 16)
    yield "null", lambda: P.pconv_quantize_mx4(p, 8, "f32", 2, 8, p, 16, 0, 16)
    yield "apart", lambda: P.pconv_quantize_mx4(p, 7, "f32", 2, 8, p, 16, p, 16)
    yield "apart", lambda: P.pconv_quantize_mx4(p, 64, "f32", 2, 64, p, 16, p, 16)
    yield "16 bytes", lambda: P.pconv_quantize_mx4(p, 8, "f32", 2, 8, p, 24, p, 16)
    yield "16 bytes", lambda: P.pconv_quantize_mx4(p, 8, "f32", 2, 8, p + 8, 16, p, 16)
    yield "8 bytes", lambda: P.pconv_quantize_mx4(p, 8, "f32", 2, 8, p, 16, p + 4, 16)
    yield "8 bytes", lambda: P.pconv_quantize_mx4(p, 8, "f32", 2, 8, p, 16, p, 20)
    yield "a row apart", lambda: P.pconv_quantize_mx4(p, 8, "f32", 2, 8, p, 16, p, 8)
    yield "8 MiB", lambda: P.pconv_quantize_mx4(p, 8, "f32", 2, 8, p, (1 << 23) + 16, p, 16)
    good = dict(a=p, lda=32, sa=p, slab_a=32, b=p, ldb=32, sb=p, slab_b=32, bias=0, y=p, ldy=4, t="f32", m=4, n=4, blocks=2)
    wrong = [("m and n", dict(m=-1)), ("m and n", dict(n=(1 << 30) + 1)), ("blocks must", dict(blocks=-1)), ("blocks must", dict(blocks=(1 << 19) + 1)),
             ("apart", dict(lda=16)), ("apart", dict(ldb=16)), ("apart", dict(ldy=3)), ("a row apart", dict(slab_a=24)), ("a row apart", dict(slab_b=24)),
             ("null", dict(a=0)), ("null", dict(b=0)), ("null", dict(sa=0)), ("null", dict(sb=0)), ("null", dict(y=0)), ("16 bytes", dict(a=p + 8)),
             ("16 bytes", dict(ldb=40)), ("8 bytes", dict(sb=p + 4)), ("8 MiB", dict(lda=1 << 24))]
    for what, change in wrong:
        yield what, lambda change=change: P.pconv_matmul_mx4(*{**good, **change}.values())
    need = P.pconv_linear_mx4_workspace(40, 40, 26000)
    assert need >= 40 * 13000
    layer = lambda work, have, x=p, k=26000: P.pconv_linear_mx4(x, k, "f32", p, 13008, p, 320, 0, p, 40, "f32", 40, 40, k, False, work, have)
    yield "work space", lambda: layer(p, need - 1)
    yield "work space", lambda: layer(0, need)
    yield "work space", lambda: layer(p + 8, need)
    yield "null", lambda: layer(p, need, x=0)
    yield "k must", lambda: layer(p, need, k=(1 << 24) + 1)


def test_c_entries_refuse_what_they_cannot_run():
    for what, call in c_calls():
        with pytest.raises(P.PconvError) as e:
            call()
        assert e.value.status == P.INVALID_ARG and what in str(e.value), (what, str(e.value))


def test_unknown_types_are_refused_at_the_c_entries():
    p = 1 << 20
    L = P.lib()
    assert L.pconv_quantize_mx4(p, 8, 7, 2, 8, p, 16, p, 16, None) == P.INVALID_ARG
    assert L.pconv_matmul_mx4(p, 32, p, 32, p, 32, p, 32, None, p, 4, 7, 4, 4, 2, 0, None, 0, None) == P.INVALID_ARG
    assert L.pconv_linear_mx4(p, 64, 7, p, 32, p, 32, None, p, 4, 0, 4, 4, 64, 0, None, 0, None) == P.INVALID_ARG


def test_calls_of_more_than_2_to_32_threads_are_unsupported():
    p, big = 1 << 20, 1 << 30
    for m, n in ((big, 1 << 20), (1 << 20, big), (1, big), (16, big)):
        with pytest.raises(P.PconvError) as e:
            P.pconv_matmul_mx4(p, 512, p, 8 * m, p, 512, p, 8 * n, 0, p, n, "f32", m, n, 32, False, p, P.pconv_matmul_mx4_workspace(m, n, 32))
        assert e.value.status == P.UNSUPPORTED and "too many workgroups" in str(e.value)


def test_calls_on_the_host_are_refused():
    import torch
    x, w, s = torch.zeros(4, 32), torch.zeros(3, 16, dtype=torch.uint8), torch.zeros(1, 3, 8, dtype=torch.uint8)
    for call in (lambda: P.quantize_mx4(x), lambda: P.linear_mx4(x, w, s), lambda: P.matmul_mx4(w, s, w, s)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


@pytest.mark.gpu
def test_wrong_tensors_are_refused():
    import torch
    z = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")
    u8 = torch.uint8
    x, w, s, b, q, sq = z(4, 40), z(3, 32, dtype=u8), z(1, 3, 8, dtype=u8), z(3), z(4, 32, dtype=u8), z(1, 4, 8, dtype=u8)
    bad = [lambda: P.quantize_mx4(x.half()), lambda: P.quantize_mx4(x.t()), lambda: P.quantize_mx4(z(1, 8).expand(4, 8)),
           lambda: P.linear_mx4(x, w.float(), s), lambda: P.linear_mx4(x, w[:, :16], s), lambda: P.linear_mx4(x, w, s.int()),
           lambda: P.linear_mx4(z(4, 65), w, s), lambda: P.linear_mx4(z(4, 32), w, s), lambda: P.linear_mx4(x, w, s[:, :2]),
           lambda: P.linear_mx4(x, w, s.transpose(0, 1)), lambda: P.linear_mx4(x, w, s.expand(2, 3, 8)), lambda: P.linear_mx4(x, w, s, b[:2]),
           lambda: P.linear_mx4(x, w, s, b, out=z(4, 4)), lambda: P.linear_mx4(x, w, s, b, out=z(4, 3), out_dtype=torch.bfloat16),
           lambda: P.linear_mx4(x, w, s, b.cpu()), lambda: P.linear_mx4(x, w, s, out=z(3, 4).t()), lambda: P.linear_mx4(x, w.view(-1), s),
           lambda: P.matmul_mx4(q, s, w, s), lambda: P.matmul_mx4(q, sq, q[:, :16], sq), lambda: P.matmul_mx4(x, sq, w, s),
           lambda: P.matmul_mx4(q, z(1, 4, 16, dtype=u8)[:, :, ::2], w, s), lambda: P.matmul_mx4(q[:, :17], sq, w, s),
           lambda: P.matmul_mx4(q, sq, w, s, out=z(4, 3, dtype=torch.float64))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    room = z(4, 64)
    over = [lambda: P.linear_mx4(room[:, :40], w, s, out=room[:, 38:41]), lambda: P.linear_mx4(x[:1], w, s, b, out=b.view(1, 3)),
            lambda: P.matmul_mx4(q, sq, w, s, out=q.view(-1).view(torch.float32)[:12].view(4, 3)),
            lambda: P.matmul_mx4(q[:1], sq[:, :1], w, s, out=sq.view(-1).view(torch.float32)[:3].view(1, 3)),
            lambda: P.matmul_mx4(q, sq, w, s, out=w.view(-1).view(torch.float32)[:12].view(4, 3))]
    for i, call in enumerate(over):
        with pytest.raises(ValueError, match="overlap"):
            call()
            pytest.fail(f"call {i} was not refused")
