"""Every form of the tiled product of 8-bit integers: each tile, with one set of waves and with two, with k whole and split, over lengths
that end with a stage of 128 bytes, with a piece of 16 and inside one; and rows that lie as far apart as its 32-bit offsets reach.

Against 64 bits on the card, with the bounds of test_i8_layers.py."""
import math
import random

import pytest

import paper_1909_05073_amd as P

from gpu_util import say

U = 2.0 ** -24

# (rows of a tile, sets of waves, whether k is split): sizes m, n, k
FORMS = {
    (32, 1, False): [(20, 40000, 1024), (1223, 1579, 560), (334, 5776, 515)],
    (32, 1, True): [(20, 4110, 16000), (19, 2234, 31984), (18, 4171, 16063)],
    (32, 2, False): [(18, 202, 640), (20, 207, 528), (18, 201, 547)],
    (32, 2, True): [(21, 209, 3968), (18, 202, 2992), (27, 207, 3005)],
    (64, 1, False): [(908, 4105, 640), (518, 6578, 528), (3387, 1161, 518)],
    (64, 1, True): [(1034, 385, 21632), (1453, 257, 17184), (1488, 258, 19310)],
    (64, 2, False): [(512, 4096, 4096), (2073, 418, 544), (2079, 392, 549)],
    (64, 2, True): [(600, 64, 8320), (335, 270, 4160), (355, 261, 4102)],
    (128, 1, False): [(5502, 1025, 640), (4960, 1187, 528), (2190, 2713, 542)],
    (128, 1, True): [(1676, 262, 75776), (1690, 281, 83088), (1692, 259, 83254)],
    (128, 2, False): [(1000, 4096, 4096), (2739, 667, 544), (1508, 1329, 529)],
    (128, 2, True): [(687, 257, 26496), (695, 268, 24160), (1378, 269, 15203)],
    (256, 1, False): [(3467, 3470, 640), (7195, 1714, 528), (4774, 2563, 526)],
    (256, 1, True): [(6299, 132, 69632), (6494, 138, 89664), (6454, 132, 78151)],
}
CASES = [(form, size) for form, sizes in FORMS.items() for size in sizes]


def form_of(m, n, k):
    p = P.pconv_debug_i8_plan(m, n, k)
    return (p.tile_m, p.sets, p.splits > 1) if p.kernel == 3 else None


def test_the_sizes_take_the_forms_that_they_are_here_for():
    for form, sizes in FORMS.items():
        assert all(form_of(*size) == form for size in sizes), form
        assert [(k % 128 == 0, k % 16 == 0) for _, _, k in sizes] == [(True, True), (False, True), (False, False)], form


def test_no_size_takes_another_form():
    rng = random.Random(0)
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    seen = {form_of(spread(1, 1 << 20), spread(1, 1 << 17), spread(1, 131071)) for _ in range(20_000)}
    assert seen - {None} <= set(FORMS)


def test_plans_of_other_kernels_and_refusals():
    assert P.pconv_debug_i8_plan(16, 4096, 8192).kernel == 1 and P.pconv_debug_i8_plan(17, 4096, 512).kernel == 2
    for m, n, k in ((0, 1, 1), (1, 0, 1), (1, 1, -1), (1 << 31, 1, 1), (1, 1, 131072)):
        with pytest.raises(P.PconvError):
            P.pconv_debug_i8_plan(m, n, k)


def rows(values, step):
    """The int8 matrix, its rows `step` bytes apart; the last ends with the memory."""
    import torch
    m, k = values.shape
    room = torch.empty((m - 1) * step + k, dtype=torch.int8, device="cuda")
    if room.numel() < 1 << 31:
        room.fill_(101)                                  # what lies between would show
    t = room.as_strided((m, k), (step, 1))
    t.copy_(values)
    return t


def operands(m, n, k):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m * 31 + n * 7 + k)
    i8 = lambda *shape: torch.randint(-127, 128, shape, generator=gen, device="cuda", dtype=torch.int8)
    some = lambda size: torch.rand(size, generator=gen, device="cuda") + 0.01
    return i8(m, k), some(m), i8(n, k), some(n), torch.randn(n, generator=gen, device="cuda")


def compare(a, sa, b, sb, bias, ra, rb):
    """Products of the rows ra and rb against the matrices a and b that they hold."""
    import torch
    acc = torch.matmul(a.double(), b.double().t().contiguous())      # (whole numbers below 2^53: exact)
    scaled = acc * sa.double()[:, None] * sb.double()
    want = scaled + bias.double()
    bound = 4 * U * (scaled.abs() + bias.double().abs())
    for dtype in (torch.float32, torch.bfloat16):
        tol = bound if dtype == torch.float32 else bound * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs() * (1 + 2.0 ** -8)
        y = P.matmul_i8(ra, sa, rb, sb, bias, out_dtype=dtype)
        wrong = (y.double() - want).abs() > tol
        assert not bool(wrong.any()), f"{dtype}: {int(wrong.sum())} of {wrong.numel()} outside, first at {wrong.nonzero()[0].tolist()}"
        assert torch.equal(P.matmul_i8(ra, sa, rb, sb, bias, relu=True, out_dtype=dtype), y.clamp(min=0))


@pytest.mark.gpu
@pytest.mark.parametrize("form,size", CASES, ids=lambda v: "x".join(map(str, v)))
def test_product_in_each_form(form, size):
    import torch
    m, n, k = size
    say(f"[case] matmul_i8 {m}x{n}x{k}: tile {form[0]}, {form[1]} sets, split {form[2]}")
    assert form_of(m, n, k) == form
    a, sa, b, sb, bias = operands(m, n, k)
    step = (k + 15) // 16 * 16
    compare(a, sa, b, sb, bias, rows(a, step), rows(b, step + 16))
    if m * k <= 10_000_000:                              # the same through the call that quantises
        x = torch.randn(m, k, device="cuda")
        q, s = P.quantize_rows(x)
        for dtype in (torch.float32, torch.bfloat16):
            assert torch.equal(P.linear_i8(x, rows(b, step + 16), sb, bias, out_dtype=dtype), P.matmul_i8(q, s, b, sb, bias, out_dtype=dtype))


FAR = 1 << 23                                            # as far as rows may lie apart to be read by 32-bit offsets


@pytest.mark.gpu
@pytest.mark.parametrize("extra", [0, 16])
@pytest.mark.parametrize("k", [640, 528, 530])
@pytest.mark.parametrize("m,n", [(512, 32700), (32700, 512), (40, 200)])
def test_tiles_of_rows_8_mebibytes_apart(m, n, k, extra):
    """The last rows of a tile of 256 begin just below 2^31 bytes behind its first; 16 bytes more, and rows are copied together first."""
    say(f"[case] matmul_i8 {m}x{n}x{k}, rows {FAR + extra} apart")
    assert form_of(m, n, k) == ((256, 1, False) if m * n > 8000 else (32, 2, False))
    a, sa, b, sb, bias = operands(m, n, k)
    near = (k + 15) // 16 * 16
    compare(a, sa, b, sb, bias, rows(a, FAR + extra if m < 1000 else near), rows(b, FAR + extra if n < 1000 else near))


@pytest.mark.gpu
@pytest.mark.parametrize("extra", [0, 16])
@pytest.mark.parametrize("m,n,k", [(100, 136, 256), (100, 136, 500), (100, 136, 1040), (3, 40, 4112), (3, 40, 4100), (16, 40, 8192)])
def test_rings_of_weights_8_mebibytes_apart(m, n, k, extra):
    """Short rows and few rows, quantised within the product and before it."""
    import torch
    say(f"[case] linear_i8 {m}x{n}x{k}, weights {FAR + extra} apart")
    _, _, b, sb, bias = operands(m, n, k)
    x = torch.randn(m, k, device="cuda")
    most = x.abs().amax(1, keepdim=True)
    scale = most / torch.full_like(most, 127.0)
    q = (x / scale).round().to(torch.int8)
    far = rows(b, FAR + extra)
    compare(q, scale[:, 0].contiguous(), b, sb, bias, q, far)
    for dtype in (torch.float32, torch.bfloat16):
        assert torch.equal(P.linear_i8(x, far, sb, bias, out_dtype=dtype), P.matmul_i8(q, scale[:, 0].contiguous(), b, sb, bias, out_dtype=dtype))
