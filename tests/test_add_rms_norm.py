"""add_rms_norm_i8 against the formula in 64 bits.

Tolerances (U = 2^-24, half a step of fp32).  The sum of two numbers rounds once; the factor 1 / sqrt(mean + eps) comes from 64 bits
and rounds once; the two products once each: with the sum's own rounding in the mean (at most U of it) h is off by at most
5 U |h| + U (|x| + |r|) f |w|, where x and r cancel.  The scale, the largest |h| over 127 rounded once, is off by the largest
of those bounds over 127 and by U.  A whole number is off by 1/2 and what these do to h / scale; the rounded sum is the nearest."""
import numpy as np
import pytest

import paper_1909_05073_amd as P

from gpu_util import say
from test_i8_layers import as_type, check, dev, make_layer8, plain_product

U = 2.0 ** -24


def plain_norm(x, r, w, eps):
    """fp64 arrays: (s, h, bound of h's error)."""
    s = x if r is None else x + r
    f = 1 / np.sqrt((s * s).mean(1, keepdims=True) + eps)
    w = np.ones(x.shape[1]) if w is None else w.astype(np.float64)
    h = s * f * w
    size = np.abs(x) if r is None else np.abs(x) + np.abs(r)
    # (the mean moves by at most the largest relative change of the sums' squares, weighted: 2 U mean(size |s|))
    moved = U * (size * np.abs(s)).mean(1, keepdims=True) * f * f
    return s, h, (5 * U + moved) * np.abs(h) + U * size * f * np.abs(w) + 2.0 ** -140


def check_norm(got, x, r, w, eps, dtype):
    """x, r: fp32 arrays of what the tensors hold."""
    import torch
    q, scale, s = got
    m, k = x.shape
    want_s, h, off = plain_norm(x.astype(np.float64), None if r is None else r.astype(np.float64), w, eps)
    if r is not None:
        nearest = torch.from_numpy(x + r).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        assert torch.equal(s.cpu().reshape(m, k), nearest), "sums"
    most = np.abs(h).max(1, initial=0)
    scale = scale.cpu().numpy().astype(np.float64).reshape(m)
    off_scale = off.max(1, initial=0) / 127 + U * most / 127 + 2.0 ** -149
    assert (np.abs(scale - most / 127) <= off_scale).all(), "scales"
    q = q.cpu().numpy().astype(np.float64).reshape(m, k)
    assert (np.abs(q) <= 127).all()
    zero = scale == 0
    assert (q[zero] == 0).all()
    live = ~zero
    ratio = h[live] / scale[live, None]
    far = np.abs(q[live] - ratio) - 0.5 - off[live] / scale[live, None] - 2 * U * np.abs(ratio)
    assert (far <= np.maximum(0, np.abs(ratio) - 127)).all(), f"values: {far.max()}"


def make(rng, m, k):
    x = rng.standard_normal((m, k)) * np.exp(rng.uniform(-3, 3, (m, 1)))
    r = rng.standard_normal((m, k)) * np.exp(rng.uniform(-2, 3, (m, 1)))
    if m > 2:
        x[1] = r[1] = 0
    return x.astype(np.float32), r.astype(np.float32), rng.uniform(-2, 2, k).astype(np.float32)


SIZES = [(1, 1), (3, 2), (1, 7), (5, 8), (33, 9), (7, 31), (40, 32), (3, 63), (257, 64), (9, 100), (5, 255), (6, 257), (4, 513), (65, 1000),
         (3, 2049), (2, 4100), (3, 8191), (2, 16385), (1, 25088), (2, 40001), (2, 70001), (20_000, 24), (3000, 520)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k", SIZES)
def test_rows_against_the_formula(m, k, dtype):
    say(f"[case] add_rms_norm_i8 {m}x{k} {dtype}")
    rng = np.random.default_rng(m * 100003 + k)
    x, r, w = make(rng, m, k)
    (xd, xv), (rd, rv) = as_type(x, dtype), as_type(r, dtype)
    check_norm(P.add_rms_norm_i8(xd, rd, dev(w)), xv, rv, w, 1e-6, dtype)
    q, scale, s = P.add_rms_norm_i8(xd, weight=dev(w), eps=0.25)
    assert s is xd
    check_norm((q, scale, s), xv, None, w, 0.25, dtype)
    check_norm(P.add_rms_norm_i8(xd, rd, eps=1e-3), xv, rv, None, np.float32(1e-3), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [5, 200, 3000, 70_000])
def test_sums_in_an_operands_place(k, dtype):
    import torch
    say(f"[case] add_rms_norm_i8 in place k={k} {dtype}")
    x, r, w = make(np.random.default_rng(k), 4, k)
    (xd, xv), (rd, rv) = as_type(x, dtype), as_type(r, dtype)
    want = P.add_rms_norm_i8(xd, rd, dev(w))
    for which in (0, 1):
        ops = [xd.clone(), rd.clone()]
        before = ops[which]._version
        got = P.add_rms_norm_i8(*ops, dev(w), out=ops[which])
        assert got[2] is ops[which] and ops[which]._version > before
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    both = xd.clone()
    got = P.add_rms_norm_i8(both, both, dev(w), out=both)
    check_norm(got, xv, xv, w, 1e-6, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("offset,extra", [(0, 4), (1, 0), (3, 5), (2, 1)])
@pytest.mark.parametrize("k", [1, 30, 333, 5000])
def test_rows_that_lie_apart_and_begin_anywhere(k, offset, extra):
    import torch
    say(f"[case] add_rms_norm_i8 k={k} offset={offset} extra={extra}")
    m = 6
    x, r, w = make(np.random.default_rng(k + offset), m, k)

    def apart(a, dtype, add):
        step = k + extra + add
        flat = torch.full((offset + m * step + 1,), float("nan"), dtype=dtype, device="cuda")
        t = torch.as_strided(flat, (m, k), (step, 1), offset)
        t.copy_(dev(a))
        return flat, t
    for dtype, name in ((torch.float32, "f32"), (torch.bfloat16, "bf16")):
        _, xd = apart(x, dtype, 0)
        _, rd = apart(r, dtype, 3)
        flat, out = apart(np.zeros_like(x), dtype, 1)
        wd = torch.cat([torch.full((offset,), float("nan"), device="cuda"), dev(w)])[offset:]
        got = P.add_rms_norm_i8(xd, rd, wd, out=out)
        check_norm(got, xd.float().cpu().numpy(), rd.float().cpu().numpy(), w, 1e-6, name)
        out.fill_(float("nan"))
        assert bool(torch.isnan(flat).all()), "values outside the rows were written"


@pytest.mark.gpu
@pytest.mark.parametrize("behind", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [1, 2, 3, 4, 5, 6, 7, 8, 9, 15, 17, 130, 513])
def test_what_lies_behind_the_weight_is_nothing(k, dtype, behind):
    """Rows shorter than one vector of 16 bytes among them."""
    import torch
    rng = np.random.default_rng(500 + k)
    m = 5
    x, r, w = make(rng, m, k)
    (xd, x), (rd, r) = as_type(x, dtype), as_type(r, dtype)
    wd = torch.cat([torch.from_numpy(w), torch.full((8,), float(behind))]).cuda()[:k]
    say(f"[case] k={k} {dtype} {behind} behind the weight")
    check_norm(P.add_rms_norm_i8(xd, rd, wd), x, r, w, 1e-6, dtype)
    check_norm(P.add_rms_norm_i8(xd, None, wd), x, None, w, 1e-6, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [5, 64, 300, 9001])
def test_rows_with_tiny_huge_infinite_and_nan_values(k):
    say(f"[case] add_rms_norm_i8 odd values k={k}")
    rng = np.random.default_rng(k)
    x = rng.standard_normal((12, k)).astype(np.float32)
    r = np.zeros_like(x)
    x[0] *= np.float32(1e-37)
    x[1] = (x[1] * 1e-30).astype(np.float32) * np.float32(1e-12)
    x[2] = np.float32(2.0 ** -149)
    x[3] = np.float32(3.0e38) * np.sign(x[3])
    x[8] = 0
    x[9] = np.float32(1e25) * x[9]
    x[10] = 0
    x[10, k - 1] = np.float32(3.4e38)
    r[11] = -x[11]                                       # a sum of zeros
    bad = {4: (k - 1, np.inf), 5: (0, -np.inf), 6: (k // 2, np.nan), 7: (k - 1, -np.nan)}
    good = [i for i in range(12) if i not in bad]
    for i, (at, value) in bad.items():
        x[i, at] = value
    q, scale, s = P.add_rms_norm_i8(dev(x), dev(r), eps=1e-12)
    check_norm((q[good], scale[good], s[good]), x[good], r[good], None, np.float32(1e-12), "f32")
    assert np.isnan(scale.cpu().numpy()[list(bad)]).all() and not bool(q[list(bad)].any())
    over = np.full((1, k), 3e38, np.float32)             # a sum that is no fp32 number
    q, scale, s = P.add_rms_norm_i8(dev(over), dev(over))
    assert bool(s.isinf().all()) and bool(scale.isnan().all()) and not bool(q.any())


@pytest.mark.gpu
def test_the_layer_that_reads_it():
    """Norm and product as they are used, [2, 7, 9, 96] as rows; one row alone gives the same bits."""
    import torch
    say("[case] add_rms_norm_i8 -> matmul_i8")
    rng = np.random.default_rng(2)
    x, r, w = make(rng, 126, 96)
    w8, sb, bias = make_layer8(rng, 40, 96)
    xd, rd, wd = dev(x).view(2, 7, 9, 96), dev(r).view(2, 7, 9, 96), dev(w)
    q, scale, s = P.add_rms_norm_i8(xd, rd, wd)
    assert q.shape == s.shape == xd.shape and scale.shape == (2, 7, 9)
    y = P.matmul_i8(q, scale, dev(w8), dev(sb), dev(bias), relu=True)
    want, bound = plain_product(q.cpu().numpy().reshape(126, 96).astype(np.int64), scale.cpu().numpy().reshape(126), w8, sb, bias, True)
    check(y.view(126, 40), want, bound, "matmul_i8 of normalised rows")
    one = P.add_rms_norm_i8(dev(x)[5], dev(r)[5], wd)
    assert all(torch.equal(a, b.reshape((126,) + a.shape)[5]) for a, b in zip(one, (q, scale, s)))


@pytest.mark.gpu
def test_ordinary_calls_and_the_long_way_give_the_same():
    """Ordinary calls are looked at in native code; an output given, or rows in more dimensions with a step, go the long way: of the
    norm and of the layer that reads it."""
    import torch
    rng = np.random.default_rng(21)
    for m, k, n in ((1, 96, 40), (37, 333, 70), (300, 1000, 130)):
        say(f"[case] both ways {m}x{k} -> {n}")
        x, r, w = (dev(rng.standard_normal(size).astype(np.float32)) for size in ((m, k), (m, k), k))
        b, sb = P.quantize_rows(dev(rng.standard_normal((n, k)).astype(np.float32)))
        apart = torch.nn.functional.pad(x, (0, 5))[:, :k].unsqueeze(1).expand(m, 1, k)
        q, scale, s = P.add_rms_norm_i8(x, r, w)
        for q2, scale2, s2 in (P.add_rms_norm_i8(x, r, w, out=torch.empty_like(x)), P.add_rms_norm_i8(apart, r.unsqueeze(1), w), P.add_rms_norm_i8(x, r, w, eps=np.float32(1e-6))):
            assert torch.equal(q2.reshape(m, k), q) and torch.equal(scale2.flatten(), scale) and torch.equal(s2.view_as(s), s)
        for half in (None, torch.float32, torch.bfloat16):
            y = P.matmul_i8(q, scale, b, sb, w[:n] if n <= k else None, True, half)
            assert torch.equal(y, P.matmul_i8(q, scale, b, sb, w[:n] if n <= k else None, True, out=torch.empty_like(y)))
            assert torch.equal(y, P.matmul_i8(q, scale.unsqueeze(1), b, sb, w[:n] if n <= k else None, True, half))


@pytest.mark.gpu
def test_steps_of_the_quantised_rows():
    """A multiple of 16 bytes, and of 128 from 1024 on."""
    import torch
    for k, step in ((40, 48), (1008, 1008), (1009, 1024), (1024, 1024), (1025, 1152)):
        say(f"[case] steps of rows of {k}")
        x, r, w = (dev(a) for a in make(np.random.default_rng(k), 6, k))
        q, scale, s = P.add_rms_norm_i8(x.view(2, 3, k), r.view(2, 3, k), w)
        assert q.shape == (2, 3, k) and q.stride() == (3 * step, step, 1)
        check_norm((q, scale, s), x.cpu().numpy(), r.cpu().numpy(), w.cpu().numpy(), np.float32(1e-6), "f32")
        q2, scale2, _ = P.add_rms_norm_i8(x.view(2, 3, k), r.view(2, 3, k), w, out=torch.empty_like(s))
        assert q2.stride() == q.stride() and torch.equal(q, q2) and torch.equal(scale, scale2)


@pytest.mark.gpu
def test_sizes_of_zero():
    import torch
    say("[case] add_rms_norm_i8, sizes of zero")
    z = lambda *shape: torch.zeros(*shape, device="cuda")
    q, scale, s = P.add_rms_norm_i8(z(0, 8), z(0, 8), z(8))
    assert q.shape == s.shape == (0, 8) and scale.shape == (0,)
    q, scale, s = P.add_rms_norm_i8(z(5, 0), z(5, 0), z(0))
    assert q.shape == (5, 0) and bool((scale == 0).all())


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    import torch
    say("[case] add_rms_norm_i8 far rows")
    m, k = 3, 40
    x, r, w = make(np.random.default_rng(0), m, k)
    step = (1 << 31) // (m - 1) // 2 + 8                 # (of fp32: beyond 2^32 bytes)
    room = torch.empty((m - 1) * step + k, dtype=torch.float32, device="cuda")
    xd = torch.as_strided(room, (m, k), (step, 1))
    xd.copy_(dev(x))
    got = P.add_rms_norm_i8(xd, dev(r), dev(w), out=xd)
    check_norm(got, x, r, w, 1e-6, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("m,k", [(1, 2048), (300, 333), (2, 70_000)])
def test_another_stream_replays_and_equal_bits(m, k):
    import torch
    say(f"[case] add_rms_norm_i8 stream and graph {m}x{k}")
    rng = np.random.default_rng(m)
    x, r, w = (dev(a) for a in make(rng, m, k))
    want = P.add_rms_norm_i8(x, r, w)
    torch.cuda.synchronize()
    stream, late = torch.cuda.Stream(), torch.zeros_like(x)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        big = torch.randn(3000, 3000, device="cuda")
        for _ in range(5):
            big = big @ big * 1e-3
        late.copy_(x)
        got = P.add_rms_norm_i8(late, r, w)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = P.add_rms_norm_i8(late, r, w)
    for i in range(4):
        late.copy_(dev(make(rng, m, k)[0]))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, P.add_rms_norm_i8(late, r, w))), f"replay {i}"


# ---- refusals ------------------------------------------------------------------------------------------------------------

def c_calls():
    p = 1 << 20
    good = dict(x=p, ldx=8, r=p, ldr=8, s=p + 4096, lds=8, t="f32", w=p, eps=1e-6, rows=2, cols=8, q=p, ldq=8, scale=p)
    for what, change in [("rows and cols", dict(rows=-1)), ("rows and cols", dict(cols=1 << 31)), ("eps", dict(eps=0.0)), ("eps", dict(eps=float("nan"))),
                         ("eps", dict(eps=float("inf"))), ("eps", dict(eps=-1.0)), ("no residual", dict(r=0)), ("null", dict(x=0)), ("null", dict(q=0)),
                         ("null", dict(scale=0)), ("apart", dict(ldx=7)), ("apart", dict(ldr=7)), ("apart", dict(lds=7)), ("apart", dict(ldq=7)),
                         ("its stride", dict(s=p, lds=9)), ("aligned", dict(x=p + 2)), ("aligned", dict(r=p + 1)), ("aligned", dict(s=p + 4098)),
                         ("aligned", dict(w=p + 2)), ("aligned", dict(x=p + 1, t="bf16"))]:
        yield what, lambda change=change: P.pconv_add_rms_norm_i8(*{**good, **change}.values())


def test_c_entry_refuses_what_it_cannot_run():
    for what, call in c_calls():
        with pytest.raises(P.PconvError) as e:
            call()
        assert e.value.status == P.INVALID_ARG and what in str(e.value), (what, str(e.value))
    assert P.lib().pconv_add_rms_norm_i8(1 << 20, 8, None, 0, None, 0, 7, None, 1e-6, 2, 8, 1 << 20, 8, 1 << 20, None) == P.INVALID_ARG


def test_calls_on_the_host_are_refused():
    import torch
    with pytest.raises(ValueError, match="CUDA"):
        P.add_rms_norm_i8(torch.zeros(4, 8), torch.zeros(4, 8), torch.ones(8))


@pytest.mark.gpu
def test_wrong_tensors_are_refused():
    import torch
    z = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")
    x, r, w = z(4, 8), z(4, 8), z(8)
    bad = [lambda: P.add_rms_norm_i8(x.half()), lambda: P.add_rms_norm_i8(x.t()), lambda: P.add_rms_norm_i8(x, r[:3]), lambda: P.add_rms_norm_i8(x, r.bfloat16()),
           lambda: P.add_rms_norm_i8(x, r, w[:7]), lambda: P.add_rms_norm_i8(x, r, w.double()), lambda: P.add_rms_norm_i8(x, r, w.cpu()),
           lambda: P.add_rms_norm_i8(x, out=z(4, 8)), lambda: P.add_rms_norm_i8(x, r, out=z(4, 9)), lambda: P.add_rms_norm_i8(x, r, out=z(4, 8).bfloat16()),
           lambda: P.add_rms_norm_i8(x, z(8).expand(4, 8)), lambda: P.add_rms_norm_i8(z(8).expand(4, 8), r)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    room, flat = z(5, 8), z(4, 20)
    over = [lambda: P.add_rms_norm_i8(room[:4], r, w, out=room[1:]), lambda: P.add_rms_norm_i8(x, flat[:, :8], out=flat[:, 4:12]),
            lambda: P.add_rms_norm_i8(x[:1], r[:1], w, out=w.view(1, 8)), lambda: P.add_rms_norm_i8(room[:4], room[1:], out=room[:4])]
    for i, call in enumerate(over):
        with pytest.raises(ValueError, match="overlap"):
            call()
            pytest.fail(f"call {i} was not refused")
    with pytest.raises(P.PconvError, match="eps"):
        P.add_rms_norm_i8(x, r, w, eps=0.0)
