"""distill_loss, its gradient and distill_loss_grad against the formulas in 64 bits, and against differences.

Tolerances (U = 2^-24).  With y = z / T, d = y - lse and L = log2(e): y rounds twice (1 / T and the product), lse once and its
logarithm and sum are off by at most (2 log2 v + 16) U and what its terms' y carry, weighted by their shares q, so d is off by
D = U (2 |y| + 2 sum q |y| + |lse| + |d| + 2 log2 v + 16), and exp(d), computed as 2^(d L), by D + U (2 |d| + 4) of itself.  Shares p
alike with the teacher's logits and top entries.  A gradient is f (exp(d) - sum p): those bounds times f, U-steps of f and of the
difference, and half a step of the type.  A loss of a row is T^2 times sum p (log p - d): p times the errors of both, the errors of
p times |log p - d|, and one U for each of top additions and products."""
import math

import numpy as np
import pytest

import paper_1909_05073_amd as P

from gpu_util import say
from test_i8_layers import as_type, dev

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


# ---- the plain implementation ----------------------------------------------------------------------------------------

def softmax64(y):
    """(log-softmax with -inf handled, bound of its fp32 error) along the last axis, fp64."""
    most = y.max(-1, keepdims=True)
    base = np.where(np.isfinite(most), most, 0)
    with np.errstate(divide="ignore", invalid="ignore"):
        lse = base + np.log(np.exp(y - base).sum(-1, keepdims=True))
        d = y - lse
    size = np.abs(np.where(np.isfinite(y), y, 0))
    fin = np.abs(np.where(np.isfinite(d), d, 0))
    share = np.where(np.isfinite(d), np.exp(np.minimum(d, 0)), 0)
    off = U * (2 * size + 2 * (share * size).sum(-1, keepdims=True) + np.abs(np.where(np.isfinite(lse), lse, 0)) + fin + 2 * math.log2(max(2, y.shape[-1])) + 16)
    return d, off


def plain_distill(z, t, c, T, weight):
    """(rows' losses, bounds, gradient with weights `weight` of the rows, bounds), fp64."""
    rows, v = z.shape
    loss, loss_off = np.zeros(rows), np.zeros(rows)
    grad, grad_off = np.zeros((rows, v)), np.zeros((rows, v))
    for r in range(rows):
        have = (c[r] >= 0) & (c[r] < v)
        have[have] = t[r][have] != -np.inf
        if not have.any():
            continue
        lq, oq = softmax64(z[r].astype(np.float64) / T)
        at = c[r][have]
        lp, op = softmax64(t[r][have].astype(np.float64) / T)
        p = np.exp(lp)
        p_off = p * (op + U * (2 * np.abs(lp) + 4))
        loss[r] = T * T * (p * (lp - lq[at])).sum()
        gap = np.abs(lp - lq[at])
        loss_off[r] = T * T * ((p * (op + oq[at] + U * gap)).sum() + (p_off * gap).sum() + (len(p) + 6) * U * (p * gap).sum())
        q = np.exp(lq)
        fin = np.where(np.isfinite(lq), np.abs(lq), 0)
        g, off = q.copy(), q * (oq + U * (2 * fin + 4))
        share, share_off = np.zeros(v), np.zeros(v)
        np.add.at(share, at, p)
        np.add.at(share_off, at, p_off + (len(p) + 1) * U * p)
        g -= share
        off += share_off + U * np.abs(g)
        f = T * weight[r]
        grad[r], grad_off[r] = f * g, np.abs(f) * (off + 4 * U * np.abs(g)) + 2.0 ** -126
    return loss, loss_off, grad, grad_off


def check_grad(got, want, off, dtype, what):
    got = got.detach().float().cpu().numpy().astype(np.float64).reshape(want.shape)
    bound = off + HALF[dtype] * (np.abs(want) + off) + (2.0 ** -134 if dtype == "bf16" else 0)
    bad = np.argwhere(~(np.abs(got - want) <= bound))
    assert bad.size == 0, f"{what}: {len(bad)} of {want.size} outside; first at {tuple(bad[0])}: {got[tuple(bad[0])]} for {want[tuple(bad[0])]}"


def make(rng, rows, v, top, ragged=False, twice=False):
    z = (rng.standard_normal((rows, v)) * 3).astype(np.float32)
    t = np.sort((rng.standard_normal((rows, top)) * 2 + 4).astype(np.float32), 1)[:, ::-1].copy()
    c = np.argsort(rng.random((rows, v)), 1)[:, :top] if top <= v and not twice else rng.integers(0, v, (rows, top))
    c = c.astype(np.int64)
    if ragged:
        c[np.arange(top)[None] >= rng.integers(0, top + 1, (rows, 1))] = -1
    return z, t, c


def run_all(z, t, c, T, dtype, tt, wide=True, z_dev=None):
    """Every entry, against the formulas."""
    import torch
    zd, zv = as_type(z, dtype)
    zd = zd if z_dev is None else z_dev
    td, tv = as_type(t, tt)
    cd = dev(c if wide else np.clip(c, -(1 << 31), (1 << 31) - 1).astype(np.int32))
    rows = len(z)
    rng = np.random.default_rng(9)
    for reduction in ("none", "sum", "mean"):
        up = rng.uniform(0.5, 2, rows) if reduction == "none" else np.full(rows, 0.75 if reduction == "sum" else 0.75 / rows)
        up = up.astype(np.float32).astype(np.float64) if reduction == "none" else up
        loss, loss_off, grad, grad_off = plain_distill(zv, tv, c, T, up)
        scale = 1 / rows if reduction == "mean" else 1
        want, bound = (loss, loss_off) if reduction == "none" else (loss.sum() * scale, (loss_off.sum() + U * np.abs(loss).sum() * 2) * scale)
        s = zd.detach().requires_grad_()
        got = P.distill_loss(s, td, cd, T, reduction)
        assert (np.abs(got.detach().cpu().numpy() - want) <= bound + 2.0 ** -140).all(), (reduction, got, want)
        got.backward(dev(up.astype(np.float32)) if reduction == "none" else torch.tensor(0.75, device="cuda"))
        check_grad(s.grad, grad, grad_off, dtype, f"autograd {reduction}")
        with torch.no_grad():
            assert torch.equal(P.distill_loss(s, td, cd, T, reduction), got.detach())
        value, g = P.distill_loss_grad(zd, td, cd, T, reduction)
        assert torch.equal(value, got.detach()), "the two calls give other losses"
        _, _, grad, grad_off = plain_distill(zv, tv, c, T, np.full(rows, scale))
        check_grad(g, grad, grad_off, dtype, f"distill_loss_grad {reduction}")


SIZES = [(1, 1, 1), (3, 2, 1), (2, 7, 7), (5, 10, 3), (33, 100, 16), (7, 1000, 16), (2, 1001, 65), (4, 4096, 50), (3, 4097, 50), (2, 10007, 128),
         (3, 16385, 5), (2, 32768, 64), (1, 50000, 100), (2, 70001, 300), (1100, 30, 4), (5, 2000, 1024)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tt", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,v,top", SIZES)
def test_losses_and_gradients_against_the_formulas(rows, v, top, dtype, tt):
    T = (1.0, 2.0, 3.0)[(rows + v) % 3]
    say(f"[case] distill {rows}x{v} top {top} {dtype} {tt} T={T}")
    rng = np.random.default_rng(rows * 1009 + v + top)
    run_all(*make(rng, rows, v, top), T, dtype, tt, wide=(v % 2 == 0))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,v,top", [(9, 40, 20), (33, 1000, 50), (6, 5000, 64), (3, 20000, 200)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lists_of_unequal_length_and_classes_named_twice(rows, v, top, dtype):
    import torch
    say(f"[case] distill ragged {rows}x{v} top {top} {dtype}")
    rng = np.random.default_rng(v)
    z, t, c = make(rng, rows, v, top, ragged=True, twice=True)
    c[0] = -1                                            # a row without an entry
    c[1] = v - 1                                         # one class for all
    c[2, ::2] = np.array([v, -5, 1 << 40, -(1 << 62)] * top)[:len(c[2, ::2])]
    run_all(z, t, c, 2.0, dtype, "f32")
    zd = dev(z).requires_grad_()
    P.distill_loss(zd, dev(t), dev(c), 2.0, "sum").backward()
    assert not bool(zd.grad[0].any()) and bool(P.distill_loss(zd.detach(), dev(t), dev(c), 2.0, "none")[0] == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("top", [63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513])
@pytest.mark.parametrize("v", [600, 9001, 21000])
def test_lists_longer_than_the_threads_of_a_row(v, top):
    """A wave, 256 or 512 threads share a row; a thread asks for its first entry, or first two, before the others."""
    say(f"[case] distill long lists 3x{v} top {top}")
    rng = np.random.default_rng(v + top)
    z, t, c = make(rng, 3, v, top, ragged=True, twice=True)
    c[0, [0, top - 1]] = c[0, top // 2] = 5              # one class first, in the middle and last
    run_all(z, t, c, 2.0, "f32", "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [5, 130, 300, 1024])
@pytest.mark.parametrize("v", [1024, 2049, 4097, 10_007, 10_241, 20_481, 21_000, 40_003])
def test_equal_bits_together_and_apart(v, top, dtype):
    """Every number of threads a row, lists shorter and longer than it."""
    import torch
    say(f"[case] distill equal bits v={v} top={top} {dtype}")
    z, t, c = make(np.random.default_rng(v + top), 9, v, top, ragged=True, twice=True)
    zd = as_type(z, dtype)[0]
    for T in (2.0, 3.0):
        loss, grad = P.distill_loss_grad(zd, dev(t), dev(c), T, "none")
        leaf = zd.clone().requires_grad_()
        apart = P.distill_loss(leaf, dev(t), dev(c), T, "none")
        apart.sum().backward()
        assert torch.equal(apart.detach(), loss) and torch.equal(leaf.grad, grad)
        with torch.no_grad():
            assert torch.equal(P.distill_loss(leaf, dev(t), dev(c), T, "none"), loss)


@pytest.mark.gpu
@pytest.mark.parametrize("v", [50, 5000, 40000])
def test_masked_classes_and_logits_of_minus_infinity(v):
    """Classes that the student may not take, teacher's logits that are none, rows of nothing else."""
    say(f"[case] distill masks v={v}")
    rng = np.random.default_rng(v)
    z, t, c = make(rng, 6, v, 8)
    z[0, rng.permutation(np.setdiff1d(np.arange(v), c[0]))[:v // 2]] = -np.inf
    t[1, 3:] = -np.inf
    t[2] = -np.inf                                       # counts as no entry
    z[3] = -np.inf
    z[3, c[3]] = 1.0                                     # all mass on the entries
    z[4, :v // 2 * 2:2] = np.finfo(np.float32).min       # the type's lowest value in masked places
    z[4, c[4]] = 2.0
    run_all(z, t, c, 2.0, "f32", "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tt", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("T", [1.0, 2.0, 0.5])
@pytest.mark.parametrize("v", [50, 5000, 40000])
def test_shares_that_vanish_count_nothing(v, T, dtype, tt):
    """A teacher masked with its type's lowest value, or far below its largest logit, where the student has -infinity."""
    import torch
    say(f"[case] distill vanishing shares v={v} T={T} {dtype} {tt}")
    rng = np.random.default_rng(v)
    z, t, c = make(rng, 5, v, 8)
    low = float(torch.finfo(torch.bfloat16 if tt == "bf16" else torch.float32).min)
    for r, value in enumerate((low, -1e30, t[2].max() - 300 * T, t[3].max() - 2000 * T)):
        t[r, 4:] = value
        z[r, c[r, 4:]] = -np.inf
    t[4, 3] = -np.inf                                    # p = 0 exactly, as well
    z[4, c[4, 3]] = -np.inf
    # (what p counts there is below exp(-300) of the others: the formulas without those entries)
    kept = c.copy()
    kept[:4, 4:] = -1
    kept[4, 3] = -1
    zd, zv = as_type(z, dtype)
    td, tv = as_type(t, tt)
    loss, loss_off, grad, grad_off = plain_distill(zv, tv, kept, T, np.ones(5))
    got, slope = P.distill_loss_grad(zd, td, dev(c), T, "none")
    assert (np.abs(got.cpu().numpy() - loss) <= loss_off + 2.0 ** -126).all(), (got, loss)
    check_grad(slope, grad, grad_off, dtype, "distill_loss_grad")
    leaf = zd.clone().requires_grad_()
    again = P.distill_loss(leaf, td, dev(c), T, "none")
    again.sum().backward()
    assert torch.equal(again.detach(), got) and torch.equal(leaf.grad, slope)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1.0, 1.3, 3.0, 5.0])
@pytest.mark.parametrize("v", [50, 5000, 40000])
def test_rows_of_huge_logits(v, T, dtype):
    """Rows whose largest logit is the type's lowest value, or so large that a step of it is an exponent's whole range."""
    import torch
    say(f"[case] distill huge logits v={v} T={T} {dtype}")
    z, t, c = make(np.random.default_rng(v), 6, v, 8)
    low = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    z[0] = low
    z[1] = low
    z[1, c[1, 0]] = 2.0
    c[1, 1:] = -1
    z[2] += 1e6
    z[3], z[4] = 3e11, -7e20
    t[5] += 1e9
    zd, zv = as_type(z, dtype)
    td, tv = as_type(t, "f32")
    loss, loss_off, grad, grad_off = plain_distill(zv, tv, c, T, np.ones(6))
    got, slope = P.distill_loss_grad(zd, td, dev(c), T, "none")
    # (of rows of equal huge logits U |lse| is more than log v: all that is asked is a number, and no share beyond 1 by more than half a step
    # of a sum near 1e6, 2^-5)
    assert bool(got.isfinite().all()) and bool(slope.isfinite().all())
    assert (np.abs(got.cpu().numpy() - loss) <= loss_off + 2.0 ** -126).all(), (got, loss)
    off = np.where(grad_off < 1, grad_off, np.inf)
    fine = ~(off.max(1) == np.inf)
    assert fine[1]
    check_grad(slope[dev(np.flatnonzero(fine))], grad[fine], off[fine], dtype, "distill_loss_grad")
    assert float(slope.abs().max()) <= T * (1 + 2.0 ** -4)
    leaf = zd.clone().requires_grad_()
    again = P.distill_loss(leaf, td, dev(c), T, "none")
    again.sum().backward()
    assert torch.equal(again.detach(), got) and torch.equal(leaf.grad, slope)


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_rows():
    import torch
    say("[case] distill NaN")
    rng = np.random.default_rng(1)
    for v in (60, 6000, 20000):
        z, t, c = make(rng, 7, v, 6)
        clean = P.distill_loss_grad(dev(z), dev(t), dev(c), 1.0, "none")
        z[1, v - 1] = np.nan
        z[2, 0] = np.inf
        t[3, 2] = np.nan
        z[4] = -np.inf
        z[5, c[5, 0]] = -np.inf                          # an entry that the student rules out: an infinite loss
        loss, grad = P.distill_loss_grad(dev(z), dev(t), dev(c), 1.0, "none")
        assert bool(loss[1:5].isnan().all()) and bool(grad[1:5].isnan().any(1).all())
        assert float(loss[5]) == math.inf and bool(grad[5].isfinite().all())
        for r in (0, 6):
            assert torch.equal(loss[r], clean[0][r]) and torch.equal(grad[r], clean[1][r])


@pytest.mark.gpu
@pytest.mark.parametrize("v", [12, 4500])
def test_gradient_against_differences(v):
    """Central differences of the loss computed in 64 bits by elementary operations; the step's own error is its square."""
    import torch
    say(f"[case] distill differences v={v}")
    rng = np.random.default_rng(v)
    z, t, c = make(rng, 3, v, 5, ragged=False, twice=True)
    T, step = 2.0, 1e-3

    def value(a):
        lq = torch.log_softmax(torch.from_numpy(a) / T, 1)
        lp = torch.log_softmax(torch.from_numpy(t.astype(np.float64)) / T, 1)
        return float((lp.exp() * (lp - lq.gather(1, torch.from_numpy(c)))).sum()) * T * T / 3
    zd = dev(z).requires_grad_()
    P.distill_loss(zd, dev(t), dev(c), T).backward()
    got = zd.grad.cpu().numpy()
    for r in range(3):
        for u in set(c[r]) | set(rng.integers(0, v, 8)):
            up, down = z.astype(np.float64), z.astype(np.float64)
            up[r, u] += step
            down[r, u] -= step
            want = (value(up) - value(down)) / (2 * step)
            # the third derivative is at most 1 / (6 T) a row: step^2 of it; 64 bits lose 1e-13 / step; the gradient's bound is below 1e-4 of it
            assert abs(got[r, u] - want) <= step ** 2 + 1e-9 + 1e-4 * abs(want) + 1e-6


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v,offset,extra", [(9, 1, 2), (1003, 3, 5), (5001, 1, 0), (20011, 2, 7)])
def test_rows_that_lie_apart_and_begin_anywhere(v, offset, extra, dtype):
    import torch
    say(f"[case] distill apart v={v} {dtype}")
    rng = np.random.default_rng(v)
    rows, top = 5, 7
    z, t, c = make(rng, rows, v, top)
    flat = torch.full((offset + rows * (v + extra) + 1,), float("nan"), dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    zd = torch.as_strided(flat, (rows, v), (v + extra, 1), offset)
    zd.copy_(dev(z))
    run_all(z, t, c, 2.0, dtype, "f32", z_dev=zd)
    wide_t, wide_c = torch.full((rows, top + 3), float("nan"), device="cuda"), torch.zeros(rows, top + 2, dtype=torch.int64, device="cuda")
    wide_t[:, 2:2 + top], wide_c[:, 1:1 + top] = dev(t), dev(c)
    room = torch.full_like(flat, 7.0)
    out = torch.as_strided(room, (rows, v), (v + extra, 1), offset)
    before = out._version
    loss, grad = P.distill_loss_grad(zd, wide_t[:, 2:2 + top], wide_c[:, 1:1 + top], 2.0, out=out)
    want = P.distill_loss_grad(zd, dev(t), dev(c), 2.0)
    assert grad is out and out._version > before and torch.equal(loss, want[0]) and torch.equal(grad, want[1])
    out.fill_(7.0)
    assert bool((room == 7).all()), "values outside the rows were written"


@pytest.mark.gpu
def test_leading_dimensions_and_sizes_of_zero():
    import torch
    say("[case] distill leading dimensions, zeros")
    rng = np.random.default_rng(0)
    z, t, c = (dev(a) for a in make(rng, 12, 50, 5))
    flat = P.distill_loss_grad(z, t, c, 2.0, "none")
    got = P.distill_loss_grad(z.view(3, 2, 2, 50), t.view(3, 2, 2, 5), c.view(3, 2, 2, 5), 2.0, "none")
    assert got[0].shape == (3, 2, 2) and torch.equal(got[0].view(-1), flat[0]) and torch.equal(got[1].view(12, 50), flat[1])
    s = z.view(3, 4, 50).clone().requires_grad_()
    P.distill_loss(s, t.view(3, 4, 5), c.view(3, 4, 5), 2.0, "none").sum().backward()
    assert torch.equal(s.grad.view(12, 50), flat[1])
    one = P.distill_loss_grad(z[3], t[3], c[3], 2.0, "none")
    assert one[0].shape == () and torch.equal(one[0], flat[0][3]) and torch.equal(one[1], flat[1][3])
    for rows, v, top in ((0, 5, 3), (4, 5, 0), (4, 0, 3), (0, 0, 0)):
        s = torch.ones(rows, v, device="cuda", requires_grad=True)
        args = torch.ones(rows, top, device="cuda"), torch.zeros(rows, top, dtype=torch.int64, device="cuda")
        for reduction in ("none", "sum", "mean"):
            value, grad = P.distill_loss_grad(s.detach(), *args, 1.0, reduction)
            assert not bool(value.any()) and not bool(grad.any()) and grad.shape == (rows, v)
            P.distill_loss(s, *args, 1.0, reduction).sum().backward()
            assert not bool(s.grad.any())


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    import torch
    say("[case] distill far rows")
    rng = np.random.default_rng(0)
    for v in (40, 5000):
        z, t, c = make(rng, 3, v, 4)
        step = (1 << 30) // 2 + 8
        room = torch.empty(2 * step + v, dtype=torch.float32, device="cuda")
        far = torch.as_strided(room, (3, v), (step, 1))
        far.copy_(dev(z))
        want = P.distill_loss_grad(dev(z), dev(t), dev(c))
        out = torch.as_strided(torch.empty(2 * step + v, device="cuda"), (3, v), (step, 1))
        got = P.distill_loss_grad(far, dev(t), dev(c), out=out)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("v", [100, 20000])
def test_another_stream_replays_and_equal_bits(v):
    """A training step captured and replayed: forward and backward on the graph's own leaf."""
    import torch
    say(f"[case] distill stream and graph v={v}")
    rng = np.random.default_rng(v)
    rows, top = 50, 9
    make_z = lambda: dev(make(rng, rows, v, top)[0])
    z, t, c = (dev(a) for a in make(rng, rows, v, top, ragged=True))
    want = P.distill_loss_grad(z, t, c, 2.0)
    torch.cuda.synchronize()
    stream, late = torch.cuda.Stream(), torch.zeros_like(z)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        big = torch.randn(3000, 3000, device="cuda")
        for _ in range(5):
            big = big @ big * 1e-3
        late.copy_(z)
        leaf = late.detach().requires_grad_()
        loss = P.distill_loss(leaf, t, c, 2.0)
        grad, = torch.autograd.grad(loss, leaf)
    stream.synchronize()
    assert torch.equal(loss.detach(), want[0]) and torch.equal(grad, want[1])
    del loss, grad, leaf
    torch.cuda.synchronize()
    static = z.clone().requires_grad_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loss = P.distill_loss(static, t, c, 2.0)
        grad, = torch.autograd.grad(loss, static)
        both = P.distill_loss_grad(static.detach(), t, c, 2.0)
    for i in range(4):
        with torch.no_grad():
            static.copy_(make_z())
        g.replay()
        torch.cuda.synchronize()
        want = P.distill_loss_grad(static.detach(), t, c, 2.0)
        assert torch.equal(loss.detach(), want[0]) and torch.equal(grad, want[1]), f"replay {i}"
        assert torch.equal(both[0], want[0]) and torch.equal(both[1], want[1]), f"replay {i}"


@pytest.mark.gpu
def test_autograd_keeps_its_rules():
    import torch
    say("[case] distill autograd")
    rng = np.random.default_rng(4)
    z, t, c = (dev(a) for a in make(rng, 6, 40, 5))
    s = z.clone().requires_grad_()
    loss = P.distill_loss(s * 1.0, t, c, 2.0)
    one, = torch.autograd.grad(loss, s, retain_graph=True)
    two, = torch.autograd.grad(loss, s)                  # a second time through the same graph
    assert torch.equal(one, two)
    y = s * 1.0
    loss = P.distill_loss(y, t, c, 2.0)
    with torch.no_grad():
        y.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        loss.backward()
    loss = P.distill_loss(s, t, c, 2.0)
    g, = torch.autograd.grad(loss, s, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
    with pytest.raises(ValueError, match="teacher"):
        P.distill_loss(s, t.clone().requires_grad_(), c)
    s.grad = None
    for _ in range(2):
        P.distill_loss(s, t, c, 2.0).backward()
    assert torch.equal(s.grad, 2 * one)


@pytest.mark.gpu
@pytest.mark.parametrize("lead", [(6,), (2, 3), ()])
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
def test_losses_may_be_changed_in_place(lead, reduction):
    import torch
    say(f"[case] distill in place {lead} {reduction}")
    z, t, c = (dev(a) for a in make(np.random.default_rng(31), 6, 40, 5))
    z, t, c = (a.view(*lead, -1) if lead else a[0] for a in (z, t, c))
    for T in (2.0, 2):
        leaf, other = z.clone().requires_grad_(), z.clone().requires_grad_()
        loss = P.distill_loss(leaf, t, c, T, reduction)
        up = torch.rand_like(loss)
        want = P.distill_loss(other, t, c, T, reduction)
        loss *= up
        loss.sum().backward()
        want.backward(up)
        assert torch.equal(leaf.grad, other.grad) and torch.equal(loss.detach(), want.detach() * up)
        value, _ = P.distill_loss_grad(z, t, c, T, reduction)
        assert value.shape == loss.shape and torch.equal(value, want.detach())


@pytest.mark.gpu
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
def test_forward_mode_and_function_transforms_are_refused(reduction):
    """A loss without its tangent, or of something that has no memory of its own, would be wrong in silence."""
    import torch
    import torch.autograd.forward_ad as fw
    say(f"[case] distill forward mode {reduction}")
    z, t, c = (dev(a) for a in make(np.random.default_rng(21), 6, 40, 5))
    want = P.distill_loss_grad(z, t, c, 2.0, reduction)
    with fw.dual_level():
        dual, dual_t, leaf = fw.make_dual(z, torch.ones_like(z)), fw.make_dual(t, torch.ones_like(t)), z.clone().requires_grad_()
        for T in (2.0, 2):                               # (in native code at once, and the long way)
            for student, teacher in ((dual, t), (z, dual_t), (fw.make_dual(leaf, torch.ones_like(z)), t)):
                with pytest.raises(NotImplementedError, match="forward mode"):
                    P.distill_loss(student, teacher, c, T, reduction)
                with torch.no_grad(), pytest.raises(NotImplementedError, match="forward mode"):
                    P.distill_loss(student, teacher, c, T, reduction)
        got = P.distill_loss_grad(fw.unpack_dual(dual).primal, t, c, 2.0, reduction)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    f = lambda s: P.distill_loss(s, t, c, 2.0, "sum")
    for call in (lambda: torch.func.jvp(f, (z,), (torch.ones_like(z),)), lambda: torch.func.grad(f)(z),
                 lambda: torch.func.vmap(lambda s: P.distill_loss(s, t[0], c[0], 2.0, "sum"))(z)):
        with pytest.raises(RuntimeError):
            call()
    assert torch.equal(P.distill_loss(z, t, c, 2.0, reduction), want[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,v,top", [(5, 10, 4), (7, 1003, 9), (6, 12001, 300)])
def test_hooks_of_saved_tensors_may_lay_them_out_otherwise(rows, v, top, dtype):
    """Rows cut out of wider ones come back from a hook without what lay between them, or with something else there."""
    import torch
    from torch.autograd.graph import save_on_cpu, saved_tensors_hooks
    say(f"[case] distill hooks {rows}x{v} top {top} {dtype}")
    z, t, c = make(np.random.default_rng(v), rows, v, top, twice=True)

    def apart(a, extra, fill, dtype=None):
        wide = torch.full((rows, a.shape[1] + extra), fill, dtype=dtype or dev(a).dtype, device="cuda")
        wide[:, :a.shape[1]] = dev(a)
        return wide[:, :a.shape[1]]
    zd = apart(z, 3, float("nan"), torch.bfloat16 if dtype == "bf16" else torch.float32).requires_grad_()
    td, cd = apart(t, 2, float("nan")), apart(c, 5, 0)
    up = dev(np.random.default_rng(1).uniform(0.5, 2, rows).astype(np.float32))
    want, = torch.autograd.grad(P.distill_loss(zd, td, cd, 2.0, "none"), zd, up)
    other = lambda t: t if t.dim() < 2 else torch.nn.functional.pad(t, (4, 7))[..., 4:-7]
    columns = lambda t: t if t.dim() < 2 else t.transpose(0, -1).contiguous().transpose(0, -1)
    packs = (lambda t: t.contiguous(), lambda t: t.clone(), other, columns)
    for hooks in [save_on_cpu()] + [saved_tensors_hooks(pack, lambda t: t) for pack in packs]:
        for wide in (lambda t: t, lambda t: t.unsqueeze(1)):
            with hooks:
                loss = P.distill_loss(wide(zd), wide(td), wide(cd), 2.0, "none")
            got, = torch.autograd.grad(loss, zd, up.view_as(loss))
            assert torch.equal(got, want)
    for pack in (lambda t: t.double() if t.is_floating_point() else t, lambda t: t[..., :1], lambda t: t.cpu()):
        with saved_tensors_hooks(pack, lambda t: t):
            loss = P.distill_loss(zd, td, cd, 2.0)
        with pytest.raises(RuntimeError, match="hook of saved tensors"):
            loss.backward()


@pytest.mark.gpu
def test_a_capture_that_torch_does_not_know_of_is_refused_where_memory_would_be_lent():
    """The rows' losses and what a gradient needs go back to torch's pool, which such a graph must not keep; calls whose every
    output is handed out are captured."""
    import ctypes as C

    import torch
    say("[case] distill captured by the HIP runtime")
    L = P.lib()

    def hip(name, *args):
        fn = getattr(L, name)
        fn.restype = C.c_int
        assert fn(*args) == 0, name
    z, t, c = (dev(a) for a in make(np.random.default_rng(8), 20, 300, 6))
    out, leaf = torch.empty_like(z), z.clone().requires_grad_()
    side = torch.cuda.Stream()
    want = P.distill_loss_grad(z, t, c, 2.0, "none")
    P.distill_loss_grad(z, t, c, 2.0, "none", out=out)
    torch.cuda.synchronize()
    st, graph, ready = C.c_void_p(side.cuda_stream), C.c_void_p(), C.c_void_p()
    with torch.cuda.stream(side):
        P.distill_loss_grad(z, t, c, 2.0, "none")            # (its memory is in the stream's pool)
        hip("hipStreamBeginCapture", st, C.c_int(2))
        for call in (lambda: P.distill_loss(z, t, c), lambda: P.distill_loss_grad(z, t, c), lambda: P.distill_loss_grad(z, t, c, out=out),
                     lambda: P.distill_loss(leaf, t, c, reduction="none")):
            with pytest.raises(RuntimeError, match="captured by others"):
                call()
        loss, grad = P.distill_loss_grad(z, t, c, 2.0, "none")
        hip("hipStreamEndCapture", st, C.byref(graph))
    hip("hipGraphInstantiate", C.byref(ready), graph, None, None, C.c_size_t(0))
    for i in range(3):
        z.copy_(dev(make(np.random.default_rng(9 + i), 20, 300, 6)[0]))
        torch.cuda.synchronize()
        hip("hipGraphLaunch", ready, st)
        torch.cuda.synchronize()
        want = P.distill_loss_grad(z, t, c, 2.0, "none")
        assert torch.equal(loss, want[0]) and torch.equal(grad, want[1]), f"replay {i}"
    hip("hipGraphExecDestroy", ready)
    hip("hipGraphDestroy", graph)


@pytest.mark.gpu
def test_a_capture_while_a_graph_of_another_stream_holds_the_student_is_refused():
    """The gradient would be added on that graph's stream, which the capture does not know."""
    import torch
    say("[case] distill captured while an eager graph lives")
    z, t, c = (dev(a) for a in make(np.random.default_rng(12), 20, 300, 6))
    leaf, y = z.clone().requires_grad_(), torch.zeros(8, device="cuda")
    alive = P.distill_loss(leaf, t, c, 2.0)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        with pytest.raises(RuntimeError, match="still holds the student"):
            P.distill_loss(leaf, t, c, 2.0)
        with torch.no_grad():
            loss = P.distill_loss(leaf, t, c, 2.0)
        y.add_(1.0)
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, alive.detach()) and float(y[0]) == i + 1
    alive.backward()
    want = P.distill_loss_grad(z, t, c, 2.0)[1]
    assert torch.equal(leaf.grad, want)
    del alive
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        grad, = torch.autograd.grad(P.distill_loss(leaf, t, c, 2.0), leaf)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad, want)


@pytest.mark.gpu
def test_ordinary_calls_and_the_long_way_give_the_same():
    """Ordinary calls are looked at in native code; a temperature that is no float, or rows in more dimensions with a step, go the long way."""
    import torch
    rng = np.random.default_rng(13)
    for rows, v, top in ((1, 5, 1), (12, 333, 9)):
        z, t, c = (dev(a) for a in make(rng, rows, v, top))
        wide = torch.nn.functional.pad(z, (0, 7))[:, :v].unsqueeze(1)            # [rows, 1, v], v + 7 apart
        for reduction in ("none", "sum", "mean"):
            say(f"[case] both ways {rows}x{v} top={top} {reduction}")
            loss, grad = P.distill_loss_grad(z, t, c, 2.0, reduction)
            assert torch.equal(loss, P.distill_loss(z, t, c, 2, reduction)) and torch.equal(loss, P.distill_loss(z, t, c, np.float32(2), reduction))
            far, slope = P.distill_loss_grad(wide, t.unsqueeze(1), c.unsqueeze(1), 2.0, reduction)
            assert far.shape == ((rows, 1) if reduction == "none" else ()) and torch.equal(far.view_as(loss), loss) and torch.equal(slope.view_as(grad), grad)
            for leaf, tt, cc in ((z.clone(), t, c), (wide.clone().expand(rows, 1, v), t.unsqueeze(1), c.unsqueeze(1))):
                leaf = leaf.requires_grad_()
                P.distill_loss(leaf, tt, cc, 2, reduction).sum().backward()
                assert torch.equal(leaf.grad.view_as(grad), grad)


# ---- refusals ------------------------------------------------------------------------------------------------------------

def c_calls():
    p, f = 1 << 20, float
    good = dict(z=p, ldz=8, zt="f32", t=p, ldt=4, tt="f32", c=p, ldc=4, size=8, rows=3, v=8, top=4, T=1.0, mean=True)
    wrong = [("rows must", dict(rows=-1)), ("rows must", dict(v=(1 << 30) + 1)), ("top must", dict(top=1025, ldt=1025, ldc=1025)), ("top must", dict(top=-1)),
             ("4 or 8", dict(size=2)), ("temperature", dict(T=0.0)), ("temperature", dict(T=f("nan"))), ("temperature", dict(T=f("inf"))), ("temperature", dict(T=-1.0)),
             ("temperature", dict(T=1e30)), ("temperature", dict(T=1e-39)), ("null", dict(z=0)), ("null", dict(t=0)), ("null", dict(c=0)), ("apart", dict(ldz=7)),
             ("apart", dict(ldt=3)), ("apart", dict(ldc=3)), ("aligned", dict(z=p + 2)), ("aligned", dict(t=p + 2)), ("aligned", dict(c=p + 4))]
    for what, change in wrong:
        args = list({**good, **change}.values())
        yield what, lambda args=args: P.pconv_distill_loss(*args, p, p, p)
        yield what, lambda args=args: P.pconv_distill_grad(*args, p, p, 0, p, 8)
        yield what, lambda args=args: P.pconv_distill_loss_grad(*args, p, p, p, 8)
    args = list(good.values())
    yield "null", lambda: P.pconv_distill_loss(*args, 0, p, p)
    yield "null", lambda: P.pconv_distill_loss_grad(*args, 0, p, p, 8)
    yield "null", lambda: P.pconv_distill_loss_grad(*args, p, p, 0, 8)
    yield "apart", lambda: P.pconv_distill_loss_grad(*args, p, p, p, 7)
    yield "aligned", lambda: P.pconv_distill_loss_grad(*args, p, p, p + 2, 8)
    yield "null", lambda: P.pconv_distill_grad(*args, 0, p, 0, p, 8)
    yield "null", lambda: P.pconv_distill_grad(*args, p, p, 0, 0, 8)
    yield "up_step", lambda: P.pconv_distill_grad(*args, p, p, 2, p, 8)


def test_c_entries_refuse_what_they_cannot_run():
    for what, call in c_calls():
        with pytest.raises(P.PconvError) as e:
            call()
        assert e.value.status == P.INVALID_ARG and what in str(e.value), (what, str(e.value))


def test_calls_on_the_host_are_refused():
    import torch
    z, t, c = torch.zeros(4, 8), torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int64)
    for call in (lambda: P.distill_loss(z, t, c), lambda: P.distill_loss(z.requires_grad_(), t, c), lambda: P.distill_loss_grad(z, t, c)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


@pytest.mark.gpu
def test_wrong_tensors_are_refused():
    import torch
    z = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")
    s, t, c = z(4, 8), z(4, 2), z(4, 2, dtype=torch.int64)
    for f in (P.distill_loss, P.distill_loss_grad):
        bad = [lambda: f(s.half(), t, c), lambda: f(s, t.double(), c), lambda: f(s, t, c.short()), lambda: f(s, t, c[:, :1]), lambda: f(s, t[:3], c[:3]),
               lambda: f(s[0], t, c), lambda: f(s.t(), t, c), lambda: f(s, t, c, reduction="batchmean"), lambda: f(s, t.cpu(), c), lambda: f(s, t[:1].expand(4, 2), c),
               lambda: f(s[:1].expand(4, 8), t, c)]
        for i, call in enumerate(bad):
            with pytest.raises(ValueError):
                call()
                pytest.fail(f"call {i} was not refused")
        for leaf in (s, s.clone().requires_grad_()):
            with pytest.raises(P.PconvError, match="temperature"):
                f(leaf, t, c, 0.0)
    for out in (z(4, 9), z(4, 8).bfloat16(), s, s.view(-1)[:32].view(4, 8)):
        with pytest.raises(ValueError):
            P.distill_loss_grad(s, t, c, out=out)
