"""Outputs given to the 8-bit layers: they may lie beside the inputs, between their rows, and nowhere over them.

The tests on the host run the binding over a library that only takes notes."""
import numpy as np
import pytest

import paper_1909_05073_amd as P

from gpu_util import say
from test_i8_layers import check, make_layer8, make_x, plain_product, plain_quantize


class FakeLibrary:
    """Notes which calls reach it."""

    def __init__(self):
        self.calls = []

    def pconv_linear_i8_workspace(self, *sizes):
        return 0

    pconv_matmul_i8_workspace = pconv_linear_i8_workspace

    def pconv_linear_i8(self, *call):
        self.calls.append("linear")
        return P.OK

    def pconv_matmul_i8(self, *call):
        self.calls.append("matmul")
        return P.OK


@pytest.fixture
def notes(monkeypatch):
    import torch
    fake = FakeLibrary()
    monkeypatch.setattr(P, "_lib", fake)
    monkeypatch.setattr(P, "_stream", lambda index: None)
    monkeypatch.setattr(P, "_device_index", lambda *tensors: 0)
    monkeypatch.setattr(P, "_linear_i8_workspace", fake.pconv_linear_i8_workspace)
    monkeypatch.setattr(P, "_matmul_i8_workspace", fake.pconv_matmul_i8_workspace)
    return fake.calls


def over(m=6, n=8, k=8):
    """(what out lies over, call) with an out that shares memory with an input."""
    import torch
    i8 = torch.int8
    x, w, s, b = torch.zeros(m, k), torch.zeros(n, k, dtype=i8), torch.ones(n), torch.zeros(n)
    q, sa = torch.zeros(m, k, dtype=i8), torch.ones(m)
    yield "x", lambda: P.linear_i8(x, w, s, b, out=x)
    half = torch.zeros(m, k, dtype=torch.bfloat16)
    yield "x, bf16", lambda: P.linear_i8(half, w, s, b, out=half)
    wide = torch.zeros(m + 1, k)
    yield "x, a row further", lambda: P.linear_i8(wide[:m], w, s, b, out=wide[1:])
    room = torch.zeros(m, 2 * k)
    yield "x, one column", lambda: P.linear_i8(room[:, :k], w, s, b, out=room[:, k - 1:2 * k - 1])
    flat = torch.zeros(4096)
    bytes_of = lambda t: t.view(i8)
    yield "w", lambda: P.linear_i8(x, bytes_of(flat)[:n * k].view(n, k), s, b, out=flat[15:15 + m * n].view(m, n))
    yield "w_scale", lambda: P.linear_i8(x, w, flat[47:47 + n], b, out=flat[:m * n].view(m, n))
    yield "bias", lambda: P.linear_i8(x, w, s, flat[:n], out=flat[7:7 + m * n].view(m, n))
    yield "a", lambda: P.matmul_i8(bytes_of(flat)[2:2 + m * k].view(m, k), sa, w, s, out=flat[:m * n].view(m, n))
    yield "a_scale", lambda: P.matmul_i8(q, flat[m * n - 1:m * n - 1 + m], w, s, out=flat[:m * n].view(m, n))
    yield "b", lambda: P.matmul_i8(q, sa, bytes_of(flat)[:n * k].view(n, k), s, out=flat[15:15 + m * n].view(m, n))
    # rows of other distances: of x 9 elements, of out 16 between rows of 8; they meet further down only
    yield "x, other distances", lambda: P.linear_i8(flat.as_strided((m, k), (9, 1), 8), w, s, b, out=flat.as_strided((m, n), (16, 1), 24))


def beside(m=6, n=8, k=8):
    import torch
    i8 = torch.int8
    x, w, s, b = torch.zeros(m, k), torch.zeros(n, k, dtype=i8), torch.ones(n), torch.zeros(n)
    q, sa = torch.zeros(m, k, dtype=i8), torch.ones(m)
    room = torch.zeros(m, 2 * k)
    yield lambda: P.linear_i8(room[:, :k], w, s, b, out=room[:, k:])
    yield lambda: P.linear_i8(room[:, k:], w, s, b, out=room[:, :k])
    room1 = torch.zeros(2 * m, k)
    yield lambda: P.linear_i8(room1[::2], w, s, b, out=room1[1::2])
    flat = torch.zeros(4096)
    yield lambda: P.linear_i8(flat[:m * k].view(m, k), w, s, b, out=flat[m * k:m * k + m * n].view(m, n))
    yield lambda: P.linear_i8(flat[m * n:m * n + m * k].view(m, k), w, s, b, out=flat[:m * n].view(m, n))
    yield lambda: P.linear_i8(x, flat.view(i8)[:n * k].view(n, k), flat[400:400 + n], flat[500:500 + n], out=flat[16:16 + m * n].view(m, n))
    yield lambda: P.matmul_i8(flat.view(i8)[:m * k].view(m, k), flat[200:200 + m], w, s, out=flat[100:100 + m * n].view(m, n))
    # rows of x at 0, 32, 64 ..; those of out, of 8, in the gaps, two of x's rows apart
    yield lambda: P.linear_i8(flat.as_strided((m, k), (32, 1), 0), w, s, b, out=flat.as_strided((m, n), (64, 1), 8))
    yield lambda: P.linear_i8(x[:0], w, s, b, out=x[:0])
    yield lambda: P.linear_i8(x, w, s, b, out=torch.zeros(m, n))
    yield lambda: P.matmul_i8(q, sa, w, s, out=torch.zeros(m, n, dtype=torch.bfloat16))


def test_outputs_over_an_input_are_refused(notes):
    for what, call in over():
        with pytest.raises(ValueError, match="overlap"):
            call()
            pytest.fail(f"out over {what} was not refused")
    assert notes == []


def test_outputs_beside_the_inputs_are_not(notes):
    calls = list(beside())
    for call in calls:
        call()
    assert len(notes) == len(calls)


def test_runs_of_rows_share_memory_as_their_bytes_do():
    """Against the sets of their bytes, for rows of all kinds of distances."""
    rng = np.random.default_rng(0)
    seen = [0, 0]
    for _ in range(4000):
        a, b = ((int(rng.integers(0, 60)), int(rng.integers(1, 7)), int(rng.integers(1, 6)), int(rng.integers(0, 20))) for _ in range(2))
        a, b = ((at, rows, size, size + apart) for at, rows, size, apart in (a, b))
        bytes_of = lambda r: {r[0] + i * r[3] + j for i in range(r[1]) for j in range(r[2])}
        want = bool(bytes_of(a) & bytes_of(b))
        seen[want] += 1
        assert P._share(a, b) == want and P._share(b, a) == want, (a, b)
    assert min(seen) > 500


@pytest.mark.gpu
def test_outputs_between_the_rows_of_the_activations():
    import torch
    say("[case] linear_i8, outputs between the rows of x")
    rng = np.random.default_rng(2)
    for m, n, k in ((3, 40, 256), (200, 136, 64), (70, 130, 700)):
        w, sb, bias = (torch.from_numpy(a).cuda() for a in make_layer8(rng, n, k))
        room = torch.zeros(m, k + n, device="cuda")
        room[:, :k] = torch.from_numpy(make_x(rng, m, k)).cuda()
        was = room[:, :k].clone()
        q, sa = plain_quantize(was.cpu().numpy())
        want, bound = plain_product(q, sa, w.cpu().numpy(), sb.cpu().numpy(), bias.cpu().numpy(), True)
        check(P.linear_i8(room[:, :k], w, sb, bias, relu=True, out=room[:, k:]), want, bound, f"{m}x{n}x{k}")
        assert torch.equal(room[:, :k], was)
    with pytest.raises(ValueError, match="overlap"):
        P.linear_i8(room[:, :k], w, sb, bias, out=room[:, k - n:k])


def test_runs_of_memory_that_share_no_byte_are_apart():
    import torch
    apart = P._tensor_list_calls().apart
    flat = torch.zeros(100)
    out = flat[20:40].view(4, 5)
    assert apart(out, flat[:20], None, flat[40:], torch.zeros(7), flat[20:20])
    assert not apart(out, flat[:21]) and not apart(out, None, flat[39:]) and not apart(out, out) and not apart(out, flat.view(torch.int8)[159:160])
    assert apart(flat[:80].view(4, 20)[:, 5:10], flat[70:]) and not apart(flat[:80].view(4, 20)[:, 5:10], flat[69:70])
    assert apart(out[:0], flat) and apart(flat[:0], flat)
    for wrong in ((out, 3), (None, out)):
        with pytest.raises(TypeError):
            apart(*wrong)
