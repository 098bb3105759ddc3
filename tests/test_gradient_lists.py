"""What a list of gradients keeps from one call to the next, and what it must not: the tensors, not where they lay.

The tests on the host run the binding over a library that only takes notes; those on the card compare with 64 bits under the
bounds of test_gradients.py."""
import ctypes as C

import numpy as np
import pytest

import paper_1909_05073_amd as P

from gpu_util import say
from test_gradients import check, host, plain


class FakeLibrary:
    """Notes what it is given."""

    def __init__(self):
        self.calls = []

    def pconv_grad_workspace(self, num):
        return 64

    def pconv_grad_norm(self, grads, counts, types, num, norm, work, size, stream):
        self.calls.append((list(grads), None, list(counts), list(types), None))
        return P.OK

    def pconv_clip_grads(self, grads, outs, counts, types, out_types, num, max_norm, eps, norm, work, size, stream):
        self.calls.append((list(grads), list(outs), list(counts), list(types), list(out_types)))
        return P.OK


@pytest.fixture
def notes(monkeypatch):
    """The calls that reach the library, with tensors in host memory."""
    import torch
    fake = FakeLibrary()
    monkeypatch.setattr(P, "_lib", fake)
    monkeypatch.setattr(P, "_stream", lambda index: None)
    monkeypatch.setattr(P, "_device_index", lambda *tensors: 0 if tensors else -1)
    monkeypatch.setattr(P, "_current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return fake.calls


def changes():
    """(name, what gives a tensor of 60 elements other memory, another size or type)."""
    import torch
    yield "data", lambda t: setattr(t, "data", torch.ones(60))
    yield "set_", lambda t: t.set_(torch.ones(60))
    yield "grown", lambda t: t.resize_(6000)
    yield "cut", lambda t: t.resize_(7)
    yield "first part", lambda t: setattr(t, "data", t.data[:11])
    yield "storage", lambda t: (t.untyped_storage().resize_(0), t.untyped_storage().resize_(4 * 60))
    yield "type", lambda t: setattr(t, "data", torch.ones(60, dtype=torch.bfloat16))
    yield "type of the same bytes", lambda t: setattr(t, "data", t.data.view(torch.bfloat16))


@pytest.mark.parametrize("which", range(8))
@pytest.mark.parametrize("side", ["in place", "gradient and output"])
def test_tensors_with_other_memory_are_seen(notes, which, side):
    import torch
    name, change = list(changes())[which]
    grads = [torch.ones(60), torch.ones(30)]
    outs = None if side == "in place" else [torch.zeros(60), torch.zeros(30)]
    plan = P.GradList(grads, outs)
    plan.clip(1.0)
    held = [torch.empty(60) for _ in range(8)]           # (so that new memory is other memory)
    for t in grads[:1] + (outs[:1] if outs else []):
        change(t)
    plan.clip(1.0)
    plan.norm()
    assert len(held) == 8 and len(notes) == 3
    for at, to, counts, types, out_types in notes[1:]:
        assert at == [g.data_ptr() for g in grads] and counts == [g.numel() for g in grads], name
        assert types == [P.BF16 if g.dtype == torch.bfloat16 else P.F32 for g in grads], name
        if to is not None:
            want = outs or grads
            assert to == [o.data_ptr() for o in want] and out_types == [P.BF16 if o.dtype == torch.bfloat16 else P.F32 for o in want], name


def test_another_order_of_dimensions_than_the_outputs_is_seen(notes):
    import torch
    grads, outs = [torch.ones(6, 10)], [torch.zeros(6, 10)]
    plan = P.GradList(grads, outs)
    grads[0].t_()
    with pytest.raises(ValueError, match="shape and the strides"):
        plan.clip(1.0)
    outs[0].t_()
    plan.clip(1.0)
    assert len(notes) == 1


def test_what_is_no_tensor_is_refused(notes):
    import torch
    plan = P.GradList([torch.ones(5)])
    plan.grads[0] = None
    for call in (plan.norm, lambda: P._tensor_list_calls().places((torch.ones(2),)), lambda: P._tensor_list_calls().places([3]),
                 lambda: P._tensor_list_calls().changed(torch.ones(2)), lambda: P._tensor_list_calls().changed([torch.ones(2), None])):
        with pytest.raises(TypeError):
            call()
    assert notes == []


def test_other_tensors_in_the_list_are_seen(notes):
    import torch
    plan = P.GradList([torch.ones(60), torch.ones(30)])
    plan.grads[1] = torch.ones(45)
    plan.clip(1.0)
    assert notes[0][0] == notes[0][1] == [g.data_ptr() for g in plan.grads] and notes[0][2] == [60, 45]


def test_changes_that_no_list_may_have_are_refused_until_they_are_gone(notes):
    import torch
    flat = torch.ones(200)
    grads = [flat[:60], flat[60:120]]
    plan = P.GradList(grads)
    was = grads[1].data
    grads[1].data = flat[59:119]                         # over the first
    for _ in range(2):
        with pytest.raises(ValueError, match="overlap"):
            plan.clip(1.0)
    grads[1].data = was
    plan.clip(1.0)
    assert len(notes) == 1 and notes[0][0] == [flat.data_ptr(), flat.data_ptr() + 240]
    grads[0].data = flat[:60].double()
    with pytest.raises(ValueError):
        plan.norm()
    assert len(notes) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("with_out", [False, True])
def test_clipping_follows_the_tensors_to_other_memory(with_out):
    import torch
    say(f"[case] clip after other memory, out {with_out}")
    rng = np.random.default_rng(4)
    fresh = lambda n: torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda()
    grads = [fresh(50_000), fresh(700), fresh(70_000)]
    outs = [torch.zeros_like(g) for g in grads] if with_out else None
    plan = P.GradList(grads, outs)
    plan.clip(1.0)
    grads[0].data = fresh(50_000)
    grads[1].set_(fresh(900))
    grads[2].resize_(90_000).normal_()
    if with_out:
        outs[1].resize_(900)
        outs[2].data = torch.zeros(90_000, device="cuda")
    else:
        outs = grads
    values = [host(g) for g in grads]
    want_norm, want = plain(values, 2.0)
    assert abs(float(plan.norm()) - want_norm) <= 1.01 * 2.0 ** -24 * want_norm
    check(plan.clip(2.0), outs, want_norm, want)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[40, 9], [300_000, 77], [50] * 170])
def test_an_infinite_limit_limits_nothing_and_a_limit_of_zero_leaves_no_nan(sizes):
    """By one workgroup, in two launches, and with a launch for the total."""
    import math
    import torch
    say(f"[case] clip, infinite norms and limits, norms and limits of zero, {len(sizes)} tensors")
    make = lambda: [torch.full((n,), 2.0, device="cuda") for n in sizes]
    for in_place in (True, False):
        grads = make()
        grads[0][3] = math.inf
        want = [g.clone() for g in grads]
        outs = grads if in_place else [torch.full_like(g, float("nan")) for g in grads]
        assert math.isinf(float(P.clip_grad_norm(grads, math.inf, out=None if in_place else outs)))
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
        grads[1][2] = math.nan                           # what is no number stays none
        assert math.isnan(float(P.clip_grad_norm(grads, math.inf, out=None if in_place else outs)))
        assert all(bool(torch.isnan(o).all()) for o in outs)
        grads = [g.zero_() for g in make()]
        outs = grads if in_place else [torch.full_like(g, float("nan")) for g in grads]
        assert float(P.clip_grad_norm(grads, 0.0, eps=0.0, out=None if in_place else outs)) == 0
        assert all(bool((o == 0).all()) for o in outs)
        grads = make()
        outs = grads if in_place else [torch.full_like(g, float("nan")) for g in grads]
        P.clip_grad_norm(grads, 0.0, eps=0.0, out=None if in_place else outs)
        assert all(bool((o == 0).all()) for o in outs)


def test_the_norm_alone_takes_tensors_that_overlap(notes):
    """Nothing is written: every tensor counts, as the formula says."""
    import torch
    flat = torch.ones(200)
    P.grad_norm([flat, flat, flat[50:90]])
    assert notes[0][0] == [flat.data_ptr(), flat.data_ptr(), flat.data_ptr() + 200] and notes[0][2] == [200, 200, 40]
    with pytest.raises(ValueError, match="overlap"):
        P.clip_grad_norm([flat, flat], 1.0)
    with pytest.raises(ValueError, match="dense"):
        P.grad_norm([flat[::2]])


@pytest.mark.gpu
def test_the_norm_of_tensors_that_overlap():
    import math
    import torch
    say("[case] grad_norm of tensors that overlap")
    flat = torch.full((50_000,), 2.0, device="cuda")
    want = math.sqrt(4.0 * 110_000)
    assert abs(float(P.grad_norm([flat, flat, flat[10:10_010]])) - want) <= 1.01 * 2.0 ** -24 * want
    assert bool((flat == 2.0).all())


def test_pointers_of_empty_tensors_are_not_looked_at():
    """The header promises it.  (The calls fail at the tensor behind the empty one, before anything is launched.)"""
    p, need = 1 << 20, P.pconv_grad_workspace(2)
    ptrs, i64, i32 = (lambda *v: (C.c_void_p * len(v))(*v)), (lambda *v: (C.c_int64 * len(v))(*v)), (lambda *v: (C.c_int32 * len(v))(*v))
    for odd in (p + 1, p + 2, None):
        with pytest.raises(P.PconvError, match="null pointer of a tensor"):
            P.pconv_grad_norm(ptrs(odd, None), i64(0, 4), i32(0, 0), 2, p, p, need)
        with pytest.raises(P.PconvError, match="null pointer of an output"):
            P.pconv_clip_grads(ptrs(odd, p), ptrs(odd, None), i64(0, 4), i32(0, 0), i32(0, 0), 2, 1.0, 0.0, p, p, need)
        with pytest.raises(P.PconvError, match="null pointer of an output"):
            P.pconv_clip_grads(ptrs(p, p), ptrs(odd, None), i64(0, 4), i32(0, 0), i32(0, 0), 2, 1.0, 0.0, p, p, need)
