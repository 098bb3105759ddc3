"""Calls whose workgroups share units of work and wait for each other, with other such calls on the same GPU."""
import os
import subprocess

import pytest

import paper_1909_05073_amd as P
from pconv_inputs import base_seed, config_layers, make_input, make_layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def shares_check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("shares") / "shares_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Wextra", "-I", os.path.join(ROOT, "paper_1909_05073_amd", "csrc"),
                    os.path.join(ROOT, "tests", "shares_check.cpp"), "-o", exe], check=True)
    return lambda *args: subprocess.run([exe, *args], capture_output=True, text=True, timeout=120)


def test_launches_end_in_whatever_order_the_xcds_start_them(shares_check):
    r = shares_check()
    assert r.returncode == 0, r.stdout


def test_places_by_id_across_xcds_would_not(shares_check):
    """Why the set of all workgroups deals its places out as they start: by their ids, launches that XCDs begin in
    different orders wait for each other for ever (and the bounded waits end in wrong outputs)."""
    r = shares_check("by_id")
    assert r.returncode == 0, r.stdout


@pytest.mark.gpu
@pytest.mark.parametrize("split_units", [1, 2])
def test_calls_that_become_ready_at_once(split_units):
    """Four streams wait for one event, so that the GPU may begin their calls in any order; each call has as many workgroups as the
    GPU has places."""
    import torch
    spec = config_layers(2)[0]
    L = make_layer(spec, base_seed(2))
    h = P.pconv_pack(L["w"], L["pattern_id"], L["conn"], L["table"], "f32")
    P.pconv_debug_set_tiling(0, -1, split_units)
    try:
        assert P.pconv_debug_plan(h, 1, spec.h, spec.w).split_units == split_units
        b = torch.from_numpy(L["bias"]).cuda()
        xs = [torch.from_numpy(make_input(spec, base_seed(2) + 7 * k)).cuda() for k in range(4)]
        refs = [P.conv2d(h, x, b, relu=True).clone() for x in xs]
        busy = torch.randn(4096, 4096, device="cuda")
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in xs]
        for turn in range(6):
            print(f"[case] split={split_units} turn {turn}", flush=True)
            busy @ busy                              # the event comes when all calls have been handed in
            event = torch.cuda.Event()
            event.record()
            outs = []
            for s, x in zip(streams, xs):
                s.wait_event(event)
                with torch.cuda.stream(s):
                    outs.append([P.conv2d(h, x, b, relu=True) for _ in range(3)])
            for s in streams:
                s.synchronize()
            for k, ys in enumerate(outs):
                for i, y in enumerate(ys):
                    assert torch.equal(y, refs[k]), f"turn {turn}, stream {k}, call {i}"
        P.pconv_get_async_error(h)                   # no wait ran out
    finally:
        P.pconv_debug_set_tiling(0, -1, -1)
        h.free()
