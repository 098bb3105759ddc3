"""quantize_rows in every shape of its launch: threads of a row, vectors that a thread keeps, rows by which the shape is chosen, rows read
past the caches (more than 64 MiB of them) and not.  Equal to the definition, computed on the card by elementary operations."""
import pytest

import paper_1909_05073_amd as P

from gpu_util import say

# (vectors of 16 bytes in a row, rows)
SHAPES = [(8, 5000), (8, 600_000), (16, 5000), (16, 300_000), (32, 5000), (32, 150_000), (64, 5000), (64, 80_000),
          (128, 4096), (128, 4097), (66, 100_000), (128, 40_000), (256, 3000), (256, 20_000), (260, 8192), (512, 8192), (257, 8193), (512, 9000),
          (300, 8000), (1000, 3000), (1024, 6000), (1500, 127), (2048, 128), (2048, 5000), (4096, 127), (4096, 128), (3000, 2000), (5000, 60),
          (8192, 700), (8300, 700)]


@pytest.mark.gpu
@pytest.mark.parametrize("short", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vecs,rows", SHAPES)
def test_quantized_rows_in_every_shape(vecs, rows, dtype, short):
    import torch
    k = vecs * (4 if dtype == "f32" else 8) - short
    say(f"[case] quantize_rows {rows}x{k} {dtype}")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + k)
    x = torch.randn(rows, k, generator=gen, device="cuda")
    x *= torch.rand(rows, 1, generator=gen, device="cuda") + 0.01
    x[rows // 2] = 0
    x[rows - 1, k - 1] = 9.0                             # the last of all is its row's largest
    x = x.to(torch.bfloat16) if dtype == "bf16" else x
    q, scale = P.quantize_rows(x)
    x = x.float()
    most = x.abs().amax(1, keepdim=True)
    want = most / torch.full_like(most, 127.0)           # (by a tensor: by a number torch multiplies with its reciprocal)
    assert torch.equal(scale, want[:, 0])
    x = torch.where(want > 0, x / want, torch.zeros_like(x)).round()
    assert torch.equal(q, x.to(torch.int8))


@pytest.mark.gpu
def test_more_rows_than_workgroups():
    import torch
    rows = 34_000_001
    say(f"[case] quantize_rows {rows}x3 bf16")
    x = torch.randn(rows, 3, device="cuda").to(torch.bfloat16)
    q, scale = P.quantize_rows(x)
    most = x.float().abs().amax(1, keepdim=True)
    want = most / torch.full_like(most, 127.0)
    assert torch.equal(scale, want[:, 0])
    assert torch.equal(q, torch.where(want > 0, x.float() / want, torch.zeros_like(most)).round().to(torch.int8))


@pytest.mark.gpu
@pytest.mark.parametrize("lead", [(6,), (2, 3)])
@pytest.mark.parametrize("k,step", [(40, 48), (1008, 1008), (1024, 1024), (1025, 1040), (2000, 2000), (4112, 4112), (25089, 25104)])
def test_rows_lie_a_multiple_of_16_bytes_apart(k, step, lead):
    """So that rows whose length is one are contiguous."""
    import torch
    say(f"[case] steps of quantised rows of {k}")
    x = torch.randn(*lead, k, device="cuda")
    for t in (x, x.bfloat16()):
        q, scale = P.quantize_rows(t)
        assert q.shape == x.shape and q.stride()[-2:] == (step, 1) and q.is_contiguous() == (k % 16 == 0)
        if k % 16 == 0:
            assert torch.equal(q.view(-1).view(6, k), P.quantize_rows(t.view(6, k))[0])
