"""From training to serving: a little network is pruned with the alternating method, its gradients limited together, and
then served with the pruned convolution and layers in 8-bit integers.

    python examples/prune_and_serve.py

Training (torch, fp32): the loss and, for the 3x3 weights W, the penalty rho/2 |W - Z + U|^2 that pulls them to the
nearest weights Z of the pruned form.  `pconv_project` finds Z from W + U every few steps; each time the penalty's gradient jumps, so
every step limits the norm of all gradients (`GradList.clip`).  Serving: the 3x3 layer is packed (`pconv_pack`, `conv2d`, channels
last), the 1x1 layer and the classifier are quantised (`quantize_rows`) and run as products of 8-bit integers
(`linear_i8`): a row for each pixel, a row for each image.
"""
import os
import sys

import numpy as np
import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1909_05073_amd as P
from pconv_inputs import PATTERN_TABLE

C_IN, C_MID, C_OUT, CLASSES, SIDE = 16, 32, 64, 10, 12


def images(count, seed):
    """Images [count, SIDE, SIDE, C_IN] of CLASSES kinds: a direction of its own over the channels for each, and noise."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1909)
    kinds = torch.randn(CLASSES, C_IN, generator=gen, device="cuda")
    gen.manual_seed(seed)
    label = torch.randint(CLASSES, (count,), generator=gen, device="cuda")
    noise = torch.randn(count, SIDE, SIDE, C_IN, generator=gen, device="cuda")
    return (kinds[label][:, None, None, :] + noise).clamp(min=0), label


def parameters(seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    make = lambda *shape, fan: (torch.randn(*shape, generator=gen, device="cuda") * (2.0 / fan) ** 0.5).requires_grad_()
    zero = lambda n: torch.zeros(n, device="cuda", requires_grad=True)
    return dict(conv=make(C_MID, C_IN, 3, 3, fan=9 * C_IN), conv_b=zero(C_MID), point=make(C_OUT, C_MID, fan=C_MID),
                point_b=zero(C_OUT), fc=make(CLASSES, C_OUT, fan=C_OUT), fc_b=zero(CLASSES))


def forward(p, x, conv=None):
    """The network in fp32: 3x3, 1x1, mean over the pixels, classifier.  (The 3x3 layer as one product over its taps.)"""
    w = p["conv"] if conv is None else conv
    taps = F.unfold(x.permute(0, 3, 1, 2), 3, padding=1).transpose(1, 2)         # [n, pixels, c_in * 9]
    y = (taps.reshape(-1, C_IN * 9) @ w.reshape(C_MID, -1).t() + p["conv_b"]).clamp(min=0)
    y = (y @ p["point"].t() + p["point_b"]).clamp(min=0)
    y = y.view(x.shape[0], -1, C_OUT).mean(1)
    return y @ p["fc"].t() + p["fc_b"]


def project(w, keep):
    """The nearest weights of the pruned form: (weights, pattern ids, connectivity)."""
    host = w.detach().cpu().numpy()
    table = PATTERN_TABLE[:8]
    pid, conn = P.pconv_project(host, table, keep)
    taps = (table[pid][:, :, None] >> np.arange(9)) & 1
    mask = (taps * conn[:, :, None]).reshape(host.shape).astype(np.float32)
    return torch.from_numpy(host * mask).to(w.device), pid, conn


def train(p, steps=60, every=15, rho=0.3, max_norm=1.0, rate=0.2, batch=64, keep=C_MID * C_IN // 2, say=print):
    """Returns the norms of the gradients before they were limited."""
    names = list(p)
    for t in p.values():
        t.grad = torch.zeros_like(t)
    grads = P.GradList([t.grad for t in p.values()])     # the buffers stay: they are cleared, not replaced
    dual = torch.zeros_like(p["conv"])
    near = project(p["conv"], keep)[0]
    norms = []
    for step in range(steps):
        x, label = images(batch, seed=step)
        loss = F.cross_entropy(forward(p, x), label) + 0.5 * rho * (p["conv"] - near + dual).square().sum()
        for t in p.values():
            t.grad.zero_()
        loss.backward()
        norms.append(grads.clip(max_norm))
        with torch.no_grad():
            for name in names:
                p[name] -= rate * p[name].grad
        if (step + 1) % every == 0:
            with torch.no_grad():
                near = project(p["conv"] + dual, keep)[0]
                dual += p["conv"] - near
            say(f"step {step + 1}: loss {loss.item():.3f}, norm of the gradients {norms[-1].item():.3f}")
    return torch.stack(norms)


class Served:
    """The trained network as it serves: packed, quantised, nothing of torch but memory and the mean over the pixels."""

    def __init__(self, p, keep=C_MID * C_IN // 2):
        self.pruned, pid, conn = project(p["conv"], keep)
        self.conv = P.pconv_pack(p["conv"].detach().cpu().numpy(), pid, conn, PATTERN_TABLE[:8], "f32")
        self.conv_b, self.point_b, self.fc_b = (p[k].detach() for k in ("conv_b", "point_b", "fc_b"))
        self.point, self.point_scale = P.quantize_rows(p["point"].detach())
        self.fc, self.fc_scale = P.quantize_rows(p["fc"].detach())

    def __call__(self, x):
        y = P.conv2d(self.conv, x, self.conv_b, relu=True, layout="nhwc")
        y = P.linear_i8(y, self.point, self.point_scale, self.point_b, relu=True)
        return P.linear_i8(y.mean((1, 2)), self.fc, self.fc_scale, self.fc_b)


def main(steps=60, say=print):
    """Trains, serves; returns (norms, accuracy, relative distance of the served logits from the pruned network's in fp32)."""
    p = parameters()
    norms = train(p, steps=steps, say=say)
    served = Served(p)
    x, label = images(256, seed=10_000)
    logits = served(x)
    with torch.no_grad():
        want = forward(p, x, conv=served.pruned)
    right = (logits.argmax(1) == label).float().mean().item()
    far = ((logits - want).norm() / want.norm()).item()
    say(f"served: {100 * right:.0f} % right, logits {100 * far:.2f} % from the pruned network in fp32")
    return norms, right, far


if __name__ == "__main__":
    main()
