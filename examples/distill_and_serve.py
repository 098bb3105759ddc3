"""A pruned network learns from the network that it was cut from, and serves in few bits.

    python examples/distill_and_serve.py

The network: a 3x3 layer and a 1x1 layer beside it, their sum normalised over the channels, a 1x1 layer, the mean over the pixels, a
classifier.  The teacher is trained on labels.  The student has the teacher's weights with the 3x3 layer pruned
(`pconv_project`) and learns, with the kernels that were cut staying zero, from the teacher's largest logits alone
(`distill_loss`), the norm of its gradients limited (`GradList.clip`).  Serving: the packed 3x3 layer (`conv2d`, channels
last), the 1x1 layer beside it (`linear_i8`), sum, norm and quantising in one (`add_rms_norm_i8`), the layer that reads it (`matmul_i8`),
the classifier in 4-bit floats (`linear_mx4`).
"""
import os
import sys

import numpy as np
import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1909_05073_amd as P
from pconv_inputs import PATTERN_TABLE

C_IN, C_MID, C_OUT, CLASSES, SIDE, TOP, EPS = 16, 32, 64, 20, 10, 5, 1e-5


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
    return dict(conv=make(C_MID, C_IN, 3, 3, fan=9 * C_IN), conv_b=zero(C_MID), beside=make(C_MID, C_IN, fan=C_IN),
                gain=torch.ones(C_MID, device="cuda", requires_grad=True), point=make(C_OUT, C_MID, fan=C_MID), point_b=zero(C_OUT),
                fc=make(CLASSES, C_OUT, fan=C_OUT), fc_b=zero(CLASSES))


def forward(p, x):
    """The network in fp32.  (The 3x3 layer as one product over its taps.)"""
    taps = F.unfold(x.permute(0, 3, 1, 2), 3, padding=1).transpose(1, 2)         # [n, pixels, c_in * 9]
    y = (taps.reshape(-1, C_IN * 9) @ p["conv"].reshape(C_MID, -1).t() + p["conv_b"]).clamp(min=0)
    s = y + x.reshape(-1, C_IN) @ p["beside"].t()
    h = s * (s.square().mean(1, keepdim=True) + EPS).rsqrt() * p["gain"]
    y = (h @ p["point"].t() + p["point_b"]).clamp(min=0)
    return y.view(x.shape[0], -1, C_OUT).mean(1) @ p["fc"].t() + p["fc_b"]


def prune(p, keep=C_MID * C_IN // 2):
    """The student: (parameters, the mask of its 3x3 layer, pattern ids, connectivity)."""
    host, table = p["conv"].detach().cpu().numpy(), PATTERN_TABLE[:8]
    pid, conn = P.pconv_project(host, table, keep)
    mask = (((table[pid][:, :, None] >> np.arange(9)) & 1) * conn[:, :, None]).reshape(host.shape).astype(np.float32)
    mask = torch.from_numpy(mask).cuda()
    student = {k: t.detach().clone() for k, t in p.items()}
    student["conv"] *= mask
    return {k: t.requires_grad_() for k, t in student.items()}, mask, pid, conn


def train(p, loss_of, steps, rate, mask=None, max_norm=1.0, batch=64):
    """Steps on loss_of(logits, images, labels), the gradients limited together; returns losses and norms before the limit."""
    for t in p.values():
        t.grad = torch.zeros_like(t)
    grads = P.GradList([t.grad for t in p.values()])     # the buffers stay: they are cleared, not replaced
    losses, norms = [], []
    for step in range(steps):
        x, label = images(batch, seed=step)
        for t in p.values():
            t.grad.zero_()
        loss = loss_of(forward(p, x), x, label)
        loss.backward()
        if mask is not None:
            p["conv"].grad *= mask
        losses.append(loss.detach())
        norms.append(grads.clip(max_norm))
        with torch.no_grad():
            for t in p.values():
                t -= rate * t.grad
    return torch.stack(losses), torch.stack(norms)


def from_teacher(teacher, temperature=2.0):
    """The student's loss: its distance from the teacher's largest logits for the same images."""
    def loss_of(logits, x, label):
        with torch.no_grad():
            top, classes = forward(teacher, x).topk(TOP, 1)
        return P.distill_loss(logits, top, classes, temperature)
    return loss_of


class Served:
    """The student as it serves."""

    def __init__(self, p, pid, conn):
        get = {k: t.detach() for k, t in p.items()}
        self.conv = P.pconv_pack(get["conv"].cpu().numpy(), pid, conn, PATTERN_TABLE[:8], "f32")
        self.conv_b, self.gain, self.point_b, self.fc_b = (get[k] for k in ("conv_b", "gain", "point_b", "fc_b"))
        self.beside, self.point, self.fc = P.quantize_rows(get["beside"]), P.quantize_rows(get["point"]), P.quantize_mx4(get["fc"])

    def __call__(self, x):
        y = P.conv2d(self.conv, x, self.conv_b, relu=True, layout="nhwc")
        q, scale, _ = P.add_rms_norm_i8(y, P.linear_i8(x, *self.beside), self.gain, EPS, out=y)
        y = P.matmul_i8(q, scale, *self.point, self.point_b, relu=True)
        return P.linear_mx4(y.mean((1, 2)), *self.fc, self.fc_b)


def main(steps=60, say=print):
    """Trains both, serves the student; returns (the student's losses, norms, accuracies of teacher, student and the served one)."""
    teacher = parameters()
    train(teacher, lambda logits, x, label: F.cross_entropy(logits, label), steps, 0.2)
    student, mask, pid, conn = prune(teacher)
    losses, norms = train(student, from_teacher(teacher), steps, 0.1, mask)
    served = Served(student, pid, conn)
    x, label = images(256, seed=10_000)
    with torch.no_grad():
        right = [(logits.argmax(1) == label).float().mean().item() for logits in (forward(teacher, x), forward(student, x), served(x))]
    say(f"loss {losses[0].item():.3f} -> {losses[-1].item():.3f}; right: teacher {100 * right[0]:.0f} %, student {100 * right[1]:.0f} %, "
        f"served {100 * right[2]:.0f} %")
    return losses, norms, right


if __name__ == "__main__":
    main()
