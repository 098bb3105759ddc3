"""Operators around the pruned convolutions, as cases to be measured.

The library prunes, packs and runs the 3x3 layers of a network.  Two more things belong to such a network.  While it
is pruned it is trained, and each step limits the norm of the gradients of all its tensors together (`GradList.clip`).
When it serves, what is no 3x3 layer is a matrix product: the 1x1 layers of a residual network with channels last (a
row for each pixel) and the fully connected layers of a classifier (a row for each image).  Those run in 8-bit
integers with a scale for each row of the activations, found in the call, and for each output channel of the weights
(`linear_i8`; or `quantize_rows` once and `matmul_i8` for each layer that reads the same activations).

    scale[m] = max_k |x[m,k]| / 127                  q[m,k] = nearest whole number, ties to even, of x[m,k] / scale[m]
    y[m,n]   = act((sum_k q[m,k] w[n,k]) * scale[m] * w_scale[n] + bias[n])

    norm = sqrt(sum over all tensors of g^2)         out = g * min(1, max_norm / (norm + 1e-6))

The scale and the quotient are numbers of 32 bits (the nearest); rows that hold only zeros have scale 0 and q 0.
"""
import math
import random

import torch

from pconv_inputs import resnet50_conv3x3_shapes, vgg16_conv_shapes

own = False

_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_EL = {"f32": 4, "bf16": 2}


# ---- cases -----------------------------------------------------------------------------------------------------------

def _linear(name, m, k, n, dtype, relu=False, bias=True, pad=0):
    """One layer; `pad`: the rows of activations and weights are that much further apart than they are long."""
    return dict(name=name, kind="linear", m=m, k=k, n=n, dtype=dtype, relu=relu, bias=bias, pad=pad)


def _shared(name, m, k, n, n2, dtype, relu=False, bias=True, pad=0):
    """Two layers that read the same activations."""
    return dict(name=name, kind="shared", m=m, k=k, n=n, n2=n2, dtype=dtype, relu=relu, bias=bias, pad=pad)


def _clip(name, net, dtype, out, max_norm, tensors=0, total=0, shape_seed=0, align=64):
    """`out`: the type of the clipped gradients; `align`: what the places of the tensors in their buffers are multiples of."""
    return dict(name=name, kind="clip", net=net, dtype=dtype, out=out, max_norm=max_norm, tensors=tensors, total=total,
                shape_seed=shape_seed, align=align)


def listed():
    return [
        # the smallest call: ten classes for one small image; launch and host time are all of it
        _linear("linear_f32_1x512_10", 1, 512, 10, "f32"),
        # the classifier of a residual network, one image at a time
        _linear("linear_bf16_1x2048_1000", 1, 2048, 1000, "bf16"),
        # the first fully connected layer of VGG-16 for single images: reading the weights is all of it
        _linear("linear_f32_1x25088_4096", 1, 25088, 4096, "f32", relu=True),
        # the same with the batch that the benchmark has
        _linear("linear_f32_32x25088_4096", 32, 25088, 4096, "f32", relu=True),
        # 1x1 layer of ResNet-50's first stage, batch 32, channels last: long and thin, activations are all of it
        _linear("linear_bf16_100352x64_256", 100352, 64, 256, "bf16"),
        # 1x1 layer of its last stage: few pixels, many channels
        _linear("linear_bf16_1568x512_2048", 1568, 512, 2048, "bf16", relu=True),
        # a wide layer over many rows, the largest: the matrix units are all of it
        _linear("linear_bf16_8192x4096_4096", 8192, 4096, 4096, "bf16"),
        # entry of a stage: two 1x1 layers read the same pixels
        _shared("shared_bf16_25088x256_128_512", 25088, 256, 128, 512, "bf16", relu=True),
        # sizes that are multiples of nothing, rows that lie apart and start anywhere, no bias
        _shared("shared_f32_odd", 777, 1155, 1001, 130, "f32", bias=False, pad=3),
        # gradients of one little layer, below the limit: launch and host time are all of it
        _clip("clip_f32_layer", "layer", "f32", "f32", 1.0),
        # the 3x3 layers of ResNet-50, bf16 gradients to fp32 ones for the weights kept in fp32
        _clip("clip_bf16_resnet50", "resnet50", "bf16", "f32", 1.0),
        # all of VGG-16, the fully connected layers too
        _clip("clip_f32_vgg16", "vgg16", "f32", "f32", 1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.35:
        total = _log_int(rng, 2000, 1.2e8)
        c = _clip("", "drawn", rng.choice(["f32", "f32", "bf16", "mixed"]), rng.choice(["same", "f32"]),
                  rng.choice([0.1, 1.0, 10.0]), tensors=_log_int(rng, 1, 300), total=total,
                  shape_seed=rng.randrange(1 << 30), align=rng.choice([64, 64, 1]))
        del c["name"]
        return c
    while True:
        m, k, n = _log_int(rng, 1, 100352), _log_int(rng, 16, 25088), _log_int(rng, 8, 4096)
        if rng.random() < 0.3:
            m = _log_int(rng, 1, 32)                 # serving: a few images
        if rng.random() < 0.6:                       # most layers have round channel counts
            k, n = max(16, k // 16 * 16), max(8, n // 8 * 8)
        pad = rng.choice([0, 0, 0, 16, 3])
        args = dict(dtype=rng.choice(["f32", "bf16"]), relu=rng.random() < 0.5, bias=rng.random() < 0.8, pad=pad)
        if rng.random() < 0.7:
            c = _linear("", m, k, n, **args)
        else:
            c = _shared("", m, k, n, _log_int(rng, 8, 2048), **args)
        del c["name"]
        w = work(c)
        if 1e4 < w["flops"] < 2.7e11 and w["bytes"] < 5e8 and m * k < 1.2e8 and k * n < 1.1e8:
            return c


def _tensors(case):
    """(elements, type) of each tensor whose gradient is clipped."""
    if case["net"] == "layer":
        sizes = [16 * 16 * 9, 16]
    elif case["net"] == "resnet50":
        sizes = [s for c, _, _ in resnet50_conv3x3_shapes() for s in (c * c * 9, c)]
    elif case["net"] == "vgg16":
        sizes = [s for ci, co, _, _ in vgg16_conv_shapes() for s in (ci * co * 9, co)]
        sizes += [25088 * 4096, 4096, 4096 * 4096, 4096, 4096 * 1000, 1000]
    else:
        rng = random.Random(case["shape_seed"])
        share = [math.exp(rng.gauss(0.0, 2.0)) for _ in range(case["tensors"])]
        sizes = [max(1, int(case["total"] * s / sum(share))) for s in share]
    mixed = case["dtype"] == "mixed"
    return [(s, ("bf16", "f32")[i % 2] if mixed else case["dtype"]) for i, s in enumerate(sizes)]


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _apart(x, pad):
    """The same rows, `pad` elements further apart."""
    if not pad:
        return x
    wide = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _layer(case, n, gen):
    """8-bit weights with the scales of their rows, and a bias: what such a program keeps of a layer."""
    k = case["k"]
    w = torch.empty(n, k, device="cuda").normal_(generator=gen)
    scale = w.abs().amax(1) / 127
    q = (w / scale[:, None]).round().clamp(-127, 127).to(torch.int8)
    bias = torch.empty(n, device="cuda").normal_(generator=gen) if case["bias"] else None
    return dict(w=_apart(q, case["pad"]), scale=scale * math.sqrt(2.0 / k), bias=bias)


def _buffers(sizes, align, like):
    """A tensor of each size, in one buffer for each type."""
    offs, end = [], {t: 0 for t in _TYPE}
    for s, t in zip(sizes, like):
        offs.append(end[t])
        end[t] = -(-(end[t] + s) // align) * align
    flat = {t: torch.zeros(e, dtype=_TYPE[t], device="cuda") for t, e in end.items() if e}
    return [flat[t][o:o + s] for o, s, t in zip(offs, sizes, like)], flat


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["kind"] == "clip":
        sizes, types = zip(*_tensors(case))
        grads, flat = _buffers(sizes, case["align"], types)
        # each tensor has its own size of gradient, as the layers of a network have
        for i, g in enumerate(grads):
            g.normal_(generator=gen).mul_(0.02 * (0.5 + (i * 7 % 5)))
        out_types = types if case["out"] == "same" else [case["out"]] * len(types)
        out, out_flat = _buffers(sizes, case["align"], out_types)
        return dict(case=case, grads=grads, flat=flat, out=out, out_flat=out_flat)
    x = torch.empty(case["m"], case["k"], device="cuda").normal_(generator=gen)
    # activations after a ReLU, the channels of different sizes
    x = x.clamp_(min=0).mul_(torch.empty(case["k"], device="cuda").uniform_(0.25, 2.0, generator=gen))
    x = _apart(x.to(_TYPE[case["dtype"]]), case["pad"])
    layers = [_layer(case, n, gen) for n in ([case["n"]] if case["kind"] == "linear" else [case["n"], case["n2"]])]
    return dict(case=case, x=x, layers=layers)


# ---- one pass --------------------------------------------------------------------------------------------------------

def _plain_quantized(x):
    x = x.float()
    most = x.abs().amax(1, keepdim=True)
    scale = most / torch.full_like(most, 127.0)      # (by a tensor: by a number torch multiplies with its reciprocal)
    return torch.where(scale > 0, (x / scale).round().clamp(-127, 127), torch.zeros_like(x)), scale


def _plain_product(q, scale, layer, relu, dtype):
    y = q @ layer["w"].float().t() * (scale * layer["scale"])
    if layer["bias"] is not None:
        y = y + layer["bias"]
    return (y.clamp(min=0) if relu else y).to(dtype)


def _plain(state):
    case = state["case"]
    if case["kind"] == "clip":
        grads = [g.float() for g in state["grads"]]
        norm = torch.stack([g.square().sum() for g in grads]).sum().sqrt()
        coef = (case["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
        _ = [o.copy_(g * coef) for o, g in zip(state["out"], grads)]
        return {"norm": norm, "clipped": state["out_flat"]}
    q, scale = _plain_quantized(state["x"])
    return [_plain_product(q, scale, ly, case["relu"], state["x"].dtype) for ly in state["layers"]]


def run(state):
    if not own:
        return _plain(state)
    import paper_1909_05073_amd as P
    case = state["case"]
    if case["kind"] == "clip":
        plan = state.get("plan")
        if plan is None:                             # made once for the tensors of a network, as its optimizer is
            plan = state["plan"] = P.GradList(state["grads"], out=state["out"])
        return {"norm": plan.clip(case["max_norm"]), "clipped": state["out_flat"]}
    x, layers, relu = state["x"], state["layers"], case["relu"]
    if case["kind"] == "linear":
        ly = layers[0]
        return [P.linear_i8(x, ly["w"], ly["scale"], ly["bias"], relu=relu)]
    q, scale = P.quantize_rows(x)
    return [P.matmul_i8(q, scale, ly["w"], ly["scale"], ly["bias"], relu=relu, out_dtype=x.dtype) for ly in layers]


# ---- what a pass cannot do without, and what is exact ---------------------------------------------------------------

def work(case):
    if case["kind"] == "clip":
        t = _tensors(case)
        out = [_EL[d if case["out"] == "same" else case["out"]] for _, d in t]
        return {"bytes": float(sum(s * (_EL[d] + o) for (s, d), o in zip(t, out)) + 4), "flops": 3.0 * sum(s for s, _ in t)}
    m, k, el = case["m"], case["k"], _EL[case["dtype"]]
    n = case["n"] + (case["n2"] if case["kind"] == "shared" else 0)
    return {"bytes": float(m * k * el + n * k + (8 if case["bias"] else 4) * n + m * n * el), "flops": 2.0 * m * n * k}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "clip":
        total = sum(float(f.double().dot(f.double())) for f in s["flat"].values())     # (the gaps hold zeros)
        norm = math.sqrt(total)
        coef = min(1.0, case["max_norm"] / (norm + 1e-6))
        flat = {t: torch.zeros(f.numel(), dtype=torch.float64, device="cuda") for t, f in s["out_flat"].items()}
        for o, g in zip(s["out"], s["grads"]):
            t = "f32" if o.dtype == torch.float32 else "bf16"
            at = o.storage_offset()
            flat[t][at:at + o.numel()] = g.double() * coef
        return {"norm": torch.tensor(norm, dtype=torch.float64), "clipped": flat}
    x = s["x"].double()
    scale = (x.abs().max(1).values / 127).float().double()
    step = torch.where(scale > 0, scale, torch.ones_like(scale))[:, None]
    q = torch.round((x / step).float()).double()
    got = []
    for ly in s["layers"]:
        y = torch.matmul(q, ly["w"].double().t().contiguous())
        y = y * scale[:, None] * ly["scale"].double()[None, :]
        if ly["bias"] is not None:
            y = y + ly["bias"].double()[None, :]
        got.append(torch.relu(y) if case["relu"] else y)
    return got
