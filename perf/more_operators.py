"""More operators around the pruned convolutions, as cases to be measured: layers in 4-bit floats, the norm before a layer in 8-bit
integers, and the loss that trains a pruned network towards its teacher.

Layers whose weights are read once a call go to 4 bits (`linear_mx4`; or `quantize_mx4` once and `matmul_mx4` for each layer that
reads the same rows).  32 neighbouring values of a row are a block with one power of two as its scale:

    scale[m,b] = 2^X,  X = floor(log2(max_k |x[m,k]|)) - 2 over the k of block b, cut to -127 .. 127
    q[m,k]     = the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives to x[m,k] / scale[m,b], ties to the even code
    y[m,n]     = act(sum_b scale[m,b] w_scale[n,b] sum_(k in b) q[m,k] w[n,k] + bias[n])

Two values are a byte, the first of them in its low half; a row is a whole number of blocks of 16 bytes, zeros behind its end.  Scales
are bytes X + 127 that lie in slabs of 8 blocks: [slab][row][8], zeros behind the last block.

Rows of a residual stream are normalised and quantised where they are added (`add_rms_norm_i8`); layers in 8-bit integers read them
(`matmul_i8`):

    s[m,k] = x[m,k] + r[m,k]     h[m,k] = s[m,k] / sqrt(mean_k s[m,k]^2 + eps) * weight[k]
    scale[m] = max_k |h[m,k]| / 127                  q[m,k] = nearest whole number, ties to even, of h[m,k] / scale[m]

What pruning and few bits lose is trained back from the largest logits that the unpruned network, the teacher, has for each row
(`distill_loss` and its gradient for autograd, `distill_loss_grad` for both at once), at temperature T:

    p[r,j] = softmax_j(teacher[r,j] / T) over the entries of row r       c[r,j] = the class of entry j; below 0: no entry
    lq[r,v] = student[r,v] / T - log sum_u exp(student[r,u] / T)
    loss = T^2 / rows * sum_r sum_j p[r,j] (log p[r,j] - lq[r,c[r,j]])
    grad[r,v] = T / rows * (exp(lq[r,v]) - sum_(j: c[r,j] = v) p[r,j]),   zeros in rows without an entry
"""
import math

import torch

own = False

_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_EL = {"f32": 4, "bf16": 2}


# ---- cases -----------------------------------------------------------------------------------------------------------

def _linear(name, m, k, n, dtype, relu=False, bias=True, pad=0):
    """One layer in 4 bits; `pad`: the rows of activations are that much further apart than they are long."""
    return dict(name=name, kind="linear", m=m, k=k, n=n, dtype=dtype, relu=relu, bias=bias, pad=pad)


def _shared(name, m, k, n, n2, dtype, relu=False, bias=True, pad=0):
    """Two layers in 4 bits that read the same activations."""
    return dict(name=name, kind="shared", m=m, k=k, n=n, n2=n2, dtype=dtype, relu=relu, bias=bias, pad=pad)


def _norm(name, m, k, n, dtype, residual=True, eps=1e-6, pad=0):
    """The norm, and the layer in 8-bit integers that reads it and gives bf16."""
    return dict(name=name, kind="norm", m=m, k=k, n=n, dtype=dtype, residual=residual, eps=eps, pad=pad)


def _distill(name, rows, classes, top, dtype, autograd, temperature=2.0, teacher="f32", ragged=False, pad=0):
    """`ragged`: rows have 0 .. `top` entries, not all of them `top`."""
    return dict(name=name, kind="distill", rows=rows, classes=classes, top=top, dtype=dtype, autograd=autograd,
                temperature=temperature, teacher=teacher, ragged=ragged, pad=pad)


def listed():
    return [
        # the smallest call: the classifier of a residual network for one image; launch and host time are all of it
        _linear("mx4_bf16_1x2048_1000", 1, 2048, 1000, "bf16"),
        # the first fully connected layer of VGG-16 for single images: reading the weights is all of it
        _linear("mx4_f32_1x25088_4096", 1, 25088, 4096, "f32", relu=True),
        # the same with the batch that the benchmark has
        _linear("mx4_bf16_32x25088_4096", 32, 25088, 4096, "bf16", relu=True),
        # a wide layer over many rows, the largest: the matrix units are all of it
        _linear("mx4_bf16_8192x4096_4096", 8192, 4096, 4096, "bf16"),
        # sizes that are multiples of nothing, rows that lie apart and start anywhere, no bias
        _shared("mx4_f32_odd", 777, 1155, 1001, 130, "f32", bias=False, pad=3),
        # one row of a residual stream and the layer behind it: latency
        _norm("norm_bf16_1x2048_512", 1, 2048, 512, "bf16"),
        # the pixels of ResNet-50's first stage, batch 32, channels last, and the narrow layer that reads them
        _norm("norm_bf16_100352x256_64", 100352, 256, 64, "bf16"),
        # long rows that are multiples of nothing and lie apart, fp32, nothing added
        _norm("norm_f32_odd", 2111, 4099, 129, "f32", residual=False, pad=5),
        # a batch of images with 1000 classes, 16 of them from the teacher: latency
        _distill("distill_f32_32x1000_16", 32, 1000, 16, "f32", False),
        # many rows and classes, loss and gradient at once
        _distill("distill_bf16_4096x32768_64", 4096, 32768, 64, "bf16", False),
        # the same step through autograd, lists of unequal length, odd sizes
        _distill("distill_f32_odd", 1999, 10007, 50, "f32", True, ragged=True, pad=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["mx4", "mx4", "norm", "distill", "distill"])
    while True:
        pad = rng.choice([0, 0, 0, 16, 3])
        if kind == "mx4":
            m, k, n = _log_int(rng, 1, 20000), _log_int(rng, 32, 25088), _log_int(rng, 8, 4096)
            if rng.random() < 0.3:
                m = _log_int(rng, 1, 32)             # serving: a few images
            if rng.random() < 0.6:                   # most layers have round channel counts
                k, n = k // 32 * 32, max(8, n // 8 * 8)
            args = dict(dtype=rng.choice(["f32", "bf16"]), relu=rng.random() < 0.5, bias=rng.random() < 0.8, pad=pad)
            c = _linear("", m, k, n, **args) if rng.random() < 0.7 else _shared("", m, k, n, _log_int(rng, 8, 2048), **args)
            fits = work(c)["flops"] < 2.7e11 and m * k < 1.2e8 and k * n < 1.1e8 and m * n < 5e7
        elif kind == "norm":
            m, k, n = _log_int(rng, 1, 100352), _log_int(rng, 64, 8192), _log_int(rng, 16, 512)
            if rng.random() < 0.6:
                k, n = max(64, k // 16 * 16), max(16, n // 8 * 8)
            c = _norm("", m, k, n, rng.choice(["f32", "bf16"]), residual=rng.random() < 0.8, eps=rng.choice([1e-5, 1e-6]), pad=pad)
            fits = m * k < 4e7
        else:
            rows, classes = _log_int(rng, 1, 8192), _log_int(rng, 10, 50000)
            if rng.random() < 0.5:
                classes = max(16, classes // 8 * 8)
            c = _distill("", rows, classes, min(classes, _log_int(rng, 1, 128)), rng.choice(["f32", "bf16"]), rng.random() < 0.5,
                         temperature=rng.choice([1.0, 2.0, 4.0]), teacher=rng.choice(["f32", "bf16"]), ragged=rng.random() < 0.4, pad=pad)
            fits = rows * classes < 1.3e8
        if fits:
            del c["name"]
            return c


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _apart(x, pad):
    """The same rows, `pad` elements further apart."""
    if not pad:
        return x
    wide = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _activations(m, k, gen):
    """Values after a ReLU, the channels of different sizes."""
    x = torch.empty(m, k, device="cuda").normal_(generator=gen)
    return x.clamp_(min=0).mul_(torch.empty(k, device="cuda").uniform_(0.25, 2.0, generator=gen))


def _layer4(k, n, bias, gen):
    """Weights in 4 bits as a layer keeps them: codes 0 .. 15 of random sign and size, scales about 1 / sqrt(k)."""
    blocks = -(-k // 32)
    q = torch.randint(0, 256, (n, blocks * 16), generator=gen, device="cuda", dtype=torch.uint8)
    if k % 32:
        q[:, (k + 1) // 2:] = 0
        if k % 2:
            q[:, k // 2] &= 15
    base = 127 - int(round(math.log2(3.0 * math.sqrt(k))))
    scale = torch.zeros(-(-blocks // 8), n, 8, dtype=torch.uint8, device="cuda")
    for s in range(scale.shape[0]):
        have = min(8, blocks - 8 * s)
        scale[s, :, :have] = torch.randint(base - 2, base + 2, (n, have), generator=gen, device="cuda", dtype=torch.uint8)
    return dict(w=q, scale=scale, bias=torch.empty(n, device="cuda").normal_(generator=gen) if bias else None)


def _layer8(k, n, gen):
    """Weights in 8-bit integers with the scales of their rows, and a bias."""
    w = torch.empty(n, k, device="cuda").normal_(generator=gen)
    scale = w.abs().amax(1) / 127
    wide = torch.zeros(n, (k + 15) // 16 * 16, dtype=torch.int8, device="cuda")
    wide[:, :k] = (w / scale[:, None]).round().clamp(-127, 127).to(torch.int8)
    return dict(w=wide[:, :k], scale=scale / math.sqrt(k), bias=torch.empty(n, device="cuda").normal_(generator=gen))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = _TYPE[case["dtype"]]
    if case["kind"] in ("linear", "shared"):
        x = _apart(_activations(case["m"], case["k"], gen).to(dtype), case["pad"])
        wide = [case["n"]] if case["kind"] == "linear" else [case["n"], case["n2"]]
        return dict(case=case, x=x, layers=[_layer4(case["k"], n, case["bias"], gen) for n in wide])
    if case["kind"] == "norm":
        # rows of different sizes, as a residual stream has
        m, k = case["m"], case["k"]
        size = torch.empty(m, 1, device="cuda").uniform_(0.5, 4.0, generator=gen)
        x = _apart(_activations(m, k, gen).sub_(0.4).mul_(size).to(dtype), case["pad"])
        residual = _apart(torch.empty(m, k, device="cuda").normal_(generator=gen).mul_(size).to(dtype), case["pad"]) if case["residual"] else None
        weight = torch.empty(k, device="cuda").uniform_(0.5, 1.5, generator=gen)
        return dict(case=case, x=x, residual=residual, weight=weight, layer=_layer8(k, case["n"], gen))
    rows, classes, top = case["rows"], case["classes"], case["top"]
    z = torch.empty(rows, classes, device="cuda").normal_(generator=gen).mul_(2.0)
    # the teacher's logits are near the student's; its largest ones
    t, c = torch.empty(rows, classes, device="cuda").normal_(generator=gen).add_(z).topk(top, 1)
    if case["ragged"]:
        have = torch.randint(0, top + 1, (rows, 1), generator=gen, device="cuda")
        c = torch.where(torch.arange(top, device="cuda")[None] < have, c, torch.full_like(c, -1))
    z = _apart(z.to(dtype), case["pad"])
    return dict(case=case, student=z.requires_grad_() if case["autograd"] else z, teacher=t.to(_TYPE[case["teacher"]]), classes=c)


# ---- one pass --------------------------------------------------------------------------------------------------------

def _plain_mx4(x):
    """Rows as the values that their 4 bits and scales stand for, [m, blocks * 32]; in 64 bits next to the borders."""
    m, k = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -k % 32)).view(m, -1, 32)
    most = x.abs().amax(2, keepdim=True)
    power = torch.where(most > 0, (torch.frexp(most)[1] - 3).clamp(-127, 127), torch.full_like(most, -127, dtype=torch.int32))
    up = torch.ldexp(torch.ones_like(most, dtype=torch.float64), power)
    v = (x.double() / up).float()                        # (exact)
    step = torch.where(v.abs() < 2, 0.5, torch.where(v.abs() < 4, 1.0, 2.0))
    v = ((v / step).round() * step).clamp(-6, 6)
    return (v * up).float().view(m, -1)


def _plain_layer4(layer):
    """The weights as values, [n, blocks * 32]."""
    q = layer["w"]
    n, blocks = q.shape[0], q.shape[1] // 16
    size = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=q.device)
    size = torch.cat([size, -size])
    v = torch.stack([size[(q & 15).int()], size[(q >> 4).int()]], 2).view(n, blocks, 32)
    power = layer["scale"].permute(1, 0, 2).reshape(n, -1)[:, :blocks].int() - 127
    return (v * torch.ldexp(torch.ones_like(power, dtype=torch.float32), power)[:, :, None]).view(n, -1)


def _plain_distill(state):
    case = state["case"]
    T, z, c = case["temperature"], state["student"].detach().float(), state["classes"]
    rows = z.shape[0]
    have = c >= 0
    t = torch.where(have, state["teacher"].float() / T, torch.full_like(c, -math.inf, dtype=torch.float32))
    some = have.any(1, keepdim=True)
    e = (t - torch.where(some, t.amax(1, keepdim=True), torch.zeros_like(t[:, :1]))).exp()
    p = torch.where(some, e / e.sum(1, keepdim=True), torch.zeros_like(e))
    z = z / T
    most = z.amax(1, keepdim=True)
    lse = most + (z - most).exp().sum(1, keepdim=True).log()
    at = c.clamp(min=0)
    each = torch.where(p > 0, p * (p.clamp(min=1e-45).log() - (z.gather(1, at) - lse)), torch.zeros_like(p))
    loss = each.double().sum().float() * (T * T / rows)
    grad = torch.where(some, (z - lse).exp(), torch.zeros_like(z)).scatter_add_(1, at, -p) * (T / rows)
    return {"loss": loss, "grad": grad.to(state["student"].dtype)}


def _plain(state):
    case = state["case"]
    if case["kind"] == "distill":
        return _plain_distill(state)
    if case["kind"] == "norm":
        s = state["x"].float() if state["residual"] is None else state["x"].float() + state["residual"].float()
        h = s.double()                                   # (a whole number next to a border)
        h = h * (h.square().mean(1, keepdim=True) + case["eps"]).rsqrt() * state["weight"].double()
        scale = (h.abs().amax(1, keepdim=True) / 127).float()
        q = torch.where(scale > 0, (h / scale.double()).round().clamp(-127, 127), torch.zeros_like(h)).float()
        ly = state["layer"]
        y = q @ ly["w"].float().t() * (scale * ly["scale"]) + ly["bias"]
        return [y.bfloat16()] + ([s.to(state["x"].dtype)] if state["residual"] is not None else [])
    x, got = _plain_mx4(state["x"]), []
    for ly in state["layers"]:
        y = x @ _plain_layer4(ly).t()
        y = y + ly["bias"] if ly["bias"] is not None else y
        got.append((y.clamp(min=0) if case["relu"] else y).to(state["x"].dtype))
    return got


def run(state):
    if not own:
        return _plain(state)
    import paper_1909_05073_amd as P
    case = state["case"]
    if case["kind"] == "distill":
        z, t, c, T = state["student"], state["teacher"], state["classes"], case["temperature"]
        if case["autograd"]:
            loss = P.distill_loss(z, t, c, T)
            return {"loss": loss.detach(), "grad": torch.autograd.grad(loss, z)[0]}
        loss, grad = P.distill_loss_grad(z, t, c, T)
        return {"loss": loss, "grad": grad}
    if case["kind"] == "norm":
        ly = state["layer"]
        q, scale, s = P.add_rms_norm_i8(state["x"], state["residual"], state["weight"], case["eps"])
        y = P.matmul_i8(q, scale, ly["w"], ly["scale"], ly["bias"], out_dtype=torch.bfloat16)
        return [y] + ([s] if state["residual"] is not None else [])
    x, layers, relu = state["x"], state["layers"], case["relu"]
    if case["kind"] == "linear":
        ly = layers[0]
        return [P.linear_mx4(x, ly["w"], ly["scale"], ly["bias"], relu=relu)]
    q, scale = P.quantize_mx4(x)
    return [P.matmul_mx4(q, scale, ly["w"], ly["scale"], ly["bias"], relu=relu, out_dtype=x.dtype) for ly in layers]


# ---- what a pass cannot do without, and what is exact ---------------------------------------------------------------

def work(case):
    el = _EL[case["dtype"]]
    if case["kind"] == "distill":
        r, v, j = case["rows"], case["classes"], case["top"]
        return {"bytes": float(2 * r * v * el + r * j * (8 + _EL[case["teacher"]]) + 4), "flops": 8.0 * r * v}
    m, k = case["m"], case["k"]
    if case["kind"] == "norm":
        n = case["n"]
        return {"bytes": float(m * k * el * (3 if case["residual"] else 1) + 4 * k + n * k + 8 * n + 2 * m * n), "flops": 2.0 * m * n * k + 8.0 * m * k}
    n = case["n"] + (case["n2"] if case["kind"] == "shared" else 0)
    blocks = -(-k // 32)
    return {"bytes": float(m * k * el + n * blocks * 17 + (4 * n if case["bias"] else 0) + m * n * el), "flops": 2.0 * m * n * k}


def _exact_mx4(x):
    m, k = x.shape
    wide = torch.zeros(m, -(-k // 32) * 32, dtype=torch.float64, device=x.device)
    wide[:, :k] = x
    wide = wide.view(m, -1, 32)
    most = wide.abs().max(2).values
    _, e = torch.frexp(most)                             # (most = f 2^e, f in [1/2, 1): its logarithm's floor is e - 1)
    up = torch.ldexp(torch.ones_like(most), (e - 3).clamp(-127, 127))[:, :, None]
    a = wide.abs() / up
    got = torch.zeros_like(a)
    # from each value to the next: beyond the middle, or on it where the next one's code is even
    for code, (low, high) in enumerate(zip((0, 0.5, 1, 1.5, 2, 3, 4), (0.5, 1, 1.5, 2, 3, 4, 6))):
        middle = (low + high) / 2
        got[(a >= middle) if code % 2 else (a > middle)] = high
    return (got * wide.sign() * up).view(m, -1)


def _exact_distill(case, s):
    T, c = case["temperature"], s["classes"]
    z, t = s["student"].detach().double() / T, s["teacher"].double() / T
    rows, loss = z.shape[0], 0.0
    grad = torch.zeros_like(z)
    for first in range(0, rows, 512):
        some = slice(first, min(rows, first + 512))
        lq = torch.log_softmax(z[some], 1)
        have = c[some] >= 0
        any_ = have.any(1)
        p = torch.softmax(t[some].masked_fill(~have, -1e300), 1) * have
        lp = torch.log(torch.where(p > 0, p, torch.ones_like(p)))
        at = c[some].clamp(min=0)
        loss += float((p * (lp - torch.gather(lq, 1, at)))[any_].sum())
        grad[some] = ((lq.exp()) * any_[:, None]).scatter_add(1, at, -p)
    return {"loss": torch.tensor(loss * T * T / rows, dtype=torch.float64), "grad": grad * (T / rows)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "distill":
        return _exact_distill(case, s)
    if case["kind"] == "norm":
        x = s["x"].double()
        if s["residual"] is not None:
            x = x + s["residual"].double()
        h = x / torch.sqrt((x * x).sum(1, keepdim=True) / x.shape[1] + case["eps"]) * s["weight"].double()
        scale = (h.abs().max(1).values / 127).float().double()[:, None]
        q = torch.round(h / torch.where(scale > 0, scale, torch.ones_like(scale)))
        ly = s["layer"]
        y = torch.matmul(q, ly["w"].double().t().contiguous()) * scale * ly["scale"].double() + ly["bias"].double()
        return [y] + ([x] if s["residual"] is not None else [])
    x, got = _exact_mx4(s["x"]), []
    for ly in s["layers"]:
        n, wide = ly["w"].shape
        w = torch.zeros(n, 2 * wide, dtype=torch.float64, device=x.device)
        for half in (0, 1):
            code = (ly["w"] >> (4 * half)) & 15
            e, f, sign = ((code >> 1) & 3).double(), (code & 1).double(), 1 - 2.0 * (code >> 3).double()
            w[:, half::2] = sign * torch.where(e > 0, torch.exp2(e - 1) * (1 + f / 2), f / 2)
        scale = ly["scale"].transpose(0, 1).reshape(n, -1)[:, :wide // 16].double()
        w = w.view(n, -1, 32) * torch.exp2(scale - 127)[:, :, None]
        y = torch.matmul(x, w.view(n, -1).t().contiguous())
        if ly["bias"] is not None:
            y = y + ly["bias"].double()
        got.append(torch.relu(y) if case["relu"] else y)
    return got
