"""The matrix operators this library is timed on: linear layers with their gradients, and the orthogonalised update.

A case is a plain dict.  `call` says what a pass is:

  forward   y = act(x w^T + bias) + residual and the pre-activation z that the gradient reads
  backward  its gradients: dx, dw and dbias from dy, x, w and z
  orth      every matrix of a list replaced by p(p(...p(G / |G|))), p(X) = a X + (b X X^T + c (X X^T)^2) X: five
            Newton-Schulz steps towards the orthogonal factor of G
  muon      the update of a list of weight matrices with it: momentum, the step above, weights and their 16-bit copy

`type` is the storage type of activations, weights and gradients.  `shapes` lists matrices, "RxC" or "RxC*N" for N of them
in a row, separated by blanks; they lie one behind the other in a flat vector, as the parameters of a network do here.  A
convolution's weight (C_out, kh, kw, C_in) is the C_out x (kh kw C_in) matrix.
"""
import math

import torch

own = False  # True: the calls go to the library's kernels; False: the same in elementary torch operations

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01


def _basic(stages):
    """Weight matrices of a residual network of basic blocks on 32 x 32 images, its 100-class head last."""
    out, c = ["64x27"], 64
    for i, n in enumerate(stages):
        w = 64 << i
        for b in range(n):
            out += ["%dx%d" % (w, 9 * c), "%dx%d" % (w, 9 * w)] + (["%dx%d" % (w, c)] if c != w else [])
            c = w
    return " ".join(out + ["100x%d" % c])


def _bottleneck(stages):
    out, c = ["64x27"], 64
    for i, n in enumerate(stages):
        w = 64 << i
        for b in range(n):
            out += ["%dx%d" % (w, c), "%dx%d" % (w, 9 * w), "%dx%d" % (4 * w, w)] + (["%dx%d" % (4 * w, c)] if c != 4 * w else [])
            c = 4 * w
    return " ".join(out + ["100x%d" % c])


def _linear(name, call, rows, cin, cout, act, dtype, residual=False):
    c = {"call": call, "rows": rows, "cin": cin, "cout": cout, "act": act, "type": dtype, "residual": residual}
    return {"name": name, **c} if name else c


def _list(name, call, shapes, dtype):
    c = {"call": call, "shapes": shapes, "type": dtype}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one sample through a wide layer, as a server does it: the weights are read once
        _linear("forward_1_row_bf16", "forward", 1, 4096, 16384, "gelu", "bf16"),
        # the classifier of the bottleneck networks on the batch of the paper's experiments: latency
        _linear("forward_head_16_fp16", "forward", 16, 2048, 100, "none", "fp16"),
        # the first half of a feed-forward block in training, at the batch of the 152-layer network times two
        _linear("forward_8192_bf16", "forward", 8192, 2048, 8192, "gelu", "bf16"),
        # odd sizes and a skip connection in fp32
        _linear("forward_odd_fp32", "forward", 1999, 1023, 1777, "relu", "fp32", True),
        # the gradients of the feed-forward layer
        _linear("backward_8192_bf16", "backward", 8192, 2048, 8192, "gelu", "bf16"),
        # a narrow layer of odd sizes with a long batch
        _linear("backward_odd_fp16", "backward", 20011, 333, 514, "silu", "fp16"),
        # the head alone, orthogonalised: latency
        _list("orth_head_fp32", "orth", "100x512", "fp32"),
        # a square matrix
        _list("orth_2048_fp32", "orth", "2048x2048", "fp32"),
        # the two matrices of a wide feed-forward block, one wide and one tall
        _list("orth_ffn_bf16", "orth", "4096x16384 16384x4096", "bf16"),
        # the smallest network that is trained here (two 3x3 layers of 8 channels, 10 classes)
        _list("muon_tiny_fp32", "muon", "8x27 8x72 10x8", "fp32"),
        # ResNet-18, gradients in fp32 as a training step gives them
        _list("muon_resnet18_fp32", "muon", _basic([2, 2, 2, 2]), "fp32"),
        # ResNet-152, every matrix, gradients in bf16
        _list("muon_resnet152_bf16", "muon", _bottleneck([3, 8, 36, 3]), "bf16"),
    ]


# ---- drawn cases -----------------------------------------------------------------------------------------------------

def _log_uniform(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def _size(rng, lo, hi):
    """Half of the sizes are multiples of 64 (or of 8 where they are small), the others any number."""
    v = _log_uniform(rng, lo, hi)
    if rng.random() < 0.5:
        step = 64 if v >= 128 else 8
        v = max(step, v // step * step)
    return v + 1 if v == 3072 else v


def draw(rng):
    call = rng.choice(["forward", "backward", "orth", "muon"])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    if call in ("forward", "backward"):
        cin, cout = _size(rng, 24, 8192), _size(rng, 10, 8192)
        most = min(20000, int(1e11 / (cin * cout)))
        rows = _size(rng, 1 if call == "forward" else 16, max(64, most))
        if call == "forward" and rng.random() < 0.3:
            rows = rng.randint(1, 64)
        return _linear("", call, rows, cin, cout, rng.choice(["none", "relu", "gelu", "silu"]), dtype,
                       call == "forward" and rng.random() < 0.5)
    if rng.random() < 0.4:  # one matrix
        m = _size(rng, 8, 4096)
        n = _size(rng, m, max(m + 8, min(16384, 8 * m)))
        return _list("", call, "%dx%d" % ((m, n) if rng.random() < 0.5 else (n, m)), dtype)
    # the convolutions of a network: a few widths, each with 3x3 and 1x1 layers
    base, first = rng.choice([16, 24, 32, 48, 64, 80]), rng.randint(1, 3)
    shapes, c = ["%dx27" % base], base
    for i in range(rng.randint(1, 4)):
        w = base << i
        shapes.append("%dx%d" % (w, 9 * c))
        shapes.append("%dx%d*%d" % (w, 9 * w, first + rng.randint(0, 3)))
        if rng.random() < 0.5:
            shapes += ["%dx%d" % (w, 4 * w), "%dx%d" % (4 * w, w)]
        c = w
    return _list("", call, " ".join(shapes + ["%dx%d" % (rng.choice([10, 100, 1000]), c)]), dtype)


def _parse(case):
    out = []
    for t in case["shapes"].split():
        t, _, n = t.partition("*")
        r, _, c = t.partition("x")
        out += [(int(r), int(c))] * int(n or 1)
    return out


def work(case):
    e = BYTES[case["type"]]
    if case["call"] in ("forward", "backward"):
        m, k, n = case["rows"], case["cin"], case["cout"]
        if case["call"] == "forward":
            return {"bytes": e * (m * k + n * k + m * n * (3 if case["residual"] else 2)) + 4 * n, "flops": 2 * m * k * n}
        return {"bytes": e * (m * n * (1 if case["act"] == "none" else 2) + 2 * m * k + 2 * n * k) + 4 * n, "flops": 4 * m * k * n}
    size = flops = 0
    for r, c in _parse(case):
        m, n = min(r, c), max(r, c)
        size += m * n
        # symmetric products cost half: X X^T, A^2 and p(A) X each step, or all steps on A and one product with X at the end
        flops += min(STEPS * (3 * m * m * n + m ** 3), 3 * m * m * n + (4 * STEPS - 3) * m ** 3)
    if case["call"] == "orth":
        return {"bytes": 2 * e * size, "flops": flops}
    return {"bytes": (e + 16 + (2 if e == 2 else 0)) * size, "flops": flops}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _matrix_like_a_gradient(r, c, gen, out):
    """A few directions that all samples share, and the samples' own: the gradients of a batch look like this."""
    k = max(1, min(r, c) // 16)
    u = torch.randn(r, k, generator=gen, device="cuda")
    v = torch.randn(k, c, generator=gen, device="cuda")
    noise = torch.randn(r, c, generator=gen, device="cuda")
    scale = torch.rand(r, 1, generator=gen, device="cuda") + 0.5  # rows of different strength
    out.copy_((torch.mm(u, v).mul_(k ** -0.5).add_(noise)).mul_(scale).mul_(1e-3))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPE[case["type"]]
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    if case["call"] in ("forward", "backward"):
        m, k, n = case["rows"], case["cin"], case["cout"]
        s = {"case": case, "act": case["act"]}
        s["x"] = randn(m, k).to(dt)
        s["w"] = (randn(n, k) * k ** -0.5).to(dt)
        if case["call"] == "forward":
            s["bias"] = randn(n) * 0.1
            s["residual"] = randn(m, n).to(dt) if case["residual"] else None
        else:
            s["z"] = randn(m, n).to(dt) if case["act"] != "none" else None
            s["dy"] = (randn(m, n) * 0.02).to(dt)
        return s
    shapes = _parse(case)
    total = sum(r * c for r, c in shapes)
    g = torch.empty(total, dtype=dt, device="cuda")
    at, by_shape = 0, {}  # where the matrices of each shape begin: the plain form takes those of one shape together
    for r, c in shapes:
        by_shape.setdefault((r, c), []).append(at)
        _matrix_like_a_gradient(r, c, gen, g[at:at + r * c].view(r, c))
        at += r * c
    s = {"case": case, "shapes": shapes, "by_shape": by_shape, "g": g}
    if case["call"] == "muon":
        s["w"] = torch.cat([(randn(r * c) * c ** -0.5) for r, c in shapes])
        s["v"] = randn(total) * 1e-3
        s["w16"] = s["w"].to(dt) if dt != torch.float32 else None
    else:
        s["out"] = torch.empty_like(g)
    if own:
        from paper_2105_00619_amd import binding as B
        s["plan"] = B.Orthogonalizer(shapes, steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _act(name, z):
    if name == "relu":
        return z.clamp_min(0)
    if name == "gelu":
        return z * 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


def _orthogonal(g):
    """Newton-Schulz steps on a stack of fp32 matrices of one shape."""
    x = g if g.shape[1] <= g.shape[2] else g.mT
    x = x * (1 / x.double().square().sum((1, 2), keepdim=True).sqrt().clamp_min(EPS)).float()
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    return x if g.shape[1] <= g.shape[2] else x.mT


def _at(flat, r, c, offsets):
    return [flat[o:o + r * c].view(r, c) for o in offsets]


def _plain(s):
    case = s["case"]
    if case["call"] == "forward":
        z = s["x"].float() @ s["w"].float().T + s["bias"]
        y = _act(s["act"], z)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(s["x"].dtype), "z": z.to(s["x"].dtype)}
    if case["call"] == "backward":
        dt = s["x"].dtype
        d = s["dy"].float()
        if s["z"] is not None:
            d = d * _act_slope(s["act"], s["z"].float())
        return {"dx": (d @ s["w"].float()).to(dt), "dw": (d.T @ s["x"].float()).to(dt), "dbias": d.sum(0)}
    if case["call"] == "orth":
        for (r, c), offsets in s["by_shape"].items():
            o = _orthogonal(torch.stack(_at(s["g"], r, c, offsets)).float())
            torch._foreach_copy_(_at(s["out"], r, c, offsets), list(o.unbind()))
        return s["out"]
    g = s["g"].float()
    s["v"].mul_(MOMENTUM).add_(g)
    u = g + MOMENTUM * s["v"]
    s["w"].mul_(1 - LR * DECAY)
    for (r, c), offsets in s["by_shape"].items():
        o = _orthogonal(torch.stack(_at(u, r, c, offsets)))
        torch._foreach_add_(_at(s["w"], r, c, offsets), list(o.unbind()), alpha=-LR * math.sqrt(max(1.0, r / c)))
    if s["w16"] is not None:
        s["w16"].copy_(s["w"])
    return {"w": s["w"], "v": s["v"], "w16": s["w16"]}


# ---- a pass ----------------------------------------------------------------------------------------------------------

def run(s):
    if not own:
        return _plain(s)
    from paper_2105_00619_amd import binding as B
    call = s["case"]["call"]
    if call == "forward":
        y, z = B.linear_forward(s["x"], s["w"], s["bias"], residual=s["residual"], activation=s["act"], save_pre=True)
        return {"y": y, "z": z}
    if call == "backward":
        dx, dw, dbias = B.linear_backward(s["dy"], s["x"], s["w"], s["z"], activation=s["act"])
        return {"dx": dx, "dw": dw, "dbias": dbias}
    if call == "orth":
        return s["plan"].orthogonalize(s["g"], s["out"])
    s["plan"].muon_update(s["w"], s["v"], s["g"], lr=LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY,
                          scale="aspect", weights16=s["w16"])
    return {"w": s["w"], "v": s["v"], "w16": s["w16"]}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _factor64(g):
    g = g.double()
    x = g / max(float(torch.linalg.vector_norm(g)), EPS)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        if x.shape[0] <= x.shape[1]:
            s = torch.mm(x, x.T.contiguous())
            p = torch.addmm(s, s, s, beta=b, alpha=c)
            x = torch.addmm(x, p, x, beta=a)
        else:
            s = torch.mm(x.T.contiguous(), x)
            p = torch.addmm(s, s, s, beta=b, alpha=c)
            x = torch.addmm(x, x, p, beta=a)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["call"] == "forward":
        z = torch.addmm(s["bias"].double(), s["x"].double(), s["w"].double().T.contiguous())
        y = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t / (1 + torch.exp(-t)),
             "gelu": lambda t: 0.5 * t * torch.special.erfc(-t / math.sqrt(2))}[case["act"]](z)
        return {"y": y if s["residual"] is None else y + s["residual"].double(), "z": z}
    if case["call"] == "backward":
        d = s["dy"].double()
        if case["act"] != "none":
            t = s["z"].double()
            if case["act"] == "relu":
                d = torch.where(t > 0, d, torch.zeros_like(d))
            elif case["act"] == "silu":
                e = torch.exp(-t)
                d = d * ((1 + e + t * e) / (1 + e) ** 2)
            else:
                d = d * (0.5 * torch.special.erfc(-t / math.sqrt(2)) + t * torch.exp(-t * t / 2) / math.sqrt(2 * math.pi))
        return {"dx": torch.mm(d, s["w"].double()), "dw": torch.mm(d.T.contiguous(), s["x"].double()), "dbias": d.sum(0)}
    parts, at = [], 0
    g = s["g"].double()
    if case["call"] == "muon":
        v = MOMENTUM * s["v"].double() + g
        w = s["w"].double()
        g = g + MOMENTUM * v
    for r, c in s["shapes"]:
        o = _factor64(g[at:at + r * c].view(r, c)).reshape(-1)
        if case["call"] == "muon":
            o = (1 - LR * DECAY) * w[at:at + r * c] - LR * math.sqrt(max(1.0, r / c)) * o
        parts.append(o)
        at += r * c
    out = torch.cat(parts)
    if case["call"] == "orth":
        return out
    return {"w": out, "v": v, "w16": out if s["w16"] is not None else None}
