"""The operators around a network's last product that this library is timed on: layer norm, and the losses over a large number of
classes whose logits are never held whole.

A case is a plain dict.  `call` says what a pass is:

  norm_forward      y = (x - mean) rstd weight + bias for every row, with mean and rstd that the gradient reads
  norm_backward     dx (plus the gradient of the skip connection beside the norm), dweight and dbias
  entropy_forward   for every row of x the cross entropy of softmax(x w^T + bias) and its label, and the log of the sum of exponentials
  entropy_backward  dx, dw and dbias of it
  distill_forward   the divergence of softmax(x w^T / temperature) from a teacher's distribution over its `top` largest logits
  distill_backward  dx and dw of it

`type` is the storage type of activations, weights, their gradients and the teacher's logits; statistics, losses, biases and the
gradients of vectors are fp32.
"""
import math

import torch

own = False  # True: the calls go to the library's kernels; False: the same in elementary torch operations

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-5
LOSS_SCALE = {"fp32": 1.0, "bf16": 1.0, "fp16": 4096.0}  # what a training step in that type multiplies the loss by


def _norm(name, call, rows, cols, dtype):
    c = {"call": call, "rows": rows, "cols": cols, "type": dtype}
    return {"name": name, **c} if name else c


def _entropy(name, call, rows, features, classes, dtype, bias=False, smoothing=0.0, z_loss=0.0):
    c = {"call": call, "rows": rows, "features": features, "classes": classes, "type": dtype, "bias": bias, "smoothing": smoothing, "z_loss": z_loss}
    return {"name": name, **c} if name else c


def _distill(name, call, rows, features, classes, top, temperature, dtype):
    c = {"call": call, "rows": rows, "features": features, "classes": classes, "top": top, "temperature": temperature, "type": dtype}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one sample of a wide layer, as a server has it: latency
        _norm("norm_forward_1_row_bf16", "norm_forward", 1, 4096, "bf16"),
        # the norm in front of a feed-forward block in training
        _norm("norm_forward_16384_bf16", "norm_forward", 16384, 4096, "bf16"),
        # its gradient
        _norm("norm_backward_16384_bf16", "norm_backward", 16384, 4096, "bf16"),
        # odd sizes in fp32
        _norm("norm_backward_odd_fp32", "norm_backward", 5003, 1777, "fp32"),
        # the likelihood of a few answers under a large vocabulary: the weights are read once
        _entropy("entropy_forward_16_bf16", "entropy_forward", 16, 2048, 65536, "bf16"),
        # a training step's loss over a large vocabulary, the log of the sum kept near zero
        _entropy("entropy_forward_8192_bf16", "entropy_forward", 8192, 4096, 128000, "bf16", z_loss=1e-4),
        # its gradient: the largest case
        _entropy("entropy_backward_8192_bf16", "entropy_backward", 8192, 4096, 128000, "bf16", z_loss=1e-4),
        # the 100-class head of the bottleneck networks on a batch of the 152-layer one, labels smoothed
        _entropy("entropy_backward_head_fp16", "entropy_backward", 4096, 2048, 100, "fp16", bias=True, smoothing=0.1),
        # odd sizes in fp32
        _entropy("entropy_backward_odd_fp32", "entropy_backward", 999, 515, 32003, "fp32", bias=True),
        # a student's loss on a batch of answers whose teacher kept 64 logits of each token
        _distill("distill_forward_4096_bf16", "distill_forward", 4096, 2048, 65536, 64, 2.0, "bf16"),
        # its gradient
        _distill("distill_backward_4096_bf16", "distill_backward", 4096, 2048, 65536, 64, 2.0, "bf16"),
        # a 1000-class student of a small batch: latency
        _distill("distill_backward_small_fp16", "distill_backward", 128, 512, 1000, 10, 4.0, "fp16"),
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
    return v


def draw(rng):
    call = rng.choice(["norm_forward", "norm_backward", "entropy_forward", "entropy_backward", "distill_forward", "distill_backward"])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    if call.startswith("norm"):
        cols = _size(rng, 16, 16384)
        return _norm("", call, _size(rng, 1, max(2, min(65536, (1 << 26) // cols))), cols, dtype)
    features, classes = _size(rng, 32, 4096), _size(rng, 10, 131072)
    # (2e11: a twentieth of the largest listed product, a fortieth in fp32)
    most = int((1e11 if dtype == "fp32" else 2e11) / (features * classes))
    rows = _size(rng, 1, max(64, min(16384, most)))
    if rng.random() < 0.2:
        rows = rng.randint(1, 64)
    if call.startswith("entropy"):
        return _entropy("", call, rows, features, classes, dtype, rng.random() < 0.5, rng.choice([0.0, 0.0, 0.1]), rng.choice([0.0, 1e-4]))
    return _distill("", call, rows, features, classes, _log_uniform(rng, 1, min(256, classes)), rng.choice([1.0, 2.0, 4.0]), dtype)


def work(case):
    e, m = BYTES[case["type"]], case["rows"]
    if case["call"].startswith("norm"):
        c = case["cols"]
        if case["call"] == "norm_forward":
            return {"bytes": 2 * e * m * c + 8 * c + 8 * m, "flops": 8 * m * c}
        return {"bytes": 4 * e * m * c + 12 * c + 8 * m, "flops": 14 * m * c}
    k, n = case["features"], case["classes"]
    small = 4 * m * 3
    if case["call"].startswith("distill"):
        small += m * case["top"] * (4 + e)
    elif case["bias"]:
        small += 4 * n
    if case["call"].endswith("forward"):
        return {"bytes": e * (m * k + n * k) + small, "flops": 2 * m * k * n}
    # the logits, which are not kept, and the two gradients
    return {"bytes": 2 * e * (m * k + n * k) + small + (4 * n if case.get("bias") else 0), "flops": 6 * m * k * n}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, m, call = DTYPE[case["type"]], case["rows"], case["call"]
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=gen, device="cuda")  # noqa: E731
    s = {"case": case}
    if call.startswith("norm"):
        c = case["cols"]
        # activations of a residual stream: rows of their own scale and offset, a few columns much larger than the others
        x = randn(m, c) * (rand(m, 1) * 4 + 0.5) + randn(m, 1)
        x *= torch.where(rand(c) < 0.01, 8.0, 1.0)
        s["x"] = x.to(dt)
        s["weight"], s["bias"] = 1 + 0.2 * randn(c), 0.1 * randn(c)
        if call == "norm_backward":
            s["dy"], s["residual"] = (randn(m, c) * 0.02).to(dt), (randn(m, c) * 0.02).to(dt)
            wide = s["x"].double()
            mean = wide.mean(1)
            s["mean"], s["rstd"] = mean.float(), ((wide - mean[:, None]).square_().mean(1) + EPS).rsqrt().float()
        return s
    k, n = case["features"], case["classes"]
    s["x"] = randn(m, k).to(dt)  # as a norm leaves them
    s["w"] = (randn(n, k) * (2.0 * k ** -0.5)).to(dt)
    s["bias"] = 0.5 * randn(n) if case.get("bias") else None
    left_out = rand(m) < 0.05  # padding
    if call.startswith("entropy"):
        labels = torch.randint(0, n, (m,), generator=gen, device="cuda", dtype=torch.int32)
        s["labels"] = torch.where(left_out, torch.full_like(labels, -1), labels)
        scale = 1.0
    else:
        # distinct classes, one of each of `top` ranges, by falling teacher's logit; a teacher that kept fewer leaves the last ones unused
        top = case["top"]
        edge = torch.arange(top + 1, device="cuda") * n // top
        at = edge[:-1] + (rand(m, top) * (edge[1:] - edge[:-1])).long().clamp_max(edge[1:] - edge[:-1] - 1)
        order = rand(m, top).argsort(1)
        kept = torch.where(rand(m, 1) < 0.1, (rand(m, 1) * top).long(), torch.full((m, 1), top, device="cuda"))
        kept[left_out] = 0
        s["indices"] = torch.where(torch.arange(top, device="cuda") < kept, at.gather(1, order), torch.full_like(at, -1)).int()
        s["teacher"] = (10 + 3 * randn(m, top)).sort(1, descending=True).values.to(dt)
        scale = case["temperature"] ** 2
    if call.endswith("backward"):
        s["dloss"] = torch.full((m,), LOSS_SCALE[case["type"]] * scale / m, device="cuda")  # of the mean
        if call.startswith("distill"):
            s["dloss"] *= rand(m) + 0.5  # answers weigh differently
        # what the forward pass kept
        tau, kept_lse = case.get("temperature", 1.0), []
        wide = s["w"].float().T
        for rows in s["x"].split(2048):
            z = torch.mm(rows.float(), wide)
            if s["bias"] is not None:
                z += s["bias"]
            kept_lse.append(torch.logsumexp(z / tau, 1))
        s["lse"] = torch.cat(kept_lse)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _plain_norm(s, backward):
    x, dt, c = s["x"].float(), s["x"].dtype, s["x"].shape[1]
    if not backward:
        mean = x.sum(1) / c
        x = x - mean[:, None]
        rstd = 1 / (x.square().sum(1) / c + EPS).sqrt()
        return {"y": (x * rstd[:, None] * s["weight"] + s["bias"]).to(dt), "mean": mean, "rstd": rstd}
    h = (x - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    u = dy * s["weight"]
    dx = (u - u.sum(1, keepdim=True) / c - h * ((u * h).sum(1, keepdim=True) / c)) * s["rstd"][:, None] + s["residual"].float()
    return {"dx": dx.to(dt), "dweight": (dy * h).sum(0), "dbias": dy.sum(0)}


def _plain_logits(s):
    z = s["x"].float() @ s["w"].float().T
    if s["bias"] is not None:
        z = z + s["bias"]
    return z


def _plain_lse(z):
    top = z.max(1).values
    return top + (z - top[:, None]).exp().sum(1).log()


def _plain_gradients(s, d):
    dt = s["x"].dtype
    out = {"dx": (d @ s["w"].float()).to(dt), "dw": (d.T @ s["x"].float()).to(dt)}
    if s["bias"] is not None:
        out["dbias"] = d.sum(0)
    return out


def _plain_entropy(s, backward):
    case, z = s["case"], _plain_logits(s)
    n, labels = z.shape[1], s["labels"].long()
    used = labels >= 0
    at = labels.clamp_min(0)[:, None]
    if not backward:
        lse = _plain_lse(z)
        loss = lse - (1 - case["smoothing"]) * z.gather(1, at)[:, 0] + case["z_loss"] * lse * lse
        if case["smoothing"]:
            loss = loss - case["smoothing"] * (z.sum(1) / n)
        return {"loss": torch.where(used, loss, torch.zeros_like(loss)), "lse": lse}
    lse = s["lse"]
    d = (z - lse[:, None]).exp()
    if case["z_loss"]:
        d = d * (1 + 2 * case["z_loss"] * lse)[:, None]
    if case["smoothing"]:
        d = d - case["smoothing"] / n
    d.scatter_add_(1, at, torch.full(at.shape, case["smoothing"] - 1, device=d.device))
    return _plain_gradients(s, d * torch.where(used, s["dloss"], torch.zeros_like(s["dloss"]))[:, None])


def _plain_distill(s, backward):
    tau = s["case"]["temperature"]
    z = _plain_logits(s) / tau
    indices = s["indices"].long()
    used = indices >= 0
    some = used.any(1)
    t = torch.where(used, s["teacher"].float() / tau, torch.full(used.shape, -math.inf, device=z.device))
    top = torch.where(some, t.max(1).values, torch.zeros_like(t[:, 0]))
    e = (t - top[:, None]).exp()
    total = e.sum(1)
    q = torch.where(some[:, None], e / total[:, None], torch.zeros_like(e))
    if not backward:
        lse = _plain_lse(z)
        log_q = t - (top + total.log())[:, None]
        terms = q * (log_q - z.gather(1, indices.clamp_min(0)) + lse[:, None])
        return {"loss": torch.where(q > 0, terms, torch.zeros_like(q)).sum(1), "lse": lse}
    d = (z - s["lse"][:, None]).exp()
    d.scatter_add_(1, indices.clamp_min(0), -q)
    return _plain_gradients(s, d * torch.where(some, s["dloss"] / tau, torch.zeros_like(s["dloss"]))[:, None])


# ---- a pass ----------------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    call, backward = case["call"], case["call"].endswith("backward")
    if not own:
        return (_plain_norm if call.startswith("norm") else _plain_entropy if call.startswith("entropy") else _plain_distill)(s, backward)
    from paper_2105_00619_amd import binding as B
    if call == "norm_forward":
        y, mean, rstd = B.layer_norm_forward(s["x"], s["weight"], s["bias"], eps=EPS, save_stats=True)
        return {"y": y, "mean": mean, "rstd": rstd}
    if call == "norm_backward":
        dx, dweight, dbias = B.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"], residual=s["residual"])
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    if call == "entropy_forward":
        loss, lse = B.cross_entropy_forward(s["x"], s["w"], s["labels"], s["bias"], label_smoothing=case["smoothing"], z_loss=case["z_loss"])
        return {"loss": loss, "lse": lse}
    if call == "distill_forward":
        loss, lse = B.distillation_forward(s["x"], s["w"], s["indices"], s["teacher"], temperature=case["temperature"])
        return {"loss": loss, "lse": lse}
    if call == "entropy_backward":
        dx, dw, dbias = B.cross_entropy_backward(s["dloss"], s["x"], s["w"], s["labels"], s["lse"], s["bias"],
                                                 label_smoothing=case["smoothing"], z_loss=case["z_loss"])
    else:
        dx, dw, dbias = B.distillation_backward(s["dloss"], s["x"], s["w"], s["indices"], s["teacher"], s["lse"], temperature=case["temperature"])
    out = {"dx": dx, "dw": dw}
    if dbias is not None:
        out["dbias"] = dbias
    return out


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    call, x = case["call"], s["x"].double()
    if call == "norm_forward":
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        return {"y": torch.addcmul(s["bias"].double(), (x - mean[:, None]) * rstd[:, None], s["weight"].double()), "mean": mean, "rstd": rstd}
    if call == "norm_backward":
        h = (x - s["mean"].double()[:, None]) * s["rstd"].double()[:, None]
        dy = s["dy"].double()
        u = dy * s["weight"].double()
        dx = s["rstd"].double()[:, None] * (u - u.mean(1, keepdim=True) - h * (u * h).mean(1, keepdim=True))
        return {"dx": dx + s["residual"].double(), "dweight": torch.sum(dy * h, 0), "dbias": torch.sum(dy, 0)}
    w = s["w"].double()
    wt = w.T.contiguous()
    m, n = x.shape[0], w.shape[0]
    tau, entropy = case.get("temperature", 1.0), call.startswith("entropy")
    loss, lse = torch.zeros(m, dtype=torch.float64, device="cuda"), torch.zeros(m, dtype=torch.float64, device="cuda")
    dx, dw, dbias = torch.zeros_like(x), torch.zeros_like(w), torch.zeros(n, dtype=torch.float64, device="cuda")
    backward = call.endswith("backward")
    for a in range(0, m, 1024):
        r = slice(a, min(a + 1024, m))
        z = torch.mm(x[r], wt)
        if s["bias"] is not None:
            z += s["bias"].double()
        z /= tau
        # the target as rows of probabilities, zero for a row without one
        target = torch.zeros_like(z)
        entropy_of_target = torch.zeros(z.shape[0], dtype=torch.float64, device="cuda")
        if entropy:
            y = s["labels"][r].long()
            used = y >= 0
            rows = used.nonzero()[:, 0]
            target[rows] = case["smoothing"] / n
            target[rows, y[rows]] += 1 - case["smoothing"]
        else:
            i = s["indices"][r].long()
            t = (s["teacher"][r].double() / tau).masked_fill(i < 0, -math.inf)
            used = (i >= 0).any(1)
            log_q = torch.log_softmax(t, 1)
            q = log_q.exp().masked_fill(i < 0, 0.0)
            target.scatter_add_(1, i.clamp_min(0), q)
            entropy_of_target = torch.where(q > 0, q * log_q, torch.zeros_like(q)).sum(1)
        zc = case.get("z_loss", 0.0)
        if not backward:
            lse[r] = torch.logsumexp(z, 1)
            loss[r] = torch.where(used, entropy_of_target - (target * z).sum(1) + lse[r] + zc * lse[r] ** 2, 0.0)
            continue
        kept = s["lse"][r].double()
        d = torch.exp_(z.sub_(kept[:, None])).mul_((1 + 2 * zc * kept)[:, None]).sub_(target)
        d *= torch.where(used, s["dloss"][r].double() / tau, 0.0)[:, None]
        dx[r] = torch.mm(d, w)
        dw.addmm_(d.T.contiguous(), x[r])
        dbias += d.sum(0)
    if not backward:
        return {"loss": loss, "lse": lse}
    return {"dx": dx, "dw": dw, "dbias": dbias} if s["bias"] is not None else {"dx": dx, "dw": dw}
