"""The operators of a training step that stand around the network, as cases that can be timed and compared.

  classes      softmax cross-entropy of a linear classifier over many classes, from features and class weights, without the
               logits being handed out: `train` is the loss with the gradients of features, weights and bias, `eval` the loss
               alone.  Rows labelled -1 are left out.
  orthogonal   the nearest orthogonal matrices of several matrices by five Newton-Schulz products (odd polynomial of degree five)
  update       one parameter update of a whole network by that rule: momentum, orthogonalised step of every filter, the small
               tensors and the head by plain momentum

Every case is one pass over data that is in device memory already.  The plain forms compute in 32 bits and round once.
"""
import math

import torch

own = False

COEFS = (3.4445, -4.7750, 2.0315)
STEPS = 5
LR, REST_LR, MOMENTUM, WEIGHT_DECAY = 0.02, 0.01, 0.95, 0.01

#: most work of one pass: rows * classes * channels of the classifier, multiplications of the orthogonalisation
MOST_CLASSES = 8192 * 32768 * 2048
MOST_ORTHOGONAL = 2 * STEPS * (4 * 2048 ** 2 * 4096 + 2 * 2048 ** 3)


def _classes(name, what, rows, channels, classes, dtype, bias=True, ignored=0.0):
    return {"name": name, "operator": "classes", "pass": what, "rows": rows, "channels": channels, "classes": classes,
            "dtype": dtype, "bias": bias, "ignored": ignored}


def _orthogonal(name, count, rows, cols, dtype):
    return {"name": name, "operator": "orthogonal", "count": count, "rows": rows, "cols": cols, "dtype": dtype}


def _update(name, net, dtype, master, nesterov):
    return {"name": name, "operator": "update", "net": net, "dtype": dtype, "master": master, "nesterov": nesterov}


def listed():
    return [
        # the smallest call anybody makes: a classifier on every position of a module of the test network (4 x 8 x 8 positions)
        _classes("positions_tiny_f32", "train", 256, 16, 10, "f32"),
        # the head of the ImageNet-sized network on its mini-batch, in full precision
        _classes("head_1000_f32", "train", 64, 2048, 1000, "f32"),
        # local classifier on every position of a module output of the wide network (128 x 8 x 8), a tenth of them unlabelled
        _classes("positions_wide", "train", 8192, 640, 100, "bf16", ignored=0.1),
        # odd sizes in full precision, no bias
        _classes("odd_f32", "train", 777, 333, 12345, "f32", bias=False, ignored=0.05),
        # a large vocabulary: the largest training call
        _classes("vocabulary", "train", 8192, 2048, 32768, "bf16", ignored=0.02),
        # one sample against many classes: reading the weights
        _classes("score_one", "eval", 1, 2048, 100003, "bf16"),
        # validation of a many-class head
        _classes("score_many", "eval", 10000, 640, 21841, "bf16"),
        # one filter of a narrow network (64 x 3x3x64)
        _orthogonal("filter_narrow_f32", 1, 64, 576, "f32"),
        # tall odd matrices, several at once
        _orthogonal("tall_odd", 6, 1001, 333, "bf16"),
        # wide matrices: the largest orthogonalisation
        _orthogonal("wide_large", 2, 2048, 4096, "bf16"),
        # parameter update of the deep narrow network: 55 filters of at most 64 x 576
        _update("update_resnet56", "resnet56", "bf16", True, True),
        # ... and of the wide one: filters of up to 640 x 5760
        _update("update_wrn28_10", "wrn28_10", "bf16", True, True),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["classes", "classes", "orthogonal", "update"])
    if kind == "classes":
        what = rng.choice(["train", "train", "eval"])
        rows, channels, classes = _spread(rng, 1, 10000), _spread(rng, 8, 2048), _spread(rng, 2, 100003)
        rows = max(1, min(rows, MOST_CLASSES // (channels * classes)))
        c = _classes("", what, rows, channels, classes, rng.choice(["f32", "bf16"]), rng.random() < 0.5, rng.choice([0.0, 0.1]))
    elif kind == "orthogonal":
        rows, cols = _spread(rng, 1, 4096), _spread(rng, 1, 4096)
        a, b = min(rows, cols), max(rows, cols)
        count = max(1, min(_spread(rng, 1, 24), MOST_ORTHOGONAL // (STEPS * (4 * a * a * b + 2 * a ** 3))))
        if STEPS * (4 * a * a * b + 2 * a ** 3) > MOST_ORTHOGONAL:
            rows, cols = max(1, rows // 2), max(1, cols // 2)
        c = _orthogonal("", count, rows, cols, rng.choice(["f32", "bf16"]))
    else:
        c = _update("", rng.choice(["tiny", "resnet20", "resnet56", "wrn28_10", "resnet50"]), rng.choice(["f32", "bf16"]),
                    rng.random() < 0.5, rng.random() < 0.5)
    del c["name"]
    return c


def _network(name):
    """(shape, whether it is orthogonalised) of every parameter tensor: filters [Cout, R, S, Cin], affine vectors of the batch
    norms, and the head's weight and bias."""
    out = []

    def conv(co, r, ci):
        out.extend([((co, r, r, ci), True), ((co,), False), ((co,), False)])

    def basic(cin, widths, per_stage):
        for s, w in enumerate(widths):
            for b in range(per_stage):
                conv(w, 3, cin)
                conv(w, 3, w)
                if cin != w or (s > 0 and b == 0):
                    conv(w, 1, cin)
                cin = w
        return cin

    if name == "tiny":
        c, classes = basic(16, [16], 2), 10
    elif name == "resnet50":
        conv(64, 7, 3)
        c, classes = 64, 1000
        for w, n in ((64, 3), (128, 4), (256, 6), (512, 3)):
            for b in range(n):
                conv(w, 1, c)
                conv(w, 3, w)
                conv(4 * w, 1, w)
                if b == 0:
                    conv(4 * w, 1, c)
                c = 4 * w
    else:
        widths, n, classes = {"resnet20": ([16, 32, 64], 3, 10), "resnet56": ([16, 32, 64], 9, 100), "wrn28_10": ([160, 320, 640], 4, 100)}[name]
        conv(16, 3, 3)
        c = basic(16, widths, n)
    return out + [((classes, c), False), ((classes,), False)]


def _layout(case):
    """Tensors of a packed set: (shape, dtype, orthogonalised, byte offset in the parameters, byte offset in the fp32 buffers).
    Filters first, then the fp32 tensors, each at a multiple of 256 bytes; the sizes of the three regions."""
    tensors = _network(case["net"])
    low = case["dtype"] == "bf16"
    table, off, goff, filters = [], 0, 0, 0
    for orth in (True, False):
        for shape, o in tensors:
            if o != orth:
                continue
            n = math.prod(shape)
            table.append((shape, "bf16" if low and orth else "f32", orth, off, goff))
            off += -(-n * (2 if low and orth else 4) // 256) * 256
            goff += -(-n * 4 // 256) * 256
        if orth:
            filters = off
    return tuple(table), off, goff, filters


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def prepare(case, seed):
    g = _generator(seed)
    dev = "cuda"
    low = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    if case["operator"] == "classes":
        n, c, v = case["rows"], case["channels"], case["classes"]
        weight = normal(v, c) / math.sqrt(c)
        labels = torch.randint(0, v, (n,), generator=g, device=dev)
        # partly trained: the score of the right class stands out by 0 to 12
        features = normal(n, c) + 12 * torch.rand((n, 1), generator=g, device=dev) * weight[labels]
        if case["ignored"]:
            labels = torch.where(torch.rand(n, generator=g, device=dev) < case["ignored"], -1, labels)
        return {"case": case, "features": features.to(low), "weight": weight.to(low), "labels": labels.to(torch.int32),
                "bias": normal(v) if case["bias"] else None}
    if case["operator"] == "orthogonal":
        m, n = case["rows"], case["cols"]
        r = max(1, min(m, n) // 4)
        # gradients: a part of low rank that the mini-batch agrees on, and noise
        return {"case": case, "matrices": [(1e-3 * (normal(m, r) @ normal(r, n) / math.sqrt(r) + 0.5 * normal(m, n))).to(low)
                                           for _ in range(case["count"])]}
    table, size, gsize, filters = _layout(case)
    s = {"case": case, "table": table, "filters": filters, "params": torch.zeros(size, dtype=torch.uint8, device=dev)}
    for k in ("grads", "velocity") + (("master",) if case["master"] else ()):
        s[k] = torch.zeros(gsize // 4, dtype=torch.float32, device=dev)
    for shape, dtype, orth, off, goff in table:
        k = math.prod(shape)
        w = normal(k) * math.sqrt(2.0 / math.prod(shape[1:])) if len(shape) > 1 else 1.0 + 0.1 * normal(k)
        p = _param(s["params"], dtype, off, k)
        p.copy_(w)
        s["grads"][goff // 4:goff // 4 + k] = 1e-3 * normal(k)
        s["velocity"][goff // 4:goff // 4 + k] = 1e-2 * normal(k)
        if case["master"]:
            s["master"][goff // 4:goff // 4 + k] = w
    return s


def _param(buf, dtype, off, n):
    return buf[off:off + 2 * n].view(torch.bfloat16) if dtype == "bf16" else buf[off:off + 4 * n].view(torch.float32)


def _cross_entropy(features, weight, bias, labels, train, real):
    """Plain form in the type `real`."""
    x, w = features.to(real), weight.to(real)
    v = weight.shape[0]
    logits = x @ w.t()
    if bias is not None:
        logits += bias.to(real)
    valid = (labels >= 0) & (labels < v)
    at = torch.where(valid, labels, 0).long().unsqueeze(1)
    top = logits.max(dim=1, keepdim=True).values
    target = logits.gather(1, at)
    e = torch.exp(logits - top)
    total = e.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    rows = torch.where(valid, (lse - target).squeeze(1), 0)
    count = valid.sum().clamp(min=1)
    out = {"loss": (rows.sum() / count).reshape(1), "row_loss": rows, "lse": lse.squeeze(1)}
    if train:
        p = e.div_(total)
        p.scatter_add_(1, at, torch.full_like(at, -1, dtype=real))
        p *= valid.unsqueeze(1)
        p /= count
        out |= {"dfeatures": p @ w, "dweight": p.t() @ torch.where(valid.unsqueeze(1), x, 0)}
        if bias is not None:
            out["dbias"] = p.sum(dim=0)
    return out


def _newton_schulz(u):
    """Plain form: X <- a X + b (X X^T) X + c (X X^T)^2 X, from X = U / |U|."""
    a, b, c = COEFS
    x = u / u.norm().clamp(min=1e-7)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    for _ in range(STEPS):
        s = x @ x.t()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if tall else x


def _plain_update(s, real, params, velocity, master):
    case = s["case"]
    for shape, dtype, orth, off, goff in s["table"]:
        n = math.prod(shape)
        part = slice(goff // 4, goff // 4 + n)
        p, v, grad = params(dtype, off, n), velocity[part], s["grads"][part].to(real)
        w = (p if master is None else master[part]).to(real)
        if orth:
            v.copy_(MOMENTUM * v + grad)
            u = grad + MOMENTUM * v if case["nesterov"] else v
            rows = shape[0]
            step = _newton_schulz(u.view(rows, -1)).reshape(-1) * math.sqrt(max(1.0, rows * rows / n))
            w = w * (1 - LR * WEIGHT_DECAY) - LR * step
        else:
            v.copy_(MOMENTUM * v + grad + WEIGHT_DECAY * w)
            w = w - REST_LR * v
        if master is not None:
            master[part] = w
        p.copy_(w)


def run(state):
    case = state["case"]
    if own:
        from paper_2112_05387_amd import ops
    if case["operator"] == "classes":
        x, w, b, y = (state[k] for k in ("features", "weight", "bias", "labels"))
        if own:
            loss, row_loss, lse = ops.linear_ce_forward(x, w, y, bias=b)
            out = {"loss": loss, "row_loss": row_loss, "lse": lse}
            if case["pass"] == "train":
                dx, dw, db = ops.linear_ce_backward(x, w, y, lse, bias=b)
                out |= {"dfeatures": dx, "dweight": dw}
                if b is not None:
                    out["dbias"] = db
            return out
        out = _cross_entropy(x, w, b, y, case["pass"] == "train", torch.float32)
        if "dfeatures" in out:
            out["dfeatures"] = out["dfeatures"].to(x.dtype)
        return out
    if case["operator"] == "orthogonal":
        if own:
            return ops.orthogonalize(state["matrices"], steps=STEPS)
        return [_newton_schulz(u.float()).to(u.dtype) for u in state["matrices"]]
    if own:
        ops.muon_update(state["table"], state["params"], state["grads"], state["velocity"], state.get("master"), lr=LR, momentum=MOMENTUM,
                        nesterov=case["nesterov"], weight_decay=WEIGHT_DECAY, rest_lr=REST_LR, steps=STEPS)
    else:
        _plain_update(state, torch.float32, lambda dtype, off, n: _param(state["params"], dtype, off, n), state["velocity"], state.get("master"))
    low = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    out = {"filters": state["params"][:state["filters"]].view(low), "rest": state["params"][state["filters"]:].view(torch.float32),
           "velocity": state["velocity"]}
    if case["master"]:
        out["master"] = state["master"]
    return out


def _cost(case):
    """(flops, bytes) that no way of computing the case can do without."""
    if case["operator"] == "classes":
        n, c, v = case["rows"], case["channels"], case["classes"]
        e = 2 if case["dtype"] == "bf16" else 4
        train = case["pass"] == "train"
        nbytes = (n * c + v * c) * e + 4 * n + 8 * n + (4 * v if case["bias"] else 0)
        if train:
            nbytes += n * c * e + 4 * v * c + (4 * v if case["bias"] else 0)
        return (6.0 if train else 2.0) * n * c * v, float(nbytes)

    def newton_schulz(m, n):
        a, b = min(m, n), max(m, n)
        return STEPS * (a * (a + 1) * b + a * a * (a + 1) + 2.0 * a * a * b)      # the two inner products are symmetric

    if case["operator"] == "orthogonal":
        m, n = case["rows"], case["cols"]
        return case["count"] * newton_schulz(m, n), 2.0 * case["count"] * m * n * (2 if case["dtype"] == "bf16" else 4)
    flops = nbytes = 0.0
    for shape, dtype, orth, _, _ in _layout(case)[0]:
        n = math.prod(shape)
        nbytes += n * (4 + 8 + (8 + (2 if dtype == "bf16" else 4) if case["master"] else 2 * (2 if dtype == "bf16" else 4)))
        flops += newton_schulz(shape[0], n // shape[0]) if orth else 4.0 * n
    return flops, nbytes


def work(case):
    flops, nbytes = _cost(case)
    return {"bytes": nbytes, "flops": flops}


def exact(case, seed):
    """The definitions in 64 bits: probabilities from the log-softmax, the polynomial applied to the singular directions by
    products of the matrix itself."""
    s = prepare(case, seed)
    if case["operator"] == "classes":
        x, w, y = s["features"].double(), s["weight"].double(), s["labels"].long()
        z = x.mm(w.t())
        if s["bias"] is not None:
            z = z.add_(s["bias"].double())
        lse = z.logsumexp(1)
        rows = torch.arange(len(y), device=y.device)
        keep = y >= 0
        index = y.clamp(min=0)
        nll = (lse - z[rows, index]) * keep
        count = max(1, int(keep.sum()))
        out = {"loss": nll.sum().reshape(1) / count, "row_loss": nll, "lse": lse}
        if case["pass"] == "train":
            d = z.sub_(lse.unsqueeze(1)).exp_()
            d[rows, index] -= 1.0
            d.mul_((keep.double() / count).unsqueeze(1))
            out |= {"dfeatures": d.mm(w), "dweight": d.t().mm(x)}
            if s["bias"] is not None:
                out["dbias"] = d.sum(0)
        return out

    def polar(u):
        a, b, c = COEFS
        wide = u if u.shape[0] <= u.shape[1] else u.t()
        y = wide / max(float(wide.pow(2).sum().sqrt()), 1e-7)
        for _ in range(STEPS):
            g = y.mm(y.t())
            gy = g.mm(y)
            y = a * y + b * gy + c * g.mm(gy)
        return y if u.shape[0] <= u.shape[1] else y.t()

    if case["operator"] == "orthogonal":
        return [polar(u.double()) for u in s["matrices"]]
    size = sum(-(-math.prod(t[0]) * 4 // 256) * 64 for t in s["table"])
    nv = torch.zeros(size, dtype=torch.float64, device="cuda")
    nm = torch.zeros_like(nv)
    low = case["dtype"] == "bf16"
    filters = torch.zeros(s["filters"] // (2 if low else 4), dtype=torch.float64, device="cuda")
    rest = torch.zeros((s["params"].numel() - s["filters"]) // 4, dtype=torch.float64, device="cuda")
    for shape, dtype, orth, off, goff in s["table"]:
        n = math.prod(shape)
        at = goff // 4
        grad, v = s["grads"][at:at + n].double(), s["velocity"][at:at + n].double()
        w = (s["master"][at:at + n] if case["master"] else _param(s["params"], dtype, off, n)).double()
        if orth:
            v = v * MOMENTUM + grad
            u = grad + MOMENTUM * v if case["nesterov"] else v
            o = polar(u.reshape(shape[0], n // shape[0])).reshape(-1)
            w = w - LR * (WEIGHT_DECAY * w + math.sqrt(max(1.0, shape[0] / (n // shape[0]))) * o)
            filters[off // (2 if low else 4):off // (2 if low else 4) + n] = w
        else:
            v = v * MOMENTUM + (grad + WEIGHT_DECAY * w)
            w = w - REST_LR * v
            o = (off - s["filters"]) // 4
            rest[o:o + n] = w
        nv[at:at + n] = v
        nm[at:at + n] = w
    out = {"filters": filters, "rest": rest, "velocity": nv}
    if case["master"]:
        out["master"] = nm
    return out
