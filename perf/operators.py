"""The operators at the end of a training step, as cases to be timed: the loss of a linear layer over many classes
with its gradients, and the orthogonalised update.

A case is one call of an entry point of ``paper_2112_05387_b200``.  Keys of a case
    op         "linear_ce"      lp_linear_cross_entropy: rows, width, classes; grads (or the loss alone); bias;
                                ignored: share of the rows whose label takes no part
               "orthogonalize"  lp_orthogonalize: batch matrices of rows x cols
               "muon"           lp_muon_update: the same matrices as weights, with their momentum
    dtype      "bf16" | "f32": type of features, weights and gradients (labels int32, losses and momentum fp32)
"""
import math

import torch

own = False

_COEFFS = (3.4445, -4.7750, 2.0315)   # quintic that drives singular values towards 1 in five steps
_STEPS, _EPS = 5, 1e-7
_LR, _MOMENTUM, _DECAY = 0.02, 0.95, 0.01


def _ce(name, rows, width, classes, dtype, grads=True, bias=False, ignored=0.0):
    case = dict(op="linear_ce", rows=rows, width=width, classes=classes, dtype=dtype, grads=grads, bias=bias,
                ignored=ignored)
    return dict(case, name=name) if name else case


def _matrix(name, op, batch, rows, cols, dtype, nesterov=True):
    case = dict(op=op, batch=batch, rows=rows, cols=cols, dtype=dtype)
    if op == "muon":
        case["nesterov"] = nesterov
    return dict(case, name=name) if name else case


def listed():
    return [
        # the head of the ImageNet-shaped workload at its own batch, in the precision of its master weights
        _ce("ce_head_f32", 64, 512, 1000, "f32", bias=True),
        # scoring one feature vector against a large set of classes
        _ce("ce_one_row", 1, 2048, 100000, "bf16", grads=False),
        # evaluation over an odd number of classes, a ragged batch
        _ce("ce_eval_odd", 2011, 1024, 50021, "bf16", grads=False, bias=True, ignored=0.1),
        # training over tens of thousands of classes
        _ce("ce_train", 4096, 2048, 32000, "bf16", ignored=0.1),
        # the same in fp32, an odd number of rows, a wide network's features
        _ce("ce_train_f32", 1001, 640, 20011, "f32", bias=True, ignored=0.1),
        # the largest: rows and classes of a large run
        _ce("ce_train_large", 8192, 4096, 128000, "bf16"),
        # 3x3 convolutions of the last stage of ResNet-56: 18 matrices of 64 x 576
        _matrix("ortho_conv64_f32", "orthogonalize", 18, 64, 576, "f32"),
        # 3x3 convolutions of the last stage of WideResNet-28-10
        _matrix("ortho_wrn", "orthogonalize", 7, 640, 5760, "bf16"),
        # a large hidden layer
        _matrix("ortho_large", "orthogonalize", 1, 4096, 16384, "bf16"),
        # one small layer: 3x3 convolution of ResNet-56's first stage
        _matrix("muon_conv16", "muon", 1, 16, 144, "f32"),
        # 1x1 convolutions of ResNet-50 that narrow and widen: tall matrices
        _matrix("muon_tall_f32", "muon", 2, 2048, 512, "f32", nesterov=False),
        # a square layer and its momentum in training
        _matrix("muon_square", "muon", 2, 4096, 4096, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if rng.random() < 0.5:
        while True:
            rows, width, classes = _log_int(rng, 1, 8192), _log_int(rng, 16, 4096), _log_int(rng, 2, 128000)
            grads = rng.random() < 0.7
            # an eighth of the largest listed case: its sizes are reached one or two at a time
            if rows * width * classes <= 8192 * 4096 * 128000 // 8 and (dtype == "bf16" or rows * width * classes <= 2 ** 36):
                return _ce(None, rows, width, classes, dtype, grads, rng.random() < 0.5, rng.choice([0.0, 0.1, 0.5]))
    while True:
        rows, cols = _log_int(rng, 1, 8192), _log_int(rng, 1, 8192)
        batch = _log_int(rng, 1, 32)
        low, high = min(rows, cols), max(rows, cols)
        if batch * low * low * high <= 4096 * 4096 * 16384 // 4 and batch * rows * cols <= 2 ** 27:
            return _matrix(None, rng.choice(["orthogonalize", "muon"]), batch, rows, cols, dtype, rng.random() < 0.5)


def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _generator(seed, k):
    return torch.Generator("cuda").manual_seed(1000003 * int(seed) + k)


def _scratch(lp, nbytes):
    """Workspace of a program: what the library asks for, on a 256-byte boundary."""
    buf = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")
    return buf, (buf.data_ptr() + 255) // 256 * 256, nbytes


def _ce_inputs(case, seed):
    T, D, V, dt = case["rows"], case["width"], case["classes"], _torch_dtype(case)
    g = _generator(seed, 1)
    w = torch.randn(V, D, generator=g, device="cuda", dtype=torch.float32).mul_(D ** -0.5).to(dt)
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    # features that lean towards their class, some more than others, as those of a network in training do
    lean = 4.0 * torch.rand(T, 1, generator=g, device="cuda")
    x = (torch.randn(T, D, generator=g, device="cuda") + lean * w[labels].float()).to(dt)
    bias = torch.randn(V, generator=g, device="cuda").mul_(0.1).to(dt) if case["bias"] else None
    out = torch.rand(T, generator=g, device="cuda") < case["ignored"]
    out[0] = False
    labels = torch.where(out, torch.full_like(labels, -100), labels).to(torch.int32)
    return x, w, bias, labels


def _matrices(case, seed):
    """Gradients as training makes them: a few strong directions over a broad floor."""
    B, m, n = case["batch"], case["rows"], case["cols"]
    g = _generator(seed, 2)
    r = max(1, min(8, m, n))
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    strong = (rand(B, m, r) * 2.0 ** -torch.arange(r, device="cuda")) @ rand(B, r, n)
    grad = (1e-3 * (rand(B, m, n) + 0.5 * strong)).to(_torch_dtype(case))
    if case["op"] != "muon":
        return grad, None, None
    weights = (rand(B, m, n) * (2.0 / n) ** 0.5).to(_torch_dtype(case))
    momentum = 2e-3 * rand(B, m, n)
    return grad, weights, momentum


def prepare(case, seed):
    state = dict(case=case)
    if case["op"] == "linear_ce":
        state["x"], state["w"], state["bias"], state["labels"] = _ce_inputs(case, seed)
    else:
        state["grad"], state["weights"], state["momentum"] = _matrices(case, seed)
    if own:
        import paper_2112_05387_b200 as lp
        dt = lp.LP_BF16 if case["dtype"] == "bf16" else lp.LP_F32
        if case["op"] == "linear_ce":
            T, D, V = case["rows"], case["width"], case["classes"]
            need = lp.lp_linear_cross_entropy_scratch_bytes(dt, T, D, V, case["grads"])
            state["loss"] = torch.empty(2, dtype=torch.float32, device="cuda")
            state["row_loss"] = torch.empty(T, dtype=torch.float32, device="cuda")
            for k, of in (("dx", "x"), ("dw", "w"), ("dbias", "bias")):
                state[k] = torch.empty_like(state[of]) if case["grads"] and state[of] is not None else None
        else:
            need = lp.lp_orthogonalize_scratch_bytes(dt, case["batch"], case["rows"], case["cols"])
            state["out"] = torch.empty_like(state["grad"]) if case["op"] == "orthogonalize" else None
        state["buffer"], state["scratch"], state["scratch_bytes"] = _scratch(lp, need)
        state["dtype"] = dt
    return state


def _plain_ce(case, s):
    x, w, labels = s["x"].float(), s["w"].float(), s["labels"].long()
    logits = x @ w.T
    if s["bias"] is not None:
        logits += s["bias"].float()
    counted = labels >= 0
    n = counted.sum().float()
    top = logits.amax(1, keepdim=True)
    at = labels.clamp(min=0).unsqueeze(1)
    target = logits.gather(1, at)
    e = logits.sub_(top).exp_()
    total = e.sum(1, keepdim=True)
    row_loss = torch.where(counted, (top + total.log() - target).squeeze(1), torch.zeros_like(top).squeeze(1))
    got = {"loss": row_loss.sum() / n, "row_loss": row_loss}
    if case["grads"]:
        weight = counted.float().unsqueeze(1) / n
        d = e.div_(total).scatter_add_(1, at, torch.full_like(target, -1.0)).mul_(weight)
        got["dx"] = (d @ w).to(s["x"].dtype)
        got["dw"] = (d.T @ x).to(s["w"].dtype)
        if s["bias"] is not None:
            got["dbias"] = d.sum(0).to(s["bias"].dtype)
    return got


def _plain_orthogonalize(g):
    a, b, c = _COEFFS
    x = g.float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.mT
    x = x / x.square().sum((1, 2), keepdim=True).sqrt().clamp(min=_EPS)
    # five steps of the iteration, written out once
    def step(x):
        gram = x @ x.mT
        return a * x + (b * gram + c * (gram @ gram)) @ x
    x = step(step(step(step(step(x)))))
    return x.mT if tall else x


def run(s):
    case = s["case"]
    if own:
        import paper_2112_05387_b200 as lp
        if case["op"] == "linear_ce":
            lp.lp_linear_cross_entropy(s["dtype"], case["rows"], case["width"], case["classes"], s["x"], s["w"], s["bias"],
                                       s["labels"], 1.0, s["loss"], s["row_loss"], s["dx"], s["dw"], s["dbias"],
                                       s["scratch"], s["scratch_bytes"])
            got = {"loss": s["loss"][0], "row_loss": s["row_loss"]}
            got.update({k: s[k] for k in ("dx", "dw", "dbias") if s[k] is not None})
            return got
        if case["op"] == "orthogonalize":
            lp.lp_orthogonalize(s["dtype"], case["batch"], case["rows"], case["cols"], s["grad"], s["out"], _STEPS, None,
                                _EPS, s["scratch"], s["scratch_bytes"])
            return s["out"]
        lp.lp_muon_update(s["dtype"], case["batch"], case["rows"], case["cols"], s["weights"], s["grad"], s["momentum"],
                          _LR, _MOMENTUM, case["nesterov"], _DECAY, _scale(case), _STEPS, None, _EPS, s["scratch"],
                          s["scratch_bytes"])
        return {"weights": s["weights"], "momentum": s["momentum"]}
    if case["op"] == "linear_ce":
        return _plain_ce(case, s)
    if case["op"] == "orthogonalize":
        return _plain_orthogonalize(s["grad"]).to(s["grad"].dtype).contiguous()
    grad, m = s["grad"].float(), s["momentum"]
    m.mul_(_MOMENTUM).add_(grad)
    o = _plain_orthogonalize(grad + _MOMENTUM * m if case["nesterov"] else m)
    w = s["weights"]
    w.copy_((1.0 - _LR * _DECAY) * w.float() - _LR * _scale(case) * o)
    return {"weights": w, "momentum": m}


def _scale(case):
    return max(1.0, case["rows"] / case["cols"]) ** 0.5


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "linear_ce":
        T, D, V = case["rows"], case["width"], case["classes"]
        reads = (T * D + V * D + (V if case["bias"] else 0)) * size + 4 * T
        if not case["grads"]:
            return {"bytes": reads + 4 * T + 4, "flops": 2.0 * T * D * V}
        return {"bytes": reads + 4 * T + 4 + (T * D + V * D + (V if case["bias"] else 0)) * size, "flops": 6.0 * T * D * V}
    B, m, n = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # X X^T and its square are symmetric: half of each
    flops = float(B) * _STEPS * (m * (m + 1.0) * n + m * (m + 1.0) * m + 2.0 * m * m * n)
    elems = B * m * n
    if case["op"] == "orthogonalize":
        return {"bytes": 2 * elems * size, "flops": flops}
    return {"bytes": 3 * elems * size + 8 * elems, "flops": flops}


def exact(case, seed):
    def linear_ce():
        x, w, bias, labels = _ce_inputs(case, seed)
        size = case["rows"] * case["width"] * case["classes"]
        if size > 2 ** 43:
            return None
        T = x.shape[0]
        w64, n = w.double(), int((labels >= 0).sum())
        losses = torch.zeros(T, dtype=torch.float64, device="cuda")
        grads = case["grads"]
        dx = torch.empty(x.shape, dtype=torch.float64, device="cuda") if grads else None
        dw = torch.zeros_like(w64) if grads else None
        db = torch.zeros(w.shape[0], dtype=torch.float64, device="cuda") if grads and bias is not None else None
        for lo in range(0, T, 1024):   # rows in blocks: the whole would not fit beside its copies
            part = slice(lo, min(T, lo + 1024))
            x64, y = x[part].double(), labels[part].long()
            z = torch.einsum("td,vd->tv", x64, w64)
            if bias is not None:
                z = z + bias.double()
            logp = torch.log_softmax(z, dim=1)
            del z
            rows = torch.nonzero(y >= 0).squeeze(1)
            losses[lo + rows] = -logp[rows, y[rows]]
            if grads:
                p = logp.exp_()
                p[rows, y[rows]] -= 1.0
                p[y < 0] = 0.0
                p /= max(n, 1)
                dx[part] = torch.einsum("tv,vd->td", p, w64)
                dw += torch.einsum("tv,td->vd", p, x64)
                if db is not None:
                    db += p.sum(0)
                del p
        got = {"loss": losses.sum() / n, "row_loss": losses}
        if grads:
            got["dx"], got["dw"] = dx, dw
            if db is not None:
                got["dbias"] = db
        return got

    def orthogonalize(g):
        """The polynomial applied through X^T X for tall and X X^T for wide matrices, one matrix at a time, in 64 bits."""
        a, b, c = _COEFFS
        out = []
        for k in range(g.shape[0]):
            x = g[k].double()
            x = x / max(float(torch.linalg.vector_norm(x)), _EPS)
            for _ in range(_STEPS):
                if x.shape[0] <= x.shape[1]:
                    s = torch.mm(x, x.t())
                    p = torch.addmm(b * s, s, s, alpha=c)
                    x = torch.addmm(x, p, x, beta=a)
                else:
                    s = torch.mm(x.t(), x)
                    p = torch.addmm(b * s, s, s, alpha=c)
                    x = torch.addmm(x, x, p, beta=a)
            out.append(x)
        return torch.stack(out)

    if case["op"] == "linear_ce":
        return linear_ce()
    grad, weights, momentum = _matrices(case, seed)
    if case["op"] == "orthogonalize":
        return orthogonalize(grad)
    g = grad.double()
    m = _MOMENTUM * momentum.double() + g
    o = orthogonalize(g + _MOMENTUM * m if case["nesterov"] else m)
    w = weights.double() * (1.0 - _LR * _DECAY) - _LR * _scale(case) * o
    return {"weights": w, "momentum": m}
