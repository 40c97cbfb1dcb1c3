"""What is measured of the operators on an 8-bit LM head: rows quantised to 8-bit integers with a scale each, the matrix product of
such rows (a scale for each token and each channel) with its gradient, and the softmax cross entropy over that head in pieces of the
vocabulary, forward and with the gradient of the hidden states.

`run` computes an operator in plain torch operations (`own` false) or through the package (`own` true).  Sizes are those
of the package's own workloads, heads of 2048 x 128256, 1024 x 151936 and 256 x 4096, and a projection of 2048 to 8192 channels.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # loading a model: its head is quantised once
        dict(name="quantize_head", op="quantize", T=128256, d=2048, dtype="bf16"),
        # a small batch of fp32 rows of odd length
        dict(name="quantize_rows_129", op="quantize", T=129, d=1003, dtype="f32"),
        # one decoding step of one sequence: fp32 logits for a sampler; the head is all there is to read
        dict(name="logits_decode_1", op="logits", T=1, d=2048, V=128256, dtype="bf16", out="f32", bias=False),
        # a decoding step of an odd batch
        dict(name="logits_decode_67", op="logits", T=67, d=1024, V=151936, dtype="bf16", out="bf16", bias=False),
        # a projection inside the model for a prompt
        dict(name="projection_2047", op="logits", T=2047, d=2048, V=8192, dtype="bf16", out="bf16", bias=True),
        # the logits of a scored batch, kept
        dict(name="logits_1000", op="logits", T=1000, d=1024, V=151936, dtype="bf16", out="bf16", bias=False),
        # gradients through the frozen projection and through the frozen head
        dict(name="projection_bwd_4096", op="logits_bwd", T=4096, d=2048, V=8192, dtype="bf16"),
        dict(name="logits_bwd_1000", op="logits_bwd", T=1000, d=1024, V=151936, dtype="bf16"),
        # evaluation: the loss of each token
        dict(name="loss_8192", op="loss", T=8192, d=2048, V=128256, dtype="bf16", masked=0.1),
        # training steps of a draft model against a frozen head: loss and gradient of the hidden states
        dict(name="loss_step_4096", op="loss_step", T=4096, d=2048, V=128256, dtype="bf16", masked=0.1),
        dict(name="loss_step_300", op="loss_step", T=300, d=1024, V=151936, dtype="bf16", masked=0.2),
        # the small head that checks of a training run use
        dict(name="loss_step_64", op="loss_step", T=64, d=256, V=4096, dtype="bf16", masked=0.0),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["quantize", "logits", "logits", "logits_bwd", "loss", "loss_step", "loss_step"])
    if op == "quantize":
        while True:
            T, d = spread(1, 160000), spread(8, 8192)
            if T * d <= 128256 * 2048:
                return dict(op=op, T=T, d=d, dtype=rng.choice(["bf16", "f32"]))
    most = dict(logits=1000 * 1024.0 * 151936, logits_bwd=1000 * 1024.0 * 151936, loss=8192 * 2048.0 * 128256, loss_step=4096 * 2048.0 * 128256)[op]
    while True:
        T, d, V = spread(1, 8192), 8 * spread(16, 512), spread(1000, 160000)
        if T * float(d) * V <= most and (op.startswith("loss") or T * V <= 1000 * 151936):
            break
    c = dict(op=op, T=T, d=d, V=V, dtype="bf16")
    if op == "logits":
        c.update(d=d - rng.choice([0, 0, 1, 4, 7]), dtype=rng.choice(["bf16", "bf16", "f32"]), out=rng.choice(["bf16", "f32"]), bias=rng.random() < 0.4)
    elif op != "logits_bwd":
        c.update(masked=rng.choice([0.0, 0.1, 0.3]))
    return c


def _quantize(x):
    """Each row in whole steps of its largest value / 127, halves to the even step; in 64 bits, where halves are exact."""
    x = x.double()
    most = x.abs().amax(1)
    steps = torch.round(x * 127.0 / torch.where(most > 0, most, 1.0).unsqueeze(1))
    return steps.to(torch.int8), (most / 127.0).float()


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    T, d, dt = case["T"], case["d"], DTYPES[case["dtype"]]

    def rand(*shape):
        return torch.rand(*shape, generator=g, device=dev)

    s = dict(case=dict(case))
    if case["op"] == "quantize":
        # rows of different lengths, as heads have
        s["X"] = (torch.randn(T, d, generator=g, device=dev) * (0.01 + 0.04 * rand(T, 1))).to(dt)
        return s
    V = case["V"]
    W = (torch.randn(V, d, generator=g, device=dev) * (0.01 + 0.02 * rand(V, 1))).to(torch.bfloat16)
    # the 8-bit head as a checkpoint holds it: rows padded to whole 16 bytes
    q = torch.zeros(V, (d + 15) // 16 * 16, dtype=torch.int8, device=dev)
    scale = torch.empty(V, device=dev)
    for i in range(0, V, 16384):
        q[i:i + 16384, :d], scale[i:i + 16384] = _quantize(W[i:i + 16384])
    s["q"], s["scale"] = q[:, :d], scale
    if case["op"] == "logits_bwd":
        ld = (V + 7) // 8 * 8
        s["dY"] = (torch.randn(T, ld, generator=g, device=dev) * rand(T, 1) / T).to(torch.bfloat16)[:, :V]
    else:
        # hidden states with a few channels that are larger than the rest
        H = torch.randn(T, d, generator=g, device=dev) * (1.0 + 5.0 * (rand(d) < 0.01))
        if case["op"] != "logits":
            labels = torch.randint(0, V, (T,), generator=g, device=dev)
            Wy = W[labels].float()
            # half of the rows know their token, as a trained model's do
            H = H + Wy * ((6.0 + 8.0 * rand(T)) * (rand(T) < 0.5) / (Wy * Wy).sum(1).clamp(min=1e-6)).unsqueeze(1)
            off = rand(T) < case["masked"]
            s["valid"] = (~off).to(torch.uint8) if case["masked"] > 0 else None
            s["labels"] = torch.where(off, torch.full_like(labels, -100), labels)
            # the upstream gradient of each token's loss: token weights over their number
            s["grad_nll"] = rand(T) / T
        s["X"] = H.to(dt)
    s["bias"] = 0.1 * torch.randn(V, generator=g, device=dev) if case.get("bias") else None
    if own:
        from paper_2605_08632_b200.api import Int8Head
        s["head"] = Int8Head.from_quantized(s["q"], s["scale"], s["bias"])
    return s


def run(s):
    return {"quantize": _run_quantize, "logits": _run_logits, "logits_bwd": _run_logits_bwd, "loss": _run_loss, "loss_step": _run_loss}[s["case"]["op"]](s)


# ---------------------------------------------------------------------------- plain forms
def _run_quantize(s):
    if own:
        from paper_2605_08632_b200.api import quantize_rows
        q, scale = quantize_rows(s["X"])
    else:
        q, scale = _quantize(s["X"])
    return {"q": q, "scale": scale}


def _product(X, q, scale):
    xq, xs = _quantize(X)
    return (xq.float() @ q.float().T) * xs.unsqueeze(1) * scale


def _run_logits(s):
    out = DTYPES[s["case"]["out"]]
    if own:
        return {"logits": s["head"].logits(s["X"], out_dtype=out)}
    z = _product(s["X"], s["q"], s["scale"])
    if s["bias"] is not None:
        z = z + s["bias"]
    return {"logits": z.to(out)}


def _run_logits_bwd(s):
    if own:
        return {"dX": s["head"].logits_backward(s["dY"])}
    return {"dX": ((s["dY"].float() * s["scale"]) @ s["q"].float()).to(torch.bfloat16)}


def _run_loss(s):
    c, X, labels, valid = s["case"], s["X"], s["labels"], s["valid"]
    if own:
        nll, lse = s["head"].loss_forward(X, labels, valid)
        if c["op"] == "loss":
            return {"nll": nll, "lse": lse}
        return {"nll": nll, "lse": lse, "dX": s["head"].loss_backward(X, labels, valid, s["grad_nll"], nll, lse)}
    V = c["V"]
    ok = (labels >= 0) & (labels < V)
    live = valid.bool() if valid is not None else torch.ones_like(ok)
    ok = ok & live
    y = labels.clamp(0, V - 1).unsqueeze(1)
    z = _product(X, s["q"], s["scale"])
    m = z.amax(1, keepdim=True)
    lse = m + torch.exp(z - m).sum(1, keepdim=True).log()
    nll = torch.where(ok, (lse - z.gather(1, y)).squeeze(1), 0.0)
    out = {"nll": nll, "lse": torch.where(live, lse.squeeze(1), 0.0)}
    if c["op"] == "loss_step":
        dz = torch.exp(z - lse)
        dz.scatter_add_(1, y, torch.full_like(lse, -1.0))
        dz *= torch.where(ok, s["grad_nll"], 0.0).unsqueeze(1)
        out["dX"] = ((dz * s["scale"]) @ s["q"].float()).to(X.dtype)
    return out


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    T, d, b = float(case["T"]), float(case["d"]), 2.0 if case["dtype"] == "bf16" else 4.0
    if case["op"] == "quantize":
        return {"bytes": T * d * (b + 1) + 4 * T, "flops": 2 * T * d}
    V = float(case["V"])
    head = V * d + 4 * V
    if case["op"] == "logits":
        return {"bytes": T * d * b + head + T * V * (2 if case["out"] == "bf16" else 4) + (4 * V if case["bias"] else 0), "flops": 2 * T * d * V}
    if case["op"] == "logits_bwd":
        return {"bytes": T * V * 2 + head + T * d * 2, "flops": 2 * T * d * V}
    step = case["op"] == "loss_step"            # one product for the logits, one more for the gradient of the hidden states
    return {"bytes": T * d * b * (2 if step else 1) + head + T * (21 if step else 17), "flops": (4 if step else 2) * T * d * V}


# ---------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    s.pop("head", None)

    def whole_steps(x):
        """The nearest whole number of steps of (largest value / 127), found from below by halves of a step, and the step."""
        size, most = x.double().abs(), x.double().abs().max(dim=1, keepdim=True).values
        halves = torch.floor(size * 254.0 / most.clamp(min=1e-300))
        border = (size * 254.0 == halves * most) & (halves % 2 == 1)
        return torch.where(border, 2 * torch.round(halves / 4), torch.floor((halves + 1) / 2)) * torch.sign(x.double()), most / 127.0

    if case["op"] == "quantize":
        return {"q": None, "scale": s["X"].double().abs().amax(1) / 127.0}
    Wd = s["q"].double() * s["scale"].double().unsqueeze(1)
    if case["op"] == "logits_bwd":
        return {"dX": s["dY"].double() @ Wd}
    T, V, dev = case["T"], case["V"], Wd.device
    rows = max(1, min(T, (1 << 28) // V))
    chunks = [slice(i, min(T, i + rows)) for i in range(0, T, rows)]

    def logits(c):
        n, step = whole_steps(s["X"][c])
        return (n * step.float().double()) @ Wd.T          # the scale is kept in 32 bits

    if case["op"] == "logits":
        z = torch.cat([logits(c) for c in chunks])
        return {"logits": z if s["bias"] is None else z + s["bias"].double()}
    valid = s["valid"].bool() if s["valid"] is not None else torch.ones(T, dtype=torch.bool, device=dev)
    ok = valid & (s["labels"] >= 0) & (s["labels"] < V)
    nll, lse = (torch.zeros(T, dtype=torch.float64, device=dev) for _ in range(2))
    dX = torch.zeros(T, case["d"], dtype=torch.float64, device=dev)
    for c in chunks:
        z = logits(c)
        lp = torch.log_softmax(z, 1)
        y = s["labels"][c].clamp(0, V - 1)
        at = torch.arange(z.shape[0], device=dev)
        lse[c] = torch.where(valid[c], z[:, 0] - lp[:, 0], 0.0)
        nll[c] = torch.where(ok[c], -lp[at, y], 0.0)
        if case["op"] == "loss_step":
            p = lp.exp()
            p[at, y] -= 1.0
            dX[c] = (torch.where(ok[c], s["grad_nll"][c].double(), 0.0).unsqueeze(1) * p) @ Wd
    return {"nll": nll, "lse": lse} if case["op"] == "loss" else {"nll": nll, "lse": lse, "dX": dX}
