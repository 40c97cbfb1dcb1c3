"""What is measured of the LM-head operators beside the CAT loss: log probabilities of given tokens with entropy and
top alternatives (forward, and backward for policy-gradient training), and the CAT-weighted distillation from a
teacher's stored top logits (forward and backward in one call).

`run` computes an operator in plain torch operations (`own` false) or through the package (`own` true).  Sizes are those
of the package's own workloads: heads of 2048 x 128256, 1024 x 151936 and 256 x 4096, draft blocks of 8 and 16 rows.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one decoding step of one sequence: the target's choice and 20 alternatives for a client; W is all there is to read
        dict(name="logprob_decode_1", op="logprob", T=1, d=2048, V=128256, top_k=20, dtype="bf16", masked=0.0, labels=False),
        # a decoding step of an odd batch with a few empty slots, few alternatives
        dict(name="logprob_decode_67", op="logprob", T=67, d=1024, V=151936, top_k=5, dtype="bf16", masked=0.1, labels=True),
        # scoring rollouts: log probabilities and entropies only
        dict(name="logprob_score_4001", op="logprob", T=4001, d=1024, V=151936, top_k=0, dtype="bf16", masked=0.1, labels=True),
        # writing a teacher's top lists for later distillation
        dict(name="logprob_teacher_8192", op="logprob", T=8192, d=2048, V=128256, top_k=64, dtype="bf16", masked=0.0, labels=True),
        # the small fp32 head that checks of a training run use
        dict(name="logprob_f32_512", op="logprob", T=512, d=256, V=4096, top_k=8, dtype="f32", masked=0.1, labels=True),
        # policy-gradient step: gradients of the log probabilities and of an entropy bonus
        dict(name="logprob_bwd_4096", op="logprob_bwd", T=4096, d=2048, V=128256, dtype="bf16", masked=0.1, entropy=True),
        # the same for a short odd batch, without an entropy bonus
        dict(name="logprob_bwd_300", op="logprob_bwd", T=300, d=1024, V=151936, dtype="bf16", masked=0.2, entropy=False),
        # the training step of the main workload with a stored top-16 list of the teacher in the place of its head
        dict(name="topk_kd_16384", op="topk_kd", T=16384, K=8, d=2048, V=128256, k=16, dtype="bf16", masked=0.0, beta=0.1,
             renormalize=True, conf="own", run_off=False),
        # long lists, longer blocks, masked rows, blocks that run past the end of the teacher's sequence
        dict(name="topk_kd_6000", op="topk_kd", T=6000, K=16, d=1024, V=151936, k=64, dtype="bf16", masked=0.1, beta=0.1,
             renormalize=False, conf="given", run_off=True),
        # a small step: one gradient-accumulation slice
        dict(name="topk_kd_512", op="topk_kd", T=512, K=8, d=2048, V=128256, k=8, dtype="bf16", masked=0.1, beta=0.0,
             renormalize=True, conf="given", run_off=False),
        # the small fp32 head
        dict(name="topk_kd_f32_512", op="topk_kd", T=512, K=8, d=256, V=4096, k=8, dtype="f32", masked=0.1, beta=0.5,
             renormalize=True, conf="own", run_off=False),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["logprob", "logprob", "logprob_bwd", "topk_kd"])
    f32 = rng.random() < 0.2
    most = 2.0 * 512 * 256 * 4096 if f32 else dict(logprob=8192, logprob_bwd=4096, topk_kd=16384)[op] * 2048.0 * 128256
    while True:
        d = 8 * spread(8, 64) if f32 else 8 * spread(16, 512)
        V = spread(500, 8192) if f32 else spread(2000, 160000)
        T = spread(1, 2048) if f32 else spread(1, 16384)
        if T * float(d) * V <= most:
            break
    c = dict(op=op, T=T, d=d, V=V, dtype="f32" if f32 else "bf16", masked=rng.choice([0.0, 0.1, 0.3]))
    if op == "logprob":
        c.update(top_k=rng.choice([0, 1, spread(2, 64), 20]), labels=rng.random() < 0.8)
    elif op == "logprob_bwd":
        c.update(entropy=rng.random() < 0.6)
    else:
        K = rng.choice([1, 4, 5, 8, 16, 32])
        c.update(T=max(1, T // K) * K, K=K, k=spread(1, 64), beta=rng.choice([0.0, 0.1, 1.0]), renormalize=rng.random() < 0.5,
                 conf=rng.choice(["own", "given"]), run_off=rng.random() < 0.4)
    return c


def _towards(H, W, token, amount):
    """Raises the logit of `token` by `amount` in each row of H, as a trained model that is sure of it does."""
    Wy = W[token].float()
    return H + Wy * (amount / (Wy * Wy).sum(1).clamp(min=1e-6)).unsqueeze(1)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    T, d, V, dt = case["T"], case["d"], case["V"], DTYPES[case["dtype"]]

    def rand(*shape):
        return torch.rand(*shape, generator=g, device=dev)

    W = (0.02 * torch.randn(V, d, generator=g, device=dev)).to(dt)
    H = torch.randn(T, d, generator=g, device=dev)
    labels = torch.randint(0, V, (T,), generator=g, device=dev)
    s = dict(case=dict(case), W=W)
    if case["op"] == "topk_kd":
        K, k = case["K"], case["k"]
        nb = T // K
        L = max(1, nb + K - 1 - (K // 2 + 1 if case["run_off"] else 0))
        start = torch.arange(nb, device=dev)
        # the teacher's stored lists: its k most likely tokens at each position, a quarter of them cut short
        sure = torch.randint(0, V, (L,), generator=g, device=dev)
        Ht = _towards(torch.randn(L, d, generator=g, device=dev), W, sure, 10.0 * rand(L))
        zt = (Ht.to(dt) @ W.T).float()
        top = zt.topk(min(k, V), dim=1)
        ids, logp = top.indices, top.values - torch.logsumexp(zt, 1, keepdim=True)
        if k > V:
            ids = torch.nn.functional.pad(ids, (0, k - V), value=-1)
            logp = torch.nn.functional.pad(logp, (0, k - V), value=-math.inf)
        keep = torch.where(rand(L) < 0.25, torch.ceil(k * rand(L)), torch.full((L,), float(k), device=dev)).clamp(min=1)
        cut = torch.arange(k, device=dev) >= keep.unsqueeze(1)
        s["top_ids"] = ids.masked_fill(cut, -1).contiguous()
        s["top_logp"] = logp.masked_fill(cut, -math.inf).contiguous()
        pos = (start.unsqueeze(1) + torch.arange(K, device=dev)).reshape(-1).clamp(max=L - 1)
        mostly = rand(T) < 0.7
        labels = torch.where(mostly, ids[pos, 0].clamp(min=0), labels)
        H = _towards(H, W, ids[pos, 0].clamp(min=0), 8.0 * rand(T) * (rand(T) < 0.6))
        s["start"] = start
        s["conf"] = rand(T).sqrt() if case["conf"] == "given" else None
    else:
        H = _towards(H, W, labels, (6.0 + 8.0 * rand(T)) * (rand(T) < 0.5))
    s["H"] = H.to(dt)
    off = rand(T) < case["masked"]
    s["valid"] = (~off).to(torch.uint8) if case["masked"] > 0 else None
    s["labels"] = torch.where(off, torch.full_like(labels, -100), labels) if case.get("labels", True) else None
    if case["op"] == "logprob_bwd":
        # what the forward pass of the step has left: log-sum-exp and entropy of each row, and the upstream gradients
        lse, entropy, _ = _statistics(_logits(s["H"], W))
        s["lse"], s["entropy"] = lse, entropy
        s["grad_logp"] = torch.randn(T, generator=g, device=dev) / T
        s["grad_entropy"] = (0.01 * torch.randn(T, generator=g, device=dev) - 0.05) / T if case["entropy"] else None
    if own:
        from paper_2605_08632_b200.api import CatLoss, TokenLogProb
        if case["op"] == "topk_kd":
            s["engine"] = CatLoss(T, d, V, case["K"], dtype=dt, dW_dtype=dt)
        else:
            s["engine"] = TokenLogProb(T, d, V, top_k=case.get("top_k", 0), dtype=dt, dW_dtype=dt)
    return s


def run(s):
    return {"logprob": _logprob, "logprob_bwd": _logprob_bwd, "topk_kd": _topk_kd}[s["case"]["op"]](s)


# ---------------------------------------------------------------------------- plain forms
def _logits(H, W):
    return H.float() @ W.float().T


def _statistics(z):
    """log-sum-exp and entropy of each row's softmax, and the softmax numerators' sum relative to the maximum."""
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1)
    return m.squeeze(1) + total.log(), total.log() - (e * (z - m)).sum(1) / total, total


def _logprob(s):
    c, H, W, labels, valid = s["case"], s["H"], s["W"], s["labels"], s["valid"]
    if own:
        r = s["engine"].forward(H, W, labels, valid)
        return {"logp": r.logp, "lse": r.lse, "entropy": r.entropy, "top_ids": r.top_ids, "top_logp": r.top_logp}
    T, V, k = c["T"], c["V"], c["top_k"]
    ok = valid.bool() if valid is not None else torch.ones(T, dtype=torch.bool, device=H.device)
    z = _logits(H, W)
    lse, entropy, _ = _statistics(z)
    logp = None
    if labels is not None:
        known = ok & (labels >= 0) & (labels < V)
        logp = torch.where(known, z.gather(1, labels.clamp(0, V - 1).unsqueeze(1)).squeeze(1) - lse, 0.0)
    top_ids = top_logp = None
    if k > 0:
        # a few more than k by their fp32 logits, then in order of their logits in 64 bits, ties to the lower index
        cand = z.topk(min(k + 8, V), dim=1).indices.sort(1).values
        zc = (W[cand].double() @ H.double().unsqueeze(2)).squeeze(2)
        zc, order = zc.sort(dim=1, descending=True, stable=True)
        n = min(k, V)
        top_ids = torch.full((T, k), -1, dtype=torch.int64, device=H.device)
        top_logp = torch.full((T, k), -math.inf, device=H.device)
        top_ids[:, :n] = torch.where(ok.unsqueeze(1), cand.gather(1, order)[:, :n], -1)
        top_logp[:, :n] = torch.where(ok.unsqueeze(1), zc[:, :n].float() - lse.unsqueeze(1), -math.inf)
    return {"logp": logp, "lse": torch.where(ok, lse, 0.0), "entropy": torch.where(ok, entropy, 0.0), "top_ids": top_ids, "top_logp": top_logp}


def _logprob_bwd(s):
    c, H, W, labels, valid = s["case"], s["H"], s["W"], s["labels"], s["valid"]
    if own:
        dH, dW = s["engine"].backward(H, W, labels, valid, s["grad_logp"], s["grad_entropy"], lse=s["lse"], entropy=s["entropy"])
        return {"dH": dH, "dW": dW}
    V = c["V"]
    ok = valid.bool() if valid is not None else torch.ones(c["T"], dtype=torch.bool, device=H.device)
    known = ok & (labels >= 0) & (labels < V)
    gl = torch.where(known, s["grad_logp"], 0.0).unsqueeze(1)
    logp = _logits(H, W) - s["lse"].unsqueeze(1)
    coef = -gl
    if s["grad_entropy"] is not None:
        ge = torch.where(ok, s["grad_entropy"], 0.0).unsqueeze(1)
        coef = coef - ge * (logp + s["entropy"].unsqueeze(1))
    dz = torch.exp(logp) * coef
    dz.scatter_add_(1, labels.clamp(0, V - 1).unsqueeze(1), gl)
    return {"dH": (dz @ W.float()).to(H.dtype), "dW": (dz.T @ H.float()).to(W.dtype)}


def _topk_kd(s):
    c, H, W, labels, valid = s["case"], s["H"], s["W"], s["labels"], s["valid"]
    if own:
        e = s["engine"]
        loss3, dH, dW = e.topk_kd_forward_backward(H, W, labels, valid, s["top_ids"], s["top_logp"], s["start"], beta=c["beta"],
                                                   renormalize=c["renormalize"], conf_ext=s["conf"])
        return {"loss": loss3, "lse": e.lse, "conf": e.conf, "weight": e.weight, "dH": dH, "dW": dW}
    T, K, V, beta = c["T"], c["K"], c["V"], c["beta"]
    L = s["top_ids"].shape[0]
    pos = (s["start"].unsqueeze(1) + torch.arange(K, device=H.device)).reshape(-1)
    ok = (labels >= 0) & (labels < V) & (pos >= 0) & (pos < L)
    if valid is not None:
        ok = ok & valid.bool()
    pos, y = pos.clamp(0, L - 1), labels.clamp(0, V - 1).unsqueeze(1)
    ids, t = s["top_ids"][pos], s["top_logp"][pos]
    there = (ids >= 0) & (ids < V) & (t > -math.inf)
    t = torch.where(there, t, -math.inf)
    if c["renormalize"]:
        t = t - torch.where(there.any(1), torch.logsumexp(t, 1), 0.0).unsqueeze(1)
    p = torch.exp(t)
    mass = p.sum(1)
    z = _logits(H, W)
    lse, _, _ = _statistics(z)
    logq = z - lse.unsqueeze(1)
    ce = -logq.gather(1, y).squeeze(1)
    kd = torch.where(there, p * (t - logq.gather(1, ids.clamp(0, V - 1))), 0.0).sum(1)
    conf = torch.where(ok, s["conf"] if s["conf"] is not None else torch.exp(-ce), 1.0)
    before = torch.nn.functional.pad(conf.view(-1, K)[:, : K - 1], (1, 0), value=1.0)
    weight = torch.where(ok, before.cumprod(1).reshape(-1), 0.0)
    n = ok.sum().clamp(min=1)
    loss_ce = (weight * ce).double().sum() / n
    loss_kd = (weight * kd).double().sum() / n
    dz = torch.exp(logq) * (beta + mass).unsqueeze(1)
    dz.scatter_add_(1, y, torch.full_like(ce, -beta).unsqueeze(1))
    dz.scatter_add_(1, ids.clamp(0, V - 1), -p)
    dz *= (weight / n).unsqueeze(1)
    dH = torch.where(ok.unsqueeze(1), dz @ W.float(), 0.0).to(H.dtype)
    return {"loss": torch.stack([beta * loss_ce + loss_kd, loss_ce, loss_kd]).float(), "lse": lse, "conf": conf, "weight": weight,
            "dH": dH, "dW": (dz.T @ H.float()).to(W.dtype)}


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    T, d, V = float(case["T"]), float(case["d"]), float(case["V"])
    b = 2.0 if case["dtype"] == "bf16" else 4.0
    heads = (T + V) * d * b                     # hidden states and head weight, or their gradients
    if case["op"] == "logprob":                 # one product of H and W; lists and row values out
        return {"bytes": heads + T * (12 * case["top_k"] + 21), "flops": 2 * T * d * V}
    if case["op"] == "logprob_bwd":             # logits are not kept by the forward pass: one product for them, two for the gradients
        return {"bytes": 2 * heads + T * 25, "flops": 6 * T * d * V}
    return {"bytes": 2 * heads + T * (12 * case["k"] / case["K"] + 25), "flops": 6 * T * d * V}


# ---------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    s.pop("engine", None)
    T, V = case["T"], case["V"]
    Wd, dev = s["W"].double(), s["W"].device
    valid = s["valid"].bool() if s["valid"] is not None else torch.ones(T, dtype=torch.bool, device=dev)
    labels = s["labels"] if s["labels"] is not None else torch.full((T,), -1, device=dev)
    named = (labels >= 0) & (labels < V)
    rows = max(1, min(T, (1 << 28) // V))
    chunks = [slice(i, min(T, i + rows)) for i in range(0, T, rows)]
    if case["op"] == "logprob":
        k = case["top_k"]
        out = dict(logp=torch.zeros(T, dtype=torch.float64, device=dev), lse=torch.zeros(T, dtype=torch.float64, device=dev),
                   entropy=torch.zeros(T, dtype=torch.float64, device=dev))
        tops = torch.full((T, k), -math.inf, dtype=torch.float64, device=dev)
        for c in chunks:
            lp = torch.log_softmax(s["H"][c].double() @ Wd.T, 1)
            z0 = s["H"][c].double() @ Wd[0]
            on = valid[c].double()
            out["lse"][c] = on * (z0 - lp[:, 0])
            out["entropy"][c] = on * -(lp.exp() * lp).sum(1)
            pick = lp.gather(1, labels[c].clamp(0, V - 1).unsqueeze(1)).squeeze(1)
            out["logp"][c] = torch.where(valid[c] & named[c], pick, 0.0)
            if k > 0:
                best = lp.topk(min(k, V), 1).values
                tops[c, : best.shape[1]] = torch.where(valid[c].unsqueeze(1), best, -math.inf)
        return {"logp": out["logp"] if s["labels"] is not None else None, "lse": out["lse"], "entropy": out["entropy"], "top_ids": None,
                "top_logp": tops if k > 0 else None}
    dH = torch.zeros(T, case["d"], dtype=torch.float64, device=dev)
    dW = torch.zeros(V, case["d"], dtype=torch.float64, device=dev)
    if case["op"] == "logprob_bwd":
        for c in chunks:
            lp = torch.log_softmax(s["H"][c].double() @ Wd.T, 1)
            p = lp.exp()
            gl = torch.where(valid[c] & named[c], s["grad_logp"][c].double(), 0.0)
            dz = -gl.unsqueeze(1) * p
            dz[torch.arange(dz.shape[0], device=dev), labels[c].clamp(0, V - 1)] += gl
            if s["grad_entropy"] is not None:
                ent = -(p * lp).sum(1, keepdim=True)
                dz -= torch.where(valid[c], s["grad_entropy"][c].double(), 0.0).unsqueeze(1) * p * (lp + ent)
            dH[c] = dz @ Wd
            dW += dz.T @ s["H"][c].double()
        return {"dH": dH, "dW": dW}
    K, k, L, beta = case["K"], case["k"], s["top_ids"].shape[0], case["beta"]
    row = torch.arange(T, device=dev)
    pos = s["start"][row // K] + row % K
    ok = valid & named & (pos >= 0) & (pos < L)
    n = max(1, int(ok.sum()))
    lse, ce, kd = (torch.zeros(T, dtype=torch.float64, device=dev) for _ in range(3))

    def teacher(c):
        at = pos[c].clamp(0, L - 1)
        ids, t = s["top_ids"][at], s["top_logp"][at].double()
        there = (ids >= 0) & (ids < V) & torch.isfinite(t)
        p = torch.where(there, t.exp(), 0.0)
        if case["renormalize"]:
            p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
        return ids.clamp(0, V - 1), p

    for c in chunks:
        lp = torch.log_softmax(s["H"][c].double() @ Wd.T, 1)
        lse[c] = s["H"][c].double() @ Wd[0] - lp[:, 0]
        ce[c] = -lp.gather(1, labels[c].clamp(0, V - 1).unsqueeze(1)).squeeze(1)
        ids, p = teacher(c)
        kd[c] = (torch.special.xlogy(p, p) - p * lp.gather(1, ids)).sum(1)
    conf = torch.where(ok, s["conf"].double() if s["conf"] is not None else torch.exp(-ce), 1.0)
    weight = torch.ones(T // K, K, dtype=torch.float64, device=dev)
    for j in range(1, K):
        weight[:, j] = weight[:, j - 1] * conf.view(-1, K)[:, j - 1]
    weight = torch.where(ok, weight.reshape(-1), 0.0)
    for c in chunks:
        q = torch.softmax(s["H"][c].double() @ Wd.T, 1)
        ids, p = teacher(c)
        dz = (beta + p.sum(1, keepdim=True)) * q
        dz.scatter_add_(1, labels[c].clamp(0, V - 1).unsqueeze(1), torch.full((dz.shape[0], 1), -beta, dtype=torch.float64, device=dev))
        dz.scatter_add_(1, ids, -p)
        dz *= (weight[c] / n).unsqueeze(1)
        dH[c] = dz @ Wd
        dW += dz.T @ s["H"][c].double()
    a, b = (weight * ce).sum() / n, (weight * kd).sum() / n
    return {"loss": torch.stack([beta * a + b, a, b]), "lse": lse, "conf": conf, "weight": weight, "dH": dH, "dW": dW}
