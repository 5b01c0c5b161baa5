"""The training losses of a large-vocabulary head, as they are measured: cases, plain forms and 64-bit references.

Two operators, each with its gradient.  Both start from activations x (T x d) and a head weight W (V x d) and never
return the logits z = x W^T + b:

  xent     loss_t = logsumexp_v z_tv - z_t,target(t); rows whose target is ignore_index or outside the vocabulary are left
           out: their loss, logsumexp and gradient are 0
  distill  loss_t = tau^2 * sum_j p_tj (log p_tj - log q_t,index(t,j)), p = softmax over the teacher's listed logits / tau,
           q = softmax over the whole vocabulary of z / tau; entries whose index is outside the vocabulary are left out, and so are
           rows with no entry

A case has "op", "pass" ("fwd": loss and logsumexp; "train": those and dx, dW and, with a bias, db for given dloss),
"dtype", the sizes T, d, V, whether there is a bias, and for distill K (listed teacher logits per token) and tau.
"""
import math

import torch

own = False

IGNORE = -100
LARGEST = 8192 * 2048 * 50021          # T * d * V of the largest listed case


def _case(name, op, pas, dtype, T, d, V, bias=False, K=0, tau=1.0):
    return {"name": name, "op": op, "pass": pas, "dtype": dtype, "T": T, "d": d, "V": V, "bias": bias, "K": K, "tau": tau}


def listed():
    return [
        # scoring a short text over a small class list: latency
        _case("xent-fwd-16x512x1000", "xent", "fwd", "bf16", 16, 512, 1000),
        # scoring a single token over a large vocabulary: the weight is read once
        _case("xent-fwd-1x1024x65536", "xent", "fwd", "bf16", 1, 1024, 65536),
        # evaluating a long text over a very large vocabulary
        _case("xent-fwd-8192x1024x131072", "xent", "fwd", "bf16", 8192, 1024, 131072),
        # a step of a fp32 classifier over a thousand classes
        _case("xent-train-f32-1024x512x1000", "xent", "train", "f32", 1024, 512, 1000, bias=True),
        # a ragged micro-batch, odd vocabulary, with a bias
        _case("xent-train-333x768x10007", "xent", "train", "bf16", 333, 768, 10007, bias=True),
        # an ordinary training step
        _case("xent-train-4096x1024x32768", "xent", "train", "bf16", 4096, 1024, 32768),
        # a large training step, odd vocabulary
        _case("xent-train-8192x2048x50021", "xent", "train", "bf16", 8192, 2048, 50021),
        # distillation loss of a short batch over a class list (validation)
        _case("distill-fwd-64x768x1000", "distill", "fwd", "bf16", 64, 768, 1000, K=16, tau=2.0),
        # a fp32 distillation step with odd sizes everywhere (rows that are not a multiple of 16 bytes)
        _case("distill-train-f32-777x501x4999", "distill", "train", "f32", 777, 501, 4999, bias=True, K=100, tau=1.5),
        # an ordinary distillation step
        _case("distill-train-2048x1024x32768", "distill", "train", "bf16", 2048, 1024, 32768, K=64, tau=2.0),
        # a large distillation step with many teacher logits
        _case("distill-train-4096x2048x65536", "distill", "train", "bf16", 4096, 2048, 65536, K=128, tau=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["xent", "distill"])
    pas = rng.choice(["fwd", "train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    while True:
        T, d, V = _log_int(rng, 1, 8192), _log_int(rng, 64, 2048), _log_int(rng, 200, 131072)
        if rng.random() < 0.5:
            d = -(-d // 64) * 64
        if T * d * V <= LARGEST // (2 if dtype == "f32" else 1):
            break
    distill = op == "distill"
    return {"op": op, "pass": pas, "dtype": dtype, "T": T, "d": d, "V": V, "bias": rng.random() < 0.3,
            "K": _log_int(rng, 1, 128) if distill else 0, "tau": rng.choice([1.0, 1.5, 2.0, 4.0]) if distill else 1.0}


def prepare(case, seed):
    """Inputs on the GPU: unit-variance activations, weights that give logits of a few units, a skewed distribution of
    targets, about one token in ten ignored; teacher logits in falling order with the tail entries of some rows left out."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, d, V, K = case["T"], case["d"], case["V"], case["K"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    s = {"op": case["op"], "pass": case["pass"], "tau": case["tau"]}
    s["x"] = normal(T, d).to(dt)
    s["w"] = (normal(V, d) * (2.0 / math.sqrt(d))).to(dt)
    s["bias"] = normal(V) * 0.5 if case["bias"] else None
    kept = uniform(T) < 0.9
    if T < 8:
        kept[:] = True
    if case["op"] == "xent":
        target = (uniform(T) ** 4 * V).to(torch.int64).clamp_(max=V - 1)
        s["target"] = torch.where(kept, target, torch.full_like(target, IGNORE))
    else:
        # K distinct indices of a row: increasing steps from a random start, in random order
        K = min(K, V)
        step = 1 + (uniform(T, K) * (V // K)).to(torch.int64).clamp_(max=max(V // K - 1, 0))
        index = ((uniform(T, 1) * V).to(torch.int64) + step.cumsum(1)) % V
        index = index.gather(1, uniform(T, K).argsort(1))
        logit = (normal(T, K) * 3.0).sort(1, descending=True).values
        count = 1 + (uniform(T, 1) * 4 * K).to(torch.int64)                  # three rows in four are full
        index = torch.where(torch.arange(K, device="cuda")[None, :] < count, index, torch.full_like(index, -1))
        s["index"] = torch.where(kept[:, None], index, torch.full_like(index, -1))
        s["logit"] = logit
    s["dloss"] = (0.5 + uniform(T)) / T
    return s


def run(s):
    if own:
        from paper_2407_12075_b200 import binding as tbn
        if s["op"] == "xent":
            loss, lse = tbn.tbn_linear_xent_fwd(s["x"], s["w"], s["target"], bias=s["bias"], ignore_index=IGNORE)
            if s["pass"] == "fwd":
                return {"loss": loss, "lse": lse}
            dx, dw, db = tbn.tbn_linear_xent_bwd(s["x"], s["w"], s["target"], lse, s["dloss"], bias=s["bias"], ignore_index=IGNORE,
                                                 need_dbias=s["bias"] is not None)
        else:
            loss, lse = tbn.tbn_linear_distill_fwd(s["x"], s["w"], s["index"], s["logit"], temperature=s["tau"], bias=s["bias"])
            if s["pass"] == "fwd":
                return {"loss": loss, "lse": lse}
            dx, dw, db = tbn.tbn_linear_distill_bwd(s["x"], s["w"], s["index"], s["logit"], lse, s["dloss"], temperature=s["tau"],
                                                    bias=s["bias"], need_dbias=s["bias"] is not None)
        out = {"loss": loss, "lse": lse, "dx": dx, "dw": dw}
        if db is not None:
            out["db"] = db
        return out

    x, w, tau = s["x"].float(), s["w"].float(), s["tau"]
    V = w.shape[0]
    z = x @ w.t()
    if s["bias"] is not None:
        z += s["bias"]
    z /= tau
    top = z.max(1, keepdim=True).values
    e = (z - top).exp_()
    total = e.sum(1, keepdim=True)
    lse = (top + total.log())[:, 0]
    if s["op"] == "xent":
        index, p = s["target"][:, None], None
        valid = (index >= 0) & (index < V)
        at = torch.where(valid, index, torch.zeros_like(index))
        p = valid.float()
        loss = torch.where(valid[:, 0], lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    else:
        valid = (s["index"] >= 0) & (s["index"] < V)
        at = torch.where(valid, s["index"], torch.zeros_like(s["index"]))
        t = torch.where(valid, s["logit"] / tau, torch.full_like(s["logit"], -math.inf))
        some = valid.any(1, keepdim=True)
        t_top = torch.where(some, t.max(1, keepdim=True).values, torch.zeros_like(lse[:, None]))
        t_exp = (t - t_top).exp()
        t_sum = torch.where(some, t_exp.sum(1, keepdim=True), torch.ones_like(t_top))
        p = t_exp / t_sum
        log_ratio = torch.where(valid, t - t_top - t_sum.log() - (z.gather(1, at) - lse[:, None]), torch.zeros_like(t))
        loss = tau * tau * (p * log_ratio).sum(1)
    live = valid.any(1, keepdim=True)
    lse = torch.where(live[:, 0], lse, torch.zeros_like(lse))
    if s["pass"] == "fwd":
        return {"loss": loss, "lse": lse}
    dz = torch.where(live, e / total, torch.zeros_like(e[:, :1]))
    del z, e
    dz.scatter_add_(1, at, -p)
    dz *= s["dloss"][:, None] * tau
    out = {"loss": loss, "lse": lse, "dx": (dz @ w).to(s["x"].dtype), "dw": (dz.t() @ x).to(s["w"].dtype)}
    if s["bias"] is not None:
        out["db"] = dz.sum(0)
    return out


def work(case):
    """Each input once, each output once; the three products of a step (logits, dx, dW), one of a forward pass."""
    T, d, V, K = case["T"], case["d"], case["V"], case["K"]
    size = 2 if case["dtype"] == "bf16" else 4
    labels = T * 8 if case["op"] == "xent" else T * K * 12
    data = (T + V) * d * size + (4 * V if case["bias"] else 0)
    total = data + labels + 8 * T
    if case["pass"] == "train":
        total += data + 4 * T
    return {"bytes": total, "flops": (6 if case["pass"] == "train" else 2) * T * d * V}


def exact(case, seed):
    """The definitions in 64 bits, in blocks of tokens."""
    s = prepare(case, seed)
    V, d, T, tau = case["V"], case["d"], case["T"], case["tau"]
    x, w, g = s["x"].double(), s["w"].double(), s["dloss"].double()
    b = s["bias"].double() if s["bias"] is not None else torch.zeros(V, dtype=torch.float64, device="cuda")
    loss, lse = torch.zeros(T, dtype=torch.float64, device="cuda"), torch.zeros(T, dtype=torch.float64, device="cuda")
    dx = torch.zeros(T, d, dtype=torch.float64, device="cuda")
    dw = torch.zeros(V, d, dtype=torch.float64, device="cuda")
    db = torch.zeros(V, dtype=torch.float64, device="cuda")
    step = max(1, min(T, (1 << 28) // V))
    for t0 in range(0, T, step):
        rows = slice(t0, min(T, t0 + step))
        logq = torch.log_softmax(torch.addmm(b, x[rows], w.t()) / tau, dim=1)
        lse[rows] = torch.logsumexp(torch.addmm(b, x[rows], w.t()) / tau, dim=1)
        teacher = torch.zeros_like(logq)
        if case["op"] == "xent":
            label = s["target"][rows]
            here = ((label >= 0) & (label < V)).nonzero()[:, 0]
            teacher[here, label[here]] = 1.0
            loss[rows] = -(teacher * logq).sum(1)
        else:
            index = s["index"][rows]
            r, j = ((index >= 0) & (index < V)).nonzero(as_tuple=True)
            listed_logits = torch.full_like(logq, -math.inf)
            listed_logits[r, index[r, j]] = s["logit"][rows][r, j].double() / tau
            full = torch.isfinite(listed_logits).any(1)
            teacher[full] = torch.softmax(listed_logits[full], dim=1)
            loss[rows] = tau * tau * (torch.special.xlogy(teacher, teacher) - teacher * logq).sum(1)
        lse[rows] *= teacher.sum(1) > 0.5
        if case["pass"] == "train":
            dz = (logq.exp() * teacher.sum(1, keepdim=True) - teacher) * (tau * g[rows])[:, None]
            dx[rows] = dz @ w
            dw += dz.t() @ x[rows]
            db += dz.sum(0)
    if case["pass"] == "fwd":
        return {"loss": loss, "lse": lse}
    out = {"loss": loss, "lse": lse, "dx": dx, "dw": dw}
    if case["bias"]:
        out["db"] = db
    return out
