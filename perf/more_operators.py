"""What a training step needs around a tiled head, as it is measured: cases, plain forms and 64-bit references.

Three operators:

  norm   LayerNorm of s = x + residual (rounded to x's type) with its statistics, and the gradient: dx (which is also the
         residual's), dgamma and dbeta; a gradient that reaches s past the norm (dsum) is added to dx
  embed  rows of a table, scaled, for token ids (ids outside the vocabulary give zeros), and the table's gradient: the sums of
         the rows of dy that share an id, as a whole table or added to the gradient that is already there (a tied head's);
         the table is a matrix, or a tiled one: bits and scaling factors
  adamw  one AdamW step over many tensors, states in 32 bits or in 8; with "clip", gradients scaled by their global norm

States in 8 bits: blocks of 256 elements of a tensor have one scale each for m and v, taken from the block's largest magnitude.
m = c |c| scale with c in -127..127, v = c^4 scale with c in 0..254.  The code is the one below or the one above, at random so
that the mean is the value: the random number of element j of tensor i comes from the seed, the step, i and j.
"""
import math

import torch

own = False

B1, B2, EPS, LR = 0.9, 0.95, 1e-8, 1e-3
BLOCK = 256
M_TOP, V_TOP = 127.0 ** 2, 254.0 ** 4          # largest code, as the value that it stands for in units of the scale
M_LEAST, V_LEAST = 2.0 ** -100, 2.0 ** -94     # no block's largest magnitude counts as less
MOST_BYTES = 4e9                               # of a drawn case


def _norm(name, pas, dtype, T, d, residual=False):
    return {"name": name, "op": "norm", "pass": pas, "dtype": dtype, "T": T, "d": d, "residual": residual}


def _embed(name, pas, dtype, T, d, V, k=0, add=False):
    return {"name": name, "op": "embed", "pass": pas, "dtype": dtype, "T": T, "d": d, "V": V, "k": k, "add": add}


def _adamw(name, bits, p, g, layers, d, odd=0, V=0, copy=False, clip=False):
    return {"name": name, "op": "adamw", "bits": bits, "p": p, "g": g, "layers": layers, "d": d, "odd": odd, "V": V, "copy": copy, "clip": clip}


def listed():
    return [
        # the last norm of a short prompt's step: latency
        _norm("norm-train-16x512", "train", "bf16", 16, 512),
        # the second norm of an encoder block over 128 images of 197 tokens, residual stream updated on the way (evaluation)
        _norm("norm-fwd-25216x768", "fwd", "bf16", 25216, 768, residual=True),
        # fp32 training with odd sizes (rows that are not a multiple of 16 bytes)
        _norm("norm-train-f32-777x501", "train", "f32", 777, 501, residual=True),
        # an ordinary training step of a wide model
        _norm("norm-train-8192x2048", "train", "bf16", 8192, 2048, residual=True),
        # a single token's row
        _embed("embed-fwd-1x1024x65536", "fwd", "bf16", 1, 1024, 65536),
        # a long prompt over a tiled table
        _embed("embed-tiled-fwd-8192x1024x32768", "fwd", "bf16", 8192, 1024, 32768, k=4),
        # an ordinary step with a tied head, whose gradient the embedding's is added to
        _embed("embed-train-add-4096x1024x32768", "train", "bf16", 4096, 1024, 32768, add=True),
        # a large step over an odd vocabulary, the gradient as a whole table
        _embed("embed-train-16384x2048x50021", "train", "bf16", 16384, 2048, 50021),
        # the gains and offsets of one norm: latency
        _adamw("adamw32-2x768", 32, "f32", "f32", 0, 768),
        # an ordinary fp32 model with a head, and a bf16 copy for the next forward pass
        _adamw("adamw32-8x1024x32768", 32, "f32", "f32", 8, 1024, V=32768, copy=True),
        # odd widths, bf16 parameters and gradients, states in 8 bits, clipped
        _adamw("adamw8-clip-6x501x4999", 8, "bf16", "bf16", 6, 501, odd=3, V=4999, clip=True),
        # a large model with states in 8 bits, bf16 gradients, clipped
        _adamw("adamw8-clip-4x2048", 8, "f32", "bf16", 4, 2048, clip=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "embed", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pas = rng.choice(["fwd", "train", "train"])
    while True:
        if op == "norm":
            case = _norm("", pas, dtype, _log_int(rng, 1, 32768), _log_int(rng, 32, 8192), residual=rng.random() < 0.5)
        elif op == "embed":
            tiled = pas == "fwd" and rng.random() < 0.5
            case = _embed("", pas, dtype, _log_int(rng, 1, 32768), _log_int(rng, 32, 2048), _log_int(rng, 100, 131072),
                          k=rng.choice([2, 4, 8]) if tiled else 0, add=pas == "train" and rng.random() < 0.5)
        else:
            p = rng.choice(["f32", "f32", "bf16"])
            case = _adamw("", rng.choice([32, 8]), p, rng.choice(["f32", "bf16"]), rng.randint(0, 8), _log_int(rng, 32, 2048),
                          odd=rng.choice([0, 0, 1, 3]), V=rng.choice([0, _log_int(rng, 100, 65536)]), copy=p == "f32" and rng.random() < 0.3,
                          clip=rng.random() < 0.5)
        if op != "adamw" and rng.random() < 0.6:
            case["d"] = -(-case["d"] // 32) * 32
        if case.get("k"):
            case["V"] = -(-case["V"] // 8) * 8
        if work(case)["bytes"] <= MOST_BYTES:
            del case["name"]
            return case


def _sizes(case):
    """Elements and weight decay of each tensor: per layer four projections, a feed-forward pair and two norms; a head and the last norm."""
    d, odd = case["d"], case["odd"]
    sizes = []
    for _ in range(case["layers"]):
        sizes += [(d * d + odd, 0.1)] * 4 + [(4 * d * d, 0.1)] * 2 + [(d, 0.0)] * 4
    if case["V"]:
        sizes.append((case["V"] * d, 0.1))
    return sizes + [(d, 0.0)] * 2


def _places(case):
    """(first element, elements, first block, blocks, weight decay) of each tensor in the flat buffers."""
    at = block = 0
    places = []
    for n, decay in _sizes(case):
        blocks = -(-n // BLOCK)
        places.append((at, n, block, blocks, decay))
        at += -(-n // 64) * 64                    # tensors begin on a line, as allocators have it
        block += blocks
    return places, at, block


def _mix(x):
    """32 bits to 32 bits; integers or int64 tensors."""
    x = x & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def prepare(case, seed):
    """Inputs on the GPU: activations of a few units with a few large columns, ids with a skewed distribution and some padding,
    gradients of the size that a mean over tokens gives, states as they are after some steps."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    s = {"case": case, "op": case["op"]}
    if case["op"] == "norm":
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        T, d = case["T"], case["d"]
        columns = 1.0 + 4.0 * (uniform(d) < 0.01) + 0.5 * normal(d)
        s["x"] = (normal(T, d) * columns + 0.3).to(dt)
        s["residual"] = normal(T, d).to(dt) if case["residual"] else None
        s["gamma"], s["beta"] = 1.0 + 0.1 * normal(d), 0.1 * normal(d)
        s["dy"] = (normal(T, d) / T).to(dt)
        s["dsum"] = (normal(T, d) / T).to(dt) if case["residual"] else None
    elif case["op"] == "embed":
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        T, d, V = case["T"], case["d"], case["V"]
        ids = (uniform(T) ** 4 * V).to(torch.int64).clamp_(max=V - 1)
        s["ids"] = torch.where(uniform(T) < 0.95, ids, torch.full_like(ids, -1)) if T >= 8 else ids
        s["scale"] = math.sqrt(d)
        s["out_dtype"] = dt
        if case["k"]:
            q = V * d // case["k"]
            words = -(-q // 128) * 4
            bits = torch.randint(-2 ** 31, 2 ** 31, (words,), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
            tail = torch.arange(words, device="cuda") * 32
            keep = (q - tail).clamp_(0, 32)
            s["tile"] = bits & ((torch.ones_like(keep) << keep) - 1).to(torch.int32)
            s["alpha"] = 0.02 * (0.5 + uniform(case["k"]))
        else:
            s["table"] = (normal(V, d) * 0.02).to(dt)
        s["dy"] = (normal(T, d) / T).to(dt)
        s["dw"] = normal(V, d) * (0.1 / T) if case["add"] else None
    else:
        kind = {"f32": torch.float32, "bf16": torch.bfloat16}
        places, n, blocks = _places(case)
        s["p"] = (normal(n) * 0.02).to(kind[case["p"]])
        s["g"] = (normal(n) * 1e-3 * (0.05 + uniform(n))).to(kind[case["g"]])
        s["copy"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda") if case["copy"] else None
        s["step"], s["seed"], s["max_norm"] = 1000, seed, 1.0
        if case["bits"] == 32:
            s["m"], s["v"] = normal(n) * 3e-4, (normal(n) * 1e-3).square_()
            s["ms"] = s["vs"] = None
        else:
            s["m"] = (normal(n) * 40.0).clamp_(-127, 127).to(torch.int8)
            s["v"] = (40.0 + 180.0 * uniform(n)).to(torch.uint8)
            s["ms"], s["vs"] = (0.5 + uniform(blocks)) * (1e-3 / M_TOP), (0.5 + uniform(blocks)) * (1e-6 / V_TOP)
            s["m_values"], s["v_values"] = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        cut = lambda name: None if s[name] is None else [s[name][a:a + m] for a, m, _, _, _ in places]  # noqa: E731
        scales = lambda name: None if s[name] is None else [s[name][b:b + m] for _, _, b, m, _ in places]  # noqa: E731
        s["tensors"] = {"params": cut("p"), "grads": cut("g"), "m": cut("m"), "v": cut("v"), "m_scale": scales("ms"), "v_scale": scales("vs"),
                        "copies": cut("copy"), "weight_decay": [decay for _, _, _, _, decay in places]}
        if case["bits"] == 8:
            s["values"] = (cut("m_values"), cut("v_values"))
        # where each block lies: its first element in the buffers and in its tensor, its length, its tensor, what weight decay leaves
        first, size, _, count, decay = (torch.tensor(c, device="cuda") for c in zip(*places))
        spread = lambda c: c.repeat_interleave(count, output_size=blocks)  # noqa: E731
        inner = (torch.arange(blocks, device="cuda") - spread(count.cumsum(0) - count)) * BLOCK
        s["layout"] = {"start": spread(first) + inner, "first": inner, "length": (spread(size) - inner).clamp_(max=BLOCK),
                       "tensor": spread(torch.arange(len(places), device="cuda")),
                       "keep": spread(1 - LR * decay.double()).float()}
        s["handle"] = None
    return s


def _run_own(s):
    from paper_2407_12075_b200 import binding as tbn
    case = s["case"]
    if s["op"] == "norm":
        y, total, mean, rstd = tbn.tbn_layernorm_train_fwd(s["x"], s["gamma"], s["beta"], EPS, residual=s["residual"])
        out = {"y": y, "mean": mean, "rstd": rstd}
        if s["residual"] is not None:
            out["sum"] = total
        if case["pass"] == "train":
            out["dx"], out["dgamma"], out["dbeta"] = tbn.tbn_layernorm_bwd(s["dy"], total, mean, rstd, s["gamma"], dsum=s["dsum"])
        return out
    if s["op"] == "embed":
        if case["k"]:
            code = tbn.BF16 if s["out_dtype"] == torch.bfloat16 else tbn.F32
            return {"y": tbn.tbn_embedding_tiled_fwd(s["ids"], case["V"], case["d"], s["tile"], case["k"], s["alpha"], tbn.ALPHA_PER_TILE,
                                                     scale=s["scale"], y_dtype=code)}
        out = {"y": tbn.tbn_embedding_fwd(s["ids"], s["table"], scale=s["scale"])}
        if case["pass"] == "train":
            out["dw"] = tbn.tbn_embedding_bwd(s["ids"], s["dy"], case["V"], scale=s["scale"], add_to=s["dw"])
        return out
    if s["handle"] is None:                       # the table of tensors, which a program makes once
        s["handle"] = tbn.tbn_adamw_tensors(**s["tensors"])
    h = s["handle"]
    out = {"p": s["p"], "m": s["m"], "v": s["v"]}
    scale = None
    if case["clip"]:
        out["norm"], scale = tbn.tbn_grad_norm(h, s["max_norm"])
    tbn.tbn_adamw_step(h, s["step"], LR, B1, B2, EPS, grad_scale=scale, seed=s["seed"])
    if case["bits"] == 8:
        tbn.tbn_adamw_unpack(h, *s["values"])
        out.update(m=s["m_values"], v=s["v_values"], ms=s["ms"], vs=s["vs"])
    if case["copy"]:
        out["copy"] = s["copy"]
    return out


def _encode(y, u, power, top):
    """Codes c, c^power <= y or one more, the one above with the probability that makes the mean y; all in 32 bits."""
    raised = lambda c: c * c if power == 2 else (c * c) * (c * c)  # noqa: E731
    c = (y.sqrt() if power == 2 else y.sqrt().sqrt()).floor()
    c -= (raised(c) > y).float()
    c += (raised(c + 1) <= y).float()
    low = raised(c)
    c += (u * (raised(c + 1) - low) < y - low).float()
    return c.clamp_(max=top)


def _adamw_plain(s, scale):
    """One step of all tensors in 32 bits, as a matrix with a row of 256 elements for each block; a tensor's last row repeats its
    last element."""
    lay, step, eight = s["layout"], s["step"], s["ms"] is not None
    of = torch.minimum(torch.arange(BLOCK, device="cuda")[None, :], lay["length"][:, None] - 1)
    at = lay["start"][:, None] + of
    g, m, v = s["g"][at].float(), s["m"][at].float(), s["v"][at].float()
    if scale is not None:
        g *= scale
    if eight:
        m, v = (m * m.abs()) * s["ms"][:, None], ((v * v) * (v * v)) * s["vs"][:, None]
    m = m * B1 + g * (1 - B1)
    v = v * B2 + (g * (1 - B2)) * g
    bc1, bc2 = 1 - B1 ** step, 1 - B2 ** step
    new = s["p"][at].float() * lay["keep"][:, None] - (m * (LR / bc1)) / (v.sqrt() * (1 / math.sqrt(bc2)) + EPS)
    s["p"][at] = new.to(s["p"].dtype)
    if s["copy"] is not None:
        s["copy"][at] = new.to(torch.bfloat16)
    if not eight:
        s["m"][at], s["v"][at] = m, v
        return
    key = _mix(_mix(_mix(s["seed"] & 0xFFFFFFFF) ^ (step & 0xFFFFFFFF)) + lay["tensor"])
    h = _mix((lay["first"][:, None] + of) ^ key[:, None])
    top = m.abs().amax(1, keepdim=True).clamp_(min=M_LEAST)
    c = _encode(m.abs() * (torch.full_like(top, M_TOP) / top), ((h & 0xFFFF).float() + 0.5) * 2.0 ** -16, 2, 127.0)
    s["m"][at] = torch.where(m < 0, -c, c).to(torch.int8)
    s["ms"].copy_(top[:, 0] * (1 / M_TOP))
    top = v.amax(1, keepdim=True).clamp_(min=V_LEAST)
    c = _encode(v * (torch.full_like(top, V_TOP) / top), ((h >> 16).float() + 0.5) * 2.0 ** -16, 4, 254.0)
    s["v"][at] = torch.where(v > 0, c.clamp(min=1.0), c).to(torch.uint8)
    s["vs"].copy_(top[:, 0] * (1 / V_TOP))
    c = s["m"][at].float()
    s["m_values"][at] = (c * c.abs()) * s["ms"][:, None]
    c = s["v"][at].float()
    s["v_values"][at] = ((c * c) * (c * c)) * s["vs"][:, None]


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    if s["op"] == "norm":
        x, gamma, dt = s["x"].float(), s["gamma"], s["x"].dtype
        out = {}
        if s["residual"] is not None:
            out["sum"] = (x + s["residual"].float()).to(dt)
            x = out["sum"].float()
        mean = x.mean(1, keepdim=True)
        centred = x - mean
        rstd = (centred.square().mean(1, keepdim=True) + EPS).rsqrt()
        h = centred * rstd
        out.update(y=(h * gamma + s["beta"]).to(dt), mean=mean[:, 0], rstd=rstd[:, 0])
        if case["pass"] == "train":
            dy = s["dy"].float()
            a = dy * gamma
            dx = (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True)) * rstd
            if s["dsum"] is not None:
                dx += s["dsum"].float()
            out.update(dx=dx.to(dt), dgamma=(dy * h).sum(0), dbeta=dy.sum(0))
        return out
    if s["op"] == "embed":
        ids, V, d = s["ids"], case["V"], case["d"]
        valid = (ids >= 0) & (ids < V)
        at = torch.where(valid, ids, torch.zeros_like(ids))
        if case["k"]:
            flat = at[:, None] * d + torch.arange(d, device=ids.device)
            q = V * d // case["k"]
            i = flat % q
            bit = (s["tile"][i >> 5] >> (i & 31).to(torch.int32)) & 1
            rows = s["alpha"][flat // q] * (2.0 * bit - 1.0)
        else:
            rows = s["table"][at].float()
        out = {"y": torch.where(valid[:, None], rows * s["scale"], torch.zeros_like(rows)).to(s["out_dtype"])}
        if case["pass"] == "train":
            dy = torch.where(valid[:, None], s["dy"].float() * s["scale"], torch.zeros_like(rows))
            dw = s["dw"] if s["dw"] is not None else torch.zeros(V, d, device=ids.device)
            dw.index_add_(0, at, dy)
            out["dw"] = dw if s["dw"] is not None else dw.to(s["out_dtype"])
        return out
    out, scale = {}, None
    if case["clip"]:
        lay = s["layout"]
        at = lay["start"][:, None] + torch.arange(BLOCK, device="cuda")
        inside = torch.arange(BLOCK, device="cuda") < lay["length"][:, None]
        g = torch.where(inside, s["g"][at.clamp_(max=s["g"].numel() - 1)].double(), 0.0)
        norm = g.square().sum().sqrt()
        scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm)).float()
        out["norm"] = norm.float().view(1)
        del g
    _adamw_plain(s, scale)
    out.update(p=s["p"], m=s["m"], v=s["v"])
    if case["bits"] == 8:
        out.update(m=s["m_values"], v=s["v_values"], ms=s["ms"], vs=s["vs"])
    if case["copy"]:
        out["copy"] = s["copy"]
    return out


def work(case):
    """Each input read once, each output written once; a few operations for each element."""
    if case["op"] == "norm":
        n, size, r = case["T"] * case["d"], 2 if case["dtype"] == "bf16" else 4, 1 if case["residual"] else 0
        total = n * size * (2 + 2 * r) + 8 * case["d"] + 8 * case["T"]
        if case["pass"] == "train":
            total += n * size * (2 + r) + 8 * case["d"]     # dy, dsum and dx; s is there
        return {"bytes": total, "flops": n * (24 if case["pass"] == "train" else 8)}
    if case["op"] == "embed":
        T, d, V, size = case["T"], case["d"], case["V"], 2 if case["dtype"] == "bf16" else 4
        distinct = min(T, int(V * (1 - math.exp(-T / V))) + 1)       # at most
        rows = V * d / case["k"] / 8 if case["k"] else distinct * d * size
        total = 8 * T + min(rows, T * d * size) + T * d * size
        if case["pass"] == "train":
            total += T * d * size + (8 * distinct * d if case["add"] else V * d * size)
        return {"bytes": total, "flops": T * d * (2 if case["pass"] == "train" else 1)}
    n = sum(m for m, _ in _sizes(case))
    sizes = {"f32": 4, "bf16": 2}
    total = n * (2 * sizes[case["p"]] + sizes[case["g"]] + (2 if case["copy"] else 0))
    total += n * 16 if case["bits"] == 32 else n * (4 + 8) + n / BLOCK * 16
    return {"bytes": total, "flops": n * (15 if case["bits"] == 32 else 60)}


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    wide = lambda t: None if t is None else t.to(torch.float64)  # noqa: E731
    if case["op"] == "norm":
        dt = s["x"].dtype
        x = s["x"].double()
        out = {}
        if s["residual"] is not None:
            out["sum"] = (s["x"].double() + s["residual"].double()).to(dt).double()   # the norm is of the rounded sum
            x = out["sum"]
        d = case["d"]
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        gamma, beta = wide(s["gamma"]), wide(s["beta"])
        out.update(y=(x - mean[:, None]) / torch.sqrt(var + EPS)[:, None] * gamma + beta, mean=mean, rstd=rstd)
        if case["pass"] == "train":
            # the gradient from the definition's two inner derivatives: of the variance and of the mean
            dy, e = wide(s["dy"]), x - mean[:, None]
            dh = dy * gamma
            dvar = -0.5 * (dh * e).sum(1) * rstd ** 3
            dmean = -(dh.sum(1) * rstd) - 2 * dvar * e.mean(1)
            dx = dh * rstd[:, None] + (2 * dvar / d)[:, None] * e + (dmean / d)[:, None]
            out["dx"] = dx + wide(s["dsum"]) if s["dsum"] is not None else dx
            out.update(dgamma=torch.einsum("td,td,t->d", dy, e, rstd), dbeta=torch.einsum("td->d", dy))
        return out
    if case["op"] == "embed":
        T, d, V = case["T"], case["d"], case["V"]
        here = ((s["ids"] >= 0) & (s["ids"] < V)).nonzero()[:, 0]
        y = torch.zeros(T, d, dtype=torch.float64, device="cuda")
        if case["k"]:
            q = V * d // case["k"]
            shifts = torch.arange(32, device="cuda")
            signs = ((s["tile"].to(torch.int64)[:, None] >> shifts) & 1).flatten()[:q].to(torch.float64) * 2 - 1
            table = (wide(s["alpha"])[:, None] * signs).reshape(V, d)
        else:
            table = s["table"]
        y[here] = wide(table[s["ids"][here]]) * s["scale"]
        out = {"y": y}
        if case["pass"] == "train":
            order = torch.argsort(s["ids"][here], stable=True)
            ids, rows = s["ids"][here][order], wide(s["dy"])[here[order]]
            seen, count = torch.unique_consecutive(ids, return_counts=True)
            out["dw"] = wide(s["dw"]) if s["dw"] is not None else torch.zeros(V, d, dtype=torch.float64, device="cuda")
            if here.numel():
                out["dw"][seen] += s["scale"] * torch.segment_reduce(rows, "sum", lengths=count, axis=0)
        return out
    places, n, blocks = _places(case)
    out = {"p": wide(s["p"])}
    factor = 1.0
    if case["clip"]:
        norm = math.sqrt(sum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in s["tensors"]["grads"]))
        factor = min(1.0, s["max_norm"] / norm)
        out["norm"] = torch.tensor([norm], dtype=torch.float64, device="cuda")
    eight = case["bits"] == 8
    # which code a value gets is settled by roundings in 32 bits, so 64 bits have no value for it; the scales they do
    out.update(m=None if eight else wide(s["m"]), v=None if eight else wide(s["v"]))
    if eight:
        out.update(ms=wide(s["ms"]), vs=wide(s["vs"]))
    t = s["step"]
    for at, size, block, count, decay in places:
        g = s["g"][at:at + size].double() * factor
        m, v = s["m"][at:at + size].double(), s["v"][at:at + size].double()
        if eight:
            of = torch.arange(size, device="cuda") // BLOCK
            m = torch.sign(m) * m ** 2 * out["ms"][block:block + count][of]
            v = v ** 4 * out["vs"][block:block + count][of]
        m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g ** 2
        step = (m / (1 - B1 ** t)) / (torch.sqrt(v / (1 - B2 ** t)) + EPS)
        p = out["p"][at:at + size]
        p -= LR * (step + decay * p)
        if eight:
            pad = torch.zeros(count * BLOCK - size, dtype=torch.float64, device="cuda")
            out["ms"][block:block + count] = torch.cat([m.abs(), pad]).view(count, BLOCK).amax(1) / 127.0 ** 2
            out["vs"][block:block + count] = torch.cat([v, pad]).view(count, BLOCK).amax(1) / 254.0 ** 4
        else:
            out["m"][at:at + size], out["v"][at:at + size] = m, v
    if case["copy"]:
        out["copy"] = wide(s["copy"])
        for at, size, _, _, _ in places:
            out["copy"][at:at + size] = out["p"][at:at + size]
    return out
