"""Plain 64-bit forms of the head losses and the error bounds their tests use."""
import math

import torch

from paper_2407_12075_b200 import binding as B

LN_EPS = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}       # half a step of the stored type, relative


def teacher_matrix(T, V, index, logit, tau):
    """Dense T x V probabilities of the listed entries, sum p log p per row, and which rows have an entry."""
    dense = torch.zeros(T, V, dtype=torch.float64)
    plogp, some = torch.zeros(T, dtype=torch.float64), torch.zeros(T, dtype=torch.bool)
    for t in range(T):
        entries = [(int(c), float(l) / tau) for c, l in zip(index[t], logit[t]) if 0 <= int(c) < V and float(l) != -math.inf]
        if not entries:
            continue
        some[t] = True
        p = torch.softmax(torch.tensor([l for _, l in entries], dtype=torch.float64), 0)
        for (c, _), q in zip(entries, p):
            dense[t, c] += q
        plogp[t] = torch.special.xlogy(p, p).sum()
    return dense, plogp, some


def reference(x, w, bias, dloss, tau, dense, plogp, some):
    """(loss, lse, dx, dw, db) and the absolute sums behind the error bounds, all in 64 bits."""
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    x, w, dense, plogp, some = x.double().to(dev), w.double().to(dev), dense.to(dev), plogp.to(dev), some.to(dev)
    b = bias.double().to(dev) if bias is not None else torch.zeros(w.shape[0], dtype=torch.float64, device=dev)
    x = torch.where(some[:, None], x, torch.zeros_like(x))
    z = (x @ w.t() + b) / tau
    lse = torch.logsumexp(z, 1)
    logq = z - lse[:, None]
    cross = torch.where(dense > 0, dense * logq, torch.zeros_like(dense)).sum(1)
    loss = torch.where(some, tau * tau * (plogp - cross), torch.zeros_like(lse))
    g = torch.where(some, dloss.double().to(dev) * tau, torch.zeros_like(lse))
    q = logq.exp()
    dz = torch.where(some[:, None], (q - dense) * g[:, None], torch.zeros_like(q))
    size = torch.where(some[:, None], (q + dense) * g.abs()[:, None], torch.zeros_like(q))
    finite_b = torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b))
    return {"loss": loss, "lse": torch.where(some, lse, torch.zeros_like(lse)), "dx": dz @ w, "dw": dz.t() @ x, "db": dz.sum(0),
            "z_abs": float((x.abs() @ w.abs().t() + finite_b).max()) / tau if x.numel() else 0.0,
            "dx_abs": dz.abs() @ w.abs(), "dw_abs": dz.abs().t() @ x.abs(), "db_abs": dz.abs().sum(0),
            "dx_size": size @ w.abs(), "dw_size": size.t() @ x.abs(), "db_size": size.sum(0),
            "g_max": float(g.abs().max()) if g.numel() else 0.0, "x_sum": x.abs().sum(0), "w_sum": w.abs().sum(0)}


def bounds(ref, x, w, tau, dw_dtype):
    """Element-wise bounds, from the roundings that take place.

    u: relative error of one product term: 0 for bf16 (products of bf16 are exact in fp32), 3 * 2^-22 for the two-halves
    form of fp32 (each operand to 2^-22, lo*lo dropped).  A sum of n terms on the tensor core adds n / 16 partial sums, each
    cut off at 2^-23 of the running magnitude, three times as many for the halves.  The logit's error enters the softmax
    as a relative error of the same size, twice (logit and lse); exp2 and the scaling add 2^-20.  dz is rounded to bf16 or
    to two halves: 2^-22 of the element, and where the low half runs out of exponent half of fp16's smallest step, 2^-25, under
    a scale that takes max |dloss tau| to 2^14 at least, i.e. 2^-39 of that maximum for every term of the sum.  The result is
    rounded once more."""
    T, d = x.shape
    V = w.shape[0]
    f32 = x.dtype == torch.float32
    u, terms = (3 * 2.0 ** -22, 3) if f32 else (0.0, 1)
    acc = lambda n: (terms * n / 16 + 8) * 2.0 ** -23
    zerr = ref["z_abs"] * (u + acc(d) + 2.0 ** -22)
    zmax = ref["z_abs"] + math.log(V)
    out = {"lse": 2 * zerr + 2.0 ** -20 + 2.0 ** -22 * zmax}
    out["loss"] = tau * tau * (3 * zerr + 2.0 ** -19 + 2.0 ** -20 * zmax) + 2.0 ** -22 * ref["loss"].abs().nan_to_num(0, 0, 0)
    rel = 2 * out["lse"] + 2.0 ** -20
    dz_round = 2.0 ** -22 if f32 else 2.0 ** -8
    floor = 2.0 ** -39 * ref["g_max"] if f32 else 0.0
    o = LN_EPS[x.dtype]
    ow = LN_EPS[torch.bfloat16 if dw_dtype == B.BF16 else torch.float32]
    out["dx"] = ref["dx_size"] * rel + ref["dx_abs"] * (dz_round + u + acc(V)) + ref["dx"].abs() * o + floor * ref["w_sum"] + 1e-30
    out["dw"] = ref["dw_size"] * rel + ref["dw_abs"] * (dz_round + u + acc(T)) + ref["dw"].abs() * ow + floor * ref["x_sum"] + 1e-30
    out["db"] = ref["db_size"] * rel + ref["db_abs"] * (T * 2.0 ** -24 + 2.0 ** -23) + 1e-30
    return out


def assert_within(got, ref, bound, what):
    got = got.double().to(ref.device)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    same = (got == ref) | (torch.isnan(got) & torch.isnan(ref))
    err = torch.where(same, torch.zeros_like(ref), (got - ref).abs())
    over = ~(err <= bound)
    assert not bool(over.any()), (f"{what}: {int(over.sum())} of {over.numel()} outside, worst error {float(err[over].max()):.3g}, "
                                  f"ratio {float((err / bound).max()):.3g}, first at {over.nonzero()[0].tolist()}")
