"""64-bit forms of the head losses with error bounds for every token and class by itself, for inputs whose tokens, classes or
features differ by many orders of magnitude."""
import math

import torch

from paper_2407_12075_b200 import binding as B

DEV = "cuda:0"


def xent_teacher(targets, V, ignore=-100):
    """Dense T x V probabilities, sum p log p per row, and which rows are kept, of a cross entropy."""
    some = (targets != ignore) & (targets >= 0) & (targets < V)
    dense = torch.zeros(targets.shape[0], V, dtype=torch.float64, device=targets.device)
    dense[some.nonzero()[:, 0], targets[some]] = 1.0
    return dense, torch.zeros(targets.shape[0], dtype=torch.float64, device=targets.device), some


def distill_teacher(index, logit, V, tau):
    """The same of a teacher's lists: a class listed twice has the sum of its probabilities."""
    valid = (index >= 0) & (index < V) & (logit != -math.inf)
    some = valid.any(1)
    l = torch.where(valid, logit.double() / tau, torch.full(logit.shape, -math.inf, dtype=torch.float64, device=logit.device))
    p = torch.softmax(torch.where(some[:, None], l, torch.zeros_like(l)), 1) * valid
    dense = torch.zeros(index.shape[0], V, dtype=torch.float64, device=index.device)
    dense.scatter_add_(1, torch.where(valid, index, torch.zeros_like(index)), p)
    return dense, torch.special.xlogy(p, p).sum(1), some


def reference(x, w, bias, dloss, tau, teacher, dw_dtype):
    """({name: value}, {name: bound}), all on the GPU in 64 bits.  The bounds, from the roundings that take place:

    logit    bf16 products are exact in fp32.  An fp32 operand is three bf16 parts, each at most 2^-8 of what the ones before
             leave over; the products of parts that are dropped (second times third, third times second, third times third) are
             below 2^-22 of |x||w|.  The tensor core cuts its running sum off at 2^-23 of its size after 16 elements.  Scaling and
             the rounded parts of lse: 2^-22.  All relative to this token's largest sum of |x||w| + |bias|.
    q        exp(logit - lse), the error of its argument E: q exp(-E) to q exp(E), and never above 1 + 2^-7.
    dz       dloss (q - p); rounded to bf16, or to three parts.  An element ends at 2^-134 (half the smallest bf16), and
             exponentials below 2^-126 are 0.
    sums     cut off as above; products below 2^-126 may be lost.  tau is multiplied in at the end; one rounding to the type."""
    f32 = x.dtype == torch.float32
    dense, plogp, some = teacher
    x, w = x.double(), w.double()
    T, d = x.shape
    V = w.shape[0]
    b = bias.double() if bias is not None else torch.zeros(V, dtype=torch.float64, device=x.device)
    x = torch.where(some[:, None], x, torch.zeros_like(x))
    z = (x @ w.t() + b) / tau
    lse = torch.logsumexp(z, 1)
    logq = z - lse[:, None]
    q = logq.exp()
    cross = torch.where(dense > 0, dense * logq, torch.zeros_like(dense)).sum(1)
    loss = tau * tau * (plogp - cross)
    g = torch.where(some, dloss.double(), torch.zeros_like(lse))
    dz = (q - dense) * g[:, None]
    finite_b = torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b))
    z_abs = (x.abs() @ w.abs().t() + finite_b).max(1).values / tau

    acc = lambda n: (n / 16 + 8) * 2.0 ** -23
    u, dz_round = (2.0 ** -22, 2.0 ** -22) if f32 else (0.0, 2.0 ** -8)
    z_err = z_abs * (u + acc(d) + 2.0 ** -22)
    z_max = z_abs + math.log(V)
    zero = torch.zeros_like(lse)
    val = {"lse": torch.where(some, lse, zero), "loss": torch.where(some, loss, zero)}
    bound = {"lse": 2 * z_err + 2.0 ** -20 + 2.0 ** -22 * z_max}
    bound["loss"] = tau * tau * (3 * z_err + 2.0 ** -19 + 2.0 ** -20 * z_max) + 2.0 ** -22 * loss.abs()
    E = (2 * bound["lse"] + 2.0 ** -20)[:, None]
    q_err = torch.maximum((logq + E).exp().clamp(max=1 + 2.0 ** -7) - q, q - (logq - E).exp())
    teacher_err = 2.0 ** -18 if plogp.any() else 2.0 ** -22
    dz_err = g.abs()[:, None] * (q_err + teacher_err * dense + 2.0 ** -126) + 2.0 ** -134
    size = dz.abs() + dz_err
    o = 2.0 ** -24 if f32 else 2.0 ** -8
    ow = 2.0 ** -24 if dw_dtype == B.F32 else 2.0 ** -8
    for name, out, rows, n, half in (("dx", dz @ w, lambda m: m @ w.abs(), V, o), ("dw", dz.t() @ x, lambda m: m.t() @ x.abs(), T, ow)):
        val[name] = out * tau
        bound[name] = tau * (rows(dz_err) + rows(size) * (dz_round + u + acc(n)) + n * 2.0 ** -126) + val[name].abs() * half + 2.0 ** -149
    val["db"] = dz.sum(0) * tau
    bound["db"] = tau * (dz_err.sum(0) + size.sum(0) * (T * 2.0 ** -24 + 2.0 ** -23)) + 2.0 ** -149
    return val, bound


def assert_close(got, val, bound, what, rows=None):
    assert got.shape == val.shape, (what, got.shape, val.shape)
    got = got.double()
    if rows is not None:
        got, val, bound = got[rows], val[rows], bound[rows]
    ok = (got - val).abs() <= bound
    top = float(torch.finfo(torch.float32).max)          # a value within the bound that fp32 and bf16 cannot hold is an infinity
    ok |= ((val + bound > top) & (got == math.inf)) | ((val - bound < -top) & (got == -math.inf))
    over = ~ok
    assert not bool(over.any()), (f"{what}: {int(over.sum())} of {over.numel()} outside, worst {float((got - val).abs()[over].nan_to_num(math.inf).max()):.3g}, "
                                  f"first at {over.nonzero()[0].tolist()}: {float(got[over][0]):.6g} for {float(val[over][0]):.6g} +- {float(bound[over][0]):.3g}")


def check(x, w, bias, dloss, tau=1.0, targets=None, index=None, logit=None, dw_dtype=B.F32, names=("lse", "loss", "dx", "dw", "db"), workspace=None):
    """Runs both calls on GPU tensors and holds every element of every output against its bound."""
    V = w.shape[0]
    if targets is not None:
        loss, lse = B.tbn_linear_xent_fwd(x, w, targets, bias=bias)
        dx, dw, db = B.tbn_linear_xent_bwd(x, w, targets, lse, dloss, bias=bias, need_dbias=True, dw_dtype=dw_dtype, workspace=workspace)
        teacher = xent_teacher(targets, V)
    else:
        loss, lse = B.tbn_linear_distill_fwd(x, w, index, logit, temperature=tau, bias=bias)
        dx, dw, db = B.tbn_linear_distill_bwd(x, w, index, logit, lse, dloss, temperature=tau, bias=bias, need_dbias=True, dw_dtype=dw_dtype,
                                              workspace=workspace)
        teacher = distill_teacher(index, logit, V, tau)
    torch.cuda.synchronize()
    assert B.tbn_last_device_status() == (0, 0)
    val, bound = reference(x, w, bias, dloss, tau, teacher, dw_dtype)
    got = {"lse": lse, "loss": loss, "dx": dx, "dw": dw, "db": db}
    for name in names:
        assert_close(got[name], val[name], bound[name], name)
    return got, val, bound
