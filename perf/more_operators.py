"""The operators around a network's logits, as cases that can be timed and compared: the transform with its bias, activation and
residual in one pass, log probabilities of given classes with entropy and top alternatives, and distillation from a teacher's
top classes, each forward and backward.

`run` computes a case in its plain form, by elementary torch operations, or, where `own` is set, by the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
ACTS = ["none", "relu", "gelu", "silu", "elu"]

# Widths of this repository's layers, and its numbers of classes; beside them any number, up to tables of entities.
WIDTHS = [47, 64, 100, 128, 200, 256, 400, 512]
CLASSES = [47, 172]


def listed():
    def act(name, call, n, K, F, dtype, act, bias=True, res="none", extra=False):
        return {"name": name, "call": call, "n": n, "K": K, "F": F, "dtype": dtype, "act": act, "bias": bias, "res": res, "extra": extra}

    def classes(name, call, n, C, dtype, k):
        return {"name": name, "call": call, "n": n, "C": C, "dtype": dtype, "k": k}

    return [
        # a hidden layer on a small sampled neighbourhood, its aggregate added before the ReLU: a launch's latency
        act("act_fwd_sampled", "act_fwd", 2_000, 128, 128, "bf16", "relu", res="first"),
        # first GraphSage layer of one worker's share of the products-sized graph: sigma(X W + b + aggregate)
        act("act_fwd_products", "act_fwd", 306_250, 100, 256, "f32", "relu", res="first"),
        # a hidden layer of a papers-sized share with a skip connection behind its GELU, in training (keeps what GELU was taken of)
        act("act_fwd_papers", "act_fwd", 867_187, 256, 256, "bf16", "gelu", res="after", extra=True),
        # the backward pass of a hidden layer with an aggregate inside an ELU, whose gradient is the error handed to the aggregation
        act("act_bwd_products", "act_bwd", 306_250, 256, 256, "f32", "elu", res="first", extra=True),
        # ... of the papers-sized hidden layer
        act("act_bwd_papers", "act_bwd", 867_187, 256, 256, "bf16", "gelu"),
        # the loss and the five likeliest classes of a worker's nodes
        classes("logp_fwd_products", "logp_fwd", 306_250, 47, "f32", 5),
        # ... of the papers-sized graph's, with the eight that a student is taught from
        classes("logp_fwd_papers", "logp_fwd", 1_734_375, 172, "bf16", 8),
        # links as classes: 64 queries against a table of 65536 entities
        classes("logp_fwd_entities", "logp_fwd", 64, 65_536, "f32", 8),
        # gradients of likelihood and entropy
        classes("logp_bwd_papers", "logp_bwd", 1_734_375, 172, "bf16", 0),
        # a student's loss against its teacher's eight likeliest classes, and the gradient
        classes("distill_fwd_papers", "distill_fwd", 1_734_375, 172, "bf16", 8),
        classes("distill_bwd_products", "distill_bwd", 306_250, 47, "f32", 8),
        # ... of 50 thousand classes, 32 of them taught
        classes("distill_bwd_entities", "distill_bwd", 4_096, 50_000, "bf16", 32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    call = rng.choice(["act_fwd", "act_bwd", "logp_fwd", "logp_bwd", "distill_fwd", "distill_bwd"])
    dtype = rng.choice(["f32", "bf16"])
    n = _log_int(rng, 1, 1_700_000)
    if call.startswith("act"):
        # one draw in three has widths off the usual ones; no more values and multiplications than the listed cases have
        K, F = (rng.randint(1, 520) if rng.random() < 1 / 3 else rng.choice(WIDTHS) for _ in range(2))
        n = max(1, min(n, 300_000_000 // (K + F), 20_000_000_000 // (K * F)))
        return {"call": call, "n": n, "K": K, "F": F, "dtype": dtype, "act": rng.choice(ACTS), "bias": rng.random() < 0.7,
                "res": rng.choice(["none", "first", "after"]) if call == "act_fwd" else rng.choice(["none", "first"]),
                "extra": rng.random() < 0.5}
    C = rng.choice(CLASSES) if rng.random() < 1 / 3 else _log_int(rng, 2, 131_072)
    k = min(C, _log_int(rng, 1, 40))
    if call == "logp_fwd":
        k -= 1
    n = max(1, min(n, (200_000_000 if call != "logp_fwd" else 2_000_000_000 // (k + 7)) // C))
    return {"call": call, "n": n, "C": C, "dtype": dtype, "k": 0 if call == "logp_bwd" else k}


# ------------------------------------------------------------------ what a program holds before the call

class State:
    pass


def _logits(randn, n, C, dt):
    """Rows as a trained network leaves them: some rows sure, some not, a few classes ahead of the others."""
    x = randn(n, C)
    x *= (0.5 + 2 * torch.rand(n, 1, device="cuda", generator=randn.g)).to(dt)
    x += (2 * randn(1, C)).to(dt)
    return x


def prepare(case, seed):
    s = State()
    s.case = case
    call, n = case["call"], case["n"]
    s.dt = dt = DTYPES[case["dtype"]]
    f32 = torch.float32
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def randn(*shape, dtype=dt):
        return torch.randn(*shape, dtype=dtype, device="cuda", generator=g)
    randn.g = g

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    s.work = None       # scratch, which a program asks for once and keeps
    if call.startswith("act"):
        K, F = case["K"], case["F"]
        s.W = randn(K, F, dtype=f32) * math.sqrt(2.0 / (K + F))
        s.X = randn(n, K)
        s.A = None
        if call == "act_fwd":
            s.bias = 0.1 * randn(F, dtype=f32) if case["bias"] else None
            s.res = randn(n, F) if case["res"] != "none" else None
            s.Y = empty(n, F)
            if case["extra"]:
                s.A = empty(n, F)
        else:
            if case["act"] != "none":
                s.A = randn(n, F)
            s.dY = randn(n, F)
            s.dW, s.dX = empty(K, F, dtype=f32), empty(n, K)
            s.db = empty(F, dtype=f32) if case["bias"] else None
            s.dA = empty(n, F) if case["extra"] else None
        return s

    C, k = case["C"], case["k"]
    s.X = _logits(randn, n, C, dt)
    if call.startswith("logp"):
        # three nodes in five have a label
        label = torch.randint(0, C, (n,), dtype=torch.int32, device="cuda", generator=g)
        s.label = torch.where(torch.rand(n, device="cuda", generator=g) < 0.6, label, -1)
        if call == "logp_fwd":
            s.logp, s.lse, s.entropy = empty(n, dtype=f32), empty(n, dtype=f32), empty(n, dtype=f32)
            s.top = (empty(n, k, dtype=f32), empty(n, k, dtype=torch.int32)) if k else None
        else:
            s.lse, s.entropy = _statistics(s.X)
            s.dlogp, s.dentropy = -0.5 - torch.rand(n, device="cuda", generator=g), 0.1 * randn(n, dtype=f32)
            s.dX = empty(n, C)
        return s
    s.temperature = 2.0
    # the teacher's likeliest classes, no class twice, and log probabilities of theirs, in descending order
    start, step = (torch.randint(0, C, (n, 1), device="cuda", generator=g) for _ in range(2))
    step = step % max(1, C // k) + 1 if C > k else torch.ones_like(step)
    index = ((start + step * torch.arange(k, device="cuda")) % C).to(torch.int32)
    value = (-torch.cumsum(0.05 + torch.rand(n, k, device="cuda", generator=g), 1)).contiguous()
    s.top = (value, index.contiguous())
    if call == "distill_fwd":
        s.loss, s.lse = empty(n, dtype=f32), empty(n, dtype=f32)
    else:
        s.lse = _statistics(s.X, s.temperature)[0]
        s.dloss = 0.5 + torch.rand(n, device="cuda", generator=g)
        s.dX = empty(n, C)
    return s


# ------------------------------------------------------------------------------------------ plain forms

def _act(name, a):
    if name == "relu":
        return a.clamp(min=0)
    if name == "gelu":
        return 0.5 * a * (1 + torch.erf(a * math.sqrt(0.5)))
    if name == "silu":
        return a / (1 + torch.exp(-a))
    if name == "elu":
        return torch.where(a > 0, a, torch.expm1(a))
    return a


def _slope(name, a):
    if name == "relu":
        return (a > 0).to(a.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(a * math.sqrt(0.5))) + a * torch.exp(-0.5 * a * a) * (1 / math.sqrt(2 * math.pi))
    if name == "silu":
        p = 1 / (1 + torch.exp(-a))
        return p * (1 + a * (1 - p))
    return torch.where(a > 0, torch.ones_like(a), torch.exp(a))


def _act_fwd(s):
    case = s.case
    a = s.X.float() @ s.W
    if s.bias is not None:
        a = a + s.bias
    if case["res"] == "first":
        a = a + s.res.float()
    y = _act(case["act"], a)
    if case["res"] == "after":
        y = y + s.res.float()
    out = {"Y": y.to(s.dt)}
    if case["extra"]:
        out["A"] = a.to(s.dt)
    return out


def _act_bwd(s):
    case = s.case
    dA = s.dY.float()
    if case["act"] != "none":
        dA = dA * _slope(case["act"], s.A.float())
    out = {"dW": s.X.float().T @ dA, "dX": (dA @ s.W.T).to(s.dt)}
    if s.db is not None:
        out["db"] = dA.sum(0)
    if s.dA is not None:
        out["dA"] = dA.to(s.dt)
    return out


def _statistics(X, temperature=1.0):
    """Log of the sum of exponentials of every row over the temperature, and the entropy of its classes."""
    x = X.float()
    if temperature != 1.0:
        x = x / temperature
    m = x.amax(1, keepdim=True)
    x = x - m
    e = torch.exp(x)
    total = e.sum(1)
    log = torch.log(total)
    return m.squeeze(1) + log, log - (e * x).sum(1) / total


def _logp_fwd(s):
    lse, entropy = _statistics(s.X)
    n, k = s.case["n"], s.case["k"]
    row = torch.arange(n, device=s.X.device)
    at = s.label.clamp(min=0).long()
    out = {"logp": torch.where(s.label >= 0, s.X[row, at].float() - lse, 0.0), "lse": lse, "entropy": entropy}
    if k:
        # the largest one, which is then taken out, k times over; argmax gives the first of several
        x = s.X.float()
        if x is s.X:
            x = x.clone()
        value, index = torch.empty(n, k, device=x.device), torch.empty(n, k, dtype=torch.int32, device=x.device)
        for j in range(k):
            i = torch.argmax(x, 1)
            index[:, j] = i.int()
            value[:, j] = x[row, i] - lse
            x[row, i] = -math.inf
        out["top_value"], out["top_index"] = value, index
    return out


def _logp_bwd(s):
    logp = s.X.float() - s.lse[:, None]
    p = torch.exp(logp)
    g = torch.where(s.label >= 0, s.dlogp, 0.0)
    d = -p * (g[:, None] + s.dentropy[:, None] * (logp + s.entropy[:, None]))
    row = torch.arange(s.case["n"], device=d.device)
    d[row, s.label.clamp(min=0).long()] += g
    return {"dX": d.to(s.dt)}


def _teacher(s):
    """The teacher's probabilities of its classes at the temperature, and their logs."""
    v = s.top[0] / s.temperature
    v = v - v.amax(1, keepdim=True)
    log = v - torch.log(torch.exp(v).sum(1, keepdim=True))
    return torch.exp(log), log


def _distill_fwd(s):
    lse, _ = _statistics(s.X, s.temperature)
    p, logp = _teacher(s)
    x = torch.gather(s.X, 1, s.top[1].long()).float() / s.temperature
    return {"loss": (p * (logp - (x - lse[:, None]))).sum(1), "lse": lse}


def _distill_bwd(s):
    p, _ = _teacher(s)
    g = (s.dloss / s.temperature)[:, None]
    d = torch.exp(s.X.float() / s.temperature - s.lse[:, None]) * g
    d.scatter_add_(1, s.top[1].long(), -p * g)
    return {"dX": d.to(s.dt)}


# ------------------------------------------------------------------------------------------- one pass

def _own(s):
    from paper_2111_06483_amd import sar
    case = s.case
    call, n = case["call"], case["n"]
    if call.startswith("act"):
        if s.work is None:
            s.work = torch.empty(sar.sar_linear_act_workspace_bytes(n, case["K"], case["F"]), dtype=torch.uint8, device="cuda")
        act = getattr(sar, "SAR_ACT_" + case["act"].upper())
        if call == "act_fwd":
            sar.sar_linear_act_fwd(s.X, s.W, s.bias, s.res, act, case["res"] == "after", s.Y, s.A, s.work)
            return {"Y": s.Y, "A": s.A} if case["extra"] else {"Y": s.Y}
        sar.sar_linear_act_bwd(s.dY, s.A, s.X, s.W, act, False, s.dW, s.db, s.dX, s.dA, s.work)
        out = {"dW": s.dW, "dX": s.dX, "db": s.db, "dA": s.dA}
        return {name: t for name, t in out.items() if t is not None}
    C, k = case["C"], case["k"]
    if call == "logp_bwd":
        sar.sar_logprob_bwd(s.X, s.label, s.lse, s.entropy, s.dlogp, s.dentropy, s.dX)
        return {"dX": s.dX}
    if call == "distill_bwd":
        sar.sar_distill_bwd(s.X, s.top, s.temperature, s.lse, s.dloss, s.dX)
        return {"dX": s.dX}
    if s.work is None:
        size = sar.sar_logprob_workspace_bytes(n, C, k) if call == "logp_fwd" else sar.sar_distill_workspace_bytes(n, C, k)
        s.work = torch.empty(size, dtype=torch.uint8, device="cuda")
    if call == "logp_fwd":
        sar.sar_logprob_fwd(s.X, s.label, s.logp, s.lse, s.entropy, s.top, s.work)
        out = {"logp": s.logp, "lse": s.lse, "entropy": s.entropy}
        if k:
            out["top_value"], out["top_index"] = s.top
        return out
    sar.sar_distill_fwd(s.X, s.top, s.temperature, s.loss, s.lse, s.work)
    return {"loss": s.loss, "lse": s.lse}


def run(s):
    if own:
        return _own(s)
    return {"act_fwd": _act_fwd, "act_bwd": _act_bwd, "logp_fwd": _logp_fwd, "logp_bwd": _logp_bwd, "distill_fwd": _distill_fwd,
            "distill_bwd": _distill_bwd}[s.case["call"]](s)


# ------------------------------------------------------------------------- work of a pass, and its values

def work(case):
    """Inputs read once, outputs written once."""
    call, n, b = case["call"], case["n"], SIZE[case["dtype"]]
    if call.startswith("act"):
        K, F = case["K"], case["F"]
        if call == "act_fwd":
            rows = 1 + (case["res"] != "none") + case["extra"]
            return {"bytes": n * (K + rows * F) * b + 4 * K * F + 4 * F * case["bias"], "flops": 2 * n * K * F}
        rows = 1 + (case["act"] != "none") + case["extra"]
        return {"bytes": n * (2 * K + rows * F) * b + 8 * K * F + 4 * F * case["bias"], "flops": 4 * n * K * F}
    C, k = case["C"], case["k"]
    if call == "logp_fwd":
        return {"bytes": n * (C * b + 16 + 8 * k), "flops": 6 * n * C}
    if call == "logp_bwd":
        return {"bytes": n * (2 * C * b + 20), "flops": 6 * n * C}
    if call == "distill_fwd":
        return {"bytes": n * (C * b + 8 + 8 * k), "flops": 4 * n * C}
    return {"bytes": n * (2 * C * b + 8 + 8 * k), "flops": 4 * n * C}


def _act_values(name, a):
    """(activation, its derivative) in 64 bits."""
    zero, one = torch.zeros_like(a), torch.ones_like(a)
    if name == "relu":
        return torch.maximum(a, zero), torch.where(a > 0, one, zero)
    if name == "gelu":
        share = 0.5 * torch.special.erfc(-a / 2.0 ** 0.5)
        return a * share, share + a * torch.exp(-a.square() / 2) / (2 * torch.pi) ** 0.5
    if name == "silu":
        share = torch.sigmoid(a)
        return a * share, share + a * share * torch.sigmoid(-a)
    if name == "elu":
        return torch.maximum(a, zero) + torch.expm1(torch.minimum(a, zero)), torch.exp(torch.minimum(a, zero))
    return a, one


def exact(case, seed):
    s = prepare(case, seed)
    call, n = case["call"], case["n"]
    x = s.X.double()
    if call == "act_fwd":
        a = torch.matmul(x, s.W.double())
        if case["bias"]:
            a += s.bias.double()
        first = case["res"] == "first"
        if first:
            a += s.res.double()
        y = _act_values(case["act"], a)[0]
        if case["res"] != "none" and not first:
            y = y + s.res.double()
        return {"Y": y, "A": a} if case["extra"] else {"Y": y}
    if call == "act_bwd":
        d = s.dY.double()
        if case["act"] != "none":
            d = d * _act_values(case["act"], s.A.double())[1]
        out = {"dW": torch.matmul(x.t(), d), "dX": torch.matmul(d, s.W.double().t())}
        if case["bias"]:
            out["db"] = d.sum(0)
        if case["extra"]:
            out["dA"] = d
        return out
    if call == "logp_fwd":
        lse = torch.logsumexp(x, 1)
        x -= lse[:, None]
        there = torch.nonzero(s.label >= 0).flatten()
        logp = torch.zeros(n, dtype=torch.float64, device=x.device)
        logp[there] = x[there, s.label[there].long()]
        out = {"logp": logp, "lse": lse, "entropy": -(torch.exp(x) * x).sum(1)}
        if case["k"]:
            # (of the values as they are given, equal ones in the order of their classes)
            order = torch.sort(s.X, dim=1, descending=True, stable=True).indices[:, :case["k"]]
            out["top_value"], out["top_index"] = torch.gather(x, 1, order), order.int()
        return out
    if call == "logp_bwd":
        x -= s.lse.double()[:, None]
        p = torch.exp(x)
        one = torch.nn.functional.one_hot(s.label.clamp(min=0).long(), case["C"]) if case["C"] <= 256 else None
        g = torch.where(s.label >= 0, s.dlogp.double(), 0.0)[:, None]
        d = -p * (x + s.entropy.double()[:, None]) * s.dentropy.double()[:, None] - g * p
        if one is not None:
            d += g * one
        else:
            d.scatter_add_(1, s.label.clamp(min=0).long()[:, None], g)
        return {"dX": d}
    x /= s.temperature
    teacher = torch.softmax(s.top[0].double() / s.temperature, 1)
    index = s.top[1].long()
    if call == "distill_fwd":
        lse = torch.logsumexp(x, 1)
        student = torch.gather(x, 1, index) - lse[:, None]
        return {"loss": (torch.special.xlogy(teacher, teacher) - teacher * student).sum(1), "lse": lse}
    p = torch.exp(x - s.lse.double()[:, None])
    p.scatter_add_(1, index, -teacher)
    return {"dX": p * (s.dloss.double() / s.temperature)[:, None]}
