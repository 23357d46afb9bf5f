"""Timed cases of the training step's loss and normalisation operators.

Three operators, through the public entry points (``own``) and in a plain form
made of elementary torch operations:

* ``top``      the K largest logits of every row with their class ids and the
               log-sum of the rest at a temperature: what a teacher keeps of
               its answer for a student (``pgcn_top_logits``);
* ``distill``  the loss of a student's logits against such top logits, with an
               optional hard-label term, and its gradient
               (``pgcn_distill_loss_fwd_bwd``);
* ``norm``     group normalisation of features-last rows with an activation,
               forward and backward (``pgcn_group_norm_fwd`` / ``_bwd``).

Widths and row counts are those of this repository's workloads (41, 47, 100
and 64 classes; 256 and 512 hidden features; 58,000 to 306,000 nodes) and
generic larger ones.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
NINF = float("-inf")


def _top(name, rows, classes, top, dtype="f32", temp=1.0, masked=False):
    return dict(name=name, op="top", rows=rows, classes=classes, top=top, dtype=dtype, temp=temp, masked=masked)


def _distill(name, rows, classes, top, dtype="f32", temp=1.0, tail=True, labels=False, masked=False):
    return dict(name=name, op="distill", rows=rows, classes=classes, top=top, dtype=dtype, temp=temp, tail=tail,
                labels=labels, masked=masked)


def _norm(name, way, samples, sample_rows, channels, groups, act, dtype="f32"):
    return dict(name=name, op="norm", way=way, samples=samples, sample_rows=sample_rows, channels=channels,
                groups=groups, act=act, dtype=dtype)


def listed():
    return [
        # the smallest partition (1,000 nodes, 8 classes): launches and latency
        _distill("distill tiny 1000x8", 1000, 8, 4, temp=2.0, labels=True),
        # the dense social graph's output layer: many short odd rows, hard labels beside the teacher
        _distill("distill reddit 58000x41", 58000, 41, 8, temp=2.0, labels=True),
        # the co-purchase graph's: more and shorter teacher lists than rows fit a cache, in bf16
        _distill("distill products 306000x47 bf16", 306000, 47, 16, dtype="bf16"),
        # an ordinary batch of rows over a large label set
        _distill("distill 4096x32000", 4096, 32000, 64, labels=True),
        # a few rows over the largest label set: one row is split over the chip
        _distill("distill 16x131071 bf16", 16, 131071, 32, dtype="bf16", temp=4.0, tail=False),
        # the teacher's side of the social graph
        _top("top reddit 58000x41", 58000, 41, 8, temp=2.0),
        # one answer at a time
        _top("top 1x100003", 1, 100003, 50),
        # an ordinary batch, whose bf16 logits hold ties
        _top("top 2048x65536 bf16", 2048, 65536, 64, dtype="bf16"),
        # between two hidden layers of the social graph: every node normalised by itself
        _norm("norm fwd reddit 58000x256", "fwd", 58000, 1, 256, 1, "relu"),
        # the widest hidden layer, backward: the largest traffic
        _norm("norm bwd yelp 239000x512", "bwd", 239000, 1, 512, 32, "silu"),
        # one sample over all nodes of the partition: a long reduction
        _norm("norm fwd whole 58000x256", "fwd", 1, 58000, 256, 8, "gelu"),
        # a batch of features-last grids in bf16, backward
        _norm("norm bwd 8x4096x320 bf16", "bwd", 8, 4096, 320, 32, "silu", dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: any operator, size (odd ones too), type and option."""
    op = rng.choice(["top", "distill", "distill", "norm", "norm"])
    dtype = rng.choice(["f32", "f32", "bf16"])
    if op != "norm":
        classes = _log(rng, 2, 140000)
        rows = _log(rng, 1, max(1, min(300000, 120_000_000 // classes)))
        top = _log(rng, 1, min(classes, 128))
        temp = rng.choice([1.0, 2.0, 0.5, round(rng.uniform(0.3, 6.0), 2)])
        masked = rng.random() < 0.3
        if op == "top":
            return dict(_top("", rows, classes, top, dtype, temp, masked))
        return dict(_distill("", rows, classes, top, dtype, temp, rng.random() < 0.6, rng.random() < 0.6, masked))
    way = rng.choice(["fwd", "bwd"])
    groups = rng.choice([1, 1, 2, 4, 8, 16, 32, 3, 5, 7])
    channels = groups * _log(rng, 2, max(2, 2048 // groups))
    total = max(1, _log(rng, 256, 100_000_000) // channels)           # rows
    sample_rows = 1 if rng.random() < 0.4 else _log(rng, 1, total)
    samples = max(1, total // sample_rows)
    return dict(_norm("", way, samples, sample_rows, channels, groups,
                      rng.choice(["none", "relu", "silu", "gelu"]), dtype))


# ------------------------------------------------------------------ inputs --

def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ld(f):
    return (f + 7) // 8 * 8


def _matrix(gen, rows, cols, dtype, scale=1.0, shift=0.0):
    """[rows, ld] with the row stride of every activation matrix; the padding columns hold nothing of use."""
    x = torch.randn(rows, _ld(cols), generator=gen, device=DEV)
    return x.mul_(scale).add_(shift).to(dtype)


def _teacher(Z, case, gen):
    """A teacher's top logits: the student's own, perturbed; one node in twenty has none."""
    C, K, T = case["classes"], case["top"], case["temp"]
    t = Z[:, :C].float()
    t = t + torch.randn(t.shape, generator=gen, device=DEV)
    v, i = torch.topk(t, K, dim=1)
    t = t.scatter_(1, i, NINF)
    tail = torch.logsumexp(t.div_(T), dim=1)
    i = torch.where(v > NINF, i, torch.full_like(i, -1)).to(torch.int32)
    none = torch.rand(Z.shape[0], generator=gen, device=DEV) < 0.05
    i[none] = -1
    return v.contiguous(), i.contiguous(), tail.contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "norm":
        rows, f = case["samples"] * case["sample_rows"], case["channels"]
        dt = _torch_dtype(case)
        s["X"] = _matrix(gen, rows, f, dt, 1.5, 0.5)
        s["gamma"] = torch.randn(f, generator=gen, device=DEV).mul_(0.2).add_(1.0)
        s["beta"] = torch.randn(f, generator=gen, device=DEV).mul_(0.2)
        s["eps"] = 1e-5
        if case["way"] == "bwd":
            s["J_out"] = _matrix(gen, rows, f, dt, 1e-3)
            x = _grouped(s["X"][:, :f].float(), case)
            mean = x.mean((1, 3))
            var = (x - mean[:, None, :, None]).square_().mean((1, 3))
            s["mean"], s["rstd"] = mean.contiguous(), (var + s["eps"]).rsqrt().contiguous()
        return s
    Z = _matrix(gen, case["rows"], case["classes"], _torch_dtype(case), 2.5)
    if case["masked"]:                                       # classes that this partition never answers with
        C = case["classes"]
        off = torch.rand(C, generator=gen, device=DEV) < 0.25
        off[0] = False
        Z[:, :C].masked_fill_(off, NINF)
    s["Z"] = Z
    if case["op"] == "distill":
        s["top_values"], s["top_ids"], s["tail_lse"] = _teacher(Z, case, gen)
        if not case["tail"]:
            s["tail_lse"] = None
        s["labels"] = None
        if case["labels"]:                                   # a third of the nodes carry no label
            y = torch.randint(0, case["classes"], (case["rows"],), generator=gen, device=DEV, dtype=torch.int32)
            if case["masked"]:
                y.zero_()
            y[torch.rand(case["rows"], generator=gen, device=DEV) < 0.33] = -1
            s["labels"] = y
        s["soft_scale"] = 0.7 * case["temp"] ** 2 / case["rows"]
        s["hard_scale"] = 0.3 / case["rows"]
    return s


# -------------------------------------------------------------- plain forms --

def _grouped(x, case):
    return x.reshape(case["samples"], case["sample_rows"], case["groups"], case["channels"] // case["groups"])


def _per_channel(v, case):
    return v.reshape(1, 1, case["groups"], -1)


def _act(u, act):
    if act == "relu":
        return torch.clamp(u, min=0.0)
    if act == "silu":
        return u * torch.sigmoid(u)
    if act == "gelu":
        return 0.5 * u * (1.0 + torch.erf(u * (1.0 / math.sqrt(2.0))))
    return u


def _act_slope(u, act):
    if act == "relu":
        return (u > 0).to(u.dtype)
    if act == "silu":
        g = torch.sigmoid(u)
        return g * (1.0 + u * (1.0 - g))
    if act == "gelu":
        phi = torch.exp(-0.5 * u * u) * (1.0 / math.sqrt(2.0 * math.pi))
        return 0.5 * (1.0 + torch.erf(u * (1.0 / math.sqrt(2.0)))) + u * phi
    return torch.ones_like(u)


def _norm_fwd_plain(s):
    case = s["case"]
    rows, f = case["samples"] * case["sample_rows"], case["channels"]
    x = _grouped(s["X"][:, :f].float(), case)
    mean = x.mean((1, 3))
    d = x - mean[:, None, :, None]
    rstd = torch.rsqrt((d * d).mean((1, 3)) + s["eps"])
    u = d * rstd[:, None, :, None] * _per_channel(s["gamma"], case) + _per_channel(s["beta"], case)
    return {"Y": _act(u, case["act"]).reshape(rows, f).to(s["X"].dtype), "mean": mean, "rstd": rstd}


def _norm_bwd_plain(s):
    case = s["case"]
    rows, f = case["samples"] * case["sample_rows"], case["channels"]
    gamma, beta = _per_channel(s["gamma"], case), _per_channel(s["beta"], case)
    rstd = s["rstd"][:, None, :, None]
    xhat = (_grouped(s["X"][:, :f].float(), case) - s["mean"][:, None, :, None]) * rstd
    du = _grouped(s["J_out"][:, :f].float(), case) * _act_slope(xhat * gamma + beta, case["act"])
    dbeta = du.sum((0, 1)).reshape(f)
    dgamma = (du * xhat).sum((0, 1)).reshape(f)
    dxhat = du * gamma
    c1 = dxhat.mean((1, 3), keepdim=True)
    c2 = (dxhat * xhat).mean((1, 3), keepdim=True)
    J_in = rstd * (dxhat - c1 - xhat * c2)
    return {"J_in": J_in.reshape(rows, f).to(s["X"].dtype), "dgamma": dgamma, "dbeta": dbeta}


def _order_key(z):
    """Whole numbers in the order of (value, lowest class first); -inf is the smallest value."""
    b = (z + 0.0).view(torch.int32).to(torch.int64)           # -0 counts as +0
    b = torch.where(b < 0, -(b & 0x7FFFFFFF), b)
    ids = torch.arange(z.shape[1], device=z.device, dtype=torch.int64)
    return b * (1 << 20) + ((1 << 20) - 1 - ids)


def _top_plain(s):
    case = s["case"]
    C, K, T = case["classes"], case["top"], case["temp"]
    z = s["Z"][:, :C].float()
    ids = torch.topk(_order_key(z), K, dim=1, largest=True, sorted=True).indices
    values = torch.gather(z, 1, ids)
    rest = torch.scatter(z, 1, ids, NINF) / T
    m = rest.amax(1, keepdim=True)
    safe = torch.where(m > NINF, m, torch.zeros_like(m))
    tail = (safe + torch.log(torch.exp(rest - safe).sum(1, keepdim=True)))[:, 0]
    return {"values": values, "ids": torch.where(values > NINF, ids, torch.full_like(ids, -1)).to(torch.int32),
            "tail_lse": tail}


def _log_sum(x, keep):
    """log of the sum of exp(x) over the kept places of a row; -inf where none is kept."""
    x = torch.where(keep, x, torch.full_like(x, NINF))
    m = x.amax(1, keepdim=True)
    safe = torch.where(m > NINF, m, torch.zeros_like(m))
    return safe + torch.log(torch.exp(x - safe).sum(1, keepdim=True))


def _times(p, x):
    """p x, and 0 where p is 0."""
    return torch.where(p > 0, p * x, torch.zeros_like(p))


def _distill_plain(s):
    case = s["case"]
    C, T = case["classes"], case["temp"]
    z = s["Z"][:, :C].float()
    zt = z / T
    ids, there = s["top_ids"].long(), s["top_ids"] >= 0
    at = torch.where(there, ids, torch.zeros_like(ids))
    t = torch.where(there, s["top_values"] / T, torch.full_like(s["top_values"], NINF))
    some = there.any(1, keepdim=True)
    L = _log_sum(t, there)
    rho = torch.zeros_like(L)
    log_rho = torch.full_like(L, NINF)
    if s["tail_lse"] is not None:
        tail = s["tail_lse"][:, None]
        m = torch.maximum(L, tail)
        total = torch.where(some, m + torch.log(torch.exp(L - m) + torch.exp(tail - m)), torch.zeros_like(m))
        log_rho = torch.where(some, tail - total, torch.full_like(tail, NINF))
        rho = torch.exp(log_rho)
        L = total
    log_p = torch.where(there, t - torch.where(some, L, torch.zeros_like(L)), torch.full_like(t, NINF))
    p = torch.exp(log_p)
    listed_ = torch.zeros(z.shape, dtype=torch.int32, device=z.device).scatter_add_(1, at, there.int()) > 0
    lse = _log_sum(zt, torch.ones_like(listed_))
    log_s = _log_sum(zt, ~listed_)                              # of the rest, before the division by all
    log_q = torch.gather(zt, 1, at) - lse
    soft = _times(p, log_p - log_q).sum(1) + _times(rho, log_rho - (log_s - lse))[:, 0]
    share = torch.exp(log_s - lse)
    r = torch.where(listed_, torch.zeros_like(zt), torch.exp(zt - torch.where(log_s > NINF, log_s, lse)))
    J = torch.where(listed_, torch.exp(zt - lse), r * (share - rho))
    J = torch.where(some, J.scatter_add(1, at, -p), torch.zeros_like(J)) * (s["soft_scale"] / T)
    loss = s["soft_scale"] * torch.where(some[:, 0], soft, torch.zeros_like(soft)).double().sum()
    if s["labels"] is not None:
        y = s["labels"].long()[:, None]
        has = y >= 0
        y = torch.where(has, y, torch.zeros_like(y))
        lse1 = _log_sum(z, torch.ones_like(listed_))
        ce = torch.where(has, lse1 - torch.gather(z, 1, y), torch.zeros_like(lse1))
        loss = loss + s["hard_scale"] * ce.double().sum()
        one = torch.zeros_like(z).scatter_(1, y, 1.0)
        J = J + torch.where(has, torch.exp(z - lse1) - one, torch.zeros_like(z)) * s["hard_scale"]
    return {"J": J.to(s["Z"].dtype), "loss": loss.float().reshape(1)}


# ------------------------------------------------------- the framework's calls --

def _own_buffers(s, B):
    """Outputs and scratch of the framework's calls, kept with the state as a training program does."""
    case = s["case"]
    s["code"] = B.PGCN_BF16 if case["dtype"] == "bf16" else B.PGCN_F32
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device=DEV)
    if case["op"] == "norm":
        n = B.pgcn_group_norm_workspace_size(s["code"], case["channels"], case["groups"], case["samples"],
                                             case["sample_rows"])
        s["act"] = {"none": B.PGCN_ACT_NONE, "relu": B.PGCN_ACT_RELU, "silu": B.PGCN_ACT_SILU,
                    "gelu": B.PGCN_ACT_GELU}[case["act"]]
        s["out"] = torch.empty_like(s["X"])
        if case["way"] == "fwd":
            s["mean"] = empty(case["samples"], case["groups"])
            s["rstd"] = empty(case["samples"], case["groups"])
        else:
            s["dgamma"], s["dbeta"] = empty(case["channels"]), empty(case["channels"])
    elif case["op"] == "top":
        n = B.pgcn_top_logits_workspace_size(s["code"], case["rows"], case["classes"], case["top"])
        s["values"] = empty(case["rows"], case["top"])
        s["ids"] = empty(case["rows"], case["top"], dtype=torch.int32)
        s["tail"] = empty(case["rows"])
    else:
        n = B.pgcn_distill_workspace_size(s["code"], case["rows"], case["classes"], case["top"])
        s["J"], s["loss"] = torch.empty_like(s["Z"]), empty(1)
    s["ws_bytes"] = max(n, 16)
    s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEV)


def _run_own(s):
    from paper_2203_10428_amd import binding as B
    if "ws" not in s:
        _own_buffers(s, B)
    case, stream = s["case"], torch.cuda.current_stream()
    if case["op"] == "norm":
        f = case["channels"]
        ld = s["X"].stride(0)
        common = dict(dtype=s["code"], act=s["act"], channels=f, groups=case["groups"], samples=case["samples"],
                      sample_rows=case["sample_rows"], ld_x=ld, X=s["X"], gamma=s["gamma"], beta=s["beta"],
                      mean=s["mean"], rstd=s["rstd"], workspace=s["ws"], workspace_bytes=s["ws_bytes"], stream=stream)
        if case["way"] == "fwd":
            B.pgcn_group_norm_fwd(ld_y=ld, eps=s["eps"], Y=s["out"], **common)
            return {"Y": s["out"][:, :f], "mean": s["mean"], "rstd": s["rstd"]}
        B.pgcn_group_norm_bwd(ld_j_out=ld, ld_j_in=ld, J_out=s["J_out"], J_in=s["out"], dgamma=s["dgamma"],
                              dbeta=s["dbeta"], **common)
        return {"J_in": s["out"][:, :f], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    C, K = case["classes"], case["top"]
    common = dict(dtype=s["code"], rows=case["rows"], classes=C, ld=s["Z"].stride(0), top=K, ld_top=K,
                  temperature=case["temp"], Z=s["Z"], workspace=s["ws"], workspace_bytes=s["ws_bytes"], stream=stream)
    if case["op"] == "top":
        B.pgcn_top_logits(top_values=s["values"], top_ids=s["ids"], tail_lse=s["tail"], **common)
        return {"values": s["values"], "ids": s["ids"], "tail_lse": s["tail"]}
    B.pgcn_distill_loss_fwd_bwd(top_values=s["top_values"], top_ids=s["top_ids"], tail_lse=s["tail_lse"],
                                labels=s["labels"], soft_scale=s["soft_scale"], hard_scale=s["hard_scale"], J=s["J"],
                                loss_out=s["loss"], **common)
    return {"J": s["J"][:, :C], "loss": s["loss"]}


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    if case["op"] == "norm":
        return _norm_fwd_plain(state) if case["way"] == "fwd" else _norm_bwd_plain(state)
    return _top_plain(state) if case["op"] == "top" else _distill_plain(state)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        n, f = case["samples"] * case["sample_rows"] * case["channels"], case["channels"]
        stats = 8 * case["samples"] * case["groups"]
        if case["way"] == "fwd":
            return {"bytes": 2 * n * e + stats + 8 * f, "flops": 10 * n}
        return {"bytes": 3 * n * e + stats + 16 * f, "flops": 20 * n}
    n, r, K = case["rows"] * case["classes"], case["rows"], case["top"]
    if case["op"] == "top":
        return {"bytes": n * e + r * (8 * K + 4), "flops": 4 * n}
    side = 8 * K + (4 if case["tail"] else 0) + (4 if case["labels"] else 0)
    return {"bytes": 2 * n * e + r * side + 4, "flops": (14 if case["labels"] else 10) * n}


# ------------------------------------------------------------- in 64 bits ----

def _exact_norm(s):
    case = s["case"]
    S, R, G, f = case["samples"], case["sample_rows"], case["groups"], case["channels"]
    x = s["X"][:, :f].double().reshape(S, R, G, f // G)
    ga, be = s["gamma"].double().view(G, f // G), s["beta"].double().view(G, f // G)
    if case["way"] == "fwd":
        mu = x.sum((1, 3)) / (R * (f // G))
        x = x - mu.view(S, 1, G, 1)
        rs = 1.0 / torch.sqrt(x.pow(2).sum((1, 3)) / (R * (f // G)) + s["eps"])
    else:
        mu, rs = s["mean"].double(), s["rstd"].double()
        x = x - mu.view(S, 1, G, 1)
    x = x * rs.view(S, 1, G, 1)
    u = x * ga + be
    a = case["act"]
    if case["way"] == "fwd":
        if a == "relu":
            y = u.relu()
        elif a == "silu":
            y = u / (1.0 + torch.exp(-u))
        elif a == "gelu":
            y = u * 0.5 * torch.special.erfc(-u / math.sqrt(2.0))
        else:
            y = u
        return {"Y": y.reshape(S * R, f), "mean": mu, "rstd": rs}
    if a == "relu":
        k = torch.where(u > 0, 1.0, 0.0).double()
    elif a == "silu":
        e = torch.exp(-u)
        k = (1.0 + e + u * e) / (1.0 + e).pow(2)
    elif a == "gelu":
        k = 0.5 * torch.special.erfc(-u / math.sqrt(2.0)) + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    else:
        k = torch.ones_like(u)
    j = s["J_out"][:, :f].double().reshape(S, R, G, f // G) * k
    del k, u
    db, dg = j.sum((0, 1)), (j * x).sum((0, 1))
    j = j * ga
    n = R * (f // G)
    first, second = j.sum((1, 3)) / n, (j * x).sum((1, 3)) / n
    out = (j - first.view(S, 1, G, 1) - x * second.view(S, 1, G, 1)) * rs.view(S, 1, G, 1)
    return {"J_in": out.reshape(S * R, f), "dgamma": dg.reshape(f), "dbeta": db.reshape(f)}


def _exact_top(s):
    case = s["case"]
    C, K, T = case["classes"], case["top"], case["temp"]
    z = s["Z"][:, :C].double()
    order = torch.sort(z, dim=1, descending=True, stable=True)
    v, i = order.values[:, :K], order.indices[:, :K]
    tail = torch.logsumexp(order.values[:, K:] / T, dim=1) if K < C else \
        torch.full((case["rows"],), NINF, dtype=torch.float64, device=z.device)
    return {"values": v.contiguous(), "ids": i.masked_fill(v == NINF, -1).to(torch.int32), "tail_lse": tail}


def _exact_distill(s):
    """Dense target rows: the listed classes' probabilities, and the rest as one more bucket."""
    case = s["case"]
    C, T, R = case["classes"], float(case["temp"]), case["rows"]
    z = s["Z"][:, :C].double()
    ids, there = s["top_ids"].long(), s["top_ids"] >= 0
    weight = torch.where(there, torch.exp((s["top_values"].double() - s["top_values"].double()[:, :1]) / T), 0.0)
    beyond = torch.zeros(R, 1, dtype=torch.float64, device=z.device)
    if s["tail_lse"] is not None:
        beyond = torch.exp(s["tail_lse"].double()[:, None] - s["top_values"].double()[:, :1] / T)
    some = there.any(1, keepdim=True)
    total = weight.sum(1, keepdim=True) + beyond
    p = torch.where(some, weight / total, 0.0)
    rho = torch.where(some, beyond / total, 0.0)
    dense = torch.zeros_like(z).scatter_add_(1, ids.clamp(min=0), p)
    inside = torch.zeros(R, C, dtype=torch.int32, device=z.device).scatter_add_(1, ids.clamp(min=0), there.int()).bool()
    log_q = torch.log_softmax(z / T, dim=1)
    q = log_q.exp()
    s_rest = torch.where(inside, 0.0, q).sum(1, keepdim=True)
    kl = torch.special.xlogy(dense, dense).sum(1) - torch.where(dense > 0, dense * log_q, 0.0).sum(1)
    kl = kl + (torch.special.xlogy(rho, rho) - torch.special.xlogy(rho, s_rest))[:, 0]
    J = q - dense
    J = torch.where(inside, J, J - q * torch.where(rho > 0, rho / s_rest, 0.0))
    J = torch.where(some, J, 0.0) * (s["soft_scale"] / T)
    loss = s["soft_scale"] * torch.where(some[:, 0], kl, 0.0).sum()
    if s["labels"] is not None:
        y = s["labels"].long()
        has = y >= 0
        lq = torch.log_softmax(z, dim=1)
        y = y.clamp(min=0)
        loss = loss - s["hard_scale"] * torch.where(has, lq.gather(1, y[:, None])[:, 0], 0.0).sum()
        h = lq.exp()
        h[torch.arange(R, device=z.device), y] -= 1.0
        J = J + torch.where(has[:, None], h, 0.0) * s["hard_scale"]
    return {"J": J, "loss": loss.reshape(1)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    return _exact_top(s) if case["op"] == "top" else _exact_distill(s)
