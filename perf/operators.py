"""Performance cases of the operators on score rows: log probabilities with top alternatives, and distillation.

``log_probs``     log probability and rank of a given class per row, log normaliser, entropy and the top
                  alternatives (``sb_log_probs``), on the booster's column-major scores or a network's row-major logits;
``distill_loss``  the distillation loss of every row against a teacher's top list (``sb_distill_loss``);
``distill_grad``  its derivatives for a boosting step: gradients, column norms and, where asked for, the diagonal
                  hessians with their row means and the loss (``sb_distill_gradients``).

Inputs are drawn on the GPU from the seed: student scores as a model part-way through training has them, teachers that
agree with the student in part, a few rows without a label and a few whose teacher list is short or empty (unused slots
hold class -1 and a value that is not a number).
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # One answer being served: the five best of 1000 classes of one row.
        dict(name="lp_1x1000_top5", op="log_probs", n=1, d=1000, order="row", dtype="f32", k=5, T=1.0, labels=False),
        # The evaluation set of a small dataset: loss, rank and three alternatives a row.
        dict(name="lp_20k_d10_top3", op="log_probs", n=20_000, d=10, order="col", dtype="f32", k=3, T=1.0, labels=True),
        # The booster's scores on the synthetic timing experiment (2M rows, 100 classes) after a round.
        dict(name="lp_2m_d100_top10", op="log_probs", n=2_000_000, d=100, order="col", dtype="f32", k=10, T=1.0,
             labels=True),
        # A many-class booster as a teacher: the lists that its student learns from, odd row count, softened.
        dict(name="lp_300k_d1000_top32", op="log_probs", n=300_007, d=1000, order="col", dtype="f32", k=32, T=2.0,
             labels=False),
        # A network as a teacher: half-precision logits of a dataset, rows one after the other.
        dict(name="lp_200k_d1000_f16_top16", op="log_probs", n=200_001, d=1000, order="row", dtype="f16", k=16, T=2.0,
             labels=True),
        # A network with a very wide output: few long rows.
        dict(name="lp_4k_d65000_bf16_top20", op="log_probs", n=4_099, d=65_000, order="row", dtype="bf16", k=20, T=1.0,
             labels=True),
        # The evaluation set of a small student.
        dict(name="dl_10k_d20_k5", op="distill_loss", n=10_000, d=20, k=5, T=2.0, alpha=0.3, teacher="logits",
             labels=True),
        # The evaluation set of a large student, log probabilities kept by the teacher.
        dict(name="dl_1m_d100_k10", op="distill_loss", n=1_000_003, d=100, k=10, T=1.0, alpha=0.0, teacher="log_probs",
             labels=False),
        # A boosting step of a small student: launches count.
        dict(name="dg_20k_d10_k3", op="distill_grad", n=20_000, d=10, k=3, T=1.0, alpha=0.5, teacher="logits",
             labels=True, hess=True),
        # A boosting step of the synthetic timing experiment with softened targets and labels.
        dict(name="dg_2m_d100_k10", op="distill_grad", n=2_000_000, d=100, k=10, T=2.0, alpha=0.3, teacher="logits",
             labels=True, hess=False),
        # A many-class student, long lists, hessians for the leaf values.
        dict(name="dg_300k_d1000_k32", op="distill_grad", n=300_007, d=1000, k=32, T=2.0, alpha=0.0, teacher="log_probs",
             labels=False, hess=True),
        # More classes than a block's registers hold.
        dict(name="dg_20k_d5003_k64", op="distill_grad", n=20_001, d=5_003, k=64, T=1.5, alpha=0.1, teacher="logits",
             labels=True, hess=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges; none costs more than the largest listed ones."""
    op = rng.choice(["log_probs", "log_probs", "distill_loss", "distill_grad", "distill_grad"])
    T = rng.choice([0.5, 1.0, 1.0, 2.0, 4.0])
    if op == "log_probs":
        order = rng.choice(["col", "row"])
        if order == "col":
            d, dtype = _log_int(rng, 2, 5_000), "f32"
        else:
            d, dtype = _log_int(rng, 2, 65_535), rng.choice(["f32", "f16", "bf16"])
        n = min(_log_int(rng, 1, 2_000_000), max(1, 200_000_000 // d))
        return dict(op=op, n=n, d=d, order=order, dtype=dtype, k=rng.randint(0, min(d, 64)), T=T,
                    labels=rng.random() < 0.7)
    d = _log_int(rng, 2, 5_000)
    n = min(_log_int(rng, 1, 2_000_000), max(1, 150_000_000 // d))
    case = dict(op=op, n=n, d=d, k=rng.randint(1, min(d, 64)), T=T, alpha=rng.choice([0.0, 0.1, 0.5]),
                teacher=rng.choice(["logits", "log_probs"]), labels=True)
    if case["alpha"] == 0.0:
        case["labels"] = False
    if op == "distill_grad":
        case["hess"] = rng.random() < 0.5
    return case


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n, d, k = case["n"], case["d"], case["k"]
    st = dict(case=case)
    if case["labels"]:
        y = torch.randint(0, d, (n,), generator=g, device=DEV, dtype=torch.int32)
        y[torch.rand(n, generator=g, device=DEV) < 0.01] = -1
        st["labels"] = y
    else:
        st["labels"] = None
    if case["op"] == "log_probs":
        shape = (d, n) if case["order"] == "col" else (n, d)
        st["F"] = (torch.randn(shape, generator=g, device=DEV) * 2.0).to(DTYPES[case["dtype"]])
        for name, t in (("logp", torch.float32), ("rank", torch.int32)):
            st[name] = torch.empty(n, dtype=t, device=DEV) if case["labels"] else None
        st["lse"] = torch.empty(n, dtype=torch.float32, device=DEV)
        st["entropy"] = torch.empty(n, dtype=torch.float32, device=DEV)
        st["top_id"] = torch.empty((k, n), dtype=torch.int32, device=DEV) if k else None
        st["top_logp"] = torch.empty((k, n), dtype=torch.float32, device=DEV) if k else None
    else:
        F = torch.randn((d, n), generator=g, device=DEV) * 1.5
        z = torch.randn((d, n), generator=g, device=DEV)
        z += F
        # the teacher's list of a row: its k largest, class by class in the framework's column-major order
        val, idx = torch.topk(z.t().contiguous(), k, dim=1)
        if case["teacher"] == "log_probs":
            val = (val - torch.logsumexp(z, 0)[:, None] * (1.0 / case["T"])) if case["T"] == 1.0 else \
                val / case["T"] - torch.logsumexp(z / case["T"], 0)[:, None]
        del z
        val, idx = val.t().contiguous(), idx.t().to(torch.int32).contiguous()
        used = torch.full((n,), k, device=DEV)
        r = torch.rand(n, generator=g, device=DEV)
        used[r < 0.05] = (k + 1) // 2
        used[r < 0.01] = 0
        unused = torch.arange(k, device=DEV)[:, None] >= used[None, :]
        idx[unused] = -1
        val[unused] = float("nan")
        st.update(F=F, t_id=idx, t_val=val, loss=torch.empty(n, dtype=torch.float32, device=DEV))
        if case["op"] == "distill_grad":
            st["G"] = torch.empty((d, n), dtype=torch.float32, device=DEV)
            st["norm2"] = torch.empty(d, dtype=torch.float64, device=DEV)
            st["hess"] = torch.empty((d, n), dtype=torch.float32, device=DEV) if case["hess"] else None
            st["h_row"] = torch.empty(n, dtype=torch.float32, device=DEV) if case["hess"] else None
    if own:
        from paper_2211_12858_amd import _lib as L
        from paper_2211_12858_amd.driver import workspace
        call = L.SB_CALL_LOG_PROBS if case["op"] == "log_probs" else L.SB_CALL_DISTILL
        st["ws"] = workspace(L.sb_workspace_bytes(call, n=n, d=d, k=k), DEV)
    return st


def _outputs(case, st):
    """The outputs that a case asks for, by name."""
    if case["op"] == "log_probs":
        names = (["logp", "rank"] if case["labels"] else []) + ["lse", "entropy"] + (
            ["top_id", "top_logp"] if case["k"] else [])
    elif case["op"] == "distill_loss":
        names = ["loss"]
    else:
        names = ["G", "norm2"] + (["hess", "h_row", "loss"] if case["hess"] else [])
    # the norms are those of the gradients as stored in 32 bits, so 32 bits of them mean something
    return {name: st[name].float() if name == "norm2" else st[name] for name in names}


def run(st):
    case = st["case"]
    if own:
        return _run_own(case, st)
    if case["op"] == "log_probs":
        return _outputs(case, _plain_log_probs(case, st))
    return _outputs(case, _plain_distill(case, st))


# ---------------------------------------------------------------- the framework's calls
def _run_own(case, st):
    from paper_2211_12858_amd import _lib as L
    n, d, k, ws = case["n"], case["d"], case["k"], st["ws"]
    if case["op"] == "log_probs":
        col = case["order"] == "col"
        L.sb_log_probs(st["F"], L.DTYPE[case["dtype"]], L.SB_COLUMN_MAJOR if col else L.SB_ROW_MAJOR, n, d, n if col else d,
                       case["T"], st["labels"], st["logp"], st["rank"], st["lse"], st["entropy"], k, st["top_id"],
                       st["top_logp"], n, ws, ws.numel())
    elif case["op"] == "distill_loss":
        L.sb_distill_loss(st["F"], n, d, n, case["T"], case["alpha"], st["labels"], L.TEACHER[case["teacher"]], k,
                          st["t_id"], st["t_val"], n, st["loss"], ws, ws.numel())
    else:
        L.sb_distill_gradients(st["F"], n, d, n, case["T"], case["alpha"], st["labels"], L.TEACHER[case["teacher"]], k,
                               st["t_id"], st["t_val"], n, st["loss"] if case["hess"] else None, st["G"], n, st["hess"], n,
                               st["h_row"], st["norm2"], ws, ws.numel())
    return _outputs(case, st)


# ---------------------------------------------------------------- plain forms, 32 bits
def _plain_log_probs(case, st):
    F = st["F"].float() if case["order"] == "row" else st["F"].t().contiguous()  # (n, d)
    d, k, T = case["d"], case["k"], case["T"]
    m = F.amax(1, keepdim=True)
    z = (F - m) / T
    e = torch.exp(z)
    s = e.sum(1)
    log_s = torch.log(s)
    out = dict(lse=m[:, 0] / T + log_s, entropy=log_s - (e * z).sum(1) / s)
    if case["labels"]:
        y = st["labels"].long()
        has = (y >= 0) & (y < d)
        a = F.gather(1, y.clamp(0, d - 1)[:, None])
        before = torch.arange(d, device=DEV)[None, :] < y[:, None]
        rank = ((F > a) | ((F == a) & before)).sum(1)
        out["logp"] = torch.where(has, (a - m)[:, 0] / T - log_s, 0.0)
        out["rank"] = torch.where(has, rank, -1).to(torch.int32)
    if k:
        # stable: equal scores stay in the order of their classes
        top, idx = torch.sort(F + 0.0, dim=1, descending=True, stable=True)
        out["top_id"] = idx[:, :k].t().to(torch.int32).contiguous()
        out["top_logp"] = ((top[:, :k] - m) / T - log_s[:, None]).t().contiguous()
    return out


def _plain_distill(case, st):
    F, T, alpha, d = st["F"], case["T"], case["alpha"], case["d"]
    m = F.amax(0)
    z = F - m
    used = (st["t_id"] >= 0) & (st["t_id"] < d)
    tid = st["t_id"].long().clamp(0, d - 1)
    if case["teacher"] == "logits":
        v = torch.where(used, st["t_val"], -torch.inf)
        u = (v - v.amax(0).clamp(min=-3e38)) / T
        e = torch.exp(u)
        total = e.sum(0)
        q = e / total.clamp(min=1e-30)
        log_q = u - torch.log(total)
    else:
        log_q = torch.where(used, st["t_val"], -torch.inf)
        q = torch.exp(log_q)
    Q = q.sum(0)
    eT = torch.exp(z / T)
    sT = eT.sum(0)
    pT = eT / sT
    log_pT = z.gather(0, tid) / T - torch.log(sT)
    out = dict(loss=(1.0 - alpha) * T * T * torch.where(q > 0, q * (log_q - log_pT), 0.0).sum(0))
    target = torch.zeros_like(F).scatter_add_(0, tid, (1.0 - alpha) * T * q)
    if alpha > 0.0:
        y = st["labels"].long()
        has = (y >= 0) & (y < d)
        yc = y.clamp(0, d - 1)[None, :]
        A = torch.where(has, alpha, 0.0)
        e1 = torch.exp(z)
        s1 = e1.sum(0)
        out["loss"] = out["loss"] - A * (z.gather(0, yc)[0] - torch.log(s1))
        if case["op"] == "distill_loss":
            return out
        p1 = e1 / s1
        target.scatter_add_(0, yc, A[None, :])
        out["G"] = A * p1 + (1.0 - alpha) * T * Q * pT - target
        h = A * (p1 * (1.0 - p1)) + (1.0 - alpha) * Q * (pT * (1.0 - pT))
    else:
        if case["op"] == "distill_loss":
            return out
        out["G"] = T * Q * pT - target
        h = Q * (pT * (1.0 - pT))
    out["hess"] = h
    out["h_row"] = h.mean(0)
    out["norm2"] = out["G"].double().square().sum(1)
    return out


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    T, d, k = case["T"], case["d"], case["k"]
    if case["op"] == "log_probs":
        a = st["F"].double() if case["order"] == "row" else st["F"].double().t()
        lse = torch.logsumexp(a / T, 1)
        lp = a / T - lse[:, None]
        out = dict(lse=lse, entropy=-(lp.exp() * lp).sum(1))
        if case["labels"]:
            y = st["labels"].long()
            out["logp"] = torch.where(y >= 0, lp.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
            out["rank"] = None
        if k:
            out["top_id"] = None
            out["top_logp"] = lp.topk(k, dim=1).values.t().contiguous()
        return _outputs(case, out)
    a = st["F"].double()
    lpT = torch.log_softmax(a / T, 0)
    on = st["t_id"] >= 0
    tid = torch.where(on, st["t_id"], 0).long()
    v = torch.where(on, st["t_val"].double(), -torch.inf)
    if case["teacher"] == "logits":
        v = v / T
        lq = torch.where(on, v - torch.logsumexp(v, 0), -torch.inf)
    else:
        lq = v
    q = lq.exp()
    soft = 1.0 - case["alpha"]
    kl = torch.where(on, q * (torch.where(on, lq, 0.0) - lpT.gather(0, tid)), 0.0).sum(0)
    out = dict(loss=soft * T * T * kl)
    Q = q.sum(0)
    pT = lpT.exp()
    del lpT
    G = soft * T * Q * pT
    h = soft * Q * pT * (1.0 - pT)
    del pT
    G.scatter_add_(0, tid, -soft * T * q)
    if case["alpha"] > 0.0:
        lp1 = torch.log_softmax(a, 0)
        y = st["labels"].long()
        A = torch.where(y >= 0, case["alpha"], 0.0).double()
        yc = y.clamp(min=0)[None, :]
        out["loss"] = out["loss"] - A * lp1.gather(0, yc)[0]
        p1 = lp1.exp_()
        G += A * p1
        h += A * p1 * (1.0 - p1)
        G.scatter_add_(0, yc, -A[None, :])
    out.update(G=G, hess=h, h_row=h.mean(0), norm2=G.square().sum(1))
    return _outputs(case, out)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    n, d, k = case["n"], case["d"], case["k"]
    labels = 4 * n if case["labels"] else 0
    if case["op"] == "log_probs":
        read = n * d * (4 if case["dtype"] == "f32" else 2) + labels
        return {"bytes": read + 8 * n + 2 * labels + 8 * n * k, "flops": 6 * n * d}
    read = 4 * n * d + 8 * n * k + labels
    if case["op"] == "distill_loss":
        return {"bytes": read + 4 * n, "flops": 6 * n * d}
    wrote = 4 * n * d + 8 * d + (4 * n * d + 8 * n if case["hess"] else 0)
    return {"bytes": read + wrote, "flops": 12 * n * d}
