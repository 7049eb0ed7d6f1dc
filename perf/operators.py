"""The operators that learn through the lens: the norm around a block, log-probabilities of listed tokens, distillation from a
teacher's top tokens, each with its gradient.

`listed()` names twelve calls, `draw()` gives others of the same ranges; `prepare`, `run`, `work` and `exact` take a case from
either.  `run` is the plain form in 32 bits, or, where `own` is set, the calls of paper_2604_06483_amd.binding.  Shapes are those of
`paper_2604_06483_amd/workloads.py` (L captured states, T tokens, hidden size d, vocabulary V, k listed tokens) and generic ragged
ones.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def _norm(name, N, d, grad, gate=None, post=False, scale=1.0):
    """gate: None, "shared" ([d]) or "rows" ([N, d]); post: the block's output has a norm of its own before it is added."""
    return dict({"kind": "norm", "N": N, "d": d, "grad": grad, "gate": gate or "none", "post": post, "scale": scale},
                **({"name": name} if name else {}))


def _lens(name, kind, N, d, V, k, **more):
    return dict({"kind": kind, "N": N, "d": d, "V": V, "k": k, "temperature": 1.0}, **more, **({"name": name} if name else {}))


def listed():
    return [
        # the newest token's states of all 33 layers through a translator's residual and the final norm: launches are most of it
        _norm("norm step d4096", 33, 4096, False, gate="shared", scale=0.5),
        # eight layers' 1500-token traces, a block with norms on both sides and a gate for every token
        _norm("norm trace d8192", 12000, 8192, False, gate="rows", post=True),
        # the gradient for all layers' traces of a small model, one gate for all rows: the parameters' sums are over 55 500 rows
        _norm("norm grad d2560", 55500, 2560, True, gate="shared", scale=0.5),
        # ragged sizes, every input there is
        _norm("norm grad ragged", 777, 1608, True, gate="rows", post=True, scale=0.5),
        # candidate answers of the newest token in all 37 layers of a small model: one read of the unembedding
        _lens("logp step d2560", "logp", 37, 2560, 151936, 10),
        # one layer's 1500-token trace, twenty candidates a token
        _lens("logp trace d4096", "logp", 1500, 4096, 128256, 20),
        # a short ragged model's sampled tokens with an entropy bonus
        _lens("logp grad ragged", "logp_grad", 111, 1608, 50257, 3, entropy=True, temperature=0.7),
        # the chosen token of a 1500-token trace, entropy bonus: a policy's step
        _lens("logp grad d2560", "logp_grad", 1500, 2560, 151936, 1, entropy=True),
        # the smallest lens anyone trains through (a toy model, a unit test)
        _lens("distill tiny", "distill", 64, 256, 4096, 5, ragged=False),
        # one row: a direction learned while decoding
        _lens("distill token d4096", "distill", 1, 4096, 128256, 20, ragged=False),
        # a prompt's rows of a few layers, softened teacher, lists that end early and rows without a teacher
        _lens("distill prompt d5120", "distill", 348, 5120, 151936, 20, ragged=True, temperature=2.0),
        # one layer's whole trace of the largest model against the last layer's read-out: the largest call
        _lens("distill trace d8192", "distill", 1500, 8192, 128256, 20, ragged=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm", "logp", "logp", "logp_grad", "logp_grad", "distill", "distill", "distill"])
    # hidden sizes: most models have whole K stages of 64, some only whole 16-byte chunks
    d = 64 * _log(rng, 4, 128) if rng.random() < 0.7 else 8 * _log(rng, 16, 1024)
    d += 64 if d == 3 * 1024 else 0
    if kind == "norm":
        N = _log(rng, 1, min(60000, 98304000 // d))
        return _norm(None, N, d, rng.random() < 0.6, gate=rng.choice([None, "shared", "rows"]), post=rng.random() < 0.5,
                     scale=rng.choice([1.0, 0.5]))
    V = _log(rng, 4000, 152064)
    N = max(1, min(1536, int(1.57e12 / (d * V)), _log(rng, 1, 1536)))
    temperature = rng.choice([1.0, 1.0, 0.7, 2.0])
    if kind == "distill":
        return _lens(None, kind, N, d, V, rng.randint(1, 32), ragged=rng.random() < 0.5, temperature=temperature)
    more = {"entropy": rng.random() < 0.5} if kind == "logp_grad" else {}
    return _lens(None, kind, N, d, V, _log(rng, 1, 64), temperature=temperature, **more)


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000 + 17)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _norm_inputs(case, seed):
    """Activations with a few outlier channels; the block's output is smaller than the stream that it joins."""
    N, d, g = case["N"], case["d"], _generator(seed)
    outliers = torch.ones((d,), device=DEV)
    outliers[torch.randint(0, d, (4,), generator=g, device=DEV)] = 20.0
    s = {"hidden": (3.0 * _normal(g, N, d) * outliers).to(BF16), "y": _normal(g, N, d).to(BF16),
         "gamma": (1.0 + 0.1 * _normal(g, d)).to(BF16), "gate": None, "gamma_y": None}
    if case["gate"] != "none":
        size = (d,) if case["gate"] == "shared" else (N, d)
        s["gate"] = (0.5 + 0.2 * _normal(g, *size)).to(BF16)
    if case["post"]:
        s["gamma_y"] = (1.0 + 0.1 * _normal(g, d)).to(BF16)
    if case["grad"]:
        s["g_hidden"] = (0.1 * _normal(g, N, d)).to(BF16)
        s["g_normed"] = (0.1 * _normal(g, N, d)).to(BF16)
    return s


def _lens_inputs(case, seed):
    """Normalised rows, each near a few tokens' own directions, so that a handful of tokens hold much of its probability."""
    N, d, V, k, g = case["N"], case["d"], case["V"], case["k"], _generator(seed)
    W = torch.empty((V, d), dtype=BF16, device=DEV)
    for v0 in range(0, V, 16384):
        W[v0:v0 + 16384] = (0.02 * _normal(g, min(16384, V - v0), d)).to(BF16)
    near = torch.randint(0, V, (N, 4), generator=g, device=DEV)
    gain = torch.rand((N, 4), generator=g, device=DEV) * 12.0      # of the logit
    a = _normal(g, N, d)
    for i in range(4):
        a += (gain[:, i:i + 1] / (0.02 * 0.02 * d)) * W[near[:, i]].float()
    a = (a / (a * a).mean(1, keepdim=True).sqrt()).to(BF16)
    ids = torch.randint(0, V, (N, k), generator=g, device=DEV)
    m = min(4, k)
    ids[:, :m] = near[:, :m]
    s = {"rows": a, "W_U": W, "ids": ids.to(torch.int32), "temperature": float(case["temperature"])}
    if case["kind"] == "distill":
        s["scores"] = -torch.cumsum(torch.empty((N, k), device=DEV).exponential_(1.0, generator=g), 1)
        s["weight"] = torch.full((N,), 1.0 / N, device=DEV)
        if case["ragged"]:                                         # lists that end early, one row in ten without a teacher
            length = torch.randint(1, k + 1, (N,), generator=g, device=DEV)
            length = torch.where(torch.rand((N,), generator=g, device=DEV) < 0.1, 0, length)
            s["ids"] = torch.where(torch.arange(k, device=DEV)[None] < length[:, None], s["ids"], -1).to(torch.int32).contiguous()
            s["weight"] = s["weight"] * torch.rand((N,), generator=g, device=DEV)
    if case["kind"] == "logp_grad":
        _, s["lse"], s["entropy"] = _logp(s)
        s["g_logp"] = _normal(g, N, k) / N
        s["g_entropy"] = -0.01 * torch.rand((N,), generator=g, device=DEV) / N if case["entropy"] else None
    return s


def _inputs(case, seed):
    return _norm_inputs(case, seed) if case["kind"] == "norm" else _lens_inputs(case, seed)


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:
        from paper_2604_06483_amd import binding as LL
        kind, N, d = case["kind"], case["N"], case["d"]
        need = 0
        if kind == "norm" and case["grad"]:
            need = LL.ll_block_norm_grad_workspace_bytes(N, d)
        elif kind == "logp":
            need = LL.ll_logp_workspace_bytes(N, d, case["V"], case["k"])
        elif kind == "logp_grad":
            need = LL.ll_logp_grad_workspace_bytes(N, d, case["V"], case["k"])
        elif kind == "distill":
            need = LL.ll_distill_workspace_bytes(N, d, case["V"], case["k"])
        s["workspace"] = torch.empty((max(need, 256),), dtype=torch.uint8, device=DEV)
    return s


# ---- plain forms, 32 bits ------------------------------------------------------------------------
def _rms(x):
    return torch.sqrt((x * x).mean(1, keepdim=True) + EPS)


def _block(s, scale):
    """The block's share u before its gate, gate * scale, and the stream x after it."""
    y = s["y"].float()
    u = y if s["gamma_y"] is None else s["gamma_y"].float() * (y / _rms(y))
    k = torch.full((1, 1), scale, device=DEV) if s["gate"] is None else scale * s["gate"].float()
    return y, u, k, s["hidden"].float() + k * u


def _norm_forward(s):
    _, _, _, x = _block(s, s["case"]["scale"])
    return x.to(BF16), (s["gamma"].float() * (x / _rms(x))).to(BF16)


def _norm_backward(s):
    scale = s["case"]["scale"]
    y, u, k, x = _block(s, scale)
    r = _rms(x)
    xh = x / r
    gn = s["g_normed"].float()
    e = gn * s["gamma"].float()
    dx = s["g_hidden"].float() + (e - xh * (e * xh).mean(1, keepdim=True)) / r
    d_gamma = (gn * xh).sum(0)
    du = k * dx
    d_gate = d_gamma_y = None
    if s["gate"] is not None:
        d_gate = scale * u * dx
        d_gate = d_gate.sum(0) if s["gate"].dim() == 1 else d_gate.to(BF16)
    dy = du
    if s["gamma_y"] is not None:
        ry = _rms(y)
        yh = y / ry
        f = du * s["gamma_y"].float()
        dy = (f - yh * (f * yh).mean(1, keepdim=True)) / ry
        d_gamma_y = (du * yh).sum(0)
    return dx.to(BF16), dy.to(BF16), d_gate, d_gamma_y, d_gamma


def _logits(s):
    return torch.matmul(s["rows"].float(), s["W_U"].float().t()) / s["temperature"]


def _logp(s):
    z = _logits(s)
    m = z.max(1, keepdim=True).values
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    entropy = lse[:, 0] - (e * z).sum(1) / total[:, 0]
    return z.gather(1, s["ids"].long()) - lse, lse[:, 0], entropy


def _logp_backward(s):
    lp = _logits(s) - s["lse"][:, None]
    share = s["g_logp"].sum(1, keepdim=True)
    if s["g_entropy"] is not None:
        share = share + s["g_entropy"][:, None] * (lp + s["entropy"][:, None])
    dz = -torch.exp(lp) * share
    dz.scatter_add_(1, s["ids"].long(), s["g_logp"])
    return torch.matmul(dz / s["temperature"], s["W_U"].float()).to(BF16)


def _distill(s):
    temperature, V = s["temperature"], s["W_U"].shape[0]
    valid = (s["ids"] >= 0) & (s["ids"] < V)
    ids = torch.where(valid, s["ids"], 0).long()
    some = valid.any(1, keepdim=True)
    t = torch.where(valid, s["scores"] / temperature, -math.inf)
    t = torch.where(some, t - torch.where(some, t.max(1, keepdim=True).values, 0.0), 0.0)
    t = torch.where(valid, torch.exp(t), 0.0)
    t = t / torch.where(some, t.sum(1, keepdim=True), 1.0)
    z = _logits(s)
    z = z - z.max(1, keepdim=True).values
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    logq = z.gather(1, ids) - torch.log(total)
    loss = temperature ** 2 * torch.where(t > 0, t * (torch.log(t) - logq), 0.0).sum(1)
    dz = torch.where(some, e / total, 0.0)
    dz.scatter_add_(1, ids, -t)
    dz = dz * (temperature * s["weight"])[:, None]
    return loss, torch.matmul(dz, s["W_U"].float()).to(BF16)


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        if kind == "norm":
            return _norm_backward(s) if case["grad"] else _norm_forward(s)
        return {"logp": _logp, "logp_grad": _logp_backward, "distill": _distill}[kind](s)
    from paper_2604_06483_amd import binding as LL
    if kind == "norm":
        options = {"gate": s["gate"], "scale": case["scale"], "gamma_y": s["gamma_y"]}
        if not case["grad"]:
            return LL.ll_block_norm(s["hidden"], s["y"], s["gamma"], EPS, **options)
        return LL.ll_block_norm_grad(s["hidden"], s["y"], s["gamma"], EPS, s["g_hidden"], s["g_normed"], workspace=s["workspace"],
                                     **options)
    if kind == "logp":
        return LL.ll_logp(s["rows"], s["W_U"], s["ids"], temperature=s["temperature"], workspace=s["workspace"])
    if kind == "logp_grad":
        return LL.ll_logp_grad(s["rows"], s["W_U"], s["ids"], s["lse"], s["entropy"], s["g_logp"], s["g_entropy"],
                               temperature=s["temperature"], workspace=s["workspace"])
    return LL.ll_distill(s["rows"], s["W_U"], s["ids"], s["scores"], temperature=s["temperature"], weight=s["weight"],
                         workspace=s["workspace"])


def work(case):
    N, d = case["N"], case["d"]
    if case["kind"] == "norm":
        rows = (6 if case["grad"] else 4) + (case["gate"] == "rows") * (2 if case["grad"] else 1)
        vectors = 2 * (1 + (case["gate"] == "shared") + case["post"])
        if case["grad"]:
            vectors += 4 * (1 + (case["gate"] == "shared") + case["post"])
        a_value = (24 if case["grad"] else 8) + case["post"] * (16 if case["grad"] else 5)
        return {"bytes": 2 * N * d * rows + d * vectors, "flops": a_value * N * d}
    V, k = case["V"], case["k"]
    table = 2 * V * d + 2 * N * d
    if case["kind"] == "logp":
        return {"bytes": table + N * (8 * k + 8), "flops": 2 * N * d * V}
    if case["kind"] == "logp_grad":
        return {"bytes": table + 2 * N * d + N * (8 * k + 4 + 8 * case["entropy"]), "flops": 4 * N * d * V}
    return {"bytes": table + 2 * N * d + N * (8 * k + 8), "flops": 4 * N * d * V}


# ---- the definitions in 64 bits ------------------------------------------------------------------
def _exact_norm(case, s):
    """Rows in blocks; the derivatives by the chain rule through every named step, x = h + c u first."""
    N, d, c = case["N"], case["d"], float(case["scale"])
    gamma = s["gamma"].to(F64)
    gamma_y = None if s["gamma_y"] is None else s["gamma_y"].to(F64)
    outs = [[] for _ in range(3)]
    sums = [torch.zeros((d,), dtype=F64, device=DEV) for _ in range(3)]      # gate, gamma_y, gamma
    for r0 in range(0, N, 4096):
        part = slice(r0, min(N, r0 + 4096))
        h, y = s["hidden"][part].to(F64), s["y"][part].to(F64)
        u = y
        if gamma_y is not None:
            inv_y = (y.pow(2).sum(1, keepdim=True) / d + EPS).pow(-0.5)
            u = y * inv_y * gamma_y
        gate = None
        if s["gate"] is not None:
            gate = s["gate"].to(F64) if case["gate"] == "shared" else s["gate"][part].to(F64)
        x = h + c * (u if gate is None else gate * u)
        inv = (x.pow(2).sum(1, keepdim=True) / d + EPS).pow(-0.5)
        if not case["grad"]:
            outs[0].append(x)
            outs[1].append(gamma * x * inv)
            continue
        gn, gh = s["g_normed"][part].to(F64), s["g_hidden"][part].to(F64)
        # n = gamma x inv(x), d inv / d x_j = -inv^3 x_j / d
        along = (gn * gamma * x).sum(1, keepdim=True)
        dx = gh + gn * gamma * inv - x * along * inv.pow(3) / d
        outs[0].append(dx)
        sums[2] += (gn * x * inv).sum(0)
        if gate is not None:
            if case["gate"] == "shared":
                sums[0] += (c * u * dx).sum(0)
            else:
                outs[2].append(c * u * dx)
        du = c * dx if gate is None else c * gate * dx
        if gamma_y is not None:
            sums[1] += (du * y * inv_y).sum(0)
            along_y = (du * gamma_y * y).sum(1, keepdim=True)
            du = du * gamma_y * inv_y - y * along_y * inv_y.pow(3) / d
        outs[1].append(du)
    if not case["grad"]:
        return torch.cat(outs[0]), torch.cat(outs[1])
    d_gate = None if s["gate"] is None else sums[0] if case["gate"] == "shared" else torch.cat(outs[2])
    return torch.cat(outs[0]), torch.cat(outs[1]), d_gate, None if gamma_y is None else sums[1], sums[2]


def _exact_lens(case, s):
    """Two sweeps over blocks of the vocabulary: the normaliser, then what the rows receive."""
    kind, N, d, V, k = (case[n] for n in ("kind", "N", "d", "V", "k"))
    T, a, W, ids = float(case["temperature"]), s["rows"].to(F64), s["W_U"], s["ids"]
    blocks = [slice(v, min(V, v + 16384)) for v in range(0, V, 16384)]
    ok = (ids >= 0) & (ids < V)
    at = ids.clamp(0, V - 1).long()
    lse = torch.full((N,), -math.inf, dtype=F64, device=DEV)
    first = torch.zeros((N,), dtype=F64, device=DEV)                          # sum of p z
    z_ids = torch.zeros((N, k), dtype=F64, device=DEV)
    z_all = [torch.mm(a, W[b].to(F64).t().contiguous()) / T for b in blocks]
    for b, z in zip(blocks, z_all):
        lse = torch.logaddexp(lse, torch.logsumexp(z, 1))
        here = (at >= b.start) & (at < b.stop)
        z_ids = torch.where(here, z.gather(1, (at - b.start).clamp(0, b.stop - b.start - 1)), z_ids)
    if kind == "logp":
        for z in z_all:
            first += (torch.exp(z - lse[:, None]) * z).sum(1)
        return z_ids - lse[:, None], lse, lse - first
    loss = None
    if kind == "logp_grad":
        lse, g = s["lse"].to(F64), s["g_logp"].to(F64)
    else:
        some = ok.any(1)
        score = torch.where(ok, s["scores"].to(F64) / T, -math.inf)
        q = torch.where(ok, torch.exp(score - torch.where(some, torch.logsumexp(score, 1), 0.0)[:, None]), 0.0)
        logq = torch.where(ok, score, 0.0) - torch.where(some, torch.logsumexp(score, 1), 0.0)[:, None]
        loss = T * T * torch.where(ok, q * (logq - (z_ids - lse[:, None])), 0.0).sum(1)
        g = q * (T * T * s["weight"].to(F64))[:, None]                        # d L / d log p_id, but for the sign
    out = torch.zeros((N, d), dtype=F64, device=DEV)
    for b, z in zip(blocks, z_all):
        lp = z - lse[:, None]
        dz = -torch.exp(lp) * g.sum(1, keepdim=True)
        if kind == "logp_grad" and s["g_entropy"] is not None:
            dz -= s["g_entropy"].to(F64)[:, None] * torch.exp(lp) * (lp + s["entropy"].to(F64)[:, None])
        here = ok & (at >= b.start) & (at < b.stop)
        dz.scatter_add_(1, torch.where(here, at - b.start, 0), torch.where(here, g, 0.0))
        out += torch.mm(dz / T, W[b].to(F64))
    return out if kind == "logp_grad" else (loss, -out)


def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_norm(case, s) if case["kind"] == "norm" else _exact_lens(case, s)
