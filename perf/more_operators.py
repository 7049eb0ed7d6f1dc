"""The operators that learn from answers through the lens, and the step that follows: the clipped policy loss with a KL term and the
preference loss, each with its gradient, the norm of many gradients, and AdamW over many tensors with states in 32 or 8 bits.

`listed()` names twelve calls, `draw()` gives others of the same ranges; `prepare`, `run`, `work` and `exact` take a case from
either.  `run` is the plain form in 32 bits (64 for sums over sequences and over gradients), or, where `own` is set, the calls of
paper_2604_06483_amd.binding.  Shapes are those of `paper_2604_06483_amd/workloads.py` (T tokens, hidden size d, vocabulary V) and of
`paper_2604_06483_amd/tune.py`'s translators (a d x d map, its offset and its gate a layer), and generic ragged ones.

States in 8 bits: m in e4m3, v in e5m2, each relative to one power of two a block of 256 elements, the smallest for which the block's
largest value fits.  Both are rounded stochastically, with 16 bits each of one hash a element; a positive v is never rounded to 0.
"""
import math

import torch

own = False

DEV = "cuda:0"
BF16, F32, F64, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
BLOCK = 256
RATE, BETA1, BETA2, TINY = 1e-3, 0.9, 0.999, 1e-8
SEED = 20240
KINDS = ("params", "m", "v", "m_scale", "v_scale", "copies")


def _lens(name, kind, N, d, V, **more):
    return dict({"kind": kind, "N": N, "d": d, "V": V, "temperature": 1.0}, **more, **({"name": name} if name else {}))


def _tensors(name, kind, L, d, rank=0, **more):
    """L translators of hidden size d: a full map (rank 0) or two factors, an offset and a gate each."""
    return dict({"kind": kind, "L": L, "d": d, "rank": rank}, **more, **({"name": name} if name else {}))


def listed():
    return [
        # one sampled token, a direction learned while decoding: one read of the unembedding
        _lens("policy token d4096", "policy", 1, 4096, 128256, kl=0.0, padded=False),
        # a short ragged model's sampled answers in a padded batch, softened
        _lens("policy ragged", "policy", 111, 1608, 50257, kl=0.05, padded=True, temperature=0.7),
        # one layer's 1500 sampled tokens: a policy's step
        _lens("policy trace d4096", "policy", 1500, 4096, 128256, kl=0.02, padded=False),
        # the smallest preference: one pair of single-token answers
        _lens("preference answers d2560", "preference", 2, 2560, 151936, pairs=1, form="logistic", mean=False, padded=False),
        # ragged pairs, some answers empty, rows behind the last; length-normalised, every pair with a weight of its own
        _lens("preference ragged", "preference", 348, 1608, 50257, pairs=9, form="square", mean=True, padded=True),
        # a batch of eight pairs of long answers: more rows than one pass holds, the largest products
        _lens("preference batch d2560", "preference", 6000, 2560, 151936, pairs=8, form="logistic", mean=False, padded=False),
        # a toy translator's gradients: launches are all of it
        _tensors("gradient norm toy", "grad_norm", 1, 256, grad="fp32"),
        # all layers' translators of a small model, gradients in bf16
        _tensors("gradient norm d2560", "grad_norm", 37, 2560, grad="bf16"),
        # a toy translator's step
        _tensors("adamw toy", "adamw", 1, 256, bits=32, param="fp32", grad="fp32", copy=False, clip=False),
        # eight layers' translators, states in 32 bits, clipped, working copies in bf16: the ordinary step
        _tensors("adamw layers d2560", "adamw", 8, 2560, bits=32, param="fp32", grad="fp32", copy=True, clip=True),
        # low-rank translators of a ragged model, parameters in bf16, states in 8 bits: sizes that end inside a block
        _tensors("adamw 8 bit ragged", "adamw", 5, 1608, 77, bits=8, param="bf16", grad="bf16", copy=False, clip=True),
        # twelve large translators, states in 8 bits, gradients in bf16: the largest step
        _tensors("adamw 8 bit d4096", "adamw", 12, 4096, bits=8, param="fp32", grad="bf16", copy=True, clip=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["policy", "policy", "preference", "preference", "grad_norm", "adamw", "adamw", "adamw"])
    # hidden sizes: most models have whole K stages of 64, some only whole 16-byte chunks
    d = 64 * _log(rng, 4, 128) if rng.random() < 0.7 else 8 * _log(rng, 16, 1024)
    if kind in ("policy", "preference"):
        V = _log(rng, 4000, 152064)
        N = max(1, min(6000, int(2.3e12 / (d * V)), _log(rng, 1, 6000)))
        temperature = rng.choice([1.0, 1.0, 0.7, 2.0])
        padded = rng.random() < 0.5
        if kind == "policy":
            return _lens(None, kind, N, d, V, kl=rng.choice([0.0, 0.05, 0.2]), padded=padded, temperature=temperature)
        N = max(2, N)
        return _lens(None, kind, N, d, V, pairs=max(1, min(64, N // 2, _log(rng, 1, 64))), form=rng.choice(["logistic", "hinge", "square"]),
                     mean=rng.random() < 0.5, padded=padded, temperature=temperature)
    rank = 0 if rng.random() < 0.5 else _log(rng, 1, 256)
    each = d * d if rank == 0 else 2 * d * rank
    L = max(1, min(_log(rng, 1, 81), int(2e8 / each)))
    if kind == "grad_norm":
        return _tensors(None, kind, L, d, rank, grad=rng.choice(["fp32", "bf16"]))
    param = rng.choice(["fp32", "fp32", "bf16"])
    return _tensors(None, kind, L, d, rank, bits=rng.choice([8, 32]), param=param, grad=rng.choice(["fp32", "bf16"]),
                    copy=param == "fp32" and rng.random() < 0.5, clip=rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000 + 29)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _lens_inputs(case, seed):
    """Normalised rows, each near a few tokens' own directions; the token of most rows is one of those, of some any."""
    N, d, V, g = case["N"], case["d"], case["V"], _generator(seed)
    W = torch.empty((V, d), dtype=BF16, device=DEV)
    for v0 in range(0, V, 16384):
        W[v0:v0 + 16384] = (0.02 * _normal(g, min(16384, V - v0), d)).to(BF16)
    near = torch.randint(0, V, (N, 4), generator=g, device=DEV)
    gain = torch.rand((N, 4), generator=g, device=DEV) * 7.0       # of the logit
    a = _normal(g, N, d)
    for i in range(4):
        a += (gain[:, i:i + 1] / (0.02 * 0.02 * d)) * W[near[:, i]].float()
    a = (a / (a * a).mean(1, keepdim=True).sqrt()).to(BF16)
    ids = torch.where(torch.rand((N,), generator=g, device=DEV) < 0.1, torch.randint(0, V, (N,), generator=g, device=DEV), near[:, 0])
    if case["padded"]:                                             # rows of a batch that hold no token
        ids = torch.where(torch.rand((N,), generator=g, device=DEV) < 0.1, -1, ids)
    s = {"rows": a, "W_U": W, "ids": ids.to(I32), "temperature": float(case["temperature"])}
    logp = torch.where(ids >= 0, _token_logp(s)[0], 0.0)
    if case["kind"] == "policy":
        s["advantage"] = _normal(g, N)
        # the policy that sampled is a few updates old; no ratio is so near a border of the clipping that its last bits decide
        ratio = torch.exp(0.2 * _normal(g, N))
        ratio = torch.where((ratio - 1.2).abs() < 1e-3, 1.198, torch.where((ratio - 0.8).abs() < 1e-3, 0.802, ratio))
        s["old_logp"] = logp - torch.log(ratio)
        s["ref_logp"] = logp + 0.3 * _normal(g, N) if case["kl"] else None
        s["weight"] = torch.full((N,), 1.0 / N, device=DEV) if not case["padded"] else torch.rand((N,), generator=g, device=DEV) / N
        return s
    P = case["pairs"]
    cuts = torch.randint(0, N + 1, (2 * P - 1,), generator=g, device=DEV).sort().values
    last = N - N // 10 if case["padded"] else N                    # rows behind the last sequence
    ends = torch.cat([torch.zeros((1,), dtype=I64, device=DEV), cuts, torch.full((1,), N, dtype=I64, device=DEV)])
    if not case["padded"]:                                         # even lengths, none empty
        ends = (torch.arange(2 * P + 1, device=DEV) * N) // (2 * P)
    s["offsets"] = ends.clamp(max=last).to(I32)
    s["ref_logp"] = logp + 0.5 * _normal(g, N) - 0.1
    s["weight"] = torch.rand((P,), generator=g, device=DEV) / P if case["padded"] else torch.full((P,), 1.0 / P, device=DEV)
    return s


def _shapes(case):
    d, r = case["d"], case["rank"]
    maps = [(d, d)] if r == 0 else [(d, r), (r, d)]
    return [size for _ in range(case["L"]) for size in maps + [(d,), (d,)]]


def _whole(n):
    return -(-n // BLOCK) * BLOCK


def _views(flat, shapes, each=1):
    """The tensors that share one buffer, each from a whole block on."""
    starts = [0]
    for size in shapes:
        starts.append(starts[-1] + _whole(math.prod(size)))
    if each != 1:
        return [flat[at // each:(at + _whole(math.prod(size))) // each] for at, size in zip(starts, shapes)]
    return [flat[at:at + math.prod(size)].view(size) for at, size in zip(starts, shapes)]


def _scaled(x, dtype, most, top):
    """x in 8 bits, to nearest, and the blocks' powers of two."""
    blocks = x.view(-1, BLOCK)
    scale = _block_scale(blocks.abs().amax(1), top)
    return (blocks / scale[:, None]).clamp(-most, most).to(dtype).view(-1), scale


def _tensor_inputs(case, seed):
    """A user's tensors; all of a kind (parameters, gradients, states) share one buffer, what is between them is 0."""
    g, shapes = _generator(seed), _shapes(case)
    total = sum(_whole(math.prod(size)) for size in shapes)
    grad = F32 if case["grad"] == "fp32" else BF16
    # gradients of a mean over rows: small, their sizes unlike from place to place
    grads = 1e-3 * _normal(g, total) * torch.exp(_normal(g, total // BLOCK)).repeat_interleave(BLOCK)
    inside = torch.zeros((total,), device=DEV)
    [t.fill_(1.0) for t in _views(inside, shapes)]
    s = {"shapes": shapes, "flat_grads": (grads * inside).to(grad)}
    s["grads"] = _views(s["flat_grads"], shapes)
    if case["kind"] == "grad_norm":
        return s
    param = F32 if case["param"] == "fp32" else BF16
    flat = {"params": (0.05 * _normal(g, total) * inside).to(param), "m": 0.3 * grads * inside + 3e-4 * _normal(g, total) * inside,
            "v": (0.5 * grads.square() + 1e-6 * torch.rand((total,), generator=g, device=DEV)) * inside}
    if case["bits"] == 8:
        flat["m"], flat["m_scale"] = _scaled(flat["m"], E4M3, 448.0, 8)
        flat["v"], flat["v_scale"] = _scaled(flat["v"], E5M2, 57344.0, 15)
    if case["copy"]:
        flat["copies"] = flat["params"].to(BF16)
    s["flat"] = flat
    for name in KINDS:
        s[name] = _views(flat[name], shapes, BLOCK if name.endswith("scale") else 1) if name in flat else None
    s["norm"] = _grad_norm(s) if case["clip"] else None
    s["max_norm"] = 0.75
    s["decay"] = 0.01
    s["step"] = 7
    return s


def _inputs(case, seed):
    return _lens_inputs(case, seed) if case["kind"] in ("policy", "preference") else _tensor_inputs(case, seed)


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:
        from paper_2604_06483_amd import binding as LL
        if case["kind"] == "policy":
            need = LL.ll_policy_workspace_bytes(case["N"], case["d"], case["V"])
        elif case["kind"] == "preference":
            need = LL.ll_preference_workspace_bytes(case["N"], case["d"], case["V"], case["pairs"])
        else:
            more = () if case["kind"] == "grad_norm" else tuple(s[n] for n in KINDS)
            s["tensors"] = LL.TensorList(s["grads"], *more)
            need = LL.ll_grad_norm_workspace_bytes(s["tensors"])
        s["workspace"] = torch.empty((max(need, 256),), dtype=torch.uint8, device=DEV)
    return s


# ---- plain forms ----------------------------------------------------------------------------------
def _token_logp(s):
    """Log-probabilities of the rows' tokens (NaN where there is none) and all exponentials over their sum."""
    V = s["W_U"].shape[0]
    z = torch.matmul(s["rows"].float(), s["W_U"].float().t()) / s["temperature"]
    z -= z.max(1, keepdim=True).values
    ids = s["ids"].long()
    valid = (ids >= 0) & (ids < V)
    token = z.gather(1, torch.where(valid, ids, 0)[:, None])[:, 0]
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    return torch.where(valid, token - torch.log(total)[:, 0], math.nan), e / total, valid


def _rows_gradient(s, p, valid, c):
    """c: what the loss gains by a row's log-probability; 0 where there is no token."""
    c = torch.where(valid, c, 0.0) / s["temperature"]
    dz = -c[:, None] * p
    dz.scatter_add_(1, torch.where(valid, s["ids"].long(), 0)[:, None], c[:, None])
    return torch.matmul(dz, s["W_U"].float()).to(BF16)


def _policy(s):
    kl = s["case"]["kl"]
    logp, p, valid = _token_logp(s)
    ratio = torch.exp(logp - s["old_logp"])
    A = s["advantage"]
    direct, clipped = ratio * A, ratio.clamp(0.8, 1.2) * A
    loss = -torch.minimum(direct, clipped)
    c = torch.where(direct <= clipped, -direct, 0.0)
    if s["ref_logp"] is not None:
        q = s["ref_logp"] - logp
        loss = loss + kl * (torch.exp(q) - q - 1.0)
        c = c + kl * (1.0 - torch.exp(q))
    return torch.where(valid, loss, 0.0), logp, _rows_gradient(s, p, valid, s["weight"] * c)


BETA = 0.1


def _pair_loss(form, h, beta):
    if form == "logistic":
        return torch.log1p(torch.exp(-h.abs())) + (-h).clamp(min=0.0), -1.0 / (1.0 + torch.exp(h))
    if form == "hinge":
        return (1.0 - h).clamp(min=0.0), torch.where(h < 1.0, -1.0, 0.0)
    return ((h - 0.5) / beta).square(), 2.0 * (h - 0.5) / (beta * beta)


def _preference(s):
    case = s["case"]
    P, N = case["pairs"], case["N"]
    logp, p, valid = _token_logp(s)
    start, end = s["offsets"][:-1], s["offsets"][1:]
    at = torch.arange(N, device=DEV)
    member = (at[None, :] >= start[:, None]) & (at[None, :] < end[:, None]) & valid[None, :]
    gain = torch.where(valid, logp - s["ref_logp"], 0.0).double()
    length = member.sum(1).clamp(min=1).double() if case["mean"] else torch.ones((2 * P,), dtype=F64, device=DEV)
    score = (member.double() * gain[None, :]).sum(1) / length
    h = BETA * (score[0::2] - score[1::2])
    loss, slope = _pair_loss(case["form"], h, BETA)
    each = s["weight"].double() * slope * BETA
    each = torch.stack([each, -each], 1).reshape(-1) / length
    c = (member.double() * each[:, None]).sum(0).float()
    return loss.float(), score.reshape(P, 2).float(), logp, _rows_gradient(s, p, valid, c)


def _grad_norm(s):
    return torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt().float().reshape(1)


def _u32(x):
    return x & 0xFFFFFFFF


def _hash(x):
    """A permutation of 32-bit words (M. O'Neill's PCG, RXS-M-XS, as a hash): x a tensor of int64, or a number."""
    s = _u32(x * 747796405 + 2891336453)
    w = _u32(((s >> ((s >> 28) + 4)) ^ s) * 277803737)
    return (w >> 22) ^ w


def _random_words(n, step, tensor):
    key = _hash(_u32(_hash(_u32(SEED + _hash(_u32(step)))) + tensor))
    return _hash(torch.arange(n, dtype=I64, device=DEV) ^ key)


def _block_scale(most, top):
    """The smallest power of two, at least 2^-126, that brings `most` to at most 1.75 2^top."""
    bits = most.float().view(I32)
    e = (bits >> 23) - 127 - top + ((bits & 0x7FFFFF) > 0x600000).to(I32)
    return ((e.clamp(min=-126) + 127) << 23).view(F32)


def _stochastic(x, r, mantissa, bias):
    """x >= 0 as the code of an 8-bit float, rounded up with the probability of its distance from the code below; r: 16 random bits."""
    step = 23 - mantissa
    normal = ((x.view(I32).long() + (r << (step - 16))) >> step) - ((127 - bias) << mantissa)
    small = torch.floor(x * 2.0 ** (bias - 1 + mantissa) + r.float() / 65536.0).long()
    return torch.where(x >= 2.0 ** (1 - bias), normal, small)


def _whole_blocks(x):
    n = x.numel()
    return torch.nn.functional.pad(x, (0, -n % BLOCK)).reshape(-1, BLOCK)


def _adamw_one(s, i):
    case = s["case"]
    step, p, g = s["step"], s["params"][i].reshape(-1).float(), s["grads"][i].reshape(-1).float()
    n, eight = p.numel(), case["bits"] == 8
    if s["norm"] is not None:
        g = g * torch.where(s["norm"] > s["max_norm"], s["max_norm"] / s["norm"], 1.0)
    m, v = s["m"][i].reshape(-1).float(), s["v"][i].reshape(-1).float()
    if eight:
        m = (_whole_blocks(m) * s["m_scale"][i][:, None]).reshape(-1)[:n]
        v = (_whole_blocks(v) * s["v_scale"][i][:, None]).reshape(-1)[:n]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    c1, c2 = 1.0 - BETA1 ** step, 1.0 - BETA2 ** step
    p = p * (1.0 - RATE * s["decay"]) - (RATE / c1) * (m / (v.sqrt() / math.sqrt(c2) + TINY))
    words = _random_words(n, step, i) if eight or case["param"] == "bf16" else None
    if eight:
        m_blocks, v_blocks = _whole_blocks(m), _whole_blocks(v)
        m_scale, v_scale = _block_scale(m_blocks.abs().amax(1), 8), _block_scale(v_blocks.amax(1), 15)
        to_m, to_v = (m_blocks / m_scale[:, None]).reshape(-1)[:n], (v_blocks / v_scale[:, None]).reshape(-1)[:n]
        m_code = _stochastic(to_m.abs(), words >> 16, 3, 7).clamp(max=0x7E)
        m_code = torch.where(torch.signbit(to_m), m_code + 128, m_code)
        v_code = _stochastic(to_v, words & 0xFFFF, 2, 15).clamp(max=0x7B)
        v_code = torch.maximum(v_code, (to_v > 0).long())
        m, v = m_code.to(torch.uint8).view(E4M3), v_code.to(torch.uint8).view(E5M2)
        s["m_scale"][i].copy_(m_scale)
        s["v_scale"][i].copy_(v_scale)
    s["m"][i].copy_(m.reshape(s["m"][i].shape))
    s["v"][i].copy_(v.reshape(s["v"][i].shape))
    if s["copies"] is not None:
        s["copies"][i].copy_(p.reshape(s["copies"][i].shape))
    if case["param"] == "bf16":
        bits = p.view(I32).long() + (_hash(words) & 0xFFFF)
        p = ((bits >> 16) << 16).to(I32).view(F32)
    s["params"][i].copy_(p.reshape(s["params"][i].shape))
    return True


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        if kind != "adamw":
            return {"policy": _policy, "preference": _preference, "grad_norm": _grad_norm}[kind](s)
        all(_adamw_one(s, i) for i in range(len(s["params"])))
        s["step"] += 1
        return s["flat"]
    from paper_2604_06483_amd import binding as LL
    if kind == "policy":
        return LL.ll_policy(s["rows"], s["W_U"], s["ids"], s["advantage"], s["old_logp"], ref_logp=s["ref_logp"], weight=s["weight"],
                            clip=(0.2, 0.2), kl=case["kl"], temperature=s["temperature"], workspace=s["workspace"])
    if kind == "preference":
        return LL.ll_preference(s["rows"], s["W_U"], s["ids"], s["offsets"], ref_logp=s["ref_logp"], weight=s["weight"], beta=BETA,
                                form=case["form"], mean=case["mean"], temperature=s["temperature"], workspace=s["workspace"])
    if kind == "grad_norm":
        return LL.ll_grad_norm(s["tensors"], workspace=s["workspace"])
    LL.ll_adamw(s["tensors"], s["step"], rate=RATE, betas=(BETA1, BETA2), eps=TINY, decay=s["decay"], norm=s["norm"],
                max_norm=s["max_norm"], seed=SEED)
    s["step"] += 1
    return s["flat"]


def work(case):
    d = case["d"]
    if case["kind"] in ("policy", "preference"):
        N, V = case["N"], case["V"]
        table = 2 * V * d + 4 * N * d
        if case["kind"] == "policy":
            return {"bytes": table + N * (24 + 4 * (case["kl"] > 0)), "flops": 4 * N * d * V}
        return {"bytes": table + N * 12 + case["pairs"] * 24, "flops": 4 * N * d * V}
    n = sum(math.prod(size) for size in _shapes(case))
    g = 4 if case["grad"] == "fp32" else 2
    if case["kind"] == "grad_norm":
        return {"bytes": n * g + 4, "flops": 2 * n}
    p = 4 if case["param"] == "fp32" else 2
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": int(n * (g + 2 * p + state + 2 * case["copy"])), "flops": 16 * n}


# ---- the definitions in 64 bits -------------------------------------------------------------------
def _exact_lens(case, s):
    """Two sweeps over blocks of the vocabulary: the normaliser, then what the rows receive."""
    N, d, V, T = case["N"], case["d"], case["V"], float(case["temperature"])
    a, W, ids = s["rows"].to(F64), s["W_U"], s["ids"].long()
    blocks = [slice(v, min(V, v + 16384)) for v in range(0, V, 16384)]
    ok = (ids >= 0) & (ids < V)
    lse = torch.full((N,), -math.inf, dtype=F64, device=DEV)
    for b in blocks:
        lse = torch.logaddexp(lse, torch.logsumexp(torch.mm(a, W[b].to(F64).t().contiguous()) / T, 1))
    token = (a * W[torch.where(ok, ids, 0)].to(F64)).sum(1) / T - lse
    logp = torch.where(ok, token, math.nan)
    if case["kind"] == "policy":
        A, kl = s["advantage"].to(F64), float(case["kl"])
        x = token - s["old_logp"].to(F64)
        bounded = torch.where(A > 0, x > math.log(1.2), x < math.log(0.8))
        held = torch.where(A > 0, 1.2 * A, 0.8 * A)
        loss = -torch.where(bounded, held, A * torch.exp(x))
        c = torch.where(bounded, 0.0, -A * torch.exp(x))
        if kl:
            q = s["ref_logp"].to(F64) - token
            loss = loss + kl * (torch.expm1(q) - q)
            c = c - kl * torch.expm1(q)
        c = c * s["weight"].to(F64)
        first = (torch.where(ok, loss, 0.0), logp)
    else:
        P, offsets = case["pairs"], s["offsets"].tolist()
        gain = torch.where(ok, token - s["ref_logp"].to(F64), 0.0)
        c = torch.zeros((N,), dtype=F64, device=DEV)
        losses, scores = [], []
        for i in range(P):
            part = [slice(offsets[2 * i + j], offsets[2 * i + j + 1]) for j in (0, 1)]
            length = [max(1.0, float(ok[q].sum())) if case["mean"] else 1.0 for q in part]
            score = [float(gain[q].sum()) / n for q, n in zip(part, length)]
            h = BETA * (score[0] - score[1])
            if case["form"] == "logistic":
                value, slope = math.log1p(math.exp(-h)), -1.0 / (1.0 + math.exp(h))
            elif case["form"] == "hinge":
                value, slope = max(0.0, 1.0 - h), -1.0 if h < 1.0 else 0.0
            else:
                value, slope = (score[0] - score[1] - 0.5 / BETA) ** 2, 2.0 * (score[0] - score[1] - 0.5 / BETA) / BETA
            for q, n, sign in zip(part, length, (1.0, -1.0)):
                c[q] = sign * BETA * slope * float(s["weight"][i]) / n
            losses.append(value)
            scores.append(score)
        first = (torch.tensor(losses, dtype=F64, device=DEV), torch.tensor(scores, dtype=F64, device=DEV), logp)
    c = torch.where(ok, c, 0.0) / T
    out = c[:, None] * W[torch.where(ok, ids, 0)].to(F64)
    for b in blocks:
        p = torch.exp(torch.mm(a, W[b].to(F64).t().contiguous()) / T - lse[:, None])
        out -= c[:, None] * torch.mm(p, W[b].to(F64))
    return first + (out,)


def _exact_step(case, s):
    """Of states in 8 bits: the values before they are rounded, relative to their block's power of two."""
    x = {k: v.to(F64) for k, v in s["flat"].items() if k != "copies"}
    g = s["flat_grads"].to(F64)
    if s["norm"] is not None:
        g = g * min(1.0, s["max_norm"] / float(torch.linalg.vector_norm(g)))
    m, v = x["m"], x["v"]
    if case["bits"] == 8:
        m, v = m * x["m_scale"].repeat_interleave(BLOCK), v * x["v_scale"].repeat_interleave(BLOCK)
    m = m + (1.0 - BETA1) * (g - m)
    v = v + (1.0 - BETA2) * (g * g - v)
    m_hat, v_hat = m / (1.0 - BETA1 ** s["step"]), v / (1.0 - BETA2 ** s["step"])
    p = x["params"] - RATE * s["decay"] * x["params"] - RATE * m_hat / (v_hat.sqrt() + TINY)
    found = {"params": p, "m": m, "v": v}
    if case["copy"]:
        found["copies"] = p
    if case["bits"] == 8:
        for key, most in (("m", 448.0), ("v", 57344.0)):
            top = found[key].view(-1, BLOCK).abs().max(1).values
            scale = torch.exp2(torch.ceil(torch.log2(top / most)).clamp(min=-126.0))
            found[key + "_scale"] = scale
            found[key] = found[key] / scale.repeat_interleave(BLOCK)
    return found


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] in ("policy", "preference"):
        return _exact_lens(case, s)
    if case["kind"] == "grad_norm":
        return torch.linalg.vector_norm(s["flat_grads"].to(F64)).reshape(1)
    return _exact_step(case, s)
