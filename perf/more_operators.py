"""The head of the policy and the report on its logits, as cases that can be timed and compared.

The last products of a model, act(x W + b) + r, give the hidden states and the logits that a rollout samples from and an
update scores; a training step takes them back through the activation to x, W and b.  From a row of logits a rollout
server reports the log-prob of the token at hand, the entropy and the likeliest alternatives with their log-probs; an
update on them (an entropy bonus, a distillation on the alternatives) takes all three back to the logits.  Each is
computed here in its plain form, elementary torch operations, and with ``own`` set through ``paper_2606_05597_amd``.

A row's words are those above -1e8.  At temperature tau, log p_v = z_v / tau - log sum exp(z / tau) over them, the entropy
is -sum p log p, the alternatives are the n likeliest words, the lowest index first among equals (-1 with log-prob -inf
where the row has fewer words).  A token outside [0, V) has log-prob 0, a word that is masked -inf; neither passes a
gradient on.  A row without words has entropy 0 and no gradient.

``listed()`` holds the fixed cases, ``draw(rng)`` gives others of the same ranges.
"""
import math

import torch

own = False

LIVE = -1e8            # logits at or below it are masked words
MAX_REPORT = 1.24e9    # elements of the largest report on logits
MAX_GRAD = 6.2e8       # elements of the largest report with its gradient
MAX_FLOPS = 6.7e12     # of the largest product with its gradients
MAX_OUT = 3.2e8        # elements of the largest product's result


# ---- the cases ----------------------------------------------------------------------------------------------------

def listed():
    return [
        # a smoke-sized rollout with five alternatives: launches and host time are all there is
        {"name": "top_tiny", "kind": "top", "dtype": "f32", "T": 4, "V": 1024, "ld": 1024, "n": 5, "tau": 1.0,
         "mask": False},
        # one sequence being decoded, twenty alternatives for each token
        {"name": "top_1_152k", "kind": "top", "dtype": "bf16", "T": 1, "V": 151936, "ld": 151936, "n": 20, "tau": 0.8,
         "mask": False},
        # a serving batch, each sequence at a temperature of its own, some restricted to the words of a grammar
        {"name": "top_64_152k", "kind": "top", "dtype": "bf16", "T": 64, "V": 151936, "ld": 151936, "n": 20,
         "tau": "rows", "mask": True},
        # the log-probs, entropies and alternatives of a batch of finished rollouts
        {"name": "top_8k_152k", "kind": "top", "dtype": "bf16", "T": 8000, "V": 151936, "ld": 151936, "n": 8, "tau": 1.0,
         "mask": False},
        # distillation on the alternatives of an odd vocabulary whose logits are kept in 32 bits
        {"name": "top_grad_3k_32k_odd", "kind": "top_grad", "dtype": "f32", "T": 3001, "V": 32003, "ld": 32003, "n": 16,
         "tau": 1.0, "mask": False},
        # an entropy bonus on a micro-batch, in the columns of a padded head, no alternatives
        {"name": "top_grad_4k_152k_padded", "kind": "top_grad", "dtype": "bf16", "T": 4000, "V": 151669, "ld": 151936,
         "n": 0, "tau": 0.8, "mask": False},
        # the head of a smoke-sized model on a few tokens, logits in 32 bits
        {"name": "linear_tiny", "kind": "linear", "M": 4, "K": 64, "N": 1000, "ldx": 64, "w": "kn", "act": "none",
         "bias": "f32", "residual": False, "out": "f32"},
        # the logits of one decoded token
        {"name": "linear_1_head", "kind": "linear", "M": 1, "K": 3584, "N": 151936, "ldx": 3584, "w": "kn", "act": "none",
         "bias": "none", "residual": False, "out": "bf16"},
        # a rollout's logits for 300 sequences, an odd vocabulary with a bias, a weight kept as [out, in]
        {"name": "linear_300_odd", "kind": "linear", "M": 300, "K": 3584, "N": 32003, "ldx": 3584, "w": "nk",
         "act": "none", "bias": "bf16", "residual": False, "out": "f32"},
        # a residual block in front of the head, as of a draft head, over a batch of tokens
        {"name": "linear_8k_block", "kind": "linear", "M": 8192, "K": 3584, "N": 3584, "ldx": 3584, "w": "nk",
         "act": "silu", "bias": "bf16", "residual": True, "out": "bf16"},
        # the same kind of block in training, on an uneven batch
        {"name": "linear_grad_4k_block", "kind": "linear_grad", "M": 4001, "K": 3584, "N": 3584, "ldx": 3584, "w": "nk",
         "act": "gelu", "bias": "f32", "residual": True, "out": "bf16"},
        # the head in training, for an objective of the caller's own on the logits
        {"name": "linear_grad_2k_head", "kind": "linear_grad", "M": 2048, "K": 3584, "N": 151936, "ldx": 3584, "w": "kn",
         "act": "none", "bias": "none", "residual": False, "out": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of the range: a multiple of 64 or of 8, or any."""
    n, step = _log_int(rng, lo, hi), rng.choice([64, 8, 8, 1])
    return max(step, n // step * step)


def draw(rng):
    kind = rng.choice(["top", "top", "top_grad", "linear", "linear", "linear_grad"])
    if kind.startswith("top"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        V = _log_int(rng, 300, 200000)
        form = rng.choice(["whole", "odd", "padded"])
        if form == "whole":
            V = V // 8 * 8
        ld = (V + 255) // 256 * 256 if form == "padded" else V
        most = (MAX_GRAD if kind == "top_grad" else MAX_REPORT) / (1 if dtype == "bf16" else 2) / ld
        return {"kind": kind, "dtype": dtype, "T": _log_int(rng, 1, max(1, min(20000, int(most)))), "V": V, "ld": ld,
                "n": rng.choice([0, 1, 5, 8, 20, 33, 64]), "tau": rng.choice([1.0, 0.7, 1.3, "rows"]),
                "mask": rng.random() < 0.25}
    K, N = _size(rng, 16, 8192), _size(rng, 16, 151936)
    flops = (6 if kind == "linear_grad" else 2) * K * N
    M = _log_int(rng, 1, max(1, min(8192, int(MAX_FLOPS / flops), int(MAX_OUT / N))))
    out = rng.choice(["bf16", "bf16", "f32"])
    return {"kind": kind, "M": M, "K": K, "N": N, "ldx": K + rng.choice([0, 0, 64, 3]), "w": rng.choice(["kn", "nk"]),
            "act": rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"]),
            "bias": rng.choice(["none", "bf16", "f32"]), "residual": rng.random() < 0.4, "out": out}


# ---- inputs --------------------------------------------------------------------------------------------------------

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _temperature(case, seed):
    """A number where all rows share it, a tensor [T] where each has its own."""
    if case["tau"] != "rows":
        return case["tau"]
    values = torch.tensor([0.6, 0.8, 1.0, 1.0, 1.3], device="cuda")
    return values[torch.randint(0, 5, (case["T"],), generator=_gen(seed), device="cuda")]


def _logits(case, seed):
    """Normal logits with 48 words of each row raised, by up to 6 in the least sure row and up to 20 in the surest; with
    `mask`, every third row has a part of its words left, down to one in 4,096, and every 64th row none."""
    T, V, ld = case["T"], case["V"], case["ld"]
    logits = torch.zeros((T, ld), dtype=_TYPES[case["dtype"]], device="cuda")
    rows = max(1, (1 << 27) // V)
    for c, a in enumerate(range(0, T, rows)):
        n = min(T, a + rows) - a
        g = _gen(seed * 7919 + c)
        z = torch.randn((n, V), generator=g, device="cuda").mul_(2.0)
        at = torch.randint(0, V, (n, 1), generator=g, device="cuda")
        at = (at + torch.arange(48, device="cuda") * max(1, V // 48)) % V
        sure = 6 + 14 * torch.rand((n, 1), generator=g, device="cuda")
        z.scatter_add_(1, at, sure * torch.rand((n, 48), generator=g, device="cuda"))
        if case["mask"]:
            row = torch.arange(a, a + n, device="cuda")[:, None]
            left = torch.exp2(-12 * torch.rand((n, 1), generator=g, device="cuda"))
            left = torch.where(row % 3 == 1, left, 1.0)
            left = torch.where(row % 64 == 63, -1.0, left)
            z.masked_fill_(torch.rand((n, V), generator=g, device="cuda") > left, -math.inf)
        logits[a:a + n, :V] = z
    return logits


def _actions(case, logits, tau, seed):
    """Words drawn from the policy at the row's temperature; one token in fifty is none (-1)."""
    T, V = case["T"], case["V"]
    act = torch.empty(T, dtype=torch.int32, device="cuda")
    rows = max(1, (1 << 27) // V)
    for c, a in enumerate(range(0, T, rows)):
        b = min(T, a + rows)
        noise = torch.rand((b - a, V), generator=_gen(seed * 104729 + c), device="cuda").clamp_(min=1e-30)
        noise = noise.log_().neg_().log_().neg_()
        noise *= tau[a:b, None] if isinstance(tau, torch.Tensor) else tau
        act[a:b] = noise.add_(logits[a:b, :V]).argmax(dim=1)
    none = torch.rand(T, generator=_gen(seed * 31 + 9), device="cuda") < 0.02
    return act.masked_fill_(none, -1)


def _normal(shape, dtype, g, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def prepare(case, seed):
    s = {"case": case}
    g = _gen(seed * 31 + 6)
    if case["kind"].startswith("top"):
        T, n = case["T"], case["n"]
        s["tau"] = _temperature(case, seed * 31 + 5)
        s["logits"] = _logits(case, seed)
        s["act"] = _actions(case, s["logits"], s["tau"], seed)
        if case["kind"] == "top_grad":
            s["dlogp"] = _normal((T,), torch.float32, g)
            s["dent"] = _normal((T,), torch.float32, g, 0.1)
            s["dtop"] = _normal((T, n), torch.float32, g, 1 / max(n, 1)) if n else None
        return s
    M, K, N, bf16 = case["M"], case["K"], case["N"], torch.bfloat16
    s["x"] = _normal((M, case["ldx"]), bf16, g)[:, :K]
    w = _normal((K, N) if case["w"] == "kn" else (N, K), bf16, g, 1 / math.sqrt(K))
    s["w"] = w if case["w"] == "kn" else w.t()
    s["bias"] = None if case["bias"] == "none" else _normal((N,), _TYPES[case["bias"]], g, 0.5)
    s["res"] = _normal((M, N), _TYPES[case["out"]], g) if case["residual"] else None
    if case["kind"] == "linear_grad":
        s["dy"] = _normal((M, N), _TYPES[case["out"]], g, 0.1)
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------

def _top(s):
    c = s["case"]
    V, n = c["V"], c["n"]
    x = s["logits"][:, :V].float()
    live = x > LIVE
    some = live.any(dim=1, keepdim=True)
    tau = s["tau"][:, None] if isinstance(s["tau"], torch.Tensor) else s["tau"]
    z = torch.where(live, x / tau, -math.inf)
    z = z - torch.where(some, z.max(dim=1, keepdim=True).values, 0.0)
    e = torch.exp(z)
    total = torch.where(some, e.sum(dim=1, keepdim=True), 1.0)
    logq = z - torch.log(total)
    p = e / total
    moment = torch.where(live, logq, 0.0)
    ent = -(p * moment).sum(dim=1, keepdim=True)
    act = s["act"].long()[:, None]
    given = (act >= 0) & (act < V)
    at = act.clamp(0, V - 1)
    logp = torch.where(given, logq.gather(1, at), 0.0)
    out = {"logp": logp[:, 0], "entropy": ent[:, 0]}
    if n:
        # values in the order of whole numbers (-0 as 0), above the index from the last up
        bits = torch.where(live, x + 0.0, -math.inf).view(torch.int32)
        bits = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
        key = (bits << 32) + (V - 1 - torch.arange(V, device=x.device))
        ids = V - 1 - (torch.topk(key, min(n, V), dim=1).values & 0xffffffff)
        ids = torch.nn.functional.pad(ids, (0, n - ids.shape[1]))
        there = (torch.arange(n, device=x.device) < live.sum(dim=1, keepdim=True))
        out["top_ids"] = torch.where(there, ids, -1).int()
        out["top_logp"] = torch.where(there, logq.gather(1, ids), -math.inf)
    if c["kind"] == "top":
        return out
    up = torch.where(given & live.gather(1, at), s["dlogp"][:, None], 0.0)
    d = torch.zeros_like(p).scatter_add_(1, at, up)
    if n:
        up_top = torch.where(there, s["dtop"], 0.0)
        d.scatter_add_(1, ids, up_top)
        up = up + up_top.sum(dim=1, keepdim=True)
    d -= p * (up + s["dent"][:, None] * (moment + ent))
    out["dlogits"] = (d / tau).to(s["logits"].dtype)
    return out


def _act(kind, z):
    """act(z) and its derivative."""
    if kind == "none":
        return z, None
    if kind == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if kind == "silu":
        g = 1 / (1 + torch.exp(-z))
        return z * g, g * (1 + z * (1 - g))
    if kind == "gelu":
        cdf = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)


def _linear(s):
    c = s["case"]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y, slope = _act(c["act"], z)
    if s["res"] is not None:
        y = y + s["res"].float()
    out = {"y": y.to(_TYPES[c["out"]])}
    if c["kind"] == "linear":
        return out
    dz = s["dy"].float()
    if slope is not None:
        dz = dz * slope
    out["dx"] = (dz @ w.t()).to(torch.bfloat16)
    dw = x.t() @ dz if c["w"] == "kn" else dz.t() @ x
    out["dw"] = dw.to(torch.bfloat16)
    if s["bias"] is not None:
        out["dbias"] = dz.sum(dim=0).to(s["bias"].dtype)
    return out


def run(s):
    c = s["case"]
    if not own:
        return _top(s) if c["kind"].startswith("top") else _linear(s)
    import paper_2606_05597_amd as grpo
    if c["kind"].startswith("top"):
        logp, ent, ids, top_logp, rows = grpo.grpo_token_logp_top(s["logits"], s["act"], c["n"], temperature=s["tau"],
                                                                 V=c["V"])
        out = {"logp": logp, "entropy": ent}
        if c["n"]:
            out["top_ids"], out["top_logp"] = ids, top_logp
        if c["kind"] == "top_grad":
            d = grpo.grpo_token_logp_top_bwd(s["logits"], s["act"], ids, rows, s["dlogp"], s["dent"], s["dtop"], V=c["V"])
            out["dlogits"] = d[:, :c["V"]] if c["V"] < c["ld"] else d
        return out
    keep = c["kind"] == "linear_grad" and c["act"] != "none"
    y, z = grpo.grpo_linear(s["x"], s["w"], s["bias"], s["res"], act=c["act"], out_dtype=_TYPES[c["out"]], keep_z=keep)
    out = {"y": y}
    if c["kind"] == "linear_grad":
        dbias = None if s["bias"] is None else torch.empty_like(s["bias"])
        out["dx"], dw, _ = grpo.grpo_linear_bwd(s["dy"], s["x"], s["w"], z, act=c["act"], dbias=dbias)
        out["dw"] = dw if c["w"] == "kn" else dw.t()
        if dbias is not None:
            out["dbias"] = dbias
    return out


def work(case):
    if case["kind"].startswith("top"):
        T, V, n, size = case["T"], case["V"], case["n"], 2 if case["dtype"] == "bf16" else 4
        small = T * (12 + 8 * n + (4 if case["tau"] == "rows" else 0))
        if case["kind"] == "top":
            return {"bytes": T * V * size + small, "flops": 6 * T * V}
        return {"bytes": 2 * T * V * size + small + T * (8 + 4 * n), "flops": 14 * T * V}
    M, K, N, out = case["M"], case["K"], case["N"], 2 if case["out"] == "bf16" else 4
    bias = {"none": 0, "bf16": 2, "f32": 4}[case["bias"]]
    n = 2 * M * K + 2 * K * N + bias * N + out * M * N * (2 if case["residual"] else 1)
    if case["kind"] == "linear":
        return {"bytes": n, "flops": 2 * M * K * N}
    return {"bytes": n + out * M * N + 2 * M * K + 2 * K * N + bias * N, "flops": 6 * M * K * N}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------

def _exact_rows(x, tau, act, n, up):
    """Rows x [r, V] in 64 bits: log-probs, entropies, the alternatives' log-probs, dlogits (None without `up`)."""
    V = x.shape[1]
    x = x.masked_fill(x <= LIVE, -math.inf)
    words = (x > -math.inf).sum(dim=1)
    empty = words == 0
    lse = torch.logsumexp(x / tau[:, None], dim=1).masked_fill(empty, 0.0)
    logq = x / tau[:, None] - lse[:, None]
    p = torch.exp(logq)
    ent = torch.special.entr(p).sum(dim=1)
    inside = (act >= 0) & (act < V)
    pick = torch.where(inside, act, 0)
    logp = torch.where(inside, logq[torch.arange(len(act), device=x.device), pick], 0.0)
    order = torch.argsort(x, dim=1, descending=True, stable=True)[:, :n] if n else None
    tops = logq.gather(1, order) if n else None
    if n > V:
        tops = torch.nn.functional.pad(tops, (0, n - V), value=-math.inf)
    if up is None:
        return logp, ent, tops, None
    dlogp, dent, dtop = up
    coef = torch.zeros_like(x)
    row = torch.arange(len(act), device=x.device)
    good = inside & (x[row, pick] > -math.inf)
    coef[row[good], pick[good]] += dlogp[good].double()
    if n:
        kept = torch.arange(order.shape[1], device=x.device) < words[:, None]
        coef.scatter_add_(1, order, dtop[:, :order.shape[1]].double() * kept)
    # d/dz of sum_v coef_v log p_v + g H
    d = coef - p * coef.sum(dim=1, keepdim=True)
    d += dent.double()[:, None] * (torch.special.entr(p) - p * ent[:, None])
    return logp, ent, tops, d / tau[:, None]


def _exact_top(s):
    c = s["case"]
    T, V, n, grad = c["T"], c["V"], c["n"], c["kind"] == "top_grad"
    tau = s["tau"].double() if isinstance(s["tau"], torch.Tensor) else torch.full((T,), float(s["tau"]),
                                                                                  dtype=torch.float64, device="cuda")
    parts = []
    rows = max(1, (1 << 26) // V)
    for a in range(0, T, rows):
        b = min(T, a + rows)
        up = (s["dlogp"][a:b], s["dent"][a:b], s["dtop"][a:b] if n else None) if grad else None
        parts.append(_exact_rows(s["logits"][a:b, :V].double(), tau[a:b], s["act"][a:b].long(), n, up))
    logp, ent, tops, d = zip(*parts)
    out = {"logp": torch.cat(logp), "entropy": torch.cat(ent)}
    if n:
        out["top_ids"], out["top_logp"] = None, torch.cat(tops)
    if grad:
        out["dlogits"] = torch.cat(d)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("top"):
        return _exact_top(s)
    x, w = s["x"].double(), s["w"].double()
    z = (torch.matmul(x, w) if s["bias"] is None else torch.addmm(s["bias"].double(), x, w)).requires_grad_()
    a = {"none": lambda t: 1.0 * t, "relu": torch.nn.functional.relu, "silu": torch.nn.functional.silu,
         "gelu": torch.nn.functional.gelu,
         "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[case["act"]](z)
    y = a.detach() if s["res"] is None else a.detach() + s["res"].double()
    out = {"y": y}
    if case["kind"] == "linear":
        return out
    dz, = torch.autograd.grad(a, z, s["dy"].double())
    out["dx"] = torch.matmul(dz, w.transpose(0, 1))
    out["dw"] = torch.matmul(x.transpose(0, 1), dz) if case["w"] == "kn" else torch.matmul(dz.transpose(0, 1), x)
    if s["bias"] is not None:
        out["dbias"] = dz.sum(0)
    return out
