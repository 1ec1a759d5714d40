"""The operators of a decode layer's feed-forward half, as measurable cases.

Four kinds of pass, each a step between a layer's attention block and the next
layer:

* ``linear``: a product with packed weights and its epilogue -- bias,
  activation, gate, residual -- in bf16 or, for a router, in fp32;
* ``route``: each token's experts and their weights from the router's logits;
* ``experts``: the chosen experts' gated products for a few tokens, weighted,
  summed and added to the residual;
* ``norm``: a block's output normed, gated, scaled and added to the residual,
  and the RMSNorm before the next block.

A case fixes how many tokens each expert is asked for by; the seed decides
which experts and tokens these are, and every value.
"""
from __future__ import annotations

import math

import numpy as np
import torch

#: False: ``run`` computes the operators with elementary torch operations; True: with the library.
own = False

EPS = 1e-6


def _linear(**kw):
    return dict(dict(kind="linear", batch=1, k=4096, n=4096, act="none", gated=False, bias=False, residual=False,
                     f32=False), **kw)


def _route(**kw):
    return dict(dict(kind="route", tokens=1, experts=128, top_k=8, scoring="softmax", renormalise=True, bias=False,
                     scale=1.0, masked=0), **kw)


def _experts(**kw):
    return dict(dict(kind="experts", tokens=1, hidden=2048, inter=768, experts=128, top_k=8, act="silu", residual=True,
                     idle=0), **kw)


def _norm(**kw):
    return dict(dict(kind="norm", rows=1, hidden=4096, post=True, pre=True, gate="none", scale=1.0, offset=0.0), **kw)


def listed():
    return [
        # a serving batch's router logits, kept in fp32: latency
        _linear(name="linear_router_b64", batch=64, k=2048, n=128, f32=True),
        # gate and up products of a dense feed-forward layer for a few requests: weight bandwidth
        _linear(name="linear_gate_up_b16", batch=16, k=4096, n=14336, act="silu", gated=True),
        # an ungated feed-forward layer with biases, an odd batch
        _linear(name="linear_gelu_b101", batch=101, k=5120, n=20480, act="gelu", bias=True),
        # the product back to the hidden size of a large batch, added to the residual stream
        _linear(name="linear_down_b200", batch=200, k=14336, n=4096, bias=True, residual=True),
        # one request's choice of experts: the smallest call
        _route(name="route_single"),
        # a large batch over 256 experts with sigmoid scores, a balancing bias and a scale
        _route(name="route_sigmoid_b256", tokens=256, experts=256, scoring="sigmoid", bias=True, scale=2.5),
        # one request over many small experts: latency
        _experts(name="experts_single"),
        # a small serving batch over the same experts: most of them are read for a token or two
        _experts(name="experts_b16", tokens=16),
        # an odd batch, some of its slots idle, experts of an odd width
        _experts(name="experts_b61_idle", tokens=61, inter=1408, experts=64, top_k=6, idle=3),
        # a large batch over a few large experts: the largest
        _experts(name="experts_b200_large", tokens=200, hidden=4096, inter=14336, experts=8, top_k=2),
        # the norms around a block of a serving batch: latency
        _norm(name="norm_b64", rows=64),
        # a prompt's rows with a gate of their own each, norm before the next block only: bandwidth
        _norm(name="norm_prompt_gated", rows=8191, hidden=5120, post=False, gate="rows", scale=0.5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(("linear",) * 4 + ("route",) * 2 + ("experts",) * 5 + ("norm",) * 2)
    if kind == "linear":
        c = _linear(batch=_log_int(rng, 1, 256), k=32 * _log_int(rng, 16, 512), n=16 * _log_int(rng, 4, 1792),
                    act=rng.choice(("none", "silu", "gelu", "gelu_tanh", "relu")), gated=rng.random() < 0.4,
                    bias=rng.random() < 0.5, residual=rng.random() < 0.4, f32=rng.random() < 0.25)
        while c["n"] * c["k"] * (2 if c["gated"] else 1) > 150_000_000:
            c["n"] = max(16, c["n"] // 32 * 16)
        return c
    if kind == "route":
        experts = rng.choice((8, 16, 60, 64, 128, 256))
        return _route(tokens=_log_int(rng, 1, 8192), experts=experts, top_k=rng.randint(1, min(8, experts)),
                      scoring=rng.choice(("softmax", "sigmoid")), renormalise=rng.random() < 0.7,
                      bias=rng.random() < 0.4, scale=rng.choice((1.0, 1.0, 2.5)),
                      masked=rng.choice((0, 0, 1, experts // 2)))
    if kind == "experts":
        experts = rng.choice((8, 16, 32, 64, 128))
        c = _experts(tokens=_log_int(rng, 1, 256), hidden=32 * _log_int(rng, 32, 160), inter=32 * _log_int(rng, 11, 448),
                     experts=experts, top_k=rng.randint(1, min(8, experts)), act=rng.choice(("silu", "silu", "gelu_tanh")),
                     residual=rng.random() < 0.6)
        while c["hidden"] * c["inter"] * experts > 450_000_000:
            c["inter"] = max(32, c["inter"] // 64 * 32)
        while c["hidden"] * c["inter"] * c["tokens"] * c["top_k"] > 20_000_000_000:
            c["tokens"] = max(1, c["tokens"] // 2)
        if c["tokens"] > 4 and rng.random() < 0.2:
            c["idle"] = rng.randint(1, c["tokens"] // 3)
        return c
    c = _norm(rows=_log_int(rng, 1, 8192), hidden=8 * _log_int(rng, 64, 1024), post=rng.random() < 0.6,
              pre=rng.random() < 0.8, gate=rng.choice(("none", "none", "features", "rows")),
              scale=rng.choice((1.0, 1.0, 0.5)), offset=rng.choice((0.0, 0.0, 1.0)))
    while c["rows"] * c["hidden"] > 41_000_000:
        c["rows"] = max(1, c["rows"] // 2)
    return c


# ------------------------------------------------------------------ inputs
def _choices(case):
    """Experts [tokens, top_k] of a case, popular ones more often, none twice for a token; idle tokens have
    none (-1).  The seed renames the experts and reorders the tokens."""
    t, e, k = case["tokens"], case["experts"], case["top_k"]
    rng = np.random.default_rng([t, e, k, 11])
    popularity = rng.normal(0.0, 0.7, size=e)
    ids = np.argsort(-(popularity + rng.gumbel(size=(t, e))), axis=1, kind="stable")[:, :k].astype(np.int32)
    ids[:case["idle"]] = -1
    return ids


class _Values:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(1_000_003 * (seed + 1))

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=self.gen)

    def hidden(self, *shape):
        """Normed hidden states: a few features much larger than the rest."""
        x = self.normal(*shape)
        x[..., 5::509] *= 8
        return x


def _inputs(case, seed):
    """Everything the seed decides; weights as a checkpoint has them, one row per output feature."""
    v = _Values(seed)
    rng = np.random.default_rng([seed, 12])
    kind = case["kind"]
    s = dict(case=case)
    if kind == "linear":
        b, k, n = case["batch"], case["k"], case["n"]
        rows = 2 * n if case["gated"] else n
        s.update(x=v.hidden(b, k), w=v.normal(rows, k, std=k ** -0.5), bias=v.normal(rows, std=0.3) if case["bias"] else None,
                 residual=v.normal(b, n) if case["residual"] else None)
    elif kind == "route":
        t, e = case["tokens"], case["experts"]
        s.update(logits=v.normal(t, e, std=1.5, dtype=torch.float32),
                 bias=v.normal(e, std=0.05, dtype=torch.float32) if case["bias"] else None)
        if case["masked"]:  # experts that no token may choose
            s["logits"][:, torch.from_numpy(rng.permutation(e)[:case["masked"]].copy()).cuda()] = -math.inf
    elif kind == "experts":
        t, h, f, e = case["tokens"], case["hidden"], case["inter"], case["experts"]
        ids = _choices(case)[rng.permutation(t)]
        ids = np.where(ids >= 0, rng.permutation(e).astype(np.int32)[ids], ids)
        weights = torch.softmax(v.normal(t, case["top_k"], dtype=torch.float32), dim=1)
        s.update(x=v.hidden(t, h), ids=torch.from_numpy(np.ascontiguousarray(ids)).cuda(), weights=weights,
                 w_gate_up=v.normal(e, 2 * f, h, std=h ** -0.5), w_down=v.normal(e, h, f, std=f ** -0.5),
                 residual=v.normal(t, h) if case["residual"] else None)
    else:
        r, h = case["rows"], case["hidden"]
        weight = lambda on: v.normal(h, mean=1.0 - case["offset"], std=0.2) if on else None
        gate = {"none": None, "features": (h,), "rows": (r, h)}[case["gate"]]
        s.update(y=v.hidden(r, h), residual=v.normal(r, h, std=2.0), post=weight(case["post"]), pre=weight(case["pre"]),
                 gate=v.normal(*gate) if gate else None)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "linear":
        s["out"] = torch.empty((case["batch"], case["n"]), dtype=torch.float32 if case["f32"] else torch.bfloat16,
                               device="cuda")
    elif kind == "route":
        shape = (case["tokens"], case["top_k"])
        s["ids"] = torch.empty(shape, dtype=torch.int32, device="cuda")
        s["weights"] = torch.empty(shape, dtype=torch.float32, device="cuda")
    elif kind == "experts":
        s["out"] = torch.empty_like(s["x"])
    else:
        s["z"] = torch.empty_like(s["y"])
        s["h"] = torch.empty_like(s["y"]) if case["pre"] else None
    if own and kind in ("linear", "experts"):  # a program packs its weights once, when it loads them
        from paper_2606_07665_amd import binding as pda
        for name in ("w", "w_gate_up", "w_down"):
            if name in s:
                w = s[name]
                s[name] = pda.pack_weights(w.flatten(0, -2)).view(w.shape)
    return s


# -------------------------------------------------------------------- pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2606_07665_amd import binding as pda
    case = s["case"]
    kind = case["kind"]
    if kind == "linear":
        return pda.linear(s["x"], s["w"], s["out"], bias=s["bias"], residual=s["residual"], activation=case["act"],
                          gated=case["gated"])
    if kind == "route":
        return pda.moe_route(s["logits"], s["ids"], s["weights"], scoring=case["scoring"], renormalise=case["renormalise"],
                             select_bias=s["bias"], scale=case["scale"])
    if kind == "experts":
        return pda.moe_experts(s["x"], s["ids"], s["weights"], s["w_gate_up"], s["w_down"], s["out"],
                               residual=s["residual"], activation=case["act"])
    out = pda.block_norm(s["y"], s["residual"], s["z"], s["h"], post_w=s["post"], pre_w=s["pre"], gate=s["gate"],
                         scale=case["scale"], weight_offset=case["offset"], eps=EPS)
    return out if case["pre"] else out[0]


# The plain forms: elementary torch operations in 32 bits.
def _plain_activation(x, name):
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    return torch.clamp_min(x, 0.0) if name == "relu" else x


def _plain_linear(s):
    case = s["case"]
    y = torch.matmul(s["x"].float(), s["w"].float().t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if case["gated"]:
        y = _plain_activation(y[:, :case["n"]], case["act"]) * y[:, case["n"]:]
    else:
        y = _plain_activation(y, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["out"].dtype)


def _plain_route(s):
    """In 64 bits: scores next to each other decide which experts are chosen."""
    case = s["case"]
    x = s["logits"].double()
    if case["scoring"] == "softmax":
        p = torch.exp(x - x.amax(1, keepdim=True))
        score = p / p.sum(1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-x))
    key = x if s["bias"] is None else torch.where(torch.isinf(x), x, score + s["bias"].double())
    ids = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :case["top_k"]]
    w = torch.gather(score, 1, ids)
    if case["renormalise"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, torch.zeros_like(w))
    return ids.int(), (w * case["scale"]).float()


def _plain_experts(s):
    case = s["case"]
    f = case["inter"]
    x = s["x"].float()
    y = torch.zeros_like(x) if s["residual"] is None else s["residual"].float()
    pairs = s["ids"].flatten()
    for e in torch.unique(pairs).tolist():
        if e < 0:
            continue
        at = torch.nonzero(pairs == e)[:, 0]
        token = at // case["top_k"]
        g = torch.matmul(x[token], s["w_gate_up"][e].float().t())
        h = _plain_activation(g[:, :f], case["act"]) * g[:, f:]
        d = torch.matmul(h, s["w_down"][e].float().t()) * s["weights"].flatten()[at][:, None]
        y.index_add_(0, token, d)
    return y.to(torch.bfloat16)


def _plain_norm(s):
    case = s["case"]

    def rms(x, w):
        return x * torch.rsqrt(x.pow(2).mean(1, keepdim=True) + EPS) * (w.float() + case["offset"])

    y = s["y"].float()
    if s["post"] is not None:
        y = rms(y, s["post"])
    if s["gate"] is not None:
        y = y * s["gate"].float()
    z = s["residual"].float() + case["scale"] * y
    if s["pre"] is None:
        return z.to(torch.bfloat16)
    return z.to(torch.bfloat16), rms(z, s["pre"]).to(torch.bfloat16)


def _run_plain(s):
    return {"linear": _plain_linear, "route": _plain_route, "experts": _plain_experts, "norm": _plain_norm}[
        s["case"]["kind"]](s)


# ---------------------------------------------------------- what it cannot do without
def work(case):
    kind = case["kind"]
    if kind == "linear":
        b, k, n = case["batch"], case["k"], case["n"]
        rows = 2 * n if case["gated"] else n
        out = 4 if case["f32"] else 2
        return {"bytes": 2 * rows * k + 2 * b * k + (2 * rows if case["bias"] else 0) + b * n * (out + 2 * case["residual"]),
                "flops": 2 * b * rows * k}
    if kind == "route":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        return {"bytes": 4 * t * e + 8 * t * k + (4 * e if case["bias"] else 0), "flops": 4 * t * e}
    if kind == "experts":
        t, h, f, k = case["tokens"], case["hidden"], case["inter"], case["top_k"]
        ids = _choices(case)
        asked = len(np.unique(ids[ids >= 0]))
        pairs = int((ids >= 0).sum())
        return {"bytes": 6 * asked * h * f + 2 * t * h * (2 + case["residual"]) + 8 * t * k, "flops": 6 * pairs * h * f}
    elements = case["rows"] * case["hidden"]
    arrays = 3 + case["pre"] + (case["gate"] == "rows")
    return {"bytes": 2 * elements * arrays, "flops": 8 * elements}


# ------------------------------------------------------------------ in 64 bits
def _exact_activation(x, name):
    if name == "silu":
        return 0.5 * x * (1.0 + torch.tanh(0.5 * x))
    if name == "gelu":
        return 0.5 * x * torch.special.erfc(-x / math.sqrt(2.0))
    if name == "gelu_tanh":  # 0.5 (1 + tanh u) = 1 / (1 + exp(-2 u))
        return x * torch.sigmoid(math.sqrt(8.0 / math.pi) * x * (1.0 + 0.044715 * x ** 2))
    return torch.where(x > 0, x, torch.zeros_like(x)) if name == "relu" else x


def _exact_linear(s):
    case = s["case"]
    x, n = s["x"].double(), case["n"]
    out = torch.empty((case["batch"], n), dtype=torch.float64, device="cuda")
    for at in range(0, n, 4096):  # output features in parts
        part = slice(at, min(n, at + 4096))

        def product(first):
            rows = slice(first + part.start, first + part.stop)
            y = torch.mm(x, s["w"][rows].double().t())
            return y if s["bias"] is None else y + s["bias"][rows].double()

        y = _exact_activation(product(0), case["act"])
        out[:, part] = y * product(n) if case["gated"] else y
    return out if s["residual"] is None else out + s["residual"].double()


def _exact_route(s):
    """Token by token on the host, the best of the experts that are left each time."""
    case = s["case"]
    x = s["logits"].double().cpu().numpy()
    bias = None if s["bias"] is None else s["bias"].double().cpu().numpy()
    ids = np.empty((case["tokens"], case["top_k"]), dtype=np.int32)
    weights = np.empty(ids.shape, dtype=np.float64)
    for t in range(case["tokens"]):
        row = x[t]
        if case["scoring"] == "softmax":
            score = np.exp(row - np.logaddexp.reduce(row))
        else:
            score = np.exp(-np.logaddexp(0.0, -row))
        key = row.copy() if bias is None else np.where(np.isinf(row), row, score + bias)
        left = np.ones(len(row), dtype=bool)
        for j in range(case["top_k"]):
            best = key[left].max()
            ids[t, j] = np.flatnonzero(left & (key == best))[0]
            left[ids[t, j]] = False
        w = score[ids[t]]
        if case["renormalise"]:
            w = w / w.sum() if w.sum() > 0 else 0.0 * w
        weights[t] = case["scale"] * w
    return torch.from_numpy(ids).cuda(), torch.from_numpy(weights).cuda()


def _exact_experts(s):
    case = s["case"]
    t, f, k = case["tokens"], case["inter"], case["top_k"]
    x = s["x"].double()
    parts = torch.zeros((t, k, case["hidden"]), dtype=torch.float64, device="cuda")
    ids = s["ids"].cpu().numpy()
    for e in range(case["experts"]):
        token, j = (torch.from_numpy(a).cuda() for a in np.nonzero(ids == e))
        if not token.numel():
            continue
        w = s["w_gate_up"][e].double()
        up = torch.mm(x[token], w[f:].t())
        h = _exact_activation(torch.mm(x[token], w[:f].t()), case["act"]) * up
        parts[token, j] = torch.mm(h, s["w_down"][e].double().t()) * s["weights"][token, j].double()[:, None]
    y = parts.sum(1)
    return y if s["residual"] is None else y + s["residual"].double()


def _exact_norm(s):
    case = s["case"]

    def norm(x, w):
        length = torch.linalg.vector_norm(x, dim=1, keepdim=True)
        return x / torch.sqrt(length ** 2 / x.shape[1] + EPS) * (w.double() + case["offset"])

    y = s["y"].double()
    if s["post"] is not None:
        y = norm(y, s["post"])
    z = s["residual"].double() + case["scale"] * (y if s["gate"] is None else y * s["gate"].double())
    return z if s["pre"] is None else (z, norm(z, s["pre"]))


def exact(case, seed):
    s = _inputs(case, seed)
    return {"linear": _exact_linear, "route": _exact_route, "experts": _exact_experts, "norm": _exact_norm}[case["kind"]](s)
