"""Performance cases of the operators of a transformer block in training: causal
attention over packed sequences, layer norm, products with bias, activation
and residual, and dropout.

A case is a dict of plain values.  ``op`` is one of
  attention    O[t] = sum over the tokens s <= t of t's sequence of P[t][s] V[s],
               P = softmax(Q K^T / sqrt(D)); with ``grad`` the gradients too
               (attention, attention_grad)
  norm         Y[t] = (X[t] - mean) / sqrt(var + eps) gamma + beta (layer_norm)
  norm_grad    its gradients: dX, and dgamma and dbeta of each worker
               (layer_norm_grad)
  linear       Y[t] = act(X[t] W_i + b_i) + R[t], and act's argument where
               ``pre`` (group_linear)
  linear_grad  dZ = dY act'(Z), and the bias gradient of each worker
               (group_linear_grad)
  dropout      Y = R + X kept / (1 - p) (dropout)
``T`` rows in ``n`` ragged groups (sequences, workers or experts).  Attention:
``heads`` heads of queries and ``kv`` of keys and values, ``D`` values each.
Products: ``d`` inputs, ``C`` outputs, ``shared`` whether all groups have the
same W and b, ``act`` the activation, ``residual`` whether there is an R.

With ``own`` false, run() computes the same in elementary torch operations.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def _named(name, case):
    return {"name": name, **case} if name else case


def _attention(name, n, T, heads, kv, D, type, grad):
    return _named(name, {"op": "attention", "n": n, "T": T, "heads": heads, "kv": kv, "D": D, "type": type, "grad": grad})


def _norm(name, op, n, T, d, type):
    return _named(name, {"op": op, "n": n, "T": T, "d": d, "type": type})


def _linear(name, n, T, d, C, type, act, residual=False, pre=False, shared=False):
    return _named(name, {"op": "linear", "n": n, "T": T, "d": d, "C": C, "type": type, "act": act, "residual": residual,
                         "pre": pre, "shared": shared})


def _linear_grad(name, n, T, C, type, act):
    return _named(name, {"op": "linear_grad", "n": n, "T": T, "C": C, "type": type, "act": act})


def _dropout(name, T, d, type, p, residual):
    return _named(name, {"op": "dropout", "T": T, "d": d, "type": type, "p": p, "residual": residual})


def listed():
    return [
        # a few short sequences of a small model: latency counts
        _attention("attention 3 seqs 200 tokens 4x64 bf16", 3, 200, 4, 4, 64, "bf16", False),
        # one long document, read through once (evaluation)
        _attention("attention 1 seq 16384 tokens 8/2x128 bf16", 1, 16384, 8, 2, 128, "bf16", False),
        # a training batch of packed sequences, grouped heads
        _attention("attention train 8 seqs 8192 tokens 16/4x128 bf16", 8, 8192, 16, 4, 128, "bf16", True),
        # many short sequences, heads of a width between the tiles
        _attention("attention train 50 seqs 5000 tokens 12x80 f16", 50, 5000, 12, 12, 80, "f16", True),
        # the norm of a large batch
        _norm("norm 16384x4096 bf16", "norm", 16, 16384, 4096, "bf16"),
        # its gradients, the weights' of each of sixteen workers
        _norm("norm grad 16 workers 8192x4096 bf16", "norm_grad", 16, 8192, 4096, "bf16"),
        # many workers with small ragged minibatches, rows at odd addresses
        _norm("norm grad 64 workers 3001x1003 f32", "norm_grad", 64, 3001, 1003, "f32"),
        # the first layer of a block, its activation's argument kept for the gradient
        _linear("linear gelu 8192x1024x4096 bf16", 16, 8192, 1024, 4096, "bf16", "gelu", pre=True, shared=True),
        # experts with few rows each, added to the residual stream
        _linear("linear silu 8 groups 300x2048x1408 f16", 8, 300, 2048, 1408, "f16", "silu", residual=True),
        # the way back through that activation
        _linear_grad("linear grad gelu 16 workers 8192x4096 bf16", 16, 8192, 4096, "bf16", "gelu"),
        # on the way into the residual stream of a large batch
        _dropout("dropout 16384x4096 bf16 with residual", 16384, 4096, "bf16", 0.1, True),
        # a small layer: latency counts
        _dropout("dropout 37x1000 f32", 37, 1000, "f32", 0.5, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "norm", "norm_grad", "norm_grad", "linear", "linear",
                     "linear_grad", "dropout"])
    if op == "attention":
        kv, share = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 1, 2, 4])
        D = rng.choice([64, 128, 64, 128, 32, 80, 96, 40])
        n = _log(rng, 1, 64)
        grad = rng.random() < 0.6
        # at most the work of the longest listed sequence; a longest sequence has at most a few times the average
        longest = math.sqrt((3e8 if grad else 2e9) / (kv * share) * 64 / max(D, 64))
        T = min(_log(rng, n, 16384), max(n, int(longest * (math.sqrt(n) if n > 1 else 1.0))))
        return _attention(None, n, T, kv * share, kv, D, rng.choice(["bf16", "f16"]), grad)
    T, n = _log(rng, 1, 16384), _log(rng, 1, 64)
    d = _log(rng, 16, 16384)
    if rng.random() < 0.7:           # most layers have widths of whole vectors
        d = (d + 7) // 8 * 8
    if op in ("norm", "norm_grad"):
        T = min(T, 16384 * 4096 // d)
        return _norm(None, op, n, T, d, rng.choice(["bf16", "f16", "f32"]))
    if op == "dropout":
        T = min(T, 16384 * 4096 // d)
        return _dropout(None, T, d, rng.choice(["bf16", "f16", "f32"]), rng.choice([0.1, 0.25, 0.5]), rng.random() < 0.5)
    act = rng.choice(["none", "relu", "gelu", "silu"])
    if op == "linear_grad":
        T = min(T, 8192 * 4096 // d)
        return _linear_grad(None, n, T, d, rng.choice(["bf16", "f16"]), act)
    d, C = min(d, 4096), _log(rng, 16, 4096)
    if d % 8 == 0:
        C = (C + 7) // 8 * 8
    T = min(T, 8192 * 1024 * 4096 // (d * C))
    return _linear(None, n, T, d, C, rng.choice(["bf16", "f16"]), act, residual=rng.random() < 0.4,
                   pre=act != "none" and rng.random() < 0.6, shared=rng.random() < 0.5)


# -- inputs ------------------------------------------------------------------


def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _lengths(rng, n, T):
    """Ragged group sizes: within a factor of seven of each other."""
    part = [rng.uniform(0.25, 1.75) for _ in range(n)]
    ends = [0]
    for p in part:
        ends.append(ends[-1] + p)
    ends = [round(T * e / ends[-1]) for e in ends]
    return [b - a for a, b in zip(ends, ends[1:])]


def prepare(case, seed):
    dev, op, T = _device(), case["op"], case["T"]
    gen = torch.Generator(device=dev).manual_seed(seed)
    rng = random.Random(seed)
    type = TYPES[case["type"]]
    normal = lambda shape, scale, dtype=type: torch.randn(shape, generator=gen, device=dev).mul_(scale).to(dtype)   # noqa: E731
    lengths = _lengths(rng, case.get("n", 1), T)
    ends = [0]
    for r in lengths:
        ends.append(ends[-1] + r)
    s = {"case": case, "ends": ends, "longest": max(lengths), "offsets": torch.tensor(ends, dtype=torch.int32, device=dev)}
    if op == "attention":
        # one array of queries, keys and values, as the product before writes it
        heads, kv, D = case["heads"], case["kv"], case["D"]
        s["qkv"] = normal((T, heads + 2 * kv, D), 1.0)
        if case["grad"]:
            s["dO"] = normal((T, heads, D), 0.02)
        return s
    if op in ("norm", "norm_grad"):
        d = case["d"]
        # the residual stream: a few columns are far larger than the others
        X = torch.randn((T, d), generator=gen, device=dev).add_(0.1)
        s["X"] = X.mul_(torch.exp(torch.randn(d, generator=gen, device=dev))).to(type)
        s["gamma"] = 1.0 + normal((d,), 0.1, torch.float32)
        s["beta"] = normal((d,), 0.1, torch.float32)
        if op == "norm_grad":
            s["dY"] = normal((T, d), 0.02)
        return s
    if op == "dropout":
        s["X"] = normal((T, case["d"]), 1.0)
        s["R"] = normal((T, case["d"]), 1.0) if case["residual"] else None
        s["seed"] = rng.getrandbits(62)
        s["step"] = torch.tensor([rng.randrange(1000)], dtype=torch.int64, device=dev)
        return s
    n, C = case["n"], case["C"]
    if op == "linear_grad":
        return s | {"dY": normal((T, C), 0.02), "Z": normal((T, C), 1.0)}
    d = case["d"]
    s["X"] = normal((T, d), 1.0)
    s["W"] = normal((d, C) if case["shared"] else (n, d, C), 1 / math.sqrt(d))
    s["b"] = normal((C,) if case["shared"] else (n, C), 0.1, torch.float32)
    s["R"] = normal((T, C), 1.0) if case["residual"] else None
    return s


# -- plain forms ---------------------------------------------------------------


def _places(s, T):
    """The group of each row, and its place there."""
    start = s["offsets"].long()
    group = torch.searchsorted(start[1:], torch.arange(T, device=start.device), right=True)
    return group, torch.arange(T, device=start.device) - start[group]


def _plain_attention(s):
    """Sequences padded to the longest, heads that share keys side by side."""
    case, qkv = s["case"], s["qkv"]
    T, n, L, kv, D = case["T"], case["n"], s["longest"], case["kv"], case["D"]
    share = case["heads"] // kv
    group, place = _places(s, T)

    def padded(rows, per):
        # [n * kv][per * L][D], zero behind a sequence's last token
        x = torch.zeros((n, L, kv, per, D), device=rows.device)
        x[group, place] = rows.float().view(T, kv, per, D)
        return x.permute(0, 2, 3, 1, 4).reshape(n * kv, per * L, D)

    def rows(x, per):
        x = x.view(n, kv, per, L, D).permute(0, 3, 1, 2, 4)
        return x[group, place].reshape(T, kv * per, D)
    heads = case["heads"]
    Q, K, V = padded(qkv[:, :heads], share), padded(qkv[:, heads:heads + kv], 1), padded(qkv[:, heads + kv:], 1)
    scale = 1 / math.sqrt(D)
    later = torch.ones((L, L), dtype=torch.bool, device=Q.device).triu(1)
    S = torch.bmm(Q, K.transpose(1, 2).contiguous()).mul_(scale).view(n * kv, share, L, L)
    S.masked_fill_(later, -math.inf)
    top = S.amax(3, keepdim=True)
    P = S.sub_(top).exp_()
    total = P.sum(3, keepdim=True)
    P = P.div_(total).view(n * kv, share * L, L)
    O = torch.bmm(P, V)                                                                                   # noqa: E741
    out = rows(O, share).to(qkv.dtype)
    if not case["grad"]:
        return out
    lse = (top + total.log()).view(n, kv * share, L).transpose(1, 2)[group, place].t().contiguous()
    dO = padded(s["dO"], share)
    dV = torch.bmm(P.transpose(1, 2).contiguous(), dO)
    dS = torch.bmm(dO, V.transpose(1, 2).contiguous()).sub_((dO * O).sum(2, keepdim=True)).mul_(P).mul_(scale)
    dQ, dK = torch.bmm(dS, K), torch.bmm(dS.transpose(1, 2).contiguous(), Q)
    return out, lse, torch.cat([rows(dQ, share), rows(dK, 1), rows(dV, 1)], 1).to(qkv.dtype)


def _of_groups(x, s):
    """Sums of the rows of each group."""
    return torch.zeros((s["case"]["n"], x.shape[1]), device=x.device).index_add_(0, _places(s, len(x))[0], x)


def _plain_norm(s):
    X = s["X"].float()
    X = X - X.mean(1, keepdim=True)
    r = (X.square().mean(1, keepdim=True) + EPS).rsqrt()
    if s["case"]["op"] == "norm":
        return (X * r * s["gamma"] + s["beta"]).to(s["X"].dtype)
    H, dY = X * r, s["dY"].float()
    dH = dY * s["gamma"]
    dX = r * (dH - dH.mean(1, keepdim=True) - H * (dH * H).mean(1, keepdim=True))
    return dX.to(s["X"].dtype), _of_groups(dY * H, s), _of_groups(dY, s)


A, B = math.sqrt(2 / math.pi), 0.044715 * math.sqrt(2 / math.pi)


def _plain_act(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return 0.5 * z * (1 + torch.tanh(A * z + B * z * z * z)) if act == "gelu" else z


def _plain_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if act == "gelu":
        t = torch.tanh(A * z + B * z * z * z)
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * (A + 3 * B * z * z)
    return torch.ones_like(z)


def _plain_linear(s):
    case, T = s["case"], s["case"]["T"]
    type, b = s["X"].dtype, s["b"]
    if case["shared"]:
        Z = s["X"].float() @ s["W"].float() + b
    else:
        group, place = _places(s, T)
        X = torch.zeros((case["n"], s["longest"], case["d"]), device=b.device)
        X[group, place] = s["X"].float()
        Z = torch.bmm(X, s["W"].float())[group, place] + b[group]
    Y = _plain_act(Z, case["act"])
    if s["R"] is not None:
        Y = Y + s["R"].float()
    return (Y.to(type), Z.to(type)) if case["pre"] else Y.to(type)


def _plain_linear_grad(s):
    dZ = s["dY"].float() * _plain_slope(s["Z"].float(), s["case"]["act"])
    return dZ.to(s["dY"].dtype), _of_groups(dZ, s)


M32 = 0xFFFFFFFF


def _philox(c, key):
    """Philox4x32-10 (Salmon et al. 2011) of counters c, four int64 arrays."""
    k0, k1 = key & M32, key >> 32
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57            # the low 64 bits are right, whatever the sign
        c = (q >> 32 & M32 ^ c[1] ^ k0, q & M32, p >> 32 & M32 ^ c[3] ^ k1, p & M32)
        k0, k1 = k0 + 0x9E3779B9 & M32, k1 + 0xBB67AE85 & M32
    return c


def _plain_dropout(s):
    case = s["case"]
    T, d, X = case["T"], case["d"], s["X"]
    cut = round(case["p"] * 65536)
    row = torch.arange(T, device=X.device).view(-1, 1)
    block = torch.arange((d + 7) // 8, device=X.device).view(1, -1)
    c = torch.broadcast_tensors(block, row, s["step"] & M32, s["step"] >> 32)
    bits = torch.stack(_philox(c, s["seed"]), 2)
    bits = torch.stack([bits & 0xFFFF, bits >> 16], 3).view(T, -1)[:, :d]
    Y = torch.where(bits >= cut, X.float() * (65536 / (65536 - cut)), 0.0)
    if s["R"] is not None:
        Y = Y + s["R"].float()
    return Y.to(X.dtype)


# -- the framework's calls -------------------------------------------------------


def _own(s):
    import paper_2004_14696_amd as dbw
    case = s["case"]
    op, at = case["op"], s["offsets"]
    if op == "attention":
        q, k = case["heads"], case["heads"] + case["kv"]
        Q, K, V = s["qkv"][:, :q], s["qkv"][:, q:k], s["qkv"][:, k:]
        O, lse = dbw.attention(Q, K, V, at, lse=case["grad"])                                            # noqa: E741
        if not case["grad"]:
            return O
        d = torch.empty_like(s["qkv"])
        dbw.attention_grad(s["dO"], Q, K, V, O, lse, at, dQ=d[:, :q], dK=d[:, q:k], dV=d[:, k:])
        return O, lse, d
    if op == "norm":
        return dbw.layer_norm(s["X"], s["gamma"], s["beta"], at, eps=EPS)
    if op == "norm_grad":
        return dbw.layer_norm_grad(s["dY"], s["X"], s["gamma"], at, eps=EPS)
    if op == "linear":
        Y, Z = dbw.group_linear(s["X"], s["W"], at, bias=s["b"], activation=case["act"], residual=s["R"], pre=case["pre"])
        return (Y, Z) if case["pre"] else Y
    if op == "linear_grad":
        return dbw.group_linear_grad(s["dY"], at, pre=s["Z"], activation=case["act"])
    return dbw.dropout(s["X"], case["p"], s["seed"], at, residual=s["R"], step=s["step"])


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return (_plain_attention if op == "attention" else _plain_linear if op == "linear" else
            _plain_linear_grad if op == "linear_grad" else _plain_dropout if op == "dropout" else _plain_norm)(state)


# -- floors ----------------------------------------------------------------------


def work(case):
    b, T, op = {"f32": 4, "bf16": 2, "f16": 2}[case["type"]], case["T"], case["op"]
    if op == "attention":
        heads, kv, D = case["heads"], case["kv"], case["D"]
        # pairs of a token and one at or before it; squares of the lengths on average (within a factor of seven)
        pairs = 0.5 * T * (T / case["n"] * (1.1875 if case["n"] > 1 else 1.0) + 1)
        rows = b * T * D
        read, written = rows * (heads + 2 * kv), rows * heads
        if case["grad"]:
            # the way back reads Q, K, V, O and dO, writes three gradients, and has five products where the way there has two
            return {"bytes": read + written + rows * (3 * heads + 2 * kv) + rows * (heads + 2 * kv) + 12 * T * heads,
                    "flops": 14 * pairs * heads * D}
        return {"bytes": read + written, "flops": 4 * pairs * heads * D}
    if op in ("norm", "norm_grad"):
        d, grad = case["d"], op == "norm_grad"
        return {"bytes": (3 if grad else 2) * b * T * d + (4 * d + 8 * case["n"] * d if grad else 8 * d),
                "flops": (16 if grad else 8) * T * d}
    if op == "dropout":
        return {"bytes": (3 if case["residual"] else 2) * b * T * case["d"], "flops": 12 * T * case["d"]}
    n, C = case["n"], case["C"]
    if op == "linear_grad":
        return {"bytes": (2 if case["act"] == "none" else 3) * b * T * C + 4 * n * C, "flops": 16 * T * C}
    groups = 1 if case["shared"] else min(n, T)
    outs = 1 + case["pre"] + case["residual"]
    return {"bytes": b * (T * case["d"] + groups * case["d"] * C + outs * T * C) + 4 * groups * C,
            "flops": 2 * T * case["d"] * C}


# -- the definitions in 64 bits ------------------------------------------------------


def _exact_attention(s):
    case = s["case"]
    heads, kv, D = case["heads"], case["kv"], case["D"]
    x = s["qkv"].double()
    O = torch.zeros((case["T"], heads, D), dtype=torch.float64, device=x.device)                          # noqa: E741
    lse, d = torch.zeros(heads, case["T"], dtype=torch.float64, device=x.device), torch.zeros_like(x)
    for a, e in zip(s["ends"], s["ends"][1:]):
        keep = torch.tril(torch.ones((e - a, e - a), dtype=torch.bool, device=x.device))
        for h in range(heads if e > a else 0):
            k, v = heads + h * kv // heads, heads + kv + h * kv // heads
            q, key, val = (x[a:e, i].contiguous() for i in (h, k, v))
            score = torch.where(keep, q @ key.t().contiguous() / math.sqrt(D), -math.inf)
            lse[h, a:e] = torch.logsumexp(score, 1)
            p = torch.exp(score - lse[h, a:e].view(-1, 1))
            O[a:e, h] = p @ val
            if case["grad"]:
                g = s["dO"][a:e, h].double()
                dp = g @ val.t().contiguous()
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(D)
                d[a:e, h] = ds @ key
                d[a:e, k] += ds.t().contiguous() @ q
                d[a:e, v] += p.t().contiguous() @ g
    return (O, lse, d) if case["grad"] else O


def _exact_norm(s):
    X = s["X"].double()
    var, mean = torch.var_mean(X, dim=1, correction=0, keepdim=True)
    H, r = (X - mean) / torch.sqrt(var + EPS), 1 / torch.sqrt(var + EPS)
    if s["case"]["op"] == "norm":
        return H * s["gamma"].double() + s["beta"].double()
    dY = s["dY"].double()
    dH, d = dY * s["gamma"].double(), X.shape[1]
    dX = (dH * d - dH.sum(1, keepdim=True) - H * (dH * H).sum(1, keepdim=True)) * r / d
    parts = list(zip(s["ends"], s["ends"][1:]))
    return (dX, torch.stack([(dY[a:e] * H[a:e]).sum(0) for a, e in parts]), torch.stack([dY[a:e].sum(0) for a, e in parts]))


def _exact_act(z, act):
    """Value and slope."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0).to(z.dtype)
    u, du = (z, 1.0) if act == "silu" else (2 * (A * z + B * z ** 3), 2 * (A + 3 * B * z ** 2))
    p = torch.sigmoid(u)
    return z * p, p + z * p * torch.sigmoid(-u) * du


def _exact_linear(s):
    case, out, pre = s["case"], [], []
    for i, (a, e) in enumerate(zip(s["ends"], s["ends"][1:])):
        W, b = (s["W"], s["b"]) if case["shared"] else (s["W"][i], s["b"][i])
        z = s["X"][a:e].double() @ W.double() + b.double()
        y = _exact_act(z, case["act"])[0]
        out.append(y if s["R"] is None else y + s["R"][a:e].double())
        pre.append(z)
    return (torch.cat(out), torch.cat(pre)) if case["pre"] else torch.cat(out)


def _exact_dropout(s):
    case, dev = s["case"], s["X"].device
    T, d = case["T"], case["d"]

    def product(m, x):          # high and low half of m x, by halves of 16 bits
        lo, hi = m % 65536, m // 65536
        middle = lo * (x // 65536) + (lo * (x % 65536)) // 65536
        cross = middle % 65536 + hi * (x % 65536)
        return middle // 65536 + hi * (x // 65536) + cross // 65536, (cross % 65536) * 65536 + (lo * (x % 65536)) % 65536
    index = torch.arange(T * ((d + 7) // 8), device=dev)
    step = int(s["step"])
    block, row = index % ((d + 7) // 8), index // ((d + 7) // 8)
    x = [block, row, torch.full_like(index, step % (1 << 32)), torch.full_like(index, step // (1 << 32))]
    for r in range(10):
        ka, kb = (s["seed"] + r * 0x9E3779B9) % (1 << 32), ((s["seed"] >> 32) + r * 0xBB67AE85) % (1 << 32)
        (h0, l0), (h1, l1) = product(0xD2511F53, x[0]), product(0xCD9E8D57, x[2])
        x = [torch.bitwise_xor(torch.bitwise_xor(h1, x[1]), torch.full_like(h1, ka)), l1,
             torch.bitwise_xor(torch.bitwise_xor(h0, x[3]), torch.full_like(h0, kb)), l0]
    draws = torch.stack([f(v) for v in x for f in (lambda v: v % 65536, lambda v: v // 65536)], 1).view(T, -1)[:, :d]
    share = 1 - round(case["p"] * 65536) / 65536
    y = s["X"].double() / share * (draws >= 65536 * (1 - share)).double()
    return y if s["R"] is None else y + s["R"].double()


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "attention":
        return _exact_attention(s)
    if op in ("norm", "norm_grad"):
        return _exact_norm(s)
    if op == "linear":
        return _exact_linear(s)
    if op == "dropout":
        return _exact_dropout(s)
    dZ = s["dY"].double() * _exact_act(s["Z"].double(), case["act"])[1]
    return dZ, torch.stack([dZ[a:e].sum(0) for a, e in zip(s["ends"], s["ends"][1:])])
