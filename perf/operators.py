"""Performance cases of the operators for language models: products of ragged
token groups, the token loss with its gradient, and the AdamW step.

A case is a dict of plain values.  ``op`` is one of
  forward      Y[t]  = X[t] W_i for the rows t of group i (group_matmul)
  input_grad   dX[t] = dY[t] W_i^T (group_input_grad)
  weight_grad  G_i = sum over the rows of group i of X[t]^T dY[t] (group_weight_grad)
  loss         mean cross entropy of each worker's tokens, and its gradient (token_loss)
  adamw        one AdamW step over a list of tensors (AdamW.step)
Products: ``n`` groups of ragged sizes, ``T`` rows, ``d`` inputs, ``C``
outputs, ``shared`` whether all groups have the same W.  Loss: ``n`` workers,
``T`` tokens, ``C`` classes, gradients times ``scale``.  AdamW: ``tensors``
tensors of ``total`` values (sizes from ``layout``), states in ``bits`` bits,
gradients in ``type``, ``low`` the type of the 16-bit copy of the weights (""
for none), ``clip`` the largest gradient norm (0: no clipping).

With ``own`` false, run() computes the same in elementary torch operations.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 256                     # values of a scale of the 8-bit states
HYPER = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "grad_scale": 0.5, "seed": 12345}


def _product(name, op, n, T, d, C, type, out, shared=False):
    case = {"op": op, "n": n, "T": T, "d": d, "C": C, "type": type, "out": out, "shared": shared}
    return {"name": name, **case} if name else case


def _loss(name, n, T, C, type):
    # gradients in fp16 are scaled, as mixed-precision training does: most lie below its smallest value
    case = {"op": "loss", "n": n, "T": T, "C": C, "type": type, "scale": 65536.0 if type == "f16" else 1.0}
    return {"name": name, **case} if name else case


def _adamw(name, tensors, total, layout, bits, type, low, clip):
    case = {"op": "adamw", "tensors": tensors, "total": total, "layout": layout, "bits": bits, "type": type,
            "low": low, "clip": clip}
    return {"name": name, **case} if name else case


def listed():
    return [
        # the logits of sixteen workers' tokens at the common weights
        _product("forward head 4096x1024x32000 bf16", "forward", 16, 4096, 1024, 32000, "bf16", "bf16", shared=True),
        # one weight matrix a group (experts), ragged groups, one of them empty
        _product("forward 32 groups 8192x2048x1536 bf16", "forward", 32, 8192, 2048, 1536, "bf16", "bf16"),
        # serving: a handful of tokens, the weights have to be read once
        _product("forward 16 groups 37x2048x1408 f16", "forward", 16, 37, 2048, 1408, "f16", "f16"),
        # backward to the inputs, with an output width off every alignment
        _product("input grad 8 groups 6000x1000x2047 f16", "input_grad", 8, 6000, 1000, 2047, "f16", "f16"),
        # the worker gradients [n][d][C] in fp32, as the server's calls take them
        _product("weight grad 16 workers 8000x784x4000 bf16", "weight_grad", 16, 8000, 784, 4000, "bf16", "f32"),
        # few workers with long minibatches and a small layer
        _product("weight grad 2 workers 30000x512x512 bf16", "weight_grad", 2, 30000, 512, 512, "bf16", "f32"),
        # a small classifier: latency counts
        _loss("loss 64x1000 f32", 4, 64, 1000, "f32"),
        # a vocabulary of odd size, a training batch of sixteen workers
        _loss("loss 8192x50257 bf16", 16, 8192, 50257, "bf16"),
        # a large vocabulary
        _loss("loss 2048x128000 f16", 1, 2048, 128000, "f16"),
        # the tensors of a small network, where launches are all there is
        _adamw("adamw 4 tensors 0.4M f32", 4, 407050, 1, 32, "f32", "", 1.0),
        # a model in training: 8-bit states, bf16 gradients and bf16 copy
        _adamw("adamw 120 tensors 128M 8 bits", 120, 128_000_000, 2, 8, "bf16", "bf16", 1.0),
        # the same kind of model with 32-bit states and fp16 gradients
        _adamw("adamw 80 tensors 64M 32 bits", 80, 64_000_000, 3, 32, "f16", "f16", 0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["forward", "forward", "input_grad", "weight_grad", "weight_grad", "loss", "loss", "adamw", "adamw"])
    if op == "loss":
        C = _log(rng, 100, 128000)
        T = min(_log(rng, 1, 16384), max(1, 8192 * 50257 // C))
        return _loss(None, min(T, _log(rng, 1, 64)), T, C, rng.choice(["f32", "bf16", "f16"]))
    if op == "adamw":
        total = _log(rng, 20000, 128_000_000)
        return _adamw(None, _log(rng, 1, 200), total, rng.randint(4, 1 << 20), rng.choice([8, 32]),
                      rng.choice(["f32", "bf16", "f16"]), rng.choice(["", "bf16", "f16"]), rng.choice([0.0, 1.0]))
    d, C = _log(rng, 64, 4096), _log(rng, 64, 4096)
    if rng.random() < 0.7:       # most layers have widths of whole vectors
        d, C = (d + 7) // 8 * 8, (C + 7) // 8 * 8
    n = _log(rng, 1, 64)
    T = min(_log(rng, 1, 16384), 4096 * 1024 * 32000 // (d * C))
    type = rng.choice(["bf16", "f16"])
    out = rng.choice(["f32", type]) if op == "weight_grad" else type
    return _product(None, op, n, T, d, C, type, out, shared=op == "forward" and rng.random() < 0.3)


# -- inputs ------------------------------------------------------------------


def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _lengths(rng, n, T):
    """Ragged group sizes: within a factor of seven of each other, one group
    in eight empty."""
    part = [rng.uniform(0.25, 1.75) if n < 8 or i % 8 != 5 else 0.0 for i in range(n)]
    ends = [0]
    for p in part:
        ends.append(ends[-1] + p)
    ends = [round(T * e / ends[-1]) for e in ends]
    return [b - a for a, b in zip(ends, ends[1:])]


def _sizes(case):
    """Sizes of the case's tensors: a few large ones, many small ones, odd."""
    rng = random.Random(case["layout"])
    part = [math.exp(rng.uniform(0.0, 6.0)) for _ in range(case["tensors"])]
    left = case["total"] - case["tensors"]
    sizes = [1 + int(left * p / sum(part)) for p in part]
    sizes[0] += case["total"] - sum(sizes)
    return sizes


def _prepare_adamw(case, gen, dev):
    sizes = _sizes(case)
    blocks = [-(-s // BLOCK) for s in sizes]
    first = [0]
    for b in blocks:
        first.append(first[-1] + b)
    flat = first[-1] * BLOCK                        # every tensor starts at a block of one flat buffer
    at = torch.tensor(first, device=dev)
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device=dev), torch.tensor(blocks, device=dev))
    start = (torch.arange(first[-1], device=dev) - at[tensor]) * BLOCK     # index of a block's first value in its tensor
    inside = torch.tensor(sizes, device=dev)[tensor].view(-1, 1) > start.view(-1, 1) + torch.arange(BLOCK, device=dev)
    decay = [0.0 if s < 5000 else 0.1 for s in sizes]                      # small tensors are biases and norms
    normal = lambda scale: torch.randn(flat, generator=gen, device=dev).mul_(scale).mul_(inside.view(-1))  # noqa: E731
    s = {"case": case, "t": 100, "sizes": sizes, "first": first, "tensor": tensor, "start": start, "decay": decay,
         "decay_of_block": torch.tensor(decay, device=dev)[tensor],
         "w": normal(0.02), "g": normal(1e-3).to(TYPES[case["type"]]),
         "low": torch.zeros(flat, dtype=TYPES[case["low"]], device=dev) if case["low"] else None}
    if case["bits"] == 32:
        s |= {"m": normal(1e-4), "v": normal(5e-4).square_()}
    else:
        # codes as the step leaves them: the largest of a block between 224 and 448
        s |= {"m": normal(100.0).clamp_(-448, 448).to(torch.float8_e4m3fn),
              "v": normal(100.0).abs_().clamp_(0.01, 448).mul_(inside.view(-1)).to(torch.float8_e4m3fn),
              "m_scale": torch.randint(105, 108, (first[-1],), generator=gen, device=dev).to(torch.uint8).view(torch.float8_e8m0fnu),
              "v_scale": torch.randint(107, 110, (first[-1],), generator=gen, device=dev).to(torch.uint8).view(torch.float8_e8m0fnu)}
    if own:
        from paper_2004_14696_amd import AdamW
        views = lambda x: [x[a * BLOCK:a * BLOCK + z] for a, z in zip(first, sizes)]                       # noqa: E731
        scales = lambda x: [x[a:b] for a, b in zip(first, first[1:])]                                      # noqa: E731
        more = {} if case["bits"] == 32 else {"m_scale": scales(s["m_scale"]), "v_scale": scales(s["v_scale"])}
        s["opt"] = AdamW(views(s["w"]), views(s["g"]), views(s["m"]), views(s["v"]),
                         low=views(s["low"]) if case["low"] else None, weight_decay=decay, step=s["t"], **more)
    return s


def prepare(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(seed)
    if case["op"] == "adamw":
        return _prepare_adamw(case, gen, dev)
    n, T, C = case["n"], case["T"], case["C"]
    lengths = _lengths(random.Random(seed), n, T)
    ends = [0]
    for r in lengths:
        ends.append(ends[-1] + r)
    type = TYPES[case["type"]]
    normal = lambda shape, scale: torch.randn(shape, generator=gen, device=dev).mul_(scale).to(type)       # noqa: E731
    s = {"case": case, "ends": ends, "longest": max(lengths), "offsets": torch.tensor(ends, dtype=torch.int32, device=dev)}
    if case["op"] == "loss":
        y = torch.randint(0, C, (T,), generator=gen, device=dev, dtype=torch.int32)
        masked = torch.rand(T, generator=gen, device=dev) < 0.1          # padding and prompt tokens have no loss
        return s | {"Z": normal((T, C), 2.0), "y": torch.where(masked, torch.full_like(y, -1), y)}
    d = case["d"]
    if case["op"] != "input_grad":
        s["X"] = normal((T, d), 1.0)
    if case["op"] != "forward":
        s["dY"] = normal((T, C), 0.01)
    if case["op"] != "weight_grad":
        s["W"] = normal((d, C) if case["shared"] else (n, d, C), 1 / math.sqrt(d))
    return s


# -- plain forms ---------------------------------------------------------------


def _padded(rows, s):
    """Rows of the groups, [n][longest][...] in 32 bits, zero behind a group's
    last row; and the group of each row with its place there."""
    start, T = s["offsets"].long(), rows.shape[0]
    group = torch.searchsorted(start[1:], torch.arange(T, device=rows.device), right=True)
    place = torch.arange(T, device=rows.device) - start[group]
    padded = torch.zeros((s["case"]["n"], s["longest"]) + tuple(rows.shape[1:]), device=rows.device)
    padded[group, place] = rows.float()
    return padded, group, place


def _plain_product(s):
    case = s["case"]
    out = TYPES[case["out"]]
    if case["op"] == "weight_grad":
        X, dY = _padded(s["X"], s)[0], _padded(s["dY"], s)[0]
        return torch.bmm(X.transpose(1, 2).contiguous(), dY).to(out)
    if case["shared"]:
        return (s["X"].float() @ s["W"].float()).to(out)
    forward = case["op"] == "forward"
    rows, group, place = _padded(s["X"] if forward else s["dY"], s)
    W = s["W"].float() if forward else s["W"].float().transpose(1, 2).contiguous()
    return torch.bmm(rows, W)[group, place].to(out)


def _plain_loss(s):
    n, y = s["case"]["n"], s["y"].long()
    start = s["offsets"].long()
    Z, live = s["Z"].float(), y >= 0
    worker = torch.searchsorted(start[1:], torch.arange(len(y), device=Z.device), right=True)
    count = torch.zeros(n, device=Z.device).index_add_(0, worker, live.float())
    share = live * s["case"]["scale"] / count.clamp(min=1.0)[worker]
    Z = Z - Z.amax(1, keepdim=True)
    at = y.clamp(min=0).view(-1, 1)
    zy = Z.gather(1, at).view(-1)
    P = Z.exp()
    sums = P.sum(1, keepdim=True)
    ce = (sums.view(-1).log() - zy) * live
    loss = torch.zeros(n, dtype=torch.float64, device=Z.device).index_add_(0, worker, ce.double()) / count.clamp(min=1.0)
    P = P / sums
    P.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
    return loss.float(), (P * share.view(-1, 1)).to(s["Z"].dtype)


M32 = 0xFFFFFFFF


def _mix(x):
    x = (x ^ (x >> 16)) * 0x9E3779B1 & M32
    x = (x ^ (x >> 15)) * 0xB7E15163 & M32
    return x ^ (x >> 16)


def _round_bits(s):
    """The 32 random bits of every value: a mix of seed, step, tensor and index."""
    key = _mix(_mix(_mix(HYPER["seed"]) + s["t"] & M32) + s["tensor"] & M32).view(-1, 1)
    index = s["start"].view(-1, 1) + torch.arange(BLOCK, device=key.device)
    return _mix((index & M32) * 0x6A09E667 + (index >> 32) * 0xBB67AE85 + key & M32)


def _exponent(x):
    """floor(log2 x) of positive normal 32-bit values."""
    return (x.view(torch.int32) >> 23) - 127


def _pow(e):
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x, bits, floor):
    """e4m3 values and e8m0 scales of x [blocks][256]: the largest value of a
    block lands in (224, 448]; rounded up where the discarded part exceeds
    1 - bits / 2^16."""
    top = x.abs().amax(1, keepdim=True).clamp(min=2.0 ** -118)
    e = _exponent(top)
    e = e - 8 + (top * _pow(-e) > 1.75)                       # scale exponent
    y = x.abs() * _pow(-e)
    step = _exponent(y.clamp(min=2.0 ** -6)) - 3
    q = torch.floor(y * _pow(-step) + bits.float() / 65536.0)
    if floor:
        q = torch.where((x > 0) & (q == 0), torch.ones_like(q), q)
    codes = torch.copysign(q * _pow(step), x).to(torch.float8_e4m3fn)
    return codes.view(-1), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu).view(-1)


def _plain_adamw(s):
    case, h = s["case"], HYPER
    s["t"] += 1
    norm, f = None, h["grad_scale"]
    if case["clip"]:
        norm = s["g"].double().square().sum().sqrt() * f
        f = (f * torch.clamp(case["clip"] / norm, max=1.0)).float()
    g = s["g"].view(-1, BLOCK).float() * f
    w = s["w"].view(-1, BLOCK)
    if case["bits"] == 32:
        m, v = s["m"].view(-1, BLOCK), s["v"].view(-1, BLOCK)
    else:
        m = s["m"].float().view(-1, BLOCK) * s["m_scale"].float().view(-1, 1)
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"].float().view(-1, 1)).square()
    m = m * h["beta1"] + g * (1 - h["beta1"])
    v = v * h["beta2"] + g * g * (1 - h["beta2"])
    r = v.sqrt()
    rate = h["lr"] / (1 - h["beta1"] ** s["t"])
    new = w * (1 - h["lr"] * s["decay_of_block"].double()).float().view(-1, 1) \
        - m / (r / math.sqrt(1 - h["beta2"] ** s["t"]) + h["eps"]) * rate
    w.copy_(new)
    if case["low"]:
        s["low"].view(-1, BLOCK).copy_(new)
    if case["bits"] == 32:
        s["m"].view(-1, BLOCK).copy_(m)
        s["v"].view(-1, BLOCK).copy_(v)
    else:
        bits = _round_bits(s)
        s["m"], s["m_scale"] = _quantise(m, bits & 0xFFFF, False)
        s["v"], s["v_scale"] = _quantise(r, bits >> 16, True)
    return _adamw_outputs(s, norm.float() if norm is not None else None)


def _adamw_outputs(s, norm):
    return {k: s[k] for k in ("w", "m", "v", "m_scale", "v_scale", "low") if s.get(k) is not None} | {"norm": norm}


# -- the framework's calls -------------------------------------------------------


def _own(s):
    import paper_2004_14696_amd as dbw
    case = s["case"]
    if case["op"] == "loss":
        return dbw.token_loss(s["Z"], s["y"], s["offsets"], scale=case["scale"])
    if case["op"] == "adamw":
        return _adamw_outputs(s, s["opt"].step(max_norm=case["clip"], **HYPER))
    out = TYPES[case["out"]]
    if case["op"] == "forward":
        return dbw.group_matmul(s["X"], s["W"], s["offsets"], out_dtype=out)
    if case["op"] == "input_grad":
        return dbw.group_input_grad(s["dY"], s["W"], s["offsets"], out_dtype=out)
    return dbw.group_weight_grad(s["X"], s["dY"], s["offsets"], out_dtype=out)


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_loss(state) if op == "loss" else _plain_adamw(state) if op == "adamw" else _plain_product(state)


# -- floors ----------------------------------------------------------------------


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2, "": 0}
    b = size[case["type"]]
    if case["op"] == "loss":
        return {"bytes": 2 * b * case["T"] * case["C"] + 4 * case["T"], "flops": 5 * case["T"] * case["C"]}
    if case["op"] == "adamw":
        state = 16 if case["bits"] == 32 else 4 + 4 / BLOCK
        return {"bytes": case["total"] * (b + 8 + state + size[case["low"]]), "flops": 20 * case["total"]}
    n, T, d, C = (case[k] for k in ("n", "T", "d", "C"))
    groups = 1 if case["shared"] else min(n, T)
    sides = {"forward": (T * d, T * C), "input_grad": (T * C, T * d), "weight_grad": (T * d + T * C, n * d * C)}
    read, written = sides[case["op"]]
    if case["op"] != "weight_grad":
        read += groups * d * C
    return {"bytes": b * read + size[case["out"]] * written, "flops": 2 * T * d * C}


# -- the definitions in 64 bits ------------------------------------------------------


def _exact_adamw(s):
    """Tensor by tensor, in 64 bits; stored states rounded by the same rule."""
    case, h, t = s["case"], HYPER, s["t"] + 1
    f, norm = h["grad_scale"], None
    if case["clip"]:
        norm = float(torch.sqrt(sum((s["g"][a * BLOCK:b * BLOCK].double() ** 2).sum() for a, b in zip(s["first"], s["first"][1:])))) * f
        f *= min(1.0, case["clip"] / norm) if norm else 1.0
    keep = {k: [] for k in ("w", "m", "v", "m_scale", "v_scale", "low")}

    def mix(x):
        for shift, factor in ((16, 0x9E3779B1), (15, 0xB7E15163)):
            x = torch.bitwise_xor(x, x >> shift)
            x = torch.remainder(x * factor, 1 << 32)
        return torch.bitwise_xor(x, x >> 16)

    def store(name, x, u, least):
        largest = x.abs().max(dim=1, keepdim=True).values.clamp(min=2.0 ** -118)
        e = torch.ceil(torch.log2(largest / 448.0))
        scaled = x.abs() / torch.exp2(e)
        step = torch.exp2(torch.floor(torch.log2(scaled.clamp(min=2.0 ** -6))) - 3)
        low = torch.floor(scaled / step)
        up = scaled / step - low >= 1.0 - u / 65536.0
        q = low + up
        if least:
            q = torch.where((q == 0) & (x > 0), 1.0, q)
        keep[name].append((q * step * torch.sign(x)).view(-1))
        keep[name + "_scale"].append(torch.exp2(e).view(-1))

    dev = s["w"].device
    for i, (a, b) in enumerate(zip(s["first"], s["first"][1:])):
        part = slice(a * BLOCK, b * BLOCK)
        w, g = s["w"][part].double(), s["g"][part].double() * f
        m, v = s["m"][part].double(), s["v"][part].double()
        if case["bits"] == 8:
            m = (m.view(-1, BLOCK) * s["m_scale"][a:b].double().view(-1, 1)).view(-1)
            v = ((v.view(-1, BLOCK) * s["v_scale"][a:b].double().view(-1, 1)) ** 2).view(-1)
        m = h["beta1"] * m + (1 - h["beta1"]) * g
        v = h["beta2"] * v + (1 - h["beta2"]) * g ** 2
        mean, spread = m / (1 - h["beta1"] ** t), torch.sqrt(v / (1 - h["beta2"] ** t))
        w = w - h["lr"] * s["decay"][i] * w - h["lr"] * mean / (spread + h["eps"])
        keep["w"].append(w)
        if case["low"]:
            keep["low"].append(w)
        if case["bits"] == 32:
            keep["m"].append(m)
            keep["v"].append(v)
            continue
        one = lambda x: torch.tensor(x, dtype=torch.int64, device=dev)                                    # noqa: E731
        key = mix((mix((mix(one(h["seed"])) + t) % (1 << 32)) + i) % (1 << 32))
        index = torch.arange((b - a) * BLOCK, device=dev)
        u = mix(((index % (1 << 32)) * 0x6A09E667 + (index // (1 << 32)) * 0xBB67AE85 + key) % (1 << 32))
        store("m", m.view(-1, BLOCK), (u % 65536).view(-1, BLOCK).double(), False)
        store("v", torch.sqrt(v).view(-1, BLOCK), (u // 65536).view(-1, BLOCK).double(), True)
    return {k: torch.cat(x) for k, x in keep.items() if x} | {"norm": norm}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s)
    ends = list(zip(s["ends"], s["ends"][1:]))
    if case["op"] == "loss":
        losses, grads = [], []
        for a, b in ends:
            z, y = s["Z"][a:b].double(), s["y"][a:b].long()
            rows = torch.nonzero(y >= 0).view(-1)
            logp = z - torch.logsumexp(z, 1, keepdim=True)
            losses.append(-logp[rows, y[rows]].mean() if len(rows) else torch.zeros((), dtype=torch.float64, device=z.device))
            grad = torch.exp(logp)
            grad[rows, y[rows]] -= 1.0
            grads.append(grad * (y >= 0).double().view(-1, 1) * case["scale"] / max(1, len(rows)))
        return torch.stack(losses), torch.cat(grads)
    if case["op"] == "weight_grad":
        return torch.stack([s["X"][a:b].double().t().contiguous() @ s["dY"][a:b].double() for a, b in ends])
    W = s["W"].double()
    if case["shared"]:
        return s["X"].double() @ W
    if case["op"] == "forward":
        return torch.cat([s["X"][a:b].double() @ W[i] for i, (a, b) in enumerate(ends)])
    return torch.cat([s["dY"][a:b].double() @ W[i].t().contiguous() for i, (a, b) in enumerate(ends)])
