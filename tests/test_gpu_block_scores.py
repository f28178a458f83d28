"""Attention whose scores are large, or far from zero, against plain 64-bit forms.

Queries and keys hold whole multiples of a power of two, fewer than 2^24 of them
in every sum, so that every score is exact in fp32 whatever the order of its
sum: what is left are the errors of the exponentials, and those may not grow
with the scores.  In natural units, with u = 2^-24 and a maximum that is at most
8 powers of two (below 6) from the row's, the exponent of a term with S - top
is off by 4 u (|S - top| + 6) for the factor scale log2(e), the difference and
their product, and its exponential by 4 u.  Rows whose scores (for gradients,
whose lse) lie below 2^10 powers of two, 710 in natural units, may form their
exponents from products instead of differences: a few u of 720 more.
"""
import math

import pytest

pb = pytest.importorskip("paper_2004_14696_amd.binding")
torch = pytest.importorskip("torch")

from test_gpu_block import BF16, F16, F32, TINY, close, gen, half_step, normal, offsets_of, parts_of, rounded, u  # noqa: E402

pytestmark = pytest.mark.gpu


def reference(Q, K, V, lengths, scale, out=None, dO=None):
    """64-bit results and bounds on the errors.  With dO: the gradients', from the
    O that the forward pass has left in `out`."""
    dtype, dev = Q.dtype, Q.device
    T, heads, D = Q.shape
    share, hs, tiny = heads // K.shape[1], half_step(dtype), TINY[dtype] / 2
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device=dev)                                        # noqa: E731
    ref = {"O": z(T, heads, D), "lse": z(heads, T), "dQ": z(*Q.shape), "dK": z(*K.shape), "dV": z(*V.shape)}
    tol = {k: torch.zeros_like(v) for k, v in ref.items()}
    for a, b in parts_of(lengths):
        N = b - a
        if N == 0:
            continue
        keep = torch.tril(torch.ones((N, N), dtype=torch.bool, device=dev))
        for h in range(heads):
            j = h // share
            q, k, v = Q[a:b, h].double().contiguous(), K[a:b, j].double().contiguous(), V[a:b, j].double().contiguous()
            S = torch.where(keep, scale * (q @ k.t().contiguous()), -math.inf)
            top = S.amax(1, keepdim=True)
            P = torch.exp(S - top)
            total = P.sum(1, keepdim=True)
            P, lsum = P / total, total.log()
            lse = top + lsum
            size = torch.where(keep, (S - top).abs() + 6, 0.0)
            near = torch.where(keep, S.abs(), 0.0).amax(1, keepdim=True).clamp(max=720)
            e_P = torch.where(keep, 4 * u * size + 4 * u + 2 * u * near, 0.0)
            e_row = (P * e_P).sum(1, keepdim=True)
            O = P @ v                                                                                      # noqa: E741
            t = 1.02 * ((P * (e_P + e_row + hs + (2 * N + 8) * u)) @ v.abs() + tiny * (keep.double() @ v.abs()))
            ref["O"][a:b, h], tol["O"][a:b, h] = O, t + rounded(O.abs() + t, dtype)
            e_sum = e_row + (N + 8) * u
            ref["lse"][h, a:b] = lse.view(-1)
            tol["lse"][h, a:b] = (1.02 * e_sum + 4 * u * (lse.abs() + top.abs())).view(-1)
            if dO is None:
                continue
            g = dO[a:b, h].double().contiguous()
            vt = v.t().contiguous()
            dP, delta = g @ vt, (g * O).sum(1, keepdim=True)
            e_G = torch.where(keep, 4 * u * size + e_sum + 8 * u + 12 * u * near, 0.0)
            e_dP = 2 * D * u * (g.abs() @ vt.abs())
            # delta is dO . O of the O that is there, or sum P dO . V
            e_delta = ((g * (out[a:b, h].double() - O)).sum(1, keepdim=True).abs() + D * u * (g * O).abs().sum(1, keepdim=True)
                       + (P * (e_dP + (e_G + N * u) * dP.abs())).sum(1, keepdim=True))
            dS = P * (dP - delta)
            e_dS = P * (e_dP + e_delta) * (1 + e_G) + dS.abs() * (e_G + 4 * u)
            e_dS = 1.02 * (e_dS + hs * (dS.abs() + e_dS) + tiny * keep.double())
            ref["dQ"][a:b, h] = scale * (dS @ k)
            tol["dQ"][a:b, h] = scale * (e_dS @ k.abs() + (2 * N + 4) * u * (dS.abs() @ k.abs()))
            back = lambda x, y: x.t().contiguous() @ y                                                     # noqa: E731
            ref["dK"][a:b, j] += scale * back(dS, q)
            tol["dK"][a:b, j] += scale * (back(e_dS, q.abs()) + (2 * N * share + 4) * u * back(dS.abs(), q.abs()))
            ref["dV"][a:b, j] += back(P, g)
            tol["dV"][a:b, j] += 1.02 * back(P * (e_G + hs + (2 * N * share + 8) * u) + tiny * keep.double(), g.abs())
    for name in ("dQ", "dK", "dV"):
        tol[name] = tol[name] + rounded(ref[name].abs() + tol[name], dtype)
    return ref, tol


def check(Q, K, V, lengths, scale=None, dO=None):
    off = offsets_of(lengths)
    O, lse = pb.attention(Q, K, V, off, scale=scale)                                                       # noqa: E741
    got = {"O": O, "lse": lse}
    if dO is not None:
        got |= dict(zip(("dQ", "dK", "dV"), pb.attention_grad(dO, Q, K, V, O, lse, off, scale=scale)))
    torch.cuda.synchronize()
    ref, tol = reference(Q, K, V, lengths, scale or Q.shape[2] ** -0.5, O, dO)
    for name, x in got.items():
        close(x, ref[name], tol[name], (name, Q.shape, K.shape, lengths, scale))
    return got


def whole(g, shape, most, dtype):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").to(dtype)


def far_from_zero(D, dtype, lengths, heads, kv):
    """Scores a multiple of 2^-3 (scale 2^-3), spread by 2 or 3 around 2^20, 2^12, 0
    and -2^20, by query and head: tiles hold rows of all kinds."""
    g, T = gen(D + heads), sum(lengths)
    Q, K, V = whole(g, (T, heads, D), 2, dtype), whole(g, (T, kv, D), 2, dtype), normal(g, (T, kv, D), dtype)
    K[:, :, 0] = 4096
    bases = torch.tensor([2048.0, 8.0, 0.0, -2048.0], device="cuda")
    Q[:, :, 0] = bases[(torch.arange(T, device="cuda").view(-1, 1) // 100 + torch.arange(heads, device="cuda")) % 4].to(dtype)
    return Q, K, V, normal(g, (T, heads, D), dtype, 0.5)


# few tiles and long sequences (eight waves a workgroup, keys' tiles shared), many (four waves), ends inside a tile
FAR = [(64, [700], 2, 1), (128, [150, 0, 333], 4, 2), (80, [257, 1], 3, 3), (128, [400, 0, 700], 64, 16), (64, [131, 129], 16, 16),
       (96, [400, 0, 700], 64, 16), (64, [400, 0, 700], 64, 32), (40, [5] * 300, 2, 2)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,lengths,heads,kv", FAR)
def test_attention_of_scores_far_from_zero(dtype, D, lengths, heads, kv):
    Q, K, V, _ = far_from_zero(D, dtype, lengths, heads, kv)
    check(Q, K, V, lengths, scale=0.125)


def large(D, dtype, lengths, heads, kv):
    """fp16 values up to 20480, bf16 ones up to 98304: the largest key of a row takes
    all, or shares with the keys that are the same."""
    g, T = gen(3 * D + heads), sum(lengths)
    unit = 2560 if dtype == F16 else 12288
    Q, K = whole(g, (T, heads, D), 8, dtype) * unit, whole(g, (T, kv, D), 8, dtype) * unit
    K[4::5] = K[3::5][:len(K[4::5])]
    return Q, K, normal(g, (T, kv, D), dtype), whole(g, (T, heads, D), 4, dtype)


LARGE = [(64, [300], 2, 1), (128, [150, 0, 333], 4, 2), (64, [400, 0, 700], 64, 16), (128, [400, 0, 700], 64, 16)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,lengths,heads,kv", LARGE)
def test_attention_of_large_values(dtype, D, lengths, heads, kv):
    Q, K, V, _ = large(D, dtype, lengths, heads, kv)
    check(Q, K, V, lengths)


def ordered(D, dtype, T, sign):
    """Keys with a different score each, of one column: the largest so far takes all."""
    g = gen(5 * D)
    Q, K = torch.zeros((T, 2, D), dtype=dtype, device="cuda"), torch.zeros((T, 1, D), dtype=dtype, device="cuda")
    Q[:, 0, 1], Q[:, 1, 1] = sign, -sign
    K[:, 0, 1] = (torch.randperm(T, generator=g, device="cuda") - T // 2).to(dtype)
    return Q, K, whole(g, (T, 1, D), 4, dtype), whole(g, (T, 2, D), 4, dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("scale", [1e5, 1e10, 1e20])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_a_large_scale(dtype, scale, D):
    T = 200
    for sign in (1, 3):
        Q, K, V, _ = ordered(D, dtype, T, sign)
        got = check(Q, K, V, [T], scale=scale)
        for h in range(2):
            k = K[:, 0, 1].double() * (1 - 2 * h)
            assert torch.equal(got["O"][:, h], V[k.cummax(0).indices, 0])


def test_attention_of_a_small_scale():
    g = gen(30)
    Q, K, V = (normal(g, (300, 2, 64), BF16, 100.0) for _ in range(3))
    O, lse = pb.attention(Q, K, V, offsets_of([300]), scale=1e-20)                                         # noqa: E741
    rows = torch.arange(1, 301, device="cuda").double()
    ref = V.double().cumsum(0) / rows.view(-1, 1, 1)
    size = V.double().abs().cumsum(0) / rows.view(-1, 1, 1)
    # all weights are the same: exponentials of scores below 1e-14 are 1, which is not rounded
    close(O, ref, 700 * u * size + rounded(ref.abs() + 700 * u * size, BF16), "O")
    close(lse, rows.log().expand(2, -1), 8 * u * rows.log().expand(2, -1) + 8 * u, "lse")


def test_attention_of_scores_that_grow_past_the_limit():
    # a row's maximum passes from exponents formed as products to those formed as differences, and back is no way
    g = gen(31)
    T, D = 500, 64
    for dtype in (BF16, F16):
        Q, K = whole(g, (T, 2, D), 2, dtype), whole(g, (T, 2, D), 2, dtype)
        Q[:, :, 0] = 8
        steps = torch.arange(T, device="cuda") // 16 * 64
        K[:, 0, 0], K[:, 1, 0] = steps.to(dtype), (steps - 1000).clamp(min=-960).to(dtype)
        check(Q, K, normal(g, (T, 2, D), dtype), [T], scale=0.125)


# -- gradients -------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,lengths,heads,kv", FAR)
def test_attention_gradients_of_scores_far_from_zero(dtype, D, lengths, heads, kv):
    Q, K, V, dO = far_from_zero(D, dtype, lengths, heads, kv)
    check(Q, K, V, lengths, scale=0.125, dO=dO)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,lengths,heads,kv", LARGE)
def test_attention_gradients_of_large_values(dtype, D, lengths, heads, kv):
    Q, K, V, dO = large(D, dtype, lengths, heads, kv)
    # (keys and queries of 20480 times dS of 1 are beyond fp16: dO of 2^-12 brings dQ and dK to its range)
    check(Q, K, V, lengths, dO=dO if dtype == BF16 else (dO * 2.0 ** -12).to(dtype))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("scale", [1e5, 1e10, 1e20])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_gradients_of_a_large_scale(dtype, scale, D):
    T = 200
    for sign in (1, 3):
        Q, K, V, dO = ordered(D, dtype, T, sign)
        off = offsets_of([T])
        O, lse = pb.attention(Q, K, V, off, scale=scale)                                                   # noqa: E741
        dQ, dK, dV = pb.attention_grad(dO, Q, K, V, O, lse, off, scale=scale)
        # weights are 1 and 0: P (dO . V - dO . O) is 0 exactly, its sums of whole numbers being exact
        assert bool((dQ == 0).all()) and bool((dK == 0).all())
        ref = torch.zeros((T, D), dtype=torch.float64, device="cuda")
        for h in range(2):
            k = K[:, 0, 1].double() * (1 - 2 * h)
            ref.index_add_(0, k.cummax(0).indices, dO[:, h].double())
        close(dV[:, 0], ref, rounded(ref, dtype), "dV")


def test_attention_gradients_of_scores_that_grow_past_the_limit():
    g = gen(32)
    T, D = 500, 64
    for dtype in (BF16, F16):
        Q, K = whole(g, (T, 2, D), 2, dtype), whole(g, (T, 2, D), 2, dtype)
        Q[:, :, 0] = 8
        steps = torch.arange(T, device="cuda") // 16 * 64
        K[:, 0, 0], K[:, 1, 0] = steps.to(dtype), (steps - 1000).clamp(min=-960).to(dtype)
        check(Q, K, normal(g, (T, 2, D), dtype), [T], scale=0.125, dO=normal(g, (T, 2, D), dtype, 0.5))


def test_attention_gradients_at_the_limits_of_the_exponents():
    # |lse| of 2^10 powers of two from both sides, in one tile and in one batch
    g = gen(33)
    T, D, limit = 400, 64, 1024 * math.log(2)
    Q, K = whole(g, (T, 4, D), 2, BF16), whole(g, (T, 4, D), 2, BF16)
    K[:, :, 0] = 16
    base = (limit / 0.125 / 16) * (1 + torch.linspace(-0.04, 0.04, T, device="cuda").view(-1, 1))
    Q[:, :, 0] = (base * torch.tensor([1, -1, 1, 0.25], device="cuda")).to(BF16)
    V, dO = normal(g, (T, 4, D), BF16), normal(g, (T, 4, D), BF16, 0.5)
    got = check(Q, K, V, [T], scale=0.125, dO=dO)
    low, high = got["lse"][0].abs() < limit, got["lse"][0].abs() > limit
    assert bool(low.any()) and bool(high.any())
    check(Q, K, V, [100, 200, 100], scale=0.125, dO=dO)


@pytest.mark.parametrize("dtype,size", [(F16, 6000.0), (BF16, 1e5), (BF16, 1e15)])
@pytest.mark.parametrize("D,lengths,heads,kv", [(64, [400], 2, 1), (128, [150, 0, 333], 4, 2), (128, [400, 0, 700], 64, 16),
                                                (64, [400, 0, 700], 64, 16)])
def test_attention_and_its_gradients_where_sums_round(dtype, size, D, lengths, heads, kv):
    """Values of which Q . K rounds by far more than 1: every pass has to find the same
    score for a query and a key.  The largest is larger than any other by more than both
    roundings (asserted), so that it takes all: P is 1 and 0, and P (dO . V - dO . O) 0."""
    g = torch.Generator().manual_seed(D + heads)
    T = sum(lengths)
    Q, K = ((torch.randn((T, h, D), generator=g).clamp(-5, 5) * size).to(dtype).cuda() for h in (heads, kv))
    V, dO = (torch.randint(-4, 5, (T, h, D), generator=g).to(dtype).cuda() for h in (kv, heads))
    O_ref, lse_ref = torch.zeros((T, heads, D), device="cuda").double(), torch.zeros((heads, T), device="cuda").double()
    dV_ref, e_lse = torch.zeros((T, kv, D), device="cuda").double(), torch.zeros_like(lse_ref)
    clear = torch.ones((T, heads), dtype=torch.bool, device="cuda")
    lone = torch.ones((T, kv), dtype=torch.bool, device="cuda")
    for a, b in parts_of(lengths):
        keep = torch.tril(torch.ones((b - a, b - a), dtype=torch.bool, device="cuda"))
        for h in range(heads if b > a else 0):
            j = h * kv // heads
            q, kt = Q[a:b, h].double(), K[a:b, j].double().t().contiguous()
            S = torch.where(keep, D ** -0.5 * (q @ kt), -math.inf)
            e_S = torch.where(keep, 2 * D * u * D ** -0.5 * (q.abs() @ kt.abs()), 0.0)
            top, at = S.max(1)
            rivals = (S + e_S >= (top - e_S.gather(1, at.view(-1, 1)).view(-1)).view(-1, 1) - 200).sum(1) > 1
            clear[a:b, h] = ~rivals
            # (keys that a row without a clear winner may give weight to)
            lone[a:b, j] &= ~((S + 2 * e_S.amax(1, keepdim=True) >= top.view(-1, 1) - 200) & rivals.view(-1, 1)).any(0)
            O_ref[a:b, h], lse_ref[h, a:b] = V[a:b, j].double()[at], top
            e_lse[h, a:b] = e_S.gather(1, at.view(-1, 1)).view(-1) + 4 * u * top.abs()
            dV_ref[a:b, j].index_add_(0, at, dO[a:b, h].double())
    assert float(clear.double().mean()) > 0.99 and float(lone.double().mean()) > 0.5
    off = offsets_of(lengths)
    O, lse = pb.attention(Q, K, V, off)                                                                    # noqa: E741
    dQ, dK, dV = pb.attention_grad(dO, Q, K, V, O, lse, off)
    torch.cuda.synchronize()
    assert torch.equal(O.double()[clear], O_ref[clear])
    close(lse[clear.t()], lse_ref[clear.t()], e_lse[clear.t()], "lse")
    assert bool((dQ[clear] == 0).all()) and bool((dK[lone] == 0).all())
    close(dV[lone], dV_ref[lone], rounded(dV_ref[lone], dtype), "dV")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lengths,heads,kv,D", [([90, 0, 300, 200], 4, 2, 64), ([90, 0, 300, 200], 96, 32, 128)])
def test_far_sequences_leave_the_others_and_the_rest_as_they_were(dtype, lengths, heads, kv, D):
    g = gen(50 + D)
    first, T = 5, sum(lengths) + 11
    Q, K, V = (normal(g, (T, h, D), dtype) for h in (heads, kv, kv))
    dO, off = normal(g, (T, heads, D), dtype), offsets_of(lengths, first)

    def run():
        arrays = [torch.full(x.shape, 7.25, dtype=dtype, device="cuda") for x in (Q, Q, K, V)]
        lse = torch.full((heads, T), 7.25, device="cuda")
        O, dQ, dK, dV = arrays                                                                             # noqa: E741
        pb.attention(Q, K, V, off, out=O, lse=lse)
        pb.attention_grad(dO, Q, K, V, O, lse, off, dQ=dQ, dK=dK, dV=dV)
        return [lse.t()] + arrays
    clean = run()
    for x in (Q, K, V, dO):
        x[:first], x[first + sum(lengths):] = float("nan"), float("inf")
    middle = slice(first + 90, first + 390)
    Q[middle, :, 0], K[middle, :, 0] = 2048, 4096
    both = run()
    assert float(both[0][middle].min()) > 1e5
    for a, b in zip(clean, both):
        for rows in (slice(0, first + 90), slice(first + 390, T)):
            assert torch.equal(a[rows], b[rows])
        assert bool(torch.isfinite(b.float()).all())


def test_attention_captured_with_scores_of_both_kinds():
    g = gen(60)
    T, D, heads, kv = 300, 64, 4, 2
    Q, K, V, dO = (normal(g, (T, h, D), BF16) for h in (heads, kv, kv, heads))
    off = offsets_of([0, 0, 0])

    def run():
        O, lse = pb.attention(Q, K, V, off)                                                                # noqa: E741
        return O, lse, *pb.attention_grad(dO, Q, K, V, O, lse, off)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for i, (lengths, far) in enumerate((([100, 200, 0], False), ([100, 200, 0], True), ([1, 0, 299], False), ([150, 140, 10], True))):
        for x in (Q, K, V, dO):
            x.copy_(normal(g, x.shape, BF16))
        if far:
            Q[:, :2, 0], K[:, :, 0] = 2048, 4096
        off.copy_(offsets_of(lengths))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        again = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, again)), i
