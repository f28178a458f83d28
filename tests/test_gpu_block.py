"""The operators of a transformer block on the GPU, against plain 64-bit forms.

Tolerances are derived, not tuned, from u = 2^-24 (a rounding to fp32) and the
output type's half step; they are computed beside each reference, from bounds
on every step's error:

Sums of N values in fp32, in any order: N u sum |x| (2 N u on the matrix cores,
which may truncate).  Layer norm's sums over a row are per thread (at most 32
values) and over a tree of at most 22 steps: 64 u.

Exponentials: 2^x of the hardware is right to 2 u; an argument's rounding is u
times its size.

Attention rounds the exponentials, and dS, to the type of its inputs: half a
step of each, which is at most that share of sum P |V| (or of the like sum).
Exponentials are relative to a maximum that is among their row's, so their sum
is at least 1 and what falls below the type's smallest value is at most half of
that each.
"""
import math

import numpy as np
import pytest

pb = pytest.importorskip("paper_2004_14696_amd.binding")
torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rounded(y, dtype):
    """The error of rounding y to dtype, at most."""
    return half_step(dtype) * y.abs() + TINY[dtype] / 2


def offsets_of(lengths, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lengths)]), dtype=torch.int32, device="cuda")


def parts_of(lengths, first=0):
    ends = np.concatenate([[first], first + np.cumsum(lengths)]).astype(int).tolist()
    return list(zip(ends, ends[1:]))


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def ragged(seed, n, T):
    cuts = np.sort(np.random.default_rng(seed).integers(0, T + 1, n - 1))
    return np.diff(np.concatenate([[0], cuts, [T]])).astype(int).tolist()


def close(got, ref, tol, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), float((err - tol)[bad].max()), float((err / tol)[bad].max()))


def inside(shape, dtype, step, fill=float("nan")):
    """An array inside a larger one, filled; columns from `step` on."""
    big = torch.full([s + 2 * step for s in shape], fill, dtype=dtype, device="cuda")
    return big, big[tuple(slice(step, step + s) for s in shape)]


# -- layer norm -------------------------------------------------------------------
def norm_parts(X, eps):
    """64-bit H, 1/sqrt(var + eps), and the errors of both (that of the second
    relative)."""
    X = X.double()
    mean, A = X.mean(1, keepdim=True), X.abs().mean(1, keepdim=True)
    c = X - mean
    var = (c * c).mean(1, keepdim=True)
    e_c = 64 * u * A + u * c.abs()
    e_var = 2 * (c.abs() * e_c + e_c * e_c).mean(1, keepdim=True) + 68 * u * var
    r = (var + eps).rsqrt()
    e_r = 0.5 * e_var / (var + eps) * (1 + e_var / (var + eps)) + 4 * u
    H = c * r
    return H, r, (e_c * r + H.abs() * (e_r + 2 * u)) * (1 + e_r), e_r


def check_norm(X, gamma, beta, lengths, first=0, eps=1e-5, out=None):
    off, T = offsets_of(lengths, first), first + sum(lengths)
    if out is None:
        out = torch.full(X.shape, 7.25, dtype=X.dtype, device="cuda")
    keep = out.clone()
    got = pb.layer_norm(X, gamma, beta, off, eps=eps, out=out)
    torch.cuda.synchronize()
    assert got is out
    H, r, e_h, e_r = norm_parts(X[first:T], eps)
    g, b = gamma.double(), beta.double() if beta is not None else torch.zeros_like(gamma).double()
    ref = H * g + b
    tol = (e_h + 2 * u * H.abs()) * g.abs() + 2 * u * b.abs()
    close(got[first:T], ref, tol + rounded(ref.abs() + tol, X.dtype), ("Y", X.shape, lengths))
    assert torch.equal(got[:first], keep[:first]) and torch.equal(got[T:], keep[T:])
    return got


def check_norm_grad(dY, X, gamma, lengths, first=0, eps=1e-5, **kw):
    off, T, n = offsets_of(lengths, first), first + sum(lengths), len(lengths)
    kw.setdefault("dX", torch.full(X.shape, 7.25, dtype=X.dtype, device="cuda"))
    keep = kw["dX"].clone()
    dX, dg, db = pb.layer_norm_grad(dY, X, gamma, off, eps=eps, **kw)
    torch.cuda.synchronize()
    H, r, e_h, e_r = norm_parts(X[first:T], eps)
    D = dY[first:T].double()
    dH = D * gamma.double()
    m1, m2 = dH.mean(1, keepdim=True), (dH * H).mean(1, keepdim=True)
    e_1 = 66 * u * dH.abs().mean(1, keepdim=True)
    e_2 = (dH.abs() * e_h).mean(1, keepdim=True) + 70 * u * (dH * H).abs().mean(1, keepdim=True) + e_r * m2.abs()
    ref = r * (dH - m1 - H * m2)
    tol = (r * (e_1 + e_h * m2.abs() + H.abs() * e_2 + 6 * u * (dH.abs() + m1.abs() + (H * m2).abs()))
           + ref.abs() * (e_r + 2 * u)) * 1.01
    close(dX[first:T], ref, tol + rounded(ref.abs() + tol, X.dtype), ("dX", X.shape, lengths))
    assert torch.equal(dX[:first], keep[:first]) and torch.equal(dX[T:], keep[T:])
    for i, (a, b) in enumerate(parts_of(lengths)):
        terms = D[a:b] * H[a:b]
        close(dg[i], terms.sum(0), (D[a:b].abs() * e_h[a:b]).sum(0) + (b - a + 4) * u * terms.abs().sum(0) + 1e-300,
              ("dgamma", i))
        if db is not None:
            close(db[i], D[a:b].sum(0), (b - a + 4) * u * D[a:b].abs().sum(0) + 1e-300, ("dbeta", i))
    return dX, dg, db


NORMS = [  # d, lengths: one token, empty groups, rows of fewer than a pack, odd widths, each width of a team
    (1, [1, 3]), (3, [2, 0, 1]), (7, [70]), (8, [1]), (64, [3, 0, 5]), (255, [9, 1]), (256, [64, 65]), (509, [130, 7]),
    (512, [8, 9, 0]), (1000, [33]), (1003, [70, 3]), (1024, [16]), (1025, [5, 6]), (2047, [9]), (2048, [1, 20]),
    (4096, [40, 3]), (4097, [7]), (8192, [3]), (10001, [4, 5]), (16383, [3, 2]), (16384, [1, 9]),
]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("d,lengths", NORMS)
def test_layer_norm_and_its_gradients(dtype, d, lengths):
    g = gen(d)
    T, first = sum(lengths), 2
    X = (normal(g, (T + 5, d), F32, 2.0) + 1.5).to(dtype)
    gamma, beta = 1 + normal(g, (d,), F32, 0.2), normal(g, (d,), F32)
    check_norm(X, gamma, beta, lengths, first=first)
    check_norm(X[:T], gamma, None, lengths)
    dY = normal(g, (T + 5, d), dtype, 0.1)
    check_norm_grad(dY, X, gamma, lengths, first=first)


@pytest.mark.parametrize("n,T,d", [(1, 9000, 96), (64, 3001, 1003), (1000, 700, 40), (3, 2500, 2304), (7, 1300, 6000)])
def test_layer_norm_of_larger_and_ragged_batches(n, T, d):
    g = gen(n + T)
    lengths = ragged(T, n, T)
    X, dY = normal(g, (T, d), BF16), normal(g, (T, d), BF16)
    gamma, beta = 1 + normal(g, (d,), F32, 0.2), normal(g, (d,), F32)
    check_norm(X, gamma, beta, lengths)
    one = check_norm_grad(dY, X, gamma, lengths)
    two = pb.layer_norm_grad(dY, X, gamma, offsets_of(lengths))
    assert all(torch.equal(a, b) for a, b in zip(one, two))       # the same bits each time


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("step", [4, 1])
def test_layer_norm_of_strided_rows_into_worker_gradients(dtype, step):
    g = gen(step)
    n, d, lengths, first, after = 3, 200, [9, 0, 30], 4, 6
    T = first + sum(lengths) + after
    (_, X), (_, dY), (bigX, dX) = inside((T, d), dtype, step), inside((T, d), dtype, step), inside((T, d), dtype, step, 3.5)
    X[first:T - after] = normal(g, (sum(lengths), d), dtype)
    dY[first:T - after] = normal(g, (sum(lengths), d), dtype)
    X[:first], dY[T - after:] = float("nan"), float("inf")
    gamma = 1 + normal(g, (d,), F32, 0.2)
    G = torch.full((n, 2 * d + 11), 3.5, device="cuda")            # the worker gradients [n][P]
    check_norm_grad(dY, X, gamma, lengths, first=first, dX=dX, dgamma=G[:, 3:3 + d], dbeta=G[:, 5 + d:5 + 2 * d])
    rest = torch.cat([G[:, :3], G[:, 3 + d:5 + d], G[:, 5 + 2 * d:]], 1)
    assert bool((rest == 3.5).all()) and bool((G[1, 3:3 + d] == 0).all())
    dX[first:T - after] = 3.5
    assert bool((bigX == 3.5).all())
    _, Y = inside((T, d), dtype, step, 3.5)
    check_norm(X, gamma, gamma, lengths, first=first, out=Y)
    dX, dg, db = pb.layer_norm_grad(dY, X, gamma, offsets_of(lengths, first), dbeta=False)
    assert db is None and torch.equal(dg, G[:, 3:3 + d])


def test_layer_norm_of_constant_large_and_broken_rows():
    d, g = 777, gen(1)
    X = normal(g, (6, d), F32)
    X[0] = 0.0
    X[1] = 3.0                                    # no variance
    X[2] = normal(g, (d,), F32) + 4096.0          # a mean far above it
    X[3, 5], X[4, 700] = float("nan"), float("inf")
    gamma, beta = torch.ones(d, device="cuda"), normal(g, (d,), F32)
    off = offsets_of([3, 1, 1, 1])
    check_norm(X[:3], gamma, beta, [3])
    Y = pb.layer_norm(X, gamma, beta, off)
    assert torch.equal(Y[0], beta) and bool(torch.isnan(Y[3:5]).all()) and bool(torch.isfinite(Y[5]).all())
    dY = normal(g, (6, d), F32)
    dX, dg, db = pb.layer_norm_grad(dY, X, gamma, off)
    assert bool(torch.isfinite(dX[[0, 1, 2, 5]]).all()) and bool(torch.isnan(dX[3:5]).all())
    assert bool(torch.isfinite(dg[[0, 3]]).all()) and bool(torch.isfinite(db).all())


def test_layer_norm_gradients_against_differences():
    # f = sum(R Y): along a direction, (f(+h) - f(-h)) / 2h in 64 bits of the formula
    g = gen(3)
    T, d, lengths, eps = 12, 90, [5, 7], 1e-5
    X, R = normal(g, (T, d), F32), normal(g, (T, d), F32)
    gamma, beta = 1 + normal(g, (d,), F32, 0.2), normal(g, (d,), F32)
    dX, dg, db = pb.layer_norm_grad(R, X, gamma, offsets_of(lengths), eps=eps)

    def f(X, gamma, beta):
        mean, var = X.mean(1, keepdim=True), X.var(1, correction=0, keepdim=True)
        return (R.double() * ((X - mean) / torch.sqrt(var + eps) * gamma + beta)).sum(1)
    x, a, b, h = X.double(), gamma.double(), beta.double(), 1e-5
    D, V = normal(g, (T, d), F32).double(), normal(g, (d,), F32).double()
    # the third derivative's part is h^2, below 1e-8 of these sums; fp32's below 1e-5
    for slope, lo, hi in ((dX.double() * D, (x - h * D, a, b), (x + h * D, a, b)),):
        change = (f(*hi) - f(*lo)) / (2 * h)
        assert float((change - slope.sum(1)).abs().max()) < 1e-4 * d ** 0.5
    for grad, lo, hi in ((dg, (x, a - h * V, b), (x, a + h * V, b)), (db, (x, a, b - h * V), (x, a, b + h * V))):
        change = (f(*hi) - f(*lo)) / (2 * h)
        for i, (p, q) in enumerate(parts_of(lengths)):
            assert abs(float(change[p:q].sum() - (grad[i].double() * V).sum())) < 1e-4 * d ** 0.5


# -- products with an epilogue ------------------------------------------------------
ACTS = ["none", "relu", "gelu", "silu"]
GELU_A, GELU_B = math.sqrt(2 / math.pi), 0.044715 * math.sqrt(2 / math.pi)


def act_of(z, act):
    """Value, slope, and the sigmoid's argument."""
    if act == "none":
        return z, torch.ones_like(z), torch.zeros_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double(), torch.zeros_like(z)
    s, ds = (z, 1.0) if act == "silu" else (2 * (GELU_A * z + GELU_B * z ** 3), 2 * (GELU_A + 3 * GELU_B * z * z))
    p = torch.sigmoid(s)
    return z * p, p + z * p * torch.sigmoid(-s) * ds, s


def check_linear(X, W, lengths, act, bias=None, residual=None, pre=False, first=0, out_dtype=None, out=None):
    off, n, T = offsets_of(lengths, first), len(lengths), X.shape[0]
    d, C = W.shape[-2:]
    dtype = out_dtype or X.dtype
    if out is None:
        out = torch.full((T, C), 7.25, dtype=dtype, device="cuda")
    keep, res = out.clone(), residual.double() if residual is not None else None     # (Y may be R)
    Y, Z = pb.group_linear(X, W, off, bias=bias, activation=act, residual=residual, pre=pre, out=out, out_dtype=dtype)
    torch.cuda.synchronize()
    assert Y is out and (Z is None) == (pre is False)
    for i, (a, b) in enumerate(parts_of(lengths, first)):
        w = (W if W.dim() == 2 else W[i]).double()
        x = X[a:b].double()
        z, size = x @ w, x.abs() @ w.abs()
        if bias is not None:
            v = (bias if bias.dim() == 1 else bias[i]).double()
            z, size = z + v, size + v.abs()
        e_z = 2 * d * u * size + 2 * u * z.abs()
        y, _, s = act_of(z, act)
        # slopes are below 1.13; the sigmoid is off by its argument's roundings (5 u of it) and 6 u
        tol = 1.13 * e_z + (0 if act in ("none", "relu") else y.abs() * u * (5 * s.abs() + 8))
        if res is not None:
            y, tol = y + res[a:b], tol + u * (y.abs() + res[a:b].abs())
        close(Y[a:b], y, tol + rounded(y.abs() + tol, dtype), ("Y", X.shape, W.shape, lengths, act))
        if Z is not None:
            close(Z[a:b], z, e_z + rounded(z.abs() + e_z, X.dtype), ("Z", X.shape, W.shape, lengths, act))
    last = first + sum(lengths)
    assert torch.equal(Y[:first], keep[:first]) and torch.equal(Y[last:], keep[last:])
    return Y, Z


LINEARS = [  # d, C, lengths: one token, empty groups, odd widths, tiles that end inside, parts of the sum
    (64, 64, [1]), (8, 8, [1, 0, 2]), (1, 1, [5, 2]), (7, 3, [1, 9]), (65, 129, [130, 1, 63]), (130, 255, [64, 65]),
    (77, 8, [64, 65]), (264, 520, [300, 17]), (512, 256, [700, 100, 513]), (200, 1000, [0, 0, 0]), (4096, 40, [3, 2]),
    (2048, 1408, [37]), (5000, 33, [4, 0, 7]),
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("d,C,lengths", LINEARS)
def test_linear_with_every_part_of_its_epilogue(dtype, act, d, C, lengths):
    g = gen(d * 1000 + C)
    n, T = len(lengths), sum(lengths)
    X, W = normal(g, (T, d), dtype), normal(g, (n, d, C), dtype, 1.5 / math.sqrt(d))
    b = normal(g, (n, C), F32)
    R = {t: normal(g, (T, C), t) for t in (dtype, F32)}
    check_linear(X, W, lengths, act, bias=b, residual=R[dtype], pre=True)
    check_linear(X, W, lengths, act, residual=R[F32], out_dtype=F32)
    check_linear(X, W, lengths, act, bias=b[0])
    check_linear(X, W[0], lengths, act, bias=b[0], pre=True, out_dtype=F32)


@pytest.mark.parametrize("T,n,d,C,shared", [(6000, 3, 1000, 2047, False), (4096, 16, 512, 4096, True), (37, 16, 2048, 1408, False),
                                            (40, 500, 64, 128, False), (9000, 1, 136, 520, True)])
def test_linear_of_larger_sizes(T, n, d, C, shared):
    g = gen(T + n)
    X, W = normal(g, (T, d), BF16), normal(g, (d, C) if shared else (n, d, C), BF16, 1 / math.sqrt(d))
    b, R = normal(g, (C,) if shared else (n, C), F32), normal(g, (T, C), BF16)
    check_linear(X, W, ragged(T + n, n, T), "gelu", bias=b, residual=R, pre=True)


@pytest.mark.parametrize("d", [72, 4096])
@pytest.mark.parametrize("step", [8, 1])
def test_linear_of_strided_arrays_and_into_the_residual(step, d):
    g = gen(step)
    C, lengths, first, after = 136, [30, 0, 7, 5], 9, 11
    n, T = len(lengths), first + sum(lengths) + after
    _, X = inside((T, d), F16, step)
    _, W = inside((n, d, C), F16, step)
    _, b = inside((n, C), F32, step)
    X[first:T - after] = normal(g, (sum(lengths), d), F16)
    W.copy_(normal(g, (n, d, C), F16, 1 / math.sqrt(d)))
    b.copy_(normal(g, (n, C), F32))
    for dtype in (F16, F32):
        bigY, Y = inside((T, C), dtype, step, 3.5)
        bigZ, Z = inside((T, C), F16, step, 3.5)
        rows = normal(g, (sum(lengths), C), dtype)
        Y[first:T - after] = rows
        check_linear(X, W, lengths, "silu", bias=b, residual=Y, pre=Z, first=first, out_dtype=dtype, out=Y)
        Y[first:T - after] = 3.5
        Z[first:T - after] = 3.5
        assert bool((bigY == 3.5).all()) and bool((bigZ == 3.5).all())


def test_linear_without_an_epilogue_is_the_product():
    g = gen(8)
    for T, d, C in ((300, 256, 512), (5, 4096, 40), (70, 33, 65)):
        X, W, off = normal(g, (T, d), BF16), normal(g, (2, d, C), BF16), offsets_of(ragged(1, 2, T))
        for dtype in (BF16, F32):
            assert torch.equal(pb.group_linear(X, W, off, out_dtype=dtype)[0], pb.group_matmul(X, W, off, out_dtype=dtype))


# -- the way back through an activation ---------------------------------------------------
def check_linear_grad(dY, Z, lengths, act, first=0, **kw):
    off, last = offsets_of(lengths, first), first + sum(lengths)
    kw.setdefault("dZ", torch.full(dY.shape, 7.25, dtype=dY.dtype, device="cuda"))
    keep = kw["dZ"].clone()
    dZ, db = pb.group_linear_grad(dY, off, pre=Z, activation=act, **kw)
    torch.cuda.synchronize()
    D, z = dY[first:last].double(), Z[first:last].double()
    _, slope, s = act_of(z, act)
    # s has a relative error of 4 u (two constants, two products, a sum), and 2 u more as an exponent of 2: e = exp(-s)
    # is off by 6 u |s| + 2 u, p = 1 / (1 + e) by (1 - p) of that and 3 u, q = e p by p of that and 4 u; z p q s' by both,
    # 2 u for its products and 4 u for s'; the last sum and the product with dY by u each.  A slope below 2^-100 may be 0.
    p, q = torch.sigmoid(s), torch.sigmoid(-s)
    big = (z.abs() * (2 * (GELU_A + 3 * GELU_B * z * z) if act == "gelu" else 1.0)).clamp(max=1e4)
    e = 2 * u * slope.abs() + 1e-30
    if act in ("gelu", "silu"):
        e = e + u * (p * q * (big * (6 * s.abs() + 15) + 6 * s.abs()) + 5 * p)
    ref, tol = D * slope, D.abs() * e
    close(dZ[first:last], ref, tol + rounded(ref.abs() + tol, dY.dtype), ("dZ", dY.shape, act))
    assert torch.equal(dZ[:first], keep[:first]) and torch.equal(dZ[last:], keep[last:])
    if db is not None:
        for i, (a, b) in enumerate(parts_of(lengths)):
            close(db[i], ref[a:b].sum(0), tol[a:b].sum(0) + (b - a + 4) * u * ref[a:b].abs().sum(0) + 1e-300, ("dbias", i, act))
    return dZ, db


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("C,lengths", [(1, [1, 3]), (3, [2, 0, 1]), (8, [300]), (33, [9, 70]), (64, [1]), (100, [17, 16, 0]),
                                       (512, [33]), (1003, [70, 3]), (4096, [40, 5]), (9001, [2, 1])])
def test_linear_grad(dtype, act, C, lengths):
    g = gen(C)
    T = sum(lengths) + 6
    dY, Z = normal(g, (T, C), dtype, 0.1), normal(g, (T, C), dtype, 2.0)
    dZ, db = check_linear_grad(dY, Z, lengths, act, first=2)
    if act == "none":
        same, db2 = pb.group_linear_grad(dY, offsets_of(lengths, 2))
        assert same is dY and torch.equal(db, db2)
    none = pb.group_linear_grad(dY, offsets_of(lengths, 2), pre=Z, activation=act, dZ=torch.zeros_like(dZ), dbias=False)
    assert none[1] is None and torch.equal(none[0][2:T - 4], dZ[2:T - 4])


def test_linear_grad_of_many_workers_strided_into_worker_gradients():
    g = gen(5)
    n, T, C = 300, 5000, 260
    lengths = ragged(3, n, T)
    (_, dY), (_, Z) = inside((T, C), BF16, 1), inside((T, C), BF16, 1)
    dY.copy_(normal(g, (T, C), BF16)), Z.copy_(normal(g, (T, C), BF16))
    G = torch.full((n, C + 20), 3.5, device="cuda")
    big, dZ = inside((T, C), BF16, 1, 3.5)
    check_linear_grad(dY, Z, lengths, "gelu", dZ=dZ, dbias=G[:, 7:7 + C])
    assert bool((G[:, :7] == 3.5).all()) and bool((G[:, 7 + C:] == 3.5).all())
    a, b = pb.group_linear_grad(dY, offsets_of(lengths), pre=Z, activation="gelu")
    assert torch.equal(a, dZ) and torch.equal(b, G[:, 7:7 + C])


def test_activations_of_extreme_arguments():
    z = torch.tensor([[0.0, -0.0, 1e-30, -1e-30, 30.0, -30.0, 200.0, -200.0, 1e20, -1e20, 3e38, -3e38, float("nan")]], device="cuda")
    one, off = torch.ones_like(z), offsets_of([1])
    for act in ("relu", "gelu", "silu"):
        dZ, _ = pb.group_linear_grad(one, off, pre=z, activation=act)
        _, slope, _ = act_of(z.double().clamp(-300, 300), act)
        close(dZ[:, :12], slope[:, :12], torch.full_like(slope[:, :12], 1e-6), act)
        assert math.isnan(float(dZ[0, 12]))


# -- dropout ------------------------------------------------------------------------------
def philox(c, k):
    """Philox4x32-10 of a counter and a key, in plain integers."""
    c, (k0, k1) = list(c), k
    for _ in range(10):
        p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [q >> 32 ^ c[1] ^ k0, q & 0xFFFFFFFF, p >> 32 ^ c[3] ^ k1, p & 0xFFFFFFFF]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def dropout_bits(T, d, seed, step):
    M = 0xFFFFFFFF
    c = np.zeros((T, (d + 7) // 8, 4), dtype=np.uint64)
    c[..., 0], c[..., 1] = np.arange((d + 7) // 8), np.arange(T)[:, None]
    c[..., 2], c[..., 3] = step & M, step >> 32
    k0, k1 = seed & M, seed >> 32
    for _ in range(10):
        p, q = np.uint64(0xD2511F53) * c[..., 0], np.uint64(0xCD9E8D57) * c[..., 2]
        sh, m = np.uint64(32), np.uint64(M)
        c = np.stack([q >> sh ^ c[..., 1] ^ np.uint64(k0), q & m, p >> sh ^ c[..., 3] ^ np.uint64(k1), p & m], -1)
        k0, k1 = k0 + 0x9E3779B9 & M, k1 + 0xBB67AE85 & M
    return np.stack([c & np.uint64(0xFFFF), c >> np.uint64(16)], -1).reshape(T, -1)[:, :d].astype(np.int64)


def check_dropout(X, p, seed, lengths, first=0, R=None, step=None, out=None):
    off, last = offsets_of(lengths, first), first + sum(lengths)
    if out is None:
        out = torch.full(X.shape, 7.25, dtype=X.dtype, device="cuda")
    x, res, keep = X.double(), R.double() if R is not None else torch.zeros_like(X).double(), out.clone()
    Y = pb.dropout(X, p, seed, off, residual=R, step=torch.tensor([step], device="cuda") if step is not None else None, out=out)
    torch.cuda.synchronize()
    q = round(65536 * p)
    kept = torch.from_numpy(dropout_bits(X.shape[0], X.shape[1], seed & (1 << 64) - 1, step or 0)).cuda() >= q
    # (a dropped value is not there, whatever it is)
    y = torch.where(kept, x * (65536 / (65536 - q) if q < 65536 else 0.0), 0.0)
    ref, tol = y + res, 2 * u * y.abs() + u * (y + res).abs()
    rows = slice(first, last)
    close(Y[rows], ref[rows], (tol + rounded(ref.abs() + tol, X.dtype))[rows], ("dropout", X.shape, p))
    assert torch.equal(Y[:first], keep[:first]) and torch.equal(Y[last:], keep[last:])
    return Y, kept


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,d", [(1, 1), (3, 7), (5, 8), (40, 33), (300, 64), (37, 1000), (9, 4099), (2, 70000)])
def test_dropout(dtype, T, d):
    g = gen(d)
    X, R = normal(g, (T + 3, d), dtype), normal(g, (T + 3, d), dtype)
    for p, seed, step in ((0.1, 1234567890123456789, None), (0.5, -5, 7), (0.25, 0, (3 << 32) + 1)):
        check_dropout(X, p, seed, [T], first=1, step=step)
        check_dropout(X, p, seed, ragged(d, 3, T), first=2, R=R, step=step)
    Y, _ = check_dropout(X, 0.0, 5, [T])
    assert torch.equal(Y[:T], X[:T])
    assert bool((check_dropout(X, 1.0, 5, [T])[0][:T] == 0).all())


def test_dropout_strided_and_in_place():
    g = gen(9)
    T, d = 21, 90
    _, X = inside((T, d), BF16, 1)
    big, Y = inside((T, d), BF16, 3, 3.5)
    X.copy_(normal(g, (T, d), BF16))
    R = normal(g, (T, d), BF16)
    want, _ = check_dropout(X, 0.3, 11, [T], R=R, out=Y)
    want = want.clone()
    Y.fill_(3.5)
    assert bool((big == 3.5).all())
    off = offsets_of([T])
    for name in ("X", "R"):
        x, r = X.clone(), R.clone()
        got = pb.dropout(x, 0.3, 11, off, residual=r, out=x if name == "X" else r)
        assert torch.equal(got, want)


def test_dropout_keeps_the_mean_and_masks_the_gradient_alike():
    T, d, p = 512, 2048, 0.25
    X = torch.ones((T, d), device="cuda")
    off = offsets_of([T])
    Y = pb.dropout(X, p, 77, off)
    dX = pb.dropout(torch.full_like(X, 2.0), p, 77, off)
    assert torch.equal(dX, 2 * Y)
    kept = (Y > 0).double()
    # a share of 2^20 fair draws: 6 standard deviations
    assert abs(float(kept.mean()) - 0.75) < 6 * math.sqrt(p * (1 - p) / (T * d))
    # rows, columns and steps draw apart: agreement of two masks is p^2 + (1 - p)^2
    other = (pb.dropout(X, p, 77, off, step=torch.ones(1, dtype=torch.int64, device="cuda")) > 0).double()
    same = p * p + (1 - p) ** 2
    for a, b in ((kept, other), (kept[:-1], kept[1:]), (kept[:, :-1], kept[:, 1:]), (kept[:, :-8], kept[:, 8:])):
        assert abs(float((a == b).double().mean()) - same) < 8 * math.sqrt(same * (1 - same) / (T * d))
    # a NaN that is dropped leaves no trace
    X[:] = float("nan")
    Y2 = pb.dropout(X, p, 77, off)
    assert torch.equal(torch.isnan(Y2), kept > 0) and bool((Y2[kept == 0] == 0).all())


# -- attention ------------------------------------------------------------------------------
def attention_ref(Q, K, V, lengths, scale, dO=None, first=0):
    """64-bit results and bounds on the errors of the kernels' steps, per array."""
    dtype, dev = Q.dtype, Q.device
    T, heads, D = Q.shape
    share, hs, tiny = heads // K.shape[1], half_step(dtype), TINY[dtype] / 2
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device=dev)                                        # noqa: E731
    out = {"O": z(T, heads, D), "lse": z(heads, T), "dQ": z(*Q.shape), "dK": z(*K.shape), "dV": z(*V.shape)}
    tol = {k: torch.zeros_like(v) for k, v in out.items()}
    for a, b in parts_of(lengths, first):
        N = b - a
        if N == 0:
            continue
        keep = torch.tril(torch.ones((N, N), dtype=torch.bool, device=dev))
        for h in range(heads):
            j = h // share
            q, k, v = Q[a:b, h].double().contiguous(), K[a:b, j].double().contiguous(), V[a:b, j].double().contiguous()
            kt, vt = k.t().contiguous(), v.t().contiguous()
            S = torch.where(keep, scale * (q @ kt), -math.inf)
            lse = torch.logsumexp(S, 1, keepdim=True)
            P = torch.exp(S - lse)
            top = S.amax(1, keepdim=True)
            e_S = 2 * D * u * scale * (q.abs() @ kt.abs())
            # exponents, from a maximum at most 8 (in powers of two) below the row's: the scale's and the sum's roundings
            size = torch.where(keep, (S - top).abs() + 6, 0.0)
            e_P = torch.where(keep, e_S + 4 * u * size + 4 * u, 0.0)
            e_row = (P * e_P).sum(1, keepdim=True)
            O = P @ v                                                                                      # noqa: E741
            t = (P * (e_P + e_row + hs + (2 * N + 8) * u)) @ v.abs() + tiny * (keep.double() @ v.abs())
            t = 1.02 * t
            out["O"][a:b, h], tol["O"][a:b, h] = O, t + rounded(O.abs() + t, dtype)
            e_lse = e_row + (N + 8) * u + 4 * u * (lse.abs() + top.abs())
            out["lse"][h, a:b], tol["lse"][h, a:b] = lse.view(-1), 1.02 * e_lse.view(-1)
            if dO is None:
                continue
            g = dO[a:b, h].double().contiguous()
            dP, delta = g @ vt, (g * O).sum(1, keepdim=True)
            # exp(S - lse): the sum's error, and both terms' roundings
            e_G = torch.where(keep, e_S + e_lse + 4 * u * (torch.where(keep, S, 0.0).abs() + lse.abs()) + 4 * u, 0.0)
            e_dP = 2 * D * u * (g.abs() @ vt.abs())
            e_delta = (g.abs() * tol["O"][a:b, h]).sum(1, keepdim=True) + D * u * (g * O).abs().sum(1, keepdim=True)
            dS = P * (dP - delta)
            e_dS = P * (e_dP + e_delta) * (1 + e_G) + dS.abs() * (e_G + 4 * u)
            e_dS = e_dS + hs * (dS.abs() + e_dS) + tiny * keep.double()
            e_dS = 1.02 * e_dS
            out["dQ"][a:b, h] = scale * (dS @ k)
            tol["dQ"][a:b, h] = scale * (e_dS @ k.abs() + (2 * N + 4) * u * (dS.abs() @ k.abs()))
            out["dK"][a:b, j] += scale * (dS.t().contiguous() @ q)
            tol["dK"][a:b, j] += scale * (e_dS.t().contiguous() @ q.abs() + (2 * N * share + 4) * u * (dS.abs().t().contiguous() @ q.abs()))
            Pt = P.t().contiguous()
            e_P2 = (P * (e_G + hs + (2 * N * share + 8) * u) + tiny * keep.double()).t().contiguous()
            out["dV"][a:b, j] += Pt @ g
            tol["dV"][a:b, j] += 1.02 * (e_P2 @ g.abs())
    for name in ("dQ", "dK", "dV"):
        tol[name] = tol[name] + rounded(out[name].abs() + tol[name], dtype)
    return out, tol


def check_attention(Q, K, V, lengths, dO=None, scale=None, first=0, out=None, grads=(None, None, None)):
    off, T, last = offsets_of(lengths, first), Q.shape[0], first + sum(lengths)
    full = lambda x: torch.full(x.shape, 7.25, dtype=x.dtype, device="cuda")                               # noqa: E731
    out = full(Q) if out is None else out
    lse = torch.full((Q.shape[1], T), 7.25, device="cuda")
    arrays = {"O": out, "lse": lse}
    if dO is not None:
        arrays |= {k: full(x) if t is None else t for k, x, t in zip(("dQ", "dK", "dV"), (Q, K, V), grads)}
    keep = {k: x.clone() for k, x in arrays.items()}
    got = pb.attention(Q, K, V, off, scale=scale, out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    if dO is not None:
        pb.attention_grad(dO, Q, K, V, out, lse, off, scale=scale, dQ=arrays["dQ"], dK=arrays["dK"], dV=arrays["dV"])
    torch.cuda.synchronize()
    ref, tol = attention_ref(Q, K, V, lengths, scale or Q.shape[2] ** -0.5, dO, first)
    for name, x in arrays.items():
        rows = (slice(None), slice(first, last)) if name == "lse" else (slice(first, last),)
        close(x[rows], ref[name][rows], tol[name][rows], (name, Q.shape, K.shape, lengths))
        for rest in (slice(0, first), slice(last, T)):
            rest = (slice(None), rest) if name == "lse" else (rest,)
            assert torch.equal(x[rest], keep[name][rest]), name
    return arrays


ATTENTIONS = [  # lengths, heads, kv_heads, D: one token, empty sequences, ends inside a tile, each width
    ([1], 1, 1, 64), ([1, 0, 2, 1], 2, 1, 8), ([31, 33], 2, 2, 64), ([32, 64], 4, 2, 128), ([65, 1, 63], 3, 3, 96),
    ([127], 4, 1, 80), ([128, 129], 2, 1, 40), ([130, 0, 0, 200], 6, 2, 64), ([257], 1, 1, 128), ([300, 5], 8, 8, 72),
    ([500, 77], 4, 4, 104), ([0, 0], 2, 2, 64), ([190, 2, 320, 33], 12, 4, 128), ([1000], 2, 1, 96), ([64], 5, 5, 16),
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lengths,heads,kv,D", ATTENTIONS)
def test_attention_and_its_gradients(dtype, lengths, heads, kv, D):
    g = gen(D + heads)
    first, T = 3, sum(lengths) + 7
    Q, K, V = normal(g, (T, heads, D), dtype), normal(g, (T, kv, D), dtype), normal(g, (T, kv, D), dtype)
    dO = normal(g, (T, heads, D), dtype, 0.5)
    for x in (Q, K, V, dO):                       # rows of no sequence reach nothing
        x[:first], x[T - 4:] = float("nan"), float("inf")
    check_attention(Q, K, V, lengths, dO, first=first)
    check_attention(Q[first:T - 4], K[first:T - 4], V[first:T - 4], lengths, scale=0.3)


@pytest.mark.parametrize("n,T,heads,kv,D", [(70, 700, 4, 2, 64), (4200, 5000, 1, 1, 32), (9, 4000, 2, 1, 128), (1, 3000, 1, 1, 64),
                                             (60, 1500, 12, 4, 128), (60, 1500, 12, 12, 80), (2, 1500, 8, 1, 128),
                                             (300, 2000, 3, 3, 96)])
def test_attention_of_many_and_long_sequences(n, T, heads, kv, D):
    g = gen(n)
    lengths = ragged(n, n, T)
    Q, K, V = normal(g, (T, heads, D), BF16), normal(g, (T, kv, D), BF16), normal(g, (T, kv, D), BF16)
    dO = normal(g, (T, heads, D), BF16)
    one = check_attention(Q, K, V, lengths, dO)
    off = offsets_of(lengths)
    O, lse = pb.attention(Q, K, V, off)                                                                    # noqa: E741
    two = (O, lse) + pb.attention_grad(dO, Q, K, V, O, lse, off)
    assert all(torch.equal(a, b) for a, b in zip(one.values(), two))      # the same bits each time
    assert pb.attention(Q, K, V, off, lse=False)[1] is None


@pytest.mark.parametrize("layout", ["packed", "heads first", "one kv head for all"])
def test_attention_of_strided_arrays(layout):
    g = gen(4)
    lengths, heads, kv, D, first = [70, 0, 140], 4, 2, 72, 2
    T = first + sum(lengths) + 3
    if layout == "packed":
        x, d = (torch.full((T, heads + 2 * kv + 1, D + 8), 3.5, dtype=BF16, device="cuda") for _ in range(2))
        x.copy_(normal(g, x.shape, BF16))
        cut = lambda y: (y[:, :heads, 8:], y[:, heads:heads + kv, :D], y[:, heads + kv:-1, :D])            # noqa: E731
    else:
        x, d = (torch.full((heads + 2 * kv, T, D), 3.5, dtype=BF16, device="cuda") for _ in range(2))
        x.copy_(normal(g, x.shape, BF16))
        cut = lambda y: tuple(p.transpose(0, 1) for p in (y[:heads], y[heads:heads + kv], y[heads + kv:]))  # noqa: E731
    Q, K, V = cut(x)
    dO, grads = normal(g, Q.shape, BF16), cut(d)
    if layout == "one kv head for all":
        K, V = K[:, :1].expand(T, kv, D), V[:, :1].expand(T, kv, D)      # a stride of 0
    check_attention(Q, K, V, lengths, dO, first=first, grads=grads)
    for y in grads:
        y[first:first + sum(lengths)] = 3.5
    assert bool((d == 3.5).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attention_of_growing_large_and_equal_scores(dtype):
    g = gen(6)
    T, D = 400, 64
    Q, K, V = normal(g, (T, 2, D), dtype), normal(g, (T, 2, D), dtype), normal(g, (T, 2, D), dtype)
    dO = normal(g, (T, 2, D), dtype)
    Q[:, 0] = Q[:1, 0]
    K[:, 0] = (K[0, 0].float() + torch.arange(T, device="cuda").view(-1, 1) * 0.02 * Q[0, 0].float()).to(dtype)   # maxima grow
    K[:, 1] = K[:1, 1]                                                                                     # all the same
    check_attention(Q, K, V, [T], dO)
    check_attention(Q, K, V, [150, 250], dO, scale=8.0)          # nearly one key a query
    check_attention(Q, K, V, [T], dO, scale=1e-6)


def test_attention_gradients_of_any_size_in_fp16():
    # dS from far below the normal range of fp16 to far above 64, in one call
    g = gen(16)
    T, D = 300, 64
    Q, K, V = normal(g, (T, 4, D), F16), normal(g, (T, 2, D), F16), normal(g, (T, 2, D), F16)
    dO = normal(g, (T, 4, D), F32)
    dO[:, 0] *= 1e-3
    dO[:, 1] *= 300.0
    dO[150:, 2] *= 2000.0
    dO[100, 3] *= 500.0
    check_attention(Q, K, V, [T], dO.to(F16))
    check_attention(Q, K, V, [40, 200, 60], dO.to(F16))


def test_attention_keeps_sequences_apart():
    g = gen(7)
    lengths, T = [40, 100, 3, 90], 233
    Q, K, V, dO = (normal(g, (T, 2, 64), BF16) for _ in range(4))
    clean = check_attention(Q, K, V, lengths, dO)
    for x in (Q, K, V, dO):
        x[40:140] = float("nan")
        x[140:143] = float("inf")
    off = offsets_of(lengths)
    O, lse = pb.attention(Q, K, V, off)                                                                    # noqa: E741
    got = (O, lse) + pb.attention_grad(dO, Q, K, V, O, lse, off)
    for x, (name, y) in zip(got, clean.items()):
        for rows in (slice(0, 40), slice(143, 233)):
            rows = (slice(None), rows) if name == "lse" else (rows,)
            assert torch.equal(x[rows], y[rows]), name


def test_attention_gradients_against_differences():
    g = gen(8)
    lengths, heads, kv, D = [9, 20], 4, 2, 16
    T, scale, h = 29, 0.25, 1e-4
    Q, K, V, R = (normal(g, (T, k, D), F16) for k in (heads, kv, kv, heads))
    off = offsets_of(lengths)
    O, lse = pb.attention(Q, K, V, off)                                                                    # noqa: E741
    grads = pb.attention_grad(R, Q, K, V, O, lse, off)

    def f(Q, K, V):
        all = 0.0
        for a, b in parts_of(lengths):
            keep = torch.tril(torch.ones((b - a, b - a), dtype=torch.bool, device="cuda"))
            for i in range(heads):
                j = i // (heads // kv)
                S = torch.where(keep, scale * (Q[a:b, i] @ K[a:b, j].t().contiguous()), -math.inf)
                all += float((R[a:b, i].double() * (torch.softmax(S, 1) @ V[a:b, j])).sum())
        return all
    x = [t.double() for t in (Q, K, V)]
    _, tol = attention_ref(Q, K, V, lengths, scale, R)
    for i, name in enumerate(("dQ", "dK", "dV")):
        D_ = normal(g, x[i].shape, F32).double()
        hi, lo = ([y + s * h * D_ if k == i else y for k, y in enumerate(x)] for s in (1, -1))
        change = (f(*hi) - f(*lo)) / (2 * h)
        # (the difference's own error: h^2 of a third derivative that is a few thousand at most, 64-bit noise / h)
        assert abs(change - float((grads[i].double() * D_).sum())) <= float((tol[name] * D_.abs()).sum()) + 1e-4, name


def test_attention_and_rows_beyond_two_to_the_31_elements():
    # token strides that put the last rows of Q, K, V and dO beyond 2^32 bytes
    T, heads, D, wide = 1200, 1, 64, (1 << 21) - 8
    store = torch.zeros((T - 1) * wide + 4 * D, dtype=BF16, device="cuda")
    g = gen(9)
    Q, K, V, dO = (store.as_strided((T, heads, D), (wide, D, 1), i * D) for i in range(4))
    for x in (Q, K, V, dO):
        x.copy_(normal(g, x.shape, BF16))
    check_attention(Q, K, V, [T - 300, 300], dO)


def test_norms_activations_and_dropout_beyond_two_to_the_31_elements():
    T, d = (1 << 17) + 5, 16384               # 2.1e9 values
    X = torch.zeros((T, d), dtype=BF16, device="cuda")
    g, tail = gen(10), 40
    X[-tail:] = normal(g, (tail, d), BF16)
    gamma = 1 + normal(g, (d,), F32, 0.2)
    off = offsets_of([T - 20, 20])
    small = X[-tail:].clone()
    s_off = offsets_of([20, 20])
    Y, Ys = pb.layer_norm(X, gamma, gamma, off), pb.layer_norm(small, gamma, gamma, s_off)
    assert torch.equal(Y[-tail:], Ys)
    dX, dg, _ = pb.layer_norm_grad(Y, X, gamma, off)
    dXs, dgs, _ = pb.layer_norm_grad(Ys, small, gamma, s_off)
    assert torch.equal(dX[-tail:], dXs)
    # (rows of zeros add nothing to dgamma; the chunks' borders differ, and with them the order of 20 terms)
    close(dg, dgs.double(), 64 * u * (Ys.double().abs().sum(0) * 130).expand(2, d), "dgamma")
    del dX, Y
    dZ, db = pb.group_linear_grad(X, off, pre=X, activation="silu")
    dZs, dbs = pb.group_linear_grad(small, s_off, pre=small, activation="silu")
    assert torch.equal(dZ[-tail:], dZs)
    close(db, dbs.double(), 64 * u * (dZs.double().abs().sum(0)).expand(2, d) + 1e-300, "dbias")
    Y = pb.dropout(X, 0.5, 3, off, out=dZ)
    for t in (T - 1, T - 7):
        bits = np.array([pb.load_library().dbw_dropout_bits(3, 0, t, c) for c in range(0, d, 97)])
        got, x = Y[t, ::97].cpu().float().numpy(), X[t, ::97].cpu().float().numpy()
        assert np.array_equal(got, np.where(bits >= 32768, 2 * x, 0))


# -- together ----------------------------------------------------------------------------------
class Block:
    """A transformer block of two products' width F, its forward and backward
    pass in calls of the framework; workers' gradients go to G [n][P]."""

    def __init__(self, d=64, heads=4, kv=2, F=160, dtype=BF16, seed=0):
        g = gen(seed)
        self.d, self.heads, self.kv, self.F, self.D, self.dtype = d, heads, kv, F, d // heads, dtype
        qkv = (heads + 2 * kv) * self.D
        shapes = {"g1": (d,), "b1": (d,), "Wqkv": (d, qkv), "bqkv": (qkv,), "Wo": (d, d), "bo": (d,), "g2": (d,), "b2": (d,),
                  "W1": (d, F), "c1": (F,), "W2": (F, d), "c2": (d,)}
        self.at, P = {}, 0
        for name, s in shapes.items():
            self.at[name] = (P, s)
            P += int(np.prod(s))
        self.P = P
        self.w = torch.zeros(P, device="cuda")
        for name, s in shapes.items():
            self.view(self.w, name).copy_(normal(g, s, F32, 0.1 if len(s) == 1 else 1 / math.sqrt(s[0])) + (name in ("g1", "g2")))
        self.low = self.w.to(dtype)
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def view(self, flat, name):
        a, s = self.at[name]
        x = flat[..., a:a + int(np.prod(s))]
        return x.view(*flat.shape[:-1], *s) if flat.dim() == 1 else x.unflatten(-1, s) if len(s) > 1 else x

    def run(self, X, workers, sequences, dY, G, p=0.1):
        w, low = (lambda n: self.view(self.w, n)), (lambda n: self.view(self.low, n))
        G_ = lambda n: self.view(G, n)                                                                    # noqa: E731
        q, k = self.heads, self.heads + self.kv
        split = lambda x: (x[:, :q], x[:, q:k], x[:, k:])                                                 # noqa: E731
        H1 = pb.layer_norm(X, w("g1"), w("b1"), workers)
        qkv = pb.group_linear(H1, low("Wqkv"), workers, bias=w("bqkv"))[0].view(len(X), -1, self.D)
        O, lse = pb.attention(*split(qkv), sequences)                                                     # noqa: E741
        A = pb.group_linear(O.view(len(X), -1), low("Wo"), workers, bias=w("bo"))[0]
        X1 = pb.dropout(A, p, 1, workers, residual=X, step=self.step)
        H2 = pb.layer_norm(X1, w("g2"), w("b2"), workers)
        M, Z = pb.group_linear(H2, low("W1"), workers, bias=w("c1"), activation="gelu", pre=True)
        B = pb.group_linear(M, low("W2"), workers, bias=w("c2"))[0]
        Y = pb.dropout(B, p, 2, workers, residual=X1, step=self.step)

        dB = pb.dropout(dY, p, 2, workers, step=self.step)
        pb.group_linear_grad(dB, workers, dbias=G_("c2"))
        pb.group_weight_grad(M, dB, workers, out=G_("W2"))
        dZ, _ = pb.group_linear_grad(pb.group_input_grad(dB, low("W2"), workers), workers, pre=Z, activation="gelu", dbias=G_("c1"))
        pb.group_weight_grad(H2, dZ, workers, out=G_("W1"))
        dH2 = pb.group_input_grad(dZ, low("W1"), workers)
        dX1 = pb.layer_norm_grad(dH2, X1, w("g2"), workers, dgamma=G_("g2"), dbeta=G_("b2"))[0] + dY
        dA = pb.dropout(dX1, p, 1, workers, step=self.step)
        pb.group_linear_grad(dA, workers, dbias=G_("bo"))
        pb.group_weight_grad(O.view(len(X), -1), dA, workers, out=G_("Wo"))
        dO = pb.group_input_grad(dA, low("Wo"), workers).view(len(X), -1, self.D)
        dqkv = torch.empty_like(qkv)
        dQ, dK, dV = split(dqkv)
        pb.attention_grad(dO, *split(qkv), O, lse, sequences, dQ=dQ, dK=dK, dV=dV)
        dqkv = dqkv.view(len(X), -1)
        pb.group_linear_grad(dqkv, workers, dbias=G_("bqkv"))
        pb.group_weight_grad(H1, dqkv, workers, out=G_("Wqkv"))
        dH1 = pb.group_input_grad(dqkv, low("Wqkv"), workers)
        dX = pb.layer_norm_grad(dH1, X, w("g1"), workers, dgamma=G_("g1"), dbeta=G_("b1"))[0] + dX1
        return Y, dX

    def plain(self, X, workers, sequences, p=0.1):
        """The same in 64 bits, from parameters [n][P] of each worker's own."""
        def f(params):
            rows = [list(range(a, b)) for a, b in parts_of(workers)]
            of = torch.cat([torch.full((len(r),), i) for i, r in enumerate(rows)]).long().cuda()
            get = lambda n: self.view(params, n)                                                          # noqa: E731

            def norm(x, g, b):
                x = x - x.mean(1, keepdim=True)
                return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5) * get(g)[of] + get(b)[of]

            def lin(x, W, b):
                return torch.cat([x[r] @ get(W)[i] for i, r in enumerate(rows)]) + get(b)[of]

            def drop(x, seed):
                kept = torch.from_numpy(dropout_bits(x.shape[0], x.shape[1], seed, int(self.step))).cuda() >= round(65536 * p)
                return x * kept / (1 - round(65536 * p) / 65536)
            qkv = lin(norm(X, "g1", "b1"), "Wqkv", "bqkv").view(len(X), -1, self.D)
            heads = []
            for h in range(self.heads):
                j = self.heads + h // (self.heads // self.kv)
                part = []
                for a, b in parts_of(sequences):
                    S = qkv[a:b, h] @ qkv[a:b, j].t() / math.sqrt(self.D)
                    S = S.masked_fill(torch.ones_like(S, dtype=torch.bool).triu(1), -math.inf)
                    part.append(torch.softmax(S, 1) @ qkv[a:b, j + self.kv])
                heads.append(torch.cat(part))
            X1 = X + drop(lin(torch.cat(heads, 1), "Wo", "bo"), 1)
            Z = lin(norm(X1, "g2", "b2"), "W1", "c1")
            return X1 + drop(lin(act_of(Z, "gelu")[0], "W2", "c2"), 2)
        return f


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_a_blocks_training_pass_together(dtype):
    block = Block(dtype=dtype)
    workers, sequences = [37, 0, 50, 13], [20, 17, 31, 19, 13]
    T = sum(workers)
    g = gen(20)
    X, dY = normal(g, (T, block.d), dtype), normal(g, (T, block.d), dtype)
    G = torch.full((len(workers), block.P), 9.0, device="cuda")
    Y, dX = block.run(X, offsets_of(workers), offsets_of(sequences), dY, G)
    # the same with every worker's own copy of the parameters, on the CPU's side of autograd
    w = block.w.double().clone()
    for name, (a, s) in block.at.items():
        if len(s) > 1:
            w[a:a + int(np.prod(s))] = block.view(block.low, name).double().view(-1)
    params = w.expand(len(workers), -1).clone().requires_grad_(True)
    x = X.double().requires_grad_(True)
    y = block.plain(x, workers, sequences)(params)
    (y * dY.double()).sum().backward()
    # some 25 arrays between input and output are rounded to 16 bits, each by at most half a step of values that the
    # block neither grows nor shrinks by more than a few: in the 2-norm, 60 half steps at most
    for got, ref, name in ((Y, y.detach(), "Y"), (dX, x.grad, "dX"), (G, params.grad, "G")):
        far = float((got.double() - ref).norm() / ref.norm())
        assert far < 60 * half_step(dtype), (name, far)
    assert bool((G[1] == 0).all())
    # what the server does with them: the mean of the fastest, and AdamW
    ctx = pb.Context(pb.make_config("softmax", len(workers), 1, block.P // 2, 2))
    ticks = torch.tensor([3, 1, 9, 2], dtype=torch.int64, device="cuda")
    grad, mask = torch.empty(block.P, device="cuda"), torch.empty(len(workers), dtype=torch.uint8, device="cuda")
    ctx.aggregate_fastest(G, ticks, 3, g=grad, mask=mask)
    ctx.sync()
    assert mask.tolist() == [1, 1, 0, 1]
    close(grad, G[[0, 1, 3]].double().mean(0), 8 * u * G.double().abs().sum(0) + 1e-300, "g")
    tensors = [[block.view(x, name) for name in block.at] for x in (block.w, grad, block.low)]
    opt = pb.AdamW(tensors[0], tensors[1], **pb.adamw_states(tensors[0]), low=tensors[2])
    before = block.w.clone()
    opt.step(lr=1e-3, max_norm=1.0)
    torch.cuda.synchronize()
    assert torch.equal(block.low, block.w.to(dtype)) and bool(torch.isfinite(block.w).all())
    assert bool((block.w != before)[grad != 0].any())


def test_a_blocks_training_pass_captured():
    # a padded batch: the captured arrays hold T rows, the offsets say how many are there
    block, T = Block(seed=1), 160
    g = gen(21)
    X, dY = normal(g, (T, block.d), BF16), normal(g, (T, block.d), BF16)
    workers, sequences = offsets_of([0, 0, 0]), offsets_of([0, 0, 0, 0])
    G = torch.zeros((3, block.P), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        block.run(X, workers, sequences, dY, G)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y, dX = block.run(X, workers, sequences, dY, G)
        block.step += 1
    for i, (a, b) in enumerate((([50, 10, 100], [60, 50, 0, 50]), ([1, 0, 0], [1, 0, 0, 0]), ([0, 90, 3], [1, 2, 80, 10]),
                                ([40, 40, 40], [30, 30, 30, 30]))):
        rows = sum(a)
        workers.copy_(offsets_of(a)), sequences.copy_(offsets_of(b))
        X.copy_(normal(g, X.shape, BF16))
        G.fill_(5.0)
        block.step.fill_(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert int(block.step) == i + 1
        block.step.fill_(i)
        G2 = torch.zeros_like(G)
        Y2, dX2 = block.run(X, workers, sequences, dY, G2)
        torch.cuda.synchronize()
        assert torch.equal(Y[:rows], Y2[:rows]) and torch.equal(dX[:rows], dX2[:rows]) and torch.equal(G, G2)


def test_calls_on_another_stream_give_the_same_bits():
    g = gen(22)
    T, d = 500, 256
    X, dY, W = normal(g, (T, d), BF16), normal(g, (T, d), BF16), normal(g, (d, d), BF16, 0.06)
    gamma, off = 1 + normal(g, (d,), F32, 0.2), offsets_of([200, 0, 300])
    Q = X.view(T, 4, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def all(**kw):
        O, lse = pb.attention(Q, Q, Q, off, **kw)                                                         # noqa: E741
        return [pb.layer_norm(X, gamma, None, off, **kw), *pb.layer_norm_grad(dY, X, gamma, off, **kw),
                *pb.group_linear(X, W, off, bias=gamma, activation="silu", residual=dY, pre=True, **kw),
                *pb.group_linear_grad(dY, off, pre=X, activation="relu", **kw), pb.dropout(X, 0.2, 5, off, residual=dY, **kw),
                O, lse, *pb.attention_grad(dY.view(T, 4, 64), Q, Q, Q, O, lse, off, **kw)]
    one = all()
    two = all(stream=s)
    torch.cuda.synchronize()
    assert len(one) == len(two) == 14
    for a, b in zip(one, two):
        assert torch.equal(a, b)


def test_calls_without_rows():
    off, w = offsets_of([0, 0]), torch.ones(64, device="cuda")
    X, Q = torch.empty((0, 64), dtype=BF16, device="cuda"), torch.empty((0, 4, 16), dtype=BF16, device="cuda")
    assert pb.layer_norm(X, w, w, off).shape == (0, 64)
    dX, dg, db = pb.layer_norm_grad(X, X, w, off, dgamma=torch.full((2, 64), 3.0, device="cuda"))
    assert dX.shape == (0, 64) and bool((dg == 0).all()) and bool((db == 0).all())
    Y, Z = pb.group_linear(X, torch.zeros((64, 8), dtype=BF16, device="cuda"), off, activation="gelu", pre=True)
    assert Y.shape == Z.shape == (0, 8)
    dZ, db = pb.group_linear_grad(X, off, pre=X, activation="gelu")
    assert dZ.shape == (0, 64) and bool((db == 0).all())
    assert pb.dropout(X, 0.5, 1, off).shape == (0, 64)
    O, lse = pb.attention(Q, Q, Q, off)                                                                    # noqa: E741
    assert O.shape == Q.shape and [x.shape for x in pb.attention_grad(Q, Q, Q, Q, O, lse, off)] == [Q.shape] * 3
    torch.cuda.synchronize()


def test_offsets_that_break_the_rules_stay_inside():
    # results are unspecified; nothing outside the arrays is touched
    g = gen(23)
    T, d, n = 90, 64, 4
    for bad in ([0, 50, 20, 70, 60], [-9, 200, -5, 300, 90], [90, 0, 90, 0, 90], [1 << 30, -(1 << 30), 5, 2, 1]):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        view = {}
        for name, shape in (("x", (T, d)), ("y", (T, d)), ("z", (T, d)), ("G", (n, d)), ("H", (n, d))):
            view[name] = inside(shape, F32 if name in "GH" else BF16, 8, 3.5)
        x, y, z, G, H = (view[k][1] for k in "xyzGH")
        x.copy_(normal(g, x.shape, BF16))
        gamma = torch.ones(d, device="cuda")
        pb.layer_norm(x, gamma, gamma, off, out=y)
        pb.layer_norm_grad(x, x, gamma, off, dX=y, dgamma=G, dbeta=H)
        pb.group_linear(x, normal(g, (n, d, d), BF16), off, bias=G.clone(), activation="gelu", pre=z, out=y)
        pb.group_linear_grad(x, off, pre=x, activation="gelu", dZ=y, dbias=G)
        pb.dropout(x, 0.5, 1, off, out=y)
        heads = lambda t: t.unflatten(1, (2, 32))                                                        # noqa: E731
        O, lse = pb.attention(heads(x), heads(x), heads(x), off, out=heads(y))                            # noqa: E741
        pb.attention_grad(heads(x), heads(x), heads(x), heads(x), O, lse, off, dQ=heads(z))
        torch.cuda.synchronize()
        for name, (big, v) in view.items():
            v.fill_(3.5)
            assert bool((big == 3.5).all()), (bad, name)
