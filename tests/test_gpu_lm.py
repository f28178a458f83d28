"""The operators for language models on the GPU, against plain 64-bit forms.

Tolerances are derived, not tuned.  u = 2^-24 is the largest relative error of
a rounding to fp32; rounding to a 16-bit type is off by half a step, eps / 2
of the value (and by half the smallest subnormal below the normal range).

A product sums K exact terms in fp32, in any order: its error is at most
2 K u sum |a b| (2: the matrix cores may truncate instead of round).

The loss of a row is log(sum) + (max - z_y).  An exponential's argument z - max
is rounded once and multiplied by log2(e) (itself rounded) in a second
rounding: 3 u |z - max| absolute, so that relative to exp; exp2 adds 2 u; the
sum of C of them, per thread and then over a tree, adds at most (64 + 16) u
(no thread sums more than 64 terms where rows are held in registers; the
streaming rows add C / 1024).  With R the spread of the logits, a probability
is off by (2 * (3 R + 2) + 80 + C / 1024) u relative.  (Where z - max is below
-104 the exponential is below 2^-149: it is 0 or the smallest value on both
sides, so R counts up to 104.)
"""
import math

import numpy as np
import pytest

from gpu_util import host

pb = pytest.importorskip("paper_2004_14696_amd.binding")
torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rounded(y, dtype):
    """The error of rounding y to dtype, at most."""
    return half_step(dtype) * y.abs() + TINY[dtype] / 2


def offsets_of(lengths, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lengths)]), dtype=torch.int32, device="cuda")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def ragged(seed, n, T):
    cuts = np.sort(np.random.default_rng(seed).integers(0, T + 1, n - 1))
    return np.diff(np.concatenate([[0], cuts, [T]])).astype(int).tolist()


# -- products -------------------------------------------------------------------
def product_ref(form, a, b, lengths, first, out):
    """64-bit result and the sum of |terms|, over the rows of the groups; rows
    of no group keep those of `out`."""
    a, b = a.double(), b.double()
    y, s = out.double(), torch.zeros_like(out, dtype=torch.float64)
    at = first
    for i, r in enumerate(lengths):
        rows = slice(at, at + r)
        at += r
        if form == "weight":
            x, z = a[rows].t().contiguous(), b[rows]
            y[i], s[i] = x @ z, x.abs() @ z.abs()
        elif r:
            W = b if b.dim() == 2 else b[i]
            W = W if form == "forward" else W.t().contiguous()
            y[rows], s[rows] = a[rows] @ W, a[rows].abs() @ W.abs()
    return y, s


def check_product(form, a, b, lengths, first=0, out_dtype=None, out=None, **kw):
    call = {"forward": pb.group_matmul, "input": pb.group_input_grad, "weight": pb.group_weight_grad}[form]
    off = offsets_of(lengths, first)
    n = len(lengths)
    d, C = (a.shape[1], b.shape[1]) if form == "weight" else b.shape[-2:]
    shape = (n, d, C) if form == "weight" else (a.shape[0], C if form == "forward" else d)
    dtype = out_dtype or (torch.float32 if form == "weight" else a.dtype)
    if out is None:
        out = torch.full(shape, 7.25, dtype=dtype, device="cuda")
    ref, size = product_ref(form, a, b, lengths, first, out)
    got = call(a, b, off, out=out, **kw)
    torch.cuda.synchronize()
    assert got is out
    K = max(lengths) if form == "weight" else (d if form == "forward" else C)
    tol = 2 * K * u * size + rounded(ref, dtype)
    bad = (got.double() - ref).abs() > tol
    assert not bool(bad.any()), (form, a.shape, b.shape, lengths, int(bad.sum()),
                                 float(((got.double() - ref).abs() - tol).max()))
    return got


SIZES = [
    # d, C, lengths: one token, empty groups, odd widths, tiles that end inside
    (64, 64, [1]), (8, 8, [1, 0, 2]), (64, 128, [3, 0, 0, 5]), (40, 72, [33, 31, 1]),
    (1, 1, [5, 2]), (7, 3, [1, 9]), (65, 129, [130, 1, 63]), (130, 255, [64, 65]),
    (9, 15, [70, 3]), (136, 201, [129, 1]), (71, 66, [300]), (8, 9, [1, 2]), (77, 8, [64, 65]), (2, 260, [40]),
    (264, 520, [300, 17]), (512, 256, [700, 100, 513]), (200, 1000, [0, 0, 0]), (96, 40, [2000]),
]


@pytest.mark.parametrize("form", ["forward", "input", "weight"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,C,lengths", SIZES)
def test_products_of_ragged_groups(form, dtype, d, C, lengths):
    g = gen(d * 1000 + C)
    n, T = len(lengths), sum(lengths)
    X, dY = normal(g, (T, d), dtype), normal(g, (T, C), dtype)
    W = normal(g, (n, d, C), dtype)
    a, b = {"forward": (X, W), "input": (dY, W), "weight": (X, dY)}[form]
    for out_dtype in (dtype, torch.float32):
        check_product(form, a, b, lengths, out_dtype=out_dtype)


@pytest.mark.parametrize("form", ["forward", "input"])
@pytest.mark.parametrize("T,d,C", [(1, 64, 64), (37, 2048, 1408), (700, 96, 4104), (5, 4096, 33), (1100, 1032, 2056)])
def test_products_of_groups_that_share_their_weights(form, T, d, C):
    g = gen(T + d)
    W = normal(g, (d, C), torch.bfloat16)
    a = normal(g, (T, d if form == "forward" else C), torch.bfloat16)
    one = check_product(form, a, W, [T])
    # how the rows are grouped does not matter, nor whether W is repeated by a stride of 0
    lengths = ragged(T, 5, T)
    assert torch.equal(one, check_product(form, a, W, lengths))
    assert torch.equal(one, check_product(form, a, W.expand(5, d, C), lengths))


@pytest.mark.parametrize("form", ["forward", "input", "weight"])
@pytest.mark.parametrize("T,n,d,C", [(6000, 3, 1000, 2047), (37, 16, 2048, 1408), (9000, 2, 136, 264), (4096, 24, 512, 1024),
                                     (3000, 1, 2500, 2304), (40, 1000, 64, 128)])
def test_products_of_larger_and_split_sizes(form, T, n, d, C):
    g = gen(T + n)
    lengths = ragged(T + n, n, T)
    X, dY = normal(g, (T, d), torch.bfloat16), normal(g, (T, C), torch.bfloat16, 0.1)
    W = normal(g, (n, d, C), torch.bfloat16) if form != "weight" else None
    a, b = {"forward": (X, W), "input": (dY, W), "weight": (X, dY)}[form]
    check_product(form, a, b, lengths)


@pytest.mark.parametrize("form", ["forward", "input", "weight"])
@pytest.mark.parametrize("wide", [True, False])
def test_products_of_strided_arrays_leave_the_rest_alone(form, wide):
    # rows, groups and columns inside larger arrays, at any offset; NaN and
    # infinities around and in rows of no group reach nothing
    g = gen(3)
    step = 8 if wide else 1
    d, C, lengths, first, after = 72, 136, [30, 0, 77, 5], 9, 11
    n, T = len(lengths), first + sum(lengths) + after

    def inside(shape, dtype, fill=float("nan")):
        big = torch.full([s + 2 * step for s in shape], fill, dtype=dtype, device="cuda")
        view = big[tuple(slice(step, step + s) for s in shape)]
        return big, view
    view = {}
    for name, shape in (("X", (T, d)), ("dY", (T, C)), ("W", (n, d, C))):
        _, v = inside(shape, torch.float16)
        v.copy_(normal(g, shape, torch.float16))
        if name != "W":
            v[:first] = float("inf")
            v[first + sum(lengths):] = float("nan")
        view[name] = v
    a, b = {"forward": (view["X"], view["W"]), "input": (view["dY"], view["W"]), "weight": (view["X"], view["dY"])}[form]
    shape = (n, d, C) if form == "weight" else (T, C if form == "forward" else d)
    for dtype in (torch.float16, torch.float32):
        big, out = inside(shape, dtype, 3.5)
        check = out.clone()
        check_product(form, a, b, lengths, first=first, out_dtype=dtype, out=out)
        if form != "weight":
            assert torch.equal(out[:first], check[:first]) and torch.equal(out[-after:], check[-after:])
        out.fill_(3.5)
        assert bool((big == 3.5).all())      # nothing written around


@pytest.mark.parametrize("form", ["forward", "input", "weight"])
def test_a_groups_nan_reaches_no_other_group(form):
    g = gen(4)
    d, C, lengths = 100, 60, [10, 40, 1, 90]
    T, n = sum(lengths), len(lengths)
    X, dY, W = normal(g, (T, d), torch.bfloat16), normal(g, (T, C), torch.bfloat16), normal(g, (n, d, C), torch.bfloat16)
    a, b = {"forward": (X, W), "input": (dY, W), "weight": (X, dY)}[form]
    a[10:50] = float("nan")
    a[50] = float("inf")
    call = {"forward": pb.group_matmul, "input": pb.group_input_grad, "weight": pb.group_weight_grad}[form]
    got = call(a, b, offsets_of(lengths))
    keep = torch.ones(n, dtype=torch.bool) if form == "weight" else torch.ones(T, dtype=torch.bool)
    keep[slice(1, 3) if form == "weight" else slice(10, 51)] = False
    keep = keep.cuda()
    assert bool(torch.isfinite(got[keep]).all()) and not bool(torch.isfinite(got[~keep]).any())


def test_gradients_of_a_product_against_differences():
    # f(X, W) = sum(R * Y): its gradients are dX = R W^T and G = X^T R, and Y is
    # linear in each, so a difference along any direction is exact up to rounding
    g = gen(5)
    d, C, lengths = 48, 80, [20, 0, 13]
    T, n = sum(lengths), len(lengths)
    off = offsets_of(lengths)
    X, W, R = (normal(g, s, torch.bfloat16) for s in ((T, d), (n, d, C), (T, C)))
    DX, DW = normal(g, (T, d), torch.bfloat16), normal(g, (n, d, C), torch.bfloat16)
    f32 = torch.float32
    dX, G = pb.group_input_grad(R, W, off, out_dtype=f32), pb.group_weight_grad(X, R, off)
    for D, grad, other in ((DX, dX, lambda: pb.group_matmul(DX, W, off, out_dtype=f32)),
                           (DW, G, lambda: pb.group_matmul(X, DW, off, out_dtype=f32))):
        change = float((R.double() * other().double()).sum())
        slope = float((grad.double() * D.double()).sum())
        # each is a sum of T d C products in fp32 sums of at most C terms
        size = T * d * C
        assert abs(change - slope) <= 2 * 80 * u * 8 * size, (change, slope)


def test_products_beyond_two_to_the_31_elements():
    T, d, C = (1 << 21) + 3, 1032, 8      # X: 2.2e9 values
    X = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    dY = torch.zeros((T, C), dtype=torch.bfloat16, device="cuda")
    X[-70:] = normal(gen(6), (70, d), torch.bfloat16)
    dY[-70:] = normal(gen(7), (70, C), torch.bfloat16)
    lengths = [T - 50, 50]
    W = normal(gen(8), (2, d, C), torch.bfloat16)
    Y = pb.group_matmul(X, W, offsets_of(lengths))
    dX = pb.group_input_grad(dY, W, offsets_of(lengths))
    G = pb.group_weight_grad(X, dY, offsets_of(lengths))
    for form, a, b, got in (("forward", X[-70:], W, Y[-70:]), ("input", dY[-70:], W, dX[-70:]),
                            ("weight", X[-70:], dY[-70:], G)):
        ref, size = product_ref(form, a, b, [20, 50], 0, torch.zeros_like(got))
        K = {"forward": d, "input": C, "weight": T}[form]
        assert bool(((got.double() - ref).abs() <= 2 * K * u * size + rounded(ref, got.dtype)).all()), form
    assert not bool(Y[:-70].any()) and not bool(dX[:-70].any())


def test_rows_around_two_to_the_31_elements_reach_their_sums():
    # rows at the start, around the 2^31st element of X (and of dX) and at the
    # end; all others are 0, and add no rounding: K is what is left of them and
    # the parts of a sum, at most 64
    T, d, C = (1 << 21) + 3, 1032, 8
    edge = (1 << 31) // d
    rows = torch.cat([torch.arange(40), torch.arange(edge - 30, edge + 30), torch.arange(T - 50, T)]).cuda()
    X = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    dY = torch.zeros((T, C), dtype=torch.bfloat16, device="cuda")
    X[rows], dY[rows] = normal(gen(60), (150, d), torch.bfloat16), normal(gen(61), (150, C), torch.bfloat16)
    W = normal(gen(62), (2, d, C), torch.bfloat16)
    lengths, some = [edge + 7, T - edge - 7], [77, 73]     # of the rows that are not 0
    off = offsets_of(lengths)
    for form, a, b, got, K in (("forward", X[rows], W, pb.group_matmul(X, W, off), d),
                               ("input", dY[rows], W, pb.group_input_grad(dY, W, off), C),
                               ("weight", X[rows], dY[rows], pb.group_weight_grad(X, dY, off), 77 + 64)):
        mine = got if form == "weight" else got[rows]
        ref, size = product_ref(form, a, b, some, 0, torch.zeros_like(mine))
        assert bool(((mine.double() - ref).abs() <= 2 * K * u * size + rounded(ref, got.dtype)).all()), form
        if form != "weight":
            got[rows] = 0
            assert not bool(got.any()), form


def test_weights_beyond_two_to_the_31_elements():
    # W and G of 2.25e9 values: the first groups, those around the 2^31st element
    # (2^32 bytes of W, and of G half way), the last
    n, d, C = 1000, 1504, 1496
    edge = (1 << 31) // (d * C)
    groups = [0, 1, edge // 2 - 1, edge // 2, edge // 2 + 1, edge - 1, edge, edge + 1, n - 2, n - 1]
    lengths = [2 + i % 2 for i in range(n)]
    off = offsets_of(lengths)
    T = sum(lengths)
    X, dY = normal(gen(63), (T, d), torch.bfloat16), normal(gen(64), (T, C), torch.bfloat16)
    W = torch.empty((n, d, C), dtype=torch.bfloat16, device="cuda").normal_(generator=gen(65))
    got = {"forward": pb.group_matmul(X, W, off), "input": pb.group_input_grad(dY, W, off),
           "weight": pb.group_weight_grad(X, dY, off)}
    for i in groups:
        rows = slice(int(off[i]), int(off[i + 1]))
        for form, a, b, K in (("forward", X, W[i], d), ("input", dY, W[i], C), ("weight", X, dY, 3)):
            mine = got[form][i:i + 1] if form == "weight" else got[form][rows]
            ref, size = product_ref(form, a[rows], b[rows] if form == "weight" else b, [lengths[i]], 0, torch.zeros_like(mine))
            assert bool(((mine.double() - ref).abs() <= 2 * K * u * size + rounded(ref, mine.dtype)).all()), (form, i)


# -- token loss -------------------------------------------------------------------
def loss_ref(Z, y, lengths, first, scale):
    Z = Z.double()
    losses, dZ = [], torch.zeros_like(Z)
    spread = gap = 0.0
    at = first
    for i, r in enumerate(lengths):
        rows = torch.arange(at, at + r, device="cuda")
        at += r
        live = rows[y[rows] >= 0]
        if len(live) == 0:
            losses.append(0.0)
            continue
        z, t = Z[live], y[live].long()
        logp = torch.log_softmax(z, 1)
        losses.append(float(-logp.gather(1, t.view(-1, 1)).mean()))
        p = logp.exp()
        p.scatter_add_(1, t.view(-1, 1), -torch.ones(len(live), 1, dtype=torch.float64, device="cuda"))
        dZ[live] = p * (scale / len(live))
        top = z.amax(1, keepdim=True)
        spread = max(spread, float((top - z).clamp(max=104.0).max()))
        gap = max(gap, float((top - z.gather(1, t.view(-1, 1))).max()))
    return torch.tensor(losses, dtype=torch.float64, device="cuda"), dZ, (spread, gap)


def check_loss(Z, y, lengths, first=0, scale=1.0, in_place=False, dZ=None):
    ref_loss, ref, (spread, gap) = loss_ref(Z, y, lengths, first, scale)
    C, dtype = Z.shape[1], Z.dtype
    before = Z.clone()
    loss, got = pb.token_loss(Z, y, offsets_of(lengths, first), scale=scale, dZ=Z if in_place else dZ)
    torch.cuda.synchronize()
    rel = (2 * (3 * spread + 2) + 80 + C / 1024) * u
    # log(sum) is off by rel and by its own roundings, then max - z_y is added
    assert bool(((loss.double() - ref_loss).abs() <= rel + 4 * u * (gap + math.log(C) + 1)).all()), (loss, ref_loss)
    at = first
    for i, r in enumerate(lengths):
        rows = slice(at, at + r)
        at += r
        count = max(1, int((y[rows] >= 0).sum()))
        # p and 1 are scaled and subtracted in fp32: 4 roundings of either
        size = ref[rows].abs() + 2 * abs(scale) / count * (torch.nn.functional.one_hot(
            y[rows].long().clamp(min=0), C).double())
        tol = (rel + 4 * u) * size + rounded(ref[rows], dtype) + rounded(ref[rows], torch.float32)
        diff = (got[rows].double() - ref[rows]).abs()
        assert bool((diff <= tol).all()), (Z.shape, dtype, i, float((diff - tol).max()))
    # rows of no group: as they were
    if in_place:
        for rows in (slice(0, first), slice(at, None)):
            assert torch.equal(got[rows].view(torch.uint8), before[rows].view(torch.uint8))
    return loss, got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("C", [1, 2, 7, 64, 1000, 2049, 4097, 5000, 16385, 32771, 65537, 140001])
def test_token_loss_over_class_counts(dtype, C):
    g = gen(C)
    lengths = [3, 0, 1, 6]
    T = 2 + sum(lengths) + 3
    Z = normal(g, (T, C), dtype, 3.0)
    y = torch.randint(0, C, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[2 + 1] = -1
    y[2 + 3] = -5            # the only row of worker 2: nothing left of it
    for scale in (1.0, -3.0) if dtype != torch.float16 else (1024.0,):
        loss, dZ = check_loss(Z, y, lengths, first=2, scale=scale)
        assert float(loss[1]) == 0.0 and float(loss[2]) == 0.0
        assert not bool(dZ[3].any()) and not bool(dZ[5].any())
    only, none = pb.token_loss(Z, y, offsets_of(lengths, 2), grad=False)
    assert none is None and torch.equal(only, loss)
    check_loss(Z, y, lengths, first=2, in_place=True)


def test_token_loss_strides_many_workers_and_one_token():
    g = gen(9)
    for n, T, C in ((1, 1, 50), (1000, 3000, 33), (64, 40, 257), (3, 700, 1000)):
        big = normal(g, (T, C + 5), torch.bfloat16, 2.0)
        out = torch.full((T, C + 9), 2.5, dtype=torch.bfloat16, device="cuda")
        y = torch.randint(-1, C, (T,), generator=g, device="cuda", dtype=torch.int32)
        check_loss(big[:, 3:C + 3], y, ragged(n, n, T), dZ=out[:, 1:C + 1])
        assert bool((out[:, 0] == 2.5).all()) and bool((out[:, C + 1:] == 2.5).all())
    loss, dZ = pb.token_loss(big[:0, :C], y[:0], offsets_of([0, 0]))
    assert host(loss).tolist() == [0.0, 0.0] and dZ.shape == (0, C)


def test_token_loss_of_more_rows_than_one_launch_starts():
    # 2^20 + 5 rows, and workers that have nearly all of them or none
    g = gen(10)
    T, C = (1 << 20) + 5, 9
    Z = normal(g, (T, C), torch.bfloat16, 2.0)
    y = torch.randint(-1, C, (T,), generator=g, device="cuda", dtype=torch.int32)
    check_loss(Z, y, [3, T - 7, 0, 4])
    check_loss(Z[:70001].float(), y[:70001], [0] * 500 + [70001] + [0] * 400)


@pytest.mark.parametrize("C", [9, 3000, 20000, 150000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_token_loss_of_masked_and_broken_logits(C, dtype):
    g = gen(C + 1)
    T = 10
    Z = normal(g, (T, C), dtype, 2.0)
    y = torch.randint(1, C, (T,), generator=g, device="cuda", dtype=torch.int32)
    low = torch.finfo(dtype).min
    Z[0, C // 2:] = -math.inf          # a grammar's mask
    y[0] = C // 3 if C // 3 else 1
    Z[1, 1:] = low                     # masked with the type's lowest value
    y[1] = 0
    Z[2] = -math.inf
    Z[2, 4] = 1.0                      # one class left
    y[2] = 4
    Z[3] = low                         # all classes equal
    Z[4] = torch.finfo(dtype).max      # equal and large
    y[5] = -1
    Z[5, 3] = math.nan                 # masked rows are not read
    check_loss(Z[:6].clone(), y[:6], [1] * 6)
    # what has no answer is a NaN, and stays in its row and worker
    Z[6, 2] = math.nan
    Z[7, 5] = math.inf
    Z[8] = -math.inf
    y[9] = C
    loss, dZ = pb.token_loss(Z, y, offsets_of([1] * 10))
    assert bool(torch.isnan(loss[6:]).all()) and bool(torch.isfinite(loss[:6]).all())
    assert bool(torch.isnan(dZ[6:]).all()) and bool(torch.isfinite(dZ[:6]).all())
    # the label's class masked: an infinite loss, as the formula says
    Z2 = normal(g, (1, C), dtype)
    Z2[0, 0] = -math.inf
    loss, dZ = pb.token_loss(Z2, torch.zeros(1, dtype=torch.int32, device="cuda"), offsets_of([1]))
    assert float(loss[0]) == math.inf and bool(torch.isfinite(dZ).all())


@pytest.mark.parametrize("C", [9, 3000, 20000, 150000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_token_loss_of_logits_of_any_magnitude(C, dtype):
    # the largest power of a row is 1 whatever its logit: rows of equal logits
    # (one masked as a whole with a large negative value among them), at every
    # power of two
    g = gen(C + 2)
    v = torch.tensor([s * 1.3 * 2.0 ** k for k in range(20, 128) for s in (1, -1)] + [3e9, 1e10, -1e10, -1e20, 1e30, -1e30],
                     dtype=torch.float64, device="cuda").to(dtype)
    T = len(v)
    y = torch.randint(0, C, (T,), generator=g, device="cuda", dtype=torch.int32)
    check_loss(v.view(-1, 1).repeat(1, C), y, [1] * T)
    # the type's next values below among them
    Z = v.view(-1, 1).repeat(1, C)
    down = torch.nextafter(v, torch.full_like(v, -math.inf))
    Z[:, 1::3] = down.view(-1, 1)
    Z[:, 2::3] = torch.nextafter(down, torch.full_like(v, -math.inf)).view(-1, 1)
    check_loss(Z, torch.zeros(T, dtype=torch.int32, device="cuda"), [1] * T)
    # one logit of that size among ordinary ones, or behind and before smaller
    # ones of a neighbouring power of two: at the label and elsewhere
    for k in (20, 29, 30, 31, 32, 40, 66, 100, 124, 125, 126, 127):
        top = 1.3 * 2.0 ** k
        Z = normal(g, (6, C), dtype, 2.0)
        Z[:2, C // 2] = top
        Z[2:4] = -top
        Z[2:4, C // 2] = 1.0
        # every thread's maximum grows on its way through the row
        Z[4:] = top / 2.0
        Z[4:, C // 2:] = top
        y = torch.tensor([C // 2, 1] * 2 + [C - 1, 0], dtype=torch.int32, device="cuda")
        for rows in (0, 1, 2, 3, 4, 5):
            check_loss(Z[rows:rows + 1].clone(), y[rows:rows + 1], [1])
    for first, then in ((0.95, 1.05), (0.5, 1.9), (1.05, 0.95)):
        for k in (30, 126):
            Z = torch.full((1, C), first * 2.0 ** k, dtype=dtype, device="cuda")
            Z[:, C // 2:] = then * 2.0 ** k
            check_loss(Z, torch.tensor([C - 1 if then > first else 0], dtype=torch.int32, device="cuda"), [1])


def test_token_loss_without_a_gradient_writes_none():
    g = gen(13)
    Z = normal(g, (5, 300), torch.bfloat16)
    y = torch.tensor([1, 0, -1, 299, 7], dtype=torch.int32, device="cuda")
    off = offsets_of([2, 3])
    want, _ = pb.token_loss(Z, y, off)
    before, buffer = Z.clone(), torch.full_like(Z, 2.0)
    for dZ in (None, buffer, Z):
        loss, none = pb.token_loss(Z, y, off, dZ=dZ, grad=False)
        assert none is None and torch.equal(loss, want) and torch.equal(Z, before)
    assert bool((buffer == 2.0).all())


def test_token_loss_gradient_against_differences():
    g = gen(11)
    T, C, lengths = 12, 40, [5, 7]
    Z = normal(g, (T, C), torch.float32)
    y = torch.randint(-1, C, (T,), generator=g, device="cuda", dtype=torch.int32)
    _, dZ = pb.token_loss(Z, y, offsets_of(lengths))
    D = normal(g, (T, C), torch.float32)
    h = 2.0 ** -6
    up, down = (pb.token_loss(Z + s * h * D, y, offsets_of(lengths), grad=False)[0].double() for s in (1, -1))
    slope = (dZ.double() * D.double())
    slope = torch.stack([slope[:5].sum(), slope[5:].sum()])
    # central difference: h^2 / 6 of the third derivative (at most max|D|^3 for
    # a log-sum-exp), and the losses' roundings over 2 h
    m = float(D.abs().max())
    assert bool((((up - down) / (2 * h) - slope).abs() <= h * h * m ** 3 + 2 * 200 * u / (2 * h)).all())


def test_token_loss_beyond_two_to_the_31_elements():
    T, C = 43000, 50001                # 2.15e9 values
    Z = torch.zeros((T, C), dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(T, dtype=torch.int32, device="cuda")
    Z[-1] = normal(gen(12), (C,), torch.bfloat16)
    y[-1] = C - 1
    ref_loss, ref, _ = loss_ref(Z[-1:], y[-1:], [1], 0, 1.0)
    loss, dZ = pb.token_loss(Z, y, offsets_of([T - 1, 1]), dZ=Z)
    assert abs(float(loss[0]) - math.log(C)) < 1e-5 and abs(float(loss[1] - ref_loss[0])) < 1e-5
    assert bool(((dZ[-1:].double() - ref).abs() <= 200 * u + rounded(ref, torch.bfloat16)).all())
    assert torch.equal(dZ[0], dZ[T - 2])


# -- AdamW ------------------------------------------------------------------------
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8)


def mix(x):
    x = (x ^ (x >> np.uint64(16))) * np.uint64(0x9E3779B1) & np.uint64(0xFFFFFFFF)
    x = (x ^ (x >> np.uint64(15))) * np.uint64(0xB7E15163) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def bits_of(seed, t, tensor, count):
    M = np.uint64(0xFFFFFFFF)
    key = mix(mix(mix(np.uint64(seed)) + np.uint64(t) & M) + np.uint64(tensor) & M)
    i = np.arange(count, dtype=np.uint64)
    return mix((i * np.uint64(0x6A09E667) + key) & M)


def encode_ref(x, bits, least):
    """e4m3 values, scales and code steps of x (64 bits), by the definition."""
    n = len(x)
    blocks = -(-n // 256)
    pad = np.zeros(blocks * 256)
    pad[:n] = x
    b = np.zeros(blocks * 256)
    b[:n] = bits
    pad, b = pad.reshape(blocks, 256), b.reshape(blocks, 256)
    top = np.maximum(np.abs(pad).max(1), 2.0 ** -118)
    scale = 2.0 ** np.ceil(np.log2(top / 448.0))
    y = np.abs(pad) / scale[:, None]
    step = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3)
    q = np.floor(y / step + b / 65536.0)
    if least:
        q = np.where((q == 0) & (pad > 0), 1.0, q)
    value = np.copysign(q * step, pad) * scale[:, None]
    return value.reshape(-1)[:n], scale, (step * scale[:, None]).reshape(-1)[:n]


def values(codes, scale):
    c = host(codes.float()).reshape(-1).astype(np.float64)
    return c * np.repeat(host(scale.float()).astype(np.float64), 256)[:len(c)]


def make(sizes, bits, g_dtype, low, seed, shift=0, decay=0.1, scale=1.0):
    """Tensors at `shift` elements from the start of their allocation."""
    g = gen(seed)

    def at(n, dtype, s):
        return normal(g, (n + shift,), dtype, s)[shift:]
    w = [at(n, torch.float32, 1.0) for n in sizes]
    grads = [at(n, g_dtype, 0.1) for n in sizes]
    st = pb.adamw_states(w, bits)
    if shift:
        st["m"], st["v"] = ([torch.zeros(n + shift, dtype=torch.uint8 if bits == 8 else torch.float32, device="cuda")[shift:]
                             .view(torch.float8_e4m3fn if bits == 8 else torch.float32) for n in sizes] for _ in "mv")
    lows = [at(n, low, 0.0) for n in sizes] if low else None
    opt = pb.AdamW(w, grads, **st, low=lows, weight_decay=decay, lr_scale=scale)
    return opt, w, grads, st, lows


def check_step(opt, w, grads, st, lows, t, seed=77, grad_scale=1.0, max_norm=0.0, decay=0.1, scale=1.0):
    n = len(w)
    decay = decay if isinstance(decay, list) else [decay] * n
    scale = scale if isinstance(scale, list) else [scale] * n
    bits8 = "m_scale" in st
    w0 = [host(x).astype(np.float64) for x in w]
    if bits8:
        m0 = [values(a, b) for a, b in zip(st["m"], st["m_scale"])]
        v0 = [values(a, b) ** 2 for a, b in zip(st["v"], st["v_scale"])]
    else:
        m0, v0 = ([host(x).astype(np.float64) for x in st[k]] for k in "mv")
    G = [host(x.float()).astype(np.float64) for x in grads]
    norm = abs(grad_scale) * math.sqrt(sum(float((x ** 2).sum()) for x in G))
    f = grad_scale * (max_norm / norm if 0 < max_norm < norm else 1.0)
    got_norm = opt.step(**HYPER, seed=seed, grad_scale=grad_scale, max_norm=max_norm)
    torch.cuda.synchronize()
    if max_norm:
        assert abs(float(got_norm) - norm) <= 2 * u * norm
    b1, b2 = HYPER["beta1"], HYPER["beta2"]
    flips = total = 0
    for i in range(n):
        x = G[i] * f
        m, v = b1 * m0[i] + (1 - b1) * x, b2 * v0[i] + (1 - b2) * x * x
        # f, the coefficients, the products and the sum are each rounded
        em = 6 * u * (b1 * np.abs(m0[i]) + (1 - b1) * np.abs(x)) + 2.0 ** -148
        ev = 8 * u * v + 2.0 ** -148
        lr = HYPER["lr"] * scale[i]
        r = np.sqrt(v)
        denom = r / math.sqrt(1 - b2 ** t) + HYPER["eps"]
        step = lr / (1 - b1 ** t) * m / denom
        want = w0[i] * (1 - lr * decay[i]) - step
        # an update's roundings: of m, of the root and quotient and products (16),
        # and of w itself (4)
        ew = lr / (1 - b1 ** t) * em / denom + 16 * u * np.abs(step) + 4 * u * (np.abs(w0[i]) + np.abs(step))
        got = host(w[i]).astype(np.float64)
        assert np.all(np.abs(got - want) <= ew), (i, np.max(np.abs(got - want) - ew))
        if lows:
            assert torch.equal(lows[i], w[i].to(lows[i].dtype)), i
        if not bits8:
            assert np.all(np.abs(host(st["m"][i]) - m) <= em) and np.all(np.abs(host(st["v"][i]) - v) <= ev), i
            continue
        b = bits_of(seed, t, i, len(m))
        for name, val, part, least in (("m", m, b & np.uint64(0xFFFF), False), ("v", r, b >> np.uint64(16), True)):
            ref, sref, code = encode_ref(val, part.astype(np.float64), least)
            s = host(st[name + "_scale"][i].float()).astype(np.float64)
            now = values(st[name][i], st[name + "_scale"][i])
            # a scale may differ where the largest value is 8 u from 448 scales
            assert np.sum(s != sref) <= 1e-3 * len(s) and np.all(np.isin(s / sref, (0.5, 1.0, 2.0))), (i, name)
            # every stored value is one of the two codes at it (of the coarser scale)
            same = np.repeat(s == sref, 256)[:len(val)]
            assert np.all(np.abs(now - val) <= np.where(same, 1.001, 2.001) * code + 16 * u * np.abs(val)), (i, name)
            if least:
                assert np.all((now > 0) == (val > 0)), i
            flips += int((now != ref)[same].sum())
            total += len(val)
    # the fp32 value decides like the 64-bit one unless its place between two
    # codes, off by 8 u of at most 16 steps, crosses the drawn threshold: 16 * 8
    # u = 2^-17 of the values
    assert flips <= 3 + total * 2.0 ** -15, (flips, total)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("g_dtype,low", [(torch.float32, None), (torch.bfloat16, torch.bfloat16),
                                         (torch.float16, torch.float16)])
def test_adamw_steps(bits, g_dtype, low):
    sizes = [1, 2, 3, 4, 5, 255, 256, 257, 1023, 4095, 4096, 4097, 10000, 70001]
    opt, w, g, st, lows = make(sizes, bits, g_dtype, low, 21)
    for t in (1, 2, 3):
        check_step(opt, w, g, st, lows, t, grad_scale=[1.0, 0.25, -2.0][t - 1], max_norm=[0.0, 1.0, 1e9][t - 1])
        for x in g:
            x.copy_(normal(gen(100 + t), x.shape, x.dtype, 0.3))
    assert opt.t == 3
    opt.t = 1000
    check_step(opt, w, g, st, lows, 1001)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [1, 3])
def test_adamw_of_unaligned_tensors_with_their_own_rates(bits, shift):
    sizes = [7, 300, 5000]
    decay, scale = [0.0, 0.1, 0.5], [1.0, 0.1, 0.0]
    opt, w, g, st, lows = make(sizes, bits, torch.float16, torch.bfloat16, 22, shift, decay, scale)
    for t in (1, 2):
        check_step(opt, w, g, st, lows, t, decay=decay, scale=scale)


def exact_codes(x, bits, floor):
    """Codes and scale exponents of fp32 values x [blocks][256], by the
    definition: the sum of a value's place and its random bits is rounded to
    fp32 (in 64 bits it is exact wherever it is near a whole number)."""
    ab = np.abs(x.astype(np.float64))
    finite = np.isfinite(ab)
    top = np.maximum(np.where(finite, ab, 0.0).max(1), 2.0 ** -118)
    mant, exp = np.frexp(top)                       # mant in [1/2, 1)
    e = exp - 1 - 8 + (mant > 0.875)
    y = np.where(finite, ab, 0.0) * 2.0 ** -e.astype(np.float64)[:, None]
    ey = np.frexp(np.maximum(y, 2.0 ** -6))[1] - 1
    q = np.floor((y * 2.0 ** (3.0 - ey) + bits / 65536.0).astype(np.float32)).astype(np.int64)
    if floor:
        q = np.where((q == 0) & (x > 0), 1, q)
    c = np.where(finite, (ey + 6) * 8 + q, 0x7F) | np.where(np.signbit(x), 0x80, 0)
    return c, e + 127


def states_that_are_known_exactly(n):
    """Gradients whose states with both betas 0 are themselves and their
    magnitudes: blocks of ordinary values, of a wide range, with zeros, of
    values whose squares are 0, subnormal or infinite, and not finite."""
    rng = np.random.default_rng(50)
    x = rng.standard_normal((n, 256)).astype(np.float32)
    x[1::16] *= np.exp2(rng.uniform(-40, 0, (len(x[1::16]), 256))).astype(np.float32)
    x[2::16] *= np.float32(2.0) ** rng.integers(-16, 1, (len(x[2::16]), 256)).astype(np.float32)
    x[3::16][rng.random((len(x[3::16]), 256)) < 0.5] = 0.0
    x[4::16] *= np.float32(2.0 ** -70)
    x[5::16] *= np.float32(2.0 ** -45)
    x[6::16, :200] *= np.float32(2.0 ** -52)
    x[7::16, 5] = 2.0 ** 80
    x[8::16, 17], x[8::32, 40] = np.inf, -np.inf
    x[9::16, 3] = np.nan
    x[10::16] = 0.0
    x[11::16] = np.float32(1.75) * np.float32(2.0) ** rng.integers(-6, 7, (len(x[11::16]), 256)).astype(np.float32)
    return x


def test_adamw_8_bit_codes_are_exactly_those_of_their_definition():
    # m = g and v = g^2 rounded, r its rounded root: no tolerance.  Two tensors,
    # the second one's last block cut short
    x = states_that_are_known_exactly(8192)
    cut = 256 * 5000 + 101
    parts = [x[:3000].reshape(-1), x[3000:].reshape(-1)[:cut]]
    w = [torch.zeros(len(p), device="cuda") for p in parts]
    grads = [torch.tensor(p, device="cuda") for p in parts]
    st = pb.adamw_states(w, 8)
    opt = pb.AdamW(w, grads, **st)
    opt.step(lr=1e-3, beta1=0.0, beta2=0.0, seed=91)
    torch.cuda.synchronize()
    for i, p in enumerate(parts):
        full = np.zeros(-(-len(p) // 256) * 256, np.float32)
        full[:len(p)] = p
        full = full.reshape(-1, 256)
        b = bits_of(91, 1, i, full.size).reshape(full.shape)
        with np.errstate(over="ignore", invalid="ignore"):
            r = np.sqrt(full * full)
        m = np.float32(0.0) + full                  # (-0 becomes 0)
        for name, val, bits, floor in (("m", m, b & np.uint64(0xFFFF), False), ("v", r, b >> np.uint64(16), True)):
            want, e = exact_codes(val, bits.astype(np.float64), floor)
            got = host(st[name][i].view(torch.uint8)).astype(np.int64)
            scale = host(st[name + "_scale"][i].view(torch.uint8)).astype(np.int64)
            want, odd = want.reshape(-1)[:len(p)], ~np.isfinite(val).reshape(-1)[:len(p)]
            assert np.array_equal(scale, e), (i, name, np.sum(scale != e))
            assert np.all((got[odd] & 0x7F) == 0x7F), (i, name)
            assert np.array_equal(got[~odd], want[~odd]), (i, name, np.sum(got[~odd] != want[~odd]))


def test_adamw_8_bit_codes_of_every_float_of_a_scale():
    # every fp32 value of [2^-6, 448], 255 to a block beside a 448 that sets the
    # scale to 1, signs in turn: m = x, r = sqrt(x^2) = |x|.  Codes against the
    # definition, whose sum of place and random bits is rounded to fp32
    first, last = 0x3C800000, 0x43E00000
    blocks = -(-(last - first + 1) // 255)
    x = torch.arange(first, first + blocks * 255, dtype=torch.int32, device="cuda").clamp(max=last).view(blocks, 255)
    x = torch.cat([torch.full((blocks, 1), last, dtype=torch.int32, device="cuda"), x], 1).view(torch.float32)
    x[:, 1::2] *= -1
    w = [torch.zeros(x.numel(), device="cuda")]
    st = pb.adamw_states(w, 8)
    opt = pb.AdamW(w, [x.view(-1)], **st)
    opt.step(lr=1e-3, beta1=0.0, beta2=0.0, seed=17)
    for name in ("m_scale", "v_scale"):
        assert bool((st[name][0].view(torch.uint8) == 127).all())
    M = 0xFFFFFFFF

    def mix_t(h):
        h = (h ^ (h >> 16)) * 0x9E3779B1 & M
        h = (h ^ (h >> 15)) * 0xB7E15163 & M
        return h ^ (h >> 16)
    key = int(mix(mix(mix(np.uint64(17)) + np.uint64(1) & np.uint64(M)) & np.uint64(M)))
    step = 1 << 24
    for at in range(0, x.numel(), step):
        val = x.view(-1)[at:at + step]
        index = torch.arange(at, at + len(val), device="cuda")
        bits = mix_t((index * 0x6A09E667 + key) & M)
        y = val.abs().double()
        ey = (val.view(torch.int32) >> 23 & 0xFF).long() - 127
        for name, part, sign in (("m", bits & 0xFFFF, val < 0), ("v", bits >> 16, None)):
            place = (y * torch.exp2(3.0 - ey) + part.double() / 65536).float()
            want = (ey + 6) * 8 + place.long() + (128 * sign if sign is not None else 0)
            got = st[name][0].view(torch.uint8)[at:at + step].long()
            assert torch.equal(got, want), (name, at, int((got != want).sum()))


def test_adamw_takes_the_same_roots_with_either_states():
    # from zero states a step's update depends on the root alone, which the two
    # kinds of states take by different instructions: the same bits for every
    # fp32 gradient of [1, 4), at several powers of four
    x = torch.arange(0x3F800000, 0x40800000, dtype=torch.int32, device="cuda").view(torch.float32)
    for power in (-20, -6, 0, 7, 28):
        g = x * 4.0 ** power
        out = []
        for bits in (32, 8):
            w = [torch.zeros_like(g)]
            pb.AdamW(w, [g], **pb.adamw_states(w, bits)).step(lr=1.0, beta1=0.9, beta2=0.99, eps=1e-30)
            out.append(w[0])
        assert torch.equal(*out) and bool((out[0] < -0.99).all()), power


def test_adamw_of_empty_and_zero_tensors():
    opt, w, g, st, lows = make([0, 300, 0], 8, torch.float32, None, 23)
    g[1].zero_()
    check_step(opt, w, g, st, lows, 1)
    assert not bool(st["m"][1].float().any()) and not bool(st["v"][1].float().any())
    empty = torch.zeros(0, device="cuda")
    pb.AdamW([empty], [empty], [empty], [empty]).step(**HYPER, max_norm=1.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_leaves_everything_when_the_norm_is_not_finite(bits):
    for bad in (math.inf, math.nan):
        opt, w, g, st, lows = make([500, 9000], bits, torch.bfloat16, torch.bfloat16, 24)
        opt.step(**HYPER, max_norm=1.0)
        keep = [x.clone() for x in w + lows + st["m"] + st["v"]]
        g[0][7] = bad
        norm = opt.step(**HYPER, max_norm=1.0)
        assert not math.isfinite(float(norm)) and opt.t == 1
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(keep, w + lows + st["m"] + st["v"]))
        # without clipping the formula holds: only that value is lost
        opt.step(**HYPER)
        assert opt.t == 2 and int((~torch.isfinite(w[0])).sum()) == 1 and bool(torch.isfinite(w[1]).all())
        if bits == 8:
            assert int(torch.isnan(st["m"][0].float()).sum()) == 1 == int(torch.isnan(st["v"][0].float()).sum())


def test_adamw_norm_of_large_and_small_gradients():
    # squares beyond fp32's range, and a long tail of small values
    opt, w, g, st, lows = make([100000, 10], 32, torch.float32, None, 25)
    g[0].fill_(1e30)
    g[1].fill_(-3e30)
    want = math.sqrt(1e5 * 1e60 + 10 * 9e60)
    assert abs(float(opt.step(**HYPER, max_norm=1.0)) - want) <= 4 * u * want
    assert bool(torch.isfinite(w[0]).all())
    norm = torch.zeros((), device="cuda")
    g[0].fill_(1e-30)
    g[1].zero_()
    assert opt.step(**HYPER, norm=norm) is norm
    assert abs(float(norm) - 1e-30 * math.sqrt(1e5)) <= 4 * u * 1e-27


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_adamw_clips_norms_whose_factor_fp32_cannot_hold(bits, dtype):
    # gradients of 2^100 to 2^127: factors down to 2^-145, below 2^-126 with
    # fewer digits than fp32 has
    for top in (100, 117, 127):
        opt, w, g, st, lows = make([70001, 500], bits, dtype, None, 26)
        for x in g:
            x.copy_(x.float().clamp(-0.5, 0.5) * 2.0 ** top)
        g[1][:400] *= 2.0 ** -30
        norm = math.sqrt(sum(float((x.double() ** 2).sum()) for x in g))

        class Plan:                                    # a norm beyond fp32 is told as infinite
            @staticmethod
            def step(**kw):
                got = float(opt.step(**kw))
                assert abs(got - norm) <= 2 * u * norm or (got == math.inf and norm > torch.finfo(torch.float32).max)
                return norm
        check_step(Plan, w, g, st, lows, 1, max_norm=1e-3 if top > 100 else 1.0)


def test_adamw_8_bit_states_keep_their_mean():
    # v moves by 1e-3 of itself a step, a code apart by 6 to 12%: only the
    # random rounding lets it decay.  After t steps without gradients the mean of
    # r^2 over N values is beta2^t of the start, within what the rounding adds
    N = 1 << 16
    w, g = [torch.zeros(N, device="cuda")], [torch.ones(N, device="cuda")]
    st = pb.adamw_states(w, 8)
    opt = pb.AdamW(w, g, **st)
    h = dict(lr=0.0, beta1=0.9, beta2=0.999, eps=1e-8)
    opt.step(**h, seed=1)
    r0 = values(st["v"][0], st["v_scale"][0]).mean()
    assert abs(r0 - math.sqrt(1e-3)) <= 0.07 * math.sqrt(1e-3) * 5 / math.sqrt(N)
    g[0].zero_()
    for s in range(200):
        opt.step(**h, seed=s)
    r = values(st["v"][0], st["v_scale"][0])
    # r is unbiased: its mean is 0.999^(200/2) of r0; its spread stays below a
    # code's step (1/8), so the mean of N is within 5 / 8 / sqrt(N)
    want = r0 * 0.999 ** 100
    assert abs(r.mean() - want) <= 5 / 8 / math.sqrt(N) * want + 1e-4 * want, (r.mean(), want)
    m = values(st["m"][0], st["m_scale"][0])
    # m, too, keeps its mean; a step rounds it by a factor whose variance is at
    # most p (1 - p) / 8^2 <= 1 / 256, so the relative variance of 200 steps is at
    # most e^(200 / 256) - 1, and the mean of N is within 5 deviations
    want = 0.1 * 0.9 ** 200
    assert abs(m.mean() - want) <= 5 * math.sqrt((math.exp(200 / 256) - 1) / N) * want, (m.mean(), want)


def test_adamw_beyond_two_to_the_32_values():
    N = (1 << 32) + 5000
    w = torch.full((N,), 0.5, device="cuda")
    g = torch.full((N,), 0.25, dtype=torch.bfloat16, device="cuda")
    st = pb.adamw_states([w], 8)
    opt = pb.AdamW([w], [g], **st)
    norm = opt.step(**HYPER, max_norm=1e9)
    assert abs(float(norm) - 0.25 * math.sqrt(N)) <= 2 * u * float(norm)
    assert float(w[0]) < 0.5
    for part in (w[1 << 30:], w[:1 << 30]):
        assert float(part.min()) == float(part.max()) == float(w[0])
    # the rounding of the last values is theirs
    last = values(st["m"][0][-5000 // 256 * 256:].contiguous(), st["m_scale"][0][-20:])
    assert 0.9 * 0.025 < np.abs(last).min() and np.abs(last).max() < 1.1 * 0.025 and len(np.unique(last)) == 2


# -- together ----------------------------------------------------------------------
def head_step(X, W, low, y, off, G, loss, opt, state):
    """A training step of a language model's head over workers with ragged
    token batches: logits, loss and its gradient, worker gradients, their mean
    over the fastest workers, AdamW."""
    Z = pb.group_matmul(X, low, off)
    loss, dZ = pb.token_loss(Z, y, off, dZ=Z, loss=loss)
    dX = pb.group_input_grad(dZ, low, off)
    pb.group_weight_grad(X, dZ, off, out=G)
    state["mean"]()
    norm = opt.step(lr=1e-2, max_norm=1.0, seed=5)
    return loss, dX, norm


def head_setup(seed, bits):
    n, d, C, lengths, k = 6, 40, 104, [30, 0, 51, 7, 64, 20], 4
    T = sum(lengths)
    g = gen(seed)
    X = normal(g, (T, d), torch.bfloat16)
    y = torch.randint(-1, C, (T,), generator=g, device="cuda", dtype=torch.int32)
    W = normal(g, (d, C), torch.float32, 0.1)
    low = W.bfloat16()
    G, grad = torch.empty((n, d, C), device="cuda"), torch.empty((d * C,), device="cuda")
    mask, loss = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(n, device="cuda")
    ticks = torch.tensor([5, 2, 9, 1, 4, 3], dtype=torch.int64, device="cuda")
    st = pb.adamw_states([W], bits)
    opt = pb.AdamW([W], [grad.view(d, C)], **st, low=[low])
    return n, d, C, lengths, k, X, y, W, low, G, grad, mask, loss, ticks, st, opt


@pytest.mark.parametrize("bits", [32, 8])
def test_a_heads_training_steps_together(bits):
    n, d, C, lengths, k, X, y, W, low, G, grad, mask, loss, ticks, st, opt = head_setup(31, bits)
    off = offsets_of(lengths)
    ctx = pb.Context(pb.make_config("softmax", n, 1, d, C))
    state = {"mean": lambda: ctx.aggregate_fastest(G.view(n, -1), ticks, k, g=grad, mask=mask)}
    for t in (1, 2, 3):
        W0, low0 = host(W).astype(np.float64), low.double()
        head_step(X, W, low, y, off, G, loss, opt, state)
        ctx.sync()
        # in 64 bits, from the same parameters
        Z = X.double() @ low0
        ref_loss, dZ, _ = loss_ref(Z, y, lengths, 0, 1.0)
        # logits in bf16 are off by 2^-8 of themselves (|z| below 4): a mean loss
        # by at most 2 * 2^-6
        assert bool(((loss.double() - ref_loss).abs() <= 2.0 ** -5).all())
        order = np.argsort(host(ticks), kind="stable")[:k]
        assert sorted(np.nonzero(host(mask))[0].tolist()) == sorted(order.tolist())
        at = np.concatenate([[0], np.cumsum(lengths)])
        mean = sum(X[at[i]:at[i + 1]].double().t().contiguous() @ dZ[at[i]:at[i + 1]] for i in order) / k
        err = (grad.view(d, C).double() - mean).norm() / mean.norm()
        # two roundings to bf16 (2^-9 each at most half a step 2^-8), the first of
        # values up to 4 through exp
        assert float(err) <= 2.0 ** -4, float(err)
        assert torch.equal(low, W.bfloat16()) and np.any(host(W) != W0) and bool(torch.isfinite(W).all())
    assert opt.t == 3


@pytest.mark.parametrize("bits", [32, 8])
def test_a_heads_training_steps_captured(bits):
    # the same steps eagerly and as replays of one captured graph: every replay
    # has the bits of the eager step, t and the rounding included
    def states(s):
        return [x.view(torch.uint8).clone() for x in [s[7], s[8], s[12]] + [t for v in s[14].values() for t in v]]
    runs = []
    for captured in (False, True):
        s = head_setup(32, bits)
        n, d, C, lengths, k, X, y, W, low, G, grad, mask, loss, ticks, st, opt = s
        off = offsets_of(lengths)
        state = {"mean": lambda: torch.mul(G[0].view(-1), 0.5, out=grad)}
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        out = []
        with torch.cuda.stream(stream):
            head_step(X, W, low, y, off, G, loss, opt, state)
            stream.synchronize()
            out.append(states(s))
            if captured:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    head_step(X, W, low, y, off, G, loss, opt, state)
            for _ in range(4):
                if captured:
                    graph.replay()
                else:
                    head_step(X, W, low, y, off, G, loss, opt, state)
                torch.cuda.synchronize()
                # unrelated eager work between the replays
                pb.group_matmul(X[:9], low, offsets_of([9]))
                out.append(states(s))
        torch.cuda.synchronize()
        assert opt.t == 5
        runs.append(out)
    for a, b in zip(*runs):
        assert all(torch.equal(x, z) for x, z in zip(a, b))


STEP_MODELS = [("softmax", dict(n=5, B=32, d=60, C=7), "none"), ("softmax", dict(n=64, B=256, d=200, C=10), "none"),
               ("softmax", dict(n=4, B=64, d=2048, C=120), "selected"), ("mlp", dict(n=6, B=32, d=50, H=40, C=5), "all")]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("model,kw,g_rows", STEP_MODELS)
def test_dbw_step_with_adamw_as_the_servers_update(model, kw, g_rows, bits):
    # every step of the simulation, with AdamW on parts of w, against an AdamW
    # step by hand on the g that the simulation made; the choice and the
    # statistics are those of SGD
    n, d, C = kw["n"], kw["d"], kw["C"]
    g = gen(41)
    X = torch.rand((n, kw["B"], d), generator=g, device="cuda")
    y = torch.randint(0, C, (n, kw["B"]), generator=g, device="cuda", dtype=torch.int32)
    ctx = pb.Context(pb.make_config(model, g_rows=g_rows, **kw))
    other = pb.Context(pb.make_config(model, g_rows=g_rows, **kw))
    P = ctx.P
    cut = P // 3 + 1
    w = normal(g, (P,), torch.float32, 0.05)
    frozen = w[-5:].clone()

    def parts(x):
        return [x[:cut], x[cut:P - 5]]
    st = pb.adamw_states(parts(w), bits)
    opt = pb.AdamW(parts(w), parts(ctx.gradient()), **st, weight_decay=[0.0, 0.1])
    hand_w, hand_g = w.clone(), torch.empty_like(w)
    hand_st = pb.adamw_states(parts(hand_w), bits)
    hand = pb.AdamW(parts(hand_w), parts(hand_g), **hand_st, weight_decay=[0.0, 0.1])
    hyper = dict(lr=0.01, max_norm=0.5, seed=9)
    ctx.use_adamw(opt, **hyper)
    for t in range(4):
        ticks = np.random.default_rng(t).integers(1, 1000, n)
        w_sgd = w.clone()
        k = ctx.step(w, X, y, ticks, wait=True)
        out = ctx.step_outputs()
        ctx.sync()
        hand_g.copy_(out["g"])
        hand.step(**hyper)
        assert torch.equal(w, hand_w) and bool(torch.isfinite(w).all()) and not torch.equal(w, w_sgd)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for m in st for a, b in zip(st[m], hand_st[m]))
        if t == 0:   # the first iteration of a context that updates by SGD has the same k and g
            assert other.step(w_sgd, X, y, ticks, wait=True) == k
            other.sync()
            assert torch.equal(other.step_outputs()["g"], out["g"])
    assert torch.equal(w[-5:], frozen) and opt.t == 4
    # a w that the plan does not update, and a plan that does not fit
    with pytest.raises(pb.DBWError):
        ctx.step(hand_w, X, y, ticks)
    four = pb.adamw_states([w[:4], w[4:8]])
    for bad in (pb.AdamW(parts(w), parts(hand_g), **st),
                pb.AdamW([w[:4], w[4:8]], [ctx.gradient()[:4], ctx.gradient()[5:9]], **four),
                pb.AdamW([w[:4], w[4:8]], [w[:4].half(), w[4:8].half()], **four)):
        with pytest.raises(pb.DBWError):
            ctx.use_adamw(bad, lr=0.1)
    with pytest.raises(pb.DBWError):
        ctx.use_adamw(opt, lr=-1.0)
    # and back to SGD
    ctx.use_adamw(None)
    before = hand_w.clone()
    ctx.step(hand_w, X, y, ticks)
    ctx.sync()
    step = before.double() - 0.1 * ctx.step_outputs()["g"].double()
    assert bool(((hand_w.double() - step).abs() <= 4 * u * (before.double().abs() + step.abs() + 1e-3)).all())
    assert opt.t == 4


def test_a_context_and_its_plan_end_with_their_last_reference():
    import gc
    import weakref

    def simulation():
        n, B, d, C = 4, 8, 1 << 21, 8                  # 64 MiB a parameter vector
        ctx = pb.Context(pb.make_config("softmax", n, B, d, C))
        w = torch.zeros(ctx.P, device="cuda")
        view = ctx.gradient()
        opt = pb.AdamW([w[:64]], [view[:64]], **pb.adamw_states([w[:64]]))
        ctx.use_adamw(opt, lr=0.1)
        return ctx, opt, w, view
    gc.collect()
    ctx, opt, w, view = simulation()
    # memory that is only a context's (torch keeps what its tensors leave)
    del opt, w, view
    ref, plan = weakref.ref(ctx), weakref.ref(ctx._adamw)
    torch.cuda.synchronize()
    held = torch.cuda.mem_get_info()[0]
    del ctx
    gc.collect()
    assert ref() is None and plan() is None
    assert torch.cuda.mem_get_info()[0] - held > 64 << 20
    # a closed context keeps no plan; a view, or a plan over it, keeps the memory
    for last in ("view", "plan"):
        ctx, opt, w, view = simulation()
        ref, plan = weakref.ref(ctx), weakref.ref(opt)
        view.fill_(3.0)
        view[:64] = 0.5
        held = torch.cuda.mem_get_info()[0]
        ctx.close()
        ctx.close()
        if last == "view":
            del opt
            assert plan() is None
        else:
            del view
        del ctx
        gc.collect()
        assert ref() is None and torch.cuda.mem_get_info()[0] - held < 64 << 20
        if last == "view":
            assert float(view[0]) == 0.5 and float(view[64:].min()) == 3.0 == float(view[64:].max())
            del view
        else:
            opt.step(lr=0.25)                         # the first step moves every weight by lr
            assert bool(((w[:64] + 0.25).abs() < 1e-5).all()) and not bool(w[64:].any())
            del opt
            assert plan() is None
        gc.collect()
        torch.cuda.synchronize()
        assert torch.cuda.mem_get_info()[0] - held > 64 << 20


def test_calls_on_another_stream_and_twice_give_the_same_bits():
    g = gen(33)
    T, d, C, n = 900, 256, 520, 7
    lengths = ragged(5, n, T)
    off = offsets_of(lengths)
    X, W, y = normal(g, (T, d), torch.bfloat16), normal(g, (n, d, C), torch.bfloat16), \
        torch.randint(-1, C, (T,), generator=g, device="cuda", dtype=torch.int32)

    def all_of(stream=None):
        Z = pb.group_matmul(X, W, off, stream=stream)
        loss, dZ = pb.token_loss(Z, y, off, stream=stream)
        return Z, loss, dZ, pb.group_input_grad(dZ, W, off, stream=stream), pb.group_weight_grad(X, dZ, off, stream=stream)
    first = all_of()
    torch.cuda.synchronize()
    again = all_of()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        there = all_of()
    # a stream given to the calls: their memory is that stream's, and what the
    # current stream allocates and fills meanwhile is not it
    given = all_of(stream=other)
    noise = [torch.full((T, C), 7.0, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    assert all(float(x[0, 0]) == 7.0 for x in noise)
    for a, b, c, e in zip(first, again, there, given):
        assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(a, e)


def test_offsets_that_break_the_rules_stay_inside():
    # each offset is taken as the nearest allowed one; nothing outside is touched
    g = gen(34)
    T, d, C = 50, 64, 72
    X, W = normal(g, (T, d), torch.bfloat16), normal(g, (3, d, C), torch.bfloat16)
    y = torch.zeros(T, dtype=torch.int32, device="cuda")
    for o in ([0, 60, 70, 80], [-5, 10, 20, 50], [10, 5, 30, 20], [50, 0, 0, 0], [-3, -2, -1, 0]):
        off = torch.tensor(o, dtype=torch.int32, device="cuda")
        big = torch.full((T + 20, C), 2.0, dtype=torch.bfloat16, device="cuda")
        pb.group_matmul(X, W, off, out=big[10:-10])
        assert bool((big[:10] == 2.0).all()) and bool((big[-10:] == 2.0).all()), o
        loss, _ = pb.token_loss(big[10:-10], y, off)
        G = pb.group_weight_grad(X, big[10:-10], off)
        torch.cuda.synchronize()
        assert loss.shape == (3,) and G.shape == (3, d, C)
    Y = torch.full((T, C), 2.0, dtype=torch.bfloat16, device="cuda")
    pb.group_matmul(X, W, torch.tensor([0, 60, 70, 80], dtype=torch.int32, device="cuda"), out=Y)
    assert torch.equal(Y, pb.group_matmul(X, W, offsets_of([50, 0, 0])))


def test_products_and_losses_in_parts_captured():
    # sums and rows in parts, in a padded batch: rows of no group before, and
    # behind, the groups keep what they held.  One graph, replayed with other
    # inputs, against the same calls made eagerly
    g = gen(35)
    T, d, C, first = 12000, 2048, 72, 5
    lengths = [0, 1, 9000, 2000]
    off = offsets_of(lengths, first)
    end = first + sum(lengths)
    few = offsets_of([3, 0, 20], first)                    # few rows of a long sum
    X = normal(g, (T, d), torch.bfloat16)
    Y0 = normal(g, (T, C), torch.bfloat16)
    y = torch.randint(-1, C, (T,), generator=g, device="cuda", dtype=torch.int32)
    W = normal(g, (3, d, C), torch.bfloat16, d ** -0.5)
    small = X[:30]
    Z, dZ = torch.empty_like(Y0), torch.full_like(Y0, 2.0)
    Y, G = torch.full((30, C), 2.0, dtype=torch.bfloat16, device="cuda"), torch.empty((4, d, C), device="cuda")
    dX = torch.full((30, d), 2.0, dtype=torch.bfloat16, device="cuda")
    loss = torch.empty(4, device="cuda")
    outs = [dZ, Y, G, dX, loss]

    def call():
        Z.copy_(Y0)
        pb.token_loss(Z, y, off, dZ=dZ, loss=loss)
        pb.group_weight_grad(X, dZ, off, out=G)
        pb.group_matmul(small, W, few, out=Y)
        pb.group_input_grad(Y, W, few, out=dX)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        for replay in range(4):
            X.normal_(generator=g)
            Y0.normal_(generator=g)
            call()
            torch.cuda.synchronize()
            want = [x.clone() for x in outs]
            for x in (dZ, Y, dX):
                x.fill_(2.0)
            G.fill_(3.0)
            loss.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            pb.group_matmul(X[:9], W[0], offsets_of([9]))   # unrelated eager work between the replays
            for a, b in zip(outs, want):
                assert torch.equal(a, b), replay
            assert bool((dZ[:first] == 2).all()) and bool((dZ[end:] == 2).all())
            assert bool((Y[:first] == 2).all()) and bool((Y[first + 23:] == 2).all())
            assert bool((dX[:first] == 2).all()) and bool((dX[first + 23:] == 2).all())
            assert bool((G[0] == 0).all())
    check_loss(Y0[first:end], y[first:end], lengths)
