"""Argument checks of the operators for language models (host only): each
refusal comes before any HIP call."""
import ctypes

import numpy as np
import pytest

pb = pytest.importorskip("paper_2004_14696_amd.binding")

P = ctypes.c_void_p(4096)
NULL = ctypes.c_void_p(0)
ODD = ctypes.c_void_p(4097)


@pytest.fixture(scope="module")
def lib():
    return pb.load_library()


def _shape(**kw):
    base = dict(form=pb.DBW_GROUP_FORWARD, dtype=pb.DBW_BF16, out_dtype=pb.DBW_BF16, n=4, d=64, C=32, T=100, ld_d=64,
                ld_C=32, ld_W=32, st_W=64 * 32)
    return pb.GroupShape(**{**base, **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(form=3), pb.DBW_EINVAL), (dict(form=-1), pb.DBW_EINVAL),
    (dict(dtype=pb.DBW_F32, out_dtype=pb.DBW_F32), pb.DBW_EUNSUPPORTED), (dict(dtype=7), pb.DBW_EINVAL),
    (dict(out_dtype=pb.DBW_F16), pb.DBW_EINVAL), (dict(n=0), pb.DBW_EINVAL), (dict(n=pb.DBW_MAX_N + 1), pb.DBW_EINVAL),
    (dict(d=0), pb.DBW_EINVAL), (dict(C=0), pb.DBW_EINVAL),
    (dict(d=(1 << 20) + 1, ld_d=(1 << 20) + 1), pb.DBW_EUNSUPPORTED),
    (dict(T=-1), pb.DBW_EINVAL), (dict(T=1 << 31), pb.DBW_EINVAL),
    (dict(ld_d=63), pb.DBW_EINVAL), (dict(ld_C=31), pb.DBW_EINVAL), (dict(ld_W=31), pb.DBW_EINVAL),
    (dict(ld_d=1 << 21), pb.DBW_EUNSUPPORTED), (dict(st_W=64 * 32 - 1), pb.DBW_EINVAL), (dict(st_W=-1), pb.DBW_EINVAL),
    (dict(st_W=1 << 40), pb.DBW_EUNSUPPORTED),
    (dict(form=pb.DBW_GROUP_WEIGHT_GRAD, st_W=0), pb.DBW_EINVAL),
    # 2^23 output tiles
    (dict(T=(1 << 31) - 1, C=1 << 20, ld_C=1 << 20, ld_W=1 << 20, st_W=1 << 26), pb.DBW_EUNSUPPORTED),
])
def test_group_product_refuses_shapes(lib, kw, status):
    s = _shape(**kw)
    need = ctypes.c_int64(-5)
    assert lib.dbw_group_workspace(ctypes.byref(s), ctypes.byref(need)) == status
    assert need.value == -5
    assert lib.dbw_group_product(ctypes.byref(s), P, P, P, P, P, 1 << 40, NULL) == status
    assert lib.dbw_last_error(None).startswith(b"dbw_group_product")


def test_group_product_refuses_pointers_and_workspaces(lib):
    def call(shape, o=P, a=P, b=P, out=P, ws=P, nbytes=1 << 40):
        return lib.dbw_group_product(ctypes.byref(shape), o, a, b, out, ws, nbytes, NULL)
    s = _shape()
    for kw in (dict(o=NULL), dict(a=NULL), dict(b=NULL), dict(out=NULL), dict(a=ODD), dict(b=ODD), dict(out=ODD),
               dict(o=ODD)):
        assert call(s, **kw) == pb.DBW_EINVAL, kw
    # a long sum over few rows is split, and needs its workspace
    long = _shape(n=1, T=1, d=65536, ld_d=65536, st_W=0)
    need = ctypes.c_int64()
    assert lib.dbw_group_workspace(ctypes.byref(long), ctypes.byref(need)) == pb.DBW_OK and need.value > 0
    assert call(long, ws=NULL) == pb.DBW_EINVAL
    assert call(long, nbytes=need.value - 1) == pb.DBW_EINVAL
    assert call(long, ws=ctypes.c_void_p(4104)) == pb.DBW_EINVAL
    assert b"workspace" in lib.dbw_last_error(None)
    assert lib.dbw_group_product(None, P, P, P, P, P, 0, NULL) == pb.DBW_EINVAL
    assert lib.dbw_group_workspace(ctypes.byref(s), None) == pb.DBW_EINVAL


def test_group_product_refuses_an_output_in_the_place_of_an_input(lib):
    other, third = ctypes.c_void_p(1 << 20), ctypes.c_void_p(1 << 21)
    for form in (pb.DBW_GROUP_FORWARD, pb.DBW_GROUP_INPUT_GRAD, pb.DBW_GROUP_WEIGHT_GRAD):
        s = _shape(form=form, d=32, ld_d=32, st_W=32 * 32)
        for a, b, out in ((P, other, P), (P, other, other)):
            assert lib.dbw_group_product(ctypes.byref(s), third, a, b, out, third, 1 << 40, NULL) == pb.DBW_EINVAL
            assert b"overlap" in lib.dbw_last_error(None)


def test_token_loss_refusals(lib):
    assert lib.dbw_token_workspace(0, 1) == -1 and lib.dbw_token_workspace(1, -1) == -1
    assert lib.dbw_token_workspace(pb.DBW_MAX_N + 1, 1) == -1 and lib.dbw_token_workspace(1, 1 << 31) == -1
    need = lib.dbw_token_workspace(4, 100)
    assert need >= 4 * 104

    def call(n=4, T=100, C=50, dtype=pb.DBW_BF16, o=P, Z=P, ld=50, y=P, scale=1.0, dZ=NULL, ldd=50, loss=P, ws=P,
             nbytes=1 << 30):
        return lib.dbw_token_loss(n, T, C, dtype, o, Z, ld, y, scale, dZ, ldd, loss, ws, nbytes, NULL)
    for kw in (dict(n=0), dict(n=pb.DBW_MAX_N + 1), dict(T=-1), dict(T=1 << 31), dict(C=0), dict(dtype=3), dict(o=NULL),
               dict(Z=NULL), dict(y=NULL), dict(loss=NULL), dict(ws=NULL), dict(Z=ODD), dict(dZ=ODD), dict(y=ODD),
               dict(ld=49), dict(dZ=P, ldd=49), dict(dZ=P, ld=60, ldd=50), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(scale=1e300), dict(nbytes=need - 1), dict(ws=ctypes.c_void_p(4100))):
        assert call(**kw) == pb.DBW_EINVAL, kw
        assert lib.dbw_last_error(None).startswith(b"dbw_token_loss")
    assert call(C=(1 << 24) + 1, ld=1 << 25) == pb.DBW_EUNSUPPORTED
    assert call(ld=1 << 32) == pb.DBW_EUNSUPPORTED


def test_adamw_refusals(lib):
    def create(cfg=None, **kw):
        t = pb.AdamWTensor(w=4096, g=4096, m=4096, v=4096, count=10, lr_scale=1.0, weight_decay=0.0)
        for k, v in kw.items():
            setattr(t, k, v)
        c = pb.AdamWConfig(**{**dict(state_bits=32, g_dtype=pb.DBW_F32, low_dtype=pb.DBW_BF16, tensors=1, t=0), **(cfg or {})})
        out = ctypes.c_void_p(1)
        return lib.dbw_adamw_create(ctypes.byref(c), ctypes.byref(t), ctypes.byref(out))
    for cfg in (dict(state_bits=16), dict(g_dtype=5), dict(low_dtype=pb.DBW_F32), dict(tensors=0), dict(tensors=65537),
                dict(t=-1), dict(state_bits=8)):
        assert create(cfg) == pb.DBW_EINVAL, cfg
    for kw in (dict(count=-1), dict(w=None), dict(g=None), dict(m=None), dict(v=None), dict(w=4098), dict(g=4097),
               dict(m=4097), dict(w_low=4097), dict(lr_scale=-1.0), dict(weight_decay=float("nan"))):
        assert create(**kw) == pb.DBW_EINVAL, kw
        assert lib.dbw_last_error(None).startswith(b"dbw_adamw_create")
    assert create(count=(1 << 40) + 1) == pb.DBW_EUNSUPPORTED
    assert create(count=1 << 37) == pb.DBW_EUNSUPPORTED      # 2^27 chunks of 1024
    assert lib.dbw_adamw_create(None, None, None) == pb.DBW_EINVAL
    h = pb.AdamWHyper(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, grad_scale=1.0)
    assert lib.dbw_adamw_step(None, ctypes.byref(h), None, None) == pb.DBW_EINVAL
    assert lib.dbw_adamw_export(None, None) == pb.DBW_EINVAL and lib.dbw_adamw_import(None, 0) == pb.DBW_EINVAL
    lib.dbw_adamw_destroy(None)


def test_adamw_bits_follow_their_definition(lib):
    M = (1 << 32) - 1

    def mix(x):
        x ^= x >> 16
        x = x * 0x9E3779B1 & M
        x ^= x >> 15
        x = x * 0xB7E15163 & M
        return x ^ x >> 16
    for seed, t, tensor, index in ((0, 1, 0, 0), (12345, 101, 7, 255), (M, 1 << 40, 65535, (1 << 39) + 5), (3, 2, 1, 1 << 32)):
        key = mix(mix(mix(seed) + t & M) + tensor & M)
        want = mix(((index & M) * 0x6A09E667 + (index >> 32) * 0xBB67AE85 + key) & M)
        assert lib.dbw_adamw_bits(seed, t, tensor, index) == want
    # uniform: the mean of N uniform 16-bit values is within 5 / sqrt(12 N) of 1/2
    N = 20000
    b = np.array([lib.dbw_adamw_bits(1, 5, 2, i) for i in range(N)])
    for part in (b & 0xFFFF, b >> 16):
        assert abs(part.mean() / 65536 - 0.5) < 5 / np.sqrt(12 * N)


def test_binding_refuses_what_the_library_cannot_see():
    torch = pytest.importorskip("torch")
    X, W, y = torch.zeros(6, 8), torch.zeros(2, 8, 4), torch.zeros(6, dtype=torch.int32)
    off = torch.tensor([0, 2, 6], dtype=torch.int32)
    Xb, Wb = X.bfloat16(), W.bfloat16()
    for call in (lambda: pb.group_matmul(Xb, Wb, off),                               # not on a GPU
                 lambda: pb.group_matmul(X, W, off),                                 # fp32 inputs
                 lambda: pb.group_matmul(Xb, W, off),                                # two types
                 lambda: pb.group_matmul(Xb, Wb[:1], off),                           # another number of groups
                 lambda: pb.group_matmul(Xb, Wb, off.long()), lambda: pb.group_matmul(Xb, Wb, off[:1]),
                 lambda: pb.group_matmul(Xb[:, :4], Wb, off), lambda: pb.group_matmul(Xb.t(), Wb, off),
                 lambda: pb.group_matmul(Xb, Wb.transpose(1, 2), off),
                 lambda: pb.group_matmul(Xb, Wb, off, out=torch.zeros(6, 5)),
                 lambda: pb.group_matmul(Xb, Wb, off, out_dtype=torch.float64),
                 lambda: pb.group_weight_grad(Xb, Xb[:4], off), lambda: pb.group_weight_grad(Xb, W.bfloat16(), off),
                 lambda: pb.token_loss(X, y, off), lambda: pb.token_loss(X.double(), y, off),
                 lambda: pb.token_loss(X, y.long(), off), lambda: pb.token_loss(X, y[:5], off),
                 lambda: pb.token_loss(X, y, off, dZ=Xb), lambda: pb.token_loss(X[:, ::2], y, off),
                 lambda: pb.AdamW([X], [X], [X], [X]), lambda: pb.AdamW([], [], [], []),
                 lambda: pb.AdamW([X], [X, X], [X], [X]), lambda: pb.AdamW([Xb], [X], [X], [X]),
                 lambda: pb.AdamW([X], [X], [X], [X], m_scale=[X]), lambda: pb.adamw_states([X], 16),
                 lambda: pb.AdamW([X], [X], [X], [X], weight_decay=[0.1, 0.2])):
        with pytest.raises(ValueError):
            call()
    # states of either kind have the shapes that AdamW asks for
    s = pb.adamw_states([torch.zeros(3, 100)], 8)
    assert s["m"][0].dtype == torch.float8_e4m3fn and s["m"][0].shape == (3, 100) and s["v_scale"][0].shape == (2,)
    assert float(s["m_scale"][0].float()[0]) == 2.0 ** -126
    assert pb.adamw_states([torch.zeros(5)])["v"][0].dtype == torch.float32


def test_unaligned_products_near_the_most_tiles_are_refused(lib):
    # 2053 x 4086 tiles of 128 x 256 are below 2^23, but lines of an odd length
    # take 128 x 128: in whole runs 2^24 workgroups of 256 threads, and a launch
    # holds fewer than 2^32 threads
    C = 4085 * 256 + 1
    s = _shape(n=1, T=2052 * 128, C=C, ld_C=C, ld_W=C, st_W=0)
    need = ctypes.c_int64(-5)
    assert lib.dbw_group_workspace(ctypes.byref(s), ctypes.byref(need)) == pb.DBW_EUNSUPPORTED
    assert lib.dbw_group_product(ctypes.byref(s), P, P, P, P, P, 1 << 40, NULL) == pb.DBW_EUNSUPPORTED
    s = _shape(n=1, T=2051 * 128, C=C, ld_C=C, ld_W=C, st_W=0)
    assert lib.dbw_group_workspace(ctypes.byref(s), ctypes.byref(need)) == pb.DBW_OK and need.value == 0


@pytest.mark.parametrize("tiles,d,C", [(1, 100, 128), (16, 512, 512), (32, 512, 1024), (33, 1408, 384), (36, 768, 768),
                                       (64, 1024, 1024), (128, 1024, 2048), (192, 1536, 2048), (256, 2048, 2048),
                                       (280, 2560, 1792), (64, 1021, 1023)])
def test_parts_of_weight_gradients(lib, tiles, d, C):
    # parts of 256 terms at least, in at most 512 workgroups and 64 parts; the
    # longest sums take more than half of what they may, at any number of tiles
    last = 1
    for T in (1, 200, 511, 512, 1024, 2048, 4096, 8192, 16384, 65536, 1 << 20, 1 << 30):
        s = _shape(form=pb.DBW_GROUP_WEIGHT_GRAD, out_dtype=pb.DBW_F32, n=1, T=T, d=d, C=C, ld_d=d, ld_C=C, ld_W=C, st_W=0)
        need = ctypes.c_int64(-5)
        assert lib.dbw_group_workspace(ctypes.byref(s), ctypes.byref(need)) == pb.DBW_OK
        parts = max(1, need.value // (4 * d * C))
        assert need.value in (0, 4 * parts * d * C)
        assert parts == 1 or (parts * tiles <= 512 and parts <= 64 and parts * 256 <= T)
        last = parts
    assert last > min(64, 512 // tiles) // 2 or 512 // tiles == 1


def test_adamw_refuses_arrays_that_overlap(lib):
    # two tensors of 300 values, states in 8 bits, each array at a place of its own
    def create(edit):
        t = (pb.AdamWTensor * 2)()
        for i in range(2):
            for j, k in enumerate(("w", "g", "m", "v", "m_scale", "v_scale", "w_low")):
                setattr(t[i], k, 65536 * (1 + 7 * i + j))
            t[i].count, t[i].lr_scale, t[i].weight_decay = 300, 1.0, 0.0
        edit(t)
        c = pb.AdamWConfig(state_bits=8, g_dtype=pb.DBW_F32, low_dtype=pb.DBW_BF16, tensors=2, t=0)
        out = ctypes.c_void_p()
        status = lib.dbw_adamw_create(ctypes.byref(c), t, ctypes.byref(out))
        lib.dbw_adamw_destroy(out)
        return status

    def at(k, size):   # the second tensor's array at a distance of the first one's
        return lambda t: setattr(t[1], k, getattr(t[0], k) + size)
    edits = [at(k, 0) for k in ("w", "m", "v", "m_scale", "v_scale", "w_low")]
    # in the last value of the first one's
    edits += [at("w", 299 * 4), at("m", 299), at("v", 299), at("m_scale", 1), at("w_low", 299 * 2)]
    # with another kind of array, written or read
    edits += [lambda t: setattr(t[0], "v", t[0].m), lambda t: setattr(t[0], "w", t[1].g),
              lambda t: setattr(t[0], "w_low", t[0].w), lambda t: setattr(t[1], "g", t[0].w + 299 * 4)]
    # a long array over a short one in its middle, where both neighbours are apart
    edits += [lambda t: setattr(t[1], "v_scale", t[0].w + 600)]
    for i, edit in enumerate(edits):
        assert create(edit) == pb.DBW_EINVAL, i
        assert b"overlap" in lib.dbw_last_error(None), i
    # one behind the other is allowed, and so is a gradient that two tensors read
    # (without a device the plan then fails to find one)
    for edit in (at("w", 300 * 4), at("m", 300), at("m_scale", 2), at("g", 0), at("g", 4)):
        assert create(edit) in (pb.DBW_OK, pb.DBW_EHIP)


class _NoLibrary:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


def test_a_closed_plan_is_refused():
    opt, ctx = pb.AdamW.__new__(pb.AdamW), pb.Context.__new__(pb.Context)
    opt.h, ctx.h, ctx.lib, opt.lib = None, ctypes.c_void_p(1), _NoLibrary(), _NoLibrary()
    with pytest.raises(ValueError, match="closed"):   # not: back to SGD
        ctx.use_adamw(opt, lr=1e-3)
    ctx._adamw = opt                                  # closed while it was in use
    with pytest.raises(ValueError, match="closed"):
        ctx.step(None, None, None, [0])
    for call in (lambda: opt.step(1e-3), lambda: opt.t, lambda: setattr(opt, "t", 3)):
        with pytest.raises(ValueError, match="closed"):
            call()


def test_a_stream_of_another_device_is_refused():
    torch = pytest.importorskip("torch")

    class Stream:
        device = torch.device("cuda", 1)
    X, W, y = torch.zeros(6, 8).bfloat16(), torch.zeros(2, 8, 4).bfloat16(), torch.zeros(6, dtype=torch.int32)
    off = torch.tensor([0, 2, 6], dtype=torch.int32)
    opt = pb.AdamW.__new__(pb.AdamW)
    opt.h, opt.lib, opt.device = ctypes.c_void_p(1), _NoLibrary(), torch.device("cuda", 0)
    for call in (lambda: pb.group_matmul(X, W, off, stream=Stream()), lambda: pb.token_loss(X, y, off, stream=Stream()),
                 lambda: opt.step(1e-3, stream=Stream())):
        with pytest.raises(ValueError, match="stream"):
            call()
    opt.h = None
