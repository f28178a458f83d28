"""Argument checks of the operators of a transformer block (host only): each
refusal comes before any HIP call."""
import ctypes

import pytest

pb = pytest.importorskip("paper_2004_14696_amd.binding")

NULL, ODD, HALF = ctypes.c_void_p(0), ctypes.c_void_p(4097), ctypes.c_void_p(4098)
A, B, C, D, E, F, G, H = (ctypes.c_void_p(i << 24) for i in range(1, 9))
BIG = 1 << 50


@pytest.fixture(scope="module")
def lib():
    return pb.load_library()


def refused(lib, call, name, status, **kw):
    assert call(**kw) == status, kw
    assert lib.dbw_last_error(None).startswith(name.encode()), kw


ROWS = [dict(n=0), dict(n=pb.DBW_MAX_N + 1), dict(T=-1), dict(T=1 << 31), dict(d=0), dict(dtype=3), dict(dtype=-1),
        dict(o=NULL), dict(o=HALF)]


def test_layer_norm_refusals(lib):
    def call(n=4, T=100, d=64, dtype=pb.DBW_BF16, o=A, X=B, ld_X=64, g=C, b=D, eps=1e-5, Y=E, ld_Y=64):
        return lib.dbw_layer_norm(n, T, d, dtype, o, X, ld_X, g, b, eps, Y, ld_Y, NULL)
    for kw in ROWS + [dict(X=NULL), dict(Y=NULL), dict(g=NULL), dict(X=ODD), dict(Y=ODD), dict(g=HALF), dict(b=HALF),
                      dict(X=HALF, dtype=pb.DBW_F32), dict(ld_X=63), dict(ld_Y=63), dict(eps=0.0), dict(eps=-1.0),
                      dict(eps=float("nan")), dict(eps=1e31), dict(Y=B), dict(Y=C), dict(Y=D)]:
        refused(lib, call, "dbw_layer_norm", pb.DBW_EINVAL, **kw)
    for kw in (dict(d=16385, ld_X=1 << 20, ld_Y=1 << 20), dict(ld_X=1 << 32), dict(ld_Y=1 << 32)):
        refused(lib, call, "dbw_layer_norm", pb.DBW_EUNSUPPORTED, **kw)


def test_layer_norm_grad_refusals(lib):
    for bad in ((0, 1, 1), (pb.DBW_MAX_N + 1, 1, 1), (1, -1, 1), (1, 1 << 31, 1), (1, 1, 0), (1, 1, 16385)):
        assert lib.dbw_layer_norm_workspace(*bad) == -1
    need = lib.dbw_layer_norm_workspace(4, 100, 64)
    assert need > 0

    def call(n=4, T=100, d=64, dtype=pb.DBW_BF16, o=A, dY=B, ld_dY=64, X=C, ld_X=64, g=D, eps=1e-5, dX=E, ld_dX=64, dg=F,
             ld_g=64, db=G, ld_b=64, ws=H, nbytes=BIG):
        return lib.dbw_layer_norm_grad(n, T, d, dtype, o, dY, ld_dY, X, ld_X, g, eps, dX, ld_dX, dg, ld_g, db, ld_b, ws,
                                       nbytes, NULL)
    for kw in ROWS + [dict(dY=NULL), dict(X=NULL), dict(dX=NULL), dict(g=NULL), dict(dg=NULL), dict(dY=ODD), dict(X=ODD),
                      dict(dX=ODD), dict(g=HALF), dict(dg=HALF), dict(db=HALF), dict(ld_dY=63), dict(ld_X=63),
                      dict(ld_dX=63), dict(ld_g=63), dict(ld_b=63), dict(eps=0.0), dict(dX=B), dict(dX=C), dict(dX=D),
                      dict(dX=F), dict(dX=G), dict(dg=B), dict(db=C), dict(db=F), dict(ws=NULL), dict(nbytes=need - 1),
                      dict(ws=ctypes.c_void_p(4104))]:
        refused(lib, call, "dbw_layer_norm_grad", pb.DBW_EINVAL, **kw)
    refused(lib, call, "dbw_layer_norm_grad", pb.DBW_EUNSUPPORTED, ld_g=1 << 32)


def test_group_linear_refusals(lib):
    def call(shape=(), epilogue=True, o=A, X=B, W=C, Y=D, ws=H, nbytes=BIG, **kw):
        s = pb.GroupShape(**{**dict(form=pb.DBW_GROUP_FORWARD, dtype=pb.DBW_BF16, out_dtype=pb.DBW_BF16, n=4, d=64, C=32,
                                    T=100, ld_d=64, ld_C=32, ld_W=32, st_W=64 * 32), **dict(shape)})
        e = pb.LinearEpilogue(**{**dict(activation=pb.DBW_ACT_GELU, bias=E.value, st_bias=32, residual=F.value,
                                        ld_residual=32, pre=G.value, ld_pre=32), **kw})
        return lib.dbw_group_linear(ctypes.byref(s), ctypes.byref(e) if epilogue else None, o, X, W, Y, ws, nbytes, NULL)
    for kw in (dict(shape=dict(n=0)), dict(shape=dict(form=pb.DBW_GROUP_INPUT_GRAD)),
               dict(shape=dict(form=pb.DBW_GROUP_WEIGHT_GRAD)), dict(shape=dict(T=1 << 31)), dict(epilogue=False),
               dict(activation=-1), dict(activation=4), dict(o=NULL), dict(X=NULL), dict(W=NULL), dict(Y=NULL), dict(X=ODD),
               dict(bias=4098), dict(residual=4097), dict(residual=4098, shape=dict(out_dtype=pb.DBW_F32)), dict(pre=4097),
               dict(st_bias=31), dict(st_bias=-1), dict(shape=dict(st_W=0)), dict(ld_residual=31), dict(ld_pre=31),
               dict(residual=D.value, ld_residual=40), dict(pre=B.value), dict(pre=C.value), dict(pre=D.value),
               dict(pre=F.value), dict(Y=B), dict(Y=C)):
        refused(lib, call, "dbw_group_linear", pb.DBW_EINVAL, **kw)
    for kw in (dict(shape=dict(dtype=pb.DBW_F32)), dict(ld_residual=1 << 21), dict(ld_pre=1 << 21), dict(st_bias=1 << 40)):
        refused(lib, call, "dbw_group_linear", pb.DBW_EUNSUPPORTED, **kw)
    long = dict(n=1, T=1, d=65536, ld_d=65536, st_W=0)       # a split sum needs its workspace
    refused(lib, call, "dbw_group_linear", pb.DBW_EINVAL, shape=long, ws=NULL)


def test_linear_grad_refusals(lib):
    for bad in ((0, 1, 1), (1, -1, 1), (1, 1 << 31, 1), (1, 1, 0), (1, 1, (1 << 20) + 1)):
        assert lib.dbw_linear_grad_workspace(*bad) == -1
    need = lib.dbw_linear_grad_workspace(4, 100, 64)

    def call(n=4, T=100, d=64, dtype=pb.DBW_BF16, act=pb.DBW_ACT_SILU, o=A, dY=B, ld_dY=64, Z=C, ld_Z=64, dZ=D, ld_dZ=64,
             db=E, ld_b=64, ws=H, nbytes=BIG):
        return lib.dbw_linear_grad(n, T, d, dtype, act, o, dY, ld_dY, Z, ld_Z, dZ, ld_dZ, db, ld_b, ws, nbytes, NULL)
    for kw in ROWS + [dict(act=-1), dict(act=4), dict(dY=NULL), dict(Z=NULL), dict(dZ=NULL), dict(dY=ODD), dict(Z=ODD),
                      dict(dZ=ODD), dict(db=HALF), dict(ld_dY=63), dict(ld_Z=63), dict(ld_dZ=63), dict(ld_b=63), dict(dZ=B),
                      dict(dZ=C), dict(dZ=E), dict(db=B), dict(db=C), dict(ws=NULL), dict(nbytes=need - 1),
                      dict(ws=ctypes.c_void_p(4104)), dict(act=pb.DBW_ACT_NONE, dZ=NULL, db=NULL)]:
        refused(lib, call, "dbw_linear_grad", pb.DBW_EINVAL, **kw)
    for kw in (dict(d=(1 << 20) + 1, ld_dY=1 << 21), dict(ld_Z=1 << 32)):
        refused(lib, call, "dbw_linear_grad", pb.DBW_EUNSUPPORTED, **kw)


def test_dropout_refusals(lib):
    def call(n=4, T=100, d=64, dtype=pb.DBW_BF16, o=A, X=B, ld_X=64, p=0.1, seed=1, step=C, R=D, ld_R=64, Y=E, ld_Y=64):
        return lib.dbw_dropout(n, T, d, dtype, o, X, ld_X, p, seed, step, R, ld_R, Y, ld_Y, NULL)
    for kw in ROWS + [dict(X=NULL), dict(Y=NULL), dict(X=ODD), dict(R=ODD), dict(Y=ODD), dict(step=ctypes.c_void_p(4100)),
                      dict(ld_X=63), dict(ld_R=63), dict(ld_Y=63), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")),
                      dict(Y=B, ld_Y=70), dict(Y=D, ld_Y=70), dict(Y=C)]:
        refused(lib, call, "dbw_dropout", pb.DBW_EINVAL, **kw)
    for kw in (dict(d=(1 << 20) + 1, ld_X=1 << 21), dict(ld_R=1 << 32)):
        refused(lib, call, "dbw_dropout", pb.DBW_EUNSUPPORTED, **kw)


def _philox(c, k0, k1):
    for _ in range(10):
        p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [q >> 32 ^ c[1] ^ k0, q & 0xFFFFFFFF, p >> 32 ^ c[3] ^ k1, p & 0xFFFFFFFF]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def test_dropout_bits(lib):
    # the generator's published answers for a counter and key of zeros, and of ones
    zero, ones = [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8], [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert _philox([0] * 4, 0, 0) == zero and _philox([0xFFFFFFFF] * 4, 0xFFFFFFFF, 0xFFFFFFFF) == ones
    for c in range(8):
        assert lib.dbw_dropout_bits(0, 0, 0, c) == zero[c // 2] >> 16 * (c % 2) & 0xFFFF
    for seed, step, t, c in ((1 << 63 | 12345, (7 << 32) + 9, (1 << 31) - 1, 12345), (3, -1, 5, 8), ((1 << 64) - 1, 1, 0, 1047)):
        words = _philox([c // 8, t, step & 0xFFFFFFFF, step >> 32 & 0xFFFFFFFF], seed & 0xFFFFFFFF, seed >> 32)
        assert lib.dbw_dropout_bits(seed, step, t, c) == words[c % 8 // 2] >> 16 * (c % 2) & 0xFFFF


def _heads(p, heads, d=64, **kw):
    return pb.Heads(**{**dict(data=p.value, token=heads * d, head=d), **kw})


SHAPE = dict(dtype=pb.DBW_BF16, n=4, heads=4, kv_heads=2, D=64, T=100, scale=0.125)


def _attention_arrays(kw):
    names = ("Q", "K", "V", "O", "dO", "dQ", "dK", "dV")
    arrays = {k: _heads(p, 2 if k in ("K", "V", "dK", "dV") else 4) for k, p in zip(names, (A, B, C, D, E, F, G, H))}
    for name, change in kw.items():
        arrays[name] = None if change is None else _heads(ctypes.c_void_p(arrays[name].data), arrays[name].token // 64, **change)
    return {k: ctypes.byref(v) if v is not None else None for k, v in arrays.items()}


BAD_SHAPES = [(kw, pb.DBW_EINVAL) for kw in (
    dict(dtype=5), dict(n=0), dict(n=65537), dict(T=-1), dict(T=1 << 31), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3),
    dict(D=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=1e21))]
BAD_SHAPES += [(kw, pb.DBW_EUNSUPPORTED) for kw in (
    dict(dtype=pb.DBW_F32), dict(D=68), dict(D=136), dict(heads=1026), dict(T=(1 << 31) - 1, heads=1024))]
BAD_ARRAYS = [({name: change}, status) for name in ("Q", "K", "V", "O") for change, status in (
    (None, pb.DBW_EINVAL), (dict(data=0), pb.DBW_EINVAL), (dict(token=-64), pb.DBW_EINVAL), (dict(head=-64), pb.DBW_EINVAL),
    (dict(data=4104), pb.DBW_EUNSUPPORTED), (dict(token=260), pb.DBW_EUNSUPPORTED), (dict(head=68), pb.DBW_EUNSUPPORTED),
    (dict(token=1 << 21), pb.DBW_EUNSUPPORTED), (dict(head=1 << 40), pb.DBW_EUNSUPPORTED))]


@pytest.mark.parametrize("grad", [False, True])
def test_attention_refusals(lib, grad):
    offsets, lse, ws = (ctypes.c_void_p(i << 24) for i in (9, 10, 11))

    def call(shape=(), o=offsets, lse=lse, ws=ws, nbytes=BIG, **kw):
        s = pb.AttentionShape(**{**SHAPE, **dict(shape)}) if shape is not None else None
        p, a = ctypes.byref(s) if s is not None else None, _attention_arrays(kw)
        if not grad:
            return lib.dbw_attention(p, o, a["Q"], a["K"], a["V"], a["O"], lse, NULL)
        return lib.dbw_attention_grad(p, o, a["dO"], a["Q"], a["K"], a["V"], a["O"], lse, a["dQ"], a["dK"], a["dV"], ws,
                                      nbytes, NULL)
    name = "dbw_attention_grad" if grad else "dbw_attention"
    for shape, status in BAD_SHAPES + [(None, pb.DBW_EINVAL)]:
        refused(lib, call, name, status, shape=shape)
        if shape is not None:
            assert lib.dbw_attention_workspace(ctypes.byref(pb.AttentionShape(**{**SHAPE, **shape}))) == -1
    for change, status in BAD_ARRAYS:
        refused(lib, call, name, status, **change)
    for kw in (dict(o=NULL), dict(o=HALF), dict(lse=HALF)):
        refused(lib, call, name, pb.DBW_EINVAL, **kw)
    if not grad:
        for kw in (dict(O=dict(token=192)), dict(O=dict(head=0)), dict(O=dict(head=56)), dict(O=dict(data=A.value)),
                   dict(O=dict(data=B.value)), dict(O=dict(data=C.value)), dict(lse=A), dict(lse=D)):
            refused(lib, call, name, pb.DBW_EINVAL, **kw)
        return
    need = lib.dbw_attention_workspace(ctypes.byref(pb.AttentionShape(**SHAPE)))
    assert need > 0
    for kw in (dict(lse=NULL), dict(dO=None), dict(dQ=None), dict(dK=None), dict(dV=None), dict(dQ=dict(token=192)),
               dict(dK=dict(token=64)), dict(dV=dict(head=0)), dict(dQ=dict(data=A.value)), dict(dK=dict(data=E.value)),
               dict(dV=dict(data=D.value)), dict(dK=dict(data=H.value)), dict(lse=F), dict(ws=NULL), dict(nbytes=need - 1),
               dict(ws=ctypes.c_void_p(4104))):
        refused(lib, call, name, pb.DBW_EINVAL, **kw)
    refused(lib, call, name, pb.DBW_EUNSUPPORTED, dQ=dict(data=4104))


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    X, off = torch.zeros(4, 8), torch.zeros(2, dtype=torch.int32)
    Q = torch.zeros(4, 2, 8, dtype=torch.bfloat16)
    for call in (lambda: pb.layer_norm(X, X[0], X[0], off), lambda: pb.layer_norm_grad(X, X, X[0], off),
                 lambda: pb.group_linear(X.bfloat16(), X.bfloat16(), off), lambda: pb.group_linear_grad(X, off),
                 lambda: pb.dropout(X, 0.1, 1, off), lambda: pb.attention(Q, Q, Q, off)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call in (lambda: pb.layer_norm(X[0], X[0], X[0], off), lambda: pb.layer_norm(X.double(), X[0], X[0], off),
                 lambda: pb.group_linear(X, X[0], off), lambda: pb.group_linear(X, X, off, activation="swish"),
                 lambda: pb.group_linear(X, X, off, bias=X.view(1, 4, 8)), lambda: pb.group_linear_grad(X, off[:1]),
                 lambda: pb.dropout(X[0], 0.1, 1, off), lambda: pb.attention(X, Q, Q, off),
                 lambda: pb.attention(Q.float(), Q, Q, off), lambda: pb.attention(Q, Q, Q, off[:1])):
        with pytest.raises(ValueError):
            call()
