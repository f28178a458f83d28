"""Limits and overlaps of the operators of a transformer block (host only), at
their borders: each refusal comes before any HIP call."""
import ctypes

import pytest

pb = pytest.importorskip("paper_2004_14696_amd.binding")

NULL = ctypes.c_void_p(0)
A, B, C, D, E, F, G, H = (ctypes.c_void_p(i << 24) for i in range(1, 9))


@pytest.fixture(scope="module")
def lib():
    return pb.load_library()


@pytest.mark.parametrize("name,kw", [("Y", dict(Y=E)), ("Z", dict(pre=E.value))])
@pytest.mark.parametrize("residual", [None, F.value])
def test_group_linear_refuses_its_bias_as_an_output(lib, name, kw, residual):
    shape = pb.GroupShape(form=pb.DBW_GROUP_FORWARD, dtype=pb.DBW_BF16, out_dtype=pb.DBW_F32, n=4, d=64, C=32, T=100, ld_d=64,
                          ld_C=32, ld_W=32, st_W=64 * 32)
    pre = kw.get("pre", G.value)
    e = pb.LinearEpilogue(activation=pb.DBW_ACT_GELU, bias=E.value, st_bias=32, residual=residual, ld_residual=32, pre=pre,
                          ld_pre=32)
    call = lib.dbw_group_linear(ctypes.byref(shape), ctypes.byref(e), A, B, C, kw.get("Y", D), H, 1 << 50, NULL)
    assert call == pb.DBW_EINVAL and b"overlap" in lib.dbw_last_error(None)


def _linear(lib, **kw):
    shape = pb.GroupShape(form=pb.DBW_GROUP_FORWARD, dtype=pb.DBW_BF16, out_dtype=pb.DBW_BF16, n=4, d=64, C=32, T=100, ld_d=64,
                          ld_C=32, ld_W=32, st_W=64 * 32)
    e = pb.LinearEpilogue(activation=pb.DBW_ACT_GELU, bias=E.value, st_bias=32, pre=kw.get("pre", G).value, ld_pre=32)
    return lib.dbw_group_linear(ctypes.byref(shape), ctypes.byref(e), A, B, C, kw.get("Y", D), H, 1 << 50, NULL)


def _norm_grad(lib, dX=E, dg=F, db=G):
    return lib.dbw_layer_norm_grad(4, 100, 64, pb.DBW_BF16, A, B, 64, C, 64, D, 1e-5, dX, 64, dg, 64, db, 64, H, 1 << 50, NULL)


def _linear_grad(lib, dZ=D, db=E):
    return lib.dbw_linear_grad(4, 100, 64, pb.DBW_BF16, pb.DBW_ACT_SILU, A, B, 64, C, 64, dZ, 64, db, 64, H, 1 << 50, NULL)


def _attention(lib, grad=False, **kw):
    s = pb.AttentionShape(dtype=pb.DBW_BF16, n=4, heads=4, kv_heads=2, D=64, T=100, scale=0.125)
    named = dict(zip(("Q", "K", "V", "O", "dO", "dQ", "dK", "dV"), (i << 32 for i in range(1, 9)))) | kw
    p = {k: ctypes.byref(pb.Heads(data=v, token=(2 if k in ("K", "V", "dK", "dV") else 4) * 64, head=64))
         for k, v in named.items() if k != "lse"}
    lse = ctypes.c_void_p(kw.get("lse", 9 << 32))
    if not grad:
        return lib.dbw_attention(ctypes.byref(s), A, p["Q"], p["K"], p["V"], p["O"], lse, NULL)
    return lib.dbw_attention_grad(ctypes.byref(s), A, p["dO"], p["Q"], p["K"], p["V"], p["O"], lse, p["dQ"], p["dK"], p["dV"],
                                  H, 1 << 50, NULL)


OFFSETS_AS_OUTPUT = {
    "layer_norm Y": lambda lib: lib.dbw_layer_norm(4, 100, 64, pb.DBW_BF16, A, B, 64, C, D, 1e-5, A, 64, NULL),
    "layer_norm_grad dX": lambda lib: _norm_grad(lib, dX=A),
    "layer_norm_grad dgamma": lambda lib: _norm_grad(lib, dg=A),
    "layer_norm_grad dbeta": lambda lib: _norm_grad(lib, db=A),
    "group_linear Y": lambda lib: _linear(lib, Y=A),
    "group_linear pre": lambda lib: _linear(lib, pre=A),
    "linear_grad dZ": lambda lib: _linear_grad(lib, dZ=A),
    "linear_grad dbias": lambda lib: _linear_grad(lib, db=A),
    "dropout Y": lambda lib: lib.dbw_dropout(4, 100, 64, pb.DBW_BF16, A, B, 64, 0.1, 1, C, D, 64, A, 64, NULL),
    "attention O": lambda lib: _attention(lib, O=A.value),
    "attention lse": lambda lib: _attention(lib, lse=A.value),
    "attention_grad dQ": lambda lib: _attention(lib, grad=True, dQ=A.value),
    "attention_grad dK": lambda lib: _attention(lib, grad=True, dK=A.value),
    "attention_grad dV": lambda lib: _attention(lib, grad=True, dV=A.value),
}


@pytest.mark.parametrize("name", OFFSETS_AS_OUTPUT)
def test_offsets_are_refused_as_an_output(lib, name):
    assert OFFSETS_AS_OUTPUT[name](lib) == pb.DBW_EINVAL
    assert b"overlap" in lib.dbw_last_error(None)


@pytest.mark.parametrize("n,T,heads", [(65536, 0, 128), (65536, 100, 128), (1, ((1 << 23) // 8 - 1) * 64, 8),
                                       (8192, 64 * 1023 + 63, 1024), (65536, 65536 * 64, 64)])
def test_attention_tiles_reach_the_stated_limit(lib, n, T, heads):
    """(floor(T / 64) + n) heads: 2^23 is refused, and what lies just below is not."""
    size = (T // 64 + n) * heads
    work = lambda n: lib.dbw_attention_workspace(ctypes.byref(pb.AttentionShape(                            # noqa: E731
        dtype=pb.DBW_BF16, n=n, heads=heads, kv_heads=heads, D=64, T=T, scale=0.125)))
    at_limit = n if size >= 1 << 23 else n + ((1 << 23) - size + heads - 1) // heads
    if at_limit <= 65536:
        assert work(at_limit) == -1
    below = ((1 << 23) - 1) // heads - T // 64
    if 1 <= below <= 65536:
        assert work(below) >= 0
