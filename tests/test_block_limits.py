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
