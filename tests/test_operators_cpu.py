"""Refusals of the operators around the layers: arguments that are turned down before anything is launched, with addresses
that are never read."""
import ctypes as C

import pytest

from paper_2010_01546_b200 import binding as B
from paper_2010_01546_b200 import build

A = 1 << 20                              # an aligned address


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_library()
    return B._lib()


def norm_forward(lib, d, rows=4, x=A, ldx=64, res=None, ldr=0, w=2 * A, s=None, lds=0, y=3 * A, ldy=64, scale=None, rstd=None):
    return lib.fw_rmsnorm_forward(C.byref(d) if d is not None else None, rows, x, ldx, res, ldr, w, s, lds, y, ldy, scale, rstd, None)


def norm_backward(lib, d, rows=4, dy=A, s=2 * A, ds=None, w=3 * A, rstd=4 * A, dx=5 * A, lddx=64, dw=6 * A, scratch=7 * A, n=1 << 24):
    return lib.fw_rmsnorm_backward(C.byref(d), rows, dy, 64, s, 64, ds, 64, w, rstd, dx, lddx, dw, scratch, n, None)


def test_norm_refusals(lib):
    ok = lambda **kw: B.fw_norm_desc_default(64, **kw)  # noqa: E731
    d = ok()
    assert (d.dtype, d.y_dtype, d.eps) == (B.FW_BF16, B.FW_BF16, pytest.approx(1e-6))
    inv, shape, ws = B.FW_ERR_INVALID_ARG, B.FW_ERR_SHAPE, B.FW_ERR_WORKSPACE
    assert norm_forward(lib, None) == inv
    for bad in (dict(dtype=2), dict(dtype=7), dict(y_dtype=B.FW_F32), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf"))):
        assert norm_forward(lib, ok(**bad)) == inv, bad
        assert B.fw_rmsnorm_scratch_bytes(ok(**bad)) == 0
    for M in (0, -1, 16385):
        assert norm_forward(lib, B.fw_norm_desc_default(M)) == shape
    for kw in (dict(x=None), dict(w=None), dict(y=None), dict(s=4 * A, lds=64), dict(scale=4 * A), dict(x=A + 1), dict(w=2 * A + 2),
               dict(rstd=A + 2), dict(y=A + 2), dict(y=A, ldy=72), dict(res=4 * A, ldr=64, s=3 * A, lds=64),
               dict(y=2 * A), dict(rstd=3 * A)):
        assert norm_forward(lib, d, **kw) == inv, kw
    for kw in (dict(rows=0), dict(rows=-3), dict(rows=1 << 31), dict(ldx=63), dict(ldy=0), dict(ldx=(1 << 30) + 1)):
        assert norm_forward(lib, d, **kw) == shape, kw
    assert norm_forward(lib, ok(y_dtype=B.FW_E4M3)) == inv                  # no place for the scales
    assert norm_forward(lib, ok(y_dtype=B.FW_E4M3), y=A, scale=4 * A) == inv   # bytes over the bf16 rows they are made from
    for kw in (dict(dy=None), dict(s=None), dict(w=None), dict(rstd=None), dict(dx=None), dict(scratch=None), dict(dx=A + 64),
               dict(dx=3 * A)):
        assert norm_backward(lib, d, **kw) == inv, kw
    assert norm_backward(lib, d, rows=0) == shape and norm_backward(lib, d, lddx=60) == shape
    assert norm_backward(lib, d, n=100) == ws and norm_backward(lib, d, scratch=7 * A + 8) == ws


def test_tensors_are_looked_at():
    import torch
    d = B.fw_norm_desc_default(8)
    x, w = torch.zeros(2, 8, dtype=torch.bfloat16), torch.ones(8)
    with pytest.raises(ValueError, match="CUDA"):
        B.fw_rmsnorm_forward(d, x, w, x)
    with pytest.raises(TypeError):
        B.fw_rmsnorm_forward(d, x.float(), w, x)
    with pytest.raises(ValueError, match="expected"):
        B.fw_rmsnorm_forward(d, x[:, :7], w, x)
    with pytest.raises(ValueError, match="next to each other"):
        B.fw_rmsnorm_forward(d, torch.zeros(8, 8, dtype=torch.bfloat16).T, w, x)
