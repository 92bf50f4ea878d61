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
               dict(y=2 * A), dict(rstd=3 * A), dict(rstd=A), dict(rstd=2 * A + 64)):
        assert norm_forward(lib, d, **kw) == inv, kw
    for kw in (dict(rows=0), dict(rows=-3), dict(rows=1 << 31), dict(ldx=63), dict(ldy=0), dict(ldx=(1 << 30) + 1)):
        assert norm_forward(lib, d, **kw) == shape, kw
    assert norm_forward(lib, ok(y_dtype=B.FW_E4M3)) == inv                  # no place for the scales
    assert norm_forward(lib, ok(y_dtype=B.FW_E4M3), y=A, scale=4 * A) == inv   # bytes over the bf16 rows they are made from
    for kw in (dict(dy=None), dict(s=None), dict(w=None), dict(rstd=None), dict(dx=None), dict(scratch=None), dict(dx=A + 64),
               dict(dx=3 * A), dict(dw=A), dict(dw=3 * A), dict(dw=7 * A + 64), dict(scratch=2 * A), dict(scratch=4 * A), dict(scratch=5 * A)):
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


def distill(lib, d, forward=True, rows=4, Z=A, ldz=104, T=2 * A, I=3 * A, tl=None, w=None, loss=4 * A, stat=5 * A, dZ=6 * A, lddz=104):
    if forward:
        return lib.fw_distill_forward(C.byref(d), Z, rows, ldz, T, I, tl, w, loss, stat, dZ, lddz, None)
    return lib.fw_distill_backward(C.byref(d), Z, rows, ldz, T, I, tl, w, stat, dZ, lddz, None)


def test_distill_refusals(lib):
    inv, shape = B.FW_ERR_INVALID_ARG, B.FW_ERR_SHAPE
    d = B.fw_distill_desc_default(100, 10)
    assert (d.z_dtype, d.t_dtype, d.index_bits, d.tau) == (B.FW_BF16, B.FW_BF16, 32, 1.0)
    assert lib.fw_distill_forward(None, A, 4, 104, 2 * A, 3 * A, None, None, 4 * A, None, None, 0, None) == inv
    for kw in (dict(z_dtype=B.FW_E4M3), dict(t_dtype=5), dict(index_bits=16), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")),
               dict(tau=1e7)):
        assert distill(lib, B.fw_distill_desc_default(100, 10, **kw)) == inv, kw
    for V, K in ((0, 1), (10, 0), (10, 11), ((1 << 20) + 1, 5), (5000, 1025)):
        assert distill(lib, B.fw_distill_desc_default(V, K), ldz=1 << 21, lddz=1 << 21) == shape, (V, K)
    for kw in (dict(Z=None), dict(T=None), dict(I=None), dict(loss=None), dict(Z=A + 1), dict(I=3 * A + 2), dict(T=2 * A + 1),
               dict(loss=4 * A + 2), dict(stat=5 * A + 1), dict(dZ=A + 208), dict(dZ=A, lddz=112), dict(dZ=2 * A), dict(loss=3 * A),
               dict(loss=A), dict(stat=4 * A + 8), dict(w=6 * A), dict(w=4 * A), dict(tl=5 * A), dict(tl=7 * A + 2)):
        assert distill(lib, d, **kw) == inv, kw
    for kw in (dict(rows=0), dict(rows=-1), dict(rows=1 << 28), dict(ldz=99), dict(lddz=99), dict(ldz=(1 << 30) + 1)):
        assert distill(lib, d, **kw) == shape, kw
    for kw in (dict(stat=None), dict(dZ=None), dict(stat=6 * A)):
        assert distill(lib, d, forward=False, **kw) == inv, kw
    assert distill(lib, B.fw_distill_desc_default(100, 10, index_bits=64), I=3 * A + 4) == inv


def test_gated_refusals(lib):
    inv, shape, ws, no = B.FW_ERR_INVALID_ARG, B.FW_ERR_SHAPE, B.FW_ERR_WORKSPACE, B.FW_ERR_UNSUPPORTED

    def make(M=64, N=32, at=A, n=1 << 30, **kw):
        d = B.fw_gated_desc()
        lib.fw_gated_desc_default(C.byref(d), M, N)
        assert (d.x_dtype, d.act, d.grad, d.max_rows) == (B.FW_BF16, B.FW_ACT_SILU, 0, 0)
        for k, v in kw.items():
            setattr(d, k, v)
        out = C.c_void_p()
        st = lib.fw_gated_create(C.byref(d), at, n, None, C.byref(out))
        assert out.value is None or st == B.FW_OK
        return st, lib.fw_gated_workspace_bytes(C.byref(d))

    for kw in (dict(x_dtype=9), dict(act=4), dict(act=-1), dict(grad=2)):
        assert make(**kw) == (inv, 0), kw
    for kw in (dict(M=0), dict(N=0), dict(M=32769), dict(N=40000), dict(grad=1), dict(grad=1, max_rows=-1), dict(grad=1, max_rows=(1 << 26) + 1)):
        assert make(**kw) == (shape, 0), kw
    assert make(x_dtype=B.FW_F32) == (no, 0) and make(x_dtype=B.FW_E4M3, grad=1, max_rows=4) == (no, 0)
    assert make(at=A + 16)[0] == ws and make(n=100)[0] == ws and make(at=None)[0] == inv
    st, n = make(grad=1, max_rows=1000)
    assert n >= 2 * 1000 * 32 * 2 and make(grad=1, max_rows=1000, n=n - 1)[0] == ws
    assert lib.fw_gated_create(None, A, 1 << 20, None, C.byref(C.c_void_p())) == inv
    for f, k in ((lib.fw_gated_destroy, 0), (lib.fw_gated_sync_status, 0)):
        assert f(None) == inv
    assert lib.fw_gated_forward(None, A, 1, 64, None, A, A, 64, None, None, None, None, A, 64, None, None, 0) == inv
    assert lib.fw_gated_backward(None, A, 1, 64, A, 64, A, A, 64, A, A, 64, A, 64, A, A, 0, A, A) == inv


def test_unknown_options_are_refused():
    """A description takes its own fields alone: a misspelt one would leave the default without a word."""
    with pytest.raises(TypeError, match="epsilon"):
        B.fw_norm_desc_default(64, epsilon=1e-3)
    with pytest.raises(TypeError, match="temperature"):
        B.fw_distill_desc_default(100, 10, temperature=2.0)
    with pytest.raises(TypeError, match="activation"):
        B.Gated(64, 32, activation=B.FW_ACT_RELU)
    assert B.fw_norm_desc_default(64, eps=0.5).eps == 0.5


def test_a_block_of_memory_elsewhere_is_refused():
    """The workspace is on the device that the kernels are launched on."""
    with pytest.raises(ValueError, match="CUDA"):
        B.Gated(64, 32, device="cpu")
    import torch
    d = B.fw_norm_desc_default(8)
    x = torch.zeros(2, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="contiguous"):         # its bytes are counted as if they lay next to each other
        B.fw_rmsnorm_backward(d, x, x, torch.ones(8), torch.ones(2), x, dw=torch.zeros(8), scratch=torch.zeros(1 << 16, 2, dtype=torch.uint8)[:, 0])
