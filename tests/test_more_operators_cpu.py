"""Refusals of the operators that joined the first ones around the layers: arguments that are turned down before anything is
launched, with addresses that are never read."""
import ctypes as C

import pytest

from paper_2010_01546_b200 import binding as B
from paper_2010_01546_b200 import build

A = 1 << 20                              # an aligned address


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_library()
    return B._lib()


def table(kind, values):
    return (kind * len(values))(*values)


def test_adamw_refusals(lib):
    inv, shape, ws = B.FW_ERR_INVALID_ARG, B.FW_ERR_SHAPE, B.FW_ERR_WORKSPACE
    D = 1 << 40                          # of the workspace

    def make(sizes=(100, 300), P=(A, 2 * A), copies=None, decay=None, at=D, n=1 << 30, **kw):
        d = B.fw_adamw_desc()
        lib.fw_adamw_desc_default(C.byref(d), len(sizes))
        assert (d.state, d.seed) == (B.FW_F32, 0) and (d.beta1, d.beta2, d.eps) == pytest.approx((0.9, 0.999, 1e-8))
        for k, v in kw.items():
            setattr(d, k, v)
        out = C.c_void_p()
        ns = table(C.c_int64, sizes)
        st = lib.fw_adamw_create(C.byref(d), ns, table(C.c_void_p, P), None if copies is None else table(C.c_void_p, copies),
                                 None if decay is None else table(C.c_float, decay), at, n, None, C.byref(out))
        assert out.value is None or st == B.FW_OK
        return st, lib.fw_adamw_workspace_bytes(C.byref(d), ns)

    for kw in (dict(state=B.FW_BF16), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0),
               dict(eps=float("inf"))):
        assert make(**kw) == (inv, 0), kw
    for kw in (dict(n=1 << 30, sizes=(0, 5)), dict(sizes=(-1, 5)), dict(sizes=((1 << 40) + 1, 5)), dict(sizes=(1 << 40, 5)),
               dict(sizes=(1 << 32, 5), state=B.FW_E4M3)):
        assert make(**kw) == (shape, 0), kw
    for n in (0, -1, 65537):
        d = B.fw_adamw_desc()
        lib.fw_adamw_desc_default(C.byref(d), n)
        assert lib.fw_adamw_workspace_bytes(C.byref(d), table(C.c_int64, (1,))) == 0
    assert lib.fw_adamw_workspace_bytes(None, table(C.c_int64, (1,))) == 0
    need = make()[1]
    assert need >= 2 * 4 * (256 + 512)
    assert make(at=D + 16)[0] == ws and make(n=need - 1)[0] == ws and make(at=None)[0] == inv
    # an address that is none, not of whole elements, twice, or over another's end
    for kw in (dict(P=(A, None)), dict(P=(A, 2 * A + 2)), dict(P=(A, A)), dict(P=(A, A + 396)), dict(P=(A, D + 64)), dict(copies=(None, 3 * A + 1)),
               dict(copies=(3 * A, 3 * A + 198)), dict(copies=(A, None)), dict(decay=(0.0, -0.1)), dict(decay=(float("nan"), 0.0))):
        assert make(**kw)[0] == inv, kw
    assert lib.fw_adamw_create(None, None, None, None, None, A, 1 << 20, None, C.byref(C.c_void_p())) == inv
    assert lib.fw_adamw_step(None, table(C.c_void_p, (A,)), None, 0.1, None, 0.0, None) == inv
    assert lib.fw_adamw_state(None, 0, C.byref(C.c_void_p()), C.byref(C.c_size_t())) == inv
    for f in (lib.fw_adamw_destroy, lib.fw_adamw_sync_status):
        assert f(None) == inv


def test_adamw_looks_at_its_tensors():
    import torch
    with pytest.raises(ValueError, match="CUDA"):
        B.AdamW([torch.zeros(8)])
    with pytest.raises(TypeError):
        B.AdamW([torch.zeros(8, dtype=torch.bfloat16)])
    with pytest.raises(ValueError, match="contiguous"):
        B.AdamW([torch.zeros(8, 8).T[1:]])
    with pytest.raises(TypeError, match="betas"):
        B.AdamW([torch.zeros(8)], betas=(0.9, 0.99))
    with pytest.raises(ValueError, match="expected one for each"):
        B.AdamW([torch.zeros(8)], decay=[0.1, 0.2])
