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


def sandwich_forward(lib, d, rows=4, o=A, x=2 * A, w1=3 * A, gate=None, w2=4 * A, h=5 * A, y=6 * A, scale=None, rstd=7 * A, ld=64, ldh=64, ldy=64):
    return lib.fw_sandwich_forward(C.byref(d) if d is not None else None, rows, o, ld, x, 64, w1, gate, w2, h, ldh, y, ldy, scale, rstd, None)


def sandwich_backward(lib, d, rows=4, dy=A, dh=2 * A, o=3 * A, h=4 * A, w1=5 * A, gate=6 * A, w2=7 * A, rstd=8 * A, dx=9 * A, d_o=10 * A, dw1=11 * A,
                      dw2=12 * A, dgate=13 * A, scratch=14 * A, n=1 << 24, lddx=64):
    return lib.fw_sandwich_backward(C.byref(d), rows, dy, 64, dh, 64, o, 64, h, 64, w1, gate, w2, rstd, dx, lddx, d_o, 64, dw1, dw2, dgate, scratch, n, None)


def test_sandwich_refusals(lib):
    inv, shape, ws = B.FW_ERR_INVALID_ARG, B.FW_ERR_SHAPE, B.FW_ERR_WORKSPACE
    ok = lambda **kw: B.fw_sandwich_desc_default(64, **kw)  # noqa: E731
    d = ok()
    assert (d.dtype, d.y_dtype, d.post, d.eps, d.alpha) == (B.FW_BF16, B.FW_BF16, 1, pytest.approx(1e-6), 1.0)
    assert sandwich_forward(lib, None) == inv
    for bad in (dict(dtype=2), dict(y_dtype=B.FW_F32), dict(post=2), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(alpha=float("nan")), dict(alpha=float("inf"))):
        assert sandwich_forward(lib, ok(**bad)) == inv and sandwich_backward(lib, ok(**bad)) == inv, bad
        assert B.fw_sandwich_scratch_bytes(ok(**bad)) == 0
    for M in (0, -1, 16385):
        assert sandwich_forward(lib, B.fw_sandwich_desc_default(M)) == shape
    for kw in (dict(o=None), dict(x=None), dict(w2=None), dict(h=None), dict(y=None), dict(scale=8 * A), dict(o=A + 1), dict(w1=3 * A + 2), dict(gate=8 * A + 1),
               dict(rstd=7 * A + 2), dict(h=6 * A + 64), dict(h=A + 64), dict(h=A, ldh=72), dict(y=2 * A + 128), dict(y=4 * A), dict(h=3 * A), dict(rstd=A),
               dict(rstd=4 * A), dict(gate=5 * A), dict(rstd=6 * A)):
        assert sandwich_forward(lib, d, **kw) == inv, kw
    for kw in (dict(rows=0), dict(rows=1 << 31), dict(ld=63), dict(ldy=0), dict(ldh=(1 << 30) + 1)):
        assert sandwich_forward(lib, d, **kw) == shape, kw
    assert sandwich_forward(lib, ok(y_dtype=B.FW_E4M3)) == inv
    assert sandwich_forward(lib, ok(y_dtype=B.FW_E4M3), y=A, scale=8 * A) == inv          # bytes over the bf16 rows they are made from
    for kw in (dict(dy=None), dict(o=None), dict(h=None), dict(w2=None), dict(rstd=None), dict(dx=None), dict(d_o=None), dict(scratch=None), dict(dx=3 * A),
               dict(dx=10 * A), dict(dx=A + 64), dict(dx=A, lddx=72), dict(dw1=A), dict(dw1=12 * A + 64), dict(dw2=14 * A + 512), dict(dgate=8 * A), dict(dgate=6 * A),
               dict(scratch=4 * A), dict(scratch=9 * A), dict(d_o=7 * A)):
        assert sandwich_backward(lib, d, **kw) == inv, kw
    assert sandwich_backward(lib, d, rows=0) == shape and sandwich_backward(lib, d, lddx=60) == shape
    assert sandwich_backward(lib, d, n=100) == ws and sandwich_backward(lib, d, scratch=14 * A + 8) == ws
    with pytest.raises(TypeError, match="beta"):
        ok(beta=1.0)


def logprob(lib, d, what="fwd", rows=4, Z=A, ldz=104, id=2 * A, logp=3 * A, stat=4 * A, dlogp=5 * A, dZ=6 * A, lddz=104):
    if what == "fwd":
        return lib.fw_logprob_forward(C.byref(d), Z, rows, ldz, id, logp, stat, None)
    return lib.fw_logprob_backward(C.byref(d), Z, rows, ldz, id, stat, dlogp, dZ, lddz, None)


def policy(lib, d, p, rows=4, Z=A, ldz=104, id=2 * A, old=7 * A, ref=None, adv=8 * A, w=None, loss=9 * A, logp=3 * A, stat=4 * A, dlogp=5 * A,
           dZ=6 * A, lddz=104):
    return lib.fw_policy_forward(C.byref(d), C.byref(p) if p is not None else None, Z, rows, ldz, id, old, ref, adv, w, loss, logp, stat, dlogp,
                                 dZ, lddz, None)


def test_logprob_and_policy_refusals(lib):
    inv, shape = B.FW_ERR_INVALID_ARG, B.FW_ERR_SHAPE
    d, p = B.fw_logprob_desc_default(100), B.fw_policy_desc_default()
    assert (d.z_dtype, d.index_bits, d.tau) == (B.FW_BF16, 32, 1.0) and (p.clip_low, p.clip_high, p.kl) == pytest.approx((0.2, 0.2, 0.0))
    calls = (lambda d, **kw: logprob(lib, d, **kw), lambda d, **kw: logprob(lib, d, "bwd", **kw), lambda d, **kw: policy(lib, d, p, **kw))
    for call in calls:
        for kw in (dict(z_dtype=B.FW_E4M3), dict(index_bits=16), dict(tau=0.0), dict(tau=float("nan")), dict(tau=1e7)):
            assert call(B.fw_logprob_desc_default(100, **kw)) == inv, kw
        for V in (0, -1, (1 << 20) + 1):
            assert call(B.fw_logprob_desc_default(V), ldz=1 << 21) == shape, V
        for kw in (dict(Z=None), dict(id=None), dict(Z=A + 1), dict(id=2 * A + 2), dict(stat=4 * A + 2)):
            assert call(d, **kw) == inv, kw
        for kw in (dict(rows=0), dict(rows=-1), dict(rows=1 << 28), dict(ldz=99), dict(ldz=(1 << 30) + 1)):
            assert call(d, **kw) == shape, kw
        assert call(B.fw_logprob_desc_default(100, index_bits=64), id=2 * A + 4) == inv
    assert lib.fw_logprob_forward(None, A, 4, 104, 2 * A, 3 * A, None, None) == inv
    for kw in (dict(logp=None), dict(logp=A), dict(logp=2 * A + 8), dict(stat=3 * A + 8)):
        assert logprob(lib, d, **kw) == inv, kw
    for kw in (dict(stat=None), dict(dlogp=None), dict(dZ=None), dict(dZ=A + 208), dict(dZ=A, lddz=112), dict(dZ=2 * A), dict(dZ=5 * A), dict(dZ=4 * A)):
        assert logprob(lib, d, "bwd", **kw) == inv, kw
    assert logprob(lib, d, "bwd", lddz=99) == shape and policy(lib, d, p, lddz=99) == shape
    for kw in (dict(old=None), dict(adv=None), dict(loss=None), dict(loss=7 * A), dict(w=5 * A), dict(logp=9 * A + 8), dict(dlogp=8 * A), dict(old=7 * A + 1),
               dict(dZ=A, lddz=112), dict(dZ=8 * A), dict(ref=9 * A)):
        assert policy(lib, d, p, **kw) == inv, kw
    for kw in (dict(clip_low=-0.1), dict(clip_low=1.0), dict(clip_high=-0.1), dict(clip_high=float("nan")), dict(kl=float("inf")), dict(kl=0.1)):
        assert policy(lib, d, B.fw_policy_desc_default(**kw)) == inv, kw                # (kl without logp_ref)
    assert policy(lib, d, None) == inv


def test_preference_refusals(lib):
    inv, shape = B.FW_ERR_INVALID_ARG, B.FW_ERR_SHAPE

    def call(d=None, p=None, logp=A, rows=100, id=2 * A, seq=3 * A, pairs=4, ref=None, w=None, loss=4 * A, sums=5 * A, dlogp=6 * A):
        d, p = d or B.fw_logprob_desc_default(50), p or B.fw_preference_desc_default()
        return lib.fw_preference_loss(C.byref(d), C.byref(p), logp, rows, id, seq, pairs, ref, w, loss, sums, dlogp, None)

    p = B.fw_preference_desc_default()
    assert (p.beta, p.margin, p.smooth, p.mean) == (pytest.approx(0.1), 0.0, 0.0, 0)
    for kw in (dict(beta=0.0), dict(beta=float("inf")), dict(margin=float("nan")), dict(smooth=1.0), dict(smooth=-0.1), dict(mean=2)):
        assert call(p=B.fw_preference_desc_default(**kw)) == inv, kw
    for kw in (dict(logp=None), dict(seq=None), dict(loss=None), dict(seq=3 * A + 2), dict(loss=A), dict(dlogp=A), dict(sums=4 * A + 8), dict(ref=5 * A),
               dict(w=4 * A), dict(dlogp=2 * A), dict(id=2 * A + 1), dict(loss=3 * A + 32)):
        assert call(**kw) == inv, kw
    for kw in (dict(rows=0), dict(rows=1 << 28), dict(pairs=0), dict(pairs=(1 << 24) + 1)):
        assert call(**kw) == shape, kw
    assert call(d=B.fw_logprob_desc_default(50, index_bits=8)) == inv and call(d=B.fw_logprob_desc_default(0)) == shape
    assert lib.fw_preference_loss(None, C.byref(p), A, 4, None, A, 1, None, None, A, None, None, None) == inv


def test_tensors_of_the_losses_are_looked_at():
    import torch
    d = B.fw_logprob_desc_default(8)
    Z, id, v = torch.zeros(2, 8, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    with pytest.raises(ValueError, match="CUDA"):
        B.fw_logprob_forward(d, Z, id, v)
    with pytest.raises(TypeError):
        B.fw_logprob_forward(d, Z.float(), id, v)
    with pytest.raises(ValueError, match="expected"):
        B.fw_logprob_forward(d, Z[:, :7], id, v)
    with pytest.raises(TypeError, match="temperature"):
        B.fw_logprob_desc_default(8, temperature=2.0)
    with pytest.raises(TypeError, match="clip"):
        B.fw_policy_desc_default(clip=0.2)
    with pytest.raises(TypeError, match="gamma"):
        B.fw_preference_desc_default(gamma=0.2)


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


@pytest.mark.parametrize("kind", ["layer", "gated", "adamw"])
@pytest.mark.parametrize("stream", [0, 0x5000])
def test_workspaces_are_of_the_stream_they_are_used_on(monkeypatch, kind, stream):
    """The memory comes from the allocator while the object's own stream is the current one: of another stream's memory the owner before
    may have work pending, which would write over states and addresses that this stream has put there."""
    import contextlib

    import torch

    class Memory:
        is_cuda = True

        def data_ptr(self):
            return 1 << 40

        def get_device(self):
            return -1

        def record_stream(self, s):
            pass

    current, taken = ["current"], []

    @contextlib.contextmanager
    def entered(s):
        current.append(s)
        yield
        current.pop()

    monkeypatch.setattr(torch, "empty", lambda *a, **kw: taken.append(current[-1]) or Memory())
    monkeypatch.setattr(torch.cuda, "stream", entered)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda s: s)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: 0)
    monkeypatch.setattr(B, "_here", lambda: -1)

    class Lib:
        def __getattr__(self, name):
            real = getattr(B_lib, name)
            return (lambda *a: 0) if name.endswith(("_create", "_destroy")) else real

    B_lib = B._lib()
    monkeypatch.setattr(B, "_lib", Lib)
    if kind == "layer":
        monkeypatch.setattr(B, "fw_layer_create", lambda *a: 0)
        B.Layer(64, 32, stream=stream)
    elif kind == "gated":
        B.Gated(64, 32, stream=stream)
    else:
        B.AdamW([torch.zeros(8)], stream=stream)
    assert taken == [stream]
