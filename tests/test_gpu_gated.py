"""Gated feed-forward block against its definition in 64 bits.

Two kinds of inputs.  Small whole numbers (and halves): every product and sum is exact in fp32, so with ReLU the outputs are
equal to the reference bit for bit at every size, which shows a lost or doubled element anywhere.  Real values: bounds
from the arithmetic (u = 2^-24).  A tensor-core sum of K products is off by at most 4 (K / 16 + 16) u of the products'
magnitudes (each addition into the accumulator truncates at 2^-23 of it); an activation by (2^-20 + 4 u (1 + a^2)) of its value and
the error of its argument times 1.13, the largest slope; bf16 results by half a step, 2^-8.
"""
import pytest
import torch

from optest_util import F64, HALF, U, captured, gen, matrix, put, surround_kept

pytestmark = pytest.mark.gpu

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
# rows, M, N
SIZES = [(1, 1, 1), (1, 64, 128), (2, 7, 300), (3, 100, 8), (17, 1000, 257), (64, 72, 513), (128, 256, 128), (129, 65, 129),
         (255, 300, 1367), (256, 128, 256), (300, 520, 640), (513, 129, 1000), (1000, 2304, 100), (33, 4000, 2050),
         # products that fill the chip: forward; the weight gradients alone; all of them
         (2600, 72, 1367), (200, 1400, 1700), (4000, 1100, 2050), (3000, 1024, 2304)]


@pytest.fixture(scope="module")
def B():
    from paper_2010_01546_b200 import binding, build
    build.build_library()
    return binding


def whole(g, rows, cols, most=2):
    return torch.randint(-most, most + 1, (rows, cols), generator=g, device="cuda").float()


def block(B, M, N, rows=0, **kw):
    return B.Gated(M, N, rows, **kw)


def bf(rows, cols, **kw):
    return matrix(rows, cols, BF16, pad=kw.pop("pad", None), **kw)


@pytest.mark.parametrize("rows,M,N", SIZES)
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_forward_exact(B, rows, M, N, kind):
    g = gen(rows + M + N)
    t = BF16 if kind == "bf16" else E4M3
    pad = 16 if M % 16 == 0 else None                         # rows further apart than they are long
    X, Wg, Wu = (put(whole(g, r, M), t, pad=pad) for r in (rows, N, N))
    bg, bu = (whole(g, 1, N, 9).flatten() / 2 for _ in range(2))
    scales = {}
    xs = ws = us = 1.0
    if kind == "e4m3":                                        # powers of two
        xs, ws, us = (2.0 ** whole(g, 1, n, 2).flatten() for n in (rows, N, N))
        scales = dict(x_scale=xs, wg_scale=ws, wu_scale=us)
        xs = xs[:, None].to(F64)
    a = X.to(F64) @ Wg.to(F64).T * xs * ws
    b = X.to(F64) @ Wu.to(F64).T * xs * us
    blk = block(B, M, N, x_dtype=B.FW_BF16 if kind == "bf16" else B.FW_E4M3, act=B.FW_ACT_RELU)
    for bias in (False, True):
        if bias:
            a, b = a + bg.to(F64), b + bu.to(F64)
            scales.update(bg=bg, bu=bu)
        H, Zg, Zu = (bf(rows, N) for _ in range(3))
        blk.forward(X, Wg, Wu, H, Zg, Zu, **scales)
        assert torch.equal(Zg, a.float().to(BF16)) and torch.equal(Zu, b.float().to(BF16))
        assert torch.equal(H, (a.float().clamp(min=0) * b.float()).to(BF16))
        H2 = bf(rows, N, shift=8)
        blk.forward(X, Wg, Wu, H2, **scales)                  # without the projections
        assert torch.equal(H2, H)
        assert all(surround_kept(v) for v in (H, Zg, Zu, H2))
    assert blk.sync_status() == B.FW_OK


@pytest.mark.parametrize("rows,M,N", SIZES)
@pytest.mark.parametrize("dw", [torch.float32, BF16])
def test_backward_exact(B, rows, M, N, dw):
    g = gen(rows + 2 * M + N)
    X, Wg, Wu, dH, Zg = (put(whole(g, r, c), BF16, pad=None) for r, c in ((rows, M), (N, M), (N, M), (rows, N), (rows, N)))
    Zu = put(whole(g, rows, N, 4) / 2, BF16, pad=None)
    blk = block(B, M, N, rows + 5, act=B.FW_ACT_RELU, grad=1)
    dX = bf(rows, M)
    dWg, dWu = (torch.full((N, M), float("nan"), dtype=dw, device="cuda") for _ in range(2))
    dbg, dbu = (torch.full((N,), float("nan"), device="cuda") for _ in range(2))
    blk.backward(dH, X, Wg, Wu, Zg, Zu, dX, dWg, dWu, dbg, dbu)
    da = dH.to(F64) * Zu.to(F64) * (Zg.to(F64) > 0)
    db = dH.to(F64) * Zg.to(F64).clamp(min=0)
    assert torch.equal(dX, (da @ Wg.to(F64) + db @ Wu.to(F64)).float().to(BF16)) and surround_kept(dX)
    assert torch.equal(dWg, (da.T @ X.to(F64)).float().to(dw)) and torch.equal(dWu, (db.T @ X.to(F64)).float().to(dw))
    assert torch.equal(dbg.to(F64), da.sum(0)) and torch.equal(dbu.to(F64), db.sum(0))
    # parts of it by themselves
    dX2 = bf(rows, M)
    blk.backward(dH, X, Wg, Wu, Zg, Zu, dX=dX2)
    assert torch.equal(dX2, dX)
    w2 = [torch.empty_like(dWg) for _ in range(2)]
    blk.backward(dH, X, Wg, Wu, Zg, Zu, dWg=w2[0], dWu=w2[1])
    assert torch.equal(w2[0], dWg) and torch.equal(w2[1], dWu)
    b2 = [torch.empty_like(dbg) for _ in range(2)]
    blk.backward(dH, X, Wg, Wu, Zg, Zu, dbg=b2[0], dbu=b2[1])
    assert torch.equal(b2[0], dbg) and torch.equal(b2[1], dbu)
    assert blk.sync_status() == B.FW_OK


def act64(name, a):
    a = a.detach().requires_grad_(True)
    f = {"silu": lambda: a * torch.sigmoid(a), "gelu": lambda: a * torch.special.ndtr(a),
         "gelu_tanh": lambda: 0.5 * a * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (a + 0.044715 * a ** 3))),
         "relu": lambda: a.clamp(min=0) + 0 * a}[name]()
    (df,) = torch.autograd.grad(f.sum(), a)
    if name == "relu":
        df = (a > 0).to(F64)
    return f.detach(), df.detach()


ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


@pytest.mark.parametrize("rows,M,N", [(1, 520, 300), (40, 1000, 257), (300, 333, 700), (513, 2304, 512)])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_forward_values(B, rows, M, N, act, kind):
    g = gen(M + ACTS.index(act))
    X, Wg, Wu = (torch.randn(r, M, generator=g, device="cuda") * s for r, s in ((rows, 1.0), (N, 2 * M ** -0.5), (N, M ** -0.5)))
    bg, bu = (torch.randn(N, generator=g, device="cuda") for _ in range(2))
    scales = {}
    if kind == "e4m3":
        q, c = zip(*(((v / (s := v.abs().amax(1, keepdim=True) / 448)), s.flatten()) for v in (X, Wg, Wu)))
        X, Wg, Wu = (put(v, E4M3, pad=None) for v in q)
        scales = dict(x_scale=c[0].contiguous(), wg_scale=c[1].contiguous(), wu_scale=c[2].contiguous())
        x64, g64, u64 = (v.to(F64) * s.to(F64)[:, None] for v, s in zip((X, Wg, Wu), c))
    else:
        X, Wg, Wu = (put(v, BF16, pad=None) for v in (X, Wg, Wu))
        x64, g64, u64 = X.to(F64), Wg.to(F64), Wu.to(F64)
    H, Zg, Zu = (bf(rows, N) for _ in range(3))
    blk = block(B, M, N, x_dtype=B.FW_E4M3 if kind == "e4m3" else B.FW_BF16, act=ACTS.index(act))
    blk.forward(X, Wg, Wu, H, Zg, Zu, bg=bg, bu=bu, **scales)
    a, b = x64 @ g64.T + bg.to(F64), x64 @ u64.T + bu.to(F64)
    c = 4 * (M / 16 + 16) * U
    ea, eb = (c * (x64.abs() @ w.abs().T) + 4 * U * (z.abs() + bias.to(F64).abs()) for w, z, bias in ((g64, a, bg), (u64, b, bu)))
    for got, want, e in ((Zg, a, ea), (Zu, b, eb)):
        assert bool(((got.to(F64) - want).abs() <= e + 2.0 ** -8 * (want.abs() + e)).all())
    f, _ = act64(act, a)
    ef = 1.13 * ea + f.abs() * (2.0 ** -20 + 4 * U * (1 + a * a)) + 1e-37
    e = ef * (b.abs() + eb) + f.abs() * eb + 2 * U * (f * b).abs()
    assert bool(((H.to(F64) - f * b).abs() <= e + 2.0 ** -8 * ((f * b).abs() + e)).all())


@pytest.mark.parametrize("act", ACTS)
def test_backward_values(B, act):
    """da and db are held in bf16 for the products: each term is off by 2^-8 of itself at most."""
    rows, M, N = 300, 333, 700
    g = gen(7 + ACTS.index(act))
    X, Wg, Wu = (put(torch.randn(r, M, generator=g, device="cuda") * s, BF16, pad=None) for r, s in ((rows, 1.0), (N, 0.1), (N, 0.1)))
    dH, Zg, Zu = (put(torch.randn(rows, N, generator=g, device="cuda") * s, BF16, pad=None) for s in (1.0, 3.0, 1.0))
    blk = block(B, M, N, rows, act=ACTS.index(act), grad=1)
    dX, dWg, dWu = bf(rows, M), torch.empty(N, M, device="cuda"), torch.empty(N, M, device="cuda")
    dbg, dbu = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    blk.backward(dH, X, Wg, Wu, Zg, Zu, dX, dWg, dWu, dbg, dbu)
    a = Zg.to(F64)
    f, df = act64(act, a)
    d = dH.to(F64)
    da, db = d * Zu.to(F64) * df, d * f
    # the derivative's terms reach 1.13 + |a| / 2 where they cancel
    ea = (d * Zu.to(F64)).abs() * (2.0 ** -20 + 4 * U * (1 + a * a)) * 2
    eb = db.abs() * (2.0 ** -20 + 4 * U * (1 + a * a)) + 1e-37
    for got, want, e in ((dbg, da, ea), (dbu, db, eb)):
        assert bool(((got.to(F64) - want.sum(0)).abs() <= e.sum(0) + 400 * U * want.abs().sum(0)).all())
    ha, hb = ea + 2.0 ** -8 * (da.abs() + ea), eb + 2.0 ** -8 * (db.abs() + eb)
    c = lambda k: 4 * (k / 16 + 16) * U  # noqa: E731
    for got, dd, h in ((dWg, da, ha), (dWu, db, hb)):
        x = X.to(F64)
        want, e = dd.T @ x, h.T @ x.abs() + c(rows) * ((dd.abs() + h).T @ x.abs())
        off = (got.to(F64) - want).abs()
        assert bool((off <= e).all())
        # roundings are not all of one sign: in the mean they are a small part of that
        assert float(off.norm() / want.norm()) <= 2.0 ** -8
    wg, wu = Wg.to(F64), Wu.to(F64)
    want = da @ wg + db @ wu
    e = ha @ wg.abs() + hb @ wu.abs() + c(2 * N) * ((da.abs() + ha) @ wg.abs() + (db.abs() + hb) @ wu.abs())
    off = (dX.to(F64) - want).abs()
    assert bool((off <= e + 2.0 ** -8 * (want.abs() + e)).all())
    assert float(off.norm() / want.norm()) <= 2 * 2.0 ** -8


def test_gradient_against_differences(B):
    """Central differences of the definition in 64 bits; the call's values are off by bf16 roundings of da, db and of the result:
    3 x 2^-8 of the terms, taken as 2^-6 of the largest."""
    rows, M, N, h = 3, 8, 5, 1e-6
    g = gen(5)
    X, Wg, Wu, c = (put(torch.randn(*s, generator=g, device="cuda"), BF16, pad=None) for s in ((rows, M), (N, M), (N, M), (rows, N)))
    bg, bu = (torch.randn(N, generator=g, device="cuda") for _ in range(2))
    v = [t.to(F64).contiguous() for t in (X, Wg, Wu, bg, bu)]
    loss = lambda: float((c.to(F64) * torch.nn.functional.silu(v[0] @ v[1].T + v[3]) * (v[0] @ v[2].T + v[4])).sum())  # noqa: E731
    H, Zg, Zu, dX = bf(rows, N), bf(rows, N), bf(rows, N), bf(rows, M)
    blk = block(B, M, N, rows, grad=1)
    blk.forward(X, Wg, Wu, H, Zg, Zu, bg=bg, bu=bu)
    dWg, dWu, dbg, dbu = torch.empty(N, M, device="cuda"), torch.empty(N, M, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    blk.backward(c, X, Wg, Wu, Zg, Zu, dX, dWg, dWu, dbg, dbu)
    for at, got in zip(v, (dX, dWg, dWu, dbg, dbu)):
        num = torch.empty_like(at)
        for i in range(at.numel()):
            x = float(at.view(-1)[i])
            at.view(-1)[i] = x + h
            up = loss()
            at.view(-1)[i] = x - h
            num.view(-1)[i] = (up - loss()) / (2 * h)
            at.view(-1)[i] = x
        assert float((got.to(F64) - num).abs().max()) <= 2.0 ** -6 * float(num.abs().max())


def test_nan_stays_in_its_row(B):
    for rows in (5, 400):
        g = gen(rows)
        X, Wg, Wu = (put(whole(g, r, 200), BF16, pad=None) for r in (rows, 130, 130))
        blk = block(B, 200, 130, act=B.FW_ACT_RELU)
        H, H2 = bf(rows, 130), bf(rows, 130)
        blk.forward(X, Wg, Wu, H)
        X[1, 3] = float("nan")
        X[3, 0] = float("inf")
        Wg[:, 0] = 1.0
        blk.forward(X, Wg, Wu, H2)
        assert bool(torch.isnan(H2[1]).all()) and not bool(torch.isfinite(H2[3].float()).all())
        X[1, 3] = X[3, 0] = 0
        blk.forward(X, Wg, Wu, H)
        keep = [r for r in range(rows) if r not in (1, 3)]
        assert torch.equal(H[keep], H2[keep])


def test_streams_graphs_and_repeats(B):
    """Two blocks on two streams at once, each captured and replayed; every replay gives the bits of the plain calls."""
    jobs = []
    for k, (rows, M, N) in enumerate(((300, 520, 1000), (70, 1000, 264), (4, 512, 2048))):
        g = gen(40 + k)
        X, Wg, Wu = (put(torch.randn(r, M, generator=g, device="cuda"), BF16, pad=None) for r in (rows, N, N))
        dH = put(torch.randn(rows, N, generator=g, device="cuda"), BF16, pad=None)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        outs = [bf(rows, N), bf(rows, N), bf(rows, N), bf(rows, M), torch.empty(N, M, device="cuda"), torch.empty(N, M, device="cuda"),
                torch.empty(N, device="cuda"), torch.empty(N, device="cuda")]
        blk = B.Gated(M, N, rows, grad=1, stream=s.cuda_stream)

        def call(blk=blk, X=X, Wg=Wg, Wu=Wu, dH=dH, o=outs):
            blk.forward(X, Wg, Wu, o[0], o[1], o[2])
            blk.backward(dH, X, Wg, Wu, o[1], o[2], o[3], o[4], o[5], o[6], o[7])

        jobs.append((s, call, outs, X, blk))
    torch.cuda.synchronize()
    graphs = []
    for s, call, outs, X, _ in jobs:
        call()
        s.synchronize()
        first = [o.clone() for o in outs]
        call()
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call()
        X.neg_()
        call()
        torch.cuda.synchronize()
        graphs.append((graph, [o.clone() for o in outs]))
        assert not torch.equal(outs[0], first[0])
        for o in outs:
            o.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for (graph, _), (s, *_r) in zip(graphs, jobs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for (_, want), (_, _, outs, _, blk) in zip(graphs, jobs):
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
        assert blk.sync_status() == B.FW_OK


def test_more_rows_than_room(B):
    blk = block(B, 64, 64, 10, grad=1)
    t = [bf(11, 64) for _ in range(4)]
    W = bf(64, 64)
    with pytest.raises(B.FwError) as e:
        blk.backward(t[0], t[1], W, W, t[2], t[3], dX=bf(11, 64))
    assert e.value.status == B.FW_ERR_SHAPE
    blk = block(B, 64, 64)
    with pytest.raises(B.FwError) as e:
        blk.backward(t[0], t[1], W, W, t[2], t[3], dX=bf(11, 64))
    assert e.value.status == B.FW_ERR_WORKSPACE


@pytest.mark.parametrize("act", ACTS)
def test_activations_at_the_ends(B, act):
    """Far from 0 the derivative is 1 or 0 and the value a or 0, up to the largest finite bf16, whose square is beyond fp32.
    At most a reciprocal (one unit, 2 u) and a product (u) are rounded: 4 u."""
    big = torch.tensor([1e6, 1e10, 1.8e19, 1.9e19, 1e25, 1e30, 1e38, torch.finfo(BF16).max])
    a = torch.cat([big, -big]).cuda()
    N = a.numel()
    Zg, Zu, dH = (put(v[None], BF16, pad=None) for v in (a, torch.ones_like(a), torch.ones_like(a)))
    blk = block(B, 64, N, 1, act=ACTS.index(act), grad=1)
    dbg, dbu = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    blk.backward(dH, None, None, None, Zg, Zu, dbg=dbg, dbu=dbu)
    want = Zg[0].to(F64)
    assert bool(((dbg.to(F64) - (want > 0).to(F64)).abs() <= 4 * U).all()), dbg
    assert bool(((dbu.to(F64) - want.clamp(min=0)).abs() <= 4 * U * want.clamp(min=0)).all()), dbu


def test_another_device_than_the_current_one(B, monkeypatch):
    """The tensors are here and the current device is said to be another: nothing is launched."""
    monkeypatch.setattr(B, "_here", lambda: 1)
    with pytest.raises(ValueError, match="cuda:0, but the current device is cuda:1"):
        B.Gated(64, 32)


def test_workspace_outlives_the_work_on_its_stream(B):
    """A block that goes while its work waits on a stream of its own: its memory is not given to anybody else before that."""
    rows, M, N = 64, 64, 128
    s = torch.cuda.Stream()
    blk = B.Gated(M, N, rows, grad=1, stream=s.cuda_stream)
    dH, Zg, Zu = (bf(rows, N, fill=1.0) for _ in range(3))
    dbg, dbu = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    blk.backward(dH, None, None, None, Zg, Zu, dbg=dbg, dbu=dbu)     # the kernels are loaded
    torch.cuda.synchronize()
    at, n = blk.workspace.data_ptr(), blk.workspace.numel()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
    blk.backward(dH, None, None, None, Zg, Zu, dbg=dbg, dbu=dbu)
    assert not s.query()
    del blk
    others = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert not s.query() and all(o.data_ptr() != at for o in others)
    torch.cuda.synchronize()
