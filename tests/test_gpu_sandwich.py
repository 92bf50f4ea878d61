"""Norms around a block with the gate and the residual addition against their definition in 64 bits.

Error bounds (u = 2^-24), built on those of the norm: rstd 36 u and 4 u of rsqrtf.  h: the block's part has rstd, the gate's product and two
more, 43 u, taken as 48 u, and the sum 2 u of both parts; y is checked from the h that is held: 48 u.  Gradients: t (of h) is within
100 u of its terms' sizes; the second norm's gradient starts from it and adds the same again: 210 u; sums over rows add a rounding a
row, whatever their order.  The held type adds half a step.
"""
import pytest
import torch

from optest_util import F64, HALF, U, captured, gen, matrix, put, surround_kept

pytestmark = pytest.mark.gpu

KINDS = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
FWD = 48 * U
SIZES = [(1, 1), (3, 7), (1, 64), (33, 100), (5, 257), (300, 1000), (17, 1537), (64, 2304), (9, 4096), (700, 4096), (2, 8192), (3, 8191),
         (2, 16384), (2, 16381)]


@pytest.fixture(scope="module")
def B():
    from paper_2010_01546_b200 import binding, build
    build.build_library()
    return binding


def desc(B, M, kind, y=None, **kw):
    code = {"f32": B.FW_F32, "bf16": B.FW_BF16, "e4m3": B.FW_E4M3}
    return B.fw_sandwich_desc_default(M, dtype=code[kind], y_dtype=code[y or kind], eps=1e-5, **kw)


def inputs(rows, M, kind, seed, **kw):
    g = gen(seed)
    rnd = lambda: torch.randn(rows, M, generator=g, device="cuda")  # noqa: E731
    f = torch.exp(torch.randn(M, generator=g, device="cuda"))
    return dict(o=put(rnd(), KINDS[kind], **kw), x=put(rnd() * f, KINDS[kind], **kw), w1=0.5 + 0.3 * torch.randn(M, generator=g, device="cuda"),
                w2=1 + 0.3 * torch.randn(M, generator=g, device="cuda"), gate=torch.randn(rows, generator=g, device="cuda"))


CASES = [dict(post=1, w1=True, gate=False, alpha=1.0, pad=None, shift=0), dict(post=1, w1=True, gate=True, alpha=0.7, pad=1, shift=1),
         dict(post=0, w1=True, gate=True, alpha=-1.5, pad=0, shift=0), dict(post=1, w1=False, gate=False, alpha=0.0, pad=None, shift=0)]


@pytest.mark.parametrize("rows,M", SIZES)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("y_kind", ["same", "e4m3"])
def test_forward(B, rows, M, kind, y_kind):
    for c in CASES:
        a = inputs(rows, M, kind, M + rows, pad=c["pad"], shift=c["shift"])
        yk = kind if y_kind == "same" else "e4m3"
        alpha = float(torch.tensor(c["alpha"]))
        h, y = matrix(rows, M, KINDS[kind], pad=c["pad"]), matrix(rows, M, KINDS[yk], pad=c["pad"], shift=c["shift"])
        scale = torch.full((rows,), 7.0, device="cuda") if yk == "e4m3" else None
        rstd = torch.full((rows, 2), 7.0, device="cuda")
        B.fw_sandwich_forward(desc(B, M, kind, yk, post=c["post"], alpha=alpha), a["o"], a["x"], a["w2"], h, y, w_post=a["w1"] if c["w1"] else None,
                              gate=a["gate"] if c["gate"] else None, y_scale=scale, rstd=rstd)
        o, x = a["o"].to(F64), a["x"].to(F64)
        r1 = (o.square().mean(1) + 1e-5).rsqrt() if c["post"] else torch.ones(rows, dtype=F64, device="cuda")
        part = o * r1[:, None]
        if c["w1"]:
            part = part * a["w1"].to(F64)
        if c["gate"]:
            part = part * a["gate"].to(F64)[:, None]
        want = part + alpha * x
        err = FWD * part.abs() + 2 * U * (part.abs() + (alpha * x).abs())
        assert bool(((h.to(F64) - want).abs() <= err + HALF[h.dtype] * (want.abs() + err)).all())
        hh = h.to(F64)
        r2 = (hh.square().mean(1) + 1e-5).rsqrt()
        assert bool(((rstd.to(F64) - torch.stack((r1, r2), 1)).abs() <= 40 * U * torch.stack((r1, r2), 1)).all())
        wy = hh * r2[:, None] * a["w2"].to(F64)
        if scale is None:
            assert bool(((y.to(F64) - wy).abs() <= (FWD + HALF[y.dtype] * (1 + FWD)) * wy.abs()).all())
        else:
            top = wy.abs().amax(1)
            ws = torch.where(top > 0, top / 448, 1.0)
            assert bool(((scale.to(F64) - ws).abs() <= (FWD + 2 * U) * ws).all())
            s = scale.to(F64)[:, None]
            assert bool(((y.to(F64) * s - wy).abs() <= 2.0 ** -4 * wy.abs() + 2.0 ** -10 * s + 2 * (FWD + 4 * U) * wy.abs()).all())
        assert surround_kept(h) and surround_kept(y)


@pytest.mark.parametrize("rows,M", SIZES + [(701, 96), (1300, 512)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_backward(B, rows, M, kind):
    for n, c in enumerate(CASES):
        a = inputs(rows, M, kind, 3 * M + rows, pad=c["pad"], shift=c["shift"])
        g = inputs(rows, M, kind, 5 * M + rows, pad=c["pad"], shift=c["shift"])
        o, h, dy, dh = a["o"], a["x"], g["o"], g["x"] if n != 2 else None
        alpha = float(torch.tensor(c["alpha"]))
        rstd = torch.stack([(v.float().square().mean(1) + 1e-5).rsqrt() for v in (o, h)], 1)
        w1, gate = a["w1"] if c["w1"] else None, a["gate"] if c["gate"] else None
        dx, do = (matrix(rows, M, KINDS[kind], pad=c["pad"], shift=c["shift"]) for _ in range(2))
        nan = lambda n: torch.full((n,), float("nan"), device="cuda")  # noqa: E731
        dw1, dw2, dgate = nan(M), nan(M), nan(rows)
        d = desc(B, M, kind, post=c["post"], alpha=alpha)
        scratch = torch.empty(B.fw_sandwich_scratch_bytes(d), dtype=torch.uint8, device="cuda")
        B.fw_sandwich_backward(d, dy, o, h, a["w2"], rstd, dx, do, w_post=w1, gate=gate, dh=dh, dw_post=dw1, dw_pre=dw2, dgate=dgate, scratch=scratch)
        r1, r2 = rstd.to(F64)[:, :1] if c["post"] else torch.ones(rows, 1, dtype=F64, device="cuda"), rstd.to(F64)[:, 1:]
        k = torch.ones(rows, 1, dtype=F64, device="cuda") if gate is None else gate.to(F64)[:, None]
        v1 = torch.ones(M, dtype=F64, device="cuda") if w1 is None else w1.to(F64)
        n2, u2 = h.to(F64) * r2, dy.to(F64) * a["w2"].to(F64)
        t = r2 * (u2 - n2 * (u2 * n2).mean(1, keepdim=True))
        ts = r2 * (u2.abs() + n2.abs() * (u2 * n2).abs().mean(1, keepdim=True))
        if dh is not None:
            t, ts = t + dh.to(F64), ts + dh.to(F64).abs()
        e = abs(alpha) * 100 * U * ts
        assert bool(((dx.to(F64) - alpha * t).abs() <= e + HALF[dx.dtype] * ((alpha * t).abs() + e)).all())
        n1, u1, us = o.to(F64) * r1, t * v1, ts * v1.abs()
        want, size = k * u1, k.abs() * us
        if c["post"]:
            want, size = k * r1 * (u1 - n1 * (u1 * n1).mean(1, keepdim=True)), k.abs() * r1 * (us + n1.abs() * (us * n1.abs()).mean(1, keepdim=True))
        assert bool(((do.to(F64) - want).abs() <= 210 * U * size + HALF[do.dtype] * (want.abs() + 210 * U * size)).all())
        q = dy.to(F64) * n2
        assert bool(((dw2.to(F64) - q.sum(0)).abs() <= (rows + 64) * U * q.abs().sum(0)).all())
        assert bool(((dw1.to(F64) - (k * t * n1).sum(0)).abs() <= (rows + 174) * U * (k.abs() * ts * n1.abs()).sum(0)).all())
        assert bool(((dgate.to(F64) - (u1 * n1).sum(1)).abs() <= 200 * U * (us * n1.abs()).sum(1)).all())
        assert surround_kept(dx) and surround_kept(do)
        # without the sums: the same gradients, no scratch; one of the sums alone
        dx2, do2 = (matrix(rows, M, KINDS[kind], pad=c["pad"], shift=c["shift"]) for _ in range(2))
        B.fw_sandwich_backward(d, dy, o, h, a["w2"], rstd, dx2, do2, w_post=w1, gate=gate, dh=dh)
        assert torch.equal(dx, dx2) and torch.equal(do, do2)
        one = nan(M)
        B.fw_sandwich_backward(d, dy, o, h, a["w2"], rstd, dx2, do2, w_post=w1, gate=gate, dh=dh, dw_post=one, scratch=scratch)
        assert torch.equal(one, dw1)
        # in the place of inputs
        if n < 2:
            B.fw_sandwich_backward(d, dy, o, h, a["w2"], rstd, h, o, w_post=w1, gate=gate, dh=dh)
            assert torch.equal(h, dx) and torch.equal(o, do) and surround_kept(h) and surround_kept(o)


@pytest.mark.parametrize("M", [640, 1152, 1280, 1536, 1601, 1793, 2304, 3585, 5120, 5121, 6144, 7168, 9216, 10240, 11777, 12288, 14336])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_of_any_number_of_warps(B, M, kind):
    """Three to fifteen warps a row, with rows for one access of a thread and for several."""
    for rows in (5, 310):
        test_forward(B, rows, M, kind, "e4m3" if rows == 5 else "same")
        test_backward(B, rows, M, kind)


def test_gradient_against_differences(B):
    """Central differences of the definition in 64 bits, step 1e-6 (1e-9 of the loss's terms); the kernel's fp32 is bounded as 1e-4
    of the largest element."""
    rows, M, alpha = 3, 12, 0.75
    a = inputs(rows, M, "f32", 11)
    cy, ch = (torch.randn(rows, M, generator=gen(s), device="cuda") for s in (12, 13))

    def loss(o, x, w1, w2, gate):
        h = alpha * x + gate[:, None] * w1 * o * (o.square().mean(1, keepdim=True) + 1e-5).rsqrt()
        return float((cy.to(F64) * h * (h.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w2 + ch.to(F64) * h).sum())
    d = desc(B, M, "f32", alpha=alpha)
    h, y, rstd = torch.empty(rows, M, device="cuda"), torch.empty(rows, M, device="cuda"), torch.empty(rows, 2, device="cuda")
    B.fw_sandwich_forward(d, a["o"], a["x"], a["w2"], h, y, w_post=a["w1"], gate=a["gate"], rstd=rstd)
    dx, do, dw1, dw2, dg = (torch.empty(s, device="cuda") for s in ((rows, M), (rows, M), M, M, rows))
    B.fw_sandwich_backward(d, cy, a["o"], h, a["w2"], rstd, dx, do, w_post=a["w1"], gate=a["gate"], dh=ch, dw_post=dw1, dw_pre=dw2, dgate=dg,
                           scratch=torch.empty(B.fw_sandwich_scratch_bytes(d), dtype=torch.uint8, device="cuda"))
    args, step = [a[k].to(F64).contiguous() for k in ("o", "x", "w1", "w2", "gate")], 1e-6
    for at, got in zip(args, (do, dx, dw1, dw2, dg)):
        num = torch.empty_like(at)
        for i in range(at.numel()):
            v = float(at.view(-1)[i])
            at.view(-1)[i] = v + step
            up = loss(*args)
            at.view(-1)[i] = v - step
            num.view(-1)[i] = (up - loss(*args)) / (2 * step)
            at.view(-1)[i] = v
        assert float((got.to(F64) - num).abs().max()) <= 1e-4 * float(num.abs().max())


def test_in_place_and_repeated(B):
    for kind, pad in (("f32", None), ("bf16", 1), ("bf16", None)):
        for h_in in ("o", "x"):
            a = inputs(50, 603, kind, 5, pad=pad)
            h, y = matrix(50, 603, KINDS[kind], pad=pad), matrix(50, 603, KINDS[kind], pad=pad)
            d = desc(B, 603, kind)
            B.fw_sandwich_forward(d, a["o"], a["x"], a["w2"], h, y, w_post=a["w1"], gate=a["gate"])
            h2, y2 = matrix(50, 603, KINDS[kind], pad=pad), matrix(50, 603, KINDS[kind], pad=pad)
            B.fw_sandwich_forward(d, a["o"], a["x"], a["w2"], h2, y2, w_post=a["w1"], gate=a["gate"])
            assert torch.equal(h, h2) and torch.equal(y, y2)
            B.fw_sandwich_forward(d, a["o"], a["x"], a["w2"], a[h_in], a["x" if h_in == "o" else "o"], w_post=a["w1"], gate=a["gate"])
            assert torch.equal(a[h_in], h) and torch.equal(a["x" if h_in == "o" else "o"], y) and surround_kept(a["o"]) and surround_kept(a["x"])


@pytest.mark.parametrize("kind,M,pad", [("f32", 1537, 0), ("bf16", 1537, 0), ("bf16", 4096, None), ("bf16", 4095, None), ("f32", 1537, None), ("f32", 5120, None), ("bf16", 603, 1), ("f32", 96, None),
                                        ("bf16", 16384, None), ("f32", 16381, 2)])
def test_backward_in_place(B, kind, M, pad):
    """Each gradient in the place of each input that the header allows: the bits of the call with outputs of their own."""
    rows = 700
    a, g = inputs(rows, M, kind, 6, pad=pad), inputs(rows, M, kind, 7, pad=pad)
    keep = dict(dy=g["o"], dh=g["x"], o=a["o"], h=a["x"])
    rstd = torch.rand(rows, 2, generator=gen(8), device="cuda") + 0.5
    d = desc(B, M, kind)
    scratch = torch.empty(B.fw_sandwich_scratch_bytes(d), dtype=torch.uint8, device="cuda")

    def call(i, dx, do):
        dw1, dw2, dgate = (torch.empty(n, device="cuda") for n in (M, M, rows))
        B.fw_sandwich_backward(d, i["dy"], i["o"], i["h"], a["w2"], rstd, dx, do, w_post=a["w1"], gate=a["gate"], dh=i["dh"], dw_post=dw1,
                               dw_pre=dw2, dgate=dgate, scratch=scratch)
        return dx, do, dw1, dw2, dgate

    want = call(keep, matrix(rows, M, KINDS[kind], pad=pad), matrix(rows, M, KINDS[kind], pad=pad))
    for x in ("dy", "dh", "h"):
        for o in ("dy", "dh", "o", "h"):
            if x == o:
                continue
            i = {k: put(v, KINDS[kind], pad=pad) for k, v in keep.items()}
            got = call(i, i[x], i[o])
            assert all(torch.equal(p, q) for p, q in zip(got, want)), (x, o)
            assert all(surround_kept(v) for v in i.values())
            assert all(torch.equal(i[k], keep[k]) for k in i if k not in (x, o))


def test_values_that_are_none(B):
    """A NaN or an infinity stays in its row; rows of zeros and squares that pass fp32 as in the norm."""
    M = 600
    for kind in ("f32", "bf16"):
        for y_kind in (kind, "e4m3"):
            a = inputs(6, M, kind, 8)
            a["o"][0, 3], a["x"][1, 7] = float("nan"), float("inf")
            a["o"][2] = 0
            a["x"][2] = 0
            a["o"][3] = 1e25
            a["x"][3] = 0
            h, y = matrix(6, M, KINDS[kind]), matrix(6, M, KINDS[y_kind])
            scale = torch.empty(6, device="cuda") if y_kind == "e4m3" else None
            rstd = torch.empty(6, 2, device="cuda")
            B.fw_sandwich_forward(desc(B, M, kind, y_kind), a["o"], a["x"], a["w2"], h, y, w_post=a["w1"], y_scale=scale, rstd=rstd)
            assert bool(h[0].isnan().all()) and bool(rstd[0].isnan().all()) and bool(y[0].float().isnan().all())
            assert int(h[1].float().isfinite().logical_not().sum()) == 1 and float(rstd[1, 1]) == 0
            assert bool((y[2].float() == 0).all()) and bool((h[2] == 0).all())
            assert float(rstd[3, 0]) == 0 and bool((h[3] == 0).all())
            assert bool(h[4:].float().isfinite().all()) and bool(y[4:].float().isfinite().all())


def test_a_step_through_both_directions_captured(B):
    rows, M = 130, 1000
    a, g = inputs(rows, M, "bf16", 1), inputs(rows, M, "bf16", 2)
    d = desc(B, M, "bf16")
    mats = {k: matrix(rows, M, torch.bfloat16) for k in ("h", "y", "dx", "do")}
    rstd, dw1, dw2, dg = torch.empty(rows, 2, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, device="cuda"), torch.empty(rows, device="cuda")
    scratch = torch.empty(B.fw_sandwich_scratch_bytes(d), dtype=torch.uint8, device="cuda")

    def call(s):
        B.fw_sandwich_forward(d, a["o"], a["x"], a["w2"], mats["h"], mats["y"], w_post=a["w1"], gate=a["gate"], rstd=rstd, stream=s)
        B.fw_sandwich_backward(d, g["o"], a["o"], mats["h"], a["w2"], rstd, mats["dx"], mats["do"], w_post=a["w1"], gate=a["gate"], dh=g["x"],
                               dw_post=dw1, dw_pre=dw2, dgate=dg, scratch=scratch, stream=s)
    graph = captured(call)
    a["o"].mul_(-0.5)
    a["x"].add_(1.0)
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (*mats.values(), rstd, dw1, dw2, dg)]
    call(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, (*mats.values(), rstd, dw1, dw2, dg)))


def test_rows_beyond_32_bits(B):
    """Rows 2^30 - 8 elements apart: the last begins 2^31 elements and more from the first."""
    ld, M = (1 << 30) - 8, 1000
    base = torch.empty(3 * ld, dtype=torch.bfloat16, device="cuda")
    big = lambda k: torch.as_strided(base, (4, M), (ld // 2, 1), k * 1024)  # noqa: E731
    a = inputs(4, M, "bf16", 3)
    o, x, h, y = (big(k) for k in range(4))
    o.copy_(a["o"])
    x.copy_(a["x"])
    d = desc(B, M, "bf16")
    h2, y2 = matrix(4, M, torch.bfloat16), matrix(4, M, torch.bfloat16)
    B.fw_sandwich_forward(d, a["o"], a["x"], a["w2"], h2, y2, w_post=a["w1"])
    with pytest.raises(B.FwError):
        B.fw_sandwich_forward(d, o, x, a["w2"], h, y, w_post=a["w1"])      # the rows lie between one another's
    del o, x, h, y, base
    ld = (1 << 30) - 8
    big = lambda: torch.as_strided(torch.empty(3 * ld + M, dtype=torch.bfloat16, device="cuda"), (4, M), (ld, 1))  # noqa: E731
    o, h = big(), big()
    o.copy_(a["o"])
    B.fw_sandwich_forward(d, o, a["x"], a["w2"], h, o, w_post=a["w1"])
    assert torch.equal(h, h2) and torch.equal(o, y2)


@pytest.mark.parametrize("kind,M,pad", [("f32", 1537, 0), ("bf16", 1537, 0), ("bf16", 4095, 3), ("bf16", 4095, None), ("f32", 1537, None), ("f32", 603, 1),
                                        ("bf16", 7001, None), ("f32", 7001, 2)])
def test_forward_in_place(B, kind, M, pad):
    """h and y in the place of o and x, rows by whole accesses though they begin or end inside one: the bits of the call with outputs of
    their own."""
    rows = 700
    keep = inputs(rows, M, kind, 9, pad=pad)
    d = desc(B, M, kind)
    h, y = matrix(rows, M, KINDS[kind], pad=pad), matrix(rows, M, KINDS[kind], pad=pad)
    B.fw_sandwich_forward(d, keep["o"], keep["x"], keep["w2"], h, y, w_post=keep["w1"], gate=keep["gate"])
    for h_in, y_in in (("o", "x"), ("x", "o"), ("o", None), ("x", None), (None, "o"), (None, "x")):
        a = {k: put(keep[k], KINDS[kind], pad=pad) for k in ("o", "x")}
        out = {n: a[k] if k else matrix(rows, M, KINDS[kind], pad=pad) for n, k in (("h", h_in), ("y", y_in))}
        B.fw_sandwich_forward(d, a["o"], a["x"], keep["w2"], out["h"], out["y"], w_post=keep["w1"], gate=keep["gate"])
        assert torch.equal(out["h"], h) and torch.equal(out["y"], y), (h_in, y_in)
        assert surround_kept(a["o"]) and surround_kept(a["x"]) and surround_kept(out["h"]) and surround_kept(out["y"])
        assert all(torch.equal(a[k], keep[k]) for k in a if k not in (h_in, y_in))


@pytest.mark.parametrize("rows,M", [(5, 6145), (310, 7001), (310, 8183)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_e4m3_from_long_odd_rows(B, rows, M, kind):
    test_forward(B, rows, M, kind, "e4m3")
