"""Residual RMS norm against its definition in 64 bits.

Error bounds (u = 2^-24).  A row's sum of squares is added in at most 32 + 5 + 32 steps (a thread's elements, lanes,
warps), all terms positive: 69 u; mean and eps 2 u more, of which the square root passes half on: 36 u; rsqrtf 2 ulp = 4 u; two
products 2 u: 42 u, taken as 48 u.  The held type adds half a step.
"""
import pytest
import torch

from optest_util import F64, HALF, U, captured, gen, matrix, put, surround_kept

pytestmark = pytest.mark.gpu

KINDS = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
FWD = 48 * U
SIZES = [(1, 1), (3, 7), (1, 64), (33, 100), (5, 257), (300, 1000), (17, 1537), (64, 2304), (9, 4096), (2, 8192), (3, 8191),
         (2, 16384), (2, 16381)]


@pytest.fixture(scope="module")
def B():
    from paper_2010_01546_b200 import binding, build
    build.build_library()
    return binding


def desc(B, M, kind, y=None, eps=1e-5):
    code = {"f32": B.FW_F32, "bf16": B.FW_BF16, "e4m3": B.FW_E4M3}
    return B.fw_norm_desc_default(M, dtype=code[kind], y_dtype=code[y or kind], eps=eps)


def inputs(rows, M, kind, seed, **kw):
    g = gen(seed)
    f = torch.exp(torch.randn(M, generator=g, device="cuda"))
    x = put(torch.randn(rows, M, generator=g, device="cuda") * f, KINDS[kind], **kw)
    r = put(torch.randn(rows, M, generator=g, device="cuda") * f, KINDS[kind], **kw)
    return x, r, 1 + 0.3 * torch.randn(M, generator=g, device="cuda")


def reference(x, r, w, eps):
    s = x.to(F64) if r is None else (x.to(F64) + r.to(F64)).to(x.dtype).to(F64)
    rstd = (s.square().mean(1) + eps).rsqrt()
    return s, rstd, s * rstd[:, None] * w.to(F64)


def check_y(y, scale, want):
    if scale is None:
        assert bool(((y.to(F64) - want).abs() <= (FWD + HALF[y.dtype] * (1 + FWD)) * want.abs()).all())
        return
    # the row's largest value fixes the scale; the held value is off by half a step, at least half of the smallest (2^-10)
    want_scale = want.abs().amax(1) / 448
    assert bool(((scale.to(F64) - want_scale).abs() <= (FWD + 2 * U) * want_scale).all())
    c = scale.to(F64)[:, None]
    off = (y.to(F64) * c - want).abs()
    assert bool((off <= 2.0 ** -4 * want.abs() + 2.0 ** -10 * c + 2 * (FWD + 4 * U) * want.abs()).all())


@pytest.mark.parametrize("rows,M", SIZES)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("y_kind", ["same", "e4m3"])
def test_forward(B, rows, M, kind, y_kind):
    for res, pad, shift in ((True, None, 0), (True, 1, 1), (False, 0, 0)):
        x, r, w = inputs(rows, M, kind, M + rows, pad=pad, shift=shift)
        r = r if res else None
        s = matrix(rows, M, KINDS[kind], pad=pad) if res else None
        yk = kind if y_kind == "same" else "e4m3"
        y = matrix(rows, M, KINDS[yk], pad=pad, shift=shift)
        scale = torch.full((rows,), 7.0, device="cuda") if yk == "e4m3" else None
        rstd = torch.empty(rows, device="cuda")
        B.fw_rmsnorm_forward(desc(B, M, kind, yk), x, w, y, res=r, sum_out=s, y_scale=scale, rstd=rstd)
        ws, wr, wy = reference(x, r, w, 1e-5)
        if res:
            assert torch.equal(s.to(F64), ws) and surround_kept(s)
        assert bool(((rstd.to(F64) - wr).abs() <= 40 * U * wr).all())
        check_y(y, scale, wy)
        assert surround_kept(y)


@pytest.mark.parametrize("rows,M", SIZES + [(701, 96), (1300, 512)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_backward(B, rows, M, kind):
    """dx within 100 u of its terms' magnitudes (the mean of u n: 69 u and 3 u for each term's products; the rest a few
    roundings) and half a step; dw within (rows + 64) u of the sum of its terms' magnitudes, in whatever order they are added."""
    for with_ds, pad, shift in ((True, None, 0), (True, 1, 1), (False, 0, 0)):
        s, ds, w = inputs(rows, M, kind, 3 * M + rows, pad=pad, shift=shift)
        dy, _, _ = inputs(rows, M, kind, 5 * M + rows, pad=pad, shift=shift)
        d = desc(B, M, kind)
        rstd = (s.float().square().mean(1) + 1e-5).rsqrt()
        dx = matrix(rows, M, KINDS[kind], pad=pad, shift=shift)
        dw = torch.full((M,), float("nan"), device="cuda")
        scratch = torch.empty(B.fw_rmsnorm_scratch_bytes(d), dtype=torch.uint8, device="cuda")
        B.fw_rmsnorm_backward(d, dy, s, w, rstd, dx, dw=dw, dsum=ds if with_ds else None, scratch=scratch)
        r = rstd.to(F64)[:, None]
        n, u = s.to(F64) * r, dy.to(F64) * w.to(F64)
        mean = (u * n).mean(1, keepdim=True)
        want = r * (u - n * mean)
        size = r * (u.abs() + n.abs() * (u * n).abs().mean(1, keepdim=True))
        if with_ds:
            want, size = want + ds.to(F64), size + ds.to(F64).abs()
        assert bool(((dx.to(F64) - want).abs() <= 100 * U * size + HALF[dx.dtype] * (want.abs() + 100 * U * size)).all())
        t = dy.to(F64) * n
        assert bool(((dw.to(F64) - t.sum(0)).abs() <= (rows + 64) * U * t.abs().sum(0)).all())
        assert surround_kept(dx)
        # without dw: the same dx, no scratch
        dx2 = matrix(rows, M, KINDS[kind], pad=pad, shift=shift)
        B.fw_rmsnorm_backward(d, dy, s, w, rstd, dx2, dsum=ds if with_ds else None)
        assert torch.equal(dx, dx2)


def test_gradient_against_differences(B):
    """Central differences of the forward definition in 64 bits, step 1e-6: truncation ~1e-12 and rounding ~1e-10 of the
    loss's terms, far below the kernel's fp32 errors (100 u of the terms' magnitudes, bounded as 1e-4 of the largest)."""
    rows, M, eps, h = 3, 12, 1e-5, 1e-6
    x, _, w = inputs(rows, M, "f32", 11)
    c = torch.randn(rows, M, generator=gen(12), device="cuda")
    loss = lambda xx, ww: float((c.to(F64) * xx * (xx.square().mean(1, keepdim=True) + eps).rsqrt() * ww).sum())  # noqa: E731
    d = desc(B, M, "f32", eps=eps)
    y, rstd, dx, dw = torch.empty_like(x.contiguous()), torch.empty(rows, device="cuda"), torch.empty(rows, M, device="cuda"), torch.empty(M, device="cuda")
    B.fw_rmsnorm_forward(d, x, w, y, rstd=rstd)
    B.fw_rmsnorm_backward(d, c, x, w, rstd, dx, dw=dw, scratch=torch.empty(B.fw_rmsnorm_scratch_bytes(d), dtype=torch.uint8, device="cuda"))
    x64, w64 = x.to(F64).contiguous(), w.to(F64)
    for at, got in ((x64, dx), (w64, dw)):
        num = torch.empty_like(at)
        for i in range(at.numel()):
            v = float(at.view(-1)[i])
            at.view(-1)[i] = v + h
            up = loss(x64, w64)
            at.view(-1)[i] = v - h
            num.view(-1)[i] = (up - loss(x64, w64)) / (2 * h)
            at.view(-1)[i] = v
        assert float((got.to(F64) - num).abs().max()) <= 1e-4 * float(num.abs().max())


def test_in_place_and_repeated(B):
    for kind in ("f32", "bf16"):
        x, r, w = inputs(50, 600, kind, 5)
        d = desc(B, 600, kind)
        s, y = matrix(50, 600, KINDS[kind]), matrix(50, 600, KINDS[kind])
        B.fw_rmsnorm_forward(d, x, w, y, res=r, sum_out=s)
        y2 = matrix(50, 600, KINDS[kind])
        B.fw_rmsnorm_forward(d, x, w, y2, res=r, sum_out=s)
        assert torch.equal(y, y2)
        x2, r2 = put(x, KINDS[kind]), put(r, KINDS[kind])
        B.fw_rmsnorm_forward(d, x2, w, x2, res=r2, sum_out=r2)
        assert torch.equal(x2, y) and torch.equal(r2, s)
        rstd = (s.float().square().mean(1) + 1e-5).rsqrt()
        dx, dy2 = matrix(50, 600, KINDS[kind]), put(x, KINDS[kind])
        B.fw_rmsnorm_backward(d, x, s, w, rstd, dx, dsum=r)
        B.fw_rmsnorm_backward(d, dy2, s, w, rstd, dy2, dsum=r)
        assert torch.equal(dx, dy2)


def test_special_rows(B):
    """Rows of zeros, with a NaN, with an infinity and with huge and tiny values: each gives what the formulas give, no other
    row is touched by it."""
    M = 520
    x, _, w = inputs(8, M, "f32", 21)
    clean = x.clone()
    x[1] = 0
    x[2, 7] = float("nan")
    x[3, 100] = float("inf")
    x[4] *= 1e-30
    x[5] *= 1e15
    for y_kind in ("f32", "e4m3"):
        d = desc(B, M, "f32", y_kind)
        out = []
        for v in (x, clean):
            y, scale = matrix(8, M, KINDS[y_kind], pad=None), torch.empty(8, device="cuda") if y_kind == "e4m3" else None
            B.fw_rmsnorm_forward(d, v, w, y, y_scale=scale)
            out.append((y.float(), scale))
        y, scale = out[0]
        assert torch.equal(y[[0, 6, 7]], out[1][0][[0, 6, 7]])
        assert bool((y[1] == 0).all()) and bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[3, 100]))
        if scale is not None:
            assert float(scale[1]) == 1 and bool(torch.isnan(scale[2]))
            assert bool(torch.isfinite(y[4]).all()) and float(scale[4]) >= 2.0 ** -120
        else:
            assert bool((y[3][torch.arange(M, device="cuda") != 100] == 0).all())
            _, _, want = reference(x[4:6], None, w, 1e-5)
            check_y(y[4:6], None, want)


def test_other_stream_and_graph(B):
    M, rows = 1000, 200
    x, r, w = inputs(rows, M, "bf16", 31, pad=None)
    d, d8 = desc(B, M, "bf16"), desc(B, M, "bf16", "e4m3")
    s, y, q = matrix(rows, M, torch.bfloat16, pad=None), matrix(rows, M, torch.bfloat16, pad=None), matrix(rows, M, torch.float8_e4m3fn, pad=None)
    scale, rstd, dw = (torch.empty(n, device="cuda") for n in (rows, rows, M))
    dx = matrix(rows, M, torch.bfloat16, pad=None)
    scratch = torch.empty(B.fw_rmsnorm_scratch_bytes(d), dtype=torch.uint8, device="cuda")

    def call(stream):
        B.fw_rmsnorm_forward(d, x, w, y, res=r, sum_out=s, rstd=rstd, stream=stream)
        B.fw_rmsnorm_forward(d8, x, w, q, res=r, y_scale=scale, stream=stream)
        B.fw_rmsnorm_backward(d, y, s, w, rstd, dx, dw=dw, dsum=x, scratch=scratch, stream=stream)

    call(0)
    torch.cuda.synchronize()
    g = captured(call)
    x.copy_(inputs(rows, M, "bf16", 32, pad=None)[0])
    g.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (s, y, q.float(), scale, rstd, dx, dw)]
    call(0)
    torch.cuda.synchronize()
    for a, b in zip(got, (s, y, q.float(), scale, rstd, dx, dw)):
        assert torch.equal(a, b)


def e4m3_of_row(s, w, eps):
    """y / c and c in 64 bits."""
    y = s.to(F64) * (s.to(F64).square().mean(1, keepdim=True) + eps).rsqrt() * w.to(F64)
    c = y.abs().amax(1, keepdim=True) / 448
    return y / c, c[:, 0]


def nearest_within(q, ratio, rel):
    """Each element of q is what some number within `rel` of `ratio` rounds to."""
    low, high = ((ratio * (1 + k * rel)).float().to(torch.float8_e4m3fn).float() for k in (-1, 1))
    q = q.float()
    return (q >= torch.minimum(low, high)) & (q <= torch.maximum(low, high))


@pytest.mark.parametrize("M", [520, 1537, 4096])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_e4m3_of_small_and_large_products(B, M, kind):
    """Rows whose |s w| is near the lower end of fp32 while y is not (448 / 1.2e-36 is beyond it), and large ones.  Zeros stay zeros.
    Squares of s below 1e-38 are 0 in fp32, as eps makes them in the definition.  What is rounded is within 7 u of y / c: s w, the largest
    of them, below 2e-36 both times rstd, 448 over that, the product, and half a step of fp32 in this test."""
    g, t = gen(M), KINDS[kind]
    for size, wsize in ((1e-36, 1.0), (1.2e-30, 1e-6), (1e-26, 1e-10), (1e9, 1e-30), (1e9, 1e25)):
        x = put(torch.rand(4, M, generator=g, device="cuda").mul_(2).sub_(1) * size, t, pad=None)
        x[:, ::5] = 0
        x[:, 1] = 1.2 * size
        w = (0.5 + 0.5 * torch.rand(M, generator=g, device="cuda")) * wsize
        y, scale = matrix(4, M, torch.float8_e4m3fn, pad=None), torch.empty(4, device="cuda")
        B.fw_rmsnorm_forward(desc(B, M, kind, "e4m3", eps=1e-6), x, w, y, y_scale=scale)
        ratio, c = e4m3_of_row(x, w, 1e-6)
        assert bool(((scale.to(F64) - c).abs() <= (FWD + 4 * U) * c).all()), (size, wsize)
        assert bool(nearest_within(y, ratio, 7 * U).all()), (size, wsize)
        assert bool((y[:, ::5].float() == 0).all())


def test_e4m3_codes(B):
    """An ordinary matrix: every code is that of a number within 5 u of y / c (s w, the largest of them, 448 over that and the
    product are rounded; one more half step in this test's own conversion)."""
    rows, M = 4096, 4096
    x, _, w = inputs(rows, M, "bf16", 1, pad=None)
    y, scale = matrix(rows, M, torch.float8_e4m3fn, pad=None), torch.empty(rows, device="cuda")
    B.fw_rmsnorm_forward(desc(B, M, "bf16", "e4m3"), x, w, y, y_scale=scale)
    ratio, _ = e4m3_of_row(x, w, 1e-5)
    assert bool(nearest_within(y, ratio, 5 * U).all())


def test_e4m3_row_beyond_the_squares(B):
    """|s| beyond 1.8e19: rstd and y are 0, a row of zeros with scale 1."""
    x = torch.full((2, 64), 1e30, device="cuda")
    y, scale, rstd = matrix(2, 64, torch.float8_e4m3fn), torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    B.fw_rmsnorm_forward(desc(B, 64, "f32", "e4m3"), x, torch.ones(64, device="cuda"), y, y_scale=scale, rstd=rstd)
    assert bool((rstd == 0).all()) and bool((y.float() == 0).all()) and bool((scale == 1).all())


def test_e4m3_row_beyond_the_products(B):
    """|s w| beyond 3.4e38 while y is not: an infinite scale says so; the other row is as ever."""
    x = torch.ones(2, 64, device="cuda")
    x[0] = 1e15
    w = torch.full((64,), 1e25, device="cuda")
    y, scale = matrix(2, 64, torch.float8_e4m3fn), torch.empty(2, device="cuda")
    B.fw_rmsnorm_forward(desc(B, 64, "f32", "e4m3"), x, w, y, y_scale=scale)
    assert float(scale[0]) == float("inf") and bool(torch.isfinite(scale[1])) and bool((y[1].float() == 448).all())
