"""Distillation loss and gradient against the definition in 64 bits.

Error bounds (u = 2^-24).  An exponential exp(-a) is computed with 2^-22 and 4 u a ln 2 of its argument; sums of exponentials
have at most 32 x 8 + 5 + 16 + 8 steps for 2^20 classes (a thread's trips, lanes, warps, CTAs), 61 u up to 131072 of them: a
probability is within E(a) = 2^-17 (1 + a / 8) of itself, 2^-15 (1 + a / 8) above that size.  Logarithms add 4 u (1 + |log|).
"""
import pytest
import torch

from optest_util import F64, HALF, captured, gen, matrix, put, surround_kept

pytestmark = pytest.mark.gpu

KINDS = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [(3, 1, 1), (1, 2, 2), (5, 100, 10), (37, 1000, 10), (9, 300, 81), (6, 512, 128), (5, 1024, 129), (7, 2047, 64), (7, 1025, 33), (4, 2048, 1024), (3, 8191, 64), (2, 50021, 33),
         (5, 3000, 256), (2, 9000, 257), (2, 131072, 64), (2, 131101, 100), (2, 250000, 256), (1, 300001, 7), (1, 1 << 20, 130)]


@pytest.fixture(scope="module")
def B():
    from paper_2010_01546_b200 import binding, build
    build.build_library()
    return binding


def desc(B, V, K, kind, t=torch.float32, bits=32, tau=1.0):
    return B.fw_distill_desc_default(V, K, z_dtype=B.FW_F32 if kind == "f32" else B.FW_BF16,
                                     t_dtype=B.FW_F32 if t == torch.float32 else B.FW_BF16, index_bits=bits, tau=tau)


def inputs(rows, V, K, kind, seed, t=torch.float32, tau=1.0, **kw):
    """Student's logits, the teacher's K largest and their classes, and the teacher's normaliser."""
    g = gen(seed)
    z = torch.randn(rows, V, generator=g, device="cuda") * 2
    teacher = 0.7 * z + torch.randn(rows, V, generator=g, device="cuda")
    top, at = teacher.topk(K, dim=1)
    return put(z, KINDS[kind], **kw), top.to(t), at.to(torch.int32), torch.logsumexp(teacher.to(F64) / tau, 1).float()


def column(v):
    return v[:, None] if torch.is_tensor(v) else v


def reference(z, T, I, tau, t_lse=None, weight=None):
    """loss, stat, dZ, and bounds of the errors of loss and dZ."""
    rows, V = z.shape
    K = T.shape[1]
    u = 2.0 ** -24
    z, t, I = z.to(F64) / tau, T.to(F64) / tau, I.long()
    w = torch.ones(rows, dtype=F64, device="cuda") if weight is None else weight.to(F64)
    there = (I >= 0) & (I < V)
    same = (I[:, :, None] == I[:, None, :]) & torch.ones(K, K, dtype=torch.bool, device="cuda").tril(-1)
    there = there & ~(same & there[:, None, :]).any(2)
    at = torch.where(there, I, 0)
    named = torch.zeros(rows, V, device="cuda").scatter_add_(1, at, there.float()) > 0
    lse = torch.logsumexp(z, 1)
    rest = torch.logsumexp(z.masked_fill(named, float("-inf")), 1)
    empty = lse == float("-inf")
    t = t.masked_fill(~there, float("-inf"))
    if t_lse is None:
        norm = torch.logsumexp(t, 1, keepdim=True)
        logp = torch.where(norm == float("-inf"), norm, t - norm)
        pt = torch.zeros(rows, dtype=F64, device="cuda")
        dpt = 0.0
    else:
        logp = t - t_lse.to(F64)[:, None]
        pt = (1 - logp.exp().sum(1)).clamp(min=0)
    p = logp.exp()
    logq = z.gather(1, at) - lse[:, None]
    qt = (rest - lse).exp()
    kl = torch.where(p == 0, 0, p * (logp - logq)).sum(1) + torch.where(pt > 0, pt * (pt.log() - qt.log()), 0)
    A = p.sum(1) + pt
    q = (z - lse[:, None]).exp()
    ratio = torch.where((pt > 0) & (qt > 0), pt / qt, 0)
    dz = torch.where(named, A[:, None] * q, q * (A - ratio)[:, None]).scatter_add(1, at, torch.where(there, -p, 0))
    live = (w != 0) & ~empty
    loss = torch.where(live, w * kl, 0)
    dz = torch.where(live[:, None], dz * (w / tau)[:, None], 0)
    stat = torch.where((w != 0)[:, None], torch.stack((lse, rest), 1), 0)
    # bounds: p within E and what rounds t / tau - t_lse, p_t what their sum is off, logarithms 4 u (1 + |log|)
    E = 2.0 ** -17 if V <= 131072 else 2.0 ** -15
    dp = p * E + 4 * u
    if t_lse is not None:
        dp = dp + p * 8 * u * (t.masked_fill(~there | torch.isinf(t), 0).abs() + t_lse.to(F64).abs()[:, None])
        dpt = dp.sum(1)
    mag = torch.where(p == 0, 0, logp.abs() + logq.abs())
    lt = torch.where(pt > 0, pt.log().abs() + qt.log().abs(), 0)
    dloss = w.abs() * ((dp * (1 + mag) + p * (E + 4 * u * (2 + mag))).sum(1) + dpt * (lt + 1) + pt * (E + 4 * u) * (2 + lt))
    Ea = E * (1 + (z.amax(1, keepdim=True) - z).clamp(max=1e4) / 8)     # beyond that q is 0, and so is what it is multiplied by
    dnamed = A[:, None] * q * Ea + column(dpt) * q + torch.zeros_like(q).scatter_add(1, at, torch.where(there, dp, 0))
    dother = q * (2 * Ea * (A + ratio)[:, None] + column(dpt) * (1 + torch.where(qt > 0, 1 / qt, 0))[:, None])
    return loss, stat, dz, dloss, torch.where(named, dnamed, dother) * (w.abs() / tau)[:, None]


def check(got, want, bound, half=0.0):
    got = got.to(F64)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    off = (got - want).abs()[fine]
    allowed = (bound + half * (want.abs() + bound))[fine] + 1e-37
    assert bool((off <= allowed).all()), float((off / allowed).max())


def check_stat(stat, want):
    fine = torch.isfinite(want)
    got = stat.to(F64)
    assert torch.equal(got[~fine], want[~fine])
    assert bool(((got - want).abs()[fine] <= 2.0 ** -15 + 8 * 2.0 ** -24 * want.abs()[fine]).all())


def stat_bound(want):
    """What the backward call's dZ may be off beyond the forward call's: its normalisers were rounded to fp32 and the student's
    probabilities are relative to them (16 u |stat| of each term; the terms' size is the bound over E)."""
    s = want[1].masked_fill(torch.isinf(want[1]), 0).abs().amax(1, keepdim=True)
    return want[4] * (1 + 2.0 ** 17 * 16 * 2.0 ** -24 * (1 + s))


@pytest.mark.parametrize("rows,V,K", SIZES)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rest", [False, True])
def test_loss_and_gradient(B, rows, V, K, kind, rest):
    for n, (pad, shift, t, bits, tau) in enumerate(((None, 0, torch.float32, 32, 1.0), (1, 1, torch.bfloat16, 64, 2.0))):
        z, T, I, t_lse = inputs(rows, V, K, kind, V + K + n, t, tau, pad=pad, shift=shift)
        if K > 2:
            I[:, K // 2] = -1 if n == 0 else V + 5          # absent
            I[0, K - 1] = I[0, 0]                           # twice: the first counts
        if V > 50 and K < V // 2:
            z[:, V // 3: V // 3 + 9] = float("-inf")        # masked classes
            I[(I >= V // 3) & (I < V // 3 + 9)] = -1
        idx = I.to(torch.int64) if bits == 64 else I
        d = desc(B, V, K, kind, t, bits, tau)
        weight = torch.rand(rows, generator=gen(V), device="cuda") + 0.5
        tl = t_lse + 0.05 if rest else None                 # the rest keeps at least 1 - exp(-0.05)
        loss, stat, dz = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda"), matrix(rows, V, KINDS[kind], pad=pad, shift=shift)
        B.fw_distill_forward(d, z, T, idx, loss, stat=stat, t_lse=tl, weight=weight, dZ=dz)
        want = reference(z, T, I, tau, tl, weight)
        check(loss, want[0], want[3])
        check_stat(stat, want[1])
        check(dz, want[2], want[4], HALF[KINDS[kind]])
        assert surround_kept(dz)
        # the loss alone is the same number; the backward call agrees with the definition on its own
        loss2 = torch.empty(rows, device="cuda")
        B.fw_distill_forward(d, z, T, idx, loss2, t_lse=tl, weight=weight)
        assert torch.equal(loss, loss2)
        dz2 = matrix(rows, V, KINDS[kind], pad=pad, shift=shift)
        B.fw_distill_backward(d, z, T, idx, stat, dz2, t_lse=tl, weight=weight)
        check(dz2, want[2], stat_bound(want), HALF[KINDS[kind]])
        assert surround_kept(dz2)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rest", [False, True])
def test_special_rows(B, kind, rest):
    """Rows of weight 0 that hold NaN, rows without entries, without any mass, with NaN, with +inf; the others as ever."""
    V, K, rows = 3001, 20, 9
    z, T, I, t_lse = inputs(rows, V, K, kind, 77)
    weight = torch.full((rows,), 0.5, device="cuda")
    z[1] = float("nan")
    weight[1] = 0
    I[2] = -1
    z[3] = float("-inf")
    z[4, 5] = float("nan")
    z[5, 6] = float("inf")
    T[6, 3:] = float("-inf")
    z[7, I[7, 1].long()] = float("-inf")
    tl = t_lse + 0.1 if rest else None
    loss, stat, dz = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda"), matrix(rows, V, KINDS[kind])
    d = desc(B, V, K, kind)
    B.fw_distill_forward(d, z, T, I, loss, stat=stat, t_lse=tl, weight=weight, dZ=dz)
    rowsum = dz.to(F64).abs().sum(1)
    for r in (1, 3) + (() if rest else (2,)):
        assert float(loss[r]) == 0 and float(rowsum[r]) == 0
    for r in (4, 5):
        assert bool(torch.isnan(loss[r])) and bool(torch.isnan(dz[r].float()).all())
    assert float(loss[7]) == float("inf") and bool(torch.isfinite(dz[7].float()).all())
    keep = [0, 2, 6, 7, 8]
    want = reference(z[keep], T[keep], I[keep], 1.0, None if tl is None else tl[keep], weight[keep])
    check(loss[keep], want[0], want[3])
    check(dz[keep], want[2], want[4], HALF[KINDS[kind]])
    # the backward call, and in place
    dz2 = matrix(rows, V, KINDS[kind])
    B.fw_distill_backward(d, z, T, I, stat, dz2, t_lse=tl, weight=weight)
    assert float(dz2.to(F64).abs().sum(1)[[1, 3]].sum()) == 0 and bool(torch.isnan(dz2[[4, 5]].float()).all())
    zz = put(z, KINDS[kind])
    B.fw_distill_backward(d, zz, T, I, stat, zz, t_lse=tl, weight=weight)
    assert torch.equal(zz[keep], dz2[keep])
    zz = put(z, KINDS[kind])
    B.fw_distill_forward(d, zz, T, I, loss, t_lse=tl, weight=weight, dZ=zz)
    assert torch.equal(zz[keep], dz[keep])


@pytest.mark.parametrize("V,rows", [(9000, 700), (50000, 150), (131072, 90)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_many_rows_with_gaps(B, V, rows, kind):
    """Several rows for every cluster, some of weight 0 among them, in runs of one to three."""
    z, T, I, t_lse = inputs(rows, V, 70, kind, V, pad=None)
    I[::5, 60:] = I[::5, :10]                               # classes named twice
    weight = torch.where(torch.rand(rows, generator=gen(4), device="cuda") < 0.4, 0.0, 1.5)
    d = desc(B, V, 70, kind)
    loss, stat, dz, dz2 = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda"), matrix(rows, V, KINDS[kind], pad=None), matrix(rows, V, KINDS[kind], pad=None)
    B.fw_distill_forward(d, z, T, I, loss, stat=stat, t_lse=t_lse + 0.05, weight=weight, dZ=dz)
    B.fw_distill_backward(d, z, T, I, stat, dz2, t_lse=t_lse + 0.05, weight=weight)
    for r0 in range(0, rows, 50):
        r = slice(r0, r0 + 50)
        want = reference(z[r], T[r], I[r], 1.0, t_lse[r] + 0.05, weight[r])
        check(loss[r], want[0], want[3])
        check_stat(stat[r], want[1])
        check(dz[r], want[2], want[4], HALF[KINDS[kind]])
        check(dz2[r], want[2], stat_bound(want), HALF[KINDS[kind]])
    assert surround_kept(dz) and surround_kept(dz2)


@pytest.mark.parametrize("V", [40000, 200003])
def test_in_place_long_rows(B, V):
    """dZ over Z where several CTAs share a row, and where the row is read twice."""
    for kind in ("f32", "bf16"):
        z, T, I, t_lse = inputs(40, V, 50, kind, V, pad=None)
        d = desc(B, V, 50, kind)
        loss, stat, dz = torch.empty(40, device="cuda"), torch.empty(40, 2, device="cuda"), matrix(40, V, KINDS[kind], pad=None)
        B.fw_distill_forward(d, z, T, I, loss, stat=stat, t_lse=t_lse, dZ=dz)
        zz = put(z, KINDS[kind], pad=None)
        B.fw_distill_forward(d, zz, T, I, loss, t_lse=t_lse, dZ=zz)
        assert torch.equal(zz, dz)
        B.fw_distill_backward(d, z, T, I, stat, dz, t_lse=t_lse)
        zz = put(z, KINDS[kind], pad=None)
        B.fw_distill_backward(d, zz, T, I, stat, zz, t_lse=t_lse)
        assert torch.equal(zz, dz)


def test_confident_student(B):
    """Nearly all of the student's mass on a named class: the rest's mass (1e-12 of the whole) is what it is, not what is left
    of a difference."""
    V, K = 5000, 8
    z, T, I, t_lse = inputs(4, V, K, "f32", 3)
    z.scatter_(1, I[:, :1].long(), 40.0)
    loss, stat, dz = torch.empty(4, device="cuda"), torch.empty(4, 2, device="cuda"), matrix(4, V, torch.float32)
    B.fw_distill_forward(desc(B, V, K, "f32"), z, T, I, loss, stat=stat, t_lse=t_lse, dZ=dz)
    want = reference(z, T, I, 1.0, t_lse)
    check(loss, want[0], want[3])
    check_stat(stat, want[1])
    check(dz, want[2], want[4], HALF[torch.float32])


@pytest.mark.parametrize("V,K", [(1500, 2), (42440, 45)])
def test_little_named_mass(B, V, K):
    """A flat teacher: nearly all mass, its and the student's, on the classes that are not named (P, Q of 1e-4 to 1e-2).  The loss is
    then of the size of P: its terms p log(p / q) within E, and p_t (log(1 - P) - log(1 - Q)) within 4 E (P + Q)."""
    tau = 4.0
    z, T, I, t_lse = inputs(20, V, K, "f32", V, tau=tau)
    loss, dz = torch.empty(20, device="cuda"), matrix(20, V, torch.float32)
    B.fw_distill_forward(desc(B, V, K, "f32", tau=tau), z, T, I, loss, t_lse=t_lse, dZ=dz)
    want = reference(z, T, I, tau, t_lse)
    logp = T.to(F64) / tau - t_lse.to(F64)[:, None]
    p = logp.exp()
    logq = z.to(F64).gather(1, I.long()) / tau - torch.logsumexp(z.to(F64) / tau, 1, keepdim=True)
    E = 2.0 ** -17 + 16 * 2.0 ** -24 * t_lse.to(F64).abs()          # t / tau - t_lse is rounded at the size of t_lse
    bound = (p * (logp.abs() + logq.abs() + 1)).sum(1) * E + 4 * E * (p.sum(1) + logq.exp().sum(1))
    assert bool(((loss.to(F64) - want[0]).abs() <= bound).all())
    check(dz, want[2], want[4], HALF[torch.float32])


def test_gradient_against_differences(B):
    """Central differences of the loss in 64 bits, step 1e-5: truncation 1e-10 of the terms."""
    V, K, tau, h = 30, 5, 2.0, 1e-5
    z, T, I, t_lse = inputs(2, V, K, "f32", 8, tau=tau)
    for tl in (None, t_lse):
        dz, loss = matrix(2, V, torch.float32), torch.empty(2, device="cuda")
        B.fw_distill_forward(desc(B, V, K, "f32", tau=tau), z, T, I, loss, t_lse=tl, dZ=dz)
        z64 = z.to(F64).contiguous()
        num = torch.empty_like(z64)
        for i in range(V):
            up, down = z64.clone(), z64.clone()
            up[:, i] += h
            down[:, i] -= h
            num[:, i] = (reference(up, T, I, tau, tl)[0] - reference(down, T, I, tau, tl)[0]) / (2 * h)
        assert float((dz.to(F64) - num).abs().max()) <= 2e-5 * float(num.abs().max())


def test_repeated_other_stream_and_graph(B):
    rows, V, K = 65, 33333, 40
    z, T, I, t_lse = inputs(rows, V, K, "bf16", 13, pad=None)
    d = desc(B, V, K, "bf16")
    loss, stat, dz, dz2 = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda"), matrix(rows, V, torch.bfloat16), matrix(rows, V, torch.bfloat16)

    def call(stream):
        B.fw_distill_forward(d, z, T, I, loss, stat=stat, t_lse=t_lse, dZ=dz, stream=stream)
        B.fw_distill_backward(d, z, T, I, stat, dz2, t_lse=t_lse, stream=stream)

    call(0)
    torch.cuda.synchronize()
    first = [t.clone() for t in (loss, stat, dz, dz2)]
    call(0)
    assert all(torch.equal(a, b) for a, b in zip(first, (loss, stat, dz, dz2)))
    g = captured(call)
    z.copy_(inputs(rows, V, K, "bf16", 14)[0])
    g.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (loss, stat, dz, dz2)]
    assert not torch.equal(got[0], first[0])
    call(0)
    assert all(torch.equal(a, b) for a, b in zip(got, (loss, stat, dz, dz2)))


@pytest.mark.parametrize("rows,V,K", [(5, 300, 4), (4, 2048, 100), (3, 9000, 64), (3, 50021, 33), (2, 131072, 64), (3, 3000, 300), (1, 300001, 7)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("gap,tau", [(60.0, 1.0), (150.0, 1.0), (900.0, 1.0), (30.0, 0.0625)])
def test_one_named_class_far_ahead(B, rows, V, K, kind, gap, tau):
    """A student sure of a class that the teacher names: the others' mass q_t is beyond fp32, their loss and gradient are not.

    In 64 bits with logarithms, so that no gap is too wide.  Bounds beyond those of the file's head, relative to an element:
    the forward call's share of the others E (1 + a / 8), a its distance from their largest; the backward call's E and, for an
    exponential of z / tau - stat in fp32, 2 u |stat| (stat's roundings), 2 u |z / tau| and 4 u of the difference.  q_t itself
    is below e^-40 of p_t here."""
    u, E, half = 2.0 ** -24, 2.0 ** -17 if V <= 131072 else 2.0 ** -15, HALF[KINDS[kind]]
    z, T, I, t_lse = inputs(rows, V, K, kind, V + K, tau=tau, pad=None)
    z.scatter_add_(1, I[:, :1].long(), torch.full((rows, 1), gap, device="cuda").to(z.dtype))
    tl = t_lse + 0.05
    weight = torch.rand(rows, generator=gen(V), device="cuda") + 0.5
    d = desc(B, V, K, kind, tau=tau)
    loss, stat = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    fwd, bwd = matrix(rows, V, KINDS[kind]), matrix(rows, V, KINDS[kind])
    B.fw_distill_forward(d, z, T, I, loss, stat=stat, t_lse=tl, weight=weight, dZ=fwd)
    B.fw_distill_backward(d, z, T, I, stat, bwd, t_lse=tl, weight=weight)

    at, w = I.long(), weight.to(F64)[:, None]
    zz, t, tl = z.to(F64) / tau, T.to(F64) / tau, tl.to(F64)[:, None]
    lse = torch.logsumexp(zz, 1, keepdim=True)
    rest = torch.logsumexp(zz.scatter(1, at, float("-inf")), 1, keepdim=True)
    logp, logq, log_qt = t - tl, zz.gather(1, at) - lse, rest - lse
    assert float(log_qt.max()) < -40
    p = logp.exp()
    pt = 1 - p.sum(1, keepdim=True)
    dp = p * (E + 8 * u * (t.abs() + tl.abs()))
    dpt = dp.sum(1, keepdim=True) + 4 * u
    mag, lt = logp.abs() + logq.abs(), pt.log().abs() + log_qt.abs()
    want = w * ((p * (logp - logq)).sum(1, keepdim=True) + pt * (pt.log() - log_qt))
    bound = w * ((dp * (1 + mag) + p * (E + 4 * u * (2 + mag))).sum(1, keepdim=True) + dpt * (lt + 1) + pt * (E + 4 * u) * (2 + lt))
    check(loss, want[:, 0], bound[:, 0])
    check_stat(stat, torch.cat((lse, rest), 1))

    share = (zz - rest).exp()
    others = w / tau * (log_qt.exp() - pt) * share
    named = w / tau * (logq.exp() - p)
    far = zz.scatter(1, at, float("-inf")).amax(1, keepdim=True) - zz
    of_stat = lambda v, s: E + 2 ** -21 + u * (2 * s.abs() + 2 * v.abs() + 4 * (v - s).abs())  # noqa: E731
    for got, rel, rel_named in ((fwd, E * (1 + far / 8), E * (1 + (zz.amax(1, keepdim=True) - zz.gather(1, at)) / 8)),
                                (bwd, of_stat(zz, rest), of_stat(zz.gather(1, at), lse))):
        dz = others.scatter(1, at, named)
        allowed = (others.abs() * (rel + dpt / pt)).scatter(1, at, w / tau * (logq.exp() * rel_named + dp))
        check(got, dz, allowed, half)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [9000, 50021, 131072])
def test_named_classes_over_their_neighbours(B, V, kind):
    """256 named classes a row, spread over every warp's stores: each holds its own gradient, forward and backward, row after row."""
    rows, K = 300, 256
    g = gen(V)
    z = put(torch.randn(rows, V, generator=g, device="cuda") * 2, KINDS[kind], pad=None)
    I = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(rows)]).to(torch.int32)
    T = torch.randn(rows, K, generator=g, device="cuda")
    d = desc(B, V, K, kind)
    loss, stat = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    for _ in range(3):
        dz, dz2 = matrix(rows, V, KINDS[kind], pad=None), matrix(rows, V, KINDS[kind], pad=None)
        B.fw_distill_forward(d, z, T, I, loss, stat=stat, dZ=dz)
        B.fw_distill_backward(d, z, T, I, stat, dz2)
        for r0 in range(0, rows, 50):
            r = slice(r0, r0 + 50)
            want = reference(z[r], T[r], I[r], 1.0)
            check(dz[r], want[2], want[4], HALF[KINDS[kind]])
            check(dz2[r], want[2], stat_bound(want), HALF[KINDS[kind]])


@pytest.mark.parametrize("rows,V,K,shift", [(5, 1000, 20, 0), (7, 5000, 20, 0), (6, 131072, 256, 0), (4, 5000, 300, 0), (3, 5000, 20, 1)])
@pytest.mark.parametrize("ignored", [8.0, 200.0, float("inf"), float("nan")])
@pytest.mark.parametrize("tau", [1.0, 0.0625])
def test_the_ignored_logit_of_a_repeated_class(B, rows, V, K, shift, ignored, tau):
    """A class named twice counts with its first logit, however large the second one is: the rest of the row is relative to the
    largest logit that counts."""
    z, T, I, t_lse = inputs(rows, V, K, "f32", V + K, tau=tau, pad=shift or None, shift=shift)
    z.mul_(tau)                                             # a student as flat as the teacher is at tau
    T.mul_(tau)
    I[:, K - 1] = I[:, 0]
    I[1:, K // 2] = I[1:, 3]
    T[:, K - 1] = T[:, 0] + ignored
    T[1:, K // 2] = T[1:, 3] + 2 * ignored
    T, I = T.contiguous(), I.contiguous()
    d = desc(B, V, K, "f32", tau=tau)
    loss, stat = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    dz, dz2 = (matrix(rows, V, torch.float32, pad=shift or None, shift=shift) for _ in range(2))
    B.fw_distill_forward(d, z, T, I, loss, stat=stat, dZ=dz)
    B.fw_distill_backward(d, z, T, I, stat, dz2)
    counted = T.clone()
    counted[:, K - 1] = 0                                   # what the definition leaves out anyway
    counted[1:, K // 2] = 0
    want = reference(z, counted, I, tau)
    assert float(want[0].min()) > 0
    check(loss, want[0], want[3])
    check(dz, want[2], want[4], HALF[torch.float32])
    check(dz2, want[2], stat_bound(want), HALF[torch.float32])


def by_logs(z, T, I, tau, t_lse=None, weight=None):
    """loss and dZ in 64 bits with their bounds, every logarithm relative to the largest logit that it is about: for logits so far
    apart, or so far from 0, that 64 bits do not hold them beside each other.  Entries are present and not repeated; some class
    is not named, and some logit of a row is finite."""
    rows, V = z.shape
    u, E = 2.0 ** -24, 2.0 ** -17 if V <= 131072 else 2.0 ** -15
    zz, t, at = z.to(F64) / tau, T.to(F64) / tau, I.long()
    w = torch.ones(rows, 1, dtype=F64, device="cuda") if weight is None else weight.to(F64)[:, None]
    m = zz.amax(1, keepdim=True)
    lse = (zz - m).exp().sum(1, keepdim=True).log()                      # relative to m
    hidden = zz.scatter(1, at, float("-inf"))
    om = hidden.amax(1, keepdim=True)
    om = torch.where(om == float("-inf"), m, om)                         # nobody there: no share, whatever it is relative to
    share = (hidden - om).exp()
    mass = share.sum(1, keepdim=True)
    log_qt = om - m + mass.log() - lse
    share = torch.where(mass > 0, share / mass, 0)
    logq = zz.gather(1, at) - m - lse
    if t_lse is None:
        logp, pt = torch.log_softmax(t, 1), torch.zeros(rows, 1, dtype=F64, device="cuda")
        dp = logp.exp() * E + 4 * u
        dpt = 0 * pt
    else:
        tl = t_lse.to(F64)[:, None]
        logp = t - tl
        pt = (1 - logp.exp().sum(1, keepdim=True)).clamp(min=0)
        dp = logp.exp() * (E + 8 * u * (t.abs() + tl.abs())) + 4 * u
        dpt = dp.sum(1, keepdim=True) + 4 * u
    p = logp.exp()
    mag, lt = logp.abs() + logq.abs(), torch.where(pt > 0, pt.log().abs() + log_qt.abs(), 0)
    loss = w * ((p * (logp - logq)).sum(1, keepdim=True) + torch.where(pt > 0, pt * (pt.log() - log_qt), 0))
    dloss = w * ((dp * (1 + mag) + p * (E + 4 * u * (2 + mag))).sum(1, keepdim=True) + dpt * (lt + 1) + pt * (E + 4 * u) * (2 + lt))
    A = p.sum(1, keepdim=True) + pt
    excess = A * log_qt.exp() - pt
    dexcess = A * log_qt.exp() * E * (1 + log_qt.abs().clamp(max=1e4) / 8) + dpt
    far = (om - zz).abs().clamp(max=1e4)
    dz = (w / tau * excess * share).scatter(1, at, w / tau * (A * logq.exp() - p))
    ddz = (w / tau * (dexcess + excess.abs() * E * (1 + far / 8)) * share).scatter(
        1, at, w / tau * (A * logq.exp() * E * (1 + logq.abs().clamp(max=1e4) / 8) + dpt * logq.exp() + dp))
    return loss[:, 0], dz, dloss[:, 0], ddz


# rows of each kernel: of a warp, of one CTA and of a cluster that stay, of a CTA for itself (many entries; not aligned), read twice
EACH_KERNEL = [(5, 1000, 20, 0), (7, 5000, 20, 0), (3, 131072, 64, 0), (4, 5000, 300, 0), (3, 5000, 20, 1), (3, 700, 20, 1), (2, 150001, 20, 1)]


@pytest.mark.parametrize("rows,V,K,shift", EACH_KERNEL)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("where", ["row", "most", "named", "one named", "others"])
@pytest.mark.parametrize("rest,tau", [(False, 1.0), (True, 1.0), (True, 4.0)])
def test_lowest_finite_value(B, rows, V, K, shift, kind, where, rest, tau):
    """torch.finfo.min as a mask is a logit like any other: a row of it alone is a flat one, beside others it has no mass, and
    where the teacher has some the loss is as large as the formula makes it."""
    z, T, I, t_lse = inputs(rows, V, K, kind, V + K, tau=tau, pad=shift or None, shift=shift)
    low, at = torch.finfo(KINDS[kind]).min, I.long()
    if where == "row":
        z[:] = low
    elif where == "most":
        z[:, torch.arange(V, device="cuda") % 7 != 3] = low
        z[:, at[0, 0]] = 1.0                                # some class has mass whatever V is
    elif where == "named":
        z.scatter_(1, at, low)
    elif where == "one named":
        z.scatter_(1, at[:, 1:2], low)
    else:
        keep = z.gather(1, at)
        z[:] = low
        z.scatter_(1, at, keep)
    tl = t_lse + 0.05 if rest else None
    weight = torch.rand(rows, generator=gen(V), device="cuda") * 0.5 + 0.25
    d = desc(B, V, K, kind, tau=tau)
    loss, loss2, dz = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), matrix(rows, V, KINDS[kind], pad=shift or None, shift=shift)
    B.fw_distill_forward(d, z, T, I, loss, t_lse=tl, weight=weight, dZ=dz)
    B.fw_distill_forward(d, z, T, I, loss2, t_lse=tl, weight=weight)
    want = by_logs(z, T, I, tau, tl, weight)
    check(loss, want[0], want[2])
    assert torch.equal(loss, loss2)
    check(dz, want[1], want[3], HALF[KINDS[kind]])


@pytest.mark.parametrize("rows,V,K,shift", EACH_KERNEL)
def test_lowest_finite_value_of_the_teacher(B, rows, V, K, shift):
    """A teacher whose named logits are all the lowest finite value is flat over them."""
    z, T, I, _ = inputs(rows, V, K, "f32", V, pad=shift or None, shift=shift)
    T[:] = torch.finfo(torch.float32).min
    loss, dz = torch.empty(rows, device="cuda"), matrix(rows, V, torch.float32, pad=shift or None, shift=shift)
    B.fw_distill_forward(desc(B, V, K, "f32"), z, T, I, loss, dZ=dz)
    want = by_logs(z, torch.zeros_like(T), I, 1.0)
    check(loss, want[0], want[2])
    check(dz, want[1], want[3], HALF[torch.float32])


STAT = 1024.0                                              # statistics up to here are taken as they are (kFineStat)


def gradient_alone(B, z, T, I, tau, tl, weight, kind, pad, shift):
    """The backward call after a forward call that leaves the statistics: into a matrix of its own and over the logits."""
    rows, V = z.shape
    d = desc(B, V, T.shape[1], kind, tau=tau)
    loss, stat = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    B.fw_distill_forward(d, z, T, I, loss, stat=stat, t_lse=tl, weight=weight)
    dz, zz = matrix(rows, V, KINDS[kind], pad=pad, shift=shift), put(z, KINDS[kind], pad=pad, shift=shift)
    B.fw_distill_backward(d, z, T, I, stat, dz, t_lse=tl, weight=weight)
    B.fw_distill_backward(d, zz, T, I, stat, zz, t_lse=tl, weight=weight)
    assert surround_kept(dz) and surround_kept(zz)
    assert torch.equal(dz.nan_to_num(nan=7.0), zz.nan_to_num(nan=7.0))
    return dz, stat


def check_alone(dz, want, tau, half):
    """The forward call's bound and, where the statistics are used, their two roundings: 2 u 1024 of each exponential.  An exponential
    below 2^-126 is 0 (fw_rows.cuh, ex2); it is multiplied by weight / tau, weight <= 1.5, and by masses and reciprocals of sums of at
    most 1."""
    relative = 2 * 2.0 ** -24 * STAT
    check(dz, want[1], want[3] + relative * (want[1].abs() + want[3] * 2.0 ** 17) + 1.5 / tau * 2.0 ** -126, half)


@pytest.mark.parametrize("rows,V,K,shift", EACH_KERNEL + [(1200, 9000, 20, 0), (300, 50021, 33, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("what", ["row", "others", "offset", "mask", "tau"])
def test_gradient_alone_where_the_statistics_are_coarse(B, rows, V, K, shift, kind, rest, what):
    """log sum exp(Z / tau) of -3e38 or 1e5 in fp32 says nothing of how many classes share the mass, or little: the gradient alone
    is still the formula's.  Every third row is an ordinary one, every seventh has weight 0."""
    tau = 2.0 ** -10 if what == "tau" else 1.0
    z, T, I, t_lse = inputs(rows, V, K, kind, V + K, tau=tau, pad=shift or None, shift=shift)
    if what == "tau":
        T = (T * tau).contiguous()                          # a teacher of ordinary size beside a student scaled by 1000
        t_lse = torch.logsumexp(T.to(F64) / tau, 1).float() + 0.5
    coarse = torch.arange(rows, device="cuda") % 3 != 1
    low, at = torch.finfo(KINDS[kind]).min, I.long()
    new = z.clone()
    if what == "row":
        new[:] = low
    elif what == "others":
        new[:] = low
        new.scatter_(1, at, z.gather(1, at))
    elif what == "offset":
        new = (z.float() - 1e5).to(z.dtype)
    elif what == "mask":
        new = (z.float() - 1e9).to(z.dtype)
    z[coarse] = new[coarse]
    weight = torch.rand(rows, generator=gen(V), device="cuda") + 0.5
    weight[6::7] = 0
    tl = t_lse + 0.05 if rest else None
    pad = shift or None
    dz, stat = gradient_alone(B, z, T, I, tau, tl, weight, kind, pad, shift)
    assert not bool((dz[6::7] != 0).any())
    for r0 in range(0, rows, 60):
        r = slice(r0, r0 + 60)
        check_alone(dz[r], by_logs(z[r], T[r], I[r], tau, None if tl is None else tl[r], weight[r]), tau, HALF[KINDS[kind]])


def test_gradient_alone_where_the_statistics_pass_fp32(B):
    """Logits of 1e38 over a tau of 1/16: the statistics are infinite, the gradient is not."""
    for rows, V, K, shift in EACH_KERNEL:
        z, T, I, _ = inputs(rows, V, K, "f32", V, pad=shift or None, shift=shift)
        z[0], z[1, : V // 2] = -1e38, 1e38
        dz, stat = gradient_alone(B, z, T, I, 0.0625, None, None, "f32", shift or None, shift)
        assert bool(torch.isinf(stat[:2, 0]).all())
        want = by_logs(z, T, I, 0.0625)
        check_alone(dz, want, 0.0625, HALF[torch.float32])
