"""Log-probabilities, policy loss and preference loss against their formulas in 64 bits.

Error bounds (u = 2^-24).  A logit's distance from the largest is rounded once, times log2(e) / tau (two more roundings): 3 u of the
scaled distance x, and ex2 is off by 2^-22 = 4 u: an exponential is off by (3 x + 6) u of itself.  A row's sum is of positive terms,
added in at most 64 + 32 + 16 steps a thread, lane and warp at the sizes here, each step with a rescaling (8 u): under 1000 u; x
e^-x is below 1/e, so that x adds 3 u to the sum.  A share q is off by (1010 + 3 x) u of itself, logp by 1010 u + 3 u |logp|.  16-bit gradients
add half a step; an exponential below 2^-126 is 0: 2^-125 times a slope over tau.  The loss's parts are exponentials of differences of log-probabilities: relative errors of |dlogp| u and a few more.
"""
import pytest
import torch

from optest_util import F64, HALF, U, captured, gen, matrix, put, surround_kept

pytestmark = pytest.mark.gpu

KINDS = {"f32": torch.float32, "bf16": torch.bfloat16}
SUM = 1010 * U
SIZES = [(1, 1), (3, 2), (5, 7), (4, 64), (33, 100), (9, 257), (70, 1000), (3, 4096), (5, 4097), (6, 5003), (3, 32000), (4, 50257), (2, 131072),
         (2, 262147), (1, 1 << 20)]
PADS = [dict(pad=None), dict(pad=0), dict(pad=1, shift=1), dict(pad=3, shift=2)]


@pytest.fixture(scope="module")
def B():
    from paper_2010_01546_b200 import binding, build
    build.build_library()
    return binding


def desc(B, V, kind, **kw):
    return B.fw_logprob_desc_default(V, z_dtype=B.FW_F32 if kind == "f32" else B.FW_BF16, **kw)


def inputs(rows, V, kind, seed, spread=3.0, **lay):
    g = gen(seed)
    Z = put(torch.randn(rows, V, generator=g, device="cuda") * spread, KINDS[kind], **lay)
    id = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int64)
    id[::3] = Z.float().argmax(1)[::3]                     # a class with much of the mass too
    return Z, id


class Ref:
    def __init__(self, Z, id, tau):
        z = Z.to(F64) / tau
        self.tau, self.z, self.id = tau, z, id
        self.q = torch.softmax(z, 1)
        self.logq = torch.log_softmax(z, 1)
        at = id.clamp(0, z.shape[1] - 1)[:, None]
        self.logp = self.logq.gather(1, at).flatten()
        # the others by themselves: of a class with most of the mass, and of logits whose logarithms take nothing on
        e = torch.exp(z - z.amax(1, keepdim=True))
        self.others = e.scatter(1, at, 0.0).sum(1) / e.sum(1)
        self.logp = torch.where(self.others < 0.4, torch.log1p(-self.others), self.logp)
        self.x = (z.amax(1, keepdim=True) - z)

    def grad(self, slope):
        dz = -self.q * (slope / self.tau)[:, None]
        return dz.scatter_(1, self.id.clamp(0, dz.shape[1] - 1)[:, None], (self.others * slope / self.tau)[:, None])

    def grad_bound(self, slope, slope_err, half):
        """slope_err: relative.  The class's own element is the others' mass: as far off as that."""
        size = self.grad(slope).abs()
        rel = (2 * SUM + 6 * U * self.x + 4 * U) + slope_err[:, None]
        rel = rel.scatter(1, self.id.clamp(0, rel.shape[1] - 1)[:, None], (2 * SUM + 6 * U * 50 + slope_err)[:, None])
        return size * (rel + half) + 2.0 ** -125 * (slope.abs().max() / self.tau + 1)


def logp_bound(r):
    """Of a class with most of the mass logp is of the size of the others' mass, and as far off as that."""
    return torch.where(r.others < 0.4, (2 * SUM + 150 * U) * r.logp.abs(), 2 * SUM + 4 * U * r.logp.abs())


@pytest.mark.parametrize("rows,V", SIZES)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_logprob(B, rows, V, kind):
    for n, lay in enumerate(PADS):
        tau = (1.0, 0.7, 2.5, 1.0)[n]
        Z, id = inputs(rows, V, kind, V + rows + n, **lay)
        if rows > 4:
            id[1], id[4] = -100, V                         # do not count
        bits = 64 if n % 2 else 32
        d = desc(B, V, kind, tau=tau, index_bits=bits)
        idt = id if bits == 64 else id.int()
        logp, stat = torch.full((rows,), 9.0, device="cuda"), torch.full((rows, 2), 9.0, device="cuda")
        B.fw_logprob_forward(d, Z, idt, logp, stat=stat)
        r = Ref(Z, id, tau)
        live = (id >= 0) & (id < V)
        assert bool(((logp.to(F64) - r.logp).abs() <= logp_bound(r))[live].all())
        assert bool((logp[~live] == 0).all()) and bool((stat[~live] == 0).all())
        assert torch.equal(stat[live, 0].to(F64), Z.to(F64).amax(1)[live])
        only = torch.empty_like(logp)
        B.fw_logprob_forward(d, Z, idt, only)
        assert torch.equal(only, logp)
        slope = torch.randn(rows, generator=gen(n), device="cuda")
        if rows > 2:
            slope[2] = 0
        # the gradient beside Z, laid out as Z is and otherwise, and in its place
        for out_lay in (lay, dict(pad=2)):
            dZ = matrix(rows, V, KINDS[kind], **out_lay)
            B.fw_logprob_backward(d, Z, idt, stat, slope, dZ)
            s = torch.where(live, slope.to(F64), 0)
            want, half = r.grad(s), HALF[dZ.dtype]
            assert bool(((dZ.to(F64) - want).abs() <= r.grad_bound(s, torch.full_like(s, 8 * U), half)).all())
            assert surround_kept(dZ)
            if rows > 2:
                assert bool((dZ[2] == 0).all())
        keep = dZ.clone()
        B.fw_logprob_backward(d, Z, idt, stat, slope, Z)
        assert torch.equal(Z, keep) and surround_kept(Z)


def policy_formula(r, live, old, ref, adv, w, low, high, kl):
    """loss, slope, and the sizes of their terms (in 64 bits)."""
    old, adv, w = old.to(F64), adv.to(F64), torch.where(live, w.to(F64), 0)
    ratio = torch.exp(r.logp - old)
    free, held = ratio * adv, ratio.clamp(1 - low, 1 + high) * adv
    loss, slope = -torch.minimum(free, held), torch.where(free <= held, -free, 0)
    size, ssize = loss.abs(), slope.abs()
    if kl:
        k = ref.to(F64) - r.logp
        loss = loss + kl * (torch.expm1(k) - k)
        slope = slope - kl * torch.expm1(k)
        # a change of logp by e moves exp(k) - 1 - k by e |exp(k) - 1|
        size = size + kl * (torch.expm1(k) - k)
        ssize = ssize + kl * torch.expm1(k).abs()
    near = ((ratio - (1 - low)).abs() < 1e-3) | ((ratio - (1 + high)).abs() < 1e-3)     # either side of the bound may be taken
    return w * loss, w * slope, w.abs() * size, w.abs() * ssize, near


@pytest.mark.parametrize("rows,V", [(1, 1), (40, 9), (64, 1000), (33, 4099), (16, 50257), (5, 131072)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("kl", [0.0, 0.2])
def test_policy(B, rows, V, kind, kl):
    """Loss and slope move with logp's error e by e times their sizes (and kl (exp(k) - 1) e: taken with the slope's size)."""
    for n, lay in enumerate(PADS):
        Z, id = inputs(rows, V, kind, 7 * V + rows + n, **lay)
        g = gen(V + n)
        rnd = lambda: torch.randn(rows, generator=g, device="cuda")  # noqa: E731
        tau = 1.0 if n % 2 else 1.3
        r = Ref(Z, id, tau)
        old, ref, adv, w = r.logp.float() + 0.3 * rnd(), r.logp.float() + (0.5 * rnd() if n else 1e-3 * rnd()), rnd(), 1 + rnd().abs()
        adv[::5] = 0
        if rows > 4:
            id[1], w[3] = V + 5, 0
        live = (id >= 0) & (id < V) & (w != 0)
        d, p = desc(B, V, kind, tau=tau, index_bits=64), B.fw_policy_desc_default(clip_low=0.2, clip_high=0.3, kl=kl)
        out = {k: torch.full((rows,), 9.0, device="cuda") for k in ("loss", "logp", "dlogp")}
        stat, dZ = torch.full((rows, 2), 9.0, device="cuda"), matrix(rows, V, KINDS[kind], **lay)
        B.fw_policy_forward(d, p, Z, id, old, adv, out["loss"], logp_ref=ref if kl else None, weight=w, logp=out["logp"], stat=stat,
                            dlogp=out["dlogp"], dZ=dZ)
        loss, slope, size, ssize, near = policy_formula(r, live, old, ref, adv, w, 0.2, 0.3, kl)
        e = logp_bound(r) + 2 * U * (r.logp.abs() + old.to(F64).abs() + ref.to(F64).abs())
        assert bool(((out["logp"].to(F64) - r.logp).abs() <= logp_bound(r))[live].all()) and bool((out["logp"][~live] == 0).all())
        assert bool(((out["loss"].to(F64) - loss).abs() <= (size + ssize) * (2 * e + 16 * U) + 2.0 ** -140)[~near].all())
        # kl (exp(k) - 1) of a small k moves by kl e
        b = ssize * (2 * e + 16 * U) + kl * w.to(F64) * e
        assert bool(((out["dlogp"].to(F64) - slope).abs() <= b)[~near].all())
        for k in ("loss", "dlogp"):
            assert bool((out[k][~live] == 0).all())
        # the gradient of the slope that the call gave
        s = out["dlogp"].to(F64)
        assert bool(((dZ.to(F64) - r.grad(s)).abs() <= r.grad_bound(s, torch.full_like(s, 8 * U), HALF[dZ.dtype])).all())
        assert surround_kept(dZ)
        # without the gradient, where sums may be added in another order (each is within its bound of the formula); and the gradient from
        # what that call left
        again, only, st2, d2 = (torch.empty_like(x) for x in (out["loss"], out["logp"], stat, dZ.contiguous()))
        slope2 = torch.empty_like(again)
        B.fw_policy_forward(d, p, Z, id, old, adv, again, logp_ref=ref if kl else None, weight=w, logp=only, stat=st2, dlogp=slope2)
        assert bool(((only.to(F64) - r.logp).abs() <= logp_bound(r))[live].all()) and torch.equal(st2[:, 0], stat[:, 0])
        assert bool(((st2 - stat)[:, 1].abs() <= 2 * SUM * stat[:, 1]).all())
        assert bool(((again.to(F64) - loss).abs() <= (size + ssize) * (2 * e + 16 * U) + 2.0 ** -140)[~near].all())
        assert bool(((slope2.to(F64) - slope).abs() <= b)[~near].all())
        for x in (again, only, slope2, st2[:, 1]):
            assert bool((x[~live] == 0).all())
        s = slope2.to(F64)
        B.fw_logprob_backward(d, Z, id, st2, slope2, d2)
        assert bool(((d2.to(F64) - r.grad(s)).abs() <= r.grad_bound(s, torch.full_like(s, 8 * U), HALF[dZ.dtype])).all())
        # in place of the logits
        B.fw_policy_forward(d, p, Z, id, old, adv, again, logp_ref=ref if kl else None, weight=w, dZ=Z)      # the same order
        assert torch.equal(again, out["loss"]) and torch.equal(Z, dZ)


@pytest.mark.parametrize("rows,V", [(3, 25087), (3, 53761), (3, 111105), (2, 134906), (2, 222210), (2, 269825), (2, 444410), (2, 888830), (3, 1 << 20)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_policy_of_long_rows(B, rows, V, kind):
    """Rows about as long as one CTA, a cluster of two, four and eight hold, and longer than that."""
    test_policy(B, rows, V, kind, 0.2)


def test_policy_gradient_against_differences(B):
    """Central differences of the loss in 64 bits, step 1e-6: 1e-9 of the loss's terms; the kernel's slope is fp32."""
    rows, V, kl, tau = 12, 20, 0.3, 1.4
    Z, id = inputs(rows, V, "f32", 5)
    g = gen(6)
    old = Ref(Z, id, tau).logp.float() + 0.3 * torch.randn(rows, generator=g, device="cuda")
    ref = old + 0.4 * torch.randn(rows, generator=g, device="cuda")
    adv, w = torch.randn(rows, generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda")
    loss, dZ = torch.empty(rows, device="cuda"), torch.empty(rows, V, device="cuda")
    B.fw_policy_forward(desc(B, V, "f32", tau=tau, index_bits=64), B.fw_policy_desc_default(kl=kl), Z, id, old, adv, loss, logp_ref=ref, weight=w, dZ=dZ)

    def total(z):
        logp = torch.log_softmax(z / tau, 1).gather(1, id[:, None]).flatten()
        ratio, k = torch.exp(logp - old.to(F64)), ref.to(F64) - logp
        pg = -torch.minimum(ratio * adv.to(F64), ratio.clamp(1 - float(torch.tensor(0.2)), 1 + float(torch.tensor(0.2))) * adv.to(F64))
        return w.to(F64) * (pg + kl * (torch.expm1(k) - k))

    z, h = Z.to(F64).contiguous(), 1e-6
    num = torch.empty_like(z)
    for j in range(V):
        up, down = z.clone(), z.clone()
        up[:, j] += h
        down[:, j] -= h
        num[:, j] = (total(up) - total(down)) / (2 * h)
    assert float((dZ.to(F64) - num).abs().max()) <= 1e-5 * float(num.abs().max())


@pytest.mark.parametrize("V", [50, 1003, 5000, 70001, 131072])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_masks_and_values_that_are_none(B, V, kind):
    lowest = torch.finfo(KINDS[kind]).min
    Z, id = inputs(12, V, kind, V)
    Z[0] = float("-inf")                                   # no class has mass
    Z[1, 1:] = float("-inf"); id[1] = 0                    # one has all
    Z[2, ::2] = float("-inf"); id[2] = 1
    Z[3, 0] = float("-inf"); id[3] = 0                     # the class itself has none
    Z[4] = lowest                                          # flat
    Z[5, :] = lowest; Z[5, 3] = 1.0; id[5] = 3
    Z[6, V // 2] = float("nan")
    Z[7, V // 2] = float("inf")
    Z[8] = torch.linspace(-2, 2, V, device="cuda") * 1e4; id[8] = V - 1      # far apart
    Z[9, 5] = 200.0; id[9] = 7                             # the class is far behind
    Z[10] = -lowest                                        # flat at the largest
    id[11] = -1
    Z[11] = float("nan")                                   # not read
    d = desc(B, V, kind, index_bits=64)
    logp, stat = torch.empty(12, device="cuda"), torch.empty(12, 2, device="cuda")
    B.fw_logprob_forward(d, Z, id, logp, stat=stat)
    slope = torch.ones(12, device="cuda")
    dZ, loss, dZ2 = matrix(12, V, KINDS[kind]), torch.empty(12, device="cuda"), matrix(12, V, KINDS[kind])
    B.fw_logprob_backward(d, Z, id, stat, slope, dZ)
    # the policy loss of ratio 1 and advantage -1 has the slope 1; of the row whose class has no mass the ratio is 0
    old, adv, dl = torch.where(logp.isfinite(), logp, 0), -torch.ones(12, device="cuda"), torch.empty(12, device="cuda")
    B.fw_policy_forward(d, B.fw_policy_desc_default(), Z, id, old, adv, loss, dlogp=dl, dZ=dZ2)
    r = Ref(Z, id, 1.0)
    for k in (1, 2, 4, 5, 8, 9, 10):
        assert abs(float(logp[k]) - float(r.logp[k])) <= float(logp_bound(r)[k]) + 1e-30, k
        want = r.grad(slope.to(F64))[k]
        bound = r.grad_bound(slope.to(F64), torch.full((12,), 8 * U, device="cuda", dtype=F64), HALF[dZ.dtype])[k]
        assert bool(((dZ[k].to(F64) - want).abs() <= bound.nan_to_num(2.0 ** -125)).all()), k
        assert bool(((dZ2[k].to(F64) - want).abs() <= bound.nan_to_num(2.0 ** -125) + 2.0 ** -20 * want.abs()).all()), k
    for k in (0, 11):
        assert float(logp[k]) == 0 and bool((stat[k] == 0).all()) and bool((dZ[k] == 0).all()) and bool((dZ2[k] == 0).all()) and float(loss[k]) == 0
    assert float(logp[3]) == float("-inf") and bool(dZ[3].isfinite().all()) and float(dZ[3, 0]) == 1
    assert float(loss[3]) == pytest.approx(0.8) and float(dl[3]) == 0 and bool((dZ2[3] == 0).all())
    for k in (6, 7):
        assert bool(logp[k].isnan()) and bool(dZ[k].isnan().all()) and bool(loss[k].isnan()) and bool(dZ2[k].isnan().all()), k
    assert surround_kept(dZ) and surround_kept(dZ2)


def test_policy_bounds(B):
    """Each side of both bounds, by each sign of the advantage: which of the two is taken, and where the slope is 0."""
    V = 10
    Z, _ = inputs(8, V, "f32", 3)
    id = torch.arange(8, device="cuda")
    logp = Ref(Z, id, 1.0).logp
    ratio = torch.tensor([0.5, 0.5, 0.95, 0.95, 1.2, 1.2, 3.0, 3.0], device="cuda", dtype=F64)
    adv = torch.tensor([1.0, -1.0] * 4, device="cuda")
    old = (logp - ratio.log()).float()
    loss, dl = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    for high, want, slope in ((0.3, [-0.5, 0.8, -0.95, 0.95, -1.2, 1.2, -1.3, 3.0], [-0.5, 0, -0.95, 0.95, -1.2, 1.2, 0, 3.0]),
                              (float("inf"), [-0.5, 0.8, -0.95, 0.95, -1.2, 1.2, -3.0, 3.0], [-0.5, 0, -0.95, 0.95, -1.2, 1.2, -3.0, 3.0])):
        p = B.fw_policy_desc_default(clip_low=0.2, clip_high=high)
        B.fw_policy_forward(desc(B, V, "f32", index_bits=64), p, Z, id, old, adv, loss, dlogp=dl)
        assert loss.tolist() == pytest.approx(want, rel=1e-5) and dl.tolist() == pytest.approx(slope, rel=1e-5)


def preference_formula(logp, id, V, seq, ref, w, beta, margin, smooth, mean):
    """In 64 bits, answer by answer."""
    rows, answers = logp.numel(), seq.numel() - 1
    live = torch.ones(rows, dtype=torch.bool, device="cuda") if id is None else (id >= 0) & (id < V)
    sums, dlogp, of = [], torch.zeros(rows, dtype=F64, device="cuda"), []
    edge = [min(max(int(x), 0), rows) for x in seq]
    for s in range(answers):
        at = torch.arange(rows, device="cuda")
        mine = (at >= edge[s]) & (at < edge[s + 1]) & live
        n = max(int(mine.sum()), 1) if mean else 1
        sums.append(logp.to(F64)[mine].sum() / n)
        of.append((mine, n))
    sums = torch.stack(sums)
    gain = sums - (0 if ref is None else ref.to(F64))
    h = beta * (gain[0::2] - gain[1::2]) - margin
    soft = lambda x: x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))  # noqa: E731
    w = torch.ones(answers // 2, dtype=F64, device="cuda") if w is None else w.to(F64)
    d = w * beta * (smooth - torch.sigmoid(-h))
    for s, (mine, n) in enumerate(of):
        dlogp[mine] = (d[s // 2] if s % 2 == 0 else -d[s // 2]) / n
    return sums, w * ((1 - smooth) * soft(-h) + smooth * soft(h)), dlogp


@pytest.mark.parametrize("mean", [0, 1])
@pytest.mark.parametrize("edges", [[0, 5, 9], [0, 0, 4, 4, 7], [2, 300, 700, 701, 1500], [0, 3, 3, 3, 3, 9, 2000], [-5, 4, 10 ** 6]])
def test_preference(B, mean, edges):
    """Sums of fp32 numbers in 64 bits, rounded once; the loss and slope are of 64-bit arguments but for beta, margin and smooth, which
    are fp32 as they are held: a few u of themselves."""
    rows, V = 1503, 60
    g = gen(sum(edges) % 1000 + mean)
    seq = torch.tensor(edges, device="cuda", dtype=torch.int32)
    pairs = (len(edges) - 1) // 2
    f = lambda x: float(torch.tensor(x))  # noqa: E731
    for n in range(4):
        logp = -torch.rand(rows, generator=g, device="cuda") * 4
        id = torch.randint(-3, V + 3, (rows,), generator=g, device="cuda", dtype=torch.int64)
        w = torch.rand(pairs, generator=g, device="cuda") if n % 2 else None
        ref = None if n == 0 else 3 * torch.randn(2 * pairs, generator=g, device="cuda")
        kw = dict(beta=f(0.3), margin=f(0.4 if n > 1 else 0.0), smooth=f(0.1 if n > 2 else 0.0))
        loss, sums, dlogp = torch.full((pairs,), 9.0, device="cuda"), torch.full((2 * pairs,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
        use = None if n == 2 else id if n % 2 else id.int()
        d = desc(B, V, "f32", index_bits=64 if n % 2 else 32)
        B.fw_preference_loss(d, B.fw_preference_desc_default(mean=mean, **kw), logp, use, seq, loss, ref=ref, weight=w, sums=sums, dlogp=dlogp)
        s, want, slope = preference_formula(logp, None if use is None else id, V, seq, ref, w, **kw, mean=mean)
        for got, ex in ((sums, s), (loss, want), (dlogp, slope)):
            assert bool(((got.to(F64) - ex).abs() <= 4 * U * ex.abs() + 1e-12).all())
        only = torch.empty_like(loss)
        B.fw_preference_loss(d, B.fw_preference_desc_default(mean=mean, **kw), logp, use, seq, only, ref=ref, weight=w)
        assert torch.equal(only, loss)


def test_preference_far_apart(B):
    """Pairs that are decided: the loss goes to 0 or to the difference, the slope to 0 or beta; nothing overflows."""
    rows = 8
    logp = torch.tensor([-1e4, 0.0, 0.0, -1e4, -1.0, -1.0, float("-inf"), -1.0], device="cuda")
    seq = torch.arange(9, device="cuda", dtype=torch.int32)
    loss, dl, w = torch.empty(4, device="cuda"), torch.empty(rows, device="cuda"), torch.ones(4, device="cuda")
    d, p = desc(B, 5, "f32"), B.fw_preference_desc_default(beta=1.0)
    B.fw_preference_loss(d, p, logp, None, seq, loss, weight=w, dlogp=dl)
    assert loss.tolist() == pytest.approx([1e4, 0.0, 0.6931472, float("inf")])
    assert dl.tolist() == pytest.approx([-1.0, 1.0, 0.0, 0.0, -0.5, 0.5, -1.0, 1.0])
    w[3] = 0                                               # a pair that does not count
    B.fw_preference_loss(d, p, logp, None, seq, loss, weight=w, dlogp=dl)
    assert float(loss[3]) == 0 and dl[6:].tolist() == [0.0, 0.0]


def test_through_the_logits(B):
    """Logits -> log-probabilities -> preference -> gradient of the logits, against differences of the whole in 64 bits (step 1e-6:
    1e-9 of the loss; fp32 log-probabilities add 1e-5 of the largest element)."""
    V, rows = 11, 14
    Z, id = inputs(rows, V, "f32", 8)
    id[5] = -1
    seq = torch.tensor([0, 4, 7, 9, 13], device="cuda", dtype=torch.int32)
    ref = torch.randn(4, generator=gen(2), device="cuda")
    d, p = desc(B, V, "f32", index_bits=64, tau=1.2), B.fw_preference_desc_default(beta=0.5, smooth=0.1)
    logp, stat, dl, loss, dZ = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(2, device="cuda"), matrix(rows, V, torch.float32)
    B.fw_logprob_forward(d, Z, id, logp, stat=stat)
    B.fw_preference_loss(d, p, logp, id, seq, loss, ref=ref, dlogp=dl)
    B.fw_logprob_backward(d, Z, id, stat, dl, dZ)
    z = Z.to(F64).contiguous()

    def total(z):
        lp = torch.log_softmax(z / float(torch.tensor(1.2)), 1).gather(1, id.clamp(min=0)[:, None]).flatten()
        return float(preference_formula(lp, id, V, seq, ref, None, 0.5, 0.0, float(torch.tensor(0.1)), 0)[1].sum())
    num, h = torch.empty_like(z), 1e-6
    for i in range(z.numel()):
        v = float(z.view(-1)[i])
        z.view(-1)[i] = v + h
        up = total(z)
        z.view(-1)[i] = v - h
        num.view(-1)[i] = (up - total(z)) / (2 * h)
        z.view(-1)[i] = v
    assert float((dZ.to(F64) - num).abs().max()) <= 1e-5 * float(num.abs().max())
    assert bool((dZ[5] == 0).all()) and bool((dZ[13] == 0).all())


def test_captured_and_on_a_stream(B):
    rows, V = 40, 5000
    Z, id = inputs(rows, V, "bf16", 9)
    old, adv = torch.zeros(rows, device="cuda") - 5, torch.ones(rows, device="cuda")
    d, p = desc(B, V, "bf16", index_bits=64), B.fw_policy_desc_default()
    loss, dZ = torch.empty(rows, device="cuda"), matrix(rows, V, torch.bfloat16)
    g = captured(lambda s: B.fw_policy_forward(d, p, Z, id, old, adv, loss, dZ=dZ, stream=s))
    Z.mul_(0.5)
    want, wantd = torch.empty_like(loss), matrix(rows, V, torch.bfloat16)
    B.fw_policy_forward(d, p, Z, id, old, adv, want, dZ=wantd)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(loss, want) and torch.equal(dZ, wantd)


@pytest.mark.parametrize("pattern", ["none", "all", "tail", "power", "chance", "one"])
def test_rows_that_do_not_count(B, pattern):
    """Wherever they lie: their results are 0, the others' are what they are by themselves."""
    for rows, V, kind in ((2500, 5003, "bf16"), (700, 50257, "bf16"), (3001, 2100, "f32"), (400, 140000, "bf16"), (300, 70000, "f32"), (9000, 600, "bf16")):
        Z, id = inputs(rows, V, kind, V, pad=0)
        n = torch.arange(rows, device="cuda")
        out = {"none": n < 0, "all": n >= 0, "tail": n > rows // 3, "power": n % 16 != 5, "chance": torch.rand(rows, generator=gen(rows), device="cuda") < 0.4,
               "one": n != rows - 2}[pattern]
        w = torch.where(out & (n % 2 == 0), 0.0, 1.5)
        use = torch.where(out & (n % 2 == 1), -7, id)
        d = desc(B, V, kind, index_bits=64)
        old, adv = -torch.rand(rows, device="cuda") * 9, torch.randn(rows, device="cuda")
        got = [torch.full((rows,), 9.0, device="cuda") for _ in range(3)]
        stat, dZ = torch.full((rows, 2), 9.0, device="cuda"), matrix(rows, V, KINDS[kind], pad=0)
        B.fw_policy_forward(d, B.fw_policy_desc_default(), Z, use, old, adv, got[0], weight=w, logp=got[1], stat=stat, dlogp=got[2], dZ=dZ)
        r = Ref(Z, id, 1.0)
        live = ~out
        assert bool(((got[1].to(F64) - r.logp).abs() <= logp_bound(r))[live].all())
        s = got[2].to(F64)
        assert bool(((dZ.to(F64) - r.grad(s)).abs() <= r.grad_bound(s, torch.full_like(s, 8 * U), HALF[dZ.dtype])).all()) and surround_kept(dZ)
        for x in (*got, stat[:, 0], stat[:, 1]):
            assert bool((x[out] == 0).all())
        assert not bool(live.any()) or bool((got[0][live & (adv != 0)] != 0).any())
        # the same rows by the two calls that follow one another
        d2, lp, st2 = matrix(rows, V, KINDS[kind], pad=0), torch.full((rows,), 9.0, device="cuda"), torch.full((rows, 2), 9.0, device="cuda")
        B.fw_logprob_forward(d, Z, torch.where(out, -1, id), lp, stat=st2)
        assert bool(((lp.to(F64) - r.logp).abs() <= logp_bound(r))[live].all()) and bool((lp[out] == 0).all())
        B.fw_logprob_backward(d, Z, id, st2, got[2], d2)
        assert bool(((d2.to(F64) - r.grad(s)).abs() <= r.grad_bound(s, torch.full_like(s, 8 * U), HALF[dZ.dtype])).all()) and surround_kept(d2)
        del r, d2, dZ


def test_many_rows_and_far_offsets(B):
    """More rows than fit the chip at once; rows that begin beyond 2^31 elements."""
    for rows, V in ((30000, 70), (3000, 5001)):
        Z, id = inputs(rows, V, "bf16", 4, pad=None)
        d = desc(B, V, "bf16", index_bits=64)
        logp, stat = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
        B.fw_logprob_forward(d, Z, id, logp, stat=stat)
        r = Ref(Z, id, 1.0)
        assert bool(((logp.to(F64) - r.logp).abs() <= logp_bound(r)).all())
        s = torch.randn(rows, generator=gen(1), device="cuda")
        dZ = matrix(rows, V, torch.bfloat16)
        B.fw_logprob_backward(d, Z, id, stat, s, dZ)
        assert bool(((dZ.to(F64) - r.grad(s.to(F64))).abs() <= r.grad_bound(s.to(F64), torch.full_like(r.logp, 8 * U), HALF[dZ.dtype])).all())
        assert surround_kept(dZ)
        del r
    ld, V = (1 << 30) - 8, 300
    big = torch.empty(4 * ld, dtype=torch.bfloat16, device="cuda")
    Z = torch.as_strided(big, (4, V), (ld, 1))
    Z.copy_(torch.randn(4, V, generator=gen(3), device="cuda"))
    id = torch.tensor([0, 5, 17, 299], device="cuda")
    loss, logp = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    keep = Z.clone()
    d = desc(B, V, "bf16", index_bits=64)
    B.fw_policy_forward(d, B.fw_policy_desc_default(), Z, id, torch.zeros(4, device="cuda"), torch.ones(4, device="cuda"), loss, logp=logp, dZ=Z)
    r = Ref(keep, id, 1.0)
    assert bool(((logp.to(F64) - r.logp).abs() <= logp_bound(r)).all())
    s = -r.logp.exp()
    assert bool(((Z.to(F64) - r.grad(s)).abs() <= r.grad_bound(s, torch.full_like(s, 3e-4), 2.0 ** -8)).all())


@pytest.mark.parametrize("V", [100, 6000])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_a_kl_term_that_is_off(B, V, kind):
    """kl = 0 with a reference model's log-probabilities at hand (a schedule that begins at 0): the bits of the call without them, however
    far off they are."""
    Z, id = inputs(8, V, kind, 71)
    Z[1, id[1]] = float("-inf")                            # the class itself is masked: logp = -inf
    d, p = desc(B, V, kind, index_bits=64), B.fw_policy_desc_default(kl=0.0)
    ref = torch.tensor([-1.0, -2.0, 120.0, float("inf"), float("-inf"), float("nan"), 0.0, -500.0], device="cuda")
    old, adv, w = torch.full((8,), -3.0, device="cuda"), torch.linspace(-1, 1, 8, device="cuda"), torch.ones(8, device="cuda")
    outs = []
    for r in (None, ref):
        loss, dl, dZ = torch.empty(8, device="cuda"), torch.empty(8, device="cuda"), matrix(8, V, KINDS[kind])
        B.fw_policy_forward(d, p, Z, id, old, adv, loss, logp_ref=r, weight=w, dlogp=dl, dZ=dZ)
        only = torch.empty(8, device="cuda")
        B.fw_policy_forward(d, p, Z, id, old, adv, only, logp_ref=r, weight=w)
        outs.append((loss, dl, dZ, only))
    assert all(torch.equal(x, y) for x, y in zip(*outs)) and all(bool(x.isfinite().all()) for x in outs[1])


@pytest.mark.parametrize("high", [0.2, float("inf")])
def test_an_advantage_of_zero(B, high):
    """A ratio beyond fp32 times an advantage of 0 is 0, as the ratio itself is a number; a NaN among the logits stays one."""
    V = 50
    Z, id = inputs(6, V, "f32", 81)
    Z[4, 7] = float("nan")
    old = torch.tensor([-200.0, -1e30, float("-inf"), -3.0, -200.0, -200.0], device="cuda")
    adv = torch.tensor([0.0, 0.0, -0.0, 0.0, 0.0, 1.0], device="cuda")
    loss, dl, dZ = torch.empty(6, device="cuda"), torch.empty(6, device="cuda"), matrix(6, V, torch.float32)
    B.fw_policy_forward(desc(B, V, "f32", index_bits=64), B.fw_policy_desc_default(clip_high=high), Z, id, old, adv, loss, dlogp=dl, dZ=dZ)
    assert bool((loss[:4] == 0).all()) and bool((dl[:4] == 0).all()) and bool((dZ[:4] == 0).all())
    assert bool(loss[4].isnan()) and bool(dl[4].isnan()) and bool(dZ[4].isnan().all())
    if high < 1:
        assert float(loss[5]) == pytest.approx(-1.2) and float(dl[5]) == 0 and bool((dZ[5] == 0).all())
    else:
        assert float(loss[5]) == float("-inf") and float(dl[5]) == float("-inf")
