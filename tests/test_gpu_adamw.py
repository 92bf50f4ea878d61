"""AdamW over many tensors against its formula in 64 bits.

Error bounds (u = 2^-24).  m: the clipped gradient and its product with the rounded 1 - beta1 have three roundings, the rounded beta1 one, the
sum one: 4 u of the two terms' sizes.  v: two clipped factors, the rounded 1 - beta2, two products, the sum: 7 u, taken as 8.  The clipping factor is a
rounded quotient (u) of the norm: sums of at most 64 squares of a thread and lanes in fp32, halved by the root: 32 u more.  P: its
product and difference have 3 u of P; of the update, m's error and 8 u / 2 of v's, the root and the quotient (2 ulp each: 8 u), three
rounded factors and a sum: 16 u, taken as 20.
Codes of 8-bit states: the kernel's m and sqrt(v) are as far off as above; the choice of a code grows with the value, so the code
lies between the choices for the value less and plus its error.
"""
import pytest
import torch

from optest_util import F64, U, captured, gen

pytestmark = pytest.mark.gpu

BLOCK = 256
SIZES = [1, 255, 256, 257, 5000, 3, 70000]


@pytest.fixture(scope="module")
def B():
    from paper_2010_01546_b200 import binding, build
    build.build_library()
    return binding


def mix(x):
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


GRID = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()          # codes that are not negative, in order


def choose(value, scale, chance, square):
    """The code for value >= 0 (held over scale) by the rule of the header."""
    grid = GRID.to(value.device)
    y = (value / scale).clamp(0, 448)
    at = (torch.searchsorted(grid, y, right=True) - 1).clamp(max=125)
    lo, hi = grid[at], grid[at + 1]
    if not square:
        return torch.where((y - lo) / (hi - lo) + chance.double() / 65536 >= 1, hi, lo)
    code = torch.where(y.square() - lo.square() > (chance.double() + 0.5) / 65536 * (hi.square() - lo.square()), hi, lo)
    return torch.where((value > 0) & (code == 0), grid[1], code)


def scale_of(top):
    return torch.exp2(torch.ceil(torch.log2(top / 448)).clamp(min=-100))


def tensors(sizes, seed, shift=0, half=()):
    """Parameters and gradients; shift: elements past an aligned address."""
    g = gen(seed)
    make = lambda n, dt, s: torch.empty(n + shift, dtype=dt, device="cuda")[shift:].copy_(torch.randn(n, generator=g, device="cuda") * s)  # noqa: E731
    P = [make(n, torch.float32, 0.1) for n in sizes]
    G = [make(n, torch.bfloat16 if i in half else torch.float32, 0.01) for i, n in enumerate(sizes)]
    return P, G


def split(flat, sizes):
    out, at = [], 0
    for n in sizes:
        out.append(flat[at:at + n])
        at += -(-n // BLOCK) * BLOCK
    return out


def states(B, opt, sizes):
    """m and v as 64-bit numbers, tensor by tensor, and the whole arrays' scales."""
    m, v = opt.state(B.FW_A_M).to(F64), opt.state(B.FW_A_V).to(F64)
    if opt.desc.state == B.FW_E4M3:
        m = (m.view(-1, BLOCK) * opt.state(B.FW_A_M_SCALE).to(F64)[:, None]).view(-1)
        v = (v.view(-1, BLOCK) * opt.state(B.FW_A_V_SCALE).to(F64)[:, None]).view(-1).square()
    return split(m, sizes), split(v, sizes)


def formula(P, G, m, v, t, lr, decay, c, beta1, beta2, eps):
    """New m, v, P and the size of m's terms."""
    f = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    eps, lr, decay = f(eps), f(lr), f(decay)
    g = G.to(F64) * c
    m1, v1 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    size = beta1 * m.abs() + (1 - beta1) * g.abs()
    rate = lr / (1 - beta1 ** t) / ((v1 / (1 - beta2 ** t)).sqrt() + eps)
    return m1, v1, P.to(F64) * (1 - lr * decay) - rate * m1, size, rate


def check_step(B, opt, P, G, copies, before, t, sizes, lr, decay, c=1.0, clip_err=0.0, beta1=0.9, beta2=0.999, eps=1e-8, seed=0):
    """P, copies and states after step t; before: (P, m, v) clones from before it."""
    P0, m0, v0 = before
    got_m, got_v = states(B, opt, sizes)
    flat_m, flat_v = opt.state(B.FW_A_M).to(F64), opt.state(B.FW_A_V).to(F64)
    at = 0
    for i, n in enumerate(sizes):
        m1, v1, p1, size, rate = formula(P0[i], G[i], m0[i], v0[i], t, lr, decay[i], c, beta1, beta2, eps)
        em, ev = (4 * U + clip_err) * size, (8 * U + 2 * clip_err) * v1
        assert bool(((P[i].to(F64) - p1).abs() <= 3 * U * P0[i].to(F64).abs() + rate * (em + (20 * U + clip_err) * m1.abs()) + U * p1.abs()).all()), i
        if copies and copies[i] is not None:
            assert torch.equal(copies[i], P[i].bfloat16())
        if opt.desc.state == B.FW_F32:
            assert bool(((got_m[i] - m1).abs() <= em).all()) and bool(((got_v[i] - v1).abs() <= ev).all()), i
        else:
            # the blocks of this tensor
            k = -(-n // BLOCK)
            pad = lambda x: torch.nn.functional.pad(x, (0, k * BLOCK - n)).view(k, BLOCK)  # noqa: E731
            x = torch.arange(at, at + k * BLOCK, device="cuda")
            chance = mix(x ^ mix((seed ^ (t * 0x9E3779B9)) & 0xFFFFFFFF)).view(k, BLOCK)
            r1 = v1.sqrt()
            er = (ev / (2 * r1)).nan_to_num(0) + 4 * U * r1
            for name, val, err, ch, square, flat in (("m", m1.abs(), em, chance & 0xFFFF, False, flat_m), ("v", r1, er, chance >> 16, True, flat_v)):
                s = opt.state(B.FW_A_M_SCALE if name == "m" else B.FW_A_V_SCALE).to(F64)[at // BLOCK:at // BLOCK + k]
                top, most = pad(val).amax(1), pad(err).amax(1)
                assert bool(((s >= scale_of(top - most)) & (s <= scale_of(top + most))).all()), (i, name)
                code = flat[at:at + k * BLOCK].view(k, BLOCK)
                lo = choose((pad(val) - pad(err)).clamp(min=0), s[:, None], ch, square)
                hi = choose(pad(val) + pad(err), s[:, None], ch, square)
                assert bool(((code.abs() >= lo) & (code.abs() <= hi)).all()), (i, name)
                # the bounds leave few choices open: a code is 1/16 of its number or more, the clipped gradient 37 u off, and m is 1/19 of
                # its terms' sizes where the gradient has just turned: 2 x 16 x 37 u x 19 = 1.4e-3 of them
                assert float((lo != hi).double().mean()) < 1e-2 or n < 5000
                if name == "m":
                    assert bool((code.sign() * pad(m1).sign() >= 0).all())
                assert bool((code.view(-1)[n:] == 0).all())                      # behind the last element
        at += -(-n // BLOCK) * BLOCK


def begin(B, opt, sizes, seed):
    """States of a training run under way."""
    g = gen(seed)
    for field, value in ((B.FW_A_M, 0.003), (B.FW_A_V, 1e-4)):
        x = opt.state(field)
        for t in split(x, sizes):
            r = torch.randn(t.numel(), generator=g, device="cuda")
            if opt.desc.state == B.FW_E4M3:
                t.copy_((r * 100 if field == B.FW_A_M else r.abs() * 100).clamp(-448, 448))
            else:
                t.copy_(r * value if field == B.FW_A_M else r.abs() * value)
    if opt.desc.state == B.FW_E4M3:
        opt.state(B.FW_A_M_SCALE).copy_(torch.full_like(opt.state(B.FW_A_M_SCALE), 2.0 ** -15, dtype=torch.float32))
        opt.state(B.FW_A_V_SCALE).copy_(torch.full_like(opt.state(B.FW_A_V_SCALE), 2.0 ** -13, dtype=torch.float32))


@pytest.mark.parametrize("kind", ["f32", "e4m3"])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("clip", [None, 0.3, 1e6, float("inf")])
def test_steps(B, kind, shift, clip):
    sizes = SIZES
    P, G = tensors(sizes, 3, shift, half=(1, 4, 5))
    copies = [torch.empty_like(p, dtype=torch.bfloat16) if i % 2 else None for i, p in enumerate(P)]
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    opt = B.AdamW(P, copies=copies, decay=decay, state=B.FW_E4M3 if kind == "e4m3" else B.FW_F32, seed=77, beta2=0.99)
    assert int(opt.state(B.FW_A_STEP)) == 0 and not bool(opt.state(B.FW_A_M).float().any()) and not bool(opt.state(B.FW_A_V).float().any())
    norm = torch.empty(1, device="cuda") if clip else None
    for t in (1, 2, 3, 4):
        if t == 3:
            begin(B, opt, sizes, 5)
        before = ([p.clone() for p in P], *states(B, opt, sizes))
        opt.step(G, 1e-2, max_norm=clip or 0.0, norm_out=norm)
        c = 1.0
        if clip:
            want = float(sum(g.to(F64).square().sum() for g in G).sqrt())
            assert abs(float(norm) - want) <= 33 * U * want
            c = min(1.0, clip / want)
        check_step(B, opt, P, G, copies, before, t, sizes, 1e-2, decay, c, 33 * U if c < 1 else 0.0, beta2=0.99, seed=77)
        assert int(opt.state(B.FW_A_STEP)) == t
        for g in G:
            g.neg_()
    assert opt.sync_status() == B.FW_OK


@pytest.mark.parametrize("n", [441, 881])
def test_hundreds_of_tensors(B, n):
    """More tensors than one launch takes; the same results as tensors by themselves."""
    sizes = [1 + (37 * i) % 700 for i in range(n)]
    P, G = tensors(sizes, 8, half=set(range(0, n, 3)))
    alone = [p.clone() for p in P[-3:]]
    opt, norm = B.AdamW(P, decay=0.1), torch.empty(1, device="cuda")
    before = ([p.clone() for p in P], *states(B, opt, sizes))
    opt.step(opt.grads(G), 1e-3, max_norm=0.5, norm_out=norm)
    want = float(sum(g.to(F64).square().sum() for g in G).sqrt())
    assert abs(float(norm) - want) <= 33 * U * want
    check_step(B, opt, P, G, None, before, 1, sizes, 1e-3, [0.1] * n, min(1.0, 0.5 / want), 33 * U)
    few = B.AdamW(alone, decay=0.1)
    opt2 = B.AdamW([p.clone() for p in before[0]], decay=0.1)
    opt2.step(G, 1e-3)
    few.step(G[-3:], 1e-3)
    assert all(torch.equal(a, b) for a, b in zip(opt2.params[-3:], alone))
    assert int(opt.state(B.FW_A_STEP)) == int(opt2.state(B.FW_A_STEP)) == 1


def test_slow_averages_move(B):
    """8-bit averages of a gradient that has changed: a step moves them by 1/100 of the way, a code is 1/16 to 1/8 apart.  A step's
    choice has the variance f (1 - f) d^2 with f d at most 0.01 v and codes' squares d at most 0.266 v apart; steps count beta2^2 each: 0.01
    x 0.266 / (1 - 0.98) v^2 = 0.133 v^2 in all, 0.365 v; 16384 elements: 0.29 %, and 1.5 % is five times that."""
    n = 16384
    P = [torch.zeros(n, device="cuda")]
    G = [torch.where(torch.arange(n, device="cuda") % 2 == 0, 1.0, -0.61)]
    opt = B.AdamW(P, state=B.FW_E4M3, beta1=0.99, beta2=0.99, seed=5)
    for _ in range(60):
        opt.step(G, 0.0)
    G[0].mul_(3)
    for _ in range(40):
        opt.step(G, 0.0)
    m, v = (x[0] for x in states(B, opt, [n]))
    g = G[0].double() / 3
    want_m = g * ((1 - 0.99 ** 60) * 0.99 ** 40 + 3 * (1 - 0.99 ** 40))
    want_v = g.square() * ((1 - 0.99 ** 60) * 0.99 ** 40 + 9 * (1 - 0.99 ** 40))
    assert abs(float((m / want_m).mean()) - 1) < 0.015 and abs(float((v / want_v).mean()) - 1) < 0.015


@pytest.mark.parametrize("kind", ["f32", "e4m3"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 1e30])
def test_a_step_that_is_left_out(B, kind, bad):
    sizes = [300, 5000]
    P, G = tensors(sizes, 4)
    C = [p.bfloat16() for p in P]
    opt = B.AdamW(P, copies=C, state=B.FW_E4M3 if kind == "e4m3" else B.FW_F32)
    opt.step(G, 1e-3, max_norm=1.0)
    before = [x.clone() for x in P + C] + [opt.state(f).view(torch.uint8).clone() for f in (B.FW_A_M, B.FW_A_V, B.FW_A_STEP)]
    keep = G[1][17].clone()
    G[1][17] = bad
    opt.step(G, 1e-3, max_norm=1.0)
    assert opt.sync_status() == B.FW_WARN_NONFINITE and opt.sync_status() == B.FW_OK
    after = [*P, *C] + [opt.state(f).view(torch.uint8) for f in (B.FW_A_M, B.FW_A_V, B.FW_A_STEP)]
    assert all(torch.equal(a, b) for a, b in zip(before, after))
    G[1][17] = keep
    opt.step(G, 1e-3, max_norm=1.0)
    assert int(opt.state(B.FW_A_STEP)) == 2 and opt.sync_status() == B.FW_OK
    # without a bound on the norm it goes into P
    if bad != bad:
        G[1][17] = bad
        opt.step(G, 1e-3)
        assert bool(P[1][17].isnan()) and int(P[1].isnan().sum()) == 1 and opt.sync_status() == B.FW_OK


def test_zero_gradients_and_new_states(B):
    for kind in (B.FW_F32, B.FW_E4M3):
        P, G = tensors([1000], 9)
        G[0][:600] = 0
        p0 = P[0].clone()
        opt = B.AdamW(P, state=kind)
        norm = torch.empty(1, device="cuda")
        opt.step(G, 1e-2, max_norm=1e9)
        assert torch.equal(P[0][:600], p0[:600])
        # the first step is lr in size, whatever the gradient
        assert bool(((P[0] - p0)[600:] + 1e-2 * G[0][600:].sign()).abs().max() < 2e-5)
        G[0].zero_()
        opt.step(G, 1e-2, max_norm=1.0, norm_out=norm)
        assert float(norm) == 0 and bool(P[0].isfinite().all())


def test_captured_steps_count_on(B):
    """A replayed step is the next step, with a schedule that lives on the device."""
    for kind in (B.FW_F32, B.FW_E4M3):
        P, G = tensors([513, 4000], 12)
        P2 = [p.clone() for p in P]
        s = torch.cuda.Stream()
        factor, norm = torch.ones(1, device="cuda"), torch.empty(1, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            opt = B.AdamW(P, stream=s.cuda_stream, state=kind, decay=0.01)
            grads = opt.grads(G)
            opt.step(grads, 1e-2, lr_factor=factor, max_norm=0.2, norm_out=norm)
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                opt.step(grads, 1e-2, lr_factor=factor, max_norm=0.2, norm_out=norm)
        for k in range(3):
            with torch.cuda.stream(s):
                factor.fill_(0.5 ** k)
            with torch.cuda.stream(s):
                g.replay()
        s.synchronize()
        assert int(opt.state(B.FW_A_STEP)) == 4
        ref = B.AdamW(P2, state=kind, decay=0.01)
        for lr in (1e-2, 1e-2, 5e-3, 2.5e-3):
            ref.step(G, lr, max_norm=0.2)
        torch.cuda.synchronize()
        for a, b in zip(P, P2):                                       # lr times factor is exact here but for the last bits of 1e-2
            assert bool(((a - b).abs() <= 4 * U * b.abs() + 1e-2 * 64 * U).all())
        del g


def test_repeated_and_two_streams(B):
    """The same bits every time; two objects on two streams at once."""
    outs = []
    for _ in range(2):
        P, G = tensors([200000, 777], 21)
        Q, H = tensors([150000, 31], 22, half=(0,))
        a, b = torch.cuda.Stream(), torch.cuda.Stream()
        torch.cuda.synchronize()
        x, y = B.AdamW(P, stream=a.cuda_stream, state=B.FW_E4M3), B.AdamW(Q, stream=b.cuda_stream)
        gx, gy = x.grads(G), y.grads(H)
        for _ in range(5):
            x.step(gx, 1e-3, max_norm=0.1)
            y.step(gy, 1e-3, max_norm=0.1)
        torch.cuda.synchronize()
        outs.append([t.clone() for t in P + Q] + [x.state(f).view(torch.uint8).clone() for f in range(4)])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_checkpoint(B):
    """States written into a new object: the next steps are the same."""
    for kind in (B.FW_F32, B.FW_E4M3):
        P, G = tensors([3000, 50], 31)
        a = B.AdamW(P, state=kind, seed=3)
        for _ in range(3):
            a.step(G, 1e-3)
        Q = [p.clone() for p in P]
        b = B.AdamW(Q, state=kind, seed=3)
        for f in (B.FW_A_M, B.FW_A_V, B.FW_A_STEP) + ((B.FW_A_M_SCALE, B.FW_A_V_SCALE) if kind == B.FW_E4M3 else ()):
            b.state(f).copy_(a.state(f))
        a.step(G, 1e-3)
        b.step(G, 1e-3)
        assert all(torch.equal(p, q) for p, q in zip(P, Q))


def test_elements_beyond_31_bits(B):
    n = (1 << 31) + 300
    P, G = torch.full((n,), 0.5, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    G[-500:] = torch.linspace(-1, 1, 500, device="cuda")
    p0, g0 = P[-1000:].clone(), G[-1000:].clone()
    opt = B.AdamW([P], state=B.FW_E4M3)
    opt.step([G], 1e-2)
    m1, v1, p1, size, rate = formula(p0, g0, torch.zeros_like(p0, dtype=F64), torch.zeros_like(p0, dtype=F64), 1, 1e-2, 0.0, 1.0, 0.9, 0.999, 1e-8)
    assert bool(((P[-1000:].to(F64) - p1).abs() <= 4 * U * p1.abs() + rate * 24 * U * size).all())
    assert bool((P[:1000] == 0.5).all()) and bool((P[1 << 30:(1 << 30) + 1000] == 0.5).all())
    s = opt.state(B.FW_A_M_SCALE).float()
    assert float(s[:4].max()) == 2.0 ** -100 and float(s[-1]) > 2.0 ** -40


@pytest.mark.parametrize("kind", ["f32", "e4m3"])
def test_gradients_that_explode(B, kind):
    """The clipping factor is 1e-21 and less, whose square is no fp32 number; the clipped gradients are ordinary ones."""
    sizes = [1000, 300]
    P, G = tensors(sizes, 41)
    for x in G:
        x.mul_(1e18)
    opt = B.AdamW(P, state=B.FW_F32 if kind == "f32" else B.FW_E4M3)
    norm = torch.empty(1, device="cuda")
    want = torch.cat([x.to(F64) for x in G]).norm()
    for t in (1, 2):
        m0, v0 = states(B, opt, sizes)
        before = ([p.clone() for p in P], m0, v0)
        opt.step(G, 1e-2, max_norm=1e-4, norm_out=norm)
        assert abs(float(norm) / float(want) - 1) <= 32 * U
        check_step(B, opt, P, G, None, before, t, sizes, 1e-2, [0.0, 0.0], 1e-4 / float(want), 33 * U)
    assert opt.sync_status() == B.FW_OK


@pytest.mark.parametrize("kind", ["f32", "e4m3"])
def test_gradients_whose_squares_are_subnormal(B, kind):
    """v is a subnormal number (half a step of them is 2^-150), whose root still matters beside an eps of 1e-30."""
    g = gen(42)
    G = 1e-19 * (1 + torch.rand(3000, generator=g, device="cuda")) * (1 - 2 * torch.randint(0, 2, (3000,), generator=g, device="cuda"))
    P = torch.zeros(3000, device="cuda")
    opt = B.AdamW([P], state=B.FW_F32 if kind == "f32" else B.FW_E4M3, eps=1e-30)
    opt.step([G], 1e-2)
    zero = torch.zeros(3000, dtype=F64, device="cuda")
    _, v1, p1, _, _ = formula(P * 0, G, zero, zero, 1, 1e-2, 0.0, 1.0, 0.9, 0.999, 1e-30)
    assert bool(((P.to(F64) - p1).abs() <= p1.abs() * (0.5 * 2.0 ** -150 / v1 + 24 * U)).all())


@pytest.mark.parametrize("kind", ["f32", "e4m3"])
@pytest.mark.parametrize("bad", [1e21, 1e25, float("-inf"), float("nan")])
def test_an_overflow_stays_in_its_element(B, kind, bad):
    """Without clipping, a gradient whose scaled square passes fp32, an infinity, a NaN: the other elements of its block, those that never
    had a gradient among them, go the way that they go where its gradients are 0.  P there: a v of infinity takes no step (m is finite), what is
    not finite in m goes into P."""
    n, at = 700, 300
    P, G = tensors([n], 51)
    G[0][256:400:3] = 0                                              # of the same block, v = 0
    G[0][at] = 0
    Q, p0 = [P[0].clone()], P[0].clone()
    state = B.FW_F32 if kind == "f32" else B.FW_E4M3
    a, b = B.AdamW(P, state=state, seed=9), B.AdamW(Q, state=state, seed=9)
    others = torch.arange(n, device="cuda") != at
    fields = (B.FW_A_M, B.FW_A_V) + ((B.FW_A_M_SCALE, B.FW_A_V_SCALE) if kind == "e4m3" else ())
    for t in range(1, 6):
        H = G[0].clone()
        H[at] = 0.01 if t != 2 else bad                              # the step before it and those behind: an ordinary gradient
        if t < 2:
            H[at] = 0
        before = P[0].clone()
        a.step([H], 1e-2)
        b.step(G, 1e-2)
        assert torch.equal(P[0][others], Q[0][others]) and bool(P[0][others].isfinite().all()), t
        for f in fields:
            x, y = a.state(f).view(torch.uint8), b.state(f).view(torch.uint8)
            if f in (B.FW_A_M, B.FW_A_V):
                x, y = (v.view(-1, 4 if kind == "f32" else 1)[:n][others] for v in (x, y))
            assert torch.equal(x, y), (t, f)
        if t >= 2:
            m, v = a.state(B.FW_A_M).float()[at], a.state(B.FW_A_V).float()[at]
            if kind == "e4m3":
                assert bool(v.isnan()) and float(m) == 0             # the codes of a v that is not finite
            if abs(bad) < float("inf"):
                assert torch.equal(P[0][at], before[at]) and torch.equal(P[0][at], p0[at])
            else:
                assert bool(P[0][at].isnan())
    zero = (G[0] == 0) & others
    moved = (G[0] != 0) & others
    assert torch.equal(P[0][zero], p0[zero]) and bool((P[0][moved] != p0[moved]).all())
    assert a.sync_status() == B.FW_OK
