"""The operators of fine-tuning as they are used: a block between its norms under a policy loss or a preference loss, the gradients
transformed by whitened layers, one step of AdamW whose bf16 copies are the block's weights; and a token through the 8-bit path."""
import pytest
import torch

from optest_util import F64, U, gen, matrix, put

pytestmark = pytest.mark.gpu

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
CLIP, KL, BETA = 0.2, 0.1, 0.1


@pytest.fixture(scope="module")
def B():
    from paper_2010_01546_b200 import binding, build
    build.build_library()
    return binding


def rel(a, b):
    return float((a.to(F64) - b).norm() / b.norm())


class Step:
    """o (what the block before gave), x -> norm, gate, sum, norm -> gated block -> classifier -> loss of sampled classes, and all of it
    back; then the transform of both weight gradients and AdamW over weights and norms."""

    def __init__(self, B, loss, rows=384, M=192, N=320, V=500, stream=0):
        g = gen(77)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.B, self.kind, self.rows, self.M, self.N, self.V, self.stream = B, loss, rows, M, N, V, stream
        self.o, self.x = put(r(rows, M), BF16), put(r(rows, M), BF16)
        self.gate = torch.rand(rows, generator=g, device="cuda") + 0.5
        self.params = [r(N, M) * M ** -0.5, r(N, M) * M ** -0.5, 1 + 0.1 * r(M), 1 + 0.1 * r(M)]          # gated block, w_post, w_pre
        self.W = [w.to(BF16) for w in self.params[:2]]
        self.down, self.head = (r(M, N) * N ** -0.5).to(BF16), (r(V, M) * 0.08).to(BF16)
        self.id = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
        self.id[::7] = -100                                                                           # a prompt's tokens
        self.adv, self.weight = r(rows), torch.full((rows,), 1.0 / rows, device="cuda")
        self.delta, self.k = torch.randint(-1, 2, (rows,), generator=g, device="cuda") * 0.6, 0.3 * r(rows)
        lengths = [4, 2, 3, 3, 1, 4, 0, 3]
        seq = torch.tensor([5] + lengths * ((rows - 5) // 40 * 2), dtype=torch.int32).cumsum(0, dtype=torch.int32)
        self.seq, self.pairs = seq.cuda(), (seq.numel() - 1) // 2
        self.ref = 0.5 * r(2 * self.pairs)
        self.pair_weight = torch.full((self.pairs,), 1.0 / self.pairs, device="cuda")
        self.norm = B.fw_sandwich_desc_default(M)
        self.classes = B.fw_logprob_desc_default(V)
        self.policy = B.fw_policy_desc_default(clip_low=CLIP, clip_high=CLIP, kl=KL)
        self.preference = B.fw_preference_desc_default(beta=BETA)
        self.block = B.Gated(M, N, rows, grad=1, stream=stream)
        self.layers = [B.Layer(M, N, stream=stream, x_dtype=B.FW_BF16, prec=B.FW_PREC_BF16, alpha=0.9, beta=0.0, gamma=1.0) for _ in range(2)]
        e = lambda *s, t=BF16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        f = torch.float32
        self.h, self.y, self.rstd = e(rows, M), e(rows, M), e(rows, 2, t=f)
        self.H, self.Zg, self.Zu = e(rows, N), e(rows, N), e(rows, N)
        self.loss, self.logp, self.stat, self.slope = e(rows if loss == "policy" else self.pairs, t=f), e(rows, t=f), e(rows, 2, t=f), e(rows, t=f)
        self.dZ, self.dX, self.dx, self.d_o, self.dgate = e(rows, V), e(rows, M), e(rows, M), e(rows, M), e(rows, t=f)
        self.G, self.Gt = [e(N, M, t=f) for _ in range(2)], [e(N, M, t=f) for _ in range(2)]
        self.dw = [e(M, t=f) for _ in range(2)]
        self.scratch = e(B.fw_sandwich_scratch_bytes(self.norm), t=torch.uint8)
        self.old, self.behind = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        with torch.no_grad():
            logp = reference(self)[-1].float()
        self.old, self.behind = logp - self.delta, logp + self.k

    def optimizer(self, state):
        self.adam = self.B.AdamW(self.params, copies=self.W + [None, None], decay=[0.01, 0.01, 0.0, 0.0], stream=self.stream, state=state)
        self.grads = self.adam.grads(self.Gt + self.dw)
        self.gnorm = torch.empty(1, device="cuda")

    def gradients(self):
        B, st = self.B, self.stream
        w_post, w_pre = self.params[2:]
        B.fw_sandwich_forward(self.norm, self.o, self.x, w_pre, self.h, self.y, w_post=w_post, gate=self.gate, rstd=self.rstd, stream=st)
        self.block.forward(self.y, *self.W, self.H, self.Zg, self.Zu)
        Z = (self.h + self.H @ self.down.T) @ self.head.T
        if self.kind == "policy":
            B.fw_policy_forward(self.classes, self.policy, Z, self.id, self.old, self.adv, self.loss, logp_ref=self.behind, weight=self.weight,
                                logp=self.logp, stat=self.stat, dlogp=self.slope, dZ=self.dZ, stream=st)
        else:
            B.fw_logprob_forward(self.classes, Z, self.id, self.logp, stat=self.stat, stream=st)
            B.fw_preference_loss(self.classes, self.preference, self.logp, self.id, self.seq, self.loss, ref=self.ref, weight=self.pair_weight,
                                 dlogp=self.slope, stream=st)
            B.fw_logprob_backward(self.classes, Z, self.id, self.stat, self.slope, self.dZ, stream=st)
        d = self.dZ @ self.head
        self.block.backward(d @ self.down, self.y, *self.W, self.Zg, self.Zu, dX=self.dX, dWg=self.G[0], dWu=self.G[1])
        B.fw_sandwich_backward(self.norm, self.dX, self.o, self.h, w_pre, self.rstd, self.dx, self.d_o, w_post=w_post, gate=self.gate, dh=d,
                               dw_post=self.dw[0], dw_pre=self.dw[1], dgate=self.dgate, scratch=self.scratch, stream=st)

    def recursion(self):
        hs = [L.handle for L in self.layers]
        self.B.fw_group_cov_update(hs, [self.y] * 2, [self.rows] * 2, [self.M] * 2)
        self.B.fw_group_cond_reduce(hs, 3, 4)

    def update(self):
        for L, G, out in zip(self.layers, self.G, self.Gt):
            L.grad_transform(G, out)
        self.adam.step(self.grads, 1e-3, max_norm=0.01, norm_out=self.gnorm)

    def results(self):
        return [self.loss, self.slope, self.dx, self.d_o, self.dgate, *self.G, *self.dw, *self.Gt, self.gnorm, *self.params, *self.W]


def reference(s):
    """The loss and its gradients in 64 bits, without any rounding between (autograd of elementary operations)."""
    leaf = lambda t: t.to(F64).clone().requires_grad_(True)  # noqa: E731
    o, x, gate, w_post, w_pre, wg, wu = leaf(s.o), leaf(s.x), leaf(s.gate), leaf(s.params[2]), leaf(s.params[3]), leaf(s.W[0]), leaf(s.W[1])
    with torch.enable_grad():
        unit = lambda t: t * (t.square().mean(1, keepdim=True) + 1e-6).rsqrt()  # noqa: E731
        h = x + gate[:, None] * w_post * unit(o)
        y = unit(h) * w_pre
        a = y @ wg.T
        out = h + (a * torch.sigmoid(a) * (y @ wu.T)) @ s.down.to(F64).T
        at = s.id.clamp(min=0).long()[:, None]
        logp = torch.log_softmax(out @ s.head.to(F64).T, 1).gather(1, at).flatten()
        counts = s.id >= 0
        if s.kind == "policy":
            ratio, k = torch.exp(logp - s.old.to(F64)), s.behind.to(F64) - logp
            adv = s.adv.to(F64)
            loss = -torch.minimum(ratio * adv, ratio.clamp(1 - CLIP, 1 + CLIP) * adv) + KL * (torch.exp(k) - 1 - k)
            loss = torch.where(counts, loss * s.weight.to(F64), 0)
        else:
            total = torch.cat([torch.zeros(1, dtype=F64, device="cuda"), torch.where(counts, logp, 0).cumsum(0)])
            sums = total[s.seq[1:].long()] - total[s.seq[:-1].long()] - s.ref.to(F64)
            loss = torch.nn.functional.softplus(-BETA * (sums[::2] - sums[1::2])) * s.pair_weight.to(F64)
        loss.sum().backward()
    return loss.detach(), x.grad, o.grad, gate.grad, wg.grad, wu.grad, w_post.grad, w_pre.grad, logp.detach()


# Between input and gradient lie thirteen roundings to bf16 (h, y, Z, H, its product, the sum, logits, dZ, the products back, da and db, dX,
# d_o), each at most 2^-8 of what it rounds.  Seven of them act on the logits, of size 2: logp is off by 7 x 2^-8 x 2 = 0.055.  The ratio of
# the policy loss moves by that share, its KL slope by KL exp(k) times it, k below 1 as a rule: 0.065 (no ratio is within 0.18 of its bounds);
# a pair's h by BETA times eight tokens' 0.055, and its slope by that share.
SLOPE = {"policy": 0.065, "preference": BETA * 8 * 0.055}


@pytest.mark.parametrize("loss", ["policy", "preference"])
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_training_step(B, loss, state):
    s = Step(B, loss)
    s.optimizer(B.FW_F32 if state == "f32" else B.FW_E4M3)
    s.gradients()
    want, dx, d_o, dgate, dwg, dwu, dw_post, dw_pre, logp = reference(s)
    counts = s.id >= 0
    assert bool(((s.logp - logp).abs() <= 0.055 * 2)[counts].all())
    assert rel(s.loss, want) <= 2 * SLOPE[loss]
    assert bool((s.slope[~counts] == 0).all()) and bool((s.dZ[~counts] == 0).all())
    for got, ref in ((s.dx, dx), (s.d_o, d_o), (s.dgate, dgate), (s.G[0], dwg), (s.G[1], dwu), (s.dw[0], dw_post), (s.dw[1], dw_pre)):
        assert rel(got, ref) <= 13 * 2.0 ** -8 + SLOPE[loss]
    # the step with each layer's own transform (TF32 products, 2^-10 of the terms, 5e-3 as for the layers)
    s.recursion()
    before = [p.to(F64) for p in s.params]
    s.update()
    for L, G, Gt in zip(s.layers, s.G, s.Gt):
        Q = L.get(B.FW_F_QS).to(F64)
        assert float((Q - torch.eye(s.M, device="cuda")).abs().max()) > 0.01          # the recursion has acted
        assert rel(Gt, G.to(F64) @ Q) <= 5e-3
    grads = [G.to(F64) for G in s.Gt + s.dw]
    norm = torch.cat([G.flatten() for G in grads]).norm()
    assert abs(float(s.gnorm) / float(norm) - 1) <= 32 * U
    c = min(1.0, 0.01 / float(norm))
    for i, (p, p0, G) in enumerate(zip(s.params, before, grads)):
        # first step: m / (1 - beta1) = c G, root of v / (1 - beta2) = |c G|
        step = 1e-3 * c * G / ((c * G).abs() + 1e-8)
        assert bool((p.to(F64) - (p0 * (1 - (1e-5 if i < 2 else 0)) - step)).abs().max() <= 4 * U * p0.abs().max() + 1e-3 * 64 * U)
    for w, p in zip(s.W, s.params):
        assert torch.equal(w, p.bfloat16())
    # and the next step is made of the new weights
    s.gradients()
    _, dx, d_o, dgate, dwg, dwu, dw_post, dw_pre, _ = reference(s)
    for got, ref in ((s.dx, dx), (s.d_o, d_o), (s.dgate, dgate), (s.G[0], dwg), (s.G[1], dwu), (s.dw[0], dw_post), (s.dw[1], dw_pre)):
        assert rel(got, ref) <= 13 * 2.0 ** -8 + SLOPE[loss]
    assert s.block.sync_status() == B.FW_OK and s.adam.sync_status() == B.FW_OK


@pytest.mark.parametrize("loss", ["policy", "preference"])
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_training_steps_in_a_graph(B, loss, state):
    """A captured step replayed gives what plain calls give, bit for bit, beside another network's steps on another stream."""
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    runs = [Step(B, loss, stream=stream.cuda_stream) for _ in range(2)]
    beside = Step(B, loss, rows=200, stream=other.cuda_stream)
    for s in (*runs, beside):
        s.optimizer(B.FW_F32 if state == "f32" else B.FW_E4M3)
    torch.cuda.synchronize()

    def whole(s):
        s.gradients()
        s.recursion()
        s.update()

    def step(s):
        s.gradients()
        s.update()

    with torch.cuda.stream(stream):
        for s in runs:
            whole(s)
            step(s)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(runs[1])
    with torch.cuda.stream(other):
        whole(beside)
    for _ in range(3):
        with torch.cuda.stream(stream):
            graph.replay()
            step(runs[0])
        with torch.cuda.stream(other):
            step(beside)
    torch.cuda.synchronize()
    assert int(runs[0].adam.state(B.FW_A_STEP)) == int(runs[1].adam.state(B.FW_A_STEP)) == 5
    for a, b in zip(runs[0].results(), runs[1].results()):
        assert torch.equal(a, b)
    fields = [B.FW_A_M, B.FW_A_V] + ([B.FW_A_M_SCALE, B.FW_A_V_SCALE] if state == "e4m3" else [])
    for f in fields:
        assert torch.equal(*(s.adam.state(f).view(torch.uint8) for s in runs))
    for s in (*runs, beside):
        assert all(bool(torch.isfinite(t).all()) for t in s.results())
        assert s.adam.sync_status() == B.FW_OK and s.block.sync_status() == B.FW_OK
    del graph


@pytest.mark.parametrize("rows", [1, 3, 40])
def test_eight_bit_tokens(B, rows):
    """Norms around the block before to e4m3 with a scale a token, into the gated block with a scale for each output: what the block
    computes is the product of the values that the 8-bit numbers stand for (4 (M / 16 + 16) u of the terms' magnitudes), rounded to bf16."""
    M, N = 1024, 768
    g = gen(rows)
    o, x = (put(torch.randn(rows, M, generator=g, device="cuda"), BF16) for _ in range(2))
    gate, w_post = torch.rand(rows, generator=g, device="cuda"), 1 + 0.1 * torch.randn(M, generator=g, device="cuda")
    W = [torch.randn(N, M, generator=g, device="cuda") * M ** -0.5 for _ in range(2)]
    c = [w.abs().amax(1) / 448 for w in W]
    q = [(w / s[:, None]).to(E4M3) for w, s in zip(W, c)]
    h, y, ys, H = matrix(rows, M, BF16), matrix(rows, M, E4M3), torch.empty(rows, device="cuda"), matrix(rows, N, BF16)
    B.fw_sandwich_forward(B.fw_sandwich_desc_default(M, y_dtype=B.FW_E4M3), o, x, torch.ones(M, device="cuda"), h, y, w_post=w_post, gate=gate,
                          y_scale=ys)
    blk = B.Gated(M, N, x_dtype=B.FW_E4M3)
    blk.forward(y, *q, H, x_scale=ys, wg_scale=c[0], wu_scale=c[1])
    v = y.to(F64) * ys.to(F64)[:, None]
    w = [a.to(F64) * b.to(F64)[:, None] for a, b in zip(q, c)]
    a, b = v @ w[0].T, v @ w[1].T
    u = 4 * (M / 16 + 16) * U
    ea, eb = (u * (v.abs() @ k.abs().T) for k in w)
    f = a * torch.sigmoid(a)
    want = f * b
    e = 1.13 * ea * (b.abs() + eb) + f.abs() * eb + want.abs() * 2.0 ** -19
    assert bool(((H.to(F64) - want).abs() <= e + 2.0 ** -8 * (want.abs() + e)).all())
    # h as it is kept, and the norm of it
    t = o.to(F64)
    t = x.to(F64) + gate.to(F64)[:, None] * w_post.to(F64) * t * (t.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    assert bool(((h.to(F64) - t).abs() <= 2.0 ** -8 * t.abs() + 2.0 ** -16 * (x.to(F64).abs() + t.abs())).all())
    n = h.to(F64)
    n = n * (n.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    assert bool(((v - n).abs() <= 2.0 ** -4 * n.abs() * (1 + 2.0 ** -17) + 2.0 ** -10 * ys.to(F64)[:, None] + 2.0 ** -17 * n.abs()).all())


@pytest.mark.parametrize("kind", ["layer", "gated", "adamw"])
def test_objects_on_a_stream_beside_pending_work(B, kind):
    """Memory that the current stream has given up while its work on it is pending: an object on another stream is not given it, so what that work
    writes in the end is in none of its states."""
    s = torch.cuda.Stream()
    P = torch.randn(5000, device="cuda")
    p0, grad = P.clone(), torch.ones(5000, device="cuda")

    def make():
        if kind == "layer":
            return B.Layer(200, 64, stream=s.cuda_stream)
        return B.Gated(256, 512, 64, grad=1, stream=s.cuda_stream) if kind == "gated" else B.AdamW([P], stream=s.cuda_stream)

    torch.cuda.empty_cache()
    n = make().nbytes + 256                                          # (the kernels of its beginning are loaded)
    before = torch.empty(n, dtype=torch.uint8, device="cuda")
    at = before.data_ptr()
    before.fill_(0)                                                  # (as is this kernel)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    before.fill_(0x7F)
    del before
    x = make()
    s.synchronize()
    assert not torch.cuda.current_stream().query()                   # the sleep's length: else nothing was pending
    assert not at <= x.workspace.data_ptr() < at + n
    torch.cuda.synchronize()
    assert x.sync_status() == B.FW_OK
    if kind == "adamw":
        assert int(x.state(B.FW_A_STEP)) == 0 and not bool(x.state(B.FW_A_M).any()) and not bool(x.state(B.FW_A_V).any())
        x.step([grad], 1e-2)
        torch.cuda.synchronize()
        assert bool(((P - p0) + 1e-2).abs().max() < 1e-6 + 4 * 2.0 ** -24 * float(p0.abs().max()))
