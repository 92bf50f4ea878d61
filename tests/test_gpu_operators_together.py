"""The operators as they are used: a training step of a gated feed-forward block whose weights are whitened layers, and a token
through the 8-bit path."""
import pytest
import torch

from optest_util import F64, gen, matrix, put

pytestmark = pytest.mark.gpu

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def B():
    from paper_2010_01546_b200 import binding, build
    build.build_library()
    return binding


def rel(a, b):
    return float((a.to(F64) - b).norm() / b.norm())


class Step:
    """x, r -> norm -> gated block -> down projection -> classifier -> loss against a teacher's top logits, and all of it back; then
    moments of the norm's output, recursion, transform of both weight gradients and the parameter step."""

    def __init__(self, B, rows=384, M=192, N=320, V=500, K=12, stream=0):
        g = gen(99)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.B, self.rows, self.M, self.N, self.V, self.K, self.stream = B, rows, M, N, V, K, stream
        self.x, self.r = put(r(rows, M), BF16), put(r(rows, M), BF16)
        self.nw = 1 + 0.1 * r(M)
        self.master = [r(N, M) * M ** -0.5 for _ in range(2)]
        self.W = [w.to(BF16) for w in self.master]
        self.down, self.head = (r(M, N) * N ** -0.5).to(BF16), (r(V, M) * 0.3).to(BF16)
        teacher = 3 * r(rows, V)
        top, at = teacher.topk(K, 1)
        self.T, self.I, self.t_lse = top.to(BF16), at.to(torch.int32), torch.logsumexp(teacher, 1)
        self.weight = torch.full((rows,), 1.0 / rows, device="cuda")
        self.norm = B.fw_norm_desc_default(M, eps=1e-5)
        self.loss_desc = B.fw_distill_desc_default(V, K)
        self.block = B.Gated(M, N, rows, grad=1, stream=stream)
        self.layers = [B.Layer(M, N, stream=stream, x_dtype=B.FW_BF16, prec=B.FW_PREC_BF16, alpha=0.9, beta=0.0, gamma=1.0) for _ in range(2)]
        e = lambda *s, t=BF16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        self.s, self.y, self.rstd, self.H, self.Zg, self.Zu = e(rows, M), e(rows, M), e(rows, t=torch.float32), e(rows, N), e(rows, N), e(rows, N)
        self.loss, self.dZ, self.dX, self.dx = e(rows, t=torch.float32), e(rows, V), e(rows, M), e(rows, M)
        self.G = [e(N, M, t=torch.float32) for _ in range(2)]
        self.dnw = e(M, t=torch.float32)
        self.scratch = e(B.fw_rmsnorm_scratch_bytes(self.norm), t=torch.uint8)

    def gradients(self):
        B, st = self.B, self.stream
        B.fw_rmsnorm_forward(self.norm, self.x, self.nw, self.y, res=self.r, sum_out=self.s, rstd=self.rstd, stream=st)
        self.block.forward(self.y, *self.W, self.H, self.Zg, self.Zu)
        out = self.s + self.H @ self.down.T
        logits = out @ self.head.T
        B.fw_distill_forward(self.loss_desc, logits, self.T, self.I, self.loss, t_lse=self.t_lse, weight=self.weight, dZ=self.dZ, stream=st)
        d_out = self.dZ @ self.head
        self.block.backward(d_out @ self.down, self.y, *self.W, self.Zg, self.Zu, dX=self.dX, dWg=self.G[0], dWu=self.G[1])
        B.fw_rmsnorm_backward(self.norm, self.dX, self.s, self.nw, self.rstd, self.dx, dw=self.dnw, dsum=d_out, scratch=self.scratch, stream=st)

    def update(self):
        hs = [L.handle for L in self.layers]
        self.B.fw_group_cov_update(hs, [self.y] * 2, [self.rows] * 2, [self.M] * 2)
        self.B.fw_group_cond_reduce(hs, 3, 4)
        self.B.fw_group_grad_transform_step(hs, self.G, self.master, None, None, 0.1)


def reference(s):
    """The loss and its gradients in 64 bits, without any rounding between (autograd of elementary operations)."""
    leaf = lambda t: t.to(F64).clone().requires_grad_(True)  # noqa: E731
    x, nw, wg, wu = leaf(s.x), leaf(s.nw), leaf(s.W[0]), leaf(s.W[1])
    u = x + s.r.to(F64)
    y = u * (u.square().mean(1, keepdim=True) + 1e-5).rsqrt() * nw
    a = y @ wg.T
    out = u + (a * torch.sigmoid(a) * (y @ wu.T)) @ s.down.to(F64).T
    logq = torch.log_softmax(out @ s.head.to(F64).T, 1)
    logp = s.T.to(F64) - s.t_lse.to(F64)[:, None]
    p, at = logp.exp(), s.I.long()
    pt = 1 - p.sum(1)
    named = torch.zeros(s.rows, s.V, dtype=torch.bool, device="cuda").scatter_(1, at, True)
    logqt = torch.logsumexp(logq.masked_fill(named, float("-inf")), 1)
    kl = (p * (logp - logq.gather(1, at))).sum(1) + pt * (pt.log() - logqt)
    loss = kl * s.weight.to(F64)
    loss.sum().backward()
    return loss.detach(), x.grad, nw.grad, wg.grad, wu.grad


def test_training_step(B):
    """Against 64 bits from end to end.  Between input and gradient lie nine roundings to bf16 (s, y, Z, H, down, logits, dZ, the
    products back, da and db, dX), each at most 2^-8 of what it rounds: 9 x 2^-8 = 0.035 of the gradients' size; the loss, in which only
    the first six act and on logits of size 5, within 6 x 2^-8 x 5 of its terms, taken as 0.1."""
    s = Step(B)
    s.gradients()
    loss, dx, dnw, dwg, dwu = reference(s)
    assert rel(s.loss, loss) <= 0.1
    for got, want in ((s.dx, dx), (s.dnw, dnw), (s.G[0], dwg), (s.G[1], dwu)):
        assert rel(got, want) <= 9 * 2.0 ** -8
    # the parameter step with each layer's own transform: W - 0.1 G Qs, TF32 products (2^-10 of the terms, 5e-3 as for the layers)
    before = [w.clone() for w in s.master]
    s.update()
    for L, w0, w, G in zip(s.layers, before, s.master, s.G):
        Q = L.get(B.FW_F_QS).to(F64)
        assert float((Q - torch.eye(s.M, device="cuda")).abs().max()) > 0.01          # the recursion has acted
        step = 0.1 * G.to(F64) @ Q
        assert rel(w0.to(F64) - w.to(F64), step) <= 5e-3
        assert L.sync_status() == B.FW_OK
    assert s.block.sync_status() == B.FW_OK


def test_training_step_in_a_graph(B):
    """The whole step captured and replayed over new inputs gives what plain calls give, bit for bit."""
    stream = torch.cuda.Stream()
    s = Step(B, stream=stream.cuda_stream)
    outs = [s.loss, s.dx, s.dnw, *s.G, s.y, s.H, *s.master]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(2):
            s.gradients()
            s.update()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            s.gradients()
        s.x.copy_(put(torch.randn(s.rows, s.M, generator=gen(5), device="cuda"), BF16))
        s.gradients()
        stream.synchronize()
        want = [o.clone() for o in outs]
        for o in outs[:7]:
            o.zero_()
        graph.replay()
        stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    assert s.block.sync_status() == B.FW_OK


@pytest.mark.parametrize("rows", [1, 3, 40])
def test_eight_bit_tokens(B, rows):
    """Norm to e4m3 with a scale a token, into the gated block with a scale for each output: what the block computes is the product of
    the values that the 8-bit numbers stand for (4 (M / 16 + 16) u of the terms' magnitudes), rounded to bf16."""
    M, N = 1024, 768
    g = gen(rows)
    x, r = (put(torch.randn(rows, M, generator=g, device="cuda"), BF16) for _ in range(2))
    W = [torch.randn(N, M, generator=g, device="cuda") * M ** -0.5 for _ in range(2)]
    c = [w.abs().amax(1) / 448 for w in W]
    q = [(w / s[:, None]).to(E4M3) for w, s in zip(W, c)]
    s, y, ys, H = matrix(rows, M, BF16), matrix(rows, M, E4M3), torch.empty(rows, device="cuda"), matrix(rows, N, BF16)
    B.fw_rmsnorm_forward(B.fw_norm_desc_default(M, y_dtype=B.FW_E4M3), x, torch.ones(M, device="cuda"), y, res=r, sum_out=s, y_scale=ys)
    blk = B.Gated(M, N, x_dtype=B.FW_E4M3)
    blk.forward(y, *q, H, x_scale=ys, wg_scale=c[0], wu_scale=c[1])
    v = y.to(F64) * ys.to(F64)[:, None]
    w = [a.to(F64) * b.to(F64)[:, None] for a, b in zip(q, c)]
    a, b = v @ w[0].T, v @ w[1].T
    u = 4 * (M / 16 + 16) * 2.0 ** -24
    ea, eb = (u * (v.abs() @ k.abs().T) for k in w)
    f = a * torch.sigmoid(a)
    want = f * b
    e = 1.13 * ea * (b.abs() + eb) + f.abs() * eb + want.abs() * 2.0 ** -19
    assert bool(((H.to(F64) - want).abs() <= e + 2.0 ** -8 * (want.abs() + e)).all())
    # and the norm's output is the norm of the sum that is kept
    n = s.to(F64)
    n = n * (n.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    assert bool(((v - n).abs() <= 2.0 ** -4 * n.abs() * (1 + 2.0 ** -17) + 2.0 ** -10 * ys.to(F64)[:, None] + 2.0 ** -17 * n.abs()).all())


def far_apart(rows, cols, dtype):
    """Rows 2^30 elements apart: the third begins at 2^31."""
    base = torch.empty((rows - 1) * 2 ** 30 + cols, dtype=dtype, device="cuda")
    return torch.as_strided(base, (rows, cols), (2 ** 30, 1))


def test_rows_beyond_32_bits(B):
    """Offsets of 2^31 elements and more in every matrix that has a leading dimension: the bits of the same call on neighbouring rows."""
    rows, M, N, V, K = 4, 264, 520, 9000, 20
    g = gen(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    x, res, w = r(rows, M), r(rows, M), 1 + r(M).float() * 0.1
    d = B.fw_norm_desc_default(M)

    def norm(x, res, s, y, dx):
        rstd = torch.empty(rows, device="cuda")
        B.fw_rmsnorm_forward(d, x, w, y, res=res, sum_out=s, rstd=rstd)
        B.fw_rmsnorm_backward(d, y, s, w, rstd, dx, dsum=x)
        return s, y, dx

    def gated(x, W, H, dX):
        blk = B.Gated(M, N, rows, grad=1)
        Zg, Zu = (torch.empty_strided((rows, N), (H.stride(0), 1), dtype=BF16, device="cuda") for _ in range(2)) if H.stride(0) == N else (far_apart(rows, N, BF16) for _ in range(2))
        blk.forward(x, *W, H, Zg, Zu)
        dWg, dWu = torch.empty(N, M, device="cuda"), torch.empty(N, M, device="cuda")
        blk.backward(H, x, *W, Zg, Zu, dX=dX, dWg=dWg, dWu=dWu)
        assert blk.sync_status() == B.FW_OK
        return H, Zg, Zu, dX, dWg, dWu

    def loss(z, dz, dz2):
        ld, out, stat = B.fw_distill_desc_default(z.shape[1], K, t_dtype=B.FW_F32), torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
        B.fw_distill_forward(ld, z, T, I[z.shape[1]], out, stat=stat, dZ=dz)
        B.fw_distill_backward(ld, z, T, I[z.shape[1]], stat, dz2)
        return out, dz, dz2

    def same(near, far):
        for a, b in zip(near, far):
            assert torch.equal(a, b) and not bool(torch.isnan(a.float()).any())

    e = lambda n: torch.empty(rows, n, dtype=BF16, device="cuda")  # noqa: E731
    far = [far_apart(rows, V, BF16) for _ in range(5)]
    put_far = lambda i, v: far[i][:, :v.shape[1]].copy_(v)  # noqa: E731
    at = lambda i, n: far[i][:, :n]  # noqa: E731
    same(norm(x, res, e(M), e(M), e(M)), norm(put_far(0, x), put_far(1, res), at(2, M), at(3, M), at(4, M)))
    W = [r(N, M) * 0.1 for _ in range(2)]
    same(gated(x, W, e(N), e(M)), gated(put_far(0, x), W, at(1, N), at(2, M)))
    T = torch.randn(rows, K, generator=g, device="cuda")
    I = {n: torch.stack([torch.randperm(n, generator=g, device="cuda")[:K] for _ in range(rows)]).to(torch.int32) for n in (1000, V)}
    for n in (1000, V):
        z = r(rows, n)
        z[2] *= 2000                                             # statistics too coarse to be used
        same(loss(z, e(n), e(n)), loss(put_far(0, z), at(1, n), at(2, n)))


def test_a_small_block_between_layer_updates(B):
    """Calls of a few rows in the stream of a bf16 layer's updates, whose products take all of the tensor memory of a SM: each waits for
    the other, and both give what they give alone."""
    g = gen(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    M, N, rows = 128, 1024, 16
    X, W, H, H2 = r(rows, M), [r(N, M) * 0.1 for _ in range(2)], torch.empty(rows, N, dtype=BF16, device="cuda"), torch.empty(rows, N, dtype=BF16, device="cuda")
    blk = B.Gated(M, N)
    blk.forward(X, *W, H)
    Y = r(4096, 576)
    layers = [B.Layer(576, 64, x_dtype=B.FW_BF16, prec=B.FW_PREC_BF16) for _ in range(2)]
    for _ in range(30):
        layers[0].cov_update(Y)
        layers[1].cov_update(Y)
        for _ in range(3):
            blk.forward(X, *W, H2)
        layers[0].cov_update(Y)
        layers[1].cov_update(Y)
    assert torch.equal(H, H2) and blk.sync_status() == B.FW_OK
    assert all(L.sync_status() == B.FW_OK for L in layers)
    assert torch.equal(layers[0].get(B.FW_F_PHIX), layers[1].get(B.FW_F_PHIX))


def test_two_streams_at_once(B):
    """Norm, block and loss on two streams, one behind the other in each and captured in one of them: the bits of calls by themselves."""
    M, N, rows, V, K = 512, 1024, 300, 20000, 40

    def job(seed, stream):
        g = gen(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
        x, res, w, W = r(rows, M), r(rows, M), 1 + r(M).float() * 0.1, [r(N, M) * 0.05 for _ in range(2)]
        z, T, I = r(rows, V), r(rows, K), torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(rows)]).to(torch.int32)
        z[5::9] *= 2000
        e = lambda *s, t=BF16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        f = torch.float32
        s, y, H, Zg, Zu, dX, dx, dz, dz2 = e(rows, M), e(rows, M), e(rows, N), e(rows, N), e(rows, N), e(rows, M), e(rows, M), e(rows, V), e(rows, V)
        rstd, dw, out, stat, G = e(rows, t=f), e(M, t=f), e(rows, t=f), e(rows, 2, t=f), [e(N, M, t=f) for _ in range(2)]
        d, ld = B.fw_norm_desc_default(M), B.fw_distill_desc_default(V, K)
        scratch, blk = e(B.fw_rmsnorm_scratch_bytes(d), t=torch.uint8), B.Gated(M, N, rows, grad=1, stream=stream)

        def call():
            B.fw_rmsnorm_forward(d, x, w, y, res=res, sum_out=s, rstd=rstd, stream=stream)
            blk.forward(y, *W, H, Zg, Zu)
            B.fw_distill_forward(ld, z, T, I, out, stat=stat, dZ=dz, stream=stream)
            B.fw_distill_backward(ld, z, T, I, stat, dz2, stream=stream)
            blk.backward(H, y, *W, Zg, Zu, dX=dX, dWg=G[0], dWu=G[1])
            B.fw_rmsnorm_backward(d, dX, s, w, rstd, dx, dw=dw, scratch=scratch, stream=stream)

        return call, [s, y, H, Zg, Zu, dX, dx, dz, dz2, rstd, dw, out, stat, *G], blk

    streams = [torch.cuda.Stream() for _ in range(2)]
    jobs = [job(k, s.cuda_stream) for k, s in enumerate(streams)]
    torch.cuda.synchronize()
    want = []
    for call, outs, _ in jobs:
        call()
        torch.cuda.synchronize()
        want.append([o.clone() for o in outs])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[1]):
        jobs[1][0]()
    for _, outs, _ in jobs:
        for o in outs:
            o.fill_(float("nan"))
    torch.cuda.synchronize()
    for _ in range(10):
        jobs[0][0]()
        with torch.cuda.stream(streams[1]):
            graph.replay()
    torch.cuda.synchronize()
    for (_, outs, blk), ref in zip(jobs, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, ref)) and blk.sync_status() == B.FW_OK
