"""More operators around a whitened layer's training step, as calls that can be timed and compared.

  sandwich    the norms behind a block and before the next one, with the gate and the residual addition between them
  policy      clipped policy loss of sampled tokens with a KL term, and its gradient for the logits
  preference  loss of pairs of answers from their tokens' log-probabilities, and its gradient for the logits
  adamw       one AdamW step over all tensors of a network, states in 32 or 8 bits

A case is a flat dict: `op` picks the operator, `way` its direction, the other entries are sizes, types and options.
Where `own` is false `run` computes an operator in elementary torch operations in 32 bits; where it is true it makes the
calls of `paper_2010_01546_b200.binding`.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}
E4M3_MAX = 448.0
EPS = 1e-5                                        # of the norms
BLOCK = 256                                       # elements of a tensor that share a scale of an 8-bit state


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------
def sandwich(way, rows, M, dtype="bf16", y="same", post=True, gate=False, alpha=1.0, pad=0):
    """way: fwd or bwd. post: the block's output is normalised. gate: a number for each row. alpha: of the residual stream.
    pad: columns that the rows are apart beyond M."""
    return {"op": "sandwich", "way": way, "rows": rows, "M": M, "dtype": dtype, "y": y, "post": post, "gate": gate, "alpha": alpha,
            "pad": pad}


def policy(way, rows, V, dtype="bf16", kl=0.0, tau=1.0, odd=False):
    """way: both (loss and gradient in one call) or loss. odd: rows next to each other whatever V is, so most are not aligned."""
    return {"op": "policy", "way": way, "rows": rows, "V": V, "dtype": dtype, "kl": kl, "tau": tau, "odd": odd}


def preference(pairs, length, V, dtype="bf16", mean=False, smooth=0.0, ref=True, odd=False):
    """length: largest number of tokens of an answer. mean: log-probabilities by token. ref: those of a reference model."""
    return {"op": "preference", "pairs": pairs, "length": length, "V": V, "dtype": dtype, "mean": mean, "smooth": smooth, "ref": ref,
            "odd": odd}


def adamw(blocks, M, N, V, g="bf16", bits=32, clip=True, copies=True):
    """A network of `blocks` blocks of width M and N with a table of V rows. g: type of the gradients of matrices. bits: of the
    states. clip: gradients clipped by their norm. copies: the step also leaves the parameters in bf16."""
    return {"op": "adamw", "blocks": blocks, "M": M, "N": N, "V": V, "g": g, "bits": bits, "clip": clip, "copies": copies}


def listed():
    return [
        # one new token between two blocks, in 8 bits for the projections that follow: latency
        dict(sandwich("fwd", 1, 4096, y="e4m3"), name="sandwich_token_e4m3"),
        # a step's tokens between two blocks
        dict(sandwich("fwd", 8192, 4096), name="sandwich_fwd_bf16"),
        # the backward pass of it, tokens that were weighted by a router's gate
        dict(sandwich("bwd", 8192, 4096, gate=True), name="sandwich_bwd_bf16"),
        # fp32 activations of an odd width, rows not on 16-byte boundaries, a damped residual stream
        dict(sandwich("bwd", 5003, 1537, dtype="f32", alpha=0.7, pad=2), name="sandwich_bwd_odd_f32"),
        # a small set of actions: latency
        dict(policy("both", 256, 1000, dtype="f32", kl=0.1), name="policy_actions1000_f32"),
        # a step's sampled tokens over a large vocabulary, with the KL term
        dict(policy("both", 4096, 131072, kl=0.04), name="policy_vocab_bf16"),
        # an odd vocabulary, rows next to each other, sampled at a higher temperature
        dict(policy("both", 2048, 50257, tau=1.3, odd=True), name="policy_odd_bf16"),
        # four pairs of short answers, fp32 logits
        dict(preference(4, 24, 8000, dtype="f32"), name="preference_short_f32"),
        # sixteen pairs of long answers; labels that may be wrong
        dict(preference(16, 160, 50257, smooth=0.1), name="preference_long_bf16"),
        # a small network of odd widths, fp32 gradients: latency
        dict(adamw(3, 192, 500, 1000, g="f32", clip=False, copies=False), name="adamw_small_f32"),
        # wide blocks and a large table: bf16 gradients clipped by their norm, bf16 copies for the next forward pass
        dict(adamw(4, 2048, 8192, 50257), name="adamw_wide_f32"),
        # hundreds of tensors of odd widths, states in 8 bits
        dict(adamw(48, 512, 1367, 32001, bits=8), name="adamw_many_e4m3"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("sandwich", "sandwich", "policy", "policy", "preference", "adamw", "adamw"))
    if op == "sandwich":
        M = _log(rng, 64, 8192)
        M -= M % rng.choice((1, 8, 8, 64)) if M >= 64 else 0
        rows = _log(rng, 1, min(16384, 8192 * 4096 // M))
        dtype, way = rng.choice(("bf16", "bf16", "f32")), rng.choice(("fwd", "bwd"))
        return sandwich(way, rows, M, dtype, rng.choice(("same", "e4m3")) if way == "fwd" else "same", rng.random() < 0.75,
                        rng.random() < 0.5, rng.choice((1.0, 1.0, 0.7)), rng.choice((0, 0, 8, 3)))
    if op == "policy":
        V = _log(rng, 100, 150000)
        rows = _log(rng, 1, max(1, min(8192, 4096 * 131072 // V // 2)))
        return policy(rng.choice(("both", "both", "loss")), rows, V, rng.choice(("bf16", "bf16", "f32")), rng.choice((0.0, 0.05)),
                      rng.choice((1.0, 1.0, 1.3)), rng.random() < 0.4)
    if op == "preference":
        V = _log(rng, 100, 150000)
        pairs = _log(rng, 1, 64)
        length = _log(rng, 2, max(2, min(2000, 16 * 160 * 50257 // V // pairs)))
        return preference(pairs, length, V, rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.4, rng.choice((0.0, 0.1)),
                          rng.random() < 0.7, rng.random() < 0.4)
    M, blocks = _log(rng, 32, 2048), _log(rng, 1, 48)
    N = _log(rng, M, 4 * M)
    if rng.random() < 0.6:
        M, N = max(32, M // 32 * 32), max(32, N // 32 * 32)
    blocks = max(1, min(blocks, 200_000_000 // (4 * M * M + 3 * M * N)))
    return adamw(blocks, M, N, _log(rng, 10, max(10, min(100000, 100_000_000 // M))), rng.choice(("bf16", "f32")), rng.choice((32, 8)),
                 rng.random() < 0.6, rng.random() < 0.6)


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _rows_apart(rows, cols, dtype, pad=0):
    """An uninitialised matrix whose rows start on multiples of 16 bytes (of one element where pad is not 0; next to each other
    where it is negative)."""
    q = 16 // dtype.itemsize
    ld = cols if pad < 0 else cols + pad if pad else -(-cols // q) * q
    return torch.empty(rows, ld, dtype=dtype, device=DEV)[:, :cols]


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _prepare_sandwich(c, g):
    t, rows, M, pad = TYPES[c["dtype"]], c["rows"], c["M"], c["pad"]
    # activations of a residual stream: a few features are far larger than the others; the block's output is smaller
    feature = torch.exp(0.5 * _randn(g, M))
    o, x = (_rows_apart(rows, M, t, pad) for _ in range(2))
    o.copy_(_randn(g, rows, M).mul_(0.3))
    x.copy_(_randn(g, rows, M).mul_(2 * feature))
    s = {"o": o, "gate": torch.rand(rows, generator=g, device=DEV) if c["gate"] else None,
         "w_post": 0.5 + 0.2 * _randn(g, M), "w_pre": 1.0 + 0.2 * _randn(g, M)}
    s["h"] = _rows_apart(rows, M, t, pad)
    if c["way"] == "fwd":
        s["x"], s["y"] = x, _rows_apart(rows, M, t if c["y"] == "same" else TYPES["e4m3"], pad)
        s["y_scale"] = torch.empty(rows, device=DEV) if c["y"] == "e4m3" else None
        s["rstd"] = torch.empty(rows, 2, device=DEV)
    else:
        v = o.float()
        r = torch.rsqrt(v.square().mean(1) + EPS)
        v = v * s["w_post"] * (r[:, None] if c["post"] else 1.0)
        s["h"].copy_(x.float() * c["alpha"] + (v * s["gate"][:, None] if c["gate"] else v))
        del v
        s["rstd"] = torch.stack((r if c["post"] else torch.ones_like(r), torch.rsqrt(s["h"].float().square().mean(1) + EPS)), 1)
        s["dy"], s["dh"], s["dx"], s["do"] = (_rows_apart(rows, M, t, pad) for _ in range(4))
        s["dy"].copy_(_randn(g, rows, M).mul_(1e-3))
        s["dh"].copy_(_randn(g, rows, M).mul_(1e-3))
        s["dw_post"], s["dw_pre"] = (torch.empty(M, device=DEV) for _ in range(2))
        s["dgate"] = torch.empty(rows, device=DEV) if c["gate"] else None
    if own:
        from paper_2010_01546_b200 import binding as B
        kinds = {"f32": B.FW_F32, "bf16": B.FW_BF16}
        s["desc"] = B.fw_sandwich_desc_default(M, dtype=kinds[c["dtype"]], eps=EPS, alpha=c["alpha"], post=int(c["post"]),
                                               y_dtype=B.FW_E4M3 if c["y"] == "e4m3" else kinds[c["dtype"]])
        if c["way"] == "bwd":
            s["scratch"] = torch.empty(B.fw_sandwich_scratch_bytes(s["desc"]), dtype=torch.uint8, device=DEV)
    return s


def _prepare_logits(c, g, rows, tau):
    """Logits, sampled tokens, and the tokens' log-probabilities."""
    V, t = c["V"], TYPES[c["dtype"]]
    z = _randn(g, rows, V).mul_(2.5)
    Z = _rows_apart(rows, V, t, -1 if c["odd"] else 0)
    Z.copy_(z)
    z.copy_(Z).div_(tau)
    lse = torch.logsumexp(z, 1)
    at = z.sub_(torch.empty_like(z).exponential_(generator=g).log_()).argmax(1)
    logp = Z.gather(1, at[:, None]).float().flatten() / tau - lse
    return Z, at.to(torch.int32), logp


def _prepare_policy(c, g):
    rows, V, tau = c["rows"], c["V"], c["tau"]
    Z, at, logp = _prepare_logits(c, g, rows, tau)
    n = torch.arange(rows, device=DEV)
    # prompt tokens and padding do not count: some by their weight, some by their class
    s = {"Z": Z, "id": torch.where(n % 16 == 9, -1, at), "weight": torch.where(n % 16 == 5, 0.0, 1.0 / rows),
         # the policy has moved since the tokens were sampled, and further from the model it began as
         "logp_old": logp + 0.15 * _randn(g, rows), "logp_ref": logp + 0.4 * _randn(g, rows) if c["kl"] else None,
         "adv": _randn(g, rows)}
    s["loss"], s["logp"] = (torch.empty(rows, device=DEV) for _ in range(2))
    s["dZ"] = _rows_apart(rows, V, Z.dtype, -1 if c["odd"] else 0) if c["way"] == "both" else None
    if own:
        from paper_2010_01546_b200 import binding as B
        s["desc"] = B.fw_logprob_desc_default(V, z_dtype=B.FW_F32 if c["dtype"] == "f32" else B.FW_BF16, tau=tau)
        s["opt"] = B.fw_policy_desc_default(clip_low=0.2, clip_high=0.28, kl=c["kl"])
    return s


def _lengths(c):
    """Tokens of each answer, by its place alone, and of the prompt before each pair's."""
    return [1 + (k * 7919 + 3571) % c["length"] for k in range(2 * c["pairs"])]


def _prepare_preference(c, g):
    lengths = _lengths(c)
    last = sum(lengths)
    rows = last + 3                               # a padded batch: rows behind the last answer belong to nobody
    Z, at, logp = _prepare_logits(c, g, rows, 1.0)
    n = torch.arange(rows, device=DEV)
    seq = torch.tensor([0] + lengths, device=DEV).cumsum(0)
    which = torch.searchsorted(seq, n, right=True) - 1          # the answer of each row
    at = torch.where((n % 11 == 3) | (n >= last), -1, at)       # tokens of the prompt inside the packed rows
    s = {"Z": Z, "id": at, "seq": seq.to(torch.int32), "which": which, "weight": torch.full((c["pairs"],), 1.0 / c["pairs"], device=DEV),
         "beta": 2.0 if c["mean"] else 0.1, "margin": 0.5 if c["mean"] else 0.0, "ref": None}
    if c["ref"]:
        live = torch.zeros(2 * c["pairs"] + 1, device=DEV, dtype=torch.float64).index_add_(0, which, torch.where(at >= 0, logp, 0).double())
        if c["mean"]:
            live = live / torch.zeros_like(live).index_add_(0, which, (at >= 0).double()).clamp_min(1)
        s["ref"] = (live[:-1] + _randn(g, 2 * c["pairs"]) * (0.2 if c["mean"] else 3.0)).float()
    s["logp"], s["dlogp"] = (torch.empty(rows, device=DEV) for _ in range(2))
    s["stat"] = torch.empty(rows, 2, device=DEV)
    s["loss"], s["sums"] = torch.empty(c["pairs"], device=DEV), torch.empty(2 * c["pairs"], device=DEV)
    s["dZ"] = _rows_apart(rows, c["V"], Z.dtype, -1 if c["odd"] else 0)
    if own:
        from paper_2010_01546_b200 import binding as B
        s["desc"] = B.fw_logprob_desc_default(c["V"], z_dtype=B.FW_F32 if c["dtype"] == "f32" else B.FW_BF16)
        s["opt"] = B.fw_preference_desc_default(beta=s["beta"], margin=s["margin"], smooth=c["smooth"], mean=int(c["mean"]))
    return s


LR, BETA1, BETA2, ADAM_EPS, DECAY, SEED, STEPS = 1e-5, 0.9, 0.95, 1e-8, 0.1, 11, 1000


def _sizes(c):
    """(elements, whether it is a matrix) of each tensor."""
    M, N = c["M"], c["N"]
    block = [(M, False)] + [(M * M, True)] * 4 + [(M, False)] + [(N * M, True)] * 3
    return [(c["V"] * M, True)] + block * c["blocks"] + [(M, False)]


def _padded(n):
    return -(-n // BLOCK) * BLOCK


def _prepare_adamw(c, g):
    sizes = _sizes(c)
    starts = [0]
    for n, _ in sizes:
        starts.append(starts[-1] + _padded(n))
    total, M = starts[-1], c["M"]
    # one arena for each kind of data, every tensor on a multiple of BLOCK elements, zeros between them
    used = torch.ones(total, dtype=torch.bool, device=DEV)
    for a, (n, _) in zip(starts, sizes):
        used[a + n:a + _padded(n)] = False
    s = {"t": STEPS}
    # parameters at their usual initial size, gradients of a training run's middle
    s["P"] = _randn(g, total).mul_(M ** -0.5).mul_(used)
    grad = _randn(g, total).mul_(torch.exp(_randn(g, total))).mul_(1e-3).mul_(used)
    matrix = torch.zeros(total // BLOCK, dtype=torch.bool, device=DEV)
    for a, (n, mat) in zip(starts, sizes):
        matrix[a // BLOCK:(a + _padded(n)) // BLOCK] = mat
    s["decay"] = torch.where(matrix, DECAY, 0.0)[:, None]       # for each block: matrices decay, vectors do not
    if c["g"] == "bf16":                          # vectors' gradients come in fp32, as the norms leave them
        s["G16"] = grad.bfloat16()
        s["G32"] = torch.where(matrix[:, None], 0.0, grad.view(-1, BLOCK)).view(-1)
        s["G16"].view(-1, BLOCK).mul_(matrix[:, None])
    else:
        s["G16"], s["G32"] = None, grad.clone()
    s["C"] = torch.empty(total, dtype=torch.bfloat16, device=DEV).copy_(s["P"]) if c["copies"] else None
    m, v = grad.mul_(0.3).add_(_randn(g, total).mul_(2e-4).mul_(used)), None
    v = torch.exp(_randn(g, total)).mul_(2e-6).mul_(used)
    s["norm"] = torch.empty(1, device=DEV) if c["clip"] else None
    s["max_norm"] = 0.5 * 2.7e-3 * math.sqrt(total) if c["clip"] else 0.0
    if c["bits"] == 8:
        scale = lambda x: torch.exp2(torch.ceil(torch.log2((x.view(-1, BLOCK).abs().amax(1) / E4M3_MAX).clamp_min(2.0 ** -100))))  # noqa: E731
        s["m_scale"], s["v_scale"] = scale(m).to(torch.float8_e8m0fnu), scale(v.sqrt()).to(torch.float8_e8m0fnu)
        s["m"] = (m.view(-1, BLOCK) / s["m_scale"].float()[:, None]).view(-1).to(torch.float8_e4m3fn)
        s["v"] = (v.sqrt().view(-1, BLOCK) / s["v_scale"].float()[:, None]).clamp_min(2.0 ** -9).view(-1).mul_(used).to(torch.float8_e4m3fn)
    else:
        s["m"], s["v"], s["m_scale"], s["v_scale"] = m, v, None, None
    del m, v, grad, used
    if own:
        from paper_2010_01546_b200 import binding as B
        cut = lambda t: None if t is None else [t[a:a + n] for a, (n, _) in zip(starts, sizes)]  # noqa: E731
        mats = [mat for _, mat in sizes]
        s["adamw"] = B.AdamW(cut(s["P"]), copies=cut(s["C"]), state=B.FW_E4M3 if c["bits"] == 8 else B.FW_F32, beta1=BETA1, beta2=BETA2,
                             eps=ADAM_EPS, seed=SEED, decay=[DECAY if mat else 0.0 for mat in mats])
        G32 = cut(s["G32"])
        s["grads"] = s["adamw"].grads(G32 if s["G16"] is None else [a if mat else b for a, b, mat in zip(cut(s["G16"]), G32, mats)])
        for field, name in ((B.FW_A_M, "m"), (B.FW_A_V, "v"), (B.FW_A_M_SCALE, "m_scale"), (B.FW_A_V_SCALE, "v_scale")):
            if s[name] is not None:
                s["adamw"].state(field).copy_(s[name])
                s[name] = s["adamw"].state(field)
        s["adamw"].state(B.FW_A_STEP).fill_(STEPS)
    return s


PREPARE = {"sandwich": _prepare_sandwich, "policy": _prepare_policy, "preference": _prepare_preference, "adamw": _prepare_adamw}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = PREPARE[case["op"]](case, g)
    s["case"] = case
    return s


# ----------------------------------------------------------------------------
# the framework's calls
# ----------------------------------------------------------------------------
def _own_sandwich(c, s):
    from paper_2010_01546_b200 import binding as B
    if c["way"] == "fwd":
        B.fw_sandwich_forward(s["desc"], s["o"], s["x"], s["w_pre"], s["h"], s["y"], w_post=s["w_post"], gate=s["gate"],
                              y_scale=s["y_scale"], rstd=s["rstd"])
    else:
        B.fw_sandwich_backward(s["desc"], s["dy"], s["o"], s["h"], s["w_pre"], s["rstd"], s["dx"], s["do"], w_post=s["w_post"],
                               gate=s["gate"], dh=s["dh"], dw_post=s["dw_post"], dw_pre=s["dw_pre"], dgate=s["dgate"],
                               scratch=s["scratch"])


def _own_policy(c, s):
    from paper_2010_01546_b200 import binding as B
    B.fw_policy_forward(s["desc"], s["opt"], s["Z"], s["id"], s["logp_old"], s["adv"], s["loss"], logp_ref=s["logp_ref"],
                        weight=s["weight"], logp=s["logp"], dZ=s["dZ"])


def _own_preference(c, s):
    from paper_2010_01546_b200 import binding as B
    B.fw_logprob_forward(s["desc"], s["Z"], s["id"], s["logp"], stat=s["stat"])
    B.fw_preference_loss(s["desc"], s["opt"], s["logp"], s["id"], s["seq"], s["loss"], ref=s["ref"], weight=s["weight"], sums=s["sums"],
                         dlogp=s["dlogp"])
    B.fw_logprob_backward(s["desc"], s["Z"], s["id"], s["stat"], s["dlogp"], s["dZ"])


def _own_adamw(c, s):
    s["adamw"].step(s["grads"], LR, max_norm=s["max_norm"], norm_out=s["norm"])


# ----------------------------------------------------------------------------
# the plain forms
# ----------------------------------------------------------------------------
def _plain_sandwich(c, s):
    gate = s["gate"][:, None] if c["gate"] else 1.0
    o, wo = s["o"].float(), s["w_post"]
    if c["way"] == "fwd":
        r1 = torch.rsqrt(o.square().mean(1) + EPS) if c["post"] else torch.ones_like(s["rstd"][:, 0])
        # the sum is kept in its own type, and normalised as it is kept
        s["h"].copy_(c["alpha"] * s["x"].float() + gate * (o * r1[:, None] * wo))
        h = s["h"].float()
        r2 = torch.rsqrt(h.square().mean(1) + EPS)
        s["rstd"].copy_(torch.stack((r1, r2), 1))
        y = h * r2[:, None] * s["w_pre"]
        if c["y"] == "e4m3":
            top = y.abs().amax(1)
            s["y_scale"].copy_(torch.where(top > 0, top / E4M3_MAX, 1.0))
            y = y / s["y_scale"][:, None]
        s["y"].copy_(y)
        return
    r1, r2 = s["rstd"][:, :1], s["rstd"][:, 1:]
    n2, dy = s["h"].float() * r2, s["dy"].float()
    u = dy * s["w_pre"]
    th = r2 * (u - n2 * (u * n2).mean(1, keepdim=True)) + s["dh"].float()
    s["dw_pre"].copy_((dy * n2).sum(0))
    s["dx"].copy_(c["alpha"] * th)
    n1 = o * r1
    s["dw_post"].copy_((gate * th * n1).sum(0))
    u = th * wo
    along = (u * n1).sum(1)
    if c["gate"]:
        s["dgate"].copy_(along)
    s["do"].copy_(gate * r1 * (u - n1 * (along / c["M"])[:, None]) if c["post"] else gate * u)


def _plain_logp(s, tau):
    """Scaled logits, their normaliser, and the log-probability of each row's token (0 where it has none)."""
    z = s["Z"].float() / tau
    top = z.amax(1)
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    there = s["id"] >= 0
    at = s["id"].clamp_min(0).long()[:, None]
    return z, lse, there, at, torch.where(there, z.gather(1, at).flatten() - lse, 0)


def _plain_dz(s, z, lse, at, dlogp):
    q = torch.exp(z - lse[:, None]) * -dlogp[:, None]
    s["dZ"].copy_(q.scatter_add_(1, at, dlogp[:, None]))


def _plain_policy(c, s):
    z, lse, there, at, logp = _plain_logp(s, c["tau"])
    there = there & (s["weight"] != 0)
    logp = torch.where(there, logp, 0)
    w, A = torch.where(there, s["weight"], 0), s["adv"]
    ratio = torch.exp(logp - s["logp_old"])
    free, held = ratio * A, ratio.clamp(0.8, 1.28) * A
    loss, d = -torch.minimum(free, held), torch.where(free <= held, -free, 0)
    if c["kl"]:
        # exp(k) - 1 - k of a small k is lost in 32 bits
        k = s["logp_ref"].double() - logp.double()
        loss = loss + c["kl"] * (torch.expm1(k) - k).float()
        d = d - c["kl"] * torch.expm1(k).float()
    s["loss"].copy_(torch.where(there, w * loss, 0))
    s["logp"].copy_(logp)
    if c["way"] == "both":
        _plain_dz(s, z, lse, at, torch.where(there, w * d, 0) / c["tau"])


def _plain_preference(c, s):
    z, lse, there, at, logp = _plain_logp(s, 1.0)
    answers, rows = 2 * c["pairs"], logp.shape[0]
    # long sums in 64 bits
    sums = torch.zeros(answers + 1, dtype=torch.float64, device=DEV).index_add_(0, s["which"], logp.double())[:-1]
    share = torch.ones(answers, dtype=torch.float64, device=DEV)
    if c["mean"]:
        share = torch.zeros(answers + 1, dtype=torch.float64, device=DEV).index_add_(0, s["which"], there.double())[:-1].clamp_min(1).reciprocal()
    sums = sums * share
    gain = sums - s["ref"].double() if c["ref"] else sums
    h = s["beta"] * (gain[0::2] - gain[1::2]) - s["margin"]
    e, w = c["smooth"], s["weight"].double()
    s["loss"].copy_(w * ((1 - e) * torch.log1p(torch.exp(-h)) + e * torch.log1p(torch.exp(h))))
    d = s["beta"] * w * (e - 1 / (1 + torch.exp(h)))            # of the chosen answer's; the other's is its negative
    d = torch.cat((torch.stack((d, -d), 1).view(-1) * share, torch.zeros(1, dtype=torch.float64, device=DEV)))
    s["sums"].copy_(sums)
    s["logp"].copy_(logp)
    s["dlogp"].copy_(torch.where(there, d[s["which"]], 0))
    _plain_dz(s, z, lse, at, s["dlogp"])


def _mix(x):
    """32 bits that look like chance, from 32 bits (as int64)."""
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _noise(n, t):
    """Two numbers below 2^16 for each of n elements of the states, at step t."""
    key = ((SEED ^ (t * 0x9E3779B9)) & 0xFFFFFFFF)
    key = int(_mix(torch.tensor(key, dtype=torch.int64)))
    x = _mix(torch.arange(n, dtype=torch.int64, device=DEV) ^ key)
    return x & 0xFFFF, x >> 16


def _power(top):
    """The least power of two (2^-100 at least) that takes `top` to 448 or less."""
    mantissa, exponent = torch.frexp(top / E4M3_MAX)            # mantissa in [1/2, 1), 0 for 0
    return torch.exp2(torch.where(top > 0, exponent - (mantissa == 0.5).to(exponent.dtype), -100).clamp_min(-100).to(top.dtype))


def _down(a):
    """The largest e4m3 value not above a (a >= 0), and the next one."""
    _, exponent = torch.frexp(a)
    step = torch.exp2((exponent - 1).clamp_min(-6).to(a.dtype) - 3)
    low = torch.floor(a / step) * step
    return low, torch.minimum(low + step, torch.full_like(low, E4M3_MAX))


def _plain_adamw(c, s):
    s["t"] += 1
    t = s["t"]
    G = s["G32"] if s["G16"] is None else s["G32"] + s["G16"].float()
    if c["clip"]:
        norm = torch.linalg.vector_norm(G, dtype=torch.float64)
        s["norm"].copy_(norm)
        G = G * (s["max_norm"] / norm).clamp(max=1.0).float()
    m, v = s["m"], s["v"]
    if c["bits"] == 8:
        m = (m.float().view(-1, BLOCK) * s["m_scale"].float()[:, None]).view(-1)
        v = (v.float().view(-1, BLOCK) * s["v_scale"].float()[:, None]).square().view(-1)
    m = BETA1 * m + (1 - BETA1) * G
    v = BETA2 * v + (1 - BETA2) * G * G
    root = torch.sqrt(v)
    P = s["P"].view(-1, BLOCK)
    step = (LR / (1 - BETA1 ** t)) * m / (root / math.sqrt(1 - BETA2 ** t) + ADAM_EPS)
    P.mul_(1 - LR * s["decay"]).sub_(step.view(-1, BLOCK))
    if c["copies"]:
        s["C"].copy_(s["P"])
    if c["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return
    # a mean is rounded up or down by chance, by its distance; a square too, from the distance of the squares
    nm, nv = _noise(m.numel(), t)
    sm, sv = (_power(x.view(-1, BLOCK).abs().amax(1)) for x in (m, root))
    a = (m.view(-1, BLOCK) / sm[:, None]).view(-1)
    low, high = _down(a.abs())
    s["m"].copy_(torch.where((a.abs() - low) / (high - low) + nm / 65536.0 >= 1, high, low) * torch.sign(a))
    a = (root.view(-1, BLOCK) / sv[:, None]).view(-1)
    low, high = _down(a)
    up = (a - low) * (a + low) > (nv + 0.5) / 65536.0 * (high - low) * (high + low)
    r = torch.where(up, high, low)
    s["v"].copy_(torch.where((v > 0) & (r == 0), 2.0 ** -9, r))
    s["m_scale"].copy_(sm)
    s["v_scale"].copy_(sv)


def _outputs(c, s):
    names = {"sandwich": ("h", "y", "y_scale", "rstd") if c.get("way") == "fwd" else ("dx", "do", "dw_post", "dw_pre", "dgate"),
             "policy": ("loss", "logp", "dZ"),
             "preference": ("logp", "sums", "loss", "dlogp", "dZ"),
             "adamw": ("P", "C", "m", "v", "m_scale", "v_scale", "norm")}[c["op"]]
    return {n: s[n] for n in names if s[n] is not None}


OWN = {"sandwich": _own_sandwich, "policy": _own_policy, "preference": _own_preference, "adamw": _own_adamw}
PLAIN = {"sandwich": _plain_sandwich, "policy": _plain_policy, "preference": _plain_preference, "adamw": _plain_adamw}


def run(state):
    c = state["case"]
    (OWN if own else PLAIN)[c["op"]](c, state)
    return _outputs(c, state)


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "sandwich":
        e, rows, M = BYTES[c["dtype"]], c["rows"], c["M"]
        n, gate = rows * M, 4 * rows if c["gate"] else 0
        if c["way"] == "fwd":
            y = e if c["y"] == "same" else 1
            return {"bytes": n * (3 * e + y) + 8 * M + gate + rows * (12 if c["y"] == "e4m3" else 8), "flops": 12 * n}
        return {"bytes": n * 6 * e + 16 * M + 2 * gate + 8 * rows, "flops": 24 * n}
    if c["op"] == "policy":
        e, rows, V = BYTES[c["dtype"]], c["rows"], c["V"]
        live = rows - len(range(5, rows, 16)) - len(range(9, rows, 16))            # the others are not read
        write = rows * V * e if c["way"] == "both" else 0
        return {"bytes": live * V * e + write + rows * (24 + (4 if c["kl"] else 0)), "flops": live * V * (6 if write else 3)}
    if c["op"] == "preference":
        e, V, last = BYTES[c["dtype"]], c["V"], sum(_lengths(c))
        rows, live = last + 3, last - len(range(3, last, 11))
        return {"bytes": (live + rows) * V * e + rows * 12 + c["pairs"] * 24, "flops": live * V * 6}
    sizes = _sizes(c)
    each = lambda mat: 8 + (2 if mat and c["g"] == "bf16" else 4) + (2 if c["copies"] else 0) + (16 if c["bits"] == 32 else 4 + 4 / BLOCK)  # noqa: E731
    return {"bytes": sum(n * each(mat) for n, mat in sizes), "flops": 14 * sum(n for n, _ in sizes)}


# ----------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------
def _exact_sandwich(c, s):
    d = torch.float64
    o, w1, w2 = s["o"].to(d), s["w_post"].to(d), s["w_pre"].to(d)
    k = s["gate"].to(d) if c["gate"] else torch.ones(c["rows"], dtype=d, device=DEV)
    if c["way"] == "fwd":
        r1 = (o.pow(2).sum(1) / c["M"] + EPS).pow(-0.5) if c["post"] else torch.ones_like(k)
        full = torch.einsum("r,rm,m->rm", k * r1, o, w1) + c["alpha"] * s["x"].to(d)
        h = full.to(s["h"].dtype).to(d)
        r2 = (h.pow(2).sum(1) / c["M"] + EPS).pow(-0.5)
        y = torch.einsum("r,rm,m->rm", r2, h, w2)
        out = {"h": full, "y": y, "rstd": torch.stack((r1, r2), 1)}
        if c["y"] == "e4m3":
            scale = y.abs().max(1).values / E4M3_MAX
            scale[scale == 0] = 1
            out["y_scale"], out["y"] = scale, (y / scale[:, None]).to(torch.float8_e4m3fn).to(d)
        return out
    r1, r2 = s["rstd"].to(d).unbind(1)
    n2, dy = s["h"].to(d) * r2[:, None], s["dy"].to(d)
    g = dy * w2                                   # of the normalised row: less its part along the row
    dh = s["dh"].to(d) + (g - n2 * (torch.einsum("rm,rm->r", g, n2) / c["M"])[:, None]) * r2[:, None]
    n1 = o * r1[:, None]
    g = dh * w1
    t = torch.einsum("rm,rm->r", g, n1)
    do = (g - n1 * (t / c["M"])[:, None]) * (r1 * k)[:, None] if c["post"] else g * k[:, None]
    out = {"dx": dh * c["alpha"], "do": do, "dw_post": torch.einsum("r,rm,rm->m", k, dh, n1), "dw_pre": torch.einsum("rm,rm->m", dy, n2)}
    return {**out, "dgate": t} if c["gate"] else out


def _exact_rows(s, tau, live):
    """Probabilities of each row and the log-probability of its token."""
    z = s["Z"].to(torch.float64).div_(tau)
    q = torch.log_softmax(z, 1)
    at = torch.where(live, s["id"], 0).long()
    logp = torch.where(live, q[torch.arange(len(at), device=DEV), at], 0)
    return q.exp_(), at, logp


def _exact_grad(q, at, slope):
    dz = q.mul_(-slope[:, None])
    dz[torch.arange(len(at), device=DEV), at] += slope
    return dz


def _exact_policy(c, s):
    d = torch.float64
    live = (s["id"] >= 0) & (s["weight"] != 0)
    q, at, logp = _exact_rows(s, c["tau"], live)
    A, w = s["adv"].to(d), torch.where(live, s["weight"].to(d), 0)
    ratio = (logp - s["logp_old"].to(d)).exp()
    low, high = torch.tensor((0.2, 0.28), dtype=d, device=DEV)
    bound = torch.where(A >= 0, (1 + high) * A, (1 - low) * A)  # what min(r A, clip(r) A) does not pass
    hit = ratio * A > bound
    loss, slope = -torch.where(hit, bound, ratio * A), torch.where(hit, 0, -ratio * A)
    if c["kl"]:
        k = s["logp_ref"].to(d) - logp
        loss, slope = loss + c["kl"] * (torch.expm1(k) - k), slope - c["kl"] * torch.expm1(k)
    out = {"loss": w * loss, "logp": logp}
    return {**out, "dZ": _exact_grad(q, at, w * slope / c["tau"])} if c["way"] == "both" else out


def _exact_preference(c, s):
    d = torch.float64
    live = s["id"] >= 0
    q, at, logp = _exact_rows(s, 1.0, live)
    total = torch.cat((torch.zeros(1, dtype=d, device=DEV), logp.cumsum(0)))
    count = torch.cat((torch.zeros(1, dtype=d, device=DEV), live.to(d).cumsum(0)))
    seq = s["seq"].long()
    sums, n = total[seq].diff(), count[seq].diff().clamp(min=1)
    if c["mean"]:
        sums = sums / n
    gain = sums - (s["ref"].to(d) if c["ref"] else 0)
    h = s["beta"] * (gain[::2] - gain[1::2]) - s["margin"]
    e, w = c["smooth"], s["weight"].to(d)
    soft = torch.nn.functional.softplus
    slope = (w * s["beta"] * (e * torch.sigmoid(h) - (1 - e) * torch.sigmoid(-h))).repeat_interleave(2)
    slope[1::2] *= -1
    if c["mean"]:
        slope = slope / n
    dlogp = torch.zeros(len(at), dtype=d, device=DEV)
    dlogp[:int(seq[-1])] = slope.repeat_interleave(seq.diff())
    dlogp[~live] = 0
    return {"logp": logp, "sums": sums, "loss": w * ((1 - e) * soft(-h, threshold=700) + e * soft(h, threshold=700)), "dlogp": dlogp,
            "dZ": _exact_grad(q, at, dlogp)}


def _exact_adamw(c, s):
    """Of the step that the plain form takes from a new state."""
    d = torch.float64
    t = s["t"] + 1
    G = s["G32"].to(d)
    if s["G16"] is not None:
        G += s["G16"]
    norm = G.pow(2).sum().sqrt()
    if c["clip"]:
        G *= min(1.0, s["max_norm"] / float(norm))
    m, v = s["m"].to(d), s["v"].to(d)
    if c["bits"] == 8:
        m *= s["m_scale"].to(d).repeat_interleave(BLOCK)
        v = (v * s["v_scale"].to(d).repeat_interleave(BLOCK)).pow(2)
    m = torch.lerp(G, m, BETA1)
    v = torch.lerp(G.pow(2), v, BETA2)
    P = s["P"].to(d) * (1 - LR * s["decay"].double().expand(-1, BLOCK).reshape(-1))
    P -= LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + ADAM_EPS)
    out = {"P": P}
    if c["copies"]:
        out["C"] = P
    if c["clip"]:
        out["norm"] = norm.view(1)
    if c["bits"] == 32:
        return {**out, "m": m, "v": v}
    i = torch.arange(m.numel(), device=DEV)
    key = (SEED ^ (t * 0x9E3779B9)) & 0xFFFFFFFF
    for shift, factor in ((16, 0x7FEB352D), (15, 0x846CA68B)):
        key = ((key ^ (key >> shift)) * factor) & 0xFFFFFFFF
    i ^= key ^ (key >> 16)
    for shift, factor in ((16, 0x7FEB352D), (15, 0x846CA68B)):
        i = ((i ^ (i >> shift)) * factor) & 0xFFFFFFFF
    i ^= i >> 16
    # all values of the 8-bit type that are not negative, in order
    grid = torch.arange(127, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn).to(d)
    for name, x, chance in (("m", m, (i & 0xFFFF).to(d) / 65536), ("v", v.sqrt(), ((i >> 16).to(d) + 0.5) / 65536)):
        top = x.abs().view(-1, BLOCK).amax(1)
        scale = torch.exp2(torch.ceil(torch.log2(top / E4M3_MAX)).clamp(min=-100))
        y = x.abs() / scale.repeat_interleave(BLOCK)
        at = (torch.searchsorted(grid, y, right=True) - 1).clamp(max=125)
        lo, hi = grid[at], grid[at + 1]
        if name == "m":
            code = torch.where(y - lo >= (1 - chance) * (hi - lo), hi, lo) * x.sign()
        else:
            code = torch.where(y.pow(2) - lo.pow(2) > chance * (hi.pow(2) - lo.pow(2)), hi, lo)
            code = torch.where((x > 0) & (code == 0), grid[1], code)
        out[name], out[name + "_scale"] = code, scale
        del y, at, lo, hi, code
    return out


def exact(case, seed):
    global own
    was, own = own, False                         # the inputs alone, no handle
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"sandwich": _exact_sandwich, "policy": _exact_policy, "preference": _exact_preference, "adamw": _exact_adamw}[case["op"]](case, s)
