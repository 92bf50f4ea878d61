"""Operators around a whitened layer's training step, as calls that can be timed and compared.

  norm     residual addition and root-mean-square norm, in the input's type or in 8 bits with a scale a row
  gated    gated feed-forward block: two projections, the activation and the product
  distill  loss against a teacher's top logits, with its gradient

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


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------
def norm(way, rows, M, dtype="bf16", y="same", res=True, pad=0):
    """way: fwd or bwd. y: "same" (the type of x) or "e4m3". pad: columns that the rows are apart beyond M."""
    return {"op": "norm", "way": way, "rows": rows, "M": M, "dtype": dtype, "y": y, "res": res, "pad": pad}


def gated(way, rows, M, N, dtype="bf16", act="silu", bias=False, keep=False):
    """way: fwd or bwd. keep: the forward call also leaves both projections, for the backward pass."""
    return {"op": "gated", "way": way, "rows": rows, "M": M, "N": N, "dtype": dtype, "act": act, "bias": bias, "keep": keep}


def distill(way, rows, V, K, dtype="bf16", rest=False, tau=1.0):
    """way: loss (no gradient), both (loss and gradient in one call) or bwd (gradient from what `loss` left).
    rest: the teacher's mass outside its top logits counts as one more class."""
    return {"op": "distill", "way": way, "rows": rows, "V": V, "K": K, "dtype": dtype, "rest": rest, "tau": tau}


def listed():
    return [
        # one new token between two blocks, in 8 bits for the projections that follow: latency
        dict(norm("fwd", 1, 4096, y="e4m3"), name="norm_token_e4m3"),
        # a long prompt, or a step's tokens, in 8 bits
        dict(norm("fwd", 8192, 4096, y="e4m3"), name="norm_rows8192_e4m3"),
        # fp32 activations of an odd width, rows not on 16-byte boundaries
        dict(norm("fwd", 5003, 1537, dtype="f32", pad=2), name="norm_odd_f32"),
        # the backward pass of a training step, with the gradient that comes along the residual
        dict(norm("bwd", 8192, 4096), name="norm_bwd_bf16"),
        # one new token: both weight matrices are read once
        dict(gated("fwd", 1, 4096, 8192), name="gated_token_bf16"),
        # a prompt in 8 bits, scales for each token and each output
        dict(gated("fwd", 2048, 4096, 8192, dtype="e4m3"), name="gated_prompt_e4m3"),
        # forward pass of a training step, both projections kept
        dict(gated("fwd", 8192, 4096, 8192, keep=True), name="gated_train_fwd_bf16"),
        # its backward pass: gradients of the input, both weights and both biases
        dict(gated("bwd", 8192, 4096, 8192, bias=True), name="gated_train_bwd_bf16"),
        # a small batch and sizes that no tile divides, biases, another activation
        dict(gated("fwd", 333, 1000, 1367, act="gelu", bias=True, keep=True), name="gated_ragged_bf16"),
        # classifier of 1000 classes, batch 256, a teacher's ten best classes: latency
        dict(distill("both", 256, 1000, 10, dtype="f32", tau=4.0), name="distill_classes1000_f32"),
        # a step's tokens over a large vocabulary, 64 logits a token and the rest's mass
        dict(distill("both", 4096, 131072, 64, rest=True), name="distill_vocab_bf16"),
        # the gradient alone, from the statistics of an earlier loss call, odd vocabulary
        dict(distill("bwd", 515, 50021, 33, dtype="f32", tau=2.0), name="distill_bwd_odd_f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "gated", "gated", "distill"))
    if op == "norm":
        M = _log(rng, 64, 8192)
        M -= M % rng.choice((1, 8, 8, 64)) if M >= 64 else 0
        rows = _log(rng, 1, min(16384, 8192 * 4096 // M))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if rng.random() < 0.35:
            return norm("bwd", rows, M, dtype, res=rng.random() < 0.7, pad=rng.choice((0, 0, 8, 3)))
        return norm("fwd", rows, M, dtype, rng.choice(("same", "e4m3")), rng.random() < 0.7, rng.choice((0, 0, 8, 3)))
    if op == "gated":
        M, N = _log(rng, 128, 4096), _log(rng, 128, 8192)
        if rng.random() < 0.6:
            M, N = max(128, M // 64 * 64), max(128, N // 64 * 64)
        rows = _log(rng, 1, 64) if rng.random() < 0.4 else _log(rng, 65, 8192)
        act, bias = rng.choice(("silu", "silu", "gelu", "gelu_tanh", "relu")), rng.random() < 0.4
        pick = rng.random()
        if pick < 0.35:
            return gated("bwd", rows, M, N, "bf16", act, bias)
        if pick < 0.6:
            return gated("fwd", rows, M, N, "e4m3", act, bias)
        return gated("fwd", rows, M, N, "bf16", act, bias, keep=rng.random() < 0.5)
    V = _log(rng, 100, 150000)
    rows = _log(rng, 1, max(1, min(8192, 4096 * 131072 // V // 2)))
    K = min(V // 2, _log(rng, 1, 128))
    return distill(rng.choice(("both", "both", "bwd", "loss")), rows, V, K, rng.choice(("bf16", "bf16", "f32")),
                   rng.random() < 0.5, rng.choice((1.0, 2.0, 4.0)))


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _rows_apart(rows, cols, dtype, pad=0):
    """An uninitialised matrix whose rows start on multiples of 16 bytes (of one element where pad is not 0)."""
    q = 16 // dtype.itemsize
    ld = cols + pad if pad else -(-cols // q) * q
    return torch.empty(rows, ld, dtype=dtype, device=DEV)[:, :cols]


def _randn(g, rows, cols, dtype, scale=1.0, pad=0):
    out = _rows_apart(rows, cols, dtype, pad)
    out.copy_(torch.randn(rows, cols, generator=g, device=DEV).mul_(scale))
    return out


def _quantised(x):
    """Rows of x in e4m3 with a scale each."""
    scale = x.abs().amax(1, keepdim=True).clamp_min(1e-20) / E4M3_MAX
    q = _rows_apart(x.shape[0], x.shape[1], torch.float8_e4m3fn)
    q.copy_(x / scale)
    return q, scale.flatten().contiguous()


def _prepare_norm(c, g):
    t, rows, M, pad = TYPES[c["dtype"]], c["rows"], c["M"], c["pad"]
    # activations of a residual stream: a few features are far larger than the others
    feature = torch.exp(0.5 * torch.randn(M, generator=g, device=DEV))
    s = {"x": _rows_apart(rows, M, t, pad), "res": _rows_apart(rows, M, t, pad) if c["res"] else None, "eps": 1e-5,
         "w": 1.0 + 0.2 * torch.randn(M, generator=g, device=DEV)}
    s["x"].copy_(torch.randn(rows, M, generator=g, device=DEV) * feature)
    if c["res"]:
        s["res"].copy_(torch.randn(rows, M, generator=g, device=DEV) * 2 * feature)
    if c["way"] == "fwd":
        s["sum"] = _rows_apart(rows, M, t, pad) if c["res"] else None
        s["y"] = _rows_apart(rows, M, t if c["y"] == "same" else TYPES["e4m3"], pad)
        s["y_scale"] = torch.empty(rows, device=DEV) if c["y"] == "e4m3" else None
        s["rstd"] = torch.empty(rows, device=DEV)
    else:
        s["s"] = s.pop("x")                       # the sum that the forward pass left
        s["dsum"] = s.pop("res")                  # the gradient that comes along the residual
        s["dy"] = _randn(g, rows, M, t, 1e-3, pad)
        s["rstd"] = torch.rsqrt(s["s"].float().square().mean(1) + s["eps"])
        s["dx"], s["dw"] = _rows_apart(rows, M, t, pad), torch.empty(M, device=DEV)
        if s["dsum"] is not None:
            s["dsum"].mul_(1e-3)
    if own:
        from paper_2010_01546_b200 import binding as B
        kinds = {"f32": B.FW_F32, "bf16": B.FW_BF16}
        s["desc"] = B.fw_norm_desc_default(M, dtype=kinds[c["dtype"]], eps=s["eps"],
                                           y_dtype=B.FW_E4M3 if c["y"] == "e4m3" else kinds[c["dtype"]])
        if c["way"] == "bwd":
            s["scratch"] = torch.empty(B.fw_rmsnorm_scratch_bytes(s["desc"]), dtype=torch.uint8, device=DEV)
    return s


def _prepare_gated(c, g):
    rows, M, N = c["rows"], c["M"], c["N"]
    bf16 = torch.bfloat16
    s = {k: None for k in ("x_scale", "wg_scale", "wu_scale", "bg", "bu", "Zg", "Zu")}
    # rows as a norm leaves them, weights of the usual initial size
    X, Wg, Wu = (torch.randn(r, M, generator=g, device=DEV) * w for r, w in ((rows, 1.0), (N, M ** -0.5), (N, M ** -0.5)))
    if c["bias"]:
        s["bg"], s["bu"] = (0.3 * torch.randn(N, generator=g, device=DEV) for _ in range(2))
    if c["dtype"] == "e4m3":
        (s["X"], s["x_scale"]), (s["Wg"], s["wg_scale"]), (s["Wu"], s["wu_scale"]) = (_quantised(v) for v in (X, Wg, Wu))
    else:
        for name, v in (("X", X), ("Wg", Wg), ("Wu", Wu)):
            s[name] = _rows_apart(v.shape[0], M, bf16)
            s[name].copy_(v)
    if c["way"] == "bwd" or c["keep"]:
        s["Zg"], s["Zu"] = (_rows_apart(rows, N, bf16) for _ in range(2))
    if c["way"] == "bwd":
        for z, w, b in (("Zg", "Wg", "bg"), ("Zu", "Wu", "bu")):
            v = (s["X"] @ s[w].T).float()
            s[z].copy_(v if s[b] is None else v + s[b])
        s["dH"] = _randn(g, rows, N, bf16, 1e-2)
        s["dX"] = _rows_apart(rows, M, bf16)
        s["dWg"], s["dWu"] = (torch.empty(N, M, dtype=bf16, device=DEV) for _ in range(2))
        s["dbg"], s["dbu"] = (torch.empty(N, device=DEV) if c["bias"] else None for _ in range(2))
    else:
        s["H"] = _rows_apart(rows, N, bf16)
    if own:
        from paper_2010_01546_b200 import binding as B
        act = {"silu": B.FW_ACT_SILU, "gelu": B.FW_ACT_GELU, "gelu_tanh": B.FW_ACT_GELU_TANH, "relu": B.FW_ACT_RELU}
        s["block"] = B.Gated(M, N, rows, x_dtype=B.FW_E4M3 if c["dtype"] == "e4m3" else B.FW_BF16, act=act[c["act"]],
                             grad=c["way"] == "bwd")
    return s


def _prepare_distill(c, g):
    rows, V, K, t = c["rows"], c["V"], c["K"], TYPES[c["dtype"]]
    z = torch.randn(rows, V, generator=g, device=DEV).mul_(2.0)
    s = {"Z": _rows_apart(rows, V, t), "tau": c["tau"], "t_lse": None, "stat": torch.empty(rows, 2, device=DEV)}
    s["Z"].copy_(z)
    # a teacher that agrees with the student to some degree; its K top logits in 16 bits, as they are kept on disk
    z.mul_(0.8).add_(torch.randn(rows, V, generator=g, device=DEV).mul_(1.5))
    top, at = torch.topk(z, K, dim=1)
    if c["rest"]:
        s["t_lse"] = torch.logsumexp(z / c["tau"], 1)
    del z
    s["T"], s["I"] = top.to(torch.bfloat16), at.to(torch.int32)
    if K > 3:
        s["I"][::7, K - 2:] = -1                  # a teacher that gave fewer for some rows
    # the mean over the rows that count: prompt tokens and padding do not
    s["weight"] = torch.where(torch.arange(rows, device=DEV) % 16 == 5, 0.0, c["tau"] ** 2 / rows)
    s["loss"] = torch.empty(rows, device=DEV)
    s["dZ"] = _rows_apart(rows, V, t) if c["way"] != "loss" else None
    if c["way"] == "bwd":
        zz = s["Z"].float() / s["tau"]
        s["stat"][:, 0] = torch.logsumexp(zz, 1)
        there = s["I"] >= 0
        zz[torch.arange(rows, device=DEV)[:, None].expand(rows, K)[there], s["I"].long()[there]] = float("-inf")
        s["stat"][:, 1] = torch.logsumexp(zz, 1)
    if own:
        from paper_2010_01546_b200 import binding as B
        s["desc"] = B.fw_distill_desc_default(V, K, z_dtype=B.FW_F32 if c["dtype"] == "f32" else B.FW_BF16, t_dtype=B.FW_BF16,
                                              tau=c["tau"])
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"norm": _prepare_norm, "gated": _prepare_gated, "distill": _prepare_distill}[case["op"]](case, g)
    s["case"] = case
    return s


# ----------------------------------------------------------------------------
# the framework's calls
# ----------------------------------------------------------------------------
def _own_norm(c, s):
    from paper_2010_01546_b200 import binding as B
    if c["way"] == "fwd":
        B.fw_rmsnorm_forward(s["desc"], s["x"], s["w"], s["y"], res=s["res"], sum_out=s["sum"], y_scale=s["y_scale"], rstd=s["rstd"])
    else:
        B.fw_rmsnorm_backward(s["desc"], s["dy"], s["s"], s["w"], s["rstd"], s["dx"], dw=s["dw"], dsum=s["dsum"], scratch=s["scratch"])


def _own_gated(c, s):
    if c["way"] == "fwd":
        s["block"].forward(s["X"], s["Wg"], s["Wu"], s["H"], Zg=s["Zg"], Zu=s["Zu"], x_scale=s["x_scale"], wg_scale=s["wg_scale"],
                           wu_scale=s["wu_scale"], bg=s["bg"], bu=s["bu"])
    else:
        s["block"].backward(s["dH"], s["X"], s["Wg"], s["Wu"], s["Zg"], s["Zu"], dX=s["dX"], dWg=s["dWg"], dWu=s["dWu"],
                            dbg=s["dbg"], dbu=s["dbu"])


def _own_distill(c, s):
    from paper_2010_01546_b200 import binding as B
    if c["way"] == "bwd":
        B.fw_distill_backward(s["desc"], s["Z"], s["T"], s["I"], s["stat"], s["dZ"], t_lse=s["t_lse"], weight=s["weight"])
    else:
        B.fw_distill_forward(s["desc"], s["Z"], s["T"], s["I"], s["loss"], stat=s["stat"], t_lse=s["t_lse"], weight=s["weight"],
                             dZ=s["dZ"])


# ----------------------------------------------------------------------------
# the plain forms
# ----------------------------------------------------------------------------
def _plain_norm(c, s):
    if c["way"] == "fwd":
        v = s["x"].float()
        if c["res"]:
            s["sum"].copy_(v + s["res"].float())   # the sum is kept in its own type, and normalised as it is kept
            v = s["sum"].float()
        s["rstd"].copy_(torch.rsqrt(v.square().mean(1) + s["eps"]))
        y = v * s["rstd"][:, None] * s["w"]
        if c["y"] == "e4m3":
            top = y.abs().amax(1)
            s["y_scale"].copy_(torch.where(top > 0, top / E4M3_MAX, 1.0))
            y = y / s["y_scale"][:, None]
        s["y"].copy_(y)
    else:
        v, u, r = s["s"].float(), s["dy"].float(), s["rstd"][:, None]
        uw = u * s["w"]
        dx = r * (uw - v * (r * r * (uw * v).mean(1, keepdim=True)))
        s["dx"].copy_(dx if s["dsum"] is None else dx + s["dsum"].float())
        s["dw"].copy_((u * v * r).sum(0))


def _act(name, a):
    if name == "silu":
        return a * torch.sigmoid(a)
    if name == "gelu":
        return 0.5 * a * (1 + torch.erf(a * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * a * (1 + torch.tanh(math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)))
    return a.clamp_min(0)


def _act_grad(name, a):
    if name == "silu":
        p = torch.sigmoid(a)
        return p * (1 + a * (1 - p))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(a * math.sqrt(0.5))) + a * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3))
        return 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * a * a)
    return (a > 0).to(a.dtype)


def _plain_gated(c, s):
    if c["way"] == "fwd":
        x = s["X"].float()
        a, b = x @ s["Wg"].float().T, x @ s["Wu"].float().T
        if s["x_scale"] is not None:
            a, b = a * s["x_scale"][:, None] * s["wg_scale"], b * s["x_scale"][:, None] * s["wu_scale"]
        if c["bias"]:
            a, b = a + s["bg"], b + s["bu"]
        if c["keep"]:
            s["Zg"].copy_(a)
            s["Zu"].copy_(b)
        s["H"].copy_(_act(c["act"], a) * b)
    else:
        a, b, dh, x = s["Zg"].float(), s["Zu"].float(), s["dH"].float(), s["X"].float()
        da, db = dh * b * _act_grad(c["act"], a), dh * _act(c["act"], a)
        s["dX"].copy_(da @ s["Wg"].float() + db @ s["Wu"].float())
        s["dWg"].copy_(da.T @ x)
        s["dWu"].copy_(db.T @ x)
        if c["bias"]:
            s["dbg"].copy_(da.sum(0))
            s["dbu"].copy_(db.sum(0))


def _teacher(s, T, t_lse):
    """Probabilities of the teacher's entries (0 for absent ones) and of the rest, in T's type."""
    there = s["I"] >= 0
    t = torch.where(there, T / s["tau"], float("-inf"))
    if t_lse is not None:
        p = torch.exp(t - t_lse[:, None])
        return p, (1 - p.sum(1)).clamp_min(0)
    p = torch.exp(t - t.amax(1, keepdim=True))
    return p / p.sum(1, keepdim=True), None


def _plain_distill(c, s):
    there, at = s["I"] >= 0, s["I"].clamp_min(0).long()
    p, rest = _teacher(s, s["T"].float(), s["t_lse"])
    z, w = s["Z"].float() / s["tau"], s["weight"]
    zk = z.gather(1, at)
    if c["way"] == "bwd":
        lse, lse_rest = s["stat"][:, 0], s["stat"][:, 1]
    else:
        top = z.amax(1)
        lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
        # the classes that the teacher does not name, by themselves; an absent entry takes nothing out
        out = torch.zeros_like(z, dtype=torch.bool).scatter_add_(1, at, there)
        other = torch.where(out, float("-inf"), z)
        high = other.amax(1).clamp_min(-1e30)
        lse_rest = high + torch.log(torch.exp(other - high[:, None]).sum(1))
        del out, other
        term = torch.where(p > 0, p * (torch.log(p) - (zk - lse[:, None])), 0).sum(1)
        if rest is not None:
            term = term + torch.where(rest > 0, rest * (torch.log(rest) - (lse_rest - lse)), 0)
        s["loss"].copy_(torch.where(w != 0, w * term, 0))
        s["stat"].copy_(torch.where(w[:, None] != 0, torch.stack((lse, lse_rest), 1), 0))
    if c["way"] != "loss":
        whole = p.sum(1) if rest is None else p.sum(1) + rest
        q = torch.exp(z - lse[:, None])
        qk = q.gather(1, at)
        outside = q * (whole if rest is None else whole - rest * torch.exp(lse - lse_rest))[:, None]
        # the entries' places: what `outside` gave them leaves, and their own gradient comes
        outside.scatter_add_(1, at, torch.where(there, whole[:, None] * qk - p - outside.gather(1, at), 0))
        s["dZ"].copy_(outside * torch.where(w != 0, w / s["tau"], 0)[:, None])


def _outputs(c, s):
    if c["op"] == "norm":
        names = ("sum", "y", "y_scale", "rstd") if c["way"] == "fwd" else ("dx", "dw")
    elif c["op"] == "gated":
        names = ("H",) + (("Zg", "Zu") if c["keep"] else ()) if c["way"] == "fwd" else ("dX", "dWg", "dWu", "dbg", "dbu")
    else:
        names = {"loss": ("loss", "stat"), "both": ("loss", "stat", "dZ"), "bwd": ("dZ",)}[c["way"]]
    return {n: s[n] for n in names if s[n] is not None}


def run(state):
    c = state["case"]
    if own:
        {"norm": _own_norm, "gated": _own_gated, "distill": _own_distill}[c["op"]](c, state)
    else:
        {"norm": _plain_norm, "gated": _plain_gated, "distill": _plain_distill}[c["op"]](c, state)
    return _outputs(c, state)


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------
def work(case):
    c, rows = case, case["rows"]
    e = BYTES[c["dtype"]]
    if c["op"] == "norm":
        n = rows * c["M"]
        if c["way"] == "fwd":
            y = e if c["y"] == "same" else 1
            return {"bytes": n * (e * (3 if c["res"] else 1) + y) + 4 * c["M"] + 4 * rows * (2 if c["y"] == "e4m3" else 1), "flops": 6 * n}
        return {"bytes": n * e * (4 if c["res"] else 3) + 8 * c["M"] + 4 * rows, "flops": 10 * n}
    if c["op"] == "gated":
        M, N = c["M"], c["N"]
        if c["way"] == "fwd":
            scales = 4 * (rows + 2 * N) if c["dtype"] == "e4m3" else 0
            return {"bytes": e * (rows * M + 2 * N * M) + 2 * rows * N * (3 if c["keep"] else 1) + scales + (8 * N if c["bias"] else 0),
                    "flops": 4 * rows * N * M}
        return {"bytes": 2 * (2 * rows * M + 4 * N * M + 3 * rows * N) + (8 * N if c["bias"] else 0), "flops": 8 * rows * N * M}
    live = rows - len(range(5, rows, 16))          # rows of weight 0 are not read
    z, entries = c["V"] * e, c["K"] * 6 + (4 if c["rest"] else 0) + 8
    write = 0 if c["way"] == "loss" else rows * z
    return {"bytes": live * (z + entries) + write + rows * (4 if c["way"] == "bwd" else 16), "flops": live * c["V"] * (3 if c["way"] == "loss" else 6)}


# ----------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------
def _exact_norm(c, s):
    d = torch.float64
    if c["way"] == "fwd":
        v = s["x"].to(d)
        if c["res"]:
            v = (v + s["res"].to(d)).to(s["x"].dtype).to(d)
        rstd = (v.pow(2).sum(1) / c["M"] + s["eps"]).pow(-0.5)
        y = v * s["w"].to(d) * rstd[:, None]
        out = {"y": y, "rstd": rstd}
        if c["res"]:
            out["sum"] = v
        if c["y"] == "e4m3":
            scale = y.abs().max(1).values / E4M3_MAX
            scale[scale == 0] = 1
            out["y_scale"], out["y"] = scale, (y / scale[:, None]).to(torch.float8_e4m3fn).to(d)
        return out
    v, dy, w, r = s["s"].to(d), s["dy"].to(d), s["w"].to(d), s["rstd"].to(d)
    n = v * r[:, None]                            # y = n w: the gradient of n, less its part along n
    dn = dy * w
    dx = (dn - n * ((dn * n).sum(1) / c["M"])[:, None]) * r[:, None]
    return {"dx": dx if s["dsum"] is None else dx + s["dsum"].to(d), "dw": torch.einsum("rm,rm->m", dy, n)}


def _exact_act(name, a):
    """Value and derivative."""
    if name == "relu":
        return torch.where(a > 0, a, 0), torch.where(a > 0, 1.0, 0.0).to(a)
    if name == "silu":
        e = torch.exp(-a)
        return a / (1 + e), 1 / (1 + e) + a * e / (1 + e) ** 2
    if name == "gelu":
        cdf = torch.special.ndtr(a)
        return a * cdf, cdf + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    k = 2 * math.sqrt(2 / math.pi)                # (1 + tanh(x)) / 2 is the logistic function of 2 x
    u = k * (a + 0.044715 * a.pow(3))
    p = 1 / (1 + torch.exp(-u))
    return a * p, p + a * p * (1 - p) * k * (1 + 0.134145 * a.pow(2))


def _exact_gated(c, s):
    d = torch.float64
    x, wg, wu = s["X"].to(d), s["Wg"].to(d), s["Wu"].to(d)
    if c["way"] == "fwd":
        if c["dtype"] == "e4m3":
            x, wg, wu = (v * t.to(d)[:, None] for v, t in ((x, s["x_scale"]), (wg, s["wg_scale"]), (wu, s["wu_scale"])))
        a, b = torch.mm(x, wg.t()), torch.mm(x, wu.t())
        if c["bias"]:
            a += s["bg"].to(d)
            b += s["bu"].to(d)
        out = {"H": _exact_act(c["act"], a)[0] * b}
        return {**out, "Zg": a, "Zu": b} if c["keep"] else out
    f, df = _exact_act(c["act"], s["Zg"].to(d))
    dh = s["dH"].to(d)
    da, db = dh * s["Zu"].to(d) * df, dh * f
    out = {"dX": torch.addmm(torch.mm(da, wg), db, wu), "dWg": torch.mm(da.t(), x), "dWu": torch.mm(db.t(), x)}
    if c["bias"]:
        out["dbg"], out["dbu"] = da.sum(0), db.sum(0)
    return out


def _exact_distill(c, s):
    d = torch.float64
    rows, V = s["Z"].shape
    z = s["Z"].to(d).div_(s["tau"])
    there = s["I"] >= 0
    row = torch.arange(rows, device=DEV)[:, None].expand_as(s["I"])[there]
    col = s["I"].long()[there]
    t = (s["T"].to(d) / s["tau"]).masked_fill(~there, float("-inf"))
    logp = t - (torch.logsumexp(t, 1) if s["t_lse"] is None else s["t_lse"].to(d))[:, None]
    logp, p = logp.masked_fill(~there, 0), logp.exp()
    pt = None if s["t_lse"] is None else (1 - p.sum(1)).clamp(min=0)
    w = s["weight"].to(d)
    if c["way"] == "bwd":
        lse, lse_rest = s["stat"].to(d).unbind(1)
    else:
        lse = torch.logsumexp(z, 1)
        hidden = z.clone()
        hidden[row, col] = float("-inf")
        lse_rest = torch.logsumexp(hidden, 1)
        del hidden
    out = {}
    if c["way"] != "bwd":
        logq = torch.zeros_like(p)
        logq[there] = z[row, col] - lse[row]
        kl = (p * (logp - logq)).sum(1)
        if pt is not None:
            kl += torch.special.xlogy(pt, pt) - torch.where(pt > 0, pt * (lse_rest - lse), 0)
        out["loss"] = torch.where(w != 0, w * kl, 0)
        out["stat"] = torch.where(w[:, None] != 0, torch.stack((lse, lse_rest), 1), 0)
    if c["way"] != "loss":
        # d loss / dZ = w / tau (softmax over all (sum p + p_t) - p_t softmax over the rest - p)
        mass = p.sum(1) + (0 if pt is None else pt)
        dz = (z - lse[:, None]).exp_()
        inside = dz[row, col] * mass[row] - p[there]
        if pt is None:
            dz *= mass[:, None]
        else:
            dz *= (mass - torch.where(pt > 0, pt * (lse - lse_rest).exp(), 0))[:, None]
        dz[row, col] = inside
        out["dZ"] = dz * (w / s["tau"])[:, None]
    return out


def exact(case, seed):
    global own
    was, own = own, False                         # the inputs alone, no handle
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"norm": _exact_norm, "gated": _exact_gated, "distill": _exact_distill}[case["op"]](case, s)
