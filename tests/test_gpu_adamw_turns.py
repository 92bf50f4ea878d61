"""AdamW over networks large enough that a warp's turn is several blocks, against its formula in 64 bits.

Error bounds: those of test_gpu_adamw.py.  m may be as near 0 as its terms cancel (0.9 m + 0.1 g is exactly 0 for g = -9 m, which bf16 holds for an
m of four bits), so its sign is open where it is less than its error, 4 u of its terms' sizes: up to 2^-22 x 448 = 2^-13 of the scale, a sixteenth of
the smallest code, which chance takes one time in sixteen.  Codes are therefore compared with their signs, between those of m less and plus its error.
"""
import pytest
import torch

from optest_util import F64, U
from test_gpu_adamw import B, BLOCK, begin, choose, formula, mix, scale_of, states, tensors  # noqa: F401

pytestmark = pytest.mark.gpu

BETA1, BETA2, SEED, LR = 0.9, 0.999, 5, 1e-2


def check_large(B, opt, P, G, copies, before, t, sizes, decay, c, clip_err):
    P0, m0, v0 = before
    got_m, got_v = states(B, opt, sizes)
    bits8 = opt.desc.state == B.FW_E4M3
    codes = [opt.state(f).to(F64) for f in (B.FW_A_M, B.FW_A_V)] if bits8 else None
    at = 0
    for i, n in enumerate(sizes):
        m1, v1, p1, size, rate = formula(P0[i], G[i], m0[i], v0[i], t, LR, decay[i], c, BETA1, BETA2, 1e-8)
        em, ev = (4 * U + clip_err) * size, (8 * U + 2 * clip_err) * v1
        assert bool(((P[i].to(F64) - p1).abs() <= 3 * U * P0[i].to(F64).abs() + rate * (em + (20 * U + clip_err) * m1.abs()) + U * p1.abs()).all()), i
        if copies[i] is not None:
            assert torch.equal(copies[i], P[i].bfloat16())
        if not bits8:
            assert bool(((got_m[i] - m1).abs() <= em).all()) and bool(((got_v[i] - v1).abs() <= ev).all()), i
        else:
            k = -(-n // BLOCK)
            pad = lambda x: torch.nn.functional.pad(x, (0, k * BLOCK - n)).view(k, BLOCK)  # noqa: E731
            chance = mix(torch.arange(at, at + k * BLOCK, device="cuda") ^ mix((SEED ^ (t * 0x9E3779B9)) & 0xFFFFFFFF)).view(k, BLOCK)
            r1 = v1.sqrt()
            er = (ev / (2 * r1)).nan_to_num(0) + 4 * U * r1
            for value, err, ch, square, field, flat in ((m1, em, chance & 0xFFFF, False, B.FW_A_M_SCALE, codes[0]),
                                                        (r1, er, chance >> 16, True, B.FW_A_V_SCALE, codes[1])):
                s = opt.state(field).to(F64)[at // BLOCK:at // BLOCK + k]
                top, most = pad(value.abs()).amax(1), pad(err).amax(1)
                assert bool(((s >= scale_of(top - most)) & (s <= scale_of(top + most))).all()), (i, field)
                code = flat[at:at + k * BLOCK].view(k, BLOCK)
                signed = lambda x: x.sign() * choose(x.abs(), s[:, None], ch, square)  # noqa: E731, B023
                lo = signed(pad(value) - pad(err) if not square else (pad(value) - pad(err)).clamp(min=0))
                hi = signed(pad(value) + pad(err))
                assert bool(((code >= lo) & (code <= hi)).all()), (i, field)
                assert float((lo != hi).double().mean()) < 1e-2 or n < 5000
                assert bool((code.view(-1)[n:] == 0).all())                      # behind the last element
        at += -(-n // BLOCK) * BLOCK


@pytest.mark.parametrize("kind,turn", [("f32", 2), ("f32", 3), ("f32", 4), ("f32", 6), ("e4m3", 2), ("e4m3", 3), ("e4m3", 5), ("e4m3", 8), ("e4m3", 9)])
@pytest.mark.parametrize("shift,clip", [(0, 0.3), (1, 0.3), (0, None)])
def test_turns_of_several_blocks(B, kind, turn, shift, clip):  # noqa: F811
    """A turn is `turn` blocks (4 at most, 8 with 8-bit states): tensors that are one turn, that end inside one, inside a block, or behind a first
    element."""
    blocks = turn * 24 * torch.cuda.get_device_properties(0).multi_processor_count + 5
    sizes = [256 * turn, 3 * 256 * turn + 256 + 17, 255, 256 * turn + 1, 100001, 2 * 256 * turn - 3]
    left = blocks - sum(-(-n // BLOCK) for n in sizes)
    sizes += [left // 2 * BLOCK - 100, (left - left // 2) * BLOCK - 255]
    P, G = tensors(sizes, 60 + turn, shift, half=(1, 4, 6))
    copies = [torch.empty_like(p, dtype=torch.bfloat16) if i % 2 == 0 else None for i, p in enumerate(P)]
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    opt = B.AdamW(P, copies=copies, decay=decay, state=B.FW_E4M3 if kind == "e4m3" else B.FW_F32, seed=SEED)
    norm = torch.empty(1, device="cuda") if clip else None
    want = float(sum(g.to(F64).square().sum() for g in G).sqrt())
    c = min(1.0, clip / want) if clip else 1.0
    for t in (1, 2):
        if t == 2:
            begin(B, opt, sizes, 61)
        before = ([p.clone() for p in P], *states(B, opt, sizes))
        opt.step(G, LR, max_norm=clip or 0.0, norm_out=norm)
        if clip:
            assert abs(float(norm) - want) <= 33 * U * want
        check_large(B, opt, P, G, copies, before, t, sizes, decay, c, 33 * U if c < 1 else 0.0)
        assert int(opt.state(B.FW_A_STEP)) == t


@pytest.mark.parametrize("size", [1e-19, 1e-17, 1e-8, 1.0, 1e9, 1e18])
def test_8_bit_states_of_any_size(B, size):  # noqa: F811
    """First steps of gradients that differ by up to fourteen orders within a block, at sizes where v is subnormal, where its scale's square or the
    inverse of it is beyond fp32, and where it is near the largest number: v within 8 u of itself and two steps of subnormal numbers."""
    n = 20 * BLOCK - 7
    g = torch.Generator(device="cuda")
    g.manual_seed(17)
    far = 10.0 ** (-14 * torch.rand(n, generator=g, device="cuda").square())
    G = torch.randn(n, generator=g, device="cuda") * far * size
    G[3 * BLOCK + 5] = 0
    P = torch.zeros(n, device="cuda")
    opt = B.AdamW([P], state=B.FW_E4M3, seed=SEED, eps=1e-36)
    opt.step([G], LR)
    gd = torch.nn.functional.pad(G.to(F64), (0, 7)).view(-1, BLOCK)
    m1, v1 = (1 - BETA1) * gd, (1 - BETA2) * gd * gd
    ev, em = 8 * U * v1 + 2.0 ** -148, 4 * U * m1.abs() + 2.0 ** -148
    chance = mix(torch.arange(gd.numel(), device="cuda") ^ mix((SEED ^ 0x9E3779B9) & 0xFFFFFFFF)).view(-1, BLOCK)
    for field, scales, low, high, ch, square in ((B.FW_A_V, B.FW_A_V_SCALE, (v1 - ev).clamp(min=0).sqrt(), (v1 + ev).sqrt() * (v1 > 0), chance >> 16, True),
                                                 (B.FW_A_M, B.FW_A_M_SCALE, (m1.abs() - em).clamp(min=0), (m1.abs() + em) * (m1 != 0), chance & 0xFFFF, False)):
        s, code = opt.state(scales).to(F64), opt.state(field).to(F64).view(-1, BLOCK).abs()
        assert bool(((s >= scale_of(low.amax(1))) & (s <= scale_of(high.amax(1)))).all()), field
        assert bool(((code >= choose(low, s[:, None], ch, square)) & (code <= choose(high, s[:, None], ch, square))).all()), field
        if square:
            held = v1 > 2.0 ** -148
            assert bool((code[held] > 0).all()) and bool((code[gd == 0] == 0).all())      # what is not 0 is not held as 0
    p1 = -LR * (m1 / (1 - BETA1)) / ((v1 / (1 - BETA2)).sqrt() + 1e-36)
    err = 24 * U + 0.5 * 2.0 ** -149 / v1.clamp(min=1e-60)
    ok = (torch.nn.functional.pad(P.to(F64), (0, 7)).view(-1, BLOCK) - p1).abs() <= err * p1.abs()
    assert bool(ok[v1 > 2.0 ** -140].all())
