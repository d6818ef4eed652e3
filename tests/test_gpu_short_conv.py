"""kata_fwd_short_conv, kata_decode_short_conv and kata_bwd_short_conv against the definition in 64 bits."""
import pytest
import torch

from paper_2607_17419_b200 import binding as kb

from mixer_ref import F32, ROUND, conv, conv_bound, live_mask, within

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}

CASES = [  # dtype, B, T, D, W, silu, bias, extra columns of the rows
    ("bf16", 2, 100, 64, 4, True, True, 0), ("f32", 2, 100, 64, 4, True, True, 0), ("bf16", 1, 1, 8, 4, True, True, 0), ("bf16", 3, 2, 24, 4, False, False, 8),
    ("f32", 1, 65, 1, 2, True, False, 0), ("bf16", 2, 130, 513, 3, True, True, 64), ("f32", 2, 7, 20, 3, False, True, 3), ("bf16", 40, 5, 136, 2, True, True, 0),
    ("bf16", 1, 1300, 1024, 4, True, True, 64), ("f32", 1, 9, 100, 4, True, False, 28), ("bf16", 300, 1, 40, 3, False, True, 0),
]


def tensors(dtype, B, T, D, W, bias, extra, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(DT[dtype])
    return n(B, T, D + extra)[..., :D], n(D, W), n(D) if bias else None, n(B, D, W - 1), n(B, T, D + extra)[..., :D], gen


def ragged(B, T, gen):
    n = torch.randint(0, T + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
    n[0] = 0
    n[-1] = T
    return n


@pytest.mark.parametrize("dtype,B,T,D,W,silu,bias,extra", CASES)
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("padded", [False, True])
def test_forward(dtype, B, T, D, W, silu, bias, extra, state, padded):
    x, w, b, s, _, gen = tensors(dtype, B, T, D, W, bias, extra)
    lengths = ragged(B, T, gen) if padded else None
    y, S, mag = conv(x, w, b, silu, s if state else None, lengths)
    live = live_mask(lengths, B, T, "cuda")
    x = x.clone().masked_fill(~live[..., None], float("nan")) if padded else x
    first = s.clone() if state else None
    last = torch.full_like(s, float("nan"))
    out = kb.kata_fwd_short_conv(x, w, b, silu=silu, s_init=first, s_final=last, lengths=lengths)
    within(out, y, conv_bound(y, mag, W, DT[dtype], silu), "out")
    assert torch.equal(last.double(), S), "state"
    assert first is None or torch.equal(first, s)
    if state:                                                   # in place, into a given output
        given = torch.full((B, T, D + 8), 3.0, device="cuda", dtype=x.dtype)
        out2 = kb.kata_fwd_short_conv(x, w, b, silu=silu, s_init=first, s_final=first, lengths=lengths, out=given[..., :D])
        assert torch.equal(out2, out) and torch.equal(first, last) and torch.all(given[..., D:] == 3)


@pytest.mark.parametrize("dtype,B,T,D,W,silu,bias,extra", CASES)
@pytest.mark.parametrize("padded", [False, True])
def test_backward(dtype, B, T, D, W, silu, bias, extra, padded):
    x, w, b, _, g, gen = tensors(dtype, B, T, D, W, bias, extra, 1)
    lengths = ragged(B, T, gen) if padded else None
    live = live_mask(lengths, B, T, "cuda")[..., None]
    x64, w64, b64 = x.double().requires_grad_(), w.double().requires_grad_(), b.double().requires_grad_() if bias else None
    y, _, mag = conv(x64, w64, b64, silu, None, lengths)
    ref = torch.autograd.grad(y, [x64, w64] + ([b64] if bias else []), g.double())
    hole = (lambda t: t.clone().masked_fill(~live, float("inf"))) if padded else (lambda t: t)
    dx, dw, db = kb.kata_bwd_short_conv(hole(g), hole(x), w, b, silu=silu, lengths=lengths)
    assert (db is None) == (not bias) and dw.dtype == torch.float32
    # g act'(z): the slope's own slope is below 1, z is off by (W + 1) roundings of its terms, the sigmoid by 2^-20
    off = ((W + 1) * F32 * mag.detach() + (2.0 ** -19 + 4 * F32) * 1.2) * g.double().abs() if silu else F32 * g.double().abs()
    off = off.masked_fill(~live, 0)
    size = (1.2 if silu else 1.0) * g.double().abs().masked_fill(~live, 0)
    pad = lambda t: torch.nn.functional.pad(t, (0, 0, 0, W - 1))
    reach = lambda t: sum(pad(t)[:, j:j + T] * w.double()[:, W - 1 - j].abs() for j in range(W))
    within(dx, ref[0], reach(off) + (W + 1) * F32 * reach(size) + 1.01 * ROUND[DT[dtype]] * ref[0].abs() + 1e-38, "dx")
    xa = torch.cat([x64.new_zeros(B, W - 1, D), x64.detach().masked_fill(~live, 0).abs()], 1)
    taps = lambda t: torch.stack([(t * xa[:, j:j + T]).sum((0, 1)) for j in range(W)], 1)
    n = min(B * T, 400)                                          # roundings in a row: 64 tokens, the segments of a block, its share of the blocks
    within(dw, ref[1], taps(off) + (n + 20) * F32 * taps(size) + 1e-38, "dw")
    if bias:
        within(db, ref[2], off.sum((0, 1)) + (n + 20) * F32 * size.sum((0, 1)) + 1e-38, "db")
    assert torch.all(dx.masked_select(~live.expand_as(dx)) == 0)
    again = kb.kata_bwd_short_conv(hole(g), hole(x), w, b, silu=silu, lengths=lengths)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    # differences of the definition along a direction
    dirx, dirw = torch.randn(B, T, D, device="cuda", generator=gen).double().masked_fill(~live, 0), torch.randn(D, W, device="cuda", generator=gen).double()
    f = lambda e: float((conv(x.double() + e * dirx, w.double() + e * dirw, b, silu, None, lengths)[0] * g.double().masked_fill(~live, 0)).sum())
    slope = (f(1e-5) - f(-1e-5)) / 2e-5
    got = float((dx.double() * dirx).sum() + (dw.double() * dirw).sum())
    slack = float(((dx.double() - ref[0]).abs() * dirx.abs()).sum() + ((dw.double() - ref[1]).abs() * dirw.abs()).sum())
    assert abs(got - slope) <= slack + 1e-4 * float(g.double().norm()) * (1 + float(w.double().norm()))


@pytest.mark.parametrize("dtype,B,D,W", [("bf16", 1, 64, 4), ("bf16", 33, 1152, 4), ("f32", 3, 7, 2), ("bf16", 2, 513, 3)])
def test_steps_are_the_forward(dtype, B, D, W):
    x, w, b, s, _, _ = tensors(dtype, B, 9, D, W, True, 8)
    whole, last = s.clone(), s.clone()
    y = kb.kata_fwd_short_conv(x, w, b, silu=True, s_init=whole, s_final=last)
    for t in range(9):
        out = kb.kata_decode_short_conv(x[:, t], w, whole, b, silu=True)
        assert torch.equal(out, y[:, t])
    assert torch.equal(whole, last)


def test_extreme_values():
    """z sigmoid(z) far out: 0 and z, never NaN."""
    x = torch.tensor([-1e30, -200.0, -90.0, 0.0, 90.0, 200.0, 1e30], device="cuda")[None, :, None].repeat(1, 1, 8)
    w = torch.tensor([0.0, 1.0], device="cuda").repeat(8, 1)
    for dt in (torch.float32, torch.bfloat16):
        y = kb.kata_fwd_short_conv(x.to(dt), w.to(dt), silu=True)
        ref = torch.where(x > 0, x, torch.zeros_like(x)).to(dt)
        assert torch.allclose(y.float(), ref.float(), rtol=1e-2, atol=1e-30)
        dx = kb.kata_bwd_short_conv(torch.ones_like(x).to(dt), x.to(dt), w.to(dt), silu=True)[0]
        assert torch.allclose(dx.float()[0, :, 0], torch.tensor([0, 0, 0, 0.5, 1, 1, 1], device="cuda"), atol=1e-2)


def test_offsets_beyond_32_bits():
    x = torch.empty((1 << 31) + 4096, device="cuda", dtype=torch.bfloat16)
    v = torch.as_strided(x, (2, 8, 64), (1 << 31, 64, 1))
    v.copy_(torch.randn(2, 8, 64, device="cuda"))
    w = torch.randn(64, 4, device="cuda").bfloat16()
    assert torch.equal(kb.kata_fwd_short_conv(v, w, silu=True), kb.kata_fwd_short_conv(v.contiguous(), w, silu=True))


@pytest.mark.parametrize("T,D", [(5, 64), (200, 64), (200, 63)])
def test_broadcast_and_shifted_views(T, D):
    """One sequence for all of a batch, and rows that begin at any entry: the same sums whatever path reads them."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    n = lambda *s: torch.randn(*s, device="cuda", generator=gen).bfloat16()
    x, w, b, g = n(1, T, D), n(D, 4), n(D), n(3, T, D)
    wide = x.expand(3, -1, -1)
    want = kb.kata_fwd_short_conv(wide.contiguous(), w, b, silu=True)
    assert torch.equal(kb.kata_fwd_short_conv(wide, w, b, silu=True), want)
    grads = kb.kata_bwd_short_conv(g, wide.contiguous(), w, b, silu=True)
    assert all(torch.equal(p, q) for p, q in zip(kb.kata_bwd_short_conv(g, wide, w, b, silu=True), grads))
    for shift in (1, 2, 8):
        room = n(3, T, D + 16)
        room[..., shift:shift + D] = x
        y = kb.kata_fwd_short_conv(room[..., shift:shift + D], w, b, silu=True)
        dx, dw, db = kb.kata_bwd_short_conv(g, room[..., shift:shift + D], w, b, silu=True)
        assert torch.equal(y, want) and torch.equal(dx, grads[0])
        # (the same 3 T terms summed in another order: 3 T roundings on each side of sums no larger than the terms' sizes, SiLU's slope
        # at most 1.1; a shifted sum of products is at most the product of the norms)
        sizes = (1.1 * g.double().norm(dim=(0, 1)) * (3.0 ** 0.5) * x.double().norm(dim=(0, 1)), 1.1 * g.double().abs().sum((0, 1)))
        for p, q, size in ((dw, grads[1], sizes[0][:, None]), (db, grads[2], sizes[1])):
            assert torch.all((p - q).abs() <= 2 * 3 * T * F32 * size)


LARGE = [  # sizes whose forward goes through shared memory: dtype, B, T, D, W, silu, bias, extra columns of the rows
    ("bf16", 5, 500, 1024, 4, True, True, 0), ("bf16", 2, 1100, 1032, 3, False, False, 8), ("bf16", 130, 129, 136, 2, True, True, 0),
    ("bf16", 3, 40000, 24, 4, True, True, 0), ("f32", 3, 2801, 1004, 4, True, True, 4),
]


@pytest.mark.parametrize("dtype,B,T,D,W,silu,bias,extra", LARGE)
@pytest.mark.parametrize("state,padded", [(False, False), (True, True)])
def test_large_forward(dtype, B, T, D, W, silu, bias, extra, state, padded):
    test_forward(dtype, B, T, D, W, silu, bias, extra, state, padded)


@pytest.mark.parametrize("dtype,B,T,D,W,silu,bias,extra", LARGE[:3])
@pytest.mark.parametrize("padded", [False, True])
def test_large_backward(dtype, B, T, D, W, silu, bias, extra, padded):
    test_backward(dtype, B, T, D, W, silu, bias, extra, padded)


@pytest.mark.parametrize("T,D", [(300, 4096), (70, 64)])
def test_long_sequences_beyond_32_bits(T, D):
    x = torch.empty((1 << 31) + T * D, device="cuda", dtype=torch.bfloat16)
    v = torch.as_strided(x, (2, T, D), (1 << 31, D, 1))
    v.copy_(torch.randn(2, T, D, device="cuda"))
    w, g = torch.randn(D, 4, device="cuda").bfloat16(), torch.randn(2, T, D, device="cuda").bfloat16()
    assert torch.equal(kb.kata_fwd_short_conv(v, w, silu=True), kb.kata_fwd_short_conv(v.contiguous(), w, silu=True))
    for a, b in ((v, v.contiguous()), (g, g)):
        assert all(p is q or torch.equal(p, q) for p, q in zip(kb.kata_bwd_short_conv(g, a, w, silu=True), kb.kata_bwd_short_conv(g, b, w, silu=True)))
    assert torch.equal(kb.kata_bwd_short_conv(v, g, w, silu=True)[0], kb.kata_bwd_short_conv(v.contiguous(), g, w, silu=True)[0])
