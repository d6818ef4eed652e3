"""kata_fwd_norm_rope and kata_bwd_norm_rope against the definition in 64 bits."""
import pytest
import torch

from paper_2607_17419_b200 import binding as kb

from mixer_ref import F32, ROUND, norm_rope, turn, within

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def freqs(r, base=10000.0):
    return [base ** (-2.0 * i / r) for i in range(r // 2)]


def forward_bound(x, w, pos, inv, inter, dtype, eps=1e-6):
    """r: d + 4 roundings of a sum of squares, halved by the root; sine and cosine: half turns rounded to fp32 (2^-24 pi) and two
    units of the function, on top of the products' four roundings."""
    y, size = norm_rope(x, w, pos, inv, inter, eps)
    return y, ((x.shape[-1] + 4) / 2 + 12) * F32 * size + 1.01 * ROUND[dtype] * y.abs() + 1e-37


CASES = [  # dtype, B, H, Hk, T, d, rot, interleaved
    ("bf16", 2, 4, 2, 37, 64, 64, False), ("f32", 2, 4, 2, 37, 64, 64, False), ("bf16", 1, 3, 1, 1, 64, 32, True), ("f32", 3, 1, 5, 65, 128, 128, True),
    ("bf16", 1, 16, 16, 300, 128, 64, False), ("bf16", 5, 7, 0, 13, 16, 16, False), ("f32", 1, 2, 2, 9, 16, 16, False), ("f32", 2, 3, 3, 33, 32, 16, False),
    ("bf16", 1, 2, 3, 70, 32, 0, False), ("bf16", 700, 1, 1, 3, 64, 48, False), ("f32", 1, 33, 2, 2, 64, 16, True),
]


def tensors(dtype, B, H, Hk, T, d, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = normal(gen, B, T, H + Hk + 1, d).to(DT[dtype])                 # (one head more: the views skip it)
    q, k = x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hk].transpose(1, 2) if Hk else None
    w = [(1 + 0.2 * normal(gen, d)).to(DT[dtype]) for _ in range(2)]
    pos = torch.randint(0, 5000, (B, T), device="cuda", generator=gen)
    return gen, q, k, w[0], w[1] if Hk else None, pos


@pytest.mark.parametrize("dtype,B,H,Hk,T,d,rot,inter", CASES)
def test_forward(dtype, B, H, Hk, T, d, rot, inter):
    _, q, k, qw, kw, pos = tensors(dtype, B, H, Hk, T, d)
    out = kb.kata_fwd_norm_rope(q, k, qw, kw, pos, rotary_dim=rot, interleaved=inter)
    assert out[0].is_contiguous() and (out[1] is None) == (k is None)
    for o, x, w in zip(out, (q, k), (qw, kw)):
        if x is not None:
            within(o, *forward_bound(x, w, pos, freqs(rot) if rot else [], inter, DT[dtype]), "out")


@pytest.mark.parametrize("dtype,B,H,Hk,T,d,rot,inter", CASES)
def test_backward(dtype, B, H, Hk, T, d, rot, inter):
    gen, q, k, qw, kw, pos = tensors(dtype, B, H, Hk, T, d, 1)
    inv = freqs(rot) if rot else []
    go = [normal(gen, *x.shape).to(x.dtype) if x is not None else None for x in (q, k)]
    dq, dk, dqw, dkw = kb.kata_bwd_norm_rope(go[0], go[1], q, k, qw, kw, pos, rotary_dim=rot, interleaved=inter)
    again = kb.kata_bwd_norm_rope(go[0], go[1], q, k, qw, kw, pos, rotary_dim=rot, interleaved=inter)
    for a, b in zip((dq, dk, dqw, dkw), again):
        assert a is None or torch.equal(a, b)
    for x, g, w, dx, dw in ((q, go[0], qw, dq, dqw), (k, go[1], kw, dk, dkw)):
        if x is None:
            assert dx is None and dw is None
            continue
        x64, w64 = x.double().requires_grad_(), w.double().requires_grad_()
        y = norm_rope(x64, w64, pos, inv, inter)[0]
        rx, rw = torch.autograd.grad(y, [x64, w64], g.double())
        # every entry of dx is r (z w - u m): z from one pair, m the mean of d products; every factor within (d + 20) roundings
        r = 1 / torch.sqrt(x.double().square().mean(-1, keepdim=True) + 1e-6)
        u = x.double() * r
        size = turn(g.double(), -pos.double(), inv, inter)[1]
        zw = size * w.double().abs()
        terms = r * (zw + u.abs() * (zw * u.abs()).mean(-1, keepdim=True))
        within(dx, rx, (d + 20) * F32 * terms + 1.01 * ROUND[DT[dtype]] * rx.abs() + 1e-37, "dx")
        n = x.shape[0] * x.shape[1] * x.shape[2]
        # a sum of n terms in runs: no entry passes more than n + 40 roundings
        within(dw, rw, (min(n, 2000) + d + 40) * F32 * (size * u.abs()).sum((0, 1, 2)), "dw")
        # and against differences of the definition along a direction
        h, dirx, dirw = 1e-5, normal(gen, *x.shape).double(), normal(gen, d).double()
        f = lambda e: float((norm_rope(x.double() + e * dirx, w.double() + e * dirw, pos, inv, inter)[0] * g.double()).sum())
        slope = (f(h) - f(-h)) / (2 * h)
        got = float((dx.double() * dirx).sum() + (dw.double() * dirw).sum())
        slack = float(((d + 20) * F32 * terms + ROUND[DT[dtype]] * 1.01 * rx.abs()).mul(dirx.abs()).sum()) + 1e-3 * float(g.double().norm())
        assert abs(got - slope) <= slack


def test_no_weights_no_norm_of_positions():
    """Without weights and positions: ones, and offset + t; any base; negative positions turn back."""
    _, q, k, _, _, _ = tensors("f32", 2, 2, 2, 11, 32)
    out = kb.kata_fwd_norm_rope(q, k, offset=-4, base=500.0, eps=1e-3)
    pos = (torch.arange(11, device="cuda") - 4)[None].expand(2, -1)
    for o, x in zip(out, (q, k)):
        within(o, *forward_bound(x, None, pos, freqs(32, 500.0), False, torch.float32, 1e-3), "out")


@pytest.mark.parametrize("first", [0, 131072, (1 << 31) - 3, 1 << 40])
def test_far_positions(first):
    """Far positions keep their angles: the fraction of a turn is exact to 2^-64 per position.  (The reference's float64 angles
    are off by 2^-53 of themselves, so it takes the turn modulo one in integers too beyond 2^31.)"""
    _, q, _, _, _, _ = tensors("f32", 1, 2, 0, 6, 64)
    pos = first + torch.arange(6, device="cuda")
    inv = freqs(64)
    got = kb.kata_fwd_norm_rope(q, None, positions=pos)[0]
    from fractions import Fraction
    import math
    two_pi = Fraction(6283185307179586476925286766559005768394, 10 ** 39)
    small = torch.tensor([[float((Fraction(int(p)) * Fraction(f) / two_pi) % 1 * two_pi) for f in inv] for p in pos.tolist()], dtype=torch.float64, device="cuda")
    x = q.double()
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    a, b = y[..., :32], y[..., 32:]
    ref = torch.cat([a * torch.cos(small) - b * torch.sin(small), a * torch.sin(small) + b * torch.cos(small)], -1)
    size = torch.cat([a.abs() + b.abs()] * 2, -1)
    # 2^-65 of a turn per position from the fixed point, and the 2^-53 of inv_freq / 2 pi in the reference's own inputs is exact
    drift = 2 * math.pi * float(first + 6) * 2.0 ** -64
    within(got, ref, ((64 + 4) / 2 + 12) * F32 * size + drift * size + F32 * ref.abs(), "far")


def test_strides_and_outputs():
    """Views of any order, broadcast inputs, given outputs, gradients into a packed tensor."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, H, T, d = 2, 3, 19, 64
    base = normal(gen, B, H, T, d).bfloat16()
    want = kb.kata_fwd_norm_rope(base)[0]
    packed = torch.full((B, T, 2, H, d), 7.0, device="cuda", dtype=torch.bfloat16)
    packed[:, :, 0] = base.transpose(1, 2)
    out = torch.full((T, B, H, 2 * d), 5.0, device="cuda", dtype=torch.bfloat16)
    view = out[..., d:].permute(1, 2, 0, 3)
    got = kb.kata_fwd_norm_rope(packed[:, :, 0].transpose(1, 2), q_out=view)[0]
    assert got.data_ptr() == view.data_ptr() and torch.equal(got, want) and torch.all(out[..., :d] == 5) and torch.all(packed[:, :, 1] == 7)
    one = base[:, :1].expand(B, H, T, d)
    assert torch.equal(kb.kata_fwd_norm_rope(one)[0], kb.kata_fwd_norm_rope(one.contiguous())[0])
    g = normal(gen, B, H, T, d).bfloat16()
    ref = kb.kata_bwd_norm_rope(g, None, base)[0]
    grads = torch.full_like(packed, 3.0)
    kb.kata_bwd_norm_rope(g, None, packed[:, :, 0].transpose(1, 2), dq=grads[:, :, 1].transpose(1, 2))
    assert torch.equal(grads[:, :, 1].transpose(1, 2), ref) and torch.all(grads[:, :, 0] == 3)


def test_misaligned_rows_are_refused():
    x = torch.zeros(2 * 3 * 5 * 64 + 8, device="cuda", dtype=torch.bfloat16)
    q = x[1:1 + 2 * 3 * 5 * 64].view(2, 3, 5, 64)
    with pytest.raises(kb.KataError):
        kb.kata_fwd_norm_rope(q)


def test_offsets_beyond_32_bits():
    """Two sequences 2^31 entries apart."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.empty((1 << 31) + 4096, device="cuda", dtype=torch.bfloat16)
    q = torch.as_strided(x, (2, 2, 8, 64), (1 << 31, 512, 64, 1))
    q.copy_(normal(gen, 2, 2, 8, 64))
    assert torch.equal(kb.kata_fwd_norm_rope(q)[0], kb.kata_fwd_norm_rope(q.contiguous())[0])


def test_large_and_small_rows():
    """Rows of any size have norm one unless eps counts; a zero row stays zero."""
    x = torch.ones(1, 1, 4, 64, device="cuda") * torch.tensor([0.0, 1e-15, 1.0, 1e15], device="cuda")[None, None, :, None]
    y = kb.kata_fwd_norm_rope(x, rotary_dim=0, eps=1e-20)[0]
    assert torch.all(y[0, 0, 0] == 0) and (y[0, 0, 2:] - 1).abs().max() < 1e-6
    assert (y[0, 0, 1].double() - 1e-15 / (1e-30 + 1e-20) ** 0.5).abs().max() < 1e-6 * 1e-5
