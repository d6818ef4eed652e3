"""kata_fwd_ssm_scan and kata_decode_ssm_step against the recurrence in 64 bits."""
import pytest
import torch

from paper_2607_17419_b200 import binding as kb

from mixer_ref import F32, ROUND, live_mask, ssm, within

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def tensors(dtype, B, H, G, T, n, d, seed=0, packed=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    x = r(B, T, H * d + 2 * G * n).to(DT[dtype])
    v = x[..., :H * d].view(B, T, H, d).transpose(1, 2)
    k = x[..., H * d:H * d + G * n].view(B, T, G, n).transpose(1, 2)
    q = x[..., H * d + G * n:].view(B, T, G, n).transpose(1, 2)
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    dt = (r(B, T, H) - 3).to(DT[dtype]).transpose(1, 2)
    A = -torch.rand(H, device="cuda", generator=gen) * 8
    A[0] = 0                                                      # (a head that forgets nothing)
    return q, k, v, dt, A, r(H), 0.3 * r(H), r(B, H, n, d), gen


def steps_bound(T, n):
    """Roundings that a term passes on its way in fp32: the decay of every token (the exponential's two units, its argument's and
    one of the product), the sum with every token, the n terms of the output."""
    return (6 * T + n + 30) * F32


def check(out, S, ref, dtype, T, n, tensor):
    y, s, mag, smag = ref
    # tensor cores: a term passes the bf16 rounding of its weight inside its chunk or, through the state, those of its scaled value
    # and of the state; its decay is a product of two exponentials, whose exponents (up to 800 in 32 tokens) are fp32 roundings
    extra = 2.02 * ROUND[torch.bfloat16] + 2.0 ** -13 if tensor else 0.0
    within(out, y, (steps_bound(T, n) + extra) * mag + 1.01 * ROUND[DT[dtype]] * y.abs() + 1e-37, "out")
    if S is not None:
        within(S, s, (steps_bound(T, n) + (2.0 ** -16 if tensor else 0)) * smag + 1e-37, "state")


CASES = [  # dtype, B, H, G, T, n, d, impl
    ("f32", 1, 2, 1, 1, 16, 16, 0), ("f32", 2, 4, 2, 50, 64, 64, 0), ("f32", 1, 2, 1, 300, 128, 32, 0), ("f32", 2, 3, 3, 17, 32, 64, 0),
    ("bf16", 1, 2, 1, 1, 64, 64, 2), ("bf16", 3, 2, 1, 40, 128, 64, 2), ("bf16", 1, 2, 1, 64, 64, 64, 0), ("bf16", 2, 4, 2, 130, 64, 64, 0), ("bf16", 2, 4, 1, 127, 128, 64, 0), ("bf16", 1, 2, 2, 129, 64, 64, 0),
    ("bf16", 1, 4, 4, 300, 128, 64, 0), ("bf16", 1, 3, 1, 640, 64, 64, 0), ("bf16", 1, 2, 1, 257, 16, 32, 0), ("bf16", 2, 2, 1, 40, 32, 16, 0),
    ("bf16", 2, 4, 2, 130, 64, 64, 1), ("bf16", 200, 1, 1, 260, 64, 64, 0), ("bf16", 1, 1, 1, 128, 128, 64, 0), ("f32", 1, 1, 1, 700, 16, 64, 0),
]


@pytest.mark.parametrize("dtype,B,H,G,T,n,d,impl", CASES)
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("padded", [False, True])
def test_forward(dtype, B, H, G, T, n, d, impl, state, padded):
    q, k, v, dt, A, D, bias, init, gen = tensors(dtype, B, H, G, T, n, d)
    lengths = None
    if padded:
        lengths = torch.randint(0, T + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
        lengths[0] = 0 if B > 1 else max(1, T - 3)
    ref = ssm(q, k, v, dt, A, D, bias, True, init if state else None, lengths)
    if padded:                                                    # what lies behind the ends may be anything
        dead = ~live_mask(lengths, B, T, "cuda")[:, None, :, None]
        q, k, v = (x.clone().masked_fill(dead, float("nan")) for x in (q, k, v))
        dt = dt.clone().masked_fill(dead[..., 0], float("inf"))
    first, last = (init.clone() if state else None), torch.full_like(init, float("nan"))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, s_init=first, s_final=last, lengths=lengths, impl=impl, device_status=err)
    tensor = kb.kata_last_impl() == kb.KATA_IMPL_TENSOR
    assert tensor == (dtype == "bf16" and n >= 64 and d == 64 and impl != 1 and (T > 64 or impl == 2))
    check(out, last, ref, dtype, T, n, tensor)
    assert int(err.item()) == 0 and (first is None or torch.equal(first, init))
    if state:                                                     # the state moved on in place, the same bits
        out2 = kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, s_init=first, s_final=first, lengths=lengths, impl=impl)
        assert torch.equal(out2, out) and torch.equal(first, last)


@pytest.mark.parametrize("dtype,H,T,n", [("bf16", 1, 5000, 64), ("bf16", 2, 3001, 128), ("f32", 1, 2100, 16)])
def test_segments(dtype, H, T, n):
    """Few heads: the token axis in segments; the same recurrence, bit for bit the same every time, also with a state in place."""
    d = 64 if dtype == "bf16" else 16
    q, k, v, dt, A, D, bias, init, gen = tensors(dtype, 1, H, 1, T, n, d, 3)
    assert kb.kata_workspace_bytes(kb.KATA_FN_SSM_SCAN, 1, H, T, n, d, 0, kb.make_opts(kb.KATA_BF16 if dtype == "bf16" else kb.KATA_F32)) > 0
    for lengths in (None, torch.tensor([T - 700], dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda")):
        ref = ssm(q, k, v, dt, A, D, bias, True, init, lengths)
        S = init.clone()
        out = kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, s_init=S, s_final=S, lengths=lengths)
        check(out, S, ref, dtype, T, n, dtype == "bf16")
        S2 = init.clone()
        assert torch.equal(kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, s_init=S2, s_final=S2, lengths=lengths), out) and torch.equal(S, S2)


def test_plain_steps_without_softplus():
    """dt as it is, no skip, no bias, contiguous tensors; a step of 0 keeps the state, a strong decay forgets it."""
    for dtype, n in (("f32", 16), ("bf16", 64)):
        q, k, v, dt, A, _, _, init, _ = tensors(dtype, 2, 2, 1, 140, n, 64, 5, packed=False)
        dt = dt.float().abs().mul(0.05).to(DT[dtype])
        dt[:, :, ::3] = 0
        dt[:, :, 100] = 60.0
        A = torch.tensor([-0.5, -8.0], device="cuda")
        ref = ssm(q, k, v, dt, A, init=init)
        S = torch.empty_like(init)
        out = kb.kata_fwd_ssm_scan(q, k, v, dt, A, s_init=init, s_final=S)
        check(out, S, ref, dtype, 140, n, dtype == "bf16")


@pytest.mark.parametrize("dtype,B,H,G,n,d", [("f32", 1, 2, 1, 16, 16), ("bf16", 3, 4, 2, 64, 64), ("bf16", 20, 16, 1, 128, 64), ("bf16", 1, 16, 1, 64, 64),
                                             ("f32", 2, 3, 3, 32, 32), ("bf16", 70, 2, 1, 32, 64), ("bf16", 100, 2, 2, 64, 32), ("f32", 5, 1, 1, 128, 16)])
def test_steps(dtype, B, H, G, n, d):
    T = 7
    q, k, v, dt, A, D, bias, init, _ = tensors(dtype, B, H, G, T, n, d, 7)
    ref = ssm(q, k, v, dt, A, D, bias, True, init)
    S = init.clone()
    outs = [kb.kata_decode_ssm_step(q[:, :, t], k[:, :, t], v[:, :, t], dt[:, :, t], A, S, D, bias, dt_softplus=True) for t in range(T)]
    check(torch.stack(outs, 2), S, ref, dtype, T, n, False)


def test_a_prompt_in_pieces_and_steps():
    """A sequence fed in pieces and then token by token is the whole sequence."""
    T, cut = 400, (0, 130, 131, 387)
    q, k, v, dt, A, D, bias, init, _ = tensors("bf16", 2, 4, 1, T, 64, 64, 9)
    ref = ssm(q, k, v, dt, A, D, bias, True, init)
    S, outs = init.clone(), []
    for a, b in zip(cut, cut[1:]):
        outs.append(kb.kata_fwd_ssm_scan(q[:, :, a:b], k[:, :, a:b], v[:, :, a:b], dt[:, :, a:b], A, D, bias, dt_softplus=True, s_init=S, s_final=S))
    for t in range(cut[-1], T):
        outs.append(kb.kata_decode_ssm_step(q[:, :, t], k[:, :, t], v[:, :, t], dt[:, :, t], A, S, D, bias, dt_softplus=True)[:, :, None])
    check(torch.cat(outs, 2), S, ref, "bf16", T, 64, True)


def test_offsets_beyond_32_bits():
    T = 140
    x = torch.empty((1 << 31) + 3 * T * 64, device="cuda", dtype=torch.bfloat16)
    q, k, v, dt, A, D, bias, _, _ = tensors("bf16", 2, 1, 1, T, 64, 64, 11)
    far = []
    for i, t in enumerate((q, k, v)):
        w = torch.as_strided(x[i * T * 64:], (2, 1, T, 64), (1 << 31, 64, 64, 1))
        w.copy_(t)
        far.append(w)
    for impl in (0, 1):
        want = kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, impl=impl)
        assert torch.equal(kb.kata_fwd_ssm_scan(*far, dt, A, D, bias, dt_softplus=True, impl=impl), want)


def test_misaligned_rows_are_refused():
    q, k, v, dt, A, D, bias, _, _ = tensors("bf16", 1, 2, 1, 20, 64, 64)
    x = torch.zeros(2 * 20 * 64 + 8, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(kb.KataError):
        kb.kata_fwd_ssm_scan(q, k, x[1:1 + 2 * 20 * 64].view(1, 2, 20, 64), dt, A)


@pytest.mark.parametrize("dtype,n", [("bf16", 64), ("bf16", 128), ("f32", 16)])
def test_broadcast_views(dtype, n):
    """Queries, keys and values shared by batches, heads or tokens (strides of 0) are what their copies are."""
    B, H, G, T, d = 3, 4, 2, 140, 64
    q, k, v, dt, A, D, bias, _, _ = tensors(dtype, B, H, G, T, n, d, 13, packed=False)
    cases = [(q[:1].expand(B, -1, -1, -1), k[:, :1].expand(-1, G, -1, -1), v), (q[:1, :1].expand(B, G, -1, -1), k, v[:, :1].expand(-1, H, -1, -1)),
             (q, k, v[:1].expand(B, -1, -1, -1))]
    for a, b, c in cases:
        got = kb.kata_fwd_ssm_scan(a, b, c, dt, A, D, bias, dt_softplus=True)
        assert torch.equal(got, kb.kata_fwd_ssm_scan(a.contiguous(), b.contiguous(), c.contiguous(), dt, A, D, bias, dt_softplus=True))
    # one key for all tokens: token by token
    one = k[:, :, :1].expand(-1, -1, T, -1)
    S, S2 = torch.empty(B, H, n, d, device="cuda"), torch.empty(B, H, n, d, device="cuda")
    got = kb.kata_fwd_ssm_scan(q, one, v, dt, A, D, bias, dt_softplus=True, s_final=S)
    assert kb.kata_last_impl() == kb.KATA_IMPL_SIMT
    want = kb.kata_fwd_ssm_scan(q, one.contiguous(), v, dt, A, D, bias, dt_softplus=True, s_final=S2, impl=kb.KATA_IMPL_SIMT)
    ref = ssm(q, one, v, dt, A, D, bias, True)                   # (the token axis may be cut elsewhere: not to the bit)
    check(got, S, ref, dtype, T, n, False)
    check(want, S2, ref, dtype, T, n, False)
    if dtype == "bf16":
        with pytest.raises(kb.KataError):
            kb.kata_fwd_ssm_scan(q, one, v, dt, A, D, bias, dt_softplus=True, impl=kb.KATA_IMPL_TENSOR)


def test_outputs_of_any_layout():
    """Outputs into a view of a larger tensor: its other entries stay."""
    B, H, T, d = 2, 4, 200, 64
    q, k, v, dt, A, D, bias, _, _ = tensors("bf16", B, H, 1, T, 64, d, 15)
    want = kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True)
    room = torch.full((B, T + 3, H, 2 * d), 7.0, device="cuda", dtype=torch.bfloat16)
    view = room[:, 1:T + 1, :, d:].transpose(1, 2)
    for lengths in (None, torch.tensor([5, 150], dtype=torch.int32, device="cuda")):
        room.fill_(7.0)
        got = kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, lengths=lengths, out=view)
        assert got.data_ptr() == view.data_ptr()
        if lengths is None:
            assert torch.equal(view, want)
        else:
            assert all(torch.equal(view[b, :, :n], want[b, :, :n]) and torch.all(view[b, :, n:] == 0) for b, n in enumerate(lengths.tolist()))
        assert torch.all(room[:, 0] == 7) and torch.all(room[:, T + 1:] == 7) and torch.all(room[..., :d] == 7)


@pytest.mark.parametrize("T", [1, 31, 32, 33, 64, 65, 127, 128, 129, 255, 257])
def test_lengths_at_the_borders(T):
    """Around the rules' and the tiles' borders, with and without a final state."""
    q, k, v, dt, A, D, bias, init, _ = tensors("bf16", 2, 2, 1, T, 64, 64, 17)
    ref = ssm(q, k, v, dt, A, D, bias, True, init)
    S = init.clone()
    check(kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, s_init=S, s_final=S), S, ref, "bf16", T, 64, True)
    check(kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, s_init=init), None, ref, "bf16", T, 64, True)


def test_steep_and_flat_decays():
    """Heads that forget everything within a token, nothing, and what lies between, on both forms."""
    B, H, T = 1, 6, 300
    q, k, v, _, _, D, _, init, _ = tensors("bf16", B, H, 1, T, 64, 64, 19)
    dt = torch.rand(B, H, T, device="cuda").bfloat16()
    dt[:, :, 40:44] = 0
    A = torch.tensor([-1000.0, -30.0, -8.0, -5.0, -1e-4, 0.0], device="cuda")
    ref = ssm(q, k, v, dt, A, D, init=init)
    for impl in (0, 1):
        S = init.clone()
        out = kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, s_init=S, s_final=S, impl=impl)
        check(out, S, ref, "bf16", T, 64, impl == 0)


@pytest.mark.parametrize("n", [64, 128])
def test_step_sizes_of_either_sign(n):
    """Without the softplus steps may be negative, and states grow in places."""
    B, H, T = 2, 3, 200
    q, k, v, _, _, D, _, init, gen = tensors("bf16", B, H, 1, T, n, 64, 21)
    dt = (0.05 * torch.randn(B, H, T, device="cuda", generator=gen)).bfloat16()
    A = torch.tensor([-2.0, 0.0, 3.0], device="cuda")
    ref = ssm(q, k, v, dt, A, D, init=init)
    for impl in (0, 1):
        S = init.clone()
        check(kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, s_init=S, s_final=S, impl=impl), S, ref, "bf16", T, n, impl == 0)


@pytest.mark.parametrize("dtype,B,H,T,n,d", [("f32", 1, 2, 512, 16, 16), ("f32", 1, 3, 3000, 64, 64), ("bf16", 1, 2, 5000, 32, 32), ("f32", 2, 2, 33, 128, 16)])
def test_segments_token_by_token(dtype, B, H, T, n, d):
    """Few heads: many short segments, the last one ragged, sequences that end before some of them begin."""
    q, k, v, dt, A, D, bias, init, _ = tensors(dtype, B, H, 1, T, n, d, 23)
    for lengths in (None, torch.tensor([T // 3, T][:B], dtype=torch.int32, device="cuda")):
        ref = ssm(q, k, v, dt, A, D, bias, True, init, lengths)
        S = init.clone()
        check(kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, s_init=S, s_final=S, lengths=lengths), S, ref, dtype, T, n, False)
        check(kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, s_init=init, lengths=lengths), None, ref, dtype, T, n, False)
