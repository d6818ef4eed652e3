"""Scan and short convolution where their arithmetic has corners: step sizes far from one another, entries that are not finite."""
import pytest
import torch

from paper_2607_17419_b200 import binding as kb

from mixer_ref import F32, conv, conv_bound, live_mask, ssm, within
from test_gpu_short_conv import ragged as conv_ragged, tensors as conv_tensors, test_backward as conv_backward
from test_gpu_ssm import check, tensors

pytestmark = pytest.mark.gpu


def both_forms(dt, A, n, seed, T):
    """Tensor cores and token by token against the recurrence, with and without a state."""
    B, H = dt.shape[:2]
    q, k, v, _, _, D, _, init, _ = tensors("bf16", B, H, 1, T, n, 64, seed)
    for first in (None, init):
        ref = ssm(q, k, v, dt, A, init=first)
        for impl in (kb.KATA_IMPL_TENSOR, kb.KATA_IMPL_SIMT):
            S = torch.empty_like(init)
            out = kb.kata_fwd_ssm_scan(q, k, v, dt, A, s_init=first, s_final=S, impl=impl)
            check(out, S, ref, "bf16", T, n, impl == kb.KATA_IMPL_TENSOR)


@pytest.mark.parametrize("n", [64, 128])
@pytest.mark.parametrize("at", [0, 7, 30, 31])
def test_one_large_step_of_a_slow_head(n, at):
    """The decay of a block is of ordinary size, the step alone is large: products of factors must not leave fp32."""
    H, T = 8, 200
    dt = torch.full((1, H, T), 0.01, device="cuda").bfloat16()
    dt[:, :, at::96] = 1000.0
    A = torch.tensor([-0.05, -0.08, -0.11, -0.14, -0.16, -0.165, -0.168, -0.17], device="cuda")
    both_forms(dt, A, n, 31, T)


@pytest.mark.parametrize("size", [2.0 ** -20, 2.0 ** -40, 2.0 ** -60])
def test_small_steps_before_a_strong_decay(size):
    """Steps of next to nothing in a block that decays by up to 2^230: their own outputs are as exact as others."""
    H, T = 4, 200
    dt = torch.full((2, H, T), size, device="cuda").bfloat16()
    dt[0, :, 20::64] = 1.0
    dt[1, :, 3::32] = 1.0
    A = torch.tensor([-60.0, -100.0, -130.0, -158.0], device="cuda")
    both_forms(dt, A, 64, 33, T)


@pytest.mark.parametrize("large,small,rate", [(1e5, 0.01, -16.0), (1000.0, 1e-4, -1000.0), (3e4, 0.05, -8.0), (40.0, 0.02, -11.0)])
def test_small_steps_around_one_that_forgets(large, small, rate):
    """A step that forgets everything, anywhere in a block, with ordinary ones before and behind it: what they lose to one another
    must not drown in what that step loses."""
    places = [0, 1, 2, 3, 5, 10, 15, 30, 31]
    T = 200
    dt = torch.full((len(places), 2, T), small, device="cuda").bfloat16()
    for b, at in enumerate(places):
        dt[b, :, at::96] = large
    both_forms(dt, torch.tensor([rate, 0.5 * rate], device="cuda"), 64, 35, T)


def test_options_without_a_truth_or_too_large():
    """An option that has no truth, or no 32 bits, raises what it raises through ctypes, and nothing is left pending."""
    two = torch.tensor([True, False])
    x, w, q = (torch.zeros(*s, device="cuda", dtype=torch.bfloat16) for s in ((2, 5, 64), (64, 4), (1, 2, 5, 64)))
    dt, A = torch.zeros(1, 2, 5, device="cuda", dtype=torch.bfloat16), torch.zeros(2, device="cuda")
    for call in (lambda: kb.kata_fwd_short_conv(x, w, silu=two), lambda: kb.kata_bwd_short_conv(x, x, w, silu=two), lambda: kb.kata_fwd_norm_rope(q, interleaved=two),
                 lambda: kb.kata_fwd_ssm_scan(q, q, q, dt, A, dt_softplus=two)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            call()
    for impl in (1 << 70, -(1 << 70), 1 << 32):
        with pytest.raises(ValueError, match="impl"):
            kb.kata_fwd_ssm_scan(q, q, q, dt, A, impl=impl)


def conv_case(T, lengths, silu, seed=5):
    """bf16 rows of whole units, 48 tokens or more: gradients through tiles; the same rows one entry further on: token by token."""
    B, D, W = 4, 1024, 4
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, device="cuda", generator=gen).bfloat16()
    x, w, b, g = n(B, T, D), n(D, W), n(D), n(B, T, D)
    room = torch.empty(B, T, D + 8, device="cuda", dtype=torch.bfloat16)
    return B, D, W, x, w, b, g, room[..., 1:1 + D]


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0))


@pytest.mark.parametrize("T", [48, 64, 150])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("what", [float("inf"), float("nan")])
def test_rows_behind_the_end_are_zeros(T, silu, what):
    """The last live inputs are not finite: what they make of a gradient stays in front of the end, whichever way rows are read."""
    lengths = torch.tensor([T, T - 2, 17, 1], dtype=torch.int32, device="cuda")
    B, D, W, x, w, b, g, shifted = conv_case(T, lengths, silu)
    for s, L in enumerate(lengths.tolist()):
        x[s, max(0, L - 2):L, 3::64] = what
    shifted.copy_(x)
    live = live_mask(lengths, B, T, "cuda")[..., None]
    tile = kb.kata_bwd_short_conv(g, x, w, b, silu=silu, lengths=lengths)
    walk = kb.kata_bwd_short_conv(g, shifted, w, b, silu=silu, lengths=lengths)
    for dx, _, _ in (tile, walk):
        assert torch.all(dx.masked_select(~live.expand_as(dx)) == 0)
    assert same(tile[0], walk[0])
    clean = torch.ones(D, dtype=torch.bool, device="cuda")
    clean[3::64] = False
    for _, dw, db in (tile, walk):
        assert torch.isfinite(dw[clean]).all() and torch.isfinite(db[clean]).all()


@pytest.mark.parametrize("T", [48, 64, 150])
@pytest.mark.parametrize("padded", [False, True])
def test_sums_take_the_tokens_of_the_sequences_alone(T, padded):
    """Without an activation an infinite last input meets one tap alone; the sums of the others have no term behind the end."""
    lengths = torch.tensor([T, T - 2, 17, 5], dtype=torch.int32, device="cuda") if padded else None
    B, D, W, x, w, b, g, shifted = conv_case(T, lengths, False)
    ends = lengths.tolist() if padded else [T] * B
    x64 = x.double()
    for s, L in enumerate(ends):
        x[s, L - 1, 3::64] = float("inf")
        g[s, L - 1, 3::64] = 1.0
    shifted.copy_(x)
    live = live_mask(lengths, B, T, "cuda")[..., None]
    g64 = g.double().masked_fill(~live, 0)
    for s, L in enumerate(ends):
        x64[s, L - 1, 3::64] = 0                                  # (its only term is that of the last tap)
    line = torch.cat([x64.new_zeros(B, W - 1, D), x64.masked_fill(~live, 0)], 1)
    ref = torch.stack([(line[:, j:j + T] * g64).sum((0, 1)) for j in range(W)], 1)
    size = torch.stack([(line[:, j:j + T] * g64).abs().sum((0, 1)) for j in range(W)], 1)
    for rows in (x, shifted):
        _, dw, db = kb.kata_bwd_short_conv(g, rows, w, b, silu=False, lengths=lengths)
        assert torch.all(dw[3::64, W - 1] == float("inf"))
        ok = torch.ones_like(dw, dtype=torch.bool)
        ok[3::64, W - 1] = False
        assert torch.isfinite(dw[ok]).all() and torch.isfinite(db).all()
        # (4 T terms in a row at most, each product and sum rounded once)
        assert torch.all(((dw - ref).abs() <= (B * T + 20) * F32 * size + 1e-38)[ok])


FILLS = [  # channels from few to many, with sequences that fill tiles of shared memory and sequences that do not: B, T, D, W
    (150, 1024, 16, 4), (1100, 128, 16, 4), (40, 512, 64, 2), (300, 130, 32, 3), (3000, 100, 8, 2), (130, 2048, 8, 4), (24, 900, 128, 2), (600, 64, 64, 3),
]


@pytest.mark.parametrize("B,T,D,W", FILLS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_convolution_of_few_and_many_channels(dtype, B, T, D, W):
    """Forward and backward whatever way rows are read; a shifted copy of the rows, which goes token by token, gives the same bits."""
    x, w, b, s, g, gen = conv_tensors(dtype, B, T, D, W, True, 0, 37)
    lengths = conv_ragged(B, T, gen)
    y, S, mag = conv(x, w, b, True, s, lengths)
    last = torch.empty_like(s)
    out = kb.kata_fwd_short_conv(x, w, b, silu=True, s_init=s, s_final=last, lengths=lengths)
    within(out, y, conv_bound(y, mag, W, x.dtype, True), "out")
    assert torch.equal(last.double(), S)
    room = torch.empty(B, T, D + 8, device="cuda", dtype=x.dtype)
    shifted = room[..., 1:1 + D]
    shifted.copy_(x)
    assert torch.equal(kb.kata_fwd_short_conv(shifted, w, b, silu=True, s_init=s, lengths=lengths), out)
    assert torch.equal(kb.kata_bwd_short_conv(g, shifted, w, b, silu=True, lengths=lengths)[0], kb.kata_bwd_short_conv(g, x, w, b, silu=True, lengths=lengths)[0])
    conv_backward(dtype, B, T, D, W, True, True, 0, True)


def test_the_time_of_few_channels_does_not_grow_with_their_tiles():
    """Sequences that fill an eighth of a tile, or less, are not worked on in tiles: with the same entries eight channels take no more
    than four times what 1024 take (the walk 1.4 times; in tiles it was 13 and 6 times)."""
    def us(f):
        f()
        a, z = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        best = 1e9
        for _ in range(5):
            torch.cuda.synchronize()
            a.record()
            for _ in range(10):
                f()
            z.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(z) * 100)
        return best

    times = {}
    for D in (8, 1024):
        B, T = (1 << 24) // (128 * D), 128
        x, w, b, _, g, _ = conv_tensors("bf16", B, T, D, 4, True, 0, 39)
        out, dx, ws = torch.empty_like(x), torch.empty_like(x), kb.Workspace()
        times[D] = (us(lambda: kb.kata_fwd_short_conv(x, w, b, silu=True, out=out)), us(lambda: kb.kata_bwd_short_conv(g, x, w, b, silu=True, dx=dx, workspace=ws)))
    assert times[8][0] <= 4 * times[1024][0] and times[8][1] <= 4 * times[1024][1], times


@pytest.mark.parametrize("B,H,T,n,dtype", [(2, 16, 3001, 64, "bf16"), (4, 16, 3001, 128, "bf16"), (3, 4, 2000, 32, "f32")])
def test_a_full_batch_with_lengths_is_the_batch_without(B, H, T, n, dtype):
    """The token axis is cut by the sizes alone: lengths that fill the batch change neither the segments nor a bit."""
    q, k, v, dt, A, D, bias, init, _ = tensors(dtype, B, H, 1, T, n, 64, 41)
    full = torch.full((B,), T, dtype=torch.int32, device="cuda")
    for state in (False, True):
        a, b = (torch.empty_like(init), torch.empty_like(init)) if state else (None, None)
        with_lengths = kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, s_init=init, s_final=a, lengths=full)
        assert torch.equal(with_lengths, kb.kata_fwd_ssm_scan(q, k, v, dt, A, D, bias, dt_softplus=True, s_init=init, s_final=b))
        assert a is None or torch.equal(a, b)
