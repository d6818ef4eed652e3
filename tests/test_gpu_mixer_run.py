"""The operators around the attention as a layer uses them: convolution, norm and rotation, attention with its state, then token by
token; convolution and scan likewise; replayed from a graph; on other streams."""
import pytest
import torch

from paper_2607_17419_b200 import binding as kb

from mixer_ref import conv, norm_rope, ssm

pytestmark = pytest.mark.gpu

B, H, T, TP, D = 2, 4, 150, 131, 64


def attention(q, k, v):
    """The definition of the attention in 64 bits."""
    w = (q.double() @ k.double().transpose(-1, -2)) / k.double().norm(dim=-1)[:, :, None, :].clamp_min(1e-300)
    w = w.square().tril()
    return (w @ v.double()) / w.sum(-1, keepdim=True)


def parts(seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, device="cuda", generator=gen).bfloat16()
    C = H * D
    return n(B, T, 3 * C), n(3 * C, 4), n(3 * C), 1 + 0.1 * n(D), 1 + 0.1 * n(D)


def heads(x):
    return x.view(*x.shape[:-1], 3, H, D).permute(2, 0, 3, 1, 4).unbind(0)


def test_attention_layer_prompt_then_tokens():
    x, w, b, qw, kw = parts()
    past = torch.zeros(B, 3 * H * D, 3, device="cuda", dtype=torch.bfloat16)
    n = kb.decode_n_psi(D)
    S, Z = torch.empty(B, H, n, D, device="cuda"), torch.empty(B, H, n, device="cuda")
    y = kb.kata_fwd_short_conv(x[:, :TP], w, b, silu=True, s_init=past, s_final=past)
    q, k, v = heads(y)
    q, k = kb.kata_fwd_norm_rope(q, k, qw, kw)
    outs = [kb.kata_fwd_chunked(q, k, v.contiguous(), s_pre=S, z_pre=Z)]
    pos = torch.full((B, 1), TP, device="cuda")
    for t in range(TP, T):
        y = kb.kata_decode_short_conv(x[:, t], w, past, b, silu=True)
        q, k, v = heads(y[:, None])
        q, k = kb.kata_fwd_norm_rope(q, k, qw, kw, pos)
        pos += 1
        outs.append(kb.kata_decode_step(q[:, :, 0], k[:, :, 0], v[:, :, 0].contiguous(), S, Z)[:, :, None])
    got = torch.cat(outs, 2).double()
    c = conv(x, w, b, True)[0]
    q, k, v = heads(c)
    at = torch.arange(T, device="cuda")[None].expand(B, -1)
    inv = [10000.0 ** (-2.0 * i / D) for i in range(D // 2)]
    ref = attention(norm_rope(q, qw, at, inv)[0], norm_rope(k, kw, at, inv)[0], v)
    # three roundings to bf16 on the way in (convolution, norm; 2^-8 each), those of the attention's own 2e-2 rule
    assert float((got - ref).norm() / ref.norm()) < 2e-2


def test_scan_layer_prompt_then_tokens():
    gen = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    G, N, C = 1, 64, H * D
    W = C + 2 * G * N
    x, w, b = n(B, T, W).bfloat16(), n(W, 4).bfloat16(), n(W).bfloat16()
    dt, A, skip, bias = (n(B, T, H) - 2).bfloat16(), -n(H).abs(), n(H), n(H)
    lengths = torch.tensor([TP, 60], dtype=torch.int32, device="cuda")
    past = torch.zeros(B, W, 3, device="cuda", dtype=torch.bfloat16)
    S = torch.zeros(B, H, N, D, device="cuda")

    def split(y):
        y = y if y.dim() == 3 else y[:, None]
        return (y[..., C + G * N:].view(*y.shape[:2], G, N).transpose(1, 2), y[..., C:C + G * N].view(*y.shape[:2], G, N).transpose(1, 2),
                y[..., :C].view(*y.shape[:2], H, D).transpose(1, 2))

    y = kb.kata_fwd_short_conv(x[:, :TP], w, b, silu=True, s_init=past, s_final=past, lengths=lengths)
    head = kb.kata_fwd_ssm_scan(*split(y), dt[:, :TP].transpose(1, 2), A, skip, bias, dt_softplus=True, s_init=S, s_final=S, lengths=lengths)
    tail = []
    for t in range(5):                                            # every sequence goes on behind its own end
        rows, i = lengths.long() + t, torch.arange(B, device="cuda")
        q, k, v = split(kb.kata_decode_short_conv(x[i, rows], w, past, b, silu=True))
        tail.append(kb.kata_decode_ssm_step(q[:, :, 0], k[:, :, 0], v[:, :, 0], dt[i, rows], A, S, skip, bias, dt_softplus=True))
    for s in range(B):
        L = int(lengths[s])
        c = conv(x[s:s + 1, :L + 5], w, b, True)[0]
        ref = ssm(*split(c), dt[s:s + 1, :L + 5].transpose(1, 2), A, skip, bias, True)[0]
        got = torch.cat([head[s:s + 1, :, :L], torch.stack([o[s:s + 1] for o in tail], 2)], 2).double()
        assert float((got - ref).norm() / ref.norm()) < 1e-2      # the convolution's rounding and the scan's, 2^-8 each at most
        assert torch.all(head[s, :, L:] == 0)


def calls():
    gen = torch.Generator(device="cuda").manual_seed(2)
    n = lambda *s: torch.randn(*s, device="cuda", generator=gen).bfloat16()
    x, w, g = n(2, 300, 128), n(128, 4), n(2, 300, 128)
    q, k, gq = n(2, 4, 300, 64), n(2, 2, 300, 64), n(2, 4, 300, 64)
    dt, A = n(2, 4, 3000), -torch.rand(4, device="cuda", generator=gen)
    qs, v = n(2, 2, 3000, 64), n(2, 4, 3000, 64)
    wq = n(64)
    return {
        "conv": lambda **kw: kb.kata_fwd_short_conv(x, w, silu=True, **kw),
        "conv_bwd": lambda **kw: kb.kata_bwd_short_conv(g, x, w, silu=True, **kw),
        "rope": lambda **kw: kb.kata_fwd_norm_rope(q, k, wq, wq, **kw),
        "rope_bwd": lambda **kw: kb.kata_bwd_norm_rope(gq, gq[:, :2], q, k, wq, wq, **kw),
        "scan": lambda **kw: kb.kata_fwd_ssm_scan(qs, qs, v, dt, A, dt_softplus=True, **kw),
        "scan_simt": lambda **kw: kb.kata_fwd_ssm_scan(qs, qs, v, dt, A, dt_softplus=True, impl=kb.KATA_IMPL_SIMT, **kw),
    }


def flat(x):
    return [t for t in (x if isinstance(x, tuple) else (x,)) if t is not None]


@pytest.mark.parametrize("name", ["conv", "conv_bwd", "rope", "rope_bwd", "scan", "scan_simt"])
def test_captured_and_replayed(name):
    f = calls()[name]
    want = [t.clone() for t in flat(f())]
    torch.cuda.synchronize()
    stream, graph, graph2 = torch.cuda.Stream(), torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            got = flat(f())
        with torch.cuda.graph(graph2, stream=stream):             # a second graph: scratch of its own
            got2 = flat(f())
        for _ in range(3):
            for t in got + got2:
                t.zero_()
            graph.replay()
            graph2.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(want, got, got2):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("name", ["conv", "conv_bwd", "rope", "rope_bwd", "scan", "scan_simt"])
def test_two_streams_at_once(name):
    f = calls()[name]
    want = flat(f())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(flat(f()))
    named = flat(f(stream=streams[0].cuda_stream))                # a stream by its handle
    torch.cuda.synchronize()
    for g in got + [named]:
        assert all(torch.equal(a, b) for a, b in zip(want, g))
