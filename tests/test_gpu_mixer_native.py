"""The calls around the attention by the native module against the same calls through ctypes (taken when a stream is named): the same
bits, the same errors, and the calls that it leaves alone."""
import pytest
import torch

from paper_2607_17419_b200 import binding as kb

pytestmark = pytest.mark.gpu


def n(*s, seed=0, dtype=torch.bfloat16):
    return torch.randn(*s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def f32(*s, seed=1):
    return n(*s, seed=seed, dtype=torch.float32)


def pos():
    return torch.arange(2 * 9, device="cuda").view(2, 9)


def lens():
    return torch.tensor([3, 9], dtype=torch.int32, device="cuda")


CALLS = {
    "rope": lambda s: kb.kata_fwd_norm_rope(n(2, 9, 4, 64).transpose(1, 2), n(2, 3, 9, 64, seed=2), n(64), n(64, seed=3), pos(), **s),
    "rope_plain": lambda s: kb.kata_fwd_norm_rope(f32(2, 3, 9, 32), offset=7, base=500.0, rotary_dim=16, interleaved=True, eps=1e-4, **s)[0],
    "rope_freq": lambda s: kb.kata_fwd_norm_rope(n(2, 3, 9, 64), None, n(64), positions=pos()[0], inv_freq=[0.5] * 16, **s)[0],
    "rope_bwd": lambda s: kb.kata_bwd_norm_rope(n(2, 4, 9, 64, seed=4), n(2, 3, 9, 64, seed=5), n(2, 9, 4, 64).transpose(1, 2), n(2, 3, 9, 64, seed=2), n(64), n(64, seed=3), pos(), **s),
    "rope_bwd_q": lambda s: [x for x in kb.kata_bwd_norm_rope(f32(2, 3, 9, 64), None, f32(2, 3, 9, 64, seed=2), None, f32(64), **s) if x is not None],
    "conv": lambda s: kb.kata_fwd_short_conv(n(2, 9, 72)[..., :64], n(64, 4), n(64, seed=2), silu=True, s_init=n(2, 64, 3), lengths=lens(), **s),
    "conv_bwd": lambda s: kb.kata_bwd_short_conv(n(2, 9, 64, seed=3), n(2, 9, 72)[..., :64], n(64, 4), n(64, seed=2), silu=True, lengths=lens(), **s),
    "conv_step": lambda s: kb.kata_decode_short_conv(f32(2, 64), f32(64, 3), f32(2, 64, 2), silu=True, **s),
    "ssm": lambda s: kb.kata_fwd_ssm_scan(n(2, 2, 900, 64), n(2, 2, 900, 64, seed=2), n(2, 900, 4, 64).transpose(1, 2), n(2, 900, 4).transpose(1, 2), -f32(4).abs(), f32(4),
                                          f32(4, seed=2), dt_softplus=True, s_init=f32(2, 4, 64, 64), s_final=f32(2, 4, 64, 64), **s),
    "ssm_simt": lambda s: kb.kata_fwd_ssm_scan(f32(2, 1, 900, 16), f32(2, 1, 900, 16, seed=2), f32(2, 4, 900, 32), f32(2, 4, 900).abs(), -f32(4).abs(), lengths=lens() * 90, **s),
    "ssm_step": lambda s: kb.kata_decode_ssm_step(n(2, 2, 64), n(2, 2, 64, seed=2), n(2, 4, 64), n(2, 4), -f32(4).abs(), f32(2, 4, 64, 64), f32(4), dt_softplus=True, **s),
    "grad": lambda s: kb.kata_fwd_short_conv(n(2, 9, 64).requires_grad_(), n(64, 4), **s),
}


def stream():
    return {"stream": torch.cuda.current_stream().cuda_stream}


def flat(x):
    return list(x) if isinstance(x, (tuple, list)) else [x]


@pytest.mark.parametrize("name", sorted(CALLS))
def test_same_bits(name, monkeypatch):
    want = flat(CALLS[name](stream()))                # (also leaves the scratch behind that the native call looks up)
    taken, mod = [], kb.native()

    class Watch:
        def __getattr__(self, attr):
            def call(*a):
                taken.append(getattr(mod, attr)(*a))
                return taken[-1]
            return call

    monkeypatch.setattr(kb, "_native", Watch())
    got = flat(CALLS[name]({}))
    assert len(taken) == 1 and taken[0] is not NotImplemented
    assert len(got) == len(want)
    for g, w in zip(got, want):
        assert g.dtype == w.dtype and g.shape == w.shape and g.stride() == w.stride() and not g.requires_grad and torch.equal(g, w)


def bad_calls():
    q, k, x, w = n(2, 4, 9, 64), n(2, 2, 9, 64), n(2, 9, 64), n(64, 4)
    ssm = dict(q=n(2, 2, 9, 64), k=n(2, 2, 9, 64), v=q, dt=n(2, 4, 9), A=-f32(4).abs())
    step = dict(q=n(2, 2, 64), k=n(2, 2, 64), v=n(2, 4, 64), dt=n(2, 4), A=-f32(4).abs(), state=f32(2, 4, 64, 64))
    return [
        lambda s: kb.kata_fwd_norm_rope(q.half(), k.half(), **s),
        lambda s: kb.kata_fwd_norm_rope(q, k.float(), **s),
        lambda s: kb.kata_fwd_norm_rope(q, k, n(32), **s),
        lambda s: kb.kata_fwd_norm_rope(q, k, rotary_dim=24, **s),
        lambda s: kb.kata_fwd_norm_rope(q, k, rotary_dim=80, **s),
        lambda s: kb.kata_fwd_norm_rope(q, k, eps=-1.0, **s),
        lambda s: kb.kata_fwd_norm_rope(q, k, positions=pos().int(), **s),
        lambda s: kb.kata_fwd_norm_rope(q, k, inv_freq=[float("nan")] * 32, **s),
        lambda s: kb.kata_fwd_norm_rope(q[..., ::2], **s),
        lambda s: kb.kata_fwd_norm_rope(n(2, 4, 9, 48), **s),
        lambda s: kb.kata_fwd_norm_rope(q, q_out=k, **s),
        lambda s: kb.kata_bwd_norm_rope(k, None, q, **s),
        lambda s: kb.kata_bwd_norm_rope(q, None, q, k, **s),
        lambda s: kb.kata_fwd_short_conv(x, n(64, 5), **s),
        lambda s: kb.kata_fwd_short_conv(x, w.float(), **s),
        lambda s: kb.kata_fwd_short_conv(x, w, lengths=lens().long(), **s),
        lambda s: kb.kata_fwd_short_conv(x, w, s_init=n(2, 64, 4), **s),
        lambda s: kb.kata_fwd_short_conv(x, w, out=n(2, 9, 32), **s),
        lambda s: kb.kata_bwd_short_conv(n(2, 8, 64), x, w, **s),
        lambda s: kb.kata_decode_short_conv(x, w, n(2, 64, 3), **s),
        lambda s: kb.kata_decode_short_conv(n(2, 64), w, None, **s),
        lambda s: kb.kata_fwd_ssm_scan(**{**ssm, "k": n(2, 2, 9, 32)}, **s),
        lambda s: kb.kata_fwd_ssm_scan(**{**ssm, "dt": n(2, 9, 4)}, **s),
        lambda s: kb.kata_fwd_ssm_scan(**{**ssm, "A": None}, **s),
        lambda s: kb.kata_fwd_ssm_scan(**{**ssm, "q": n(2, 3, 9, 64), "k": n(2, 3, 9, 64)}, **s),
        lambda s: kb.kata_fwd_ssm_scan(**{**ssm, "v": n(2, 4, 9, 128)}, **s),
        lambda s: kb.kata_fwd_ssm_scan(**ssm, impl=7, **s),
        lambda s: kb.kata_fwd_ssm_scan(**ssm, s_init=f32(2, 4, 64, 32), **s),
        lambda s: kb.kata_decode_ssm_step(**{**step, "state": f32(2, 4, 32, 64)}, **s),
        lambda s: kb.kata_decode_ssm_step(**{**step, "state": None}, **s),
        lambda s: kb.kata_decode_ssm_step(**{**step, "dt": n(4, 2)}, **s),
    ]


def test_same_errors():
    for i, call in enumerate(bad_calls()):
        seen = []
        for s in (stream(), {}):
            with pytest.raises(Exception) as e:
                call(s)
            seen.append((type(e.value), str(e.value)))
        assert seen[0] == seen[1], i
