"""Host-side checks of the operators around the attention (no GPU): argument structs, status codes before anything is launched,
and what the binding refuses by itself."""
import ctypes
import os
import re

import pytest
import torch

from paper_2607_17419_b200 import binding as kb
from paper_2607_17419_b200 import build as kbuild

INV, SHAPE, ALIGN, WS = -1, -2, -3, -4
P = 4096                                                     # a pointer that is never followed
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    kbuild.build()
    return kb.lib()


def test_structs_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "kata.h")).read(), flags=re.S)
    for name, cls in (("kata_norm_rope_args", kb.NormRopeArgs), ("kata_short_conv_args", kb.ShortConvArgs), ("kata_ssm_args", kb.SsmArgs)):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
        fields = []
        for decl in body.split(";"):
            decl = decl.strip()
            if decl:
                kind, names = re.match(r"((?:const )?\w+)\s*(.*)", decl, flags=re.S).groups()
                for x in names.split(","):
                    fields.append((re.search(r"\w+", x).group(0), "*" in x, int((re.search(r"\[(\d)\]", x) or [0, 0])[1]), kind))
        assert [f[0] for f in fields] == [f[0] for f in cls._fields_]
        sizes = {"uint32_t": 4, "int32_t": 4, "double": 8, "int64_t": 8}
        for (_, pointer, count, kind), (_, ctype) in zip(fields, cls._fields_):
            assert ctypes.sizeof(ctype) == (8 if pointer else sizes[kind] * max(1, count))


def opts(**kw):
    return kb.make_opts(kw.pop("dtype", kb.KATA_BF16), **kw)


def call(L, name, a, o):
    return getattr(L, name)(ctypes.byref(a), ctypes.byref(o))


def rope(**kw):
    a = kb.NormRopeArgs(struct_size=ctypes.sizeof(kb.NormRopeArgs), B=2, T=5, H_q=4, H_k=2, d=64, rotary_dim=64, eps=1e-6, q=P, k=P, q_out=P,
                        k_out=P, q_weight=P, k_weight=P, dq=P, dk=P, dq_weight=P, dk_weight=P)
    a.keep = (ctypes.c_double * 64)()
    a.inv_freq = ctypes.addressof(a.keep)
    for f in ("q", "k", "q_out", "k_out", "dq", "dk"):
        getattr(a, f + "_stride")[:] = (1280, 320, 64)
    for key, x in kw.items():
        if isinstance(x, tuple):
            getattr(a, key)[:] = x
        else:
            setattr(a, key, x)
    return a


@pytest.mark.parametrize("fn", ["kata_fwd_norm_rope", "kata_bwd_norm_rope"])
def test_norm_rope_arguments(L, fn):
    o = lambda **kw: opts(workspace=P, workspace_bytes=1 << 30, **kw)
    assert getattr(L, fn)(None, ctypes.byref(o())) == INV
    assert getattr(L, fn)(ctypes.byref(rope()), None) == INV
    for bad in (dict(struct_size=8), dict(B=0), dict(T=0), dict(H_q=0), dict(H_k=-1), dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(inv_freq=None), dict(rotary_dim=-16),
                dict(q_stride=(-1280, 320, 64)), dict(positions=P, pos_stride=(-1, 1))):
        assert call(L, fn, rope(**bad), o()) == INV, bad
    nan = rope()
    nan.keep[3] = float("nan")
    assert call(L, fn, nan, o()) == INV
    for bad in (dict(d=48), dict(d=256), dict(rotary_dim=8), dict(rotary_dim=80), dict(rotary_dim=128), dict(H_q=32768), dict(B=1 << 20, T=1 << 11)):
        assert call(L, fn, rope(**bad), o()) == SHAPE, bad
    for bad in (dict(q=P + 8), dict(k_out=P + 2), dict(q_stride=(1280, 324, 64)), dict(k_stride=(1280, 320, 65)), dict(q_weight=P + 1), dict(positions=P + 4)):
        assert call(L, fn, rope(**bad), o()) == ALIGN, bad
    assert call(L, fn, rope(), o(impl=kb.KATA_IMPL_TENSOR)) == SHAPE
    assert call(L, fn, rope(), o(s_pre=P, z_pre=P)) == INV and call(L, fn, rope(), opts(dtype=5)) == INV
    if fn == "kata_bwd_norm_rope":
        assert call(L, fn, rope(dq=None), o()) == INV and call(L, fn, rope(dk_stride=(0, 320, 64)), o()) == INV
        assert call(L, fn, rope(q_weight=None), o()) == INV and call(L, fn, rope(dk=P + 8), o()) == ALIGN
        need = kb.kata_workspace_bytes(kb.KATA_FN_BWD_NORM_ROPE, 2, 6, 5, 64, 0, 0, opts())
        assert need > 0 and call(L, fn, rope(), opts()) == WS
        assert call(L, fn, rope(), opts(workspace=P, workspace_bytes=need - 1)) == WS
        assert call(L, fn, rope(), opts(workspace=P + 16, workspace_bytes=1 << 30)) == ALIGN
    else:
        assert call(L, fn, rope(q_out_stride=(1280, 0, 64)), o()) == INV          # an output that is written twice


def conv(**kw):
    a = kb.ShortConvArgs(struct_size=ctypes.sizeof(kb.ShortConvArgs), B=2, T=5, D=64, width=4, silu=1, x=P, weight=P, bias=P, out=P, s_init=P,
                         s_final=P, dout=P, dx=P, dweight=P, dbias=P)
    for f in ("x", "out", "dout", "dx"):
        getattr(a, f + "_stride")[:] = (320, 64)
    for key, x in kw.items():
        if isinstance(x, tuple):
            getattr(a, key)[:] = x
        else:
            setattr(a, key, x)
    return a


@pytest.mark.parametrize("fn", ["kata_fwd_short_conv", "kata_decode_short_conv", "kata_bwd_short_conv"])
def test_short_conv_arguments(L, fn):
    o = lambda **kw: opts(workspace=P, workspace_bytes=1 << 30, **kw)
    bwd = {"s_init": None, "s_final": None} if fn == "kata_bwd_short_conv" else {}
    make = lambda **kw: conv(**{**bwd, **kw})
    assert getattr(L, fn)(None, ctypes.byref(o())) == INV
    for bad in (dict(struct_size=8), dict(B=0), dict(D=0), dict(width=0), dict(x=None), dict(weight=None), dict(x_stride=(-320, 64))):
        assert call(L, fn, make(**bad), o()) == INV, bad
    for bad in (dict(width=1), dict(width=5), dict(D=1 << 25), dict(B=1 << 30, D=1 << 20)):
        assert call(L, fn, make(**bad), o()) == SHAPE, bad
    for bad in (dict(x=P + 1), dict(weight=P + 1), dict(bias=P + 1)):
        assert call(L, fn, make(**bad), o()) == ALIGN, bad
    assert call(L, fn, make(), o(impl=kb.KATA_IMPL_TENSOR)) == SHAPE and call(L, fn, make(), o(s_init=P, z_init=P)) == INV
    if fn == "kata_decode_short_conv":
        assert call(L, fn, make(s_init=None), o()) == INV and call(L, fn, make(s_final=None), o()) == INV and call(L, fn, make(lengths=P), o()) == INV
    else:
        assert call(L, fn, make(T=0), o()) == INV and call(L, fn, make(lengths=P + 2), o()) == ALIGN
    if fn == "kata_bwd_short_conv":
        assert call(L, fn, make(s_init=P), o()) == INV and call(L, fn, make(s_final=P), o()) == INV and call(L, fn, make(bias=None), o()) == INV
        assert call(L, fn, make(dout=None), o()) == INV and call(L, fn, make(dx_stride=(320, 0)), o()) == INV
        need = kb.kata_workspace_bytes(kb.KATA_FN_BWD_SHORT_CONV, 2, 64, 5, 4, 0, 0, opts())
        assert need > 0 and call(L, fn, make(), opts()) == WS and call(L, fn, make(), opts(workspace=P, workspace_bytes=need - 1)) == WS
    else:
        assert call(L, fn, make(out=None), o()) == INV and call(L, fn, make(out_stride=(0, 64)), o()) == INV
        assert call(L, fn, make(s_final=P + 1), o()) == ALIGN


def ssm(**kw):
    a = kb.SsmArgs(struct_size=ctypes.sizeof(kb.SsmArgs), B=2, T=5, H=4, G=2, n=64, d_v=64, q=P, k=P, v=P, dt=P, out=P, A=P, D=P, dt_bias=P, s_init=P,
                   s_final=P)
    for f in ("q", "k", "v", "out"):
        getattr(a, f + "_stride")[:] = (1280, 320, 64)
    a.dt_stride[:] = (20, 5, 1)
    for key, x in kw.items():
        if isinstance(x, tuple):
            getattr(a, key)[:] = x
        else:
            setattr(a, key, x)
    return a


@pytest.mark.parametrize("fn", ["kata_fwd_ssm_scan", "kata_decode_ssm_step"])
def test_ssm_arguments(L, fn):
    o = lambda **kw: opts(workspace=P, workspace_bytes=1 << 30, **kw)
    assert getattr(L, fn)(None, ctypes.byref(o())) == INV
    for bad in (dict(struct_size=8), dict(B=0), dict(H=0), dict(G=0), dict(G=3), dict(n=0), dict(q=None), dict(k=None), dict(v=None), dict(dt=None),
                dict(out=None), dict(A=None), dict(dt_stride=(-20, 5, 1)), dict(out_stride=(0, 320, 64)), dict(out_stride=(1280, 0, 64))):
        assert call(L, fn, ssm(**bad), o()) == INV, bad
    for bad in (dict(n=48), dict(n=256), dict(d_v=128), dict(d_v=8), dict(B=65536, H=2)) + ((dict(T=(1 << 30) + 1),) if fn == "kata_fwd_ssm_scan" else ()):
        assert call(L, fn, ssm(**bad), o()) == SHAPE, bad
    for bad in (dict(q=P + 8), dict(v_stride=(1280, 321, 64)), dict(out=P + 4), dict(dt=P + 1), dict(A=P + 2), dict(s_init=P + 8, s_final=P + 8)):
        assert call(L, fn, ssm(**bad), o()) == ALIGN, bad
    assert call(L, fn, ssm(), o(dtype=kb.KATA_F32, impl=kb.KATA_IMPL_TENSOR)) == SHAPE and call(L, fn, ssm(), o(s_pre=P, z_pre=P)) == INV
    if fn == "kata_decode_ssm_step":
        for bad in (dict(s_init=None), dict(s_final=None), dict(s_final=2 * P), dict(lengths=P)):
            assert call(L, fn, ssm(**bad), o()) == INV, bad
        assert call(L, fn, ssm(), o(impl=kb.KATA_IMPL_TENSOR)) == SHAPE
    else:
        assert call(L, fn, ssm(T=0), o()) == INV and call(L, fn, ssm(lengths=P + 1), o()) == ALIGN
        for bf16 in (kb.KATA_BF16, kb.KATA_F32):
            need = kb.kata_workspace_bytes(kb.KATA_FN_SSM_SCAN, 1, 2, 9000, 64, 64, 0, opts(dtype=bf16))
            long = lambda: ssm(B=1, H=2, T=9000)
            assert need > 0 and call(L, fn, long(), opts(dtype=bf16)) == WS
            assert call(L, fn, long(), opts(dtype=bf16, workspace=P, workspace_bytes=need - 1)) == WS


def test_workspace_of_bad_sizes_is_zero(L):
    ws = kb.kata_workspace_bytes
    assert ws(kb.KATA_FN_SSM_SCAN, 1, 2, 9000, 48, 64, 0, opts()) == 0 and ws(kb.KATA_FN_SSM_SCAN, 0, 2, 9000, 64, 64, 0, opts()) == 0
    up = lambda n: (n + 255) // 256 * 256
    assert ws(kb.KATA_FN_SSM_SCAN, 64, 16, 4096, 64, 32, 0, opts()) == 0           # heads enough: one segment
    assert ws(kb.KATA_FN_SSM_SCAN, 64, 16, 4096, 64, 64, 0, opts()) == up(64 * 16 * 2 * (64 * 64 + 1) * 4)   # (with a final state)
    assert ws(kb.KATA_FN_BWD_SHORT_CONV, 1, 64, 100, 7, 0, 0, opts()) == 0 and ws(kb.KATA_FN_BWD_NORM_ROPE, 1, 4, 100, 48, 0, 0, opts()) == 0
    assert ws(kb.KATA_FN_SSM_SCAN | kb.KATA_FN_HOST_IO, 1, 2, 9000, 64, 64, 0, opts()) == 0


# ---- the binding's own refusals (host tensors end at the latest with "runs on a CUDA device") ----
def z(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def refused_calls():
    q, k, w = z(2, 4, 5, 64), z(2, 2, 5, 64), z(64)
    yield "rope host", lambda: kb.kata_fwd_norm_rope(q, k)
    yield "rope axes", lambda: kb.kata_fwd_norm_rope(q[0], k)
    yield "rope empty", lambda: kb.kata_fwd_norm_rope(q[:, :, :0])
    yield "rope k type", lambda: kb.kata_fwd_norm_rope(q, k.bfloat16())
    yield "rope k rows", lambda: kb.kata_fwd_norm_rope(q, k[..., :32])
    yield "rope inner", lambda: kb.kata_fwd_norm_rope(q.transpose(2, 3).contiguous().transpose(2, 3))
    yield "rope weight", lambda: kb.kata_fwd_norm_rope(q, k, z(32))
    yield "rope weight type", lambda: kb.kata_fwd_norm_rope(q, k, w.bfloat16())
    yield "rope weight of no k", lambda: kb.kata_fwd_norm_rope(q, None, w, w)
    yield "rope positions", lambda: kb.kata_fwd_norm_rope(q, k, positions=z(5, dtype=torch.int32))
    yield "rope positions shape", lambda: kb.kata_fwd_norm_rope(q, k, positions=z(6, dtype=torch.int64))
    yield "rope freq", lambda: kb.kata_fwd_norm_rope(q, k, inv_freq=[1.0] * 3, rotary_dim=64)
    yield "rope out", lambda: kb.kata_fwd_norm_rope(q, k, q_out=z(2, 4, 5, 32))
    yield "rope out of no k", lambda: kb.kata_fwd_norm_rope(q, k_out=q)
    yield "rope bwd grad", lambda: kb.kata_bwd_norm_rope(q[:, :3], k, q, k)
    yield "rope bwd no k", lambda: kb.kata_bwd_norm_rope(q, k, q)
    yield "rope bwd missing", lambda: kb.kata_bwd_norm_rope(q, None, q, k)
    x, cw = z(2, 5, 64), z(64, 4)
    yield "conv host", lambda: kb.kata_fwd_short_conv(x, cw)
    yield "conv axes", lambda: kb.kata_fwd_short_conv(x[0], cw)
    yield "conv weight", lambda: kb.kata_fwd_short_conv(x, z(4, 64))
    yield "conv weight order", lambda: kb.kata_fwd_short_conv(x, z(4, 64).T)
    yield "conv bias", lambda: kb.kata_fwd_short_conv(x, cw, z(63))
    yield "conv state", lambda: kb.kata_fwd_short_conv(x, cw, s_init=z(2, 64, 4))
    yield "conv state type", lambda: kb.kata_fwd_short_conv(x, cw, s_final=z(2, 64, 3, dtype=torch.bfloat16))
    yield "conv lengths", lambda: kb.kata_fwd_short_conv(x, cw, lengths=z(2, dtype=torch.int64))
    yield "conv inner", lambda: kb.kata_fwd_short_conv(x.transpose(1, 2), z(5, 4))
    yield "conv out", lambda: kb.kata_fwd_short_conv(x, cw, out=z(2, 5, 63))
    yield "conv step state", lambda: kb.kata_decode_short_conv(z(2, 64), cw, None)
    yield "conv step axes", lambda: kb.kata_decode_short_conv(x, cw, z(2, 64, 3))
    yield "conv bwd", lambda: kb.kata_bwd_short_conv(x[:, :4], x, cw)
    a = dict(q=z(2, 2, 5, 64), k=z(2, 2, 5, 64), v=z(2, 4, 5, 64), dt=z(2, 4, 5), A=z(4))
    yield "ssm host", lambda: kb.kata_fwd_ssm_scan(**a)
    for name, bad in (("q", z(2, 2, 5, 32)), ("k", z(2, 1, 5, 64)), ("v", z(2, 4, 6, 64)), ("dt", z(2, 5, 4)), ("dt", z(2, 4, 5, dtype=torch.bfloat16)),
                      ("A", z(4, dtype=torch.float64)), ("A", z(2)), ("A", None), ("D", z(5)), ("dt_bias", z(1)), ("s_init", z(2, 4, 64, 32)),
                      ("s_final", z(2, 4, 64, 64, dtype=torch.bfloat16)), ("lengths", z(3, dtype=torch.int32)), ("out", z(2, 4, 5, 32))):
        yield f"ssm {name} {tuple(bad.shape) if bad is not None else None}", lambda name=name, bad=bad: kb.kata_fwd_ssm_scan(**{**a, name: bad})
    s = dict(q=z(2, 2, 64), k=z(2, 2, 64), v=z(2, 4, 64), dt=z(2, 4), A=z(4), state=z(2, 4, 64, 64))
    yield "step host", lambda: kb.kata_decode_ssm_step(**s)
    yield "step state", lambda: kb.kata_decode_ssm_step(**{**s, "state": z(2, 4, 32, 64)})
    yield "step axes", lambda: kb.kata_decode_ssm_step(**{**s, "q": z(2, 2, 1, 64)})


CALLS = dict(refused_calls())


@pytest.mark.parametrize("name", list(CALLS))
def test_refused(name):
    with pytest.raises(ValueError):
        CALLS[name]()


def test_no_unbounded_wait_between_the_warps():
    """The scan's tensor-core kernels meet at barriers with a bounded wait and at __syncthreads behind all roles, nowhere else."""
    text = open(os.path.join(ROOT, "paper_2607_17419_b200", "csrc", "kata_tc_ssm.cu")).read()
    assert not re.search(r"\bbar(rier)?\.(cta\.)?(sync|red)|named_barrier|__nanosleep|while \(", text)
    for role in re.split(r"// =+ ", text)[1:]:
        assert "__syncthreads" not in role.split("// ---------------- teardown")[0]
    # no sum across lanes stands in one side of a choice (a lane that does not take part is waited for without a limit)
    for name in ("kata_norm_rope.cu", "kata_short_conv.cu", "kata_simt_ssm.cu", "kata_ssm_step.cu", "kata_tc_ssm.cu"):
        for line in open(os.path.join(ROOT, "paper_2607_17419_b200", "csrc", name)):
            code = line.split("//")[0]
            assert not re.search(r"\?.*(row_sum|_sync)\s*\(", code), (name, line)


def test_offset_of_more_than_64_bits():
    import torch
    q = torch.zeros(1, 1, 2, 16)
    for offset in (1 << 63, -(1 << 63) - 1):
        with pytest.raises(ValueError, match="offset"):
            kb._rope_args(q, None, None, None, None, offset, (1.0,) * 8, False, 1e-6)
    assert kb._rope_args(q, None, None, None, None, (1 << 63) - 1, (1.0,) * 8, False, 1e-6).pos_offset == (1 << 63) - 1
