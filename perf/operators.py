"""Performance cases of the operators around the attention forms: the selective state space scan, the short causal
convolution before it, and the norm with rotation of queries and keys.

Every case is a plain dict; ``prepare`` makes its inputs on the GPU from the seed, ``run`` is one pass through an operator (its
plain form in elementary torch operations, or, where ``own`` is true, the public entry points of
``paper_2607_17419_b200.binding``), ``work`` the bytes and operations that the result cannot do without and ``exact`` the result
by the definition in 64 bits.

Keys of a case: ``path`` (which operator), ``B, T`` (sequences, tokens of the longest), ``dtype``; of the scan ``H, G`` (heads,
groups of heads that share queries and keys), ``n, d`` (state rows and columns); of the convolution ``D`` (channels), ``W``
(width); of the rotation ``H, Hk`` (query and key heads), ``d``, ``rot`` (rotated entries of a row), ``pairs`` (how they are
paired); ``ragged`` (prompts of unlike lengths in one padded batch), ``state`` (state handed in and out), ``train`` (gradients
too).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _scan(name, B, H, T, n, d, G=1, dtype="bf16", ragged=False, state=False, step=False):
    return {"name": name, "path": "scan_step" if step else "scan", "B": B, "H": H, "T": T, "n": n, "d": d, "G": G, "dtype": dtype,
            "ragged": ragged, "state": state}


def _conv(name, B, T, D, W=4, dtype="bf16", silu=True, bias=True, ragged=False, state=False, train=False, step=False):
    return {"name": name, "path": "conv_step" if step else "conv", "B": B, "T": T, "D": D, "W": W, "dtype": dtype, "silu": silu,
            "bias": bias, "ragged": ragged, "state": state, "train": train}


def _rope(name, B, H, Hk, T, d, rot, pairs="halves", dtype="bf16", train=False, far=0):
    return {"name": name, "path": "rope", "B": B, "H": H, "Hk": Hk, "T": T, "d": d, "rot": rot, "pairs": pairs, "dtype": dtype,
            "train": train, "far": far}


def listed():
    return [
        # one token of one sequence in an interactive session: the latency of a call that moves half a megabyte
        _scan("scan_step_b1", 1, 16, 1, 64, 64, step=True),
        # one token of a large serving batch: the states stream from memory and back
        _scan("scan_step_b128", 128, 16, 1, 128, 64, step=True),
        # the tiny fp32 configuration: a small model in full precision, state handed on
        _scan("scan_tiny_f32", 1, 2, 512, 16, 16, dtype="f32", state=True),
        # prompts of unlike lengths in one padded batch, states handed over for decoding
        _scan("scan_prompt_ragged", 4, 16, 3001, 128, 64, ragged=True, state=True),
        # a layer of a 340M-parameter model at its training shape
        _scan("scan_layer", 8, 16, 4096, 64, 64),
        # long context, one sequence
        _scan("scan_long", 1, 16, 131072, 64, 64),
        # the convolution of one decode step of sixteen sequences
        _conv("conv_step_b16", 16, 1, 1024, step=True, state=True),
        # the convolution of the ragged prompts: values, keys and queries of a layer side by side
        _conv("conv_prompt_ragged", 4, 3001, 1280, ragged=True, state=True),
        # a training step of one layer: forward and gradients
        _conv("conv_train", 8, 4096, 1024, train=True),
        # queries and keys of one decode step of sixteen sequences, each at its own far position
        _rope("rope_step_b16", 16, 16, 16, 1, 64, 64, far=131072),
        # queries and keys of a prompt, views of one packed projection
        _rope("rope_prompt", 2, 16, 16, 3001, 64, 64),
        # a training step of one layer: forward and gradients
        _rope("rope_train", 8, 16, 16, 4096, 64, 64, train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    kind = rng.choice(["scan_step", "scan", "scan", "conv_step", "conv", "conv", "rope", "rope"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "scan_step":
        c = _scan("", _log_int(rng, 1, 128), rng.choice([4, 8, 12, 16]), 1, rng.choice([16, 32, 64, 128]), rng.choice([16, 32, 64]),
                  G=rng.choice([1, 2, 4]), dtype=dtype, step=True)
    elif kind == "scan":
        T = _log_int(rng, 1, 131072)
        wide = rng.random() < 0.75
        G, n, d = rng.choice([1, 1, 2, 4]), rng.choice([64, 128] if wide else [16, 32]), 64 if wide else rng.choice([16, 32])
        most = (1 << 21 if dtype == "bf16" else 1 << 18) // max(1, G * n // 64)      # tokens x heads
        heads = max(G, min(2048, _log_int(rng, 256, most) // T))
        H = rng.choice([h for h in (1, 2, 4, 8, 12, 16) if h <= heads and h % G == 0])
        c = _scan("", max(1, heads // H), H, min(T, most // G), n, d, G=G, dtype=dtype, ragged=rng.random() < 0.4,
                  state=rng.random() < 0.5)
    elif kind == "conv_step":
        c = _conv("", _log_int(rng, 1, 256), 1, rng.choice([128, 1000, 1024, 1152, 2048]), W=rng.choice([2, 3, 4]), dtype=dtype,
                  silu=rng.random() < 0.8, bias=rng.random() < 0.7, state=True, step=True)
    elif kind == "conv":
        T = _log_int(rng, 1, 32768)
        train = rng.random() < 0.5
        c = _conv("", max(1, _log_int(rng, 64, 32768) // T), T, rng.choice([8, 100, 128, 513, 1000, 1024]), W=rng.choice([2, 3, 4]),
                  dtype=dtype, silu=rng.random() < 0.8, bias=rng.random() < 0.7, ragged=rng.random() < 0.4,
                  state=not train and rng.random() < 0.6, train=train)
    else:
        T = _log_int(rng, 1, 32768)
        H, d = rng.choice([1, 4, 8, 12, 16]), rng.choice([16, 32, 64, 64])
        c = _rope("", max(1, _log_int(rng, 16, 32768) // T), H, rng.choice([h for h in (1, 4, 8, 12, 16) if h <= H]), T, d,
                  rng.choice([r for r in (0, 16, 32, 64) if r <= d]), pairs=rng.choice(["halves", "halves", "neighbours"]),
                  dtype=dtype, train=rng.random() < 0.4, far=rng.choice([0, 1000, 1 << 20]))
    del c["name"]
    while work(c)["bytes"] > 5.7e8:                                          # what the long scan moves
        c["B"], c["T"] = ((c["B"] + 1) // 2, c["T"]) if c["B"] > 1 else (1, c["T"] // 2)
    return c


def _lengths(case, gen):
    """Lengths of the sequences of a padded batch: the longest fills it."""
    if not case["ragged"]:
        return None
    n = torch.randint(1, case["T"] + 1, (case["B"],), device="cuda", generator=gen, dtype=torch.int32)
    n[-1] = case["T"]
    return n


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def uniform(lo, hi, *shape):
        return torch.rand(*shape, device="cuda", generator=gen) * (hi - lo) + lo

    B, T = case["B"], case["T"]
    s = {"case": dict(case)}
    if case["path"] in ("scan", "scan_step"):
        H, G, n, d = case["H"], case["G"], case["n"], case["d"]
        # values, keys and queries side by side in the rows that the convolution before them writes
        x = normal(B, T, H * d + 2 * G * n)
        x = (x * torch.sigmoid(x)).to(dt)
        v = x[..., :H * d].view(B, T, H, d).transpose(1, 2)
        k = x[..., H * d:H * d + G * n].view(B, T, G, n).transpose(1, 2)
        q = x[..., H * d + G * n:].view(B, T, G, n).transpose(1, 2)
        step = torch.exp(uniform(math.log(1e-3), math.log(0.1), H))          # step sizes at a raw step of 0
        s.update(A=-uniform(1.0, 16.0, H), D=1 + 0.1 * normal(H), bias=step + torch.log(-torch.expm1(-step)),
                 lengths=_lengths(case, gen))
        dts = (0.5 * normal(B, T, H)).to(dt).transpose(1, 2)
        if case["path"] == "scan_step":
            s.update(q=q[:, :, 0], k=k[:, :, 0], v=v[:, :, 0], dt=dts[:, :, 0], S=normal(B, H, n, d))
        else:
            s.update(q=q, k=k, v=v, dt=dts, S=normal(B, H, n, d) if case["state"] else None)
    elif case["path"] in ("conv", "conv_step"):
        D, W = case["D"], case["W"]
        s.update(w=(normal(D, W) / math.sqrt(W)).to(dt), bias=(0.1 * normal(D)).to(dt) if case["bias"] else None,
                 lengths=_lengths(case, gen), S=normal(B, D, W - 1).to(dt) if case["state"] else None)
        x = normal(B, T, D + 64).to(dt)[..., :D]                             # the front of wider projection rows
        s["x"] = x[:, 0] if case["path"] == "conv_step" else x
        if case["train"]:
            s["dout"] = normal(B, T, D).to(dt)
    else:
        H, Hk, d = case["H"], case["Hk"], case["d"]
        x = normal(B, T, H + Hk, d).to(dt)                                   # one packed projection
        s.update(q=x[:, :, :H].transpose(1, 2), k=x[:, :, H:].transpose(1, 2), qw=(1 + 0.1 * normal(d)).to(dt),
                 kw=(1 + 0.1 * normal(d)).to(dt), inv_freq=[10000.0 ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)])
        s["freqs"] = torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda")
        first = torch.randint(0, case["far"] + 1, (B, 1), device="cuda", generator=gen)
        s["pos"] = first + torch.arange(T, device="cuda")                    # every sequence goes on from its own position
        if case["train"]:
            s["dq"], s["dk"] = normal(B, H, T, d).to(dt), normal(B, Hk, T, d).to(dt)
    return s


def _live(lengths, B, T):
    """[B, T]: whether a token is one of its sequence's."""
    t = torch.arange(T, device="cuda")
    return (t < lengths[:, None]) if lengths is not None else (t < T).expand(B, T)


def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-torch.abs(x)))


CHUNK = 128


def _scan_plain(q, k, v, dt, A, D, bias, S0, lengths):
    """S_t = exp(dt_t A) S_{t-1} + dt_t k_t v_t^T, o_t = q_t^T S_t + D v_t: products inside chunks, states before chunks."""
    B, H, T, d = v.shape
    G, n = k.shape[1], k.shape[3]
    live = _live(lengths, B, T)[:, None]
    steps = torch.where(live, _softplus(dt.float() + bias[:, None]), 0.0)
    pad = -T % CHUNK
    chunks = (T + pad) // CHUNK

    def cut(x, rows):
        x = torch.nn.functional.pad(x, (0, 0, 0, pad)).reshape(B, x.shape[1], chunks, CHUNK, x.shape[-1])
        return x if x.shape[1] == rows else x.repeat_interleave(rows // x.shape[1], 1)

    qf, kf = (torch.where(live[..., None], x.float(), 0.0) for x in (q, k))
    vf = torch.where(live[..., None], v.float(), 0.0)
    qc, kc, vc, sc = cut(qf, G), cut(kf, G), cut(vf, H), cut(steps[..., None], H)[..., 0]
    cum = torch.cumsum(sc.double() * A.double()[:, None, None], -1)          # log decay inside a chunk up to a token
    ends = torch.cumsum(cum[..., -1], -1)                                    # and up to the end of a chunk
    below = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda").tril()
    weights = torch.where(below, torch.exp((cum[..., :, None] - cum[..., None, :]).float()), 0.0) * sc[..., None, :]
    weights = weights * (qc @ kc.transpose(-1, -2)).repeat_interleave(H // G, 1)
    out = weights @ vc
    kh, qh = kc.repeat_interleave(H // G, 1), qc.repeat_interleave(H // G, 1)
    left = torch.exp((cum[..., -1:] - cum).float()) * sc
    local = ((kh * left[..., None]).transpose(-1, -2) @ vc).reshape(B, H, chunks, n * d)
    before = torch.cat([torch.zeros_like(ends[..., :1]), ends], -1)          # [B, H, chunks + 1]
    earlier = torch.arange(chunks + 1, device="cuda")[:, None] > torch.arange(chunks, device="cuda")
    carry = torch.where(earlier, torch.exp((before[..., :, None] - ends[..., None, :]).float()), 0.0)
    states = carry @ local
    if S0 is not None:
        states = states + torch.exp(before.float())[..., None] * S0.reshape(B, H, 1, n * d)
    states = states.reshape(B, H, chunks + 1, n, d)
    out = out + torch.exp(cum.float())[..., None] * (qh @ states[:, :, :-1])
    out = out.reshape(B, H, T + pad, d)[:, :, :T]
    out = out + D[:, None, None] * vf
    return torch.where(live[..., None], out, 0.0).to(v.dtype), states[:, :, -1]


def _scan_step_plain(q, k, v, dt, A, D, bias, S):
    B, H, d = v.shape
    per = H // k.shape[1]
    steps = _softplus(dt.float() + bias)
    kh, qh = k.float().repeat_interleave(per, 1), q.float().repeat_interleave(per, 1)
    new = torch.exp(steps * A)[..., None, None] * S + (steps[..., None] * kh)[..., None] * v.float()[..., None, :]
    S.copy_(new)
    return ((qh[..., None] * new).sum(-2) + D[:, None] * v.float()).to(v.dtype)


def _conv_taps(x, S, W):
    """[B, T, D, W]: the inputs that the taps of a token meet, oldest first."""
    B, T, D = x.shape
    past = S.transpose(1, 2).float() if S is not None else x.new_zeros(B, W - 1, D, dtype=torch.float32)
    return torch.cat([past, x.float()], 1).unfold(1, W, 1)


def _conv_plain(x, w, bias, S, lengths, silu):
    B, T, D = x.shape
    W = w.shape[1]
    live = _live(lengths, B, T)[..., None]
    x = torch.where(live, x, torch.zeros((), device="cuda", dtype=x.dtype))
    pre = (_conv_taps(x, S, W) * w.float()).sum(-1)
    if bias is not None:
        pre = pre + bias.float()
    out = torch.where(live, pre * torch.sigmoid(pre) if silu else pre, 0.0).to(x.dtype)
    if S is not None:                                                        # the last W - 1 inputs of every sequence
        n = lengths.long() if lengths is not None else torch.full((B,), T, device="cuda")
        at = n[:, None] + torch.arange(W - 1, device="cuda")
        line = torch.cat([S.transpose(1, 2), x], 1)
        S.copy_(torch.gather(line, 1, at[..., None].expand(-1, -1, D)).transpose(1, 2))
    return out


def _conv_bwd_plain(dout, x, w, bias, lengths, silu):
    B, T, D = x.shape
    W = w.shape[1]
    live = _live(lengths, B, T)[..., None]
    taps = _conv_taps(torch.where(live, x, torch.zeros((), device="cuda", dtype=x.dtype)), None, W)
    g = torch.where(live, dout.float(), 0.0)
    if silu:
        pre = (taps * w.float()).sum(-1)
        if bias is not None:
            pre = pre + bias.float()
        sig = torch.sigmoid(pre)
        g = g * sig * (1 + pre * (1 - sig))
    ahead = torch.nn.functional.pad(g, (0, 0, 0, W - 1)).unfold(1, W, 1)     # the tokens that an input is a tap of
    dx = torch.where(live, (ahead * w.float().flip(1)).sum(-1), 0.0).to(x.dtype)
    return dx, (taps * g[..., None]).sum((0, 1)), g.sum((0, 1)) if bias is not None else None


EPS = 1e-6


def _angles(pos, freqs):
    a = pos.double()[:, None, :, None] * freqs
    return torch.cos(a).float(), torch.sin(a).float()


def _rotate(x, cos, sin, rot, pairs):
    r = x[..., :rot]
    a, b = (r[..., :rot // 2], r[..., rot // 2:]) if pairs == "halves" else (r[..., 0::2], r[..., 1::2])
    a, b = a * cos - b * sin, a * sin + b * cos
    r = torch.cat([a, b], -1) if pairs == "halves" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([r, x[..., rot:]], -1)


def _rope_plain(x, w, cos, sin, rot, pairs):
    x = x.float()
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    return _rotate(y, cos, sin, rot, pairs)


def _rope_bwd_plain(dout, x, w, cos, sin, rot, pairs):
    g = _rotate(dout.float(), cos, -sin, rot, pairs)
    xf = x.float()
    r = 1 / torch.sqrt((xf * xf).mean(-1, keepdim=True) + EPS)
    unit = xf * r
    gw = g * w.float()
    dx = r * (gw - unit * (gw * unit).mean(-1, keepdim=True))
    return dx.to(x.dtype), (g * unit).sum((0, 1, 2))


def run(state):
    if own:
        return _run_own(state)
    case, path = state["case"], state["case"]["path"]
    if path == "scan":
        a = (state[x] for x in ("q", "k", "v", "dt", "A", "D", "bias", "S", "lengths"))
        out, S = _scan_plain(*a)
        if state["S"] is None:
            return out
        state["S"].copy_(S)
        return out, state["S"]
    if path == "scan_step":
        out = _scan_step_plain(*(state[x] for x in ("q", "k", "v", "dt", "A", "D", "bias", "S")))
        return out, state["S"]
    if path == "conv_step":
        out = _conv_plain(state["x"][:, None], state["w"], state["bias"], state["S"], None, case["silu"])
        return out[:, 0], state["S"]
    if path == "conv":
        out = _conv_plain(*(state[x] for x in ("x", "w", "bias", "S", "lengths")), case["silu"])
        if case["train"]:
            return (out, *_conv_bwd_plain(state["dout"], state["x"], state["w"], state["bias"], state["lengths"], case["silu"]))
        return out, state["S"]
    cos, sin = _angles(state["pos"], state["freqs"])
    rot, pairs, dt = case["rot"], case["pairs"], state["q"].dtype
    q = _rope_plain(state["q"], state["qw"], cos, sin, rot, pairs).to(dt)
    k = _rope_plain(state["k"], state["kw"], cos, sin, rot, pairs).to(dt)
    if not case["train"]:
        return q, k
    dq, dqw = _rope_bwd_plain(state["dq"], state["q"], state["qw"], cos, sin, rot, pairs)
    dk, dkw = _rope_bwd_plain(state["dk"], state["k"], state["kw"], cos, sin, rot, pairs)
    return q, k, dq, dk, dqw, dkw


def _run_own(state):
    from paper_2607_17419_b200 import binding as kb

    case, path = state["case"], state["case"]["path"]
    if path == "scan":
        out = kb.kata_fwd_ssm_scan(state["q"], state["k"], state["v"], state["dt"], state["A"], state["D"], state["bias"],
                                   dt_softplus=True, s_init=state["S"], s_final=state["S"], lengths=state["lengths"])
        return out if state["S"] is None else (out, state["S"])
    if path == "scan_step":
        out = kb.kata_decode_ssm_step(state["q"], state["k"], state["v"], state["dt"], state["A"], state["S"], state["D"],
                                      state["bias"], dt_softplus=True)
        return out, state["S"]
    if path == "conv_step":
        out = kb.kata_decode_short_conv(state["x"], state["w"], state["S"], state["bias"], silu=case["silu"])
        return out, state["S"]
    if path == "conv":
        out = kb.kata_fwd_short_conv(state["x"], state["w"], state["bias"], silu=case["silu"], s_init=state["S"],
                                     s_final=state["S"], lengths=state["lengths"])
        if case["train"]:
            return (out, *kb.kata_bwd_short_conv(state["dout"], state["x"], state["w"], state["bias"], silu=case["silu"],
                                                 lengths=state["lengths"]))
        return out, state["S"]
    kw = {"inv_freq": state["inv_freq"], "interleaved": case["pairs"] != "halves", "eps": EPS}
    a = (state["q"], state["k"], state["qw"], state["kw"], state["pos"])
    q, k = kb.kata_fwd_norm_rope(*a, **kw)
    if not case["train"]:
        return q, k
    return (q, k, *kb.kata_bwd_norm_rope(state["dq"], state["dk"], *a, **kw))


def work(case):
    """Inputs read once, outputs written once; the operations of the recurrence, of the taps, of the norm and rotation."""
    B, T, e = case["B"], case["T"], 4 if case["dtype"] == "f32" else 2
    if case["path"].startswith("scan"):
        H, G, n, d = case["H"], case["G"], case["n"], case["d"]
        io = B * T * (2 * H * d + 2 * G * n + H) * e
        states = 2 * B * H * n * d * 4 if case["state"] or case["path"] == "scan_step" else 0
        return {"bytes": io + states, "flops": B * T * H * n * d * 5}
    if case["path"].startswith("conv"):
        D, W = case["D"], case["W"]
        io = B * T * D * e * (5 if case["train"] else 2)                     # x, out; x, dout, dx
        states = 2 * B * D * (W - 1) * e if case["state"] else 0
        return {"bytes": io + states, "flops": B * T * D * (2 * W + 4) * (3 if case["train"] else 1)}
    rows = B * T * (case["H"] + case["Hk"])
    return {"bytes": rows * case["d"] * e * (5 if case["train"] else 2) + B * T * 8, "flops": rows * case["d"] * 8 * (3 if case["train"] else 1)}


def _scan_exact(s):
    """The recurrence, one token after the other."""
    q, k, v = (s[x].double() for x in ("q", "k", "v"))
    if s["case"]["path"] == "scan_step":
        q, k, v, dt = q[:, :, None], k[:, :, None], v[:, :, None], s["dt"].double()[..., None]
    else:
        dt = s["dt"].double()
    B, H, T, d = v.shape
    n, per = k.shape[-1], H // k.shape[1]
    raw = dt + s["bias"].double()[:, None]
    steps = torch.logaddexp(raw, torch.zeros_like(raw))
    stop = s["lengths"].tolist() if s["lengths"] is not None else [T] * B
    for b in range(B):
        steps[b, :, stop[b]:] = 0
    kept = torch.exp(steps * s["A"].double()[:, None])[..., None, None].transpose(0, 2).contiguous()        # [T, H, B, 1, 1]
    add = (steps[..., None] * k.repeat_interleave(per, 1)).permute(2, 1, 0, 3)[..., None].contiguous()      # [T, H, B, n, 1]
    vt = v.permute(2, 1, 0, 3)[..., None, :].contiguous()                                                   # [T, H, B, 1, d]
    qt = q.repeat_interleave(per, 1).permute(2, 1, 0, 3)[..., None, :].contiguous()                         # [T, H, B, 1, n]
    S = s["S"].double().transpose(0, 1).contiguous() if s["S"] is not None else v.new_zeros(H, B, n, d)
    out = v.new_empty(T, H, B, 1, d)
    for o, a, x, y, z in zip(out.unbind(0), kept.unbind(0), add.unbind(0), vt.unbind(0), qt.unbind(0)):
        S.mul_(a).addcmul_(x, y)
        torch.matmul(z, S, out=o)
    o = out[:, :, :, 0].permute(2, 1, 0, 3) + s["D"].double()[:, None, None] * v
    for b in range(B):
        o[b, :, stop[b]:] = 0
    return o, S.transpose(0, 1)


def _conv_exact(s, case):
    """Tap by tap; gradients by differentiation."""
    step = case["path"] == "conv_step"
    x = (s["x"][:, None] if step else s["x"]).double()
    B, T, D = x.shape
    W = case["W"]
    stop = s["lengths"].tolist() if s["lengths"] is not None else [T] * B
    alive = torch.zeros(B, T, 1, dtype=torch.bool, device="cuda")
    for b in range(B):
        alive[b, :stop[b]] = True
    with torch.enable_grad():
        x = x.masked_fill(~alive, 0).requires_grad_(case["train"])
        w = s["w"].double().requires_grad_(case["train"])
        bias = s["bias"].double().requires_grad_(case["train"]) if s["bias"] is not None else None
        past = s["S"].double().transpose(1, 2) if s["S"] is not None else x.new_zeros(B, W - 1, D)
        line = torch.cat([past, x], 1)
        y = sum(line[:, j:j + T] * w[:, j] for j in range(W))
        y = y + bias if bias is not None else y
        y = (y / (1 + torch.exp(-y)) if case["silu"] else y).masked_fill(~alive, 0)
        if case["train"]:
            wrt = [x, w] + ([bias] if bias is not None else [])
            g = torch.autograd.grad(y, wrt, s["dout"].double())
    if case["train"]:
        return y.detach(), g[0].masked_fill(~alive, 0), g[1], g[2] if bias is not None else None
    S = None
    if s["S"] is not None:
        S = torch.stack([line[b, stop[b]:stop[b] + W - 1].T for b in range(B)])
    return (y[:, 0] if step else y), S


def _rope_exact(s, case):
    """The pairs as complex numbers turned by their angles; gradients by differentiation."""
    rot, halves = case["rot"], case["pairs"] == "halves"
    angle = s["pos"].double()[:, None, :, None] * torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones_like(angle), angle)
    outs, grads = [], []
    for x, w, g in ((s["q"], s["qw"], s.get("dq")), (s["k"], s["kw"], s.get("dk"))):
        with torch.enable_grad():
            x, w = x.double().requires_grad_(case["train"]), w.double().requires_grad_(case["train"])
            y = w * x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
            if rot:
                r = y[..., :rot]
                z = torch.complex(r[..., :rot // 2], r[..., rot // 2:]) if halves else torch.complex(r[..., ::2], r[..., 1::2])
                z = z * turn
                r = torch.cat([z.real, z.imag], -1) if halves else torch.view_as_real(z).flatten(-2)
                y = torch.cat([r, y[..., rot:]], -1)
            if case["train"]:
                grads.append(torch.autograd.grad(y, [x, w], g.double()))
            outs.append(y.detach())
    if not case["train"]:
        return tuple(outs)
    return (*outs, grads[0][0], grads[1][0], grads[0][1], grads[1][1])


def exact(case, seed):
    s = prepare(case, seed)
    if case["path"].startswith("scan"):
        out, S = _scan_exact(s)
        return out if s["S"] is None else (out, S)
    return _conv_exact(s, case) if case["path"].startswith("conv") else _rope_exact(s, case)
