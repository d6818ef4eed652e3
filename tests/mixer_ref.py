"""Plain definitions in 64 bits of the operators around the attention, with the sums of absolute terms that the error bounds of
the tests are stated in.  Tensors are torch tensors on any device; everything is computed in float64."""
import torch

ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}        # half a step, relative
F32 = 2.0 ** -24


def live_mask(lengths, B, T, device):
    t = torch.arange(T, device=device)
    if lengths is None:
        return torch.ones(B, T, dtype=torch.bool, device=device)
    return t[None] < lengths.to(device).long().clamp(0, T)[:, None]


def within(got, ref, bound, what=""):
    got, ref = got.double(), ref.double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - ref).abs() - bound
    worst = int(over.argmax())
    assert over.max() <= 0, f"{what}: off by {float((got - ref).abs().reshape(-1)[worst]):.3e} at {worst}, allowed {float((bound + torch.zeros_like(ref)).reshape(-1)[worst]):.3e}"


# ---- convolution ----
def conv(x, w, bias=None, silu=False, past=None, lengths=None):
    """(out, state, sum of absolute terms before the activation)"""
    B, T, D = x.shape
    W = w.shape[1]
    live = live_mask(lengths, B, T, x.device)
    x64 = x.double().masked_fill(~live[..., None], 0)
    line = torch.cat([past.double().transpose(1, 2) if past is not None else x64.new_zeros(B, W - 1, D), x64], 1)
    z = sum(line[:, j:j + T] * w.double()[:, j] for j in range(W))
    mag = sum((line[:, j:j + T] * w.double()[:, j]).abs() for j in range(W))
    if bias is not None:
        z, mag = z + bias.double(), mag + bias.double().abs()
    y = z * torch.sigmoid(z) if silu else z
    n = live.sum(1)
    state = torch.stack([line[b, n[b]:n[b] + W - 1].T for b in range(B)])
    return y.masked_fill(~live[..., None], 0), state, mag


def conv_bound(y, mag, W, dtype, silu):
    # z: W + 1 roundings of partial sums below mag; z sigmoid(z) has a slope below 1.1; the sigmoid is within 2^-20 of itself
    return 1.1 * (W + 1) * F32 * mag + (ROUND[dtype] * 1.01 + (2.0 ** -20 if silu else 0)) * y.abs() + 1e-38


# ---- norm and rotation ----
def turn(x, pos, inv_freq, interleaved):
    """x [B,H,T,d], pos [B,T] (or broadcastable); also the sizes of the pairs that entries come from."""
    r = 2 * len(inv_freq)
    if r == 0:
        return x, x.abs()
    ang = pos.double()[:, None, :, None] * torch.tensor(list(inv_freq), dtype=torch.float64, device=x.device)
    c, s = torch.cos(ang), torch.sin(ang)
    head = x[..., :r]
    a, b = (head[..., 0::2], head[..., 1::2]) if interleaved else (head[..., :r // 2], head[..., r // 2:])
    ya, yb, size = a * c - b * s, a * s + b * c, a.abs() + b.abs()
    join = (lambda p, q: torch.stack([p, q], -1).flatten(-2)) if interleaved else (lambda p, q: torch.cat([p, q], -1))
    return torch.cat([join(ya, yb), x[..., r:]], -1), torch.cat([join(size, size), x[..., r:].abs()], -1)


def norm_rope(x, w, pos, inv_freq, interleaved=False, eps=1e-6):
    x64 = x.double()
    y = x64 / torch.sqrt(x64.square().mean(-1, keepdim=True) + eps)
    if w is not None:
        y = y * w.double()
    return turn(y, pos, inv_freq, interleaved)


# ---- scan ----
def ssm(q, k, v, dt, A, D=None, bias=None, softplus=False, init=None, lengths=None):
    """(out, final state, magnitudes of both: the same recurrence over absolute values)"""
    B, H, T, d = v.shape
    per, n = H // k.shape[1], k.shape[3]
    live = live_mask(lengths, B, T, v.device)[:, None]
    s = dt.double() + (bias.double()[:, None] if bias is not None else 0)
    s = torch.logaddexp(s, torch.zeros_like(s)) if softplus else s
    s = s.masked_fill(~live, 0)
    k64, q64 = (x.double().masked_fill(~live[..., None], 0).repeat_interleave(per, 1) for x in (k, q))
    v64 = v.double().masked_fill(~live[..., None], 0)
    a = torch.exp(s * A.double()[:, None])
    S = init.double().clone() if init is not None else v64.new_zeros(B, H, n, d)
    M, out, mag = S.abs(), torch.empty_like(v64), torch.empty_like(v64)
    skip = D.double()[:, None, None] if D is not None else torch.zeros((), dtype=torch.float64, device=v.device)
    for t in range(T):
        add = (s[:, :, t, None] * k64[:, :, t])[..., None] * v64[:, :, t, None, :]
        S = a[:, :, t, None, None] * S + add
        M = a[:, :, t, None, None] * M + add.abs()
        out[:, :, t] = (q64[:, :, t, :, None] * S).sum(2)
        mag[:, :, t] = (q64[:, :, t, :, None].abs() * M).sum(2)
    out, mag = out + skip * v64, mag + (skip * v64).abs()
    return out.masked_fill(~live[..., None], 0), S, mag, M
