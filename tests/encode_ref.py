"""The prompt encoder's operators in 64 bits on the CPU, and how far a result
computed in fp32 and rounded once may be from them.

U32 and U16 are the unit roundoffs of fp32 and bf16. A sum of n terms in fp32,
in any order, is off by at most n U32 times the sum of the terms' magnitudes
(first order); a rounded result by its type's roundoff times its magnitude.
"""
import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8
UNIT = {torch.float32: U32, torch.bfloat16: U16}
TINY = 1e-37


def close(got, want, slack, what=""):
    """Every element of `got` within `slack` of the 64-bit `want`; NaN and
    infinities in the same places."""
    got, want, slack = got.detach().cpu().double(), want.double(), slack.double() + TINY
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[bad & ~torch.isnan(want)], want[bad & ~torch.isnan(want)]), what
    over = ((got - want).abs() - slack)[~bad]
    if over.numel():
        worst = float(over.max())
        assert worst <= 0, f"{what}: off by {worst:.3g} more than allowed"


def prompt_of(offsets, T):
    """Prompt of every token, -1 for none."""
    bag = torch.full((T,), -1, dtype=torch.long)
    for q in range(len(offsets) - 1):
        bag[offsets[q]:offsets[q + 1]] = q
    return bag


def embed(tokens, table, scale, offsets, mean):
    """(result, sum of the terms' magnitudes, largest number of terms)."""
    t, E = tokens.cpu().long(), table.cpu().double() * scale
    ok = (t >= 0) & (t < E.shape[0])
    if offsets is None:
        out = torch.zeros(len(t), E.shape[1], dtype=torch.float64)
        out[ok] = E[t[ok]]
        return out, out.abs(), 1
    off = offsets.cpu().tolist()
    bag = prompt_of(off, len(t))
    ok &= bag >= 0
    Q = len(off) - 1
    out, mag = torch.zeros(Q, E.shape[1], dtype=torch.float64), torch.zeros(Q, E.shape[1], dtype=torch.float64)
    out.index_add_(0, bag[ok], E[t[ok]])
    mag.index_add_(0, bag[ok], E[t[ok]].abs())
    n = torch.bincount(bag[ok], minlength=Q).double() if Q else torch.zeros(0, dtype=torch.float64)
    most = int(n.max()) if Q else 0
    if mean:
        out, mag = out / n.clamp_min(1)[:, None], mag / n.clamp_min(1)[:, None]
    return out, mag, most


def embed_grad(tokens, grad, V, scale, offsets, mean, add):
    t, g = tokens.cpu().long(), grad.cpu().double() * scale
    ok = (t >= 0) & (t < V)
    src = torch.arange(len(t))
    if offsets is not None:
        off = offsets.cpu().tolist()
        src = prompt_of(off, len(t))
        ok &= src >= 0
        if mean:
            n = torch.bincount(src[ok], minlength=len(off) - 1).double()
            g = g / n.clamp_min(1)[:, None]
    out = add.cpu().double().clone() if add is not None else torch.zeros(V, grad.shape[1], dtype=torch.float64)
    mag = out.abs()
    out.index_add_(0, t[ok], g[src[ok]])
    mag.index_add_(0, t[ok], g[src[ok]].abs())
    most = int(torch.bincount(t[ok], minlength=1).max()) if ok.any() else 0
    return out, mag, most


def rms_norm(x, residual, gain, eps):
    s = x.cpu().double() + (residual.cpu().double() if residual is not None else 0.0)
    return s, s / torch.sqrt((s * s).mean(1, keepdim=True) + eps) * gain.cpu().double()


def rms_norm_grad(grad, total, gain, eps, grad_total):
    """(grad_x, grad_gain, their slacks in units of U32)."""
    s, dy, g = total.cpu().double(), grad.cpu().double(), gain.cpu().double()
    d = s.shape[1]
    w = 1.0 / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    u = dy * g
    dx = w * u - s * w ** 3 * (u * s).mean(1, keepdim=True)
    # w: its d-term sum, halved by the root, cubed at most; sum(u s): d terms.
    slack = (d + 16) * ((w * u).abs() * 0.5 + s.abs() * w ** 3 * (u * s).abs().mean(1, keepdim=True) * 2.5)
    if grad_total is not None:
        dx = dx + grad_total.cpu().double()
        slack = slack + grad_total.cpu().double().abs() + dx.abs()
    dgain = (dy * s * w).sum(0)
    return dx, dgain, slack, (s.shape[0] + 0.5 * d + 16) * (dy * s * w).abs().sum(0)


def quantize(x, block="row", transpose=False):
    """The definition in fp32 (each step one rounding): bytes and scales."""
    x = x.cpu().float()
    x = x.t().contiguous() if transpose else x
    R, C = x.shape
    kb, rb = -(-C // 128), -(-R // 128)
    mag = torch.where(torch.isfinite(x), x.abs(), torch.zeros(()))
    mag = torch.nn.functional.pad(mag, (0, kb * 128 - C)).view(R, kb, 128).amax(2)
    if block == "square":
        mag = torch.nn.functional.pad(mag, (0, 0, 0, rb * 128 - R)).view(rb, 128, kb).amax(1)
    scales = (mag / 448.0).clamp_min(2.0 ** -126)
    inv = 1.0 / scales
    per_row = inv.repeat_interleave(128, 0)[:R] if block == "square" else inv
    y = x * per_row.repeat_interleave(128, 1)[:, :C]
    y = torch.where(torch.isfinite(x), y, torch.full((), float("nan")))
    q = torch.nn.functional.pad(y, (0, -C % 16)).to(torch.float8_e4m3fn)
    return q, scales.t().contiguous()


def dequantize(q, scales, block="row"):
    v = q.cpu().float().double()
    s = scales.cpu().double().t()
    s = s.repeat_interleave(128, 0)[:v.shape[0]] if block == "square" else s
    return v * s.repeat_interleave(128, 1)[:, :v.shape[1]]


def same_e4m3(got, want, what=""):
    """The same values (any NaN is as good as another)."""
    g, w = got.cpu().float(), want.cpu().float()
    assert g.shape == w.shape, (what, g.shape, w.shape)
    assert torch.equal(torch.isnan(g), torch.isnan(w)), what
    assert torch.equal(torch.nan_to_num(g), torch.nan_to_num(w)), what


def matmul(a, a_scales, b, b_scales, b_block, bias, relu):
    """(result, sum of the terms' magnitudes)."""
    x, y = dequantize(a, a_scales), dequantize(b, b_scales, b_block)
    out, mag = x @ y.t(), x.abs() @ y.abs().t()
    if bias is not None:
        out, mag = out + bias.cpu().double(), mag + bias.cpu().double().abs()
    return (torch.where(out < 0, torch.zeros_like(out), out) if relu else out), mag


def fast_slack(a, a_scales, b, b_scales, b_block):
    """How far the 8-bit matrix instructions' sums may be off: of 8 products
    with neighbouring k, all but the largest may lose what is below 2^-13 of it."""
    x, y = dequantize(a, a_scales).abs(), dequantize(b, b_scales, b_block).abs()
    pad = (0, -x.shape[1] % 8)
    x, y = (torch.nn.functional.pad(v, pad).view(v.shape[0], -1, 8) for v in (x, y))
    out = torch.zeros(x.shape[0], y.shape[0], dtype=torch.float64)
    for g in range(x.shape[1]):
        out += (x[:, None, g] * y[None, :, g]).amax(2)
    return 7 * 2.0 ** -13 * out
