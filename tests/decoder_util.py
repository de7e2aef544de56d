"""Plain implementations, in 64 bits, of the operators around a decoder's attention, and the tolerances of their tests."""
import math

import torch

# Half a step of the type, relative to a value: what one rounding does at most.
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # half the smallest subnormal


def tables(n, rd, device="cuda", base=10000.0):
    a = torch.outer(torch.arange(n, dtype=torch.float64), base ** (-torch.arange(0, rd, 2, dtype=torch.float64) / rd))
    return a.cos().float().to(device), a.sin().float().to(device)


def rotate(y, cos, sin, interleaved):
    """y [..., N, d] by cos, sin [..., N, rd / 2]."""
    rd = 2 * cos.shape[-1]
    out = y.clone()
    first, second = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, rd // 2), slice(rd // 2, rd))
    a, b = y[..., first], y[..., second]
    out[..., first], out[..., second] = a * cos - b * sin, b * cos + a * sin
    return out


def norm_rope(x, w, cos, sin, positions, eps, interleaved):
    """[B,H,N,d] in 64 bits; a row with a negative position is zero.  Differentiable."""
    x = x.double()
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if w is not None:
        y = y * w.double()
    if positions is None:
        positions = torch.arange(x.shape[2], device=x.device).expand(x.shape[0], -1)
    live = (positions >= 0)[:, None, :, None]
    if cos is not None:
        at = positions.long().clamp(min=0)
        y = rotate(y, cos.double()[at][:, None], sin.double()[at][:, None], interleaved)
    return torch.where(live, y, torch.zeros_like(y))


def norm_rope_grads(x, w, cos, sin, positions, eps, interleaved, dout):
    """(dx, dw) by the formulas of the operator, in 64 bits."""
    x, dout = x.double(), dout.double()
    B, _, N, d = x.shape
    if positions is None:
        positions = torch.arange(N, device=x.device).expand(B, -1)
    live = (positions >= 0)[:, None, :, None]
    dy = dout
    if cos is not None:
        at = positions.long().clamp(min=0)
        dy = rotate(dout, cos.double()[at][:, None], -sin.double()[at][:, None], interleaved)
    dy = torch.where(live, dy, torch.zeros_like(dy))
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n = x * r
    t = dy if w is None else dy * w.double()
    dx = r * (t - n * (t * n).mean(-1, keepdim=True))
    return torch.where(live, dx, torch.zeros_like(dx)), torch.where(live, dy * n, torch.zeros_like(n)).sum((0, 1, 2))


def close(got, want, bound, label):
    """|got - want| <= bound, entry by entry; infinities and NaN in the same places."""
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~same & ~((got - want).abs() <= bound)
    assert not bool(bad.any()), (label, int(bad.sum()), float((got - want).abs()[bad].max()),
                                 [tuple(i) for i in bad.nonzero()[:4].tolist()])
