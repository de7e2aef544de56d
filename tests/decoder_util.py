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


def prefix_mask(G, B, Nq, P, S, causal, prefix_lens, q_lens, s_lens):
    """[B, Nq, P + S]: the keys that a query sees."""
    pl = torch.full((G,), P) if prefix_lens is None else prefix_lens.cpu().long()
    ql = torch.full((B,), Nq) if q_lens is None else q_lens.cpu().long()
    sl = torch.full((B,), S) if s_lens is None else s_lens.cpu().long()
    mask = torch.zeros(B, Nq, P + S, dtype=torch.bool)
    for b in range(B):
        n, p, m = int(ql[b].clamp(0, Nq)), int(pl[b // (B // G)].clamp(0, P)), int(sl[b].clamp(0, S))
        mask[b, :n, :p] = True
        for i in range(n):
            mask[b, i, P:P + (max(0, min(m, i + m - n + 1)) if causal else m)] = True
    return mask


def prefix_attention(Q, Kp, Vp, Ks, Vs, scale, mask, dO=None):
    """Plain attention in 64 bits with every key of every sequence laid out; unseen keys' values are not used at all.
    Returns a dict: O, LSE, P |V| (for the rounding of P), and with dO the gradients and their magnitudes."""
    B, H, Nq, d = Q.shape
    G, Hkv, P = Kp.shape[:3]
    S = Ks.shape[2]
    r, grp = H // Hkv, torch.arange(B, device=Q.device) // (B // G)
    mask = mask.to(Q.device)
    used = mask.any(1)[:, None, :, None]  # a key that no query sees reads as zero

    def keys(p, s):
        x = torch.cat((p.double()[grp], s.double()), 2)
        return torch.where(used, x, torch.zeros_like(x)).repeat_interleave(r, 1)

    K, V, q = keys(Kp, Ks), keys(Vp, Vs), Q.double()
    live = mask.any(-1)[:, None, :, None]
    q = torch.where(live, q, torch.zeros_like(q))
    x = (q @ K.mT * scale).masked_fill(~mask[:, None], -math.inf)
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[..., None])
    out = {"O": p @ V, "LSE": lse, "absO": p @ V.abs()}
    if dO is None:
        return out
    do = torch.where(live, dO.double(), torch.zeros_like(q))
    dp = do @ V.mT
    D = (do * out["O"]).sum(-1, keepdim=True)
    ds = p * (dp - D) * scale

    def back(x):  # [B,H,P+S,d] -> prefix [G,Hkv,P,d], suffix [B,Hkv,S,d]
        x = x.reshape(B, Hkv, r, P + S, d).sum(2)
        return x[:, :, :P].reshape(G, B // G, Hkv, P, d).sum(1), x[:, :, P:]

    out["dQ"] = ds @ K
    out["dKp"], out["dKs"] = back(ds.mT @ q)
    out["dVp"], out["dVs"] = back(p.mT @ do)
    # magnitudes: what one relative error in P, dP, D or dS is multiplied by
    a = p * (do.abs() @ V.abs().mT + (do.abs() * out["absO"]).sum(-1, keepdim=True)) * scale
    out["abs_dQ"] = a @ K.abs()
    out["abs_dKp"], out["abs_dKs"] = back(a.mT @ q.abs())
    out["abs_dVp"], out["abs_dVs"] = back(p.mT @ do.abs())
    return out
