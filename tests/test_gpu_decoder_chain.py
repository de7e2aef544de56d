"""The operators around a decoder's attention as they are used together: a training step of answers to shared prompts, and
tokens generated one by one into a cache.

Tolerances of the chain.  Between the operators queries and keys are rounded once: a score is off by 2 h sum|q k| scale, at most
2 h M with M the largest such sum, and so, relatively, is P.  With the bounds of the single operators (tests/test_gpu_prefix_*.py)
O is off by (h + 5e-4 + 2 * 2 h M) sum P|V| and half a step, the gradients of the rotated rows by
(3 h + 3e-3 + 3 * 2 h M + h) of their magnitudes (P enters dS three times: itself, and through O in D).  The last operator is linear in
those: its own bound, and its formula with absolute values applied to their errors."""
import threading

import pytest
import torch

from tests import decoder_util as du
from tests.test_gpu_prefix_fwd import BF16, F16, ints, make

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def spread(delta, x, w, rd, eps):
    """Magnitude of dx for a gradient of magnitude delta: |dy| of a pair is at most the sum of both."""
    pair = delta.clone()
    both = delta[..., :rd // 2] + delta[..., rd // 2:rd]
    pair[..., :rd // 2], pair[..., rd // 2:rd] = both, both
    r = 1 / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + eps)
    n, t = x.double().abs() * r, pair * w.double().abs()
    return r * (t + n * (t * n).mean(-1, keepdim=True))


@pytest.mark.parametrize("dtype, d, rd", [(F16, 64, 64), (BF16, 128, 128), (F16, 80, 48)])
def test_a_training_step(dtype, d, rd):
    from paper_2502_12784_amd import (spark_mha_prefix_bwd, spark_mha_prefix_fwd, spark_qk_norm_rope_bwd,
                                      spark_qk_norm_rope_fwd)
    G, B, H, Hkv, N, P = 2, 6, 4, 2, 150, 130
    ql = [150, 3, 64, 129, 1, 77]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(B, N, H + 2 * Hkv, d, generator=g, device="cuda").to(dtype).permute(0, 2, 1, 3)  # the projection
    Q, K, V = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
    _, Kp, Vp, _, _ = make(G, 1, 1, Hkv, 1, P, 1, d, dtype, 2)
    dO = torch.randn(B, N, H, d, generator=g, device="cuda").to(dtype).permute(0, 2, 1, 3)
    wq, wk = (1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2))
    cos, sin = du.tables(P + N, rd)
    lens = ints([100, P]), ints(ql), ints(ql)
    start = torch.tensor([100, P], device="cuda").repeat_interleave(B // G)[:, None]
    positions = start + torch.arange(N, device="cuda")
    positions = torch.where(torch.arange(N, device="cuda") < lens[1][:, None], positions, -1).to(torch.int32)
    scale, eps = d ** -0.5, 1e-6
    # the chain
    Qr, Kr = spark_qk_norm_rope_fwd(Q, K, wq, wk, cos, sin, positions)
    O, LSE = spark_mha_prefix_fwd(Qr, Kp, Vp, Kr, V, scale, True, *lens)
    dQr, dKp, dVp, dKr, dV = spark_mha_prefix_bwd(Qr, Kp, Vp, Kr, V, O, LSE, dO, scale, True, *lens)
    dQ, dK, dwq, dwk = spark_qk_norm_rope_bwd(Q, K, wq, wk, cos, sin, dQr, dKr, positions)
    # in 64 bits, from end to end
    q = du.norm_rope(Q, wq, cos, sin, positions, eps, False)
    k = du.norm_rope(K, wk, cos, sin, positions, eps, False)
    mask = du.prefix_mask(G, B, N, P, N, True, *lens)
    want = du.prefix_attention(q, Kp, Vp, k, V, scale, mask, dO)
    h = du.HALF[dtype]
    M = scale * float(max((q.abs() @ t.repeat_interleave(n, 1).abs().mT).max() for t, n in
                          ((k, H // Hkv), (Kp.double()[torch.arange(B, device="cuda") // (B // G)], H // Hkv))))
    du.close(O, want["O"], h * want["O"].abs() + (h + 5e-4 + 4 * h * M) * (1 + h) * want["absO"] + du.TINY[dtype], "O")
    far = (4 * h + 3e-3 + 6 * h * M) * (1 + h)
    for n, got in (("dKp", dKp), ("dVp", dVp), ("dVs", dV)):
        du.close(got, want[n], h * want[n].abs() + far * want["abs_" + n] + du.TINY[dtype], n)
    for n, rows, w, got, dw in (("dQ", Q, wq, dQ, dwq), ("dKs", K, wk, dK, dwk)):
        dx, dw_want = du.norm_rope_grads(rows, w, cos, sin, positions, eps, False, want[n])
        delta = h * want[n].abs() + far * want["abs_" + n]
        delta = torch.where((positions >= 0)[:, None, :, None], delta, torch.zeros_like(delta))
        bound = spread(delta + 80 * U * want[n].abs(), rows, w, rd, eps)
        du.close(got, dx, h * dx.abs() + bound * (1 + h) + du.TINY[dtype], n)
        r = 1 / torch.sqrt((rows.double() ** 2).mean(-1, keepdim=True) + eps)
        pair = delta + 320 * U * want[n].abs()
        both = pair[..., :rd // 2] + pair[..., rd // 2:rd]
        pair = torch.cat((both, both, pair[..., rd:]), -1)
        du.close(dw, dw_want, (pair * rows.double().abs() * r).sum((0, 1, 2)), "dw")
    # padding: zeros all the way
    for b, n in enumerate(ql):
        assert not bool(O[b, :, n:].any()) and not bool(dQ[b, :, n:].any()) and not bool(dK[b, :, n:].any())
        assert not bool(dV[b, :, n:].any())


def test_tokens_one_by_one_and_all_at_once():
    """Eight sequences behind a prompt: every token's key is rotated into the cache, its value copied, and attended to; the same
    rows come from one call over all tokens."""
    from paper_2502_12784_amd import spark_mha_prefix_fwd, spark_qk_norm_rope_fwd
    B, H, Hkv, P, T, S, d = 8, 8, 2, 500, 21, 40, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn(B, T, H + 2 * Hkv, d, generator=g, device="cuda").to(BF16).permute(0, 2, 1, 3)
    _, Kp, Vp, _, _ = make(1, 1, 1, Hkv, 1, P, 1, d, BF16, 4)
    w = 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
    cos, sin = du.tables(P + T, d)
    Kc, Vc = (torch.full((B, Hkv, S, d), float("nan"), dtype=BF16, device="cuda") for _ in range(2))
    outs = []
    for t in range(T):
        new = x[:, :, t:t + 1]
        positions = torch.full((B, 1), P + t, dtype=torch.int32, device="cuda")
        q, _ = spark_qk_norm_rope_fwd(new[:, :H], new[:, H:H + Hkv], w, w, cos, sin, positions, Kr=Kc[:, :, t:t + 1])
        Vc[:, :, t:t + 1] = new[:, H + Hkv:]
        s_lens = torch.full((B,), t + 1, dtype=torch.int32, device="cuda")
        outs.append(spark_mha_prefix_fwd(q, Kp, Vp, Kc, Vc, d ** -0.5, True, s_lens=s_lens))
    positions = (P + torch.arange(T, device="cuda")).expand(B, -1).contiguous().to(torch.int32)
    q, k = spark_qk_norm_rope_fwd(x[:, :H], x[:, H:H + Hkv], w, w, cos, sin, positions)
    assert torch.equal(k, Kc[:, :, :T])
    O, LSE = spark_mha_prefix_fwd(q, Kp, Vp, k, x[:, H + Hkv:], d ** -0.5, True)
    want = du.prefix_attention(q, Kp, Vp, k, x[:, H + Hkv:], d ** -0.5, du.prefix_mask(1, B, T, P, T, True, None, None, None))
    h = du.HALF[BF16]
    for got_o, got_l in ((O, LSE), (torch.cat([o for o, _ in outs], 2), torch.cat([l for _, l in outs], 2))):
        du.close(got_l, want["LSE"], torch.full_like(want["LSE"], 2e-4), "LSE")
        du.close(got_o, want["O"], h * want["O"].abs() + (h + 5e-4) * (1 + h) * want["absO"], "O")


def test_gradients_of_a_broadcast_input_are_whole():
    """A key tensor with a zero stride gets a gradient of its full shape, to be summed by the caller."""
    from paper_2502_12784_amd import spark_mha_prefix_bwd, spark_mha_prefix_fwd
    Q, Kp, Vp, Ks, Vs = make(1, 3, 2, 2, 40, 100, 40, 64, F16, 5)
    dO = make(1, 3, 2, 1, 40, 1, 1, 64, F16, 6)[0]
    wide = (Q, Kp, Vp, Ks[:1].expand(3, -1, -1, -1), Vs[:, :1].expand(-1, 2, -1, -1))
    dense = [t.contiguous() for t in wide]
    out = [spark_mha_prefix_fwd(*x, 0.125) for x in (wide, dense)]
    grads = [spark_mha_prefix_bwd(*x, *o, dO, 0.125) for x, o in zip((wide, dense), out)]
    for a, b in zip((*out[0], *grads[0]), (*out[1], *grads[1])):
        assert a.shape == b.shape and torch.equal(a, b)


def test_two_threads_on_streams_of_their_own():
    from paper_2502_12784_amd import spark_mha_prefix_bwd, spark_mha_prefix_fwd
    xs = [make(1, 8, 4, 2, 5, 700, 60, 128, BF16, 20 + i) for i in range(2)]
    dOs = [make(1, 8, 4, 1, 5, 1, 1, 128, BF16, 30 + i)[0] for i in range(2)]

    def run(x, dO):
        out = spark_mha_prefix_fwd(*x, 0.1)
        return (*out, *spark_mha_prefix_bwd(*x, *out, dO, 0.1))

    want = [run(x, dO) for x, dO in zip(xs, dOs)]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = run(xs[i], dOs[i])
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                    bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_allocated_outputs_have_the_layouts_of_empty_like():
    from paper_2502_12784_amd import spark_mha_prefix_bwd, spark_mha_prefix_fwd, spark_qk_norm_rope_fwd
    x = torch.randn(3, 20, 8, 64, device="cuda").to(F16).permute(0, 2, 1, 3)  # [B, heads, N, d], heads inside
    w = torch.ones(64, device="cuda")
    cos, sin = du.tables(20, 64)
    views = [(x[:, :4], x[:, 4:6], x[:, 6:]), (x[:, :4].contiguous(), x[:, 4:6], x[:1, 6:].expand(3, -1, -1, -1)),
             (x[:, :4, :1], x[:, 4:6, :1], x[:, 6:, :1]), (x[:1, :1], x[:1, 4:5], x[:1, 6:7])]
    for Q, K, V in views:
        q, k = spark_qk_norm_rope_fwd(Q, K, w, w, cos, sin)
        Kp = torch.randn(1, K.shape[1], 30, 64, device="cuda").to(F16)
        O, LSE = spark_mha_prefix_fwd(Q, Kp, Kp, K, V, 0.125)
        grads = spark_mha_prefix_bwd(Q, Kp, Kp, K, V, O, LSE, O, 0.125)
        for got, like in zip((q, k, O, *grads), (Q, K, Q, Q, Kp, Kp, K, V)):
            want = torch.empty_like(like)
            assert got.shape == want.shape and got.stride() == want.stride() and got.dtype == want.dtype
