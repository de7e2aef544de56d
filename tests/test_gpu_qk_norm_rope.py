"""spark_qk_norm_rope_fwd / _bwd against their formulas in 64 bits.

Tolerances.  Everything between the inputs and the one rounding of a result is fp32, u = 2^-24: the sum of d <= 128
squares (a chain of 16 products and sums in a lane, 4 more additions across lanes), mean, 1/sqrt, two products for n w and
the two products and the sum of the rotation.  That is at most 30 roundings of relative size u on the way to a term
|y c| + |z s|, so a result is off by half a step of its type and 40 u of |y c| + |z s|.  The backward adds a second sum
of d products (20 roundings) and three products: 80 u of r (|t| + |n| mean|t n|).  dw is a sum over R rows of products
with at most 20 roundings each, added in fp32 in chains: of a lane's tokens and heads, then over lanes, waves and
workgroups; the longest chain here is below 300 additions, so 320 u of the sum of magnitudes."""
import pytest
import torch

from tests import decoder_util as du

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F16, BF16 = torch.float16, torch.bfloat16


def make(B, H, Hkv, N, d, dtype, layout, seed, sigma=1.0):
    """Two pairs (Q, K): inputs and gradients."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = []
    for _ in range(2):
        if layout == "packed":
            x = (torch.randn(B, N, H + 2 * Hkv, d, generator=g, device="cuda") * sigma).to(dtype)
            out += [x[:, :, :H].permute(0, 2, 1, 3), x[:, :, H:H + Hkv].permute(0, 2, 1, 3)]
        else:
            out += [(torch.randn(B, n, N, d, generator=g, device="cuda") * sigma).to(dtype) for n in (H, Hkv)]
    w = [1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2)]
    return out, w


def fwd_bound(x, w, cos, sin, positions, eps, interleaved, want, dtype):
    """Half a step of the result and 40 u of |y c| + |z s|."""
    mag = du.norm_rope(x.double().abs(), None if w is None else w.abs(), None if cos is None else cos.abs(),
                       None if sin is None else -sin.abs(), positions, eps, interleaved)
    # with both signs positive only one of a pair's two results is the sum of magnitudes: take the other's with +
    mag2 = du.norm_rope(x.double().abs(), None if w is None else w.abs(), None if cos is None else cos.abs(),
                        None if sin is None else sin.abs(), positions, eps, interleaved)
    return want.abs() * du.HALF[dtype] + 40 * U * torch.maximum(mag.abs(), mag2.abs()) * (1 + du.HALF[dtype]) + du.TINY[dtype]


def check(B, H, Hkv, N, d, rd, dtype, interleaved=False, layout="packed", positions=None, weights="fp32", eps=1e-6, seed=1,
          table=None, sigma=1.0):
    from paper_2502_12784_amd import spark_qk_norm_rope_bwd, spark_qk_norm_rope_fwd
    (Q, K, dQr, dKr), (wq, wk) = make(B, H, Hkv, N, d, dtype, layout, seed, sigma)
    if weights == "none":
        wq = wk = None
    elif weights == "same":
        wq, wk = wq.to(dtype), wk.to(dtype)
    cos, sin = du.tables(table or N, rd) if rd else (None, None)
    before = Q.clone(), K.clone()
    out = spark_qk_norm_rope_fwd(Q, K, wq, wk, cos, sin, positions, eps, interleaved)
    grads = spark_qk_norm_rope_bwd(Q, K, wq, wk, cos, sin, dQr, dKr, positions, eps, interleaved)
    torch.cuda.synchronize()
    assert torch.equal(Q, before[0]) and torch.equal(K, before[1])
    for x, w, got, dout, dx, dw, name in ((Q, wq, out[0], dQr, grads[0], grads[2], "q"),
                                          (K, wk, out[1], dKr, grads[1], grads[3], "k")):
        args = (cos, sin, positions, eps, interleaved)
        want = du.norm_rope(x, w, *args)
        du.close(got, want, fwd_bound(x, w, *args, want, dtype), name)
        want_dx, want_dw = du.norm_rope_grads(x, w, *args, dout)
        r = 1 / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + eps)
        n = x.double().abs() * r
        # |dy| <= |a c| + |b s| <= sqrt(2) of the pair's length, at most |a| + |b|
        pair = dout.double().abs()
        if rd:
            first, second = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, rd // 2), slice(rd // 2, rd))
            both = pair[..., first] + pair[..., second]
            pair = pair.clone()
            pair[..., first], pair[..., second] = both, both
        t = pair * (1 if w is None else w.double().abs())
        mag = r * (t + n * (t * n).mean(-1, keepdim=True))
        du.close(dx, want_dx, want_dx.abs() * du.HALF[dtype] + 80 * U * mag * (1 + du.HALF[dtype]) + du.TINY[dtype], "d" + name)
        du.close(dw, want_dw, 320 * U * (pair * n).sum((0, 1, 2)), "dw" + name)
        assert dw.dtype == torch.float32


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("d, rd", [(128, 128), (64, 64), (96, 96), (80, 48), (72, 72), (8, 8), (24, 16), (120, 8), (128, 0),
                                   (48, 40), (112, 112), (56, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_sizes_of_heads_and_rotation(d, rd, interleaved, dtype):
    check(2, 3, 2, 37, d, rd, dtype, interleaved)


@pytest.mark.parametrize("B, H, Hkv, N", [(1, 1, 1, 1), (7, 5, 1, 1), (1, 33, 17, 3), (3, 4, 4, 1333), (64, 16, 8, 1),
                                          (2, 1, 3, 500), (1, 2, 2, 33000)])
@pytest.mark.parametrize("layout", ["packed", "bhnd"])
def test_numbers_of_heads_and_tokens(B, H, Hkv, N, layout):
    check(B, H, Hkv, N, 64, 64, BF16, layout=layout, seed=3)


@pytest.mark.parametrize("weights", ["fp32", "same", "none"])
def test_weights(weights):
    check(2, 4, 2, 65, 128, 64, BF16, weights=weights, seed=4)
    check(2, 4, 2, 65, 72, 72, F16, weights=weights, seed=4)


def test_positions_in_any_order_far_ones_and_padding():
    g = torch.Generator().manual_seed(5)
    positions = torch.randint(0, 40000, (3, 50), generator=g).to(torch.int32)
    positions[0, 7:] = -1          # padding behind a sequence
    positions[1, :20] = -5         # and in front of one
    positions[2, 4] = positions[2, 5]
    for interleaved in (False, True):
        check(3, 4, 2, 50, 128, 128, BF16, interleaved, positions=positions.cuda(), table=40000, seed=6)
    check(3, 4, 2, 50, 64, 0, F16, positions=positions.cuda(), seed=6)  # padding without a rotation


@pytest.mark.parametrize("sigma, eps", [(1e-4, 1e-6), (0.0, 1e-6), (200.0, 1e-5), (1.0, 0.5)])
def test_small_zero_and_large_rows(sigma, eps):
    check(1, 2, 2, 40, 128, 128, F16, eps=eps, sigma=sigma, seed=7)
    check(1, 2, 2, 40, 64, 64, BF16, eps=eps, sigma=sigma, seed=7)


def test_a_position_behind_the_table_gives_nan_and_reads_nothing():
    from paper_2502_12784_amd import spark_qk_norm_rope_fwd
    (Q, K, _, _), (wq, wk) = make(1, 2, 1, 4, 64, BF16, "bhnd", 8)
    cos, sin = du.tables(16, 32)
    positions = torch.tensor([[3, 16, 2 ** 31 - 1, 15]], dtype=torch.int32, device="cuda")
    q, _ = spark_qk_norm_rope_fwd(Q, K, wq, wk, cos, sin, positions)
    nan = torch.isnan(q)
    assert bool(nan[:, :, 1:3, :32].all()) and int(nan.sum()) == 2 * 2 * 32
    assert torch.isfinite(q[:, :, [0, 3]]).all() and torch.isfinite(q[..., 32:]).all()


def test_in_place_into_a_cache_and_given_gradients():
    from paper_2502_12784_amd import spark_qk_norm_rope_bwd, spark_qk_norm_rope_fwd
    (Q, K, dQr, dKr), (wq, wk) = make(2, 4, 2, 5, 128, BF16, "packed", 9)
    cos, sin = du.tables(64, 128)
    want = spark_qk_norm_rope_fwd(Q, K, wq, wk, cos, sin)
    cache = torch.full((2, 2, 40, 128), 7.0, dtype=BF16, device="cuda")
    Q2 = Q.clone()
    got = spark_qk_norm_rope_fwd(Q2, K, wq, wk, cos, sin, Qr=Q2, Kr=cache[:, :, 11:16])
    assert torch.equal(got[0], want[0]) and torch.equal(cache[:, :, 11:16], want[1])
    assert bool((cache[:, :, :11] == 7).all()) and bool((cache[:, :, 16:] == 7).all())
    grads = spark_qk_norm_rope_bwd(Q, K, wq, wk, cos, sin, dQr, dKr)
    again = spark_qk_norm_rope_bwd(Q, K, wq, wk, cos, sin, dQr, dKr, dQ=dQr, dK=dKr)
    for a, b in zip(grads, again):
        assert torch.equal(a, b)  # in place, and the same bits in every run


def test_one_token_of_a_long_cache():
    """The row stride of a tensor with one row does not matter; a cache of more than 4 GiB is written behind that."""
    from paper_2502_12784_amd import spark_qk_norm_rope_fwd
    (Q, K, _, _), (wq, wk) = make(3, 2, 2, 1, 128, BF16, "bhnd", 10)
    cos, sin = du.tables(8, 128)
    want = spark_qk_norm_rope_fwd(Q, K, wq, wk, cos, sin)
    cache = torch.zeros(3, 2, 3_000_000, 128, dtype=BF16, device="cuda")  # 4.6 GB, a head 768 MB
    spark_qk_norm_rope_fwd(Q, K, wq, wk, cos, sin, Kr=cache[:, :, 2_999_999:])
    assert torch.equal(cache[:, :, 2_999_999:], want[1]) and not bool(cache[:, :, 2_999_998].any())


def test_gradients_against_differences():
    """The gradient of sum(c out) in 64 bits, by central differences of the plain forward at a few entries."""
    (Q, K, dQr, _), (wq, _) = make(1, 2, 1, 6, 32, F16, "bhnd", 11)
    cos, sin = du.tables(6, 24)
    dx, dw = du.norm_rope_grads(Q, wq, cos, sin, None, 1e-6, False, dQr)
    f = lambda x, w: float((du.norm_rope(x, w, cos, sin, None, 1e-6, False) * dQr.double()).sum())  # noqa: E731
    x, w, h = Q.double(), wq.double(), 1e-5
    for at in ((0, 0, 0, 0), (0, 1, 5, 31), (0, 0, 3, 13), (0, 1, 2, 23)):
        e = torch.zeros_like(x)
        e[at] = h
        assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - float(dx[at])) <= 1e-6
    for i in (0, 12, 30):
        e = torch.zeros_like(w)
        e[i] = h
        assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - float(dw[i])) <= 1e-6


def test_on_another_stream_and_in_a_graph():
    from paper_2502_12784_amd import spark_qk_norm_rope_bwd, spark_qk_norm_rope_fwd
    (Q, K, dQr, dKr), (wq, wk) = make(2, 4, 2, 300, 128, BF16, "packed", 12)
    cos, sin = du.tables(300, 128)

    def step():
        return (*spark_qk_norm_rope_fwd(Q, K, wq, wk, cos, sin), *spark_qk_norm_rope_bwd(Q, K, wq, wk, cos, sin, dQr, dKr))

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(3):
        Q.add_(0.25)
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, held):
            assert torch.equal(a, b)
