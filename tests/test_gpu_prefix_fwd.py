"""spark_mha_prefix_fwd against plain attention in 64 bits, at the lengths, masks and layouts where it can go wrong.

Tolerances.  With h half a step of the type (decoder_util.HALF) and u = 2^-24:
* LSE: scores are fp32 sums of d <= 128 products of exactly represented inputs, off by at most 130 u sum|q k| scale; the
  exponentials' argument adds a few u of its size (log2 units up to some 30), v_exp and v_log are good to a few u, the sum
  of up to 20000 positive terms is off by a relative 20000 u / 64 (64 partial chains at least) = 2e-5.  Inputs of unit
  variance and scale 1/sqrt(d) give sum|q k| scale < 15 for d = 128 (mean 7.2): 1.2e-4 + 2e-5.  Asserted: 2e-4.
* O: P is rounded to the type once before the product with V: h sum P|V|.  The exponents' error (as for LSE) is a relative
  error of P of at most 2 * 2e-4, the sum in fp32 2e-5 more: 5e-4 sum P|V|.  The result is rounded once: h |O|."""
import pytest
import torch

from tests import decoder_util as du

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def make(G, B, H, Hkv, Nq, P, S, d, dtype, seed=1, layout="cache"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    if layout == "packed":  # queries and suffix are slices of a projection [B, N, heads, d]: Nq = S
        x = normal(B, Nq, H + 2 * Hkv, d).permute(0, 2, 1, 3)
        Q, Ks, Vs = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
        kv = normal(G, P, 2, Hkv, d).permute(2, 0, 3, 1, 4)
        return Q, kv[0], kv[1], Ks, Vs
    return normal(B, H, Nq, d), normal(G, Hkv, P, d), normal(G, Hkv, P, d), normal(B, Hkv, S, d), normal(B, Hkv, S, d)


def check_fwd(x, scale, causal, pl, ql, sl, got, dtype):
    Q, Kp, Vp, Ks, Vs = x
    G, Hkv, P = Kp.shape[:3]
    B, H, Nq, d = Q.shape
    want = du.prefix_attention(*x, scale, du.prefix_mask(G, B, Nq, P, Ks.shape[2], causal, pl, ql, sl))
    O, LSE = got
    du.close(LSE, want["LSE"], torch.full_like(want["LSE"], 2e-4), "LSE")
    h = du.HALF[dtype]
    du.close(O, want["O"], h * want["O"].abs() + (h + 5e-4) * (1 + h) * want["absO"] + du.TINY[dtype], "O")
    return want


def check(G, B, H, Hkv, Nq, P, S, d, dtype, causal=True, pl=None, ql=None, sl=None, layout="cache", seed=1, spoil=True):
    from paper_2502_12784_amd import spark_mha_prefix_fwd
    x = make(G, B, H, Hkv, Nq, P, S, d, dtype, seed, layout)
    if spoil:  # what stands behind a length is not used
        for t, lens, n in ((x[1], pl, P), (x[2], pl, P), (x[3], sl, S), (x[4], sl, S), (x[0], ql, Nq)):
            for b, m in enumerate(lens or ()):
                t[b, :, max(0, min(m, n)):] = float("nan") if t is not x[4] else float("inf")
    pl, ql, sl = ints(pl), ints(ql), ints(sl)
    scale = d ** -0.5
    for workspace in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):  # what the call asks for; none
        got = spark_mha_prefix_fwd(*x, scale, causal, pl, ql, sl, workspace=workspace)
        torch.cuda.synchronize()
        check_fwd(x, scale, causal, pl, ql, sl, got, dtype)
    return x, got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("d", [8, 40, 64, 72, 96, 104, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("more", [0, 704, 2600])  # few keys are one kernel's, more of them others'
def test_head_sizes(d, causal, dtype, more):
    check(1, 2, 4, 2, 70, 131 + more, 70, d, dtype, causal)


@pytest.mark.parametrize("P, S, Nq", [(1, 1, 1), (64, 1, 1), (63, 5, 1), (65, 64, 1), (200, 16, 1), (0, 7, 1), (0, 130, 130),
                                      (5, 0, 3), (128, 0, 200), (1, 257, 257), (300, 300, 129), (64, 100, 300), (2000, 33, 4),
                                      (640, 513, 500), (127, 127, 127), (64, 64, 64), (1000, 3, 257)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("more", [0, 704, 2600])
def test_lengths(P, S, Nq, causal, more):
    check(1, 3, 2, 2, Nq, P + more, S, 64, F16, causal, seed=2)
    check(1, 3, 2, 1, Nq, P + more, S, 128, BF16, causal, seed=2)


def test_long_suffixes():
    check(2, 4, 3, 3, 1, 30, 1500, 64, F16, seed=2)
    check(2, 4, 6, 2, 7, 0, 1500, 128, BF16, seed=2, sl=[1500, 7, 0, 1111], ql=[7, 7, 3, 5])
    check(1, 2, 3, 1, 600, 64, 700, 72, BF16, seed=2, sl=[700, 333], ql=[600, 400])


def test_many_runs_of_keys():
    check(1, 1, 4, 1, 1, 0, 20000, 128, BF16, seed=16)
    check(1, 2, 4, 2, 3, 9000, 9000, 64, F16, seed=16, sl=[9000, 12], ql=[3, 1])
    check(1, 1, 2, 2, 2, 19000, 5, 40, F16, seed=16, pl=[18111])


@pytest.mark.parametrize("G, B, H, Hkv, Nq", [(1, 1, 1, 1, 1), (1, 64, 8, 2, 1), (3, 12, 8, 2, 5), (2, 2, 12, 4, 33), (5, 5, 6, 1, 1),
                                             (4, 8, 16, 16, 1), (1, 7, 32, 1, 2), (1, 200, 2, 2, 1)])
@pytest.mark.parametrize("more", [0, 704, 2600])
def test_groups_and_shared_heads(G, B, H, Hkv, Nq, more):
    check(G, B, H, Hkv, Nq, 333 + more, 77, 64, BF16, seed=3)
    check(G, B, H, Hkv, Nq, 150 + more, 70, 128, F16, seed=3)


@pytest.mark.parametrize("d, dtype", [(64, F16), (128, BF16), (80, BF16)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("P", [257, 961, 4100])  # a kernel for few keys, and others
def test_ragged_lengths_and_empty_rows(d, dtype, causal, P):
    pl, sl = [0, 130, P], [0, 1, 64, 130, 200, 77]
    check(3, 6, 4, 2, 1, P, 200, d, dtype, causal, pl=pl, sl=sl, seed=4)
    check(3, 6, 4, 2, 200, P, 200, d, dtype, causal, pl=pl, sl=sl, ql=sl, seed=4)
    check(3, 6, 6, 2, 9, P, 200, d, dtype, causal, pl=pl, sl=sl, ql=[9, 3, 0, 1, 9, 8], seed=4)
    # more queries than suffix keys: the first rows see the prefix alone, or nothing
    check(3, 6, 4, 2, 150, P, 200, d, dtype, causal, pl=pl, sl=sl, ql=[150, 70, 150, 1, 0, 149], seed=4)
    check(3, 6, 15, 3, 20, P, 200, d, dtype, causal, pl=pl, sl=sl, ql=[20, 7, 20, 1, 0, 19], seed=4)


@pytest.mark.parametrize("d", [72, 128])
def test_workgroups_of_eight_waves(d):
    """Long sequences with more tiles of 128 rows than CUs, and not as many of 256."""
    check(1, 2, 8, 8, 2100, 100, 2100, d, BF16, seed=14, sl=[2100, 1990], ql=[2100, 1990])
    check(2, 2, 16, 4, 1050, 1100, 1050, d, F16, False, seed=14, pl=[1100, 1025], sl=[1000, 1050], ql=[1050, 1049])


def test_lengths_out_of_range_are_cut():
    check(2, 4, 2, 2, 5, 900, 40, 64, F16, True, pl=[2 ** 31 - 1, -3], ql=[7, -1, 5, 2 ** 31 - 1], sl=[41, 12, -2 ** 31, 1000], seed=5)
    check(2, 4, 2, 2, 5, 100, 40, 64, F16, True, pl=[2 ** 31 - 1, -3], ql=[7, -1, 5, 2 ** 31 - 1], sl=[41, 12, -2 ** 31, 1000], seed=5)


@pytest.mark.parametrize("d", [64, 80, 128])
def test_slices_of_packed_projections(d):
    check(2, 4, 6, 2, 150, 200, 150, d, BF16, layout="packed", seed=6)
    check(2, 4, 6, 2, 1, 70, 1, d, F16, layout="packed", seed=6)


def test_broadcast_keys_and_a_given_output():
    from paper_2502_12784_amd import spark_mha_prefix_fwd
    Q, Kp, Vp, Ks, Vs = make(2, 4, 4, 4, 40, 100, 40, 64, F16, 7)
    x = (Q, Kp[:1].expand(2, -1, -1, -1), Vp[:1].expand(2, -1, -1, -1), Ks[:, :1].expand(-1, 4, -1, -1), Vs[:1].expand(4, -1, -1, -1))
    O = torch.full((4, 40, 4, 64), 3.0, dtype=F16, device="cuda").permute(0, 2, 1, 3)
    LSE = torch.empty(4, 4, 40, device="cuda")
    got = spark_mha_prefix_fwd(*x, 0.125, O=O, LSE=LSE)
    assert got[0] is O and got[1] is LSE
    check_fwd(x, 0.125, True, None, None, None, got, F16)


def test_agrees_with_attention_over_the_keys_laid_out():
    from paper_2502_12784_amd import spark_mha_fwd, spark_mha_prefix_fwd
    Q, Kp, Vp, Ks, Vs = make(1, 3, 4, 4, 333, 0, 333, 128, BF16, 8)
    a, b = spark_mha_prefix_fwd(Q, Kp, Vp, Ks, Vs, 0.1), spark_mha_fwd(Q, Ks.contiguous(), Vs.contiguous(), 0.1, True)
    # the same sums in another order: fp32 differences, and where they meet a border one rounding of the result
    assert float((a[1] - b[1]).abs().max()) <= 1e-5
    assert float((a[0].float() - b[0].float()).abs().max()) <= 2.0 ** -7 * float(b[0].float().abs().max())


def test_peaked_scores():
    """Scores of hundreds: a few keys carry a row, and the running maximum moves."""
    from paper_2502_12784_amd import spark_mha_prefix_fwd
    Q, Kp, Vp, Ks, Vs = make(1, 4, 4, 2, 3, 500, 90, 64, F16, 9)
    Kp[:, :, 400:] *= 8
    Ks[:, :, 80:] *= 16
    x = (Q * 4, Kp, Vp, Ks, Vs)
    O, LSE = spark_mha_prefix_fwd(*x, 0.125)
    want = du.prefix_attention(*x, 0.125, du.prefix_mask(1, 4, 3, 500, 90, True, None, None, None))
    # sum|q k| scale is up to 4 * 16 * 7: the bounds of LSE and of P's relative error 64 times as wide
    du.close(LSE, want["LSE"], torch.full_like(want["LSE"], 64 * 1.2e-4), "LSE")
    h = du.HALF[F16]
    du.close(O, want["O"], h * want["O"].abs() + (h + 128 * 1.2e-4) * want["absO"], "O")


def test_another_stream_and_graphs_with_workspaces_of_their_own():
    from paper_2502_12784_amd import spark_mha_prefix_fwd
    x = make(2, 8, 8, 2, 1, 2000, 100, 128, BF16, 10)
    y = make(2, 8, 8, 2, 1, 2000, 100, 128, BF16, 11)
    want = [spark_mha_prefix_fwd(*t, 0.1) for t in (x, y)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = spark_mha_prefix_fwd(*x, 0.1)
    side.synchronize()
    assert torch.equal(got[0], want[0][0]) and torch.equal(got[1], want[0][1])
    held = []
    for t in (x, y):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = spark_mha_prefix_fwd(*t, 0.1)
        held.append((graph, out))
    for _ in range(3):
        for t in (x, y):
            t[0].mul_(1.0625)
        want = [[v.clone() for v in spark_mha_prefix_fwd(*t, 0.1)] for t in (x, y)]
        torch.cuda.synchronize()
        for graph, out in held:
            out[0].zero_()
            graph.replay()
        torch.cuda.synchronize()
        for (_, out), w in zip(held, want):
            assert torch.equal(out[0], w[0]) and torch.equal(out[1], w[1])
