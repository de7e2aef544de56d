"""spark_mha_prefix_bwd against the formulas in 64 bits, at the lengths, masks and layouts where it can go wrong.

Tolerances.  With h half a step of the type: dS = P o (dP - D) is rounded to the type before its products (h |dS|), and so
is P before the product with dO (h P).  D is formed from the forward's rounded O, which is off by h |O| and (h + 5e-4)
sum P|V| (tests/test_gpu_prefix_fwd.py); with |O| <= sum P|V| that is (2 h + 5e-4) |dO| . sum P|V|.  P itself is formed in
fp32 from scores and LSE, a relative 2e-4 each and another 2e-4 for its exponential; dP and the accumulations are fp32 sums
of up to 20000 terms in chains, a relative 1e-3 at most.  With a = P (|dO| . |V|^T + |dO| . sum P|V|) scale, all of it is at most
(3 h + 3e-3) of a times the other factor, (h + 2e-3) of P |dO| for dV, and the result's own rounding h."""
import pytest
import torch

from tests import decoder_util as du
from tests.test_gpu_prefix_fwd import BF16, F16, check_fwd, ints, make

pytestmark = pytest.mark.gpu


def step(x, dO, scale, causal, lens):
    from paper_2502_12784_amd import spark_mha_prefix_bwd, spark_mha_prefix_fwd
    out = spark_mha_prefix_fwd(*x, scale, causal, *lens)
    return out, spark_mha_prefix_bwd(*x, *out, dO, scale, causal, *lens)


def check_bwd(x, dO, scale, causal, lens, grads, dtype):
    Q, Kp, Vp, Ks, Vs = x
    mask = du.prefix_mask(Kp.shape[0], Q.shape[0], Q.shape[2], Kp.shape[2], Ks.shape[2], causal, *lens)
    want = du.prefix_attention(*x, scale, mask, dO)
    h = du.HALF[dtype]
    for n, got in zip(("dQ", "dKp", "dVp", "dKs", "dVs"), grads):
        far = h + 2e-3 if n[1] == "V" else 3 * h + 3e-3
        du.close(got, want[n], h * want[n].abs() + far * (1 + h) * want["abs_" + n] + du.TINY[dtype], n)


def check(G, B, H, Hkv, Nq, P, S, d, dtype, causal=True, pl=None, ql=None, sl=None, layout="cache", seed=1):
    x = make(G, B, H, Hkv, Nq, P, S, d, dtype, seed, layout)
    dO = make(1, B, H, 1, Nq, 1, 1, d, dtype, seed + 100)[0]
    if layout == "packed":
        dO = dO.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    for t, lens, n in ((x[1], pl, P), (x[2], pl, P), (x[3], sl, S), (x[4], sl, S), (x[0], ql, Nq), (dO, ql, Nq)):
        for b, m in enumerate(lens or ()):
            t[b, :, max(0, min(m, n)):] = float("nan")  # behind a length: not used
    lens = [ints(v) for v in (pl, ql, sl)]
    out, grads = step(x, dO, d ** -0.5, causal, lens)
    torch.cuda.synchronize()
    check_fwd(x, d ** -0.5, causal, *lens, out, dtype)
    check_bwd(x, dO, d ** -0.5, causal, lens, grads, dtype)
    return x, dO, out, grads


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("d", [8, 40, 64, 72, 96, 104, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_head_sizes(d, causal, dtype):
    check(1, 2, 4, 2, 70, 131, 70, d, dtype, causal)


@pytest.mark.parametrize("P, S, Nq", [(1, 1, 1), (64, 1, 1), (63, 5, 1), (129, 64, 1), (0, 7, 1), (0, 130, 130), (5, 0, 3), (128, 0, 200),
                                      (1, 257, 257), (300, 300, 129), (64, 100, 300), (700, 33, 4), (640, 513, 500), (127, 127, 127),
                                      (64, 64, 64), (500, 3, 257), (256, 192, 192)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(P, S, Nq, causal):
    check(1, 3, 2, 2, Nq, P, S, 64, F16, causal, seed=2)
    check(1, 3, 2, 1, Nq, P, S, 128, BF16, causal, seed=2)


@pytest.mark.parametrize("G, B, H, Hkv, Nq", [(1, 1, 1, 1, 1), (1, 40, 8, 2, 1), (3, 12, 8, 2, 5), (2, 2, 12, 4, 33), (5, 5, 6, 1, 70),
                                             (4, 8, 16, 16, 65), (1, 7, 32, 1, 130)])
def test_groups_and_shared_heads(G, B, H, Hkv, Nq):
    check(G, B, H, Hkv, Nq, 333, 77, 64, BF16, seed=3)
    check(G, B, H, Hkv, Nq, 150, 70, 128, F16, seed=3)


@pytest.mark.parametrize("d, dtype", [(64, F16), (128, BF16), (80, BF16)])
@pytest.mark.parametrize("causal", [False, True])
def test_ragged_lengths_and_empty_rows(d, dtype, causal):
    pl, sl = [0, 130, 257], [0, 1, 64, 130, 200, 77]
    check(3, 6, 4, 2, 200, 257, 200, d, dtype, causal, pl=pl, sl=sl, ql=sl, seed=4)
    check(3, 6, 4, 2, 9, 257, 200, d, dtype, causal, pl=pl, sl=sl, ql=[9, 3, 0, 1, 9, 8], seed=4)
    check(3, 6, 4, 2, 150, 257, 200, d, dtype, causal, pl=pl, sl=sl, ql=[150, 70, 150, 1, 0, 149], seed=4)
    check(1, 6, 4, 2, 150, 257, 200, d, dtype, causal, sl=sl, ql=[0, 0, 0, 0, 0, 0], seed=4)


@pytest.mark.parametrize("G, B, H, Hkv, N, P, d, dtype", [(2, 44, 16, 16, 20, 150, 64, F16), (1, 16, 16, 16, 40, 200, 128, BF16),
                                                          (5, 20, 32, 16, 33, 130, 80, BF16), (1, 70, 8, 8, 3, 900, 48, BF16),
                                                          (2, 28, 24, 8, 50, 0, 112, F16)])
@pytest.mark.parametrize("causal", [False, True])
def test_a_grid_for_each_side(G, B, H, Hkv, N, P, d, dtype, causal):
    """Enough tiles of queries for dQ to have a grid of its own."""
    check(G, B, H, Hkv, N, P, N, d, dtype, causal, seed=15)
    sl = [(7 * b) % (N + 1) for b in range(B)]
    check(G, B, H, Hkv, N, P, N, d, dtype, causal, pl=[P - g for g in range(G)], sl=sl, ql=sl[::-1], seed=15)


@pytest.mark.parametrize("d", [64, 80, 128])
def test_slices_of_packed_projections(d):
    check(2, 4, 6, 2, 150, 200, 150, d, BF16, layout="packed", seed=6)
    check(1, 8, 4, 4, 200, 100, 200, d, F16, layout="packed", sl=[200, 3, 150, 64, 65, 199, 128, 1], ql=[200, 3, 150, 64, 65, 199, 128, 1],
          seed=6)


def test_rows_shared_by_several_workgroups_and_given_outputs():
    """Many sequences behind one tile of a prefix: its rows are split; the same bits in every run, and in given tensors."""
    from paper_2502_12784_amd import spark_mha_prefix_bwd, spark_mha_prefix_bwd_workspace_bytes
    x, dO, out, grads = check(1, 24, 4, 2, 100, 129, 100, 128, BF16, seed=7)
    stats = (24 * 4 * 100 * 8 + 255) // 256 * 256
    assert spark_mha_prefix_bwd_workspace_bytes(1, 24, 4, 2, 100, 129, 100, 128, True, 1) > stats
    mine = [torch.full_like(g, float("nan")) for g in grads]
    again = spark_mha_prefix_bwd(*x, *out, dO, 128 ** -0.5, dQ=mine[0], dKp=mine[1], dVp=mine[2], dKs=mine[3], dVs=mine[4])
    for a, b, c in zip(grads, again, mine):
        assert torch.equal(a, b) and b is c


def test_gradients_against_differences():
    """Central differences in 64 bits of the plain forward, at a few entries of each input."""
    lens = [ints([70, 33]), ints([20, 7, 20, 0]), ints([20, 30, 11, 4])]
    x = make(2, 4, 4, 2, 20, 70, 30, 16, F16, 9)
    dO = make(1, 4, 4, 1, 20, 1, 1, 16, F16, 10)[0]
    mask = du.prefix_mask(2, 4, 20, 70, 30, True, *lens)
    want = du.prefix_attention(*x, 0.3, mask, dO)
    xs = [t.double() for t in x]
    e = 1e-5
    for i, n in enumerate(("dQ", "dKp", "dVp", "dKs", "dVs")):
        for at in ((0, 0, 0, 0), (1, 1, 6, 15), (0, 1, 19, 3), (1, 0, 32, 7)):
            if at[2] >= xs[i].shape[2]:
                continue
            vals = []
            for sign in (1, -1):
                y = [t.clone() for t in xs]
                y[i][at] += sign * e
                vals.append(float((du.prefix_attention(*y, 0.3, mask)["O"] * dO.double()).sum()))
            assert abs((vals[0] - vals[1]) / (2 * e) - float(want[n][at])) <= 1e-5, (n, at)


def test_agrees_with_the_backward_over_one_sequence():
    from paper_2502_12784_amd import spark_mha_bwd
    x, dO, out, grads = check(1, 3, 4, 4, 333, 0, 333, 128, BF16, seed=8)
    old = spark_mha_bwd(x[0], x[3], x[4], out[0], out[1], dO, 128 ** -0.5, True)
    for a, b in zip((grads[0], grads[3], grads[4]), old):
        # the same products, sums and roundings of operands: where fp32 sums in another order meet a border, one step
        assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -7 * float(b.float().abs().max())


def test_another_stream_and_a_graph():
    x = make(2, 6, 4, 2, 100, 200, 100, 64, F16, 10)
    dO = make(1, 6, 4, 1, 100, 1, 1, 64, F16, 11)[0]
    run = lambda: sum((list(t) for t in step(x, dO, 0.125, True, (None, None, None))), [])  # noqa: E731
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for _ in range(3):
        x[0].mul_(1.0625)
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, held))


def test_general_path_of_the_binding_gives_the_same():
    """A call that the native path leaves to the Python one (a tensor subclass), forward and backward, both operators."""
    from paper_2502_12784_amd import spark_qk_norm_rope_bwd, spark_qk_norm_rope_fwd
    x = make(2, 4, 4, 2, 33, 70, 33, 64, BF16, 12)
    dO = make(1, 4, 4, 1, 33, 1, 1, 64, BF16, 13)[0]
    lens = [ints([70, 9]), ints([33, 1, 0, 20]), ints([30, 1, 2, 33])]
    a = step(x, dO, 0.125, True, lens)
    y = [torch.nn.Parameter(x[0], requires_grad=False)] + list(x[1:])
    b = step(y, dO, 0.125, True, lens)
    for s, t in zip(a, b):
        assert all(torch.equal(u, v) for u, v in zip(s, t))
    w = torch.ones(64, device="cuda")
    cos, sin = du.tables(33, 64)
    for Q in (x[0], y[0]):
        got = (*spark_qk_norm_rope_fwd(Q, x[3], w, w, cos, sin),
               *spark_qk_norm_rope_bwd(Q, x[3], w, w, cos, sin, dO, x[4]))
        want = got if Q is x[0] else want  # noqa: F821
        assert all(torch.equal(u, v) for u, v in zip(got, want))
