"""What the operators around a decoder's attention refuse, before anything reaches a device."""
import pytest
import torch

import paper_2502_12784_amd as pkg

OK, E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_WS = 0, -1, -2, -3, -4, -5
S = pkg.Strides


@pytest.fixture(scope="module")
def lib():
    return pkg.load_library()


def qk_fwd(lib, q=0x1000, kr=0x4000, cos=0x6000, positions=None, sq=S(64, 64, 64), skr=S(64, 64, 64), B=1, N=1, H=1, Hkv=1,
           d=64, rd=64, table=8, eps=1e-6, dtype=0):
    one = S(64, 64, 64)
    return lib.spark_qk_norm_rope_fwd(q, 0x2000, None, None, cos, 0x7000, positions, 0x3000, kr, sq, one, one, skr, B, N, H, Hkv,
                                      d, rd, table, eps, 0, 1, dtype, None)


def test_qk_forward(lib):
    assert qk_fwd(lib, q=None) == E_NULL
    assert qk_fwd(lib, cos=None) == E_NULL
    assert qk_fwd(lib, sq=None) == E_NULL
    assert qk_fwd(lib, dtype=2) == E_DTYPE
    for bad in (dict(B=0), dict(N=0), dict(H=0), dict(Hkv=0), dict(d=60), dict(d=136), dict(d=0), dict(rd=12), dict(rd=72),
                dict(rd=-8), dict(table=0), dict(N=9), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(eps=-1.0), dict(eps=1e-50), dict(B=1 << 16, N=1 << 16), dict(H=40000), dict(sq=S(64, 64, 32), N=2),
                dict(sq=S(-64, 64, 64), B=2), dict(skr=S(0, 64, 64), B=2), dict(skr=S(64, 0, 64), Hkv=2)):
        assert qk_fwd(lib, **bad) == E_SHAPE, bad
    assert qk_fwd(lib, sq=S(64, 64, 68), N=2) == E_ALIGN
    assert qk_fwd(lib, kr=0x4008) == E_ALIGN
    assert qk_fwd(lib, cos=0x6004) == E_ALIGN


def test_qk_backward(lib):
    def call(dwq=0x9000, ws=0xA000, ws_bytes=1 << 20, d=64, dtype=0, sdk=S(64, 64, 64), Hkv=1, N=1):
        one = S(64, 64, 64)
        return lib.spark_qk_norm_rope_bwd(0x1000, 0x2000, None, None, 0x6000, 0x7000, None, 0x3000, 0x4000, 0x5000, 0x8000, dwq,
                                          0xB000, one, one, one, one, one, sdk, ws, ws_bytes, 1, N, 1, Hkv, d, 64, 8, 1e-6, 0, 1,
                                          dtype, None)
    assert call(dwq=None) == E_NULL
    assert call(ws=None) == E_NULL
    assert call(d=68) == E_SHAPE
    assert call(N=9) == E_SHAPE
    assert call(dtype=5) == E_DTYPE
    assert call(sdk=S(64, 0, 64), Hkv=2) == E_SHAPE
    assert call(ws=0xA008) == E_ALIGN
    need = pkg.spark_qk_norm_rope_bwd_workspace_bytes(1, 1, 1, 1, 64, 64, 0)
    assert need == 2 * 64 * 4
    assert call(ws_bytes=need - 1) == E_WS
    assert pkg.spark_qk_norm_rope_bwd_workspace_bytes(1, 1, 1, 1, 60, 0, 0) == 0
    for B, N, H, Hkv in ((64, 4096, 32, 8), (1, 1, 64, 64), (1, 1 << 20, 1, 1), (1, 1 << 20, 5000, 4000)):
        assert pkg.spark_qk_norm_rope_bwd_workspace_bytes(B, N, H, Hkv, 128, 128, 1) <= (2048 + H + Hkv) * 128 * 4


def test_binding_refuses_tensors_that_are_not_on_the_device():
    x, w, c = torch.zeros(1, 1, 8, 64, dtype=torch.float16), torch.ones(64), torch.ones(8, 32)
    with pytest.raises(ValueError):
        pkg.spark_qk_norm_rope_fwd(x, x, w, w, c, c)
    with pytest.raises(ValueError):
        pkg.spark_qk_norm_rope_bwd(x, x, w, w, c, c, x, x)


def prefix_fwd(lib, q=0x1000, kp=0x2000, ks=0x4000, o=0x6000, lse=0x7000, ws=None, ws_bytes=0, G=1, B=2, H=4, Hkv=2, Nq=8, P=64,
               S=16, d=64, scale=0.125, causal=1, dtype=0, **strides):
    def c(h, n):
        return S_(h * n * d, n * d, d)
    S_ = S_type
    st = {"sQ": c(H, Nq), "sKp": c(Hkv, P), "sVp": c(Hkv, P), "sKs": c(Hkv, S), "sVs": c(Hkv, S), "sO": c(H, Nq)}
    st.update(strides)
    return lib.spark_mha_prefix_fwd(q, kp, 0x3000, ks, 0x5000, o, lse, *st.values(), None, None, None, ws, ws_bytes, G, B, H, Hkv, Nq,
                                    P, S, d, scale, causal, dtype, None)


S_type = S


def test_prefix_forward(lib):
    for bad in ("q", "kp", "ks", "o", "lse"):
        assert prefix_fwd(lib, **{bad: None}) == E_NULL, bad
    assert prefix_fwd(lib, sVs=None) == E_NULL
    assert prefix_fwd(lib, dtype=2) == E_DTYPE
    for bad in (dict(G=0), dict(B=0), dict(H=0), dict(Hkv=0), dict(Nq=0), dict(P=-1), dict(S=-1), dict(P=0, S=0), dict(B=3, G=2), dict(H=5),
                dict(d=60), dict(d=136), dict(scale=0.0), dict(scale=float("nan")), dict(scale=-1.0), dict(B=1 << 22, H=8),
                dict(P=1 << 25, d=128), dict(sQ=S(0, 0, 32)), dict(sKs=S(-8, 64, 64)), dict(sO=S(0, 512, 64)), dict(sO=S(2048, 0, 64)),
                dict(sKp=S(0, 0, 1 << 24)), dict(Nq=1 << 20, H=1 << 11, Hkv=1, B=1)):
        assert prefix_fwd(lib, **bad) == E_SHAPE, bad
    assert prefix_fwd(lib, sKs=S(2048, 1024, 68)) == E_ALIGN
    assert prefix_fwd(lib, q=0x1008) == E_ALIGN
    assert prefix_fwd(lib, ws=0x8008, ws_bytes=1 << 30) == E_ALIGN
    need = pkg.spark_mha_prefix_fwd_workspace_bytes(1, 32, 16, 16, 1, 4096, 256, 128, 1)
    assert need > 0 and need % (32 * 16 * 132 * 4) == 0
    assert prefix_fwd(lib, ws=0x8000, ws_bytes=need - 1, B=32, H=16, Hkv=16, Nq=1, P=4096, S=256, d=128) == E_WS
    assert pkg.spark_mha_prefix_fwd_workspace_bytes(1, 8, 16, 16, 512, 4096, 512, 128, 1) == 0  # every tile by itself
    assert pkg.spark_mha_prefix_fwd_workspace_bytes(1, 8, 16, 5, 1, 4096, 512, 128, 1) == 0     # no such problem


def test_prefix_backward(lib):
    def call(dq=0x9000, dkp=0xA000, lse=0x7000, ws=0xF000, ws_bytes=1 << 30, dtype=0, P=64, d=64, **strides):
        H, Hkv, Nq, S_, B = 4, 2, 8, 16, 2

        def c(h, n):
            return S(h * n * d, n * d, d)
        q, kp, ks = c(H, Nq), c(Hkv, P), c(Hkv, S_)
        st = {"sQ": q, "sKp": kp, "sVp": kp, "sKs": ks, "sVs": ks, "sO": q, "sdO": q, "sdQ": q, "sdKp": kp, "sdVp": kp, "sdKs": ks,
              "sdVs": ks}
        st.update(strides)
        return lib.spark_mha_prefix_bwd(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, lse, 0x8000, dq, dkp, 0xB000, 0xC000, 0xD000,
                                        *st.values(), None, None, None, ws, ws_bytes, 1, B, H, Hkv, Nq, P, S_, d, 0.125, 1, dtype, None)
    assert call(dq=None) == E_NULL
    assert call(dkp=None) == E_NULL
    assert call(lse=None) == E_NULL
    assert call(ws=None) == E_NULL
    assert call(sdKs=None) == E_NULL
    assert call(dtype=7) == E_DTYPE
    assert call(d=72 + 4) == E_SHAPE
    assert call(sdKs=S(0, 1024, 64)) == E_SHAPE      # a gradient that every sequence would write
    assert call(sdVp=S(0, 0, 64)) == E_SHAPE
    assert call(sdO=S(2048, 512, 66)) == E_ALIGN
    assert call(ws=0xF004) == E_ALIGN
    need = pkg.spark_mha_prefix_bwd_workspace_bytes(1, 2, 4, 2, 8, 64, 16, 64, True, 0)
    assert need >= 2 * 2 * 4 * 8 * 4
    assert call(ws_bytes=need - 1) == E_WS
    assert pkg.spark_mha_prefix_bwd_workspace_bytes(1, 2, 4, 3, 8, 64, 16, 64, True, 0) == 0


def test_prefix_binding_refuses_tensors_that_are_not_on_the_device():
    q, kp, ks = (torch.zeros(*s, dtype=torch.float16) for s in ((2, 4, 1, 64), (1, 2, 64, 64), (2, 2, 16, 64)))
    with pytest.raises(ValueError):
        pkg.spark_mha_prefix_fwd(q, kp, kp, ks, ks, 0.125)
    with pytest.raises(ValueError):
        pkg.spark_mha_prefix_bwd(q, kp, kp, ks, ks, q, torch.zeros(2, 4, 1), q, 0.125)
