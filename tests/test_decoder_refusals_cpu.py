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
