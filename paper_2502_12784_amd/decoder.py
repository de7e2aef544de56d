"""The operators around a decoder's attention: norm and rotation of queries and keys, attention behind a shared prefix.

Argument marshalling only, as in ``binding``: the work is done by the HIP kernels of ``libspark_mha.so``.  Ordinary calls are
marshalled by the extension ``_spark_host``; what it does not take (and every error) goes through the code here.
"""
from __future__ import annotations

from . import binding
from .binding import Strides, _check, _dtype_code, _native, _stream_ptr, load_library


def _same_device(*tensors):
    """All tensors given (None: not given) on the current device; the kernels run there."""
    import torch
    for name, t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("%s must be a device tensor" % name)
        if t.device.index != torch.cuda.current_device():
            raise ValueError("%s is on %s, not on the current device %d" % (name, t.device, torch.cuda.current_device()))


def _rows(t, shape, dtype, name):
    """Check a [B,H,N,d] view whose last dimension is contiguous; return its spark_strides_t."""
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or (t.stride(3) != 1 and t.shape[3] != 1):
        raise ValueError("%s must be a %s view of shape %s with contiguous last dimension"
                         % (name, dtype, tuple(shape)))
    return Strides(t.stride(0), t.stride(1), t.stride(2))


def _ints(t, shape, name):
    """An optional contiguous int32 tensor; its address."""
    import torch
    if t is None:
        return None
    if tuple(t.shape) != tuple(shape) or t.dtype != torch.int32 or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of shape %s" % (name, tuple(shape)))
    return t.data_ptr()


def _scratch(workspace, need, like):
    import torch
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=like.device)
    elif not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace, workspace.numel() * workspace.element_size()


def _qk_problem(Q, K, wq, wk, cos, sin, positions, eps, interleaved):
    """(tensors' addresses, sizes, flags) shared by both directions of spark_qk_norm_rope."""
    import torch
    if Q.dim() != 4 or K.dim() != 4:
        raise ValueError("Q must be [B,H,N,d] and K [B,Hkv,N,d]")
    B, H, N, d = Q.shape
    code = _dtype_code(Q)
    _same_device(("Q", Q), ("K", K), ("wq", wq), ("wk", wk), ("cos", cos), ("sin", sin), ("positions", positions))
    given = [w for w in (wq, wk) if w is not None]
    for w in given:
        if tuple(w.shape) != (d,) or w.dtype not in (torch.float32, Q.dtype) or not w.is_contiguous():
            raise ValueError("wq and wk must be contiguous [%d] tensors of float32 or %s" % (d, Q.dtype))
    if len(given) == 2 and wq.dtype != wk.dtype:
        raise ValueError("wq and wk must have the same type")
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin are given together")
    table = rd = 0
    if cos is not None:
        if cos.dim() != 2:
            raise ValueError("cos and sin must be [positions, rd / 2]")
        table, rd = cos.shape[0], 2 * cos.shape[1]
        for t, n in ((cos, "cos"), (sin, "sin")):
            if tuple(t.shape) != tuple(cos.shape) or t.dtype != torch.float32 or not t.is_contiguous():
                raise ValueError("%s must be a contiguous float32 tensor of shape %s" % (n, tuple(cos.shape)))
    at = _ints(positions, (B, N), "positions")
    address = [None if t is None else t.data_ptr() for t in (wq, wk, cos, sin)] + [at]
    fp32 = int(bool(given) and given[0].dtype == torch.float32)
    sizes = (B, N, H, K.shape[1], d, rd, table, float(eps), int(bool(interleaved)), fp32, code)
    return address, sizes


def spark_qk_norm_rope_fwd(Q, K, wq, wk, cos, sin, positions=None, eps: float = 1e-6, interleaved: bool = False, Qr=None,
                           Kr=None):
    """Qr, Kr: every head's row of Q [B,H,N,d] and K [B,Hkv,N,d] divided by its root mean square, scaled by wq, wk ([d],
    fp32 or the tensors' type; None: not scaled) and its first 2 * cos.shape[1] elements rotated by its position's row of
    cos, sin ([positions, rd / 2] fp32; None: no rotation).  positions: [B,N] int32 (None: 0 ... N-1); a negative one marks
    padding, whose results are zeros.  Any strides; Qr and Kr may be given, as Q and K themselves or as rows of a cache."""
    import torch
    lib = load_library()
    out = binding._host.qk_fwd(Q, K, wq, wk, cos, sin, positions, eps, interleaved, Qr, Kr)
    if out is not None:
        return _native(out)
    address, sizes = _qk_problem(Q, K, wq, wk, cos, sin, positions, eps, interleaved)
    B, N, H, Hkv, d = sizes[:5]
    Qr = torch.empty_like(Q) if Qr is None else Qr
    Kr = torch.empty_like(K) if Kr is None else Kr
    _same_device(("Qr", Qr), ("Kr", Kr))
    qs, ks = (B, H, N, d), (B, Hkv, N, d)
    st = [_rows(Q, qs, Q.dtype, "Q"), _rows(K, ks, Q.dtype, "K"), _rows(Qr, qs, Q.dtype, "Qr"), _rows(Kr, ks, Q.dtype, "Kr")]
    _check(lib.spark_qk_norm_rope_fwd(Q.data_ptr(), K.data_ptr(), *address, Qr.data_ptr(), Kr.data_ptr(), *st, *sizes,
                                      _stream_ptr()))
    return Qr, Kr


def spark_qk_norm_rope_bwd_workspace_bytes(B: int, N: int, H: int, Hkv: int, d: int, rd: int, dtype_code: int) -> int:
    return int(load_library().spark_qk_norm_rope_bwd_workspace_bytes(B, N, H, Hkv, d, rd, dtype_code))


def spark_qk_norm_rope_bwd(Q, K, wq, wk, cos, sin, dQr, dKr, positions=None, eps: float = 1e-6, interleaved: bool = False,
                           dQ=None, dK=None, dwq=None, dwk=None, workspace=None):
    """dQ, dK, dwq, dwk for the problem of spark_qk_norm_rope_fwd, whose Q and K must still hold the forward's inputs.
    dwq and dwk are fp32."""
    import torch
    lib = load_library()
    if workspace is None:
        out = binding._host.qk_bwd(Q, K, wq, wk, cos, sin, dQr, dKr, positions, eps, interleaved, dQ, dK, dwq, dwk)
        if out is not None:
            return _native(out)
    address, sizes = _qk_problem(Q, K, wq, wk, cos, sin, positions, eps, interleaved)
    B, N, H, Hkv, d, rd = sizes[:6]
    dQ = torch.empty_like(Q) if dQ is None else dQ
    dK = torch.empty_like(K) if dK is None else dK
    dwq = torch.empty(d, dtype=torch.float32, device=Q.device) if dwq is None else dwq
    dwk = torch.empty(d, dtype=torch.float32, device=Q.device) if dwk is None else dwk
    _same_device(("dQr", dQr), ("dKr", dKr), ("dQ", dQ), ("dK", dK), ("dwq", dwq), ("dwk", dwk), ("workspace", workspace))
    for t, n in ((dwq, "dwq"), (dwk, "dwk")):
        binding._require(t, (d,), torch.float32, n)
    qs, ks = (B, H, N, d), (B, Hkv, N, d)
    st = [_rows(Q, qs, Q.dtype, "Q"), _rows(K, ks, Q.dtype, "K"), _rows(dQr, qs, Q.dtype, "dQr"),
          _rows(dKr, ks, Q.dtype, "dKr"), _rows(dQ, qs, Q.dtype, "dQ"), _rows(dK, ks, Q.dtype, "dK")]
    need = spark_qk_norm_rope_bwd_workspace_bytes(B, N, H, Hkv, d, rd, sizes[-1])
    workspace, nbytes = _scratch(workspace, need, Q)
    _check(lib.spark_qk_norm_rope_bwd(Q.data_ptr(), K.data_ptr(), *address, dQr.data_ptr(), dKr.data_ptr(), dQ.data_ptr(),
                                      dK.data_ptr(), dwq.data_ptr(), dwk.data_ptr(), *st, workspace.data_ptr(), nbytes,
                                      *sizes, _stream_ptr()))
    return dQ, dK, dwq, dwk


def _prefix_problem(Q, Kp, Vp, Ks, Vs, prefix_lens, q_lens, s_lens):
    """(sizes G, B, H, Hkv, Nq, P, S, d; strides of the five tensors; addresses of the lengths)"""
    for t, n in ((Q, "Q"), (Kp, "Kp"), (Vp, "Vp"), (Ks, "Ks"), (Vs, "Vs")):
        if t.dim() != 4:
            raise ValueError("%s must have four dimensions" % n)
    _same_device(("Q", Q), ("Kp", Kp), ("Vp", Vp), ("Ks", Ks), ("Vs", Vs), ("prefix_lens", prefix_lens), ("q_lens", q_lens),
                 ("s_lens", s_lens))
    B, H, Nq, d = Q.shape
    G, Hkv, P = Kp.shape[:3]
    S = Ks.shape[2]
    _dtype_code(Q)
    strides = [_rows(Q, (B, H, Nq, d), Q.dtype, "Q")]
    strides += [_rows(t, (G, Hkv, P, d), Q.dtype, n) for t, n in ((Kp, "Kp"), (Vp, "Vp"))]
    strides += [_rows(t, (B, Hkv, S, d), Q.dtype, n) for t, n in ((Ks, "Ks"), (Vs, "Vs"))]
    lens = [_ints(prefix_lens, (G,), "prefix_lens"), _ints(q_lens, (B,), "q_lens"), _ints(s_lens, (B,), "s_lens")]
    return (G, B, H, Hkv, Nq, P, S, d), strides, lens


def spark_mha_prefix_fwd_workspace_bytes(G: int, B: int, H: int, Hkv: int, Nq: int, P: int, S: int, d: int,
                                         dtype_code: int) -> int:
    return int(load_library().spark_mha_prefix_fwd_workspace_bytes(G, B, H, Hkv, Nq, P, S, d, dtype_code))


def spark_mha_prefix_fwd(Q, Kp, Vp, Ks, Vs, scale: float, causal: bool = True, prefix_lens=None, q_lens=None, s_lens=None,
                         O=None, LSE=None, workspace=None):
    """O, LSE of Q [B,H,Nq,d] attending to the prefix Kp, Vp [G,Hkv,P,d] that B / G sequences in a row share, and to their
    own suffixes Ks, Vs [B,Hkv,S,d].  prefix_lens [G], q_lens, s_lens [B]: int32 on the device, how much of P, Nq, S is in
    use.  causal: query i sees suffix keys j <= i + s_lens - q_lens.  Rows from q_lens on, and rows that see no key, give
    O = 0 and LSE = -inf.  Any strides.  workspace: allocated here if not given; with an empty one every query tile is one
    workgroup's, which for few rows is slow; one kept for several problems has the largest of their sizes (a smaller problem
    may need more)."""
    import torch
    lib = load_library()
    if workspace is None:
        out = binding._host.prefix_fwd(Q, Kp, Vp, Ks, Vs, scale, causal, prefix_lens, q_lens, s_lens, O, LSE)
        if out is not None:
            return _native(out)
    sizes, strides, lens = _prefix_problem(Q, Kp, Vp, Ks, Vs, prefix_lens, q_lens, s_lens)
    G, B, H, Hkv, Nq, P, S, d = sizes
    code = _dtype_code(Q)
    O = torch.empty_like(Q) if O is None else O
    LSE = torch.empty((B, H, Nq), dtype=torch.float32, device=Q.device) if LSE is None else LSE
    _same_device(("O", O), ("LSE", LSE), ("workspace", workspace))
    strides.append(_rows(O, (B, H, Nq, d), Q.dtype, "O"))
    binding._require(LSE, (B, H, Nq), torch.float32, "LSE")
    workspace, nbytes = _scratch(workspace, spark_mha_prefix_fwd_workspace_bytes(*sizes, code), Q)
    _check(lib.spark_mha_prefix_fwd(Q.data_ptr(), Kp.data_ptr(), Vp.data_ptr(), Ks.data_ptr(), Vs.data_ptr(), O.data_ptr(),
                                    LSE.data_ptr(), *strides, *lens, workspace.data_ptr(), nbytes, *sizes, float(scale),
                                    int(bool(causal)), code, _stream_ptr()))
    return O, LSE


def spark_mha_prefix_bwd_workspace_bytes(G: int, B: int, H: int, Hkv: int, Nq: int, P: int, S: int, d: int, causal: bool,
                                         dtype_code: int) -> int:
    return int(load_library().spark_mha_prefix_bwd_workspace_bytes(G, B, H, Hkv, Nq, P, S, d, int(bool(causal)), dtype_code))


def spark_mha_prefix_bwd(Q, Kp, Vp, Ks, Vs, O, LSE, dO, scale: float, causal: bool = True, prefix_lens=None, q_lens=None,
                         s_lens=None, dQ=None, dKp=None, dVp=None, dKs=None, dVs=None, workspace=None):
    """dQ, dKp, dVp, dKs, dVs for the problem of spark_mha_prefix_fwd and its O and LSE.  dKp and dVp sum over the sequences
    that share the prefix; what is not in use is zero.  Gradients default to the layouts of Q, Kp, Vp, Ks, Vs."""
    import torch
    lib = load_library()
    if workspace is None:
        out = binding._host.prefix_bwd(Q, Kp, Vp, Ks, Vs, O, LSE, dO, scale, causal, prefix_lens, q_lens, s_lens, dQ, dKp, dVp,
                                       dKs, dVs)
        if out is not None:
            return _native(out)
    sizes, strides, lens = _prefix_problem(Q, Kp, Vp, Ks, Vs, prefix_lens, q_lens, s_lens)
    G, B, H, Hkv, Nq, P, S, d = sizes
    code = _dtype_code(Q)
    dQ, dKp, dVp, dKs, dVs = (torch.empty_like(like) if t is None else t for t, like in
                              ((dQ, Q), (dKp, Kp), (dVp, Vp), (dKs, Ks), (dVs, Vs)))
    _same_device(("O", O), ("LSE", LSE), ("dO", dO), ("dQ", dQ), ("dKp", dKp), ("dVp", dVp), ("dKs", dKs), ("dVs", dVs),
                 ("workspace", workspace))
    qs, ps, ss = (B, H, Nq, d), (G, Hkv, P, d), (B, Hkv, S, d)
    strides += [_rows(t, shape, Q.dtype, n) for t, shape, n in
                ((O, qs, "O"), (dO, qs, "dO"), (dQ, qs, "dQ"), (dKp, ps, "dKp"), (dVp, ps, "dVp"), (dKs, ss, "dKs"),
                 (dVs, ss, "dVs"))]
    binding._require(LSE, (B, H, Nq), torch.float32, "LSE")
    workspace, nbytes = _scratch(workspace, spark_mha_prefix_bwd_workspace_bytes(*sizes, causal, code), Q)
    _check(lib.spark_mha_prefix_bwd(*(t.data_ptr() for t in (Q, Kp, Vp, Ks, Vs, O, LSE, dO, dQ, dKp, dVp, dKs, dVs)), *strides,
                                    *lens, workspace.data_ptr(), nbytes, *sizes, float(scale), int(bool(causal)), code,
                                    _stream_ptr()))
    return dQ, dKp, dVp, dKs, dVs
