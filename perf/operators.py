"""The operators around a decoder's attention: what their performance is judged on, and their plain forms.

Two operators, each forward and backward:

* ``spark_qk_norm_rope_*``: every head's query and key vector is divided by its root mean square, scaled by a
  learned vector and rotated by its token's position (the step between the projection and the attention).
* ``spark_mha_prefix_*``: attention of a batch whose sequences come in groups that share a long prefix: the keys and
  values of a group's prefix exist once, each sequence has its own suffix behind it.

A case is one pass of a user's program: a forward ("fwd") or a training step, forward and then backward ("step").
Inputs are normal random numbers, as everywhere in this repository; rotation tables are those of base 10000.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def _qk(name, what, B, N, H, Hkv, d, rd, dtype, interleaved=False, layout="packed", far=0):
    c = {"op": "qk", "pass": what, "B": B, "N": N, "H": H, "Hkv": Hkv, "d": d, "rd": rd, "dtype": dtype,
         "interleaved": interleaved, "layout": layout, "far": far}
    return dict(c, name=name) if name else c


def _prefix(name, what, G, B, H, Hkv, Nq, P, S, d, dtype, causal=True, ragged=False):
    c = {"op": "prefix", "pass": what, "G": G, "B": B, "H": H, "Hkv": Hkv, "Nq": Nq, "P": P, "S": S, "d": d,
         "dtype": dtype, "causal": causal, "ragged": ragged}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token in each of eight sequences of a decoder, at positions of their own: launches count.
        _qk("qk-one-token-fwd", "fwd", 8, 1, 16, 16, 128, 128, "bf16", far=4000),
        # A prompt of 2048 tokens in four sequences, slices of the packed projection.
        _qk("qk-prompt-fwd", "fwd", 4, 2048, 16, 16, 128, 128, "bf16"),
        # Training on ragged lengths, a head size between the tiles, part of it rotated, neighbours paired.
        _qk("qk-ragged-step", "step", 3, 1333, 12, 4, 80, 48, "f16", interleaved=True),
        # One sequence of 16384 tokens, narrow heads, four queries to a key, heads outermost.
        _qk("qk-long-step", "step", 1, 16384, 32, 8, 64, 64, "f16", layout="bhnd"),
        # Two short answers to one short prompt: the smallest call.
        _prefix("decode-two-fwd", "fwd", 1, 2, 4, 4, 1, 200, 16, 64, "f16"),
        # 32 requests behind one system prompt, one new token each, a head of keys for every head of queries.
        _prefix("decode-shared-fwd", "fwd", 1, 32, 16, 16, 1, 4096, 256, 128, "bf16", ragged=True),
        # 64 samples behind a long document, four heads of queries to one of keys: the prefix is a matrix product.
        _prefix("decode-grouped-fwd", "fwd", 1, 64, 32, 8, 1, 16384, 512, 128, "bf16", ragged=True),
        # Five drafted tokens a sequence are looked at together; three prompts of odd lengths, four sequences each.
        _prefix("draft-five-fwd", "fwd", 3, 12, 32, 8, 5, 4001, 333, 64, "f16", ragged=True),
        # The requests' own 512 tokens behind a prompt that is in the cache already.
        _prefix("extend-prompt-fwd", "fwd", 1, 8, 16, 16, 512, 4096, 512, 128, "bf16"),
        # Training on eight sampled answers each to two prompts, answers of different lengths.
        _prefix("group-step", "step", 2, 16, 16, 4, 512, 1024, 512, 128, "bf16", ragged=True),
        # The same with odd sizes everywhere and a head size between the tiles.
        _prefix("group-odd-step", "step", 3, 6, 6, 2, 333, 700, 333, 80, "f16", ragged=True),
        # Long answers to a long prompt: the largest case.
        _prefix("group-long-step", "step", 1, 8, 16, 16, 1024, 4096, 1024, 128, "bf16"),
    ]


def _scores(c):
    """Entries of the score matrix, which the plain form holds whole."""
    return c["B"] * c["H"] * c["Nq"] * (c["P"] + c["S"])


def draw(rng):
    def size(lo, hi):  # spread over the logarithm, odd values among them
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n if rng.random() < 0.5 else max(lo, min(hi, (n + 63) // 64 * 64))

    while True:
        kind = rng.choice(["qk", "qk", "decode", "decode", "draft", "extend", "group", "group"])
        d = rng.choice([64, 128, 64, 128, 8 * rng.randint(4, 16)])
        dtype = rng.choice(["f16", "bf16"])
        Hkv = rng.choice([1, 2, 4, 8, 16])
        H = Hkv * rng.choice([1, 1, 2, 4])
        if kind == "qk":
            what = rng.choice(["fwd", "step"])
            N = 1 if what == "fwd" and rng.random() < 0.4 else size(16, 16384)
            B = size(1, 64) if N == 1 else max(1, min(16, size(1, 32768) // N))
            rd = d if rng.random() < 0.7 else 8 * rng.randint(1, d // 8)
            c = _qk(None, what, B, N, H, Hkv, d, rd, dtype, rng.random() < 0.3, rng.choice(["packed", "bhnd"]),
                    4000 if N == 1 else 0)
        else:
            G, Bg = rng.choice([1, 1, 2, 3]), rng.choice([1, 2, 4, 5, 8, 16, 32, 64])
            P, S = size(64, 16384), size(16, 1024)
            if kind == "decode":
                c = _prefix(None, "fwd", G, G * Bg, H, Hkv, 1, P, S, d, dtype, ragged=rng.random() < 0.6)
            elif kind == "draft":
                c = _prefix(None, "fwd", G, G * Bg, H, Hkv, rng.randint(2, 12), P, S, d, dtype, ragged=rng.random() < 0.6)
            else:
                N = size(16, 1024)
                c = _prefix(None, "fwd" if kind == "extend" else "step", G, G * min(Bg, 16), H, Hkv, N, min(P, 8192), N, d,
                            dtype, rng.random() < 0.85, rng.random() < 0.6)
        w, most = work(c), work(listed()[-1])
        scores = 0 if kind == "qk" else _scores(c)
        if w["flops"] <= most["flops"] and w["bytes"] <= 2e9 and scores <= _scores(listed()[-1]):
            return c


def _lengths(case):
    """Suffix lengths of a case's sequences, and how many of the Nq query rows of each are in use."""
    B, S, Nq = case["B"], case["S"], case["Nq"]
    s = [S - (b * 1597) % (S // 2 + 1) if case["ragged"] else S for b in range(B)]
    return s, ([min(Nq, n) for n in s] if Nq == S else [Nq] * B)


def _prefix_lengths(case):
    P = case["P"]
    return [P - (g * 977) % (P // 3 + 1) if case["ragged"] else P for g in range(case["G"])]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    d = case["d"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(dt)

    if case["op"] == "qk":
        B, N, H, Hkv, rd = (case[k] for k in ("B", "N", "H", "Hkv", "rd"))

        def pair():
            if case["layout"] == "packed":  # [B, N, heads of Q, K and V, d]
                x = normal(B, N, H + 2 * Hkv, d)
                return x[:, :, :H].permute(0, 2, 1, 3), x[:, :, H:H + Hkv].permute(0, 2, 1, 3)
            return normal(B, H, N, d), normal(B, Hkv, N, d)

        s = {"case": case}
        s["Q"], s["K"] = pair()
        s["dQr"], s["dKr"] = pair()
        s["wq"], s["wk"] = (1 + 0.1 * torch.randn(d, generator=g, device="cuda") for _ in range(2))
        first = torch.randint(0, case["far"] + 1, (B, 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(N, device="cuda")).to(torch.int32) if case["far"] else None
        angles = torch.outer(torch.arange(N + case["far"], dtype=torch.float64, device="cuda"),
                             10000.0 ** (-torch.arange(0, rd, 2, dtype=torch.float64, device="cuda") / rd))
        s["cos"], s["sin"] = angles.cos().float(), angles.sin().float()
        return s
    G, B, H, Hkv, Nq, P, S = (case[k] for k in ("G", "B", "H", "Hkv", "Nq", "P", "S"))
    s = {"case": case, "scale": 1.0 / math.sqrt(d)}
    if case["pass"] == "step":  # slices of the packed projection of the answers, [B, N, heads, d]
        x = normal(B, Nq, H + 2 * Hkv, d).permute(0, 2, 1, 3)
        s["Q"], s["Ks"], s["Vs"] = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
        s["dO"] = normal(B, Nq, H, d).permute(0, 2, 1, 3)
    else:  # a cache, [B, Hkv, S, d]
        s["Q"], s["Ks"], s["Vs"] = normal(B, H, Nq, d), normal(B, Hkv, S, d), normal(B, Hkv, S, d)
    s["Kp"], s["Vp"] = normal(G, Hkv, P, d), normal(G, Hkv, P, d)
    lens = {"prefix_lens": _prefix_lengths(case), "s_lens": _lengths(case)[0], "q_lens": _lengths(case)[1]}
    for k, v in lens.items():
        s[k] = torch.tensor(v, dtype=torch.int32, device="cuda") if case["ragged"] else None
    return s


def run(s):
    if s["case"]["op"] == "qk":
        return _run_qk(s)
    return _run_prefix(s)


def _run_qk(s):
    c = s["case"]
    if own:
        from paper_2502_12784_amd import spark_qk_norm_rope_bwd, spark_qk_norm_rope_fwd
        args, how = (s["Q"], s["K"], s["wq"], s["wk"], s["cos"], s["sin"]), (s["positions"], EPS, c["interleaved"])
        out = spark_qk_norm_rope_fwd(*args, *how)
        return tuple(out) + (tuple(spark_qk_norm_rope_bwd(*args, s["dQr"], s["dKr"], *how)) if c["pass"] == "step" else ())
    if s["positions"] is None:
        cos, sin = s["cos"][:c["N"]], s["sin"][:c["N"]]
    else:
        cos, sin = s["cos"][s["positions"].long()][:, None], s["sin"][s["positions"].long()][:, None]
    q, k = _norm_rope(s["Q"], s["wq"], cos, sin, c), _norm_rope(s["K"], s["wk"], cos, sin, c)
    if c["pass"] == "fwd":
        return q, k
    dq, dwq = _norm_rope_grad(s["Q"], s["wq"], cos, sin, c, s["dQr"])
    dk, dwk = _norm_rope_grad(s["K"], s["wk"], cos, sin, c, s["dKr"])
    return q, k, dq, dk, dwq, dwk


def _rotate(y, cos, sin, c):
    rd = c["rd"]
    a, b = (y[..., 0:rd:2], y[..., 1:rd:2]) if c["interleaved"] else (y[..., :rd // 2], y[..., rd // 2:rd])
    u, v = a * cos - b * sin, b * cos + a * sin
    both = torch.stack((u, v), -1).flatten(-2) if c["interleaved"] else torch.cat((u, v), -1)
    return torch.cat((both, y[..., rd:]), -1)


def _norm_rope(x, w, cos, sin, c):
    x32 = x.float()
    y = x32 * torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + EPS) * w
    return _rotate(y, cos, sin, c).to(x.dtype)


def _norm_rope_grad(x, w, cos, sin, c, dout):
    x32 = x.float()
    r = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + EPS)
    dy = _rotate(dout.float(), cos, -sin, c)
    n = x32 * r
    t = dy * w
    dx = r * (t - n * (t * n).mean(-1, keepdim=True))
    return dx.to(x.dtype), (dy * n).sum((0, 1, 2), dtype=torch.float64).float()


def _run_prefix(s):
    c, scale = s["case"], s["scale"]
    if own:
        from paper_2502_12784_amd import spark_mha_prefix_bwd, spark_mha_prefix_fwd
        x = (s["Q"], s["Kp"], s["Vp"], s["Ks"], s["Vs"])
        how = (scale, c["causal"], s["prefix_lens"], s["q_lens"], s["s_lens"])
        out = spark_mha_prefix_fwd(*x, *how)
        return tuple(out) + (tuple(spark_mha_prefix_bwd(*x, *out, s["dO"], *how)) if c["pass"] == "step" else ())
    G, B, H, Hkv, Nq, P, S, d = (c[k] for k in ("G", "B", "H", "Hkv", "Nq", "P", "S", "d"))
    dt, dev = DTYPES[c["dtype"]], s["Q"].device

    def full(t, n, m):
        return torch.full((n,), m, dtype=torch.int32, device=dev) if t is None else t

    pl, ql, sl = full(s["prefix_lens"], G, P), full(s["q_lens"], B, Nq), full(s["s_lens"], B, S)
    i, j = torch.arange(Nq, device=dev), torch.arange(S, device=dev)
    live = i < ql[:, None]  # [B, Nq]
    seen = (j < sl[:, None])[:, None, :].expand(B, Nq, S)
    if c["causal"]:
        seen = seen & (j <= (i + (sl - ql)[:, None])[:, :, None])
    seen_p = (torch.arange(P, device=dev) < pl[:, None]).repeat_interleave(B // G, 0)  # [B, P]
    # keys of the prefix, then of the suffix; heads [Hkv, H / Hkv]
    mask = torch.cat((seen_p[:, None, :].expand(B, Nq, P), seen), -1) & live[:, :, None]  # [B, Nq, P + S]
    mask = mask[:, None, None]

    def by_prefix(t):  # [B, Hkv, H / Hkv, Nq, n] -> [G, Hkv, rows of the group, n]
        return t.reshape(G, B // G, Hkv, -1, t.shape[-1]).transpose(1, 2).reshape(G, Hkv, -1, t.shape[-1])

    def by_head(t):  # and back
        return t.reshape(G, Hkv, B // G, -1, t.shape[-1]).transpose(1, 2).reshape(B, Hkv, H // Hkv, Nq, t.shape[-1])

    def rows(t):  # [B, Hkv, H / Hkv, Nq, n] -> [B, Hkv, rows of the sequence, n]
        return t.reshape(B, Hkv, -1, t.shape[-1])

    def heads(t):
        return t.reshape(B, Hkv, H // Hkv, Nq, t.shape[-1])

    Q = heads(s["Q"].float())
    Kp, Vp, Ks, Vs = (s[n].float() for n in ("Kp", "Vp", "Ks", "Vs"))
    x = torch.cat((by_head(by_prefix(Q) @ Kp.mT.contiguous()), heads(rows(Q) @ Ks.mT.contiguous())), -1) * scale
    x = x.masked_fill(~mask, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    x = torch.exp(x - top)
    total = x.sum(-1, keepdim=True)
    lse = (torch.log(total) + top).reshape(B, H, Nq)
    x = x / torch.where(total == 0, torch.ones_like(total), total)
    O = by_head(by_prefix(x[..., :P]) @ Vp) + heads(rows(x[..., P:]) @ Vs)
    out = (O.reshape(B, H, Nq, d).to(dt), lse)
    if c["pass"] == "fwd":
        return out
    dO = heads(s["dO"].float()) * live[:, None, None, :, None]
    dx = torch.cat((by_head(by_prefix(dO) @ Vp.mT.contiguous()), heads(rows(dO) @ Vs.mT.contiguous())), -1)
    dx = x * (dx - (dO * O).sum(-1, keepdim=True)) * scale
    dQ = by_head(by_prefix(dx[..., :P]) @ Kp) + heads(rows(dx[..., P:]) @ Ks)
    Qg, dOg = by_prefix(Q), by_prefix(dO)
    grads = (dQ.reshape(B, H, Nq, d), by_prefix(dx[..., :P]).mT.contiguous() @ Qg, by_prefix(x[..., :P]).mT.contiguous() @ dOg,
             rows(dx[..., P:]).mT.contiguous() @ rows(Q), rows(x[..., P:]).mT.contiguous() @ rows(dO))
    return out + tuple(t.to(dt) for t in grads)


def work(case):
    d = case["d"]
    if case["op"] == "qk":
        n = float(case["B"] * case["N"] * (case["H"] + case["Hkv"]) * d)
        step = case["pass"] == "step"
        # x and the result; backward: x, the result's gradient and dx; tables, weights and positions are small
        tables = 4.0 * case["N"] * case["rd"] + 8.0 * d
        return {"bytes": n * 2 * (5 if step else 2) + tables, "flops": n * (20 if step else 8)}
    G, B, H, Hkv, Nq, P = (case[k] for k in ("G", "B", "H", "Hkv", "Nq", "P"))
    s, q = _lengths(case)
    pre = _prefix_lengths(case)
    pairs = 0.0
    for b in range(B):
        pairs += q[b] * float(pre[b // (B // G)])
        if case["causal"]:  # row i sees min(s, i + s - q + 1) keys of the suffix
            pairs += sum(max(0, i + s[b] - q[b] + 1) for i in range(q[b]))
        else:
            pairs += q[b] * float(s[b])
    flops = 4.0 * H * pairs * d
    keys = 4.0 * d * Hkv * (sum(pre) + sum(s))  # K and V, 16 bits
    rows = 2.0 * d * H * sum(q)
    nbytes = keys + 2 * rows + 4.0 * B * H * Nq
    if case["pass"] == "step":
        flops *= 3.5
        nbytes += 2 * keys + 4 * rows + 4.0 * B * H * Nq  # and again with O and dO, dQ and the keys' gradients written
    return {"bytes": nbytes, "flops": flops}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_qk(case, s) if case["op"] == "qk" else _exact_prefix(case, s)


def _exact_qk(case, s):
    """Rotations as products of complex numbers, gradients by torch's differentiation, in 64 bits."""
    rd, half = case["rd"], case["rd"] // 2
    at = torch.arange(case["N"], device="cuda")[None] if s["positions"] is None else s["positions"].long()
    turn = torch.complex(s["cos"].double(), s["sin"].double())[at][:, None]

    def forward(x, w):
        x = x / ((x ** 2).sum(-1, keepdim=True) / case["d"] + EPS) ** 0.5 * w
        r = x[..., :rd].unflatten(-1, (half, 2) if case["interleaved"] else (2, half))
        r = r if case["interleaved"] else r.transpose(-1, -2)
        z = torch.view_as_real(torch.complex(r[..., 0], r[..., 1]) * turn)
        z = z if case["interleaved"] else z.transpose(-1, -2)
        return torch.cat((z.flatten(-2), x[..., rd:]), -1)

    leaves = [s[n].double().requires_grad_(case["pass"] == "step") for n in ("Q", "K", "wq", "wk")]
    outs = [forward(leaves[0], leaves[2]), forward(leaves[1], leaves[3])]
    if case["pass"] == "fwd":
        return tuple(outs)
    grads = torch.autograd.grad(outs, leaves, [s["dQr"].double(), s["dKr"].double()])
    return tuple(o.detach() for o in outs) + tuple(grads)


def _exact_prefix(case, s):
    """Sequence by sequence, head of keys by head of keys, over the keys that exist, in 64 bits."""
    G, B, H, Hkv, Nq, S, d = (case[k] for k in ("G", "B", "H", "Hkv", "Nq", "S", "d"))
    slen, qlen = _lengths(case)
    plen = _prefix_lengths(case)
    r, step = H // Hkv, case["pass"] == "step"
    if 4.0 * B * H * Nq * d * (max(plen) + max(slen)) * (3.5 if step else 1) > 2e12:
        return None
    O = torch.zeros(B, H, Nq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, Nq), -math.inf, dtype=torch.float64, device="cuda")
    dQ = torch.zeros_like(O)
    dKp, dVp, dKs, dVs = (torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("Kp", "Vp", "Ks", "Vs"))
    for b in range(B):
        g = b // (B // G)
        n, m, p = qlen[b], slen[b], plen[g]
        hidden = torch.zeros(n, p + m, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden[:, p:] = torch.ones(n, m, dtype=torch.bool, device="cuda").triu(m - n + 1)
        K = torch.cat((s["Kp"][g, :, :p], s["Ks"][b, :, :m]), 1).double()
        V = torch.cat((s["Vp"][g, :, :p], s["Vs"][b, :, :m]), 1).double()
        q = s["Q"][b, :, :n].double()
        for h in range(H):
            k, v = K[h // r], V[h // r]
            t = (q[h] @ k.T * s["scale"]).masked_fill(hidden, -math.inf)
            l = torch.logsumexp(t, 1)
            w = torch.exp(t - l[:, None])
            O[b, h, :n], lse[b, h, :n] = w @ v, l
            if step:
                do = s["dO"][b, h, :n].double()
                dw = do @ v.T
                dt = w * (dw - (w * dw).sum(1, keepdim=True)) * s["scale"]
                dQ[b, h, :n] = dt @ k
                dk, dv = dt.T @ q[h], w.T @ do
                dKp[g, h // r, :p] += dk[:p]
                dVp[g, h // r, :p] += dv[:p]
                dKs[b, h // r, :m] += dk[p:]
                dVs[b, h // r, :m] += dv[p:]
    return (O, lse, dQ, dKp, dVp, dKs, dVs) if step else (O, lse)
