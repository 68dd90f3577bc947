"""Cases and plain forms of the operators of a layer around its attention: the norm with an output in 8 bits, the product of two
matrices held in 8 bits, and the storing of new keys and values with the rotation by position.

Three operators; activations are bf16, 8-bit values int8 or e4m3 with a scale in f32 for every row (a token of activations, an
output channel of weights):

  norm     h = x + residual, kept on request; root-mean-square or layer norm of h, or h itself; the result in bf16, in 8 bits with
           a scale per row, or in both                                                              llmcache_norm
  dense    act(a w^T) + residual for a and w in 8 bits; int8 is summed in whole numbers              llmcache_dense
  append   queries and keys of new tokens are rotated by their positions, keys and values go to their places in a paged cache
                                                                                                     llmcache_kv_append

`run` computes them from elementary torch operations in 32 bits (angles in 64), or, with `own` set, through the library's entry
points.  Values in int8 are handed back in the activations' type, as the numbers that they stand for.
"""
import math

import numpy as np
import torch

own = False

DH = 64
DEV = "cuda"
BF = torch.bfloat16
E4M3 = torch.float8_e4m3fn
TOP = {"int8": 127.0, "e4m3": 448.0}                     # largest magnitude of each type


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token on its way into a layer's first product: latency
        _norm("norm one token", rows=1, cols=1024, kind="rms", residual=True, total=True, out=False, to="e4m3"),
        # a batch behind the attention of an encoder layer: the next product takes the 8 bits, the next residual the bf16 rows
        _norm("norm of an encoder's batch, int8", rows=12288, cols=768, kind="layer", residual=False, total=False, out=True, to="int8"),
        # the residual stream of a long batch between two layers
        _norm("norm of a long residual stream", rows=131072, cols=1024, kind="rms", residual=True, total=True, out=False, to="e4m3"),
        # wide rows of a feed-forward block, an odd number of them, that only change their type
        _norm("to 8 bits, wide rows", rows=4001, cols=4096, kind="none", residual=False, total=False, out=False, to="e4m3"),
        # one token through the first feed-forward product: latency, and the reading of the weights
        _dense("dense one token", M=1, N=4096, K=1024, to="int8", bias=True, act="gelu_tanh"),
        # the next tokens of 64 sequences through the q|k|v product
        _dense("dense next tokens of a batch", M=64, N=2304, K=768, to="int8", bias=True),
        # a batch of misses through the first feed-forward product
        _dense("dense feed-forward of a batch", M=32768, N=4096, K=1024, to="int8", bias=True, act="gelu_erf"),
        # the second feed-forward product of a larger batch, onto the residual
        _dense("dense second feed-forward, e4m3", M=65536, N=1024, K=4096, to="e4m3", bias=True, residual=True),
        # scores over a vocabulary, for the last tokens of a ragged batch: nothing is a multiple of a tile
        _dense("dense over a vocabulary", M=1001, N=50257, K=768, to="int8"),
        # the next token of one sequence: latency
        _append("append one token", B=1, lo=517, hi=517, rows=1, H=12, HK=12, page=16, dims=64, interleaved=False, far=False),
        # the next tokens of 64 sequences of uneven lengths, grouped heads, positions far beyond the kept slots, neighbours paired
        _append("append next tokens of a batch", B=64, lo=301, hi=4100, rows=1, H=16, HK=4, page=64, dims=32, interleaved=True, far=True),
        # prompts of 1,024 tokens
        _append("append prompts", B=32, lo=1024, hi=1024, rows=1024, H=16, HK=16, page=64, dims=64, interleaved=False, far=False),
    ]


def _norm(name, rows, cols, kind, residual, total, out, to):
    return dict(name=name, op="norm", rows=rows, cols=cols, kind=kind, residual=residual, total=total, out=out, to=to)


def _dense(name, M, N, K, to, bias=False, act="none", residual=False):
    return dict(name=name, op="dense", M=M, N=N, K=K, to=to, bias=bias, act=act, residual=residual)


def _append(name, B, lo, hi, rows, H, HK, page, dims, interleaved, far):
    return dict(name=name, op="append", B=B, lo=lo, hi=hi, rows=rows, H=H, HK=HK, page=page, dims=dims, interleaved=interleaved, far=far)


def _spread(rng, lo, hi, step=1):
    """A multiple of step from lo to hi, even over its logarithm."""
    x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))
    return min(hi, max(lo, x // step * step))


def draw(rng):
    op = rng.choice(["norm", "dense", "append"])
    if op == "norm":
        cols = _spread(rng, 64, 16384, 8)
        kind = rng.choice(["none", "layer", "rms", "rms"])
        c = _norm("", rows=_spread(rng, 1, min(131072, 131072 * 1024 // cols)), cols=cols, kind=kind, residual=rng.random() < 0.6,
                  total=rng.random() < 0.5, out=rng.random() < 0.4, to=rng.choice(["int8", "e4m3"]))
    elif op == "dense":
        N, K = _spread(rng, 64, 50257), _spread(rng, 64, 8192, 16)
        most = max(1, min(65536, 65536 * 1024 * 4096 // (N * K), 65536 * 4096 // max(N, K)))
        c = _dense("", M=_spread(rng, 1, most), N=N, K=K, to=rng.choice(["int8", "e4m3"]), bias=rng.random() < 0.6,
                   act=rng.choice(["none", "gelu_erf", "gelu_tanh"]), residual=rng.random() < 0.4)
    else:
        H, HK = rng.choice([(12, 12), (16, 16), (16, 4), (12, 2), (8, 1), (6, 2)])
        rows = rng.choice([1, _spread(rng, 1, 1024)])
        hi = max(rows, _spread(rng, 1, 16000))
        most = max(1, min(64, 32 * 1024 * 96 // (rows * (2 * H + 4 * HK)), 1024 * 1024 * 4 // (hi * HK)))
        c = _append("", B=_spread(rng, 1, most), lo=max(rows, int(hi * rng.uniform(0.1, 1.0))), hi=hi, rows=rows, H=H, HK=HK,
                    page=rng.choice([16, 32, 64, 128]), dims=rng.choice([16, 32, 48, 64, 64]), interleaved=rng.random() < 0.5,
                    far=rng.random() < 0.5)
    del c["name"]
    return c


def _lengths(case):
    """The batch's cache lengths, from lo to hi in even steps (every seed deals the same lengths out in another order)."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    return [hi if B == 1 else lo + (hi - lo) * b // (B - 1) for b in range(B)]


def _chunks(case):
    """How many new tokens each sequence brings: `rows`, every fourth sequence about two thirds of them."""
    return [max(1, case["rows"] * 2 // 3) if b % 4 == 1 else case["rows"] for b in range(case["B"])]


def work(case):
    if case["op"] == "norm":
        n = case["rows"] * case["cols"]
        per = 2 + 2 * case["residual"] + 2 * case["total"] + 2 * case["out"] + 1
        return {"bytes": n * per + 4 * case["rows"] + (0 if case["kind"] == "none" else 4 * case["cols"]), "flops": 0}
    if case["op"] == "dense":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": (M + N) * (K + 4) + M * N * (2 + 2 * case["residual"]) + 4 * N * case["bias"], "flops": 2 * M * N * K}
    # queries and keys and values read, written; lengths and page numbers of the new rows
    return {"bytes": sum(_chunks(case)) * (2 * case["H"] + 4 * case["HK"]) * DH * 2 + 12 * case["B"], "flops": 0}


# --------------------------------------------------------------------------------------------------------- inputs
def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV).to(BF)


def _eight(case, x):
    """x in the case's 8-bit type."""
    return x.round().clamp(-127, 127).to(torch.int8) if case["to"] == "int8" else x.clamp(-448, 448).to(E4M3)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    st = {"case": case}
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        # a few columns are several times as large as the others, as in a trained model's residual stream
        wide = torch.where(torch.rand(cols, generator=g, device=DEV) < 0.01, 6.0, 1.0)
        st["x"] = (torch.randn((rows, cols), generator=g, device=DEV) * wide).to(BF)
        st["residual"] = _normal(g, rows, cols) if case["residual"] else None
        normed = case["kind"] != "none"
        st["gain"] = torch.rand(cols, generator=g, device=DEV) + 0.5 if normed else None
        st["bias"] = torch.randn(cols, generator=g, device=DEV) * 0.1 if case["kind"] == "layer" else None
        st["total"] = torch.empty((rows, cols), dtype=BF, device=DEV) if case["total"] else None
        st["out"] = torch.empty((rows, cols), dtype=BF, device=DEV) if case["out"] else None
        st["q"] = torch.empty((rows, cols), dtype=torch.int8 if case["to"] == "int8" else E4M3, device=DEV)
        st["scale"] = torch.empty(rows, device=DEV)
        st["values"] = torch.empty((rows, cols), dtype=BF, device=DEV) if case["to"] == "int8" else None
        return st
    if case["op"] == "dense":
        M, N, K = case["M"], case["N"], case["K"]
        # 8-bit values as a quantised normal distribution leaves them; products of the size of one
        spread = 30.0 if case["to"] == "int8" else 100.0
        st["a"] = _eight(case, torch.randn((M, K), generator=g, device=DEV) * spread)
        st["w"] = _eight(case, torch.randn((N, K), generator=g, device=DEV) * spread)
        st["a_scale"] = (torch.rand(M, generator=g, device=DEV) + 0.5) / spread
        st["w_scale"] = (torch.rand(N, generator=g, device=DEV) + 0.5) / (spread * math.sqrt(K))
        st["bias"] = torch.randn(N, generator=g, device=DEV) * 0.2 if case["bias"] else None
        pitch = -(-N // 8) * 8                           # rows of the result start on 16 bytes
        st["residual"] = _normal(g, M, pitch)[:, :N] if case["residual"] else None
        st["out"] = torch.empty((M, pitch), dtype=BF, device=DEV)[:, :N]
        return st
    order = np.random.RandomState(seed % (1 << 31))
    H, HK, ps, B = case["H"], case["HK"], case["page"], case["B"]
    lens = [_lengths(case)[i] for i in order.permutation(B)]
    rows = [min(r, n) for r, n in zip(_chunks(case), lens)]
    need = [-(-n // ps) for n in lens]
    pages = sum(need) + 3
    ids = order.permutation(pages).astype(np.int32)      # pages in the order in which an allocator has handed them out
    table = np.full((B, max(need)), -1, dtype=np.int32)
    at = 0
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
    T = sum(rows)
    st["host_lens"], st["rows"] = lens, rows
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    st["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32), device=DEV)
    st["pages"] = torch.from_numpy(table).to(DEV)
    st["k"], st["v"] = _normal(g, pages, HK, ps, DH), _normal(g, pages, HK, ps, DH)
    qkv = _normal(g, T, H + 2 * HK, DH)                  # one matrix with the columns q | k | v, as a projection writes it
    st["q"], st["k_new"], st["v_new"] = qkv[:, :H], qkv[:, H:H + HK], qkv[:, H + HK:]
    st["q_out"] = torch.empty((T, H, DH), dtype=BF, device=DEV)
    # angles per position: a geometric series, as rotary models have it
    half = case["dims"] // 2
    st["inv_freq"] = torch.tensor([10000.0 ** (-i / half) for i in range(half)], dtype=torch.float64, device=DEV)
    st["first"] = None
    if case["far"]:                                      # earlier slots were dropped: positions run ahead of the slots
        st["first"] = torch.tensor([int(x) for x in order.randint(100000, 1000000, B)], dtype=torch.int32, device=DEV)
    if own:
        from paper_2512_16843_b200 import binding as L
        st["rotation"] = L.make_rotation(st["inv_freq"], interleaved=case["interleaved"])
        st["cache"] = L.KVCache(st["k"], st["v"], heads=H, max_seqs=B, max_rows=T, max_len=max(need) * ps)
    return st


# ------------------------------------------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    if own:
        from paper_2512_16843_b200 import binding as L
        if case["op"] == "norm":
            L.llmcache_norm(st["x"], kind=case["kind"], gain=st["gain"], bias=st["bias"], residual=st["residual"], total=st["total"],
                            out=st["out"], q=st["q"], scale=st["scale"])
            if case["to"] == "int8":
                torch.mul(st["q"], st["scale"].unsqueeze(1), out=st["values"])
            return _norm_answer(st, st["total"], st["out"], st["values"] if case["to"] == "int8" else st["q"], st["scale"])
        if case["op"] == "dense":
            L.llmcache_dense(st["a"], st["a_scale"], st["w"], st["w_scale"], st["out"], bias=st["bias"], act=case["act"],
                              residual=st["residual"])
            return {"out": st["out"]}
        st["cache"].append(st["k_new"], st["v_new"], cu_rows=st["cu"], lens=st["lens"], pages=st["pages"], q=st["q"], q_out=st["q_out"],
                           rotation=st["rotation"], first=st["first"])
        return {"q": st["q_out"], "k": st["k"], "v": st["v"]}
    return {"norm": _plain_norm, "dense": _plain_dense, "append": _plain_append}[case["op"]](st)


def _norm_answer(st, total, out, values, scale):
    answer = {"values": values, "scale": scale}
    if st["case"]["total"]:
        answer["total"] = total
    if st["case"]["out"]:
        answer["out"] = out
    return answer


def _plain_norm(st):
    case = st["case"]
    h = st["x"].float()
    if st["residual"] is not None:
        h = h + st["residual"].float()
    y = h
    if case["kind"] == "layer":
        y = h - h.mean(-1, keepdim=True)
    if case["kind"] != "none":
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-5) * st["gain"]
    if st["bias"] is not None:
        y = y + st["bias"]
    top = TOP[case["to"]]
    scale = y.abs().amax(-1, keepdim=True) / top
    q = (y / scale).clamp(-top, top)
    values = (q.round() * scale).to(BF) if case["to"] == "int8" else q.to(E4M3)
    return _norm_answer(st, h.to(BF), y.to(BF), values, scale.squeeze(-1))


def _plain_dense(st):
    case = st["case"]
    y = torch.matmul(st["a"].float(), st["w"].float().t()) * (st["a_scale"].unsqueeze(1) * st["w_scale"])
    if st["bias"] is not None:
        y = y + st["bias"]
    if case["act"] == "gelu_erf":
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    elif case["act"] == "gelu_tanh":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return {"out": y.to(BF)}


def _turned(x, cos, sin, dims, interleaved):
    """x [rows, heads, 64] in 32 bits with its first `dims` columns rotated pair by pair; cos, sin [rows, dims / 2]."""
    cos, sin = cos.unsqueeze(1), sin.unsqueeze(1)
    part = x[..., :dims]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :dims // 2], part[..., dims // 2:])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((turned, x[..., dims:]), -1)


def _plain_append(st):
    case, cu, lens = st["case"], st["cu"].long(), st["lens"].long()
    count = cu[1:] - cu[:-1]
    row = torch.arange(st["q"].shape[0], device=DEV)
    seq = torch.searchsorted(cu[1:], row, right=True)
    slot = lens[seq] - count[seq] + row - cu[seq]
    position = slot if st["first"] is None else st["first"].long()[seq] + row - cu[seq]
    angle = position.double().unsqueeze(1) * st["inv_freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    page = st["pages"][seq, slot // case["page"]].long()
    st["k"][page, :, slot % case["page"]] = _turned(st["k_new"].float(), cos, sin, case["dims"], case["interleaved"]).to(BF)
    st["v"][page, :, slot % case["page"]] = st["v_new"]
    return {"q": _turned(st["q"].float(), cos, sin, case["dims"], case["interleaved"]).to(BF), "k": st["k"], "v": st["v"]}


# ------------------------------------------------------------------------------------------- the definition, exactly
def exact(case, seed):
    """What run() returns, from the definition in 64 bits."""
    st, f8 = prepare(case, seed), torch.float64
    if case["op"] == "norm":
        total, out, values, scales = [], [], [], []
        for lo in range(0, case["rows"], 16384):         # some rows at a time: 64 bits are large
            part = slice(lo, lo + 16384)
            z = st["x"][part].to(f8)
            if case["residual"]:
                z = z + st["residual"][part].to(f8)
            total.append(z)
            if case["kind"] == "layer":
                mu = z.sum(1) / case["cols"]
                z = z - mu[:, None]
            if case["kind"] != "none":
                size = torch.sqrt(torch.sum(z ** 2, 1) / case["cols"] + 1e-5)
                z = z / size[:, None] * st["gain"].to(f8)[None]
            if case["kind"] == "layer":
                z = z + st["bias"].to(f8)[None]
            out.append(z)
            s = torch.maximum(z.max(1).values, -z.min(1).values) / TOP[case["to"]]
            scales.append(s)
            z = z / s[:, None]
            values.append(torch.round(z) * s[:, None] if case["to"] == "int8" else z.to(E4M3).to(f8))
        answer = {"values": torch.cat(values), "scale": torch.cat(scales), "total": torch.cat(total), "out": torch.cat(out)}
        return {k: v for k, v in answer.items() if k in ("values", "scale") or case[k]}
    if case["op"] == "dense":
        M, N = case["M"], case["N"]
        y = torch.empty((M, N), dtype=f8, device=DEV)
        wt = st["w"].to(f8)
        for lo in range(0, M, 8192):
            part = slice(lo, lo + 8192)
            z = st["a"][part].to(f8) @ wt.T              # (whole numbers below 2^53 in int8: exact)
            z = z * st["a_scale"][part].to(f8)[:, None] * st["w_scale"].to(f8)[None]
            if case["bias"]:
                z = z + st["bias"].to(f8)[None]
            if case["act"] == "gelu_erf":
                z = z * torch.special.ndtr(z)
            if case["act"] == "gelu_tanh":
                z = z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
            if case["residual"]:
                z = z + st["residual"][part].to(f8)
            y[part] = z
        return {"out": y}
    half, ps = case["dims"] // 2, case["page"]
    k, v = st["k"].to(f8), st["v"].to(f8)
    q = torch.empty(st["q"].shape, dtype=f8, device=DEV)
    r0 = 0
    for b, (n, r) in enumerate(zip(st["host_lens"], st["rows"])):
        slot = torch.arange(n - r, n, device=DEV)
        at = slot if st["first"] is None else int(st["first"][b]) + torch.arange(r, device=DEV)
        turn = torch.polar(torch.ones((), dtype=f8, device=DEV), at.to(f8)[:, None] * st["inv_freq"])[:, None]    # [r, 1, half]

        def rotated(x):
            x = x[r0:r0 + r].to(f8).clone()
            i = torch.arange(half, device=DEV)
            re, im = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
            z = torch.complex(x[..., re], x[..., im]) * turn
            x[..., re], x[..., im] = z.real, z.imag
            return x

        q[r0:r0 + r] = rotated(st["q"])
        page = st["pages"][b].long()[slot // ps]
        k[page, :, slot % ps] = rotated(st["k_new"])
        v[page, :, slot % ps] = st["v_new"][r0:r0 + r].to(f8)
        r0 += r
    return {"q": q, "k": k, "v": v}
