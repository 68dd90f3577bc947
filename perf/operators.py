"""Cases and plain forms of the attention, paged-cache and cache-eviction operators.

Three operators, all with heads of 64 columns and bf16 activations:

  attention  softmax(mod(q k^T)) v over whole sequences; mod caps the scores with a tanh, adds a bias that depends on
             the distance, and masks (causal, prefix, documents)                       llmcache_attention
  chunk      new tokens (one or many per sequence) are stored in a paged cache and attend to all of it; on request the
             attention that every cached key received is recorded                      llmcache_kv_attention
  evict      per key/value head the entries that received the most attention, the newest and the first ones move to
             fresh pages, the others are dropped                                       llmcache_kv_evict

`run` computes them from elementary torch operations in 32 bits, or, with `own` set, through the library's entry points.
"""
import math

import numpy as np
import torch

own = False

DH = 64
DEV = "cuda"


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one sentence of 128 tokens through a 12-head layer, biased by a learned table over distances: latency
        _attention("attention one sentence, distance table", S=1, n=128, H=12, HK=12, causal=False, bias="table"),
        # an encoder's batch of rows of 384 tokens with several documents packed into each row, padded at the end
        _attention("attention packed documents", S=64, n=384, H=12, HK=12, causal=False, docs=4),
        # prompts of 1,024 tokens whose first 512 (a shared document) are seen in both directions
        _attention("attention prefix of 512", S=32, n=1024, H=12, HK=12, causal=True, prefix=512),
        # two long rows of packed documents with grouped heads, capped scores and a linear bias, in [sequence, head, token]
        # layout
        _attention("attention capped, long, grouped heads", S=2, n=4001, H=16, HK=4, causal=True, cap=30.0, bias="slopes",
                   docs=2, layout="heads_first"),
        # the next token of one sequence: latency
        _chunk("chunk one token", B=1, lo=517, hi=517, rows=1, H=12, HK=12, page=16),
        # the next token of 64 sequences of uneven lengths, with the received attention recorded
        _chunk("chunk next tokens of a batch, weights", B=64, lo=301, hi=4100, rows=1, H=16, HK=4, page=64, weights=True),
        # 512 tokens behind a cached prefix of 512, for 32 sequences
        _chunk("chunk of 512 behind a prefix", B=32, lo=1024, hi=1024, rows=512, H=12, HK=12, page=64),
        # the last tokens of two long prompts: their attention decides what the cache keeps
        _chunk("chunk over long caches, capped, weights", B=2, lo=17003, hi=30001, rows=250, H=16, HK=4, page=32, cap=30.0,
               bias="slopes", weights=True),
        # a batch goes on after an eviction: the entries of every head have positions of their own
        _chunk("chunk after an eviction, table", B=16, lo=513, hi=640, rows=33, H=12, HK=12, page=16, bias="table", evicted=True,
               weights=True),
        # one sequence goes back from 640 entries to 512: latency
        _evict("evict one sequence", B=1, lo=640, hi=640, HK=12, page=16, budget=512, recent=64, sinks=4),
        # a batch of uneven lengths is cut to 512 entries
        _evict("evict a batch", B=64, lo=400, hi=1500, HK=12, page=64, budget=512, recent=64, sinks=4),
        # long prompts are cut to 8,192 entries before the answer is generated
        _evict("evict long prompts", B=4, lo=20011, hi=32000, HK=16, page=64, budget=8192, recent=256, sinks=16),
    ]


def _attention(name, S, n, H, HK, causal, cap=0.0, bias="none", docs=0, prefix=0, layout="fused"):
    return dict(name=name, op="attention", S=S, n=n, H=H, HK=HK, causal=causal, cap=cap, bias=bias, docs=docs, prefix=prefix,
                layout=layout)


def _chunk(name, B, lo, hi, rows, H, HK, page, cap=0.0, bias="none", weights=False, evicted=False):
    return dict(name=name, op="chunk", B=B, lo=lo, hi=hi, rows=rows, H=H, HK=HK, page=page, cap=cap, bias=bias, weights=weights,
                evicted=evicted)


def _evict(name, B, lo, hi, HK, page, budget, recent, sinks):
    return dict(name=name, op="evict", B=B, lo=lo, hi=hi, HK=HK, page=page, budget=budget, recent=recent, sinks=sinks)


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["attention", "chunk", "evict"])
    H, HK = rng.choice([(12, 12), (16, 16), (16, 4), (12, 2), (8, 1), (6, 2)])
    cap = rng.choice([0.0, 30.0, 50.0])
    bias = rng.choice(["none", "slopes", "table"])
    if op == "attention":
        n = _spread(rng, 1, 4001)
        most = max(1, min(64, int(32 * 1024 * 1024 * 12 / (n * n * H))))
        causal = rng.random() < 0.5
        c = _attention("", S=_spread(rng, 1, most), n=n, H=H, HK=HK, causal=causal, cap=cap, bias=bias,
                       docs=rng.choice([0, 0, 3, 7]), prefix=rng.randrange(0, n + 1) if causal and rng.random() < 0.5 else 0,
                       layout=rng.choice(["fused", "heads_first"]))
    elif op == "chunk":
        rows = rng.choice([1, 1, _spread(rng, 1, 512)])
        hi = max(rows, _spread(rng, 1, 30000))
        most = max(1, min(64, int(32 * 512 * 1024 * 12 / (rows * hi * H)), int(64 * 4100 * 4 * 2 / (hi * HK))))
        c = _chunk("", B=_spread(rng, 1, most), lo=max(rows, int(hi * rng.uniform(0.1, 1.0))), hi=hi, rows=rows, H=H, HK=HK,
                   page=rng.choice([16, 32, 64, 128]), cap=cap, bias=bias, weights=rng.random() < 0.5,
                   evicted=rng.random() < 0.25)
    else:
        hi = _spread(rng, 1, 32000)
        budget = _spread(rng, 1, min(8192, hi))
        recent = rng.randrange(0, budget // 2 + 1)
        most = max(1, min(64, int(4 * 32000 * 16 / (hi * HK))))
        c = _evict("", B=_spread(rng, 1, most), lo=max(1, int(hi * rng.uniform(0.3, 1.0))), hi=hi, HK=HK,
                   page=rng.choice([16, 32, 64, 128]), budget=budget, recent=recent, sinks=rng.randrange(0, budget - recent + 1))
    del c["name"]
    return c


def _lengths(case):
    """The batch's cache lengths, from lo to hi in even steps (every seed deals the same lengths out in another order)."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    return [hi if B == 1 else lo + (hi - lo) * b // (B - 1) for b in range(B)]


def _chunks(case):
    """How many new tokens each sequence brings: `rows`, every fourth sequence about two thirds of them."""
    return [max(1, case["rows"] * 2 // 3) if b % 4 == 1 else case["rows"] for b in range(case["B"])]


def _pieces(case):
    """The lengths of the documents in a row of n tokens; the last piece is padding."""
    n, docs = case["n"], case["docs"]
    parts = [1 + 2 * i for i in range(docs)] + [1]
    got = [n * p // sum(parts) for p in parts]
    got[-2] += n - sum(got)
    return got


def work(case):
    H, HK = case.get("H", 0), case["HK"]
    if case["op"] == "attention":
        S, n = case["S"], case["n"]
        parts = _pieces(case)[:-1] if case["docs"] else [n]
        pairs, at = 0, 0
        for p in parts:
            if case["causal"]:
                pairs += p * (p + 1) // 2
                inside = max(0, min(case["prefix"] - at, p))          # keys of this piece that every query may see
                pairs += inside * (inside - 1) // 2
            else:
                pairs += p * p
            at += p
        bytes_ = S * n * (2 * H + 2 * HK) * DH * 2 + S * n * H * 4
        return {"bytes": bytes_, "flops": 4 * DH * S * H * pairs}
    lens = _lengths(case)
    if case["op"] == "chunk":
        rows = _chunks(case)
        pairs = sum(r * (n - r) + r * (r + 1) // 2 for r, n in zip(rows, lens))
        T, keys = sum(rows), sum(lens)
        # cached keys and values read, new ones read and written, queries read, outputs written, a weight per key written
        bytes_ = (keys - T) * HK * DH * 4 + 2 * T * HK * DH * 4 + T * H * (DH * 4 + 4) + keys * HK * (4 * case["weights"] + 4 * case["evicted"])
        return {"bytes": bytes_, "flops": (6 if case["weights"] else 4) * DH * H * pairs}
    kept = sum(min(n, case["budget"]) for n in lens)
    # every entry's weight and position is read; kept rows are read and written, their weights and positions written
    return {"bytes": HK * (sum(lens) * 8 + kept * (2 * DH * 4 + 12)), "flops": 0}


# --------------------------------------------------------------------------------------------------------- inputs
def _normal(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(torch.bfloat16)


def _bias(case, g):
    """(slopes, table): per head a factor of the distance, or a value for every distance up to 64, as a trained model has."""
    H = case["H"]
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=DEV) if case["bias"] == "slopes" else None
    table = torch.randn((H, 2 * 64 + 1), generator=g, device=DEV) if case["bias"] == "table" else None
    return slopes, table


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    order = np.random.RandomState(seed % (1 << 31))
    st = {"case": case}
    if case["op"] == "attention":
        S, n, H, HK = case["S"], case["n"], case["H"], case["HK"]
        if case["layout"] == "fused":                    # one matrix with the columns q | k | v, as a projection writes it
            qkv = _normal(g, S, n, H + 2 * HK, DH)
            st["q"], st["k"], st["v"] = qkv[:, :, :H], qkv[:, :, H:H + HK], qkv[:, :, H + HK:]
        else:
            st["q"], st["k"], st["v"] = (_normal(g, S, h, n, DH).transpose(1, 2) for h in (H, HK, HK))
        st["q"].mul_(2.0)                                # scores with a spread of two, as trained heads have
        st["slopes"], st["table"] = _bias(case, g)
        st["doc"] = st["prefix"] = None
        if case["docs"]:
            parts = _pieces(case)
            rows = []
            for _ in range(S):
                lens = [parts[i] for i in order.permutation(len(parts) - 1)] + [parts[-1]]
                rows.append(np.repeat(list(range(len(lens) - 1)) + [-1], lens))
            st["doc"] = torch.from_numpy(np.stack(rows).astype(np.int32)).to(DEV)
        if case["prefix"]:
            st["prefix"] = torch.full((S,), case["prefix"], dtype=torch.int32, device=DEV)
        st["out"] = torch.empty((S, n, H, DH), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.empty((S, n, H), dtype=torch.float32, device=DEV)
        if own:
            from paper_2512_16843_b200 import binding as L
            st["mods"] = L.make_score_mods(causal=case["causal"], cap=case["cap"], slopes=st["slopes"], table=st["table"],
                                           doc=st["doc"], prefix=st["prefix"])
        return st

    HK, ps, B = case["HK"], case["page"], case["B"]
    lens = [_lengths(case)[i] for i in order.permutation(B)]
    need = [-(-n // ps) for n in lens]
    fresh = -(-case["budget"] // ps) if case["op"] == "evict" else 0
    pages = sum(need) + B * fresh + 3
    ids = order.permutation(pages).astype(np.int32)      # pages in the order in which an allocator has handed them out
    table = np.full((B, max(need)), -1, dtype=np.int32)
    at = 0
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
    st["host_lens"] = lens
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    st["pages"] = torch.from_numpy(table).to(DEV)
    st["k"], st["v"] = _normal(g, pages, HK, ps, DH), _normal(g, pages, HK, ps, DH)
    # slots behind the last entry of a sequence, and pages that nobody has, were never written
    used = torch.zeros((pages, ps), dtype=torch.bool, device=DEV)
    slot = torch.arange(max(need) * ps, device=DEV).view(1, -1, ps)
    inside = slot < st["lens"].view(B, 1, 1)
    used[st["pages"].long().clamp(min=0).view(-1)] = inside.reshape(-1, ps)
    if at < pages:
        used[torch.from_numpy(ids[at:]).long().to(DEV)] = False
    for b in range(B):                                   # (a page id of -1 was clamped to 0: set that page again)
        hit = np.nonzero(table[b] == 0)[0]
        if len(hit):
            used[0] = torch.arange(ps, device=DEV) + int(hit[0]) * ps < lens[b]
    if 0 in ids[at:]:
        used[0] = False
    for t in (st["k"], st["v"]):
        t.masked_fill_(~used.view(pages, 1, ps, 1), float("nan"))
    width = max(need) * ps

    if case["op"] == "chunk":
        H = case["H"]
        rows = [min(r, n) for r, n in zip(_chunks(case), lens)]
        T = sum(rows)
        st["rows"], st["most_rows"] = rows, max(rows)
        st["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32), device=DEV)
        qkv = _normal(g, T, H + 2 * HK, DH)
        st["q"], st["k_new"], st["v_new"] = qkv[:, :H], qkv[:, H:H + HK], qkv[:, H + HK:]
        st["q"].mul_(2.0)
        st["slopes"], st["bias"] = _bias(case, g)
        st["weights"] = torch.zeros((B, HK, width), dtype=torch.float32, device=DEV) if case["weights"] else None
        st["positions"] = st["first"] = None
        if case["evicted"]:                              # entries of positions with gaps, the new rows behind them
            gaps = torch.randint(1, 4, (B, HK, width), generator=g, device=DEV)
            st["positions"] = (gaps.cumsum(-1) - 1).int()
            st["first"] = torch.tensor([3 * n for n in lens], dtype=torch.int32, device=DEV)
        st["out"] = torch.empty((T, H, DH), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.empty((T, H), dtype=torch.float32, device=DEV)
        if own:
            from paper_2512_16843_b200 import binding as L
            st["mods"] = L.make_score_mods(causal=True, cap=case["cap"], slopes=st["slopes"], table=st["bias"])
            st["cache"] = L.KVCache(st["k"], st["v"], heads=H, max_seqs=B, max_rows=T, max_len=width)
        return st

    # weights as attention leaves them: most entries got little, some a lot
    st["weights"] = torch.exp(1.5 * torch.randn((B, HK, width), generator=g, device=DEV) - 2.0)
    st["positions"] = torch.arange(width, dtype=torch.int32, device=DEV).expand(B, HK, width).contiguous()
    st["new_weights"] = torch.zeros((B, HK, case["budget"]), device=DEV)
    st["new_positions"] = torch.zeros((B, HK, case["budget"]), dtype=torch.int32, device=DEV)
    new = ids[at:at + B * fresh].reshape(B, fresh)
    st["new_pages"] = torch.from_numpy(np.ascontiguousarray(new)).to(DEV)
    st["new_lens"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    st["kept"] = torch.empty((B, HK, case["budget"]), dtype=torch.int32, device=DEV)
    if own:
        from paper_2512_16843_b200 import binding as L
        st["cache"] = L.KVCache(st["k"], st["v"], heads=HK, max_seqs=B, max_rows=B, max_len=width)
    return st


# ------------------------------------------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    if own:
        from paper_2512_16843_b200 import binding as L
        if case["op"] == "attention":
            L.llmcache_attention(st["q"], st["k"], st["v"], st["out"], mods=st["mods"], lse=st["lse"])
            return {"out": st["out"], "lse": st["lse"]}
        if case["op"] == "chunk":
            # the weights of this chunk's queries alone (decay 0): what earlier chunks gave is forgotten
            st["cache"].attention(st["q"], st["out"], cu_rows=st["cu"], lens=st["lens"], pages=st["pages"],
                                  longest=st["most_rows"], k_new=st["k_new"], v_new=st["v_new"], lse=st["lse"],
                                  mods=st["mods"], weights=st["weights"], decay=0.0, positions=st["positions"], first=st["first"])
            return _chunk_answer(st, st["out"], st["lse"])
        st["cache"].evict(lens=st["lens"], pages=st["pages"], weights=st["weights"], positions=st["positions"],
                          new_pages=st["new_pages"], new_lens=st["new_lens"], new_weights=st["new_weights"],
                          new_positions=st["new_positions"], kept=st["kept"], budget=case["budget"], recent=case["recent"],
                          sinks=case["sinks"])
        return _evict_answer(st, st["new_weights"], st["new_positions"], st["new_lens"], st["kept"])
    return {"attention": _plain_attention, "chunk": _plain_chunk, "evict": _plain_evict}[case["op"]](st)


def _chunk_answer(st, out, lse):
    answer = {"out": out, "lse": lse, "k": st["k"], "v": st["v"]}
    if st["weights"] is not None:
        answer["weights"] = st["weights"]
    if st["positions"] is not None:
        answer["positions"] = st["positions"]
    return answer


def _evict_answer(st, weights, positions, new_lens, kept):
    return {"k": st["k"], "v": st["v"], "weights": weights, "positions": positions, "new_lens": new_lens, "kept": kept}


def _softmax(s, seen):
    """(weights, log of the sum of exponentials); a row that sees nothing has weights of zero and a logarithm of -inf."""
    s = torch.where(seen, s, float("-inf"))
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = torch.exp(s - top)
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total), (top + torch.log(total)).squeeze(-1)


def _modified(s, case, slopes, table, apart):
    """The scaled products s [.., HK, G, rows, keys], capped and biased; apart [.., 1 or HK, 1, rows, keys]: key position -
    query position."""
    HK, G = case["HK"], case["H"] // case["HK"]
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    if slopes is not None:
        s = s - slopes.view(HK, G, 1, 1) * apart.abs().float()
    if table is not None:
        reach = table.shape[1] // 2
        hk, g = torch.arange(HK, device=DEV).view(HK, 1, 1, 1), torch.arange(G, device=DEV).view(G, 1, 1)
        s = s + table.view(HK, G, 2 * reach + 1)[hk, g, (apart.clamp(-reach, reach) + reach).long()]
    return s


def _plain_attention(st):
    case = st["case"]
    S, n, H, HK = case["S"], case["n"], case["H"], case["HK"]
    q = st["q"].float().view(S, n, HK, H // HK, DH).permute(0, 2, 3, 1, 4)
    k, v = (st[x].float().permute(0, 2, 1, 3).unsqueeze(2) for x in ("k", "v"))
    at = torch.arange(n, device=DEV)
    apart = at.view(1, n) - at.view(n, 1)
    s = _modified(torch.matmul(q, k.transpose(-1, -2)) * DH ** -0.5, case, st["slopes"], st["table"], apart.view(1, 1, n, n))
    seen = torch.ones((1, n, n), dtype=torch.bool, device=DEV)
    if case["causal"]:
        seen = (apart <= 0).view(1, n, n)
        if st["prefix"] is not None:
            seen = seen | (at.view(1, 1, n) < st["prefix"].view(S, 1, 1))
    if st["doc"] is not None:
        seen = seen & (st["doc"].view(S, n, 1) == st["doc"].view(S, 1, n)) & (st["doc"].view(S, 1, n) >= 0)
    p, lse = _softmax(s, seen.view(-1, 1, 1, n, n))
    out = torch.matmul(p, v)
    return {"out": out.permute(0, 3, 1, 2, 4).reshape(S, n, H, DH).to(torch.bfloat16),
            "lse": lse.permute(0, 3, 1, 2).reshape(S, n, H)}


def _slots(st, width):
    """For every sequence and slot below `width`: page, place in the page, and whether an entry is there."""
    ps = st["case"]["page"]
    j = torch.arange(width, device=DEV)
    page = st["pages"][:, j // ps].long()
    return page.clamp(min=0), (j % ps).view(1, -1).expand_as(page), (j.view(1, -1) < st["lens"].view(-1, 1)) & (page >= 0)


def _plain_chunk(st):
    case, cu, lens = st["case"], st["cu"].long(), st["lens"].long()
    B, H, HK, most = case["B"], case["H"], case["HK"], st["most_rows"]
    T, width = st["q"].shape[0], st["pages"].shape[1] * case["page"]
    count = cu[1:] - cu[:-1]
    # the new rows go to the last slots of their sequences
    row = torch.arange(T, device=DEV)
    seq = torch.searchsorted(cu[1:], row, right=True)
    slot = lens[seq] - count[seq] + row - cu[seq]
    page = st["pages"][seq, slot // case["page"]].long()
    st["k"][page, :, slot % case["page"]] = st["k_new"]
    st["v"][page, :, slot % case["page"]] = st["v_new"]
    page, place, there = _slots(st, width)
    k, v = (torch.where(there.view(B, width, 1, 1), st[x][page, :, place].float(), 0.0).transpose(1, 2).unsqueeze(2) for x in ("k", "v"))
    i = torch.arange(most, device=DEV)
    real = i.view(1, most) < count.view(B, 1)
    q = st["q"].float()[(cu[:-1].view(B, 1) + i.view(1, most)).clamp(max=T - 1)]
    q = q.view(B, most, HK, H // HK, DH).permute(0, 2, 3, 1, 4)
    behind = torch.arange(width, device=DEV).view(1, 1, 1, 1, width) - ((lens - count).view(B, 1) + i.view(1, most)).view(B, 1, 1, most, 1)
    apart = behind
    if st["positions"] is not None:
        st["positions"].transpose(1, 2)[seq, slot] = (st["first"][seq] + (row - cu[seq]).int()).view(T, 1)
        apart = st["positions"].view(B, HK, 1, 1, width) - (st["first"].view(B, 1) + i.view(1, most)).view(B, 1, 1, most, 1)
    s = _modified(torch.matmul(q, k.transpose(-1, -2)) * DH ** -0.5, case, st["slopes"], st["bias"], apart)
    seen = (behind <= 0) & there.view(B, 1, 1, 1, width) & real.view(B, 1, 1, most, 1)
    p, lse = _softmax(s, seen)
    out = torch.matmul(p, v).permute(0, 3, 1, 2, 4).reshape(B, most, H, DH)
    if st["weights"] is not None:
        st["weights"].copy_(torch.where(there.view(B, 1, width), p.sum((2, 3)), st["weights"]))
    pick = (seq, row - cu[seq])
    return _chunk_answer(st, out[pick].to(torch.bfloat16), lse.permute(0, 3, 1, 2).reshape(B, most, H)[pick])


def _plain_evict(st):
    case = st["case"]
    B, HK, budget, ps = case["B"], case["HK"], case["budget"], case["page"]
    width = st["pages"].shape[1] * ps
    page, place, there = _slots(st, width)
    w, pos = st["weights"], st["positions"]                                  # [B, HK, width]
    there = there.unsqueeze(1).expand_as(w)
    last = torch.where(there, pos, -1).amax(-1, keepdim=True)
    safe = (pos < case["sinks"]) | (pos > last - case["recent"])
    rank = torch.where(there, torch.where(safe, float("inf"), w), -1.0)
    size = max(width, budget)
    rank = torch.nn.functional.pad(rank, (0, size - width), value=-1.0)
    first = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :budget]
    new_lens = torch.minimum(st["lens"], torch.full_like(st["lens"], budget))
    real = torch.arange(budget, device=DEV).view(1, 1, budget) < new_lens.view(B, 1, 1)
    kept = torch.where(real, first, size).sort(-1).values                    # ascending, the places that stay empty last
    src = kept.clamp(max=width - 1)
    head = torch.arange(HK, device=DEV).view(1, HK, 1).expand_as(src)
    from_page, from_place = page.unsqueeze(1).expand(B, HK, width).gather(2, src), src % ps
    to = torch.arange(budget, device=DEV)
    to_page = st["new_pages"].long()[:, to // ps].unsqueeze(1).expand_as(src)
    to_place = (to % ps).view(1, 1, -1).expand_as(src)
    for t in (st["k"], st["v"]):
        moved, before = t[from_page, head, from_place], t[to_page, head, to_place]
        t[to_page, head, to_place] = torch.where(real.unsqueeze(-1), moved, before)
    new_weights, new_positions = torch.where(real, w.gather(2, src), 0.0), torch.where(real, pos.gather(2, src), 0)
    return _evict_answer(st, new_weights, new_positions, new_lens, torch.where(real, kept, -1).to(torch.int32))


# ------------------------------------------------------------------------------------------- the definition, exactly
def exact(case, seed):
    """What run() returns, from the sums themselves in 64 bits, head by head.  (Eviction moves rows and returns whole numbers.)"""
    if case["op"] == "evict":
        return None
    st = prepare(case, seed)
    G, f8 = case["H"] // case["HK"], torch.float64

    def head(q, k, v, h, qpos, kpos, visible):
        z = (q.to(f8) @ k.to(f8).T) / 8.0
        if case["cap"]:
            z = torch.tanh(z / case["cap"]) * case["cap"]
        gap = kpos[None, :] - qpos[:, None]
        if case["bias"] == "slopes":
            z = z - st["slopes"][h].to(f8) * gap.abs()
        if case["bias"] == "table":
            t = (st["table"] if case["op"] == "attention" else st["bias"])[h].to(f8)
            z = z + t[gap.clamp(-64, 64) + 64]
        z = z.masked_fill(~visible, -math.inf)
        lse = torch.logsumexp(z, 1)
        p = torch.exp(z - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
        return p @ v.to(f8), lse, p

    if case["op"] == "attention":
        S, n, H = case["S"], case["n"], case["H"]
        out, lse = torch.empty((S, n, H, DH), dtype=f8, device=DEV), torch.empty((S, n, H), dtype=f8, device=DEV)
        at = torch.arange(n, device=DEV)
        for s in range(S):
            vis = torch.ones((n, n), dtype=torch.bool, device=DEV)
            if case["causal"]:
                vis = at[None, :] <= at[:, None]
                if case["prefix"]:
                    vis = vis | (at[None, :] < case["prefix"])
            if case["docs"]:
                d = st["doc"][s]
                vis = vis & (d[None, :] == d[:, None]) & (d[None, :] >= 0)
            for h in range(H):
                out[s, :, h], lse[s, :, h], _ = head(st["q"][s, :, h], st["k"][s, :, h // G], st["v"][s, :, h // G], h, at, at, vis)
        return {"out": out, "lse": lse}

    T, H, ps = st["q"].shape[0], case["H"], case["page"]
    out, lse = torch.empty((T, H, DH), dtype=f8, device=DEV), torch.empty((T, H), dtype=f8, device=DEV)
    weights = torch.zeros((case["B"], case["HK"], st["pages"].shape[1] * ps), dtype=f8, device=DEV)
    t0 = 0
    for b, (n, r) in enumerate(zip(st["host_lens"], st["rows"])):
        slot = torch.arange(n, device=DEV)
        vis = slot[None, :] <= slot[n - r:, None]
        kpos, qpos = slot, slot[n - r:]
        page, place = st["pages"][b].long()[slot // ps], slot % ps
        for hk in range(case["HK"]):
            k = torch.cat([st["k"][page, hk, place][:n - r], st["k_new"][t0:t0 + r, hk]])
            v = torch.cat([st["v"][page, hk, place][:n - r], st["v_new"][t0:t0 + r, hk]])
            if case["evicted"]:
                qpos = int(st["first"][b]) + slot[:r]
                kpos = torch.cat([st["positions"][b, hk, :n - r].long(), qpos])
            for h in range(hk * G, hk * G + G):
                out[t0:t0 + r, h], lse[t0:t0 + r, h], p = head(st["q"][t0:t0 + r, h], k, v, h, qpos, kpos, vis)
                weights[b, hk, :n] += p.sum(0)
        t0 += r
    answer = {"out": out, "lse": lse, "k": None, "v": None, "positions": None}
    if case["weights"]:
        answer["weights"] = weights
    return answer
