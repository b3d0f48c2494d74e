"""The 4-bit latent cache's operators as programs call them: tokens written into the cache (normed, rotated,
quantised) and read back, latent attention over it for single tokens and for prompts, with and without the sums
of each cached token's attention weights, and the eviction of tokens by those sums.

With ``own`` false the operators are computed in plain torch; with ``own`` true by the library.

A cached row has Dc + Dr values in groups of 64 (the last group is the rotated key, Dr values). A group holds 4-bit
codes q, a step s and a middle z (fp16), and stands for s (q - 8) + z. A page of P tokens is, in bytes, the latents'
codes [P][Dc / 2] (two a byte, the first in the low half), the keys' codes [P][Dr / 2], the steps [G][P] and the
middles [G][P].

Shapes: the dimensions and lengths of the fp16 cache's own cases (a 3.1k-token prompt, ragged serving batches,
chunks on cached context), generic head layouts and lengths, and budgets of a fraction of them.
"""

import math

import torch

own = False

EPS = 1e-6  # of the RMS norm, as everywhere in the library

WIDE = {"Dc": 512, "Dr": 64, "Dn": 128, "Dv": 128}
SMALL = {"Dc": 256, "Dr": 32, "Dn": 64, "Dv": 64}


def listed():
    return [
        # the new token of 16 decoding sequences, and a whole 3.1k-token prompt, into the cache and read back
        dict(WIDE, name="append_t16", kind="append", T=16, seqs=16, H=32, page=64, reach=4000),
        dict(WIDE, name="append_t3100", kind="append", T=3100, seqs=3, H=32, page=64, reach=3100),
        # one decode token over a short context: the smallest attention call
        dict(WIDE, name="decode_b1", kind="decode", B=1, H=32, most=700, ragged=False, page=64, sums=False, steps=0),
        # a serving batch of ragged lengths up to 16k, with padding rows
        dict(WIDE, name="decode_b48_ragged", kind="decode", B=48, H=32, most=16384, ragged=True, page=64, sums=False, steps=0),
        # many heads: the products bound it rather than the cache
        dict(WIDE, name="decode_h128", kind="decode", B=8, H=128, most=12000, ragged=True, page=128, sums=False, steps=0),
        # a batch that keeps its tokens' weights for a later eviction, and one long sequence that does
        dict(SMALL, name="decode_sums_b20", kind="decode", B=20, H=20, most=3001, ragged=True, page=16, sums=True, steps=1000),
        dict(WIDE, name="decode_sums_long", kind="decode", B=1, H=16, most=40000, ragged=False, page=64, sums=True, steps=900),
        # a whole prompt; a ragged batch of chunks on top of cached context; one long chunk that keeps its weights
        dict(WIDE, name="prefill_t3100", kind="prefill", B=1, H=32, T=3100, most=3100, page=64, sums=False, steps=0),
        dict(SMALL, name="prefill_chunks", kind="prefill", B=5, H=8, T=777, most=5000, page=16, sums=False, steps=0),
        dict(WIDE, name="prefill_sums", kind="prefill", B=2, H=16, T=1555, most=2600, page=32, sums=True, steps=2000),
        # one layer of one sequence back to its budget, and a stack of 24 layers on 8 sequences
        dict(SMALL, name="evict_one", kind="evict", layers=1, seqs=1, most=1100, ragged=False, budget=500, sinks=4, recent=100, page=16),
        dict(WIDE, name="evict_stack", kind="evict", layers=24, seqs=8, most=6000, ragged=True, budget=2000, sinks=4, recent=256, page=64),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["append", "decode", "decode", "decode", "prefill", "prefill", "evict", "evict"])
    dims = dict(rng.choice([WIDE, WIDE, SMALL, {"Dc": 512, "Dr": 64, "Dn": 64, "Dv": 128}, {"Dc": 128, "Dr": 32, "Dn": 64, "Dv": 64},
                            {"Dc": 256, "Dr": 64, "Dn": 128, "Dv": 64}]), page=rng.choice([16, 32, 64, 128]))
    H = rng.choice([1, 5, 8, 20, 32, 64])
    sums = rng.random() < 0.5
    steps = _log_int(rng, 300, 3000) if sums else 0
    if kind == "append":
        seqs = _log_int(rng, 1, 40)
        return dict(dims, kind=kind, H=min(H, 32), T=max(seqs, _log_int(rng, 1, 3100)), seqs=seqs, reach=_log_int(rng, 3100, 9000))
    if kind == "decode":
        B = _log_int(rng, 1, 64)
        H = rng.choice([H, 128]) if B <= 16 else H
        most = _log_int(rng, 1, min(40000, 380000 // B))
        # (weights of a few tokens alone are no sums that a program evicts by)
        return dict(dims, kind=kind, B=B, H=H, most=max(most, 500) if sums else most, ragged=rng.random() < 0.7, sums=sums, steps=steps)
    if kind == "prefill":
        B = _log_int(rng, 1, 6)
        T = _log_int(rng, B, 2000)
        H = max(H, 8) if sums else H
        return dict(dims, kind=kind, B=B, H=min(H, 32), T=T, most=T + _log_int(rng, 600 if sums else 1, 4000), sums=sums, steps=steps)
    layers, seqs = _log_int(rng, 1, 24), _log_int(rng, 1, 16)
    most = _log_int(rng, 40, min(30000, 900000 // (layers * seqs)))
    budget = max(20, int(most * rng.uniform(0.1, 0.8)))
    return dict(dims, kind=kind, layers=layers, seqs=seqs, most=most, ragged=rng.random() < 0.7, budget=budget,
                sinks=rng.randint(0, 4), recent=rng.randint(1, budget // 2))


# ---- inputs -------------------------------------------------------------------


def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + stream) % (1 << 62))
    return g


def _host(seed, stream):
    g = torch.Generator()
    g.manual_seed((seed * 1_000_003 + stream) % (1 << 62))
    return g


def _normal(g, shape, std=1.0, dtype=torch.float16):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _lengths(c, n):
    """Context lengths of a batch of n: the case's, so that every seed does the same work."""
    most = c["most"]
    if not c["ragged"]:
        return [most] * n
    k = [max(1, int(round(most * ((i * 0.6180339887 + 0.37) % 1.0)))) for i in range(n)]
    k[0] = most
    for i in range(5, n, 20):
        k[i] = 0  # a padding row of the batch
    return k


def _chunks(c):
    """(query tokens, context tokens with them) of each sequence of a prefill batch."""
    B, T = c["B"], c["T"]
    share = [1.0 + (i * 0.6180339887) % 1.0 for i in range(B)]
    q = [max(1, int(T * s / sum(share))) for s in share]
    q[0] = max(1, q[0] + T - sum(q))
    return [(n, n + int((c["most"] - n) * ((i * 0.381966 + 1.0) % 1.0 if i else 1.0)) if c["most"] > n else n) for i, n in enumerate(q)]


def _groups(c):
    return c["Dc"] // 64 + 1


def _row_bytes(c):
    return (c["Dc"] + c["Dr"]) // 2 + 4 * _groups(c)


def _views(c, pages):
    """The parts of pages uint8 [n, page bytes]: latents' codes, keys' codes, steps, middles."""
    P, G = c["page"], _groups(c)
    a, b = P * c["Dc"] // 2, P * (c["Dc"] + c["Dr"]) // 2
    n = pages.shape[0]
    half = pages[:, b:].view(torch.float16).view(n, 2, G, P)
    return pages[:, :a].view(n, P, -1), pages[:, a:b].view(n, P, -1), half[:, 0], half[:, 1]


def _quantised(v, c):
    """Rows v [n, Dc + Dr] (fp32 or fp64) as (codes uint8 [n, Dc + Dr], s fp16 [n, G], z fp16 [n, G])."""
    parts = []
    for x in (v[:, :c["Dc"]].reshape(-1, c["Dc"] // 64, 64), v[:, None, c["Dc"]:]):
        lo, hi = x.amin(-1), x.amax(-1)
        s = ((hi - lo) / 15).float().half()
        z = (lo + 8 * s.to(v.dtype)).float().half()
        step = s.to(v.dtype)[..., None]
        q = torch.round((x - z.to(v.dtype)[..., None]) / torch.where(step == 0, torch.ones_like(step), step)) + 8
        parts.append((q.clamp(0, 15).to(torch.uint8).flatten(1), s, z))
    return tuple(torch.cat(p, 1) for p in zip(*parts))


def _store(c, pages, page, at, rows):
    """Rows into the pages `page` at the places `at` of them."""
    lat, key, step, mid = _views(c, pages)
    q, s, z = _quantised(rows, c)
    q = q[:, 0::2] | (q[:, 1::2] << 4)
    lat[page, at], key[page, at] = q[:, :c["Dc"] // 2], q[:, c["Dc"] // 2:]
    step[page, :, at], mid[page, :, at] = s, z


def _table(c, seed, lengths, slack=0):
    """Page tables of sequences whose pages lie in any order, the number of pages, and the pages left over."""
    P = c["page"]
    per = [-(-n // P) for n in lengths]
    n_pages = sum(per) + slack + 1
    order = torch.randperm(n_pages, generator=_host(seed, 1)).to(torch.int32)
    table = torch.zeros(len(lengths), max(1, max(per)), dtype=torch.int32)
    at = 0
    for b, k in enumerate(per):
        table[b, :k] = order[at:at + k]
        at += k
    return table.cuda(), n_pages, order[at:].cuda()


def _filled(c, seed, n_pages):
    """Pages full of quantised unit-variance rows."""
    pages = torch.zeros(n_pages, c["page"] * _row_bytes(c), dtype=torch.uint8, device="cuda")
    g, n = _gen(seed, 2), n_pages * c["page"]
    for i in range(0, n, 1 << 16):
        k = torch.arange(i, min(n, i + (1 << 16)), device="cuda")
        _store(c, pages, k // c["page"], k % c["page"], _normal(g, (len(k), c["Dc"] + c["Dr"]), dtype=torch.float32))
    return pages


def _history(c, seed, rows, lengths, width):
    """Sums that all heads of each sequence's own tokens, and of `steps` that have been evicted since, left on it."""
    s = torch.exp(torch.randn(rows, width, generator=_gen(seed, 8), device="cuda"))
    n = torch.tensor(lengths, device="cuda")[:, None]
    s = s * (torch.arange(width, device="cuda") < n)
    return s * ((n + c["steps"]) * c["H"] / s.sum(-1, keepdim=True).clamp_min(1.0))


def _scale(c):
    return 1.0 / math.sqrt(c["Dn"] + c["Dr"])


def prepare(case, seed):
    c = case
    s = {"case": c}
    Dc, Dr, Dn, Dv = (c[k] for k in ("Dc", "Dr", "Dn", "Dv"))
    g = _gen(seed, 7)
    if c["kind"] == "evict":
        n = _lengths(c, c["seqs"])
        need = -(-c["budget"] // c["page"])
        s["table"], n_pages, rest = _table(c, seed, n, slack=need * c["seqs"])
        # rows are moved, not computed with: any bytes
        s["pages"] = torch.randint(0, 256, (c["layers"], n_pages, c["page"] * _row_bytes(c)), generator=g, device="cuda", dtype=torch.uint8)
        s["to"] = rest[:need * c["seqs"]].view(c["seqs"], need).contiguous()
        s["len"], s["n"] = _i32(n), n
        # sums over a few orders of magnitude; those of tokens that little attends to are alike, and some zero
        v = torch.exp(1.5 * torch.randn(c["layers"], c["seqs"], c["most"], generator=g, device="cuda"))
        s["sums"] = torch.where(v < 0.5, torch.floor(v * 8) / 8, v).contiguous()
        s["sums_out"] = torch.zeros_like(s["sums"])
        s["keep"] = torch.zeros(c["layers"], c["seqs"], c["budget"], dtype=torch.int32, device="cuda")
        return s
    H = c["H"]
    if c["kind"] == "append":
        T, S = c["T"], c["seqs"]
        per = [T // S + (1 if i < T % S else 0) for i in range(S)]
        ends = [min(c["reach"], per[i] + (i * 977) % max(1, c["reach"] - per[i] + 1)) for i in range(S)]
        s["table"], n_pages, _ = _table(c, seed, ends)
        s["pages"] = _filled(c, seed, n_pages)
        s["seq"] = _i32([i for i in range(S) for _ in range(per[i])])
        slot = [ends[i] - per[i] + k for i in range(S) for k in range(per[i])]
        # (positions run ahead of places in sequences that have been evicted from)
        s["slot"], s["pos"] = _i32(slot), _i32([k + 500 for k in slot])
        s["kv"] = _normal(g, (T, Dc + Dr), dtype=torch.float32)
        s["gamma"] = (1.0 + 0.1 * torch.randn(Dc, generator=g, device="cuda")).half()
        angle = torch.arange(c["reach"] + 500, dtype=torch.float64, device="cuda")[:, None] * (
            10000.0 ** (-torch.arange(0, Dr, 2, dtype=torch.float64, device="cuda") / Dr))[None]
        s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        s["qin"] = _normal(g, (T, H, Dn + Dr))
        s["qout"] = torch.zeros_like(s["qin"])
        s["rows"] = torch.zeros(T, Dc + Dr, dtype=torch.float16, device="cuda")
        return s
    s["w"] = _normal(g, (H, Dn + Dv, Dc), 1.0 / math.sqrt(Dc))
    if c["kind"] == "decode":
        n = _lengths(c, c["B"])
        s["len"], rows, seen = _i32(n), c["B"], n
    else:
        both = _chunks(c)
        n, qs, ks = [k for _, k in both], [0], [0]
        for q, k in both:
            qs.append(qs[-1] + q)
            ks.append(ks[-1] + k)
        s["q_start"], s["kv_start"], s["both"] = _i32(qs), _i32(ks), both
        rows, seen = qs[-1], [k - q for q, k in both]
    s["table"], n_pages, _ = _table(c, seed, n)
    s["pages"] = _filled(c, seed, n_pages)
    s["qin"] = _normal(g, (rows, H, Dn + Dr), 1.5)
    s["sums"] = _history(c, seed, c["B"], seen, max(n)) if c["sums"] else None
    return s


# ---- one pass -----------------------------------------------------------------


def _values(c, pages, ids):
    """fp32 rows [..., P, Dc + Dr] of the pages `ids`."""
    lat, key, step, mid = _views(c, pages)
    out = []
    for codes, a, b in ((lat, 0, _groups(c) - 1), (key, _groups(c) - 1, _groups(c))):
        q = codes[ids]
        q = torch.stack([q & 15, q >> 4], -1).flatten(-2).float() - 8
        q = q.unflatten(-1, (b - a, -1))
        s, z = (v[:, a:b][ids].transpose(-1, -2).float()[..., None] for v in (step, mid))
        out.append((q * s + z).flatten(-2))
    return torch.cat(out, -1)


def _rotated(v, cs):
    a, b = v[..., 0::2], v[..., 1::2]
    return torch.stack([a * cs[..., 0] - b * cs[..., 1], a * cs[..., 1] + b * cs[..., 0]], -1).flatten(-2)


def _plain_append(s):
    c = s["case"]
    Dc, Dn, P = c["Dc"], c["Dn"], c["page"]
    # in 64 bits: a code next to a border goes one way or the other by the last bit
    kv, slot, seq = s["kv"].double(), s["slot"].long(), s["seq"].long()
    lat = kv[:, :Dc]
    lat = lat / torch.sqrt(lat.square().mean(-1, keepdim=True) + EPS) * s["gamma"].double()
    cs = s["rope"][s["pos"].long()]
    page, at = s["table"][seq, slot // P].long(), slot % P
    _store(c, s["pages"], page, at, torch.cat([lat, _rotated(kv[:, Dc:], cs.double())], -1))
    q = s["qin"].float()
    s["qout"].copy_(torch.cat([q[..., :Dn], _rotated(q[..., Dn:], cs[:, None])], -1))
    lat, key, step, mid = _views(c, s["pages"])
    parts = []
    for codes, a, b in ((lat, 0, _groups(c) - 1), (key, _groups(c) - 1, _groups(c))):
        v = codes[page, at]
        v = torch.stack([v & 15, v >> 4], -1).flatten(-2).float().unflatten(-1, (b - a, -1)) - 8
        parts.append((v * step[page, :, at][:, a:b, None].float() + mid[page, :, at][:, a:b, None].float()).flatten(-2))
    s["rows"].copy_(torch.cat(parts, -1))
    return s["rows"], s["qout"]


def _softmax(score, keep):
    """Softmax over the kept scores; rows that keep nothing are zero."""
    score = score.masked_fill(~keep, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    return p / p.sum(-1, keepdim=True).clamp_min(1e-30)


def _plain_decode(s):
    c = s["case"]
    B, Dc, Dn = c["B"], c["Dc"], c["Dn"]
    w, q = s["w"].float(), s["qin"].float()
    lat_q = torch.matmul(q[..., :Dn].transpose(0, 1), w[:, :Dn]).transpose(0, 1)
    full = torch.cat([lat_q, q[..., Dn:]], -1) * _scale(c)
    rows = _values(c, s["pages"], s["table"].long()).view(B, -1, Dc + c["Dr"])
    score = full @ rows.transpose(1, 2)
    keep = torch.arange(rows.shape[1], device="cuda") < s["len"][:, None]
    p = _softmax(score, keep[:, None].expand_as(score))
    o = p @ rows[..., :Dc]
    out = torch.matmul(o.transpose(0, 1), w[:, Dn:].transpose(1, 2)).transpose(0, 1).half().contiguous()
    if s["sums"] is None:
        return out
    s["sums"] += p.sum(1)[:, :s["sums"].shape[1]]
    return out, s["sums"]


def _plain_prefill(s):
    c = s["case"]
    B, H, Dc, Dn = c["B"], c["H"], c["Dc"], c["Dn"]
    w, q = s["w"].float(), s["qin"].float()
    rows = _values(c, s["pages"], s["table"].long()).view(B, -1, Dc + c["Dr"])
    heads = torch.matmul(rows[:, None, :, :Dc], w.transpose(1, 2))
    k = torch.cat([heads[..., :Dn], rows[:, None, :, Dc:].expand(-1, H, -1, -1)], -1)
    n_q = s["q_start"][1:] - s["q_start"][:-1]
    n_kv = s["kv_start"][1:] - s["kv_start"][:-1]
    i = torch.arange(max(n for n, _ in s["both"]), device="cuda")
    real = i < n_q[:, None]
    padded = torch.zeros(B, len(i), H, q.shape[-1], device="cuda")
    padded[real] = q
    score = torch.matmul(padded.transpose(1, 2) * _scale(c), k.transpose(2, 3))
    last = (n_kv - n_q)[:, None] + i
    keep = torch.arange(rows.shape[1], device="cuda") <= torch.where(real, last, torch.full_like(last, -1))[..., None]
    p = _softmax(score, keep[:, None])
    out = (p @ heads[..., Dn:]).transpose(1, 2)[real].half()
    if s["sums"] is None:
        return out
    s["sums"] += p.sum((1, 2))[:, :s["sums"].shape[1]]
    return out, s["sums"]


def _plain_evict(s):
    c = s["case"]
    P, K, n = c["page"], c["budget"], s["len"][None, :, None]
    at = torch.arange(c["most"], device="cuda")
    fixed = (at < c["sinks"]) | (at >= n - c["recent"])
    rank = torch.where(fixed, math.inf, s["sums"]).masked_fill(at >= n, -math.inf)
    # (a stable sort: of equal sums the first stay)
    first = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :K]
    stays = torch.arange(K, device="cuda") < n.clamp_max(K)
    if first.shape[-1] < K:
        first = torch.nn.functional.pad(first, (0, K - first.shape[-1]), value=c["most"])
    first = torch.where(stays, first, c["most"]).sort(-1).values
    s["keep"].copy_(torch.where(stays, first, -1))
    from_slot = first.clamp_max(c["most"] - 1)
    moved = torch.gather(s["sums"], 2, from_slot) * stays
    s["sums_out"].zero_()
    w = min(K, c["most"])
    s["sums_out"][..., :w] = moved[..., :w]
    # every kept row: from its page and place to the next place of its sequence's new pages
    layer, seq, i = stays.expand_as(first).nonzero(as_tuple=True)
    slot = first[layer, seq, i]
    a, b = s["table"][seq, slot // P].long(), s["to"][seq, i // P].long()
    flat = s["pages"].view(-1, s["pages"].shape[-1])
    n_pages = s["pages"].shape[1]
    for v in _views(c, flat)[:2]:
        v[layer * n_pages + b, i % P] = v[layer * n_pages + a, slot % P]
    for v in _views(c, flat)[2:]:
        v = v.view(torch.int16)
        v[layer * n_pages + b, :, i % P] = v[layer * n_pages + a, :, slot % P]
    return s["keep"], s["sums_out"], s["pages"]


def _kept(s):
    """What a program makes once and keeps beside its weights and cache: descriptions, workspaces, outputs."""
    if "kept" in s:
        return s["kept"]
    from paper_2609_18063_amd import binding as B
    c = s["case"]
    k = s["kept"] = {"B": B, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    k["spec"] = B.make_latent_spec(c.get("H", 1), c["Dc"], c["Dr"], c["Dn"], c["Dv"], c["page"], _scale(c))
    if c["kind"] != "evict":
        k["cache"] = B.latent4_cache(k["spec"], s["pages"], s["table"])
    n = 0
    if c["kind"] == "decode":
        n = B.latent4_decode_workspace_bytes(k["spec"], c["B"], c["most"], sums=c["sums"])
    elif c["kind"] == "prefill":
        k["kv_total"], k["max_q"] = sum(n for _, n in s["both"]), max(n for n, _ in s["both"])
        n = B.latent4_prefill_workspace_bytes(k["spec"], s["qin"].shape[0], c["B"], k["kv_total"], sums=c["sums"])
    k["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    if "qin" in s:
        k["out"] = torch.empty(s["qin"].shape[0], c["H"], c["Dv"], dtype=torch.float16, device="cuda")
    return k


def _own(s):
    c, k = s["case"], _kept(s)
    B = k["B"]
    if c["kind"] == "append":
        B.latent4_append(k["spec"], k["cache"], s["kv"], s["gamma"], s["rope"], s["seq"], s["slot"], s["pos"], k["status"],
                         q=s["qin"], q_out=s["qout"])
        B.latent4_read(k["spec"], k["cache"], s["seq"], s["slot"], s["rows"], k["status"])
        return s["rows"], s["qout"]
    if c["kind"] == "decode":
        B.latent4_decode(k["spec"], k["cache"], s["w"], s["qin"], s["len"], c["most"], k["out"], k["status"], k["ws"], sums=s["sums"])
    elif c["kind"] == "prefill":
        B.latent4_prefill(k["spec"], k["cache"], s["w"], s["qin"], s["q_start"], s["kv_start"], k["kv_total"], k["max_q"], k["out"],
                          k["status"], k["ws"], sums=s["sums"])
    else:
        B.evict_select(s["sums"], s["len"], c["budget"], c["sinks"], c["recent"], s["keep"], s["sums_out"], k["status"])
        B.latent4_move(k["spec"], s["pages"], s["table"], s["keep"], s["to"], k["status"])
        return s["keep"], s["sums_out"], s["pages"]
    return k["out"] if s["sums"] is None else (k["out"], s["sums"])


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "decode": _plain_decode, "prefill": _plain_prefill, "evict": _plain_evict}[state["case"]["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------


def work(case):
    c = case
    row = _row_bytes(c)
    if c["kind"] == "evict":
        n = _lengths(c, c["seqs"])
        kept = sum(min(k, c["budget"]) for k in n)
        return {"bytes": c["layers"] * (8 * sum(n) + kept * (4 + 2 * row)), "flops": 0}
    H, Dc, Dr, Dn, Dv = (c[k] for k in ("H", "Dc", "Dr", "Dn", "Dv"))
    if c["kind"] == "append":
        return {"bytes": c["T"] * ((Dc + Dr) * 6 + 2 * row + H * (Dn + Dr) * 4 + 12), "flops": c["T"] * (12 * Dc + 3 * (H + 4) * Dr)}
    weights = 2 * H * (Dn + Dv) * Dc
    if c["kind"] == "decode":
        B, n = c["B"], sum(_lengths(c, c["B"]))
        return {"bytes": n * (row + (8 if c["sums"] else 0)) + weights + 2 * B * H * (Dn + Dr + Dv),
                "flops": 2 * H * (2 * Dc + Dr) * n + 2 * B * H * Dc * (Dn + Dv)}
    both = _chunks(c)
    pairs = sum(q * (k - q) + q * (q + 1) // 2 for q, k in both)
    T, kv = sum(q for q, _ in both), sum(k for _, k in both)
    return {"bytes": kv * (row + (8 if c["sums"] else 0)) + weights + 2 * T * H * (Dn + Dr + Dv),
            "flops": 2 * H * (Dn + Dr + Dv) * pairs + 2 * kv * H * (Dn + Dv) * Dc}


# ---- the same from the definitions, in 64 bits --------------------------------------


def _row64(c, s, b, n):
    """The first n tokens of sequence b, in 64 bits: [n, Dc + Dr]."""
    P, Dc, Dr, G = c["page"], c["Dc"], c["Dr"], _groups(c)
    raw = s["pages"].index_select(0, s["table"][b].long())
    a, e = P * Dc // 2, P * (Dc + Dr) // 2
    out = torch.empty(raw.shape[0], P, Dc + Dr, dtype=torch.float64, device="cuda")
    for lo, hi, first in ((0, a, 0), (a, e, Dc)):
        code = raw[:, lo:hi].reshape(raw.shape[0], P, -1)
        last = first + 2 * code.shape[-1]
        out[:, :, first:last:2], out[:, :, first + 1:last:2] = (code % 16).double(), torch.div(code, 16, rounding_mode="floor").double()
    tail = raw[:, e:].contiguous().view(torch.float16).double().reshape(raw.shape[0], 2 * G, P)
    for i in range(G):
        cut = slice(64 * i, 64 * i + 64 if i < G - 1 else Dc + Dr)
        out[:, :, cut] = (out[:, :, cut] - 8.0) * tail[:, i, :, None] + tail[:, G + i, :, None]
    return out.view(-1, Dc + Dr)[:n]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    f64 = torch.float64
    if c["kind"] == "evict":
        return _exact_evict(c, s)
    H, Dc, Dr, Dn = c["H"], c["Dc"], c["Dr"], c["Dn"]
    if c["kind"] == "append":
        kv = s["kv"].to(f64)
        at = s["rope"].to(f64)[s["pos"].long()]
        turn = torch.complex(at[..., 0], at[..., 1])

        def rot(v):
            z = torch.view_as_complex(v.reshape(*v.shape[:-1], -1, 2).contiguous())
            return torch.view_as_real(z * (turn if v.dim() == 2 else turn[:, None])).flatten(-2)

        norm = torch.linalg.vector_norm(kv[:, :Dc], dim=-1, keepdim=True).square() / Dc + EPS
        row = torch.cat([kv[:, :Dc] / norm.sqrt() * s["gamma"].to(f64), rot(kv[:, Dc:])], -1)
        for lo in range(0, Dc + Dr, 64):
            x = row[:, lo:lo + 64]
            low, high = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
            step = ((high - low) / 15.0).half().to(f64)
            mid = (low + 8.0 * step).half().to(f64)
            row[:, lo:lo + 64] = torch.clamp(torch.round((x - mid) / step), -8.0, 7.0) * step + mid
        q = s["qin"].to(f64)
        return row, torch.cat([q[..., :Dn], rot(q[..., Dn:])], -1)
    w, q = s["w"].to(f64), s["qin"].to(f64)

    def attend(b, qs, n, seen):
        """qs [k, H, Dn + Dr] over the n tokens of sequence b, row i seeing the first seen[i] (None: all) of them: the
        outputs, and each token's weights over all rows and heads."""
        out = torch.zeros(qs.shape[0], H, c["Dv"], dtype=f64, device="cuda")
        total = torch.zeros(n, dtype=f64, device="cuda")
        if not n:
            return out, total
        rows = _row64(c, s, b, n)
        if qs.shape[0] == 1:
            # (one row: through the latents, all heads at a time)
            lat = torch.cat([(qs[0, :, None, :Dn] @ w[:, :Dn])[:, 0], qs[0, :, Dn:]], -1)
            p = torch.softmax(lat @ rows.t().contiguous() / math.sqrt(Dn + Dr), -1)
            return (w[:, Dn:] @ (p @ rows[:, :Dc])[..., None])[None, ..., 0], p.sum(0)
        mask = torch.arange(n, device="cuda")[None] >= seen[:, None]
        for h in range(H):
            k = torch.cat([rows[:, :Dc] @ w[h, :Dn].t().contiguous(), rows[:, Dc:]], -1)
            p = torch.softmax(((qs[:, h] @ k.t().contiguous()) / math.sqrt(Dn + Dr)).masked_fill(mask, -math.inf), -1)
            out[:, h] = p @ (rows[:, :Dc] @ w[h, Dn:].t().contiguous())
            total += p.sum(0)
        return out, total

    if c["kind"] == "decode":
        todo = [(b, b, b + 1, n) for b, n in enumerate(_lengths(c, c["B"]))]
    else:
        start = s["q_start"].tolist()
        todo = [(b, start[b], start[b + 1], k) for b, (_, k) in enumerate(s["both"])]
    got, sums = [], None if s["sums"] is None else s["sums"].to(f64)
    for b, lo, hi, n in todo:
        o, total = attend(b, q[lo:hi], n, torch.arange(n - (hi - lo), n, device="cuda") + 1)
        got.append(o)
        if sums is not None:
            sums[b, :n] += total
    return torch.cat(got) if sums is None else (torch.cat(got), sums)


def _exact_evict(c, s):
    P, K, half = c["page"], c["budget"], c["page"] * (c["Dc"] + c["Dr"]) // 2
    keep = torch.full((c["layers"], c["seqs"], K), -1, dtype=torch.int32)
    out = torch.zeros(c["layers"], c["seqs"], c["most"], dtype=torch.float64)
    weight, to, pages = s["sums"].double().cpu().numpy(), s["to"].long(), s["pages"]
    for layer in range(c["layers"]):
        for b, n in enumerate(s["n"]):
            tail = range(max(0, n - c["recent"]), n)
            chosen = {j for j in tail} | set(range(min(c["sinks"], n)))
            middle = [j for j in range(min(c["sinks"], n), max(0, n - c["recent"]))]
            row = weight[layer, b].tolist()
            middle.sort(key=lambda j: (-row[j], j))
            chosen = sorted(chosen | set(middle[:max(0, min(n, K) - len(chosen))]))
            keep[layer, b, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
            out[layer, b, :len(chosen)] = torch.tensor([row[j] for j in chosen], dtype=torch.float64)
            if not chosen:
                continue
            j, i = torch.tensor(chosen, device="cuda"), torch.arange(len(chosen), device="cuda")
            was, now = pages[layer].index_select(0, s["table"][b, j // P].long()), to[b, i // P]
            for lo, hi in ((0, P * c["Dc"] // 2), (P * c["Dc"] // 2, half)):
                rows = pages[layer, :, lo:hi].unflatten(1, (P, -1))
                rows[now, i % P] = was[:, lo:hi].unflatten(1, (P, -1))[i, j % P]
            tail = pages[layer, :, half:].unflatten(1, (-1, P, 2))
            tail[now, :, i % P] = was[:, half:].unflatten(1, (-1, P, 2))[i, :, j % P]
    return keep, out, pages
