"""The attention block's operators as programs call them: int4 projections with
an unmerged adapter, the latent cache's writes, latent attention for single
tokens (absorbed, with and without a prefix that the batch shares) and for
prompts (expanded), and the moves of cache pages.

With ``own`` false the operators are computed in plain torch; with ``own`` true
by the library. Weights and tokens have the distributions of the seeded test
inputs: uniform int4 codes, scales near 0.02 / sqrt(255 / 12), LoRA A ~ N(0, 1/r)
and B ~ N(0, 0.01), unit-variance activations.

Shapes: hidden sizes and token counts of the 35B-class layer (2048) and the 8B
tier (4096), a 3.1k-token prompt, generic head layouts and lengths.
"""

import math

import torch

own = False

EPS = 1e-6  # of the RMS norm, as everywhere in the library

WIDE = {"Dc": 512, "Dr": 64, "Dn": 128, "Dv": 128}
SMALL = {"Dc": 256, "Dr": 32, "Dn": 64, "Dv": 64}


def listed():
    return [
        # query projection of one decode token of the 35B-class layer (32 heads of 192): launch latency and 7 MB of weights
        {"name": "linear_t1", "kind": "linear", "T": 1, "n_in": 2048, "n_out": 6144, "r": 16, "out": "f16"},
        # output projection of a small decode batch of the 8B tier, fp32 for the residual
        {"name": "linear_t13", "kind": "linear", "T": 13, "n_in": 4096, "n_out": 4096, "r": 16, "out": "f32"},
        # a prompt's tokens through a projection, an odd number of outputs
        {"name": "linear_t1555", "kind": "linear", "T": 1555, "n_in": 4096, "n_out": 5001, "r": 16, "out": "f32"},
        # the new token of 16 decoding sequences, and a whole 3.1k-token prompt, into the cache
        dict(WIDE, name="append_t16", kind="append", T=16, seqs=16, H=32, page=64, reach=4000),
        dict(WIDE, name="append_t3100", kind="append", T=3100, seqs=3, H=32, page=64, reach=3100),
        # one decode token over a short context: the smallest attention call
        dict(WIDE, name="decode_b1", kind="decode", B=1, H=32, most=700, ragged=False, page=64, prefix=0),
        # a serving batch of ragged lengths up to 16k, with padding rows
        dict(WIDE, name="decode_b48_ragged", kind="decode", B=48, H=32, most=16384, ragged=True, page=64, prefix=0),
        # samples that share a long prompt
        dict(WIDE, name="decode_shared", kind="decode", B=32, H=64, most=500, ragged=True, page=32, prefix=12000),
        # a whole prompt, and a ragged batch of chunks on top of cached context
        dict(WIDE, name="prefill_t3100", kind="prefill", B=1, H=32, T=3100, most=3100, page=64),
        dict(SMALL, name="prefill_chunks", kind="prefill", B=5, H=8, T=777, most=5000, page=16),
        # forking 24 sequences (their last, partly filled pages) over 24 layers; closing the gaps of a large cache
        {"name": "pages_fork", "kind": "pages", "layers": 24, "pages": 128, "moves": 24, "page": 64, "row": 576, "entries": 600},
        {"name": "pages_compact", "kind": "pages", "layers": 8, "pages": 900, "moves": 400, "page": 64, "row": 576, "entries": 2000},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "append", "decode", "decode", "decode", "prefill", "prefill", "pages"])
    if kind == "linear":
        return {"kind": kind, "T": _log_int(rng, 1, 1555), "n_in": 64 * _log_int(rng, 8, 64), "n_out": _log_int(rng, 64, 6144),
                "r": rng.choice([0, 4, 8, 16, 16, 64]), "out": rng.choice(["f16", "f32"])}
    if kind == "pages":
        moves = _log_int(rng, 1, 300)
        return {"kind": kind, "layers": _log_int(rng, 1, 12), "pages": 2 * moves + rng.randint(1, 100), "moves": moves,
                "page": rng.choice([16, 32, 64]), "row": rng.choice([160, 288, 320, 576]), "entries": _log_int(rng, 3, 2000)}
    dims = dict(rng.choice([WIDE, WIDE, SMALL, {"Dc": 512, "Dr": 64, "Dn": 64, "Dv": 128}, {"Dc": 128, "Dr": 32, "Dn": 64, "Dv": 64},
                            {"Dc": 256, "Dr": 64, "Dn": 128, "Dv": 64}]), page=rng.choice([16, 32, 64, 128]))
    H = rng.choice([1, 5, 8, 20, 32, 64])
    if kind == "append":
        seqs = _log_int(rng, 1, 40)
        return dict(dims, kind=kind, H=min(H, 32), T=max(seqs, _log_int(rng, 1, 3100)), seqs=seqs, reach=_log_int(rng, 3100, 9000))
    if kind == "decode":
        if rng.random() < 0.35:
            return dict(dims, kind=kind, B=_log_int(rng, 2, 32), H=H, most=_log_int(rng, 1, 1000), ragged=True,
                        prefix=_log_int(rng, 100, 12000))
        B = _log_int(rng, 1, 64)
        H = rng.choice([H, 128]) if B <= 16 else H
        return dict(dims, kind=kind, B=B, H=H, most=_log_int(rng, 1, min(40000, 400000 // B)), ragged=rng.random() < 0.7, prefix=0)
    B = _log_int(rng, 1, 6)
    T = _log_int(rng, B, 2000)
    return dict(dims, kind=kind, B=B, H=min(H, 32), T=T, most=T + _log_int(rng, 1, 4000))


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


def _lengths(c):
    """Own context lengths of a decode batch: the case's, so that every seed does the same work."""
    B, most = c["B"], c["most"]
    if not c["ragged"]:
        return [most] * B
    n = [max(1, int(round(most * ((i * 0.6180339887 + 0.37) % 1.0)))) for i in range(B)]
    n[0] = most
    for i in range(5, B, 20):
        n[i] = 0  # a padding row of the batch
    return n


def _chunks(c):
    """(query tokens, context tokens with them) of each sequence of a prefill batch."""
    B, T = c["B"], c["T"]
    share = [1.0 + (i * 0.6180339887) % 1.0 for i in range(B)]
    q = [max(1, int(T * s / sum(share))) for s in share]
    q[0] = max(1, q[0] + T - sum(q))
    return [(n, n + int((c["most"] - n) * ((i * 0.381966 + 1.0) % 1.0 if i else 1.0)) if c["most"] > n else n) for i, n in enumerate(q)]


def _paged(c, seed, lengths, slack=0):
    """A cache whose pages lie in any order, and the page table of the sequences."""
    P = c["page"]
    per = [-(-n // P) for n in lengths]
    n_pages = sum(per) + slack + 1
    order = torch.randperm(n_pages, generator=_host(seed, 1)).to(torch.int32)
    table = torch.zeros(len(lengths), max(1, max(per)), dtype=torch.int32)
    at = 0
    for b, k in enumerate(per):
        table[b, :k] = order[at:at + k]
        at += k
    pages = _normal(_gen(seed, 2), (n_pages, P, c["Dc"] + c["Dr"]))
    return pages, table.cuda(), order[at:].cuda()


def _scale(c):
    return 1.0 / math.sqrt(c["Dn"] + c["Dr"])


def prepare(case, seed):
    c = case
    s = {"case": c}
    if c["kind"] == "linear":
        g = _gen(seed, 3)
        n_in, n_out, r = c["n_in"], c["n_out"], c["r"]
        s["q"] = torch.randint(0, 256, (n_out, n_in // 2), generator=g, device="cuda", dtype=torch.uint8)
        scale = (torch.rand(n_out, n_in // 64, generator=g, device="cuda") * 0.2 + 0.9) * (0.02 / math.sqrt(255 / 12))
        u = torch.rand(n_out, n_in // 64, generator=g, device="cuda") * 2 - 1
        s["sz"] = torch.stack([scale, -7.5 * scale + 0.005 * u], -1).half()
        s["x"] = _normal(g, (c["T"], n_in))
        s["a"] = _normal(g, (r, n_in), 1.0 / r) if r else None
        s["b"] = _normal(g, (n_out, r), 0.01) if r else None
        return s
    if c["kind"] == "pages":
        g = _gen(seed, 4)
        n, m = c["pages"], c["moves"]
        s["pages"] = _normal(g, (c["layers"], n, c["page"], c["row"]))
        # no page is both a source and a target, as in a fork's and a compaction's plan
        order = torch.randperm(n, generator=_host(seed, 5))
        s["pairs"] = torch.stack([order[:m], order[m:2 * m]], -1).to(torch.int32).cuda()
        remap = torch.arange(n, dtype=torch.int32)
        remap[order[:m]] = order[m:2 * m].to(torch.int32)
        s["remap"] = remap.cuda()
        # page tables: entries of all sequences, -1 where a sequence has no page yet
        table = torch.randint(-1, n, (c["entries"],), generator=_host(seed, 6)).to(torch.int32)
        s["table"] = table.cuda()
        s["table_out"] = torch.zeros_like(s["table"])
        return s
    H, Dc, Dr, Dn, Dv = (c[k] for k in ("H", "Dc", "Dr", "Dn", "Dv"))
    g = _gen(seed, 7)
    if c["kind"] == "append":
        T, S = c["T"], c["seqs"]
        per = [T // S + (1 if i < T % S else 0) for i in range(S)]
        ends = [min(c["reach"], per[i] + (i * 977) % max(1, c["reach"] - per[i] + 1)) for i in range(S)]
        s["pages"], s["table"], _ = _paged(c, seed, ends)
        s["seq"] = _i32([i for i in range(S) for _ in range(per[i])])
        s["pos"] = _i32([ends[i] - per[i] + k for i in range(S) for k in range(per[i])])
        s["kv"] = _normal(g, (T, Dc + Dr), dtype=torch.float32)
        s["gamma"] = (1.0 + 0.1 * torch.randn(Dc, generator=g, device="cuda")).half()
        angle = torch.arange(c["reach"], dtype=torch.float64, device="cuda")[:, None] * (
            10000.0 ** (-torch.arange(0, Dr, 2, dtype=torch.float64, device="cuda") / Dr))[None]
        s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        s["qin"] = _normal(g, (T, H, Dn + Dr))
        s["qout"] = torch.zeros_like(s["qin"])
        return s
    s["w"] = _normal(g, (H, Dn + Dv, Dc), 1.0 / math.sqrt(Dc))
    if c["kind"] == "decode":
        own_len = _lengths(c)
        need = -(-c["prefix"] // c["page"])
        s["pages"], s["table"], rest = _paged(c, seed, own_len, slack=need)
        s["prefix"] = rest[:need].contiguous() if need else None
        s["len"] = _i32(own_len)
        s["qin"] = _normal(g, (c["B"], H, Dn + Dr), 1.5)
        return s
    both = _chunks(c)
    s["pages"], s["table"], _ = _paged(c, seed, [k for _, k in both])
    qs, ks = [0], [0]
    for q, k in both:
        qs.append(qs[-1] + q)
        ks.append(ks[-1] + k)
    s["q_start"], s["kv_start"], s["both"] = _i32(qs), _i32(ks), both
    s["qin"] = _normal(g, (qs[-1], H, Dn + Dr), 1.5)
    return s


# ---- one pass -----------------------------------------------------------------


def _codes(s):
    q = s["q"]
    return torch.stack([q & 15, q >> 4], -1).reshape(q.shape[0], -1)


def _plain_linear(s):
    c = s["case"]
    sz = s["sz"].float()
    w = _codes(s).float().view(c["n_out"], -1, 64) * sz[..., :1] + sz[..., 1:]
    x = s["x"].float()
    y = x @ w.view(c["n_out"], -1).t()
    if c["r"]:
        y = y + 2.0 * ((x @ s["a"].float().t()) @ s["b"].float().t())
    return y.half() if c["out"] == "f16" else y


def _rotated(v, cs):
    a, b = v[..., 0::2], v[..., 1::2]
    return torch.stack([a * cs[..., 0] - b * cs[..., 1], a * cs[..., 1] + b * cs[..., 0]], -1).flatten(-2)


def _plain_append(s):
    c = s["case"]
    Dc, Dn, P = c["Dc"], c["Dn"], c["page"]
    kv, pos, seq = s["kv"], s["pos"].long(), s["seq"].long()
    lat = kv[:, :Dc]
    lat = lat * torch.rsqrt(lat.square().mean(-1, keepdim=True) + EPS) * s["gamma"].float()
    cs = s["rope"][pos]
    row = torch.cat([lat, _rotated(kv[:, Dc:], cs)], -1).half()
    s["pages"][s["table"][seq, pos // P].long(), pos % P] = row
    q = s["qin"].float()
    s["qout"].copy_(torch.cat([q[..., :Dn], _rotated(q[..., Dn:], cs[:, None])], -1))
    return s["pages"], s["qout"]


def _weighted(score, keep, values):
    """softmax over the kept scores times the values; rows that keep nothing give zeros."""
    score = score.masked_fill(~keep, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    return (p @ values) / p.sum(-1, keepdim=True).clamp_min(1e-30)


def _plain_decode(s):
    c = s["case"]
    B, H, Dc, Dn, P = c["B"], c["H"], c["Dc"], c["Dn"], c["page"]
    w, q = s["w"].float(), s["qin"].float()
    lat_q = torch.matmul(q[..., :Dn].transpose(0, 1), w[:, :Dn]).transpose(0, 1)
    full = torch.cat([lat_q, q[..., Dn:]], -1) * _scale(c)
    rows = s["pages"][s["table"].long()].view(B, -1, Dc + c["Dr"]).float()
    score = full @ rows.transpose(1, 2)
    keep = torch.arange(rows.shape[1], device="cuda") < s["len"][:, None]
    rows = torch.where(keep[..., None], rows, torch.zeros_like(rows))
    keep = keep[:, None].expand_as(score)
    if s["prefix"] is None:
        o = _weighted(score, keep, rows[..., :Dc])
    else:
        shared = s["pages"][s["prefix"].long()].view(-1, Dc + c["Dr"])[:c["prefix"]].float()
        first = full @ shared.t()
        top = torch.maximum(first.amax(-1, keepdim=True), score.masked_fill(~keep, -math.inf).amax(-1, keepdim=True))
        p1, p2 = torch.exp(first - top), torch.exp(score.masked_fill(~keep, -math.inf) - top)
        o = (p1 @ shared[:, :Dc] + p2 @ rows[..., :Dc]) / (p1.sum(-1, keepdim=True) + p2.sum(-1, keepdim=True))
    return torch.matmul(o.transpose(0, 1), w[:, Dn:].transpose(1, 2)).transpose(0, 1).half().contiguous()


def _plain_prefill(s):
    c = s["case"]
    B, H, Dc, Dn, P = c["B"], c["H"], c["Dc"], c["Dn"], c["page"]
    w, q = s["w"].float(), s["qin"].float()
    rows = s["pages"][s["table"].long()].view(B, -1, Dc + c["Dr"]).float()
    L = rows.shape[1]
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
    keep = torch.arange(L, device="cuda") <= torch.where(real, last, torch.full_like(last, -1))[..., None]
    o = _weighted(score, keep[:, None], heads[..., Dn:])
    return o.transpose(1, 2)[real].half()


def _plain_pages(s):
    src, dst = s["pairs"].long().unbind(-1)
    s["pages"][:, dst] = s["pages"][:, src]
    t = s["table"].long()
    s["table_out"].copy_(torch.where(t >= 0, s["remap"][t.clamp_min(0)], s["table"]))
    return s["pages"], s["table_out"]


def _kept(s):
    """What a program makes once and keeps beside its weights and cache: descriptions, workspaces, outputs."""
    if "kept" in s:
        return s["kept"]
    from paper_2609_18063_amd import binding as B
    c = s["case"]
    k = s["kept"] = {"B": B, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}

    def ws(n):
        return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")

    if c["kind"] == "linear":
        k["proj"] = B.MoeProj(*(t.data_ptr() if t is not None else None for t in (s["q"], s["sz"], s["a"], s["b"])))
        k["y"] = torch.empty(c["T"], c["n_out"], dtype=torch.float16 if c["out"] == "f16" else torch.float32, device="cuda")
        k["ws"] = ws(B.linear_workspace_bytes(c["n_out"], c["n_in"], c["r"], c["T"]))
    elif c["kind"] != "pages":
        k["spec"] = B.make_latent_spec(c["H"], c["Dc"], c["Dr"], c["Dn"], c["Dv"], c["page"], _scale(c))
        k["cache"] = B.latent_cache(s["pages"], s["table"])
        if c["kind"] == "decode":
            k["ws"] = ws(B.latent_decode_workspace_bytes(k["spec"], c["B"], c["most"], c["prefix"]))
        elif c["kind"] == "prefill":
            k["kv_total"], k["max_q"] = sum(n for _, n in s["both"]), max(n for n, _ in s["both"])
            k["ws"] = ws(B.latent_prefill_workspace_bytes(k["spec"], c["B"], k["kv_total"]))
        if c["kind"] != "append":
            k["out"] = torch.empty(s["qin"].shape[0], c["H"], c["Dv"], dtype=torch.float16, device="cuda")
    return k


def _own(s):
    c, k = s["case"], _kept(s)
    B = k["B"]
    if c["kind"] == "linear":
        B.linear_int4(k["proj"], c["n_out"], c["n_in"], c["r"], 2.0, s["x"], k["y"], k["ws"])
        return k["y"]
    if c["kind"] == "append":
        B.latent_append(k["spec"], k["cache"], s["kv"], s["gamma"], s["rope"], s["seq"], s["pos"], k["status"], q=s["qin"],
                        q_out=s["qout"])
        return s["pages"], s["qout"]
    if c["kind"] == "decode":
        B.latent_decode(k["spec"], k["cache"], s["w"], s["qin"], s["len"], c["most"], k["out"], k["status"], k["ws"],
                        prefix=s["prefix"], prefix_len=c["prefix"])
        return k["out"]
    if c["kind"] == "prefill":
        B.latent_prefill(k["spec"], k["cache"], s["w"], s["qin"], s["q_start"], s["kv_start"], k["kv_total"], k["max_q"], k["out"],
                         k["status"], k["ws"])
        return k["out"]
    B.page_copy(s["pages"], s["pairs"], k["status"])
    B.page_remap(s["table"], s["remap"], s["table_out"], k["status"])
    return s["pages"], s["table_out"]


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "append": _plain_append, "decode": _plain_decode, "prefill": _plain_prefill,
            "pages": _plain_pages}[state["case"]["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------


def work(case):
    c = case
    if c["kind"] == "linear":
        T, i, o, r = c["T"], c["n_in"], c["n_out"], c["r"]
        return {"bytes": o * i // 2 + o * i // 16 + 2 * r * (i + o) + 2 * T * i + T * o * (2 if c["out"] == "f16" else 4),
                "flops": 2 * T * (o * i + r * (i + o))}
    if c["kind"] == "pages":
        return {"bytes": 2 * c["layers"] * c["moves"] * c["page"] * c["row"] * 2 + 8 * c["moves"] + 8 * c["entries"], "flops": 0}
    H, Dc, Dr, Dn, Dv = (c[k] for k in ("H", "Dc", "Dr", "Dn", "Dv"))
    if c["kind"] == "append":
        return {"bytes": c["T"] * ((Dc + Dr) * 6 + H * (Dn + Dr) * 4 + 8), "flops": c["T"] * (4 * Dc + 3 * (H + 1) * Dr)}
    weights = 2 * H * (Dn + Dv) * Dc
    if c["kind"] == "decode":
        B, own_len = c["B"], sum(_lengths(c))
        return {"bytes": (own_len + c["prefix"]) * (Dc + Dr) * 2 + weights + 2 * B * H * (Dn + Dr + Dv),
                "flops": 2 * H * (2 * Dc + Dr) * (own_len + B * c["prefix"]) + 2 * B * H * Dc * (Dn + Dv)}
    both = _chunks(c)
    pairs = sum(q * (k - q) + q * (q + 1) // 2 for q, k in both)
    T, kv = sum(q for q, _ in both), sum(k for _, k in both)
    return {"bytes": kv * (Dc + Dr) * 2 + weights + 2 * T * H * (Dn + Dr + Dv),
            "flops": 2 * H * (Dn + Dr + Dv) * pairs + 2 * kv * H * (Dn + Dv) * Dc}


# ---- the same from the definitions, in 64 bits --------------------------------------


def exact(case, seed):
    c, s = case, prepare(case, seed)
    f64 = torch.float64
    if c["kind"] == "linear":
        lo, hi = (s["q"] & 15).to(f64), (s["q"] >> 4).to(f64)
        w = torch.empty(c["n_out"], c["n_in"], dtype=f64, device="cuda")
        w[:, 0::2], w[:, 1::2] = lo, hi
        sz = s["sz"].to(f64).repeat_interleave(64, 1)
        w = w * sz[..., 0] + sz[..., 1]
        if c["r"]:
            w = w + 2.0 * (s["b"].to(f64) @ s["a"].to(f64))
        return torch.mm(s["x"].to(f64), w.t().contiguous())
    if c["kind"] == "pages":
        was = s["pages"].clone()
        for a, b in s["pairs"].tolist():
            s["pages"][:, b] = was[:, a]
        remap = s["remap"].tolist()
        return s["pages"].to(f64), torch.tensor([remap[t] if t >= 0 else t for t in s["table"].tolist()], dtype=torch.int32)
    H, Dc, Dr, Dn, P = c["H"], c["Dc"], c["Dr"], c["Dn"], c["page"]
    if c["kind"] == "append":
        pages = s["pages"].to(f64)
        kv, pos, seq = s["kv"].to(f64), s["pos"].long(), s["seq"].long()
        at = s["rope"].to(f64)[pos]
        turn = torch.complex(at[..., 0], at[..., 1])

        def rot(v):
            z = torch.view_as_complex(v.reshape(*v.shape[:-1], -1, 2).contiguous())
            return torch.view_as_real(z * (turn if v.dim() == 2 else turn[:, None])).flatten(-2)

        norm = torch.linalg.vector_norm(kv[:, :Dc], dim=-1, keepdim=True).square() / Dc + EPS
        row = torch.cat([kv[:, :Dc] / norm.sqrt() * s["gamma"].to(f64), rot(kv[:, Dc:])], -1)
        pages.view(-1, Dc + Dr)[s["table"][seq, pos // P].long() * P + pos % P] = row
        q = s["qin"].to(f64)
        return pages, torch.cat([q[..., :Dn], rot(q[..., Dn:])], -1)
    w, q = s["w"].to(f64), s["qin"].to(f64)

    def context(ids, n):
        return s["pages"].index_select(0, ids.long()).reshape(-1, Dc + Dr)[:n].to(f64)

    def attend(qs, rows, seen):
        """qs [n, H, Dn + Dr] over the rows, row i seeing the first seen[i] of them."""
        out = torch.zeros(qs.shape[0], H, c["Dv"], dtype=f64, device="cuda")
        if not len(rows):
            return out
        mask = torch.arange(len(rows), device="cuda")[None] >= seen[:, None]
        for h in range(H):
            k = torch.cat([rows[:, :Dc] @ w[h, :Dn].t().contiguous(), rows[:, Dc:]], -1)
            a = (qs[:, h] @ k.t().contiguous()) / math.sqrt(Dn + Dr)
            out[:, h] = torch.softmax(a.masked_fill(mask, -math.inf), -1) @ (rows[:, :Dc] @ w[h, Dn:].t().contiguous())
        return out

    if c["kind"] == "decode":
        if sum(_lengths(c)) + c["B"] * c["prefix"] > 500_000 or c["B"] * H > 2048:
            # (expanded keys for every head and sequence: too long here, so through the latents)
            return _exact_latent(c, s, w, q, context)
        first = context(s["prefix"], c["prefix"]) if s["prefix"] is not None else context(s["table"][0, :0], 0)
        got = []
        for b, n in enumerate(_lengths(c)):
            rows = torch.cat([first, context(s["table"][b], n)])
            got.append(attend(q[b:b + 1], rows, torch.tensor([len(rows)], device="cuda")))
        return torch.cat(got)
    got, at = [], 0
    for b, (n, k) in enumerate(s["both"]):
        got.append(attend(q[at:at + n], context(s["table"][b], k), torch.arange(k - n, k, device="cuda") + 1))
        at += n
    return torch.cat(got)


def _exact_latent(c, s, w, q, context):
    Dc, Dn = c["Dc"], c["Dn"]
    first = context(s["prefix"], c["prefix"]) if s["prefix"] is not None else None
    got = []
    for b, n in enumerate(_lengths(c)):
        rows = context(s["table"][b], n)
        if first is not None:
            rows = torch.cat([first, rows])
        if not len(rows):
            got.append(torch.zeros(c["H"], c["Dv"], dtype=torch.float64, device="cuda"))
            continue
        lat = torch.cat([(q[b, :, None, :Dn] @ w[:, :Dn])[:, 0], q[b, :, Dn:]], -1)
        p = torch.softmax(lat @ rows.t().contiguous() / math.sqrt(Dn + c["Dr"]), -1)
        got.append((w[:, Dn:] @ (p @ rows[:, :Dc])[..., None])[..., 0])
    return torch.stack(got)
