"""The attention block in front of a MoE layer: int4 projections with their adapters, latent attention and its
paged cache, through the C ABI.

The paper's decoder runs attention before each MoE layer (§3.2, Motivation), its 8B tier latent attention (§2),
with adapters on the attention projections (§3.3). A block is, on the residual r:

    x = rmsnorm(r);  q = W_q x;  (c, k_r) = W_kv x;  the token's cache row and the rotated query (latent_append);
    o = latent attention of q over the sequence's rows;  r = r + W_o o.

:class:`LatentCache` holds the pages of all layers and one page table for them; pages are counted by the
library's pool, so that sequences fork (a full page is shared, the last, partly filled one copied), end and move
together without the device being read back.
"""

import torch

from . import binding as B


class LatentCache:
    """Pages of every layer and the page tables of up to ``n_seqs`` sequences (the same page ids in every layer).
    Tables and pages change on the current stream, which has to be the one that reads them."""

    def __init__(self, spec, n_layers, n_pages, n_seqs, max_tokens):
        P = spec.page_tokens
        self.spec, self.n_layers, self.max_pages = spec, n_layers, -(-max_tokens // P)
        self.pages = torch.zeros(n_layers, n_pages, P, spec.d_latent + spec.d_rope, dtype=torch.float16, device="cuda")
        self.table = torch.full((n_seqs, self.max_pages), -1, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.layers = [B.latent_cache(self.pages[n], self.table) for n in range(n_layers)]
        self.pool = B.PagePool(n_pages, P)
        self.ids = [None] * n_seqs       # host copy of each sequence's pages; None: no such sequence
        self.tokens = [0] * n_seqs

    def _publish(self, seq):
        row = torch.full((self.max_pages,), -1, dtype=torch.int32)
        row[:len(self.ids[seq])] = torch.tensor(self.ids[seq], dtype=torch.int32)
        self.table[seq].copy_(row)

    def start(self):
        """A free sequence number, with no tokens."""
        if None not in self.ids:
            raise ValueError("all %d sequences are in use" % len(self.ids))
        seq = self.ids.index(None)
        self.ids[seq], self.tokens[seq] = [], 0
        return seq

    def _live(self, seq):
        if not 0 <= seq < len(self.ids) or self.ids[seq] is None:
            raise ValueError("there is no sequence %d" % seq)

    def grow(self, seq, n):
        """Room for ``n`` more tokens of ``seq``; returns the position of the first."""
        self._live(seq)
        if n < 0:
            raise ValueError("sequence %d cannot grow by %d tokens" % (seq, n))
        at = self.tokens[seq]
        need = -(-(at + n) // self.spec.page_tokens) - len(self.ids[seq])
        if len(self.ids[seq]) + need > self.max_pages:
            raise ValueError("sequence %d: %d tokens are more than its table holds" % (seq, at + n))
        if need > 0:
            self.ids[seq] = self.ids[seq] + self.pool.alloc(need)
            self._publish(seq)
        self.tokens[seq] = at + n
        return at

    def fork(self, seq):
        """A new sequence with ``seq``'s tokens: its full pages shared, the last one copied."""
        self._live(seq)
        new = self.start()
        try:
            self.ids[new], pairs = self.pool.fork(self.ids[seq], self.tokens[seq])
        except B.MoeError:
            self.ids[new] = None
            raise
        self.tokens[new] = self.tokens[seq]
        if pairs:
            B.page_copy(self.pages, torch.tensor(pairs, dtype=torch.int32).cuda(), self.status)
        self._publish(new)
        return new

    def end(self, seq):
        """Give ``seq``'s pages back. Its table row is cleared: a call that still names it flags
        ``MOE_STATUS_BAD_PAGE`` and touches no page that another sequence has by then."""
        self._live(seq)
        self.pool.free(self.ids[seq])
        self.ids[seq], self.tokens[seq] = None, 0
        self.table[seq].fill_(-1)

    def compact(self):
        """Move the live pages to the lowest ids, in the tables too; returns the number of pages moved."""
        moves, remap = self.pool.compact()
        if len(moves):
            B.page_copy(self.pages, torch.from_numpy(moves.copy()).cuda(), self.status)
            B.page_remap(self.table, torch.from_numpy(remap).cuda(), self.table, self.status)
            self.ids = [None if s is None else [int(remap[i]) for i in s] for s in self.ids]
        return len(moves)

    def close(self):
        self.pool.close()


def rope_table(max_pos, d_rope, base=10000.0):
    """fp32 ``[max_pos, d_rope / 2, 2]`` of (cos, sin) on the GPU, the angles in 64 bits."""
    angle = torch.arange(max_pos, dtype=torch.float64)[:, None] * (
        base ** (-torch.arange(0, d_rope, 2, dtype=torch.float64) / d_rope))[None]
    return torch.stack([angle.cos(), angle.sin()], -1).float().cuda()


class LatentBlock:
    """One layer's weights: ``q``, ``kv``, ``o`` (MoeProj of device pointers), ``w_kvb`` fp16 ``[H, d_nope + d_v,
    d_latent]`` and ``gamma`` fp16 ``[d_latent]``; ``rank`` and ``lora_scale`` of the adapters. ``keep``: what
    the projections point into."""

    def __init__(self, q, kv, o, w_kvb, gamma, rank=0, lora_scale=0.0, keep=None):
        self.q, self.kv, self.o, self.w_kvb, self.gamma = q, kv, o, w_kvb, gamma
        self.rank, self.lora_scale, self.keep = rank, lora_scale, keep


class LatentAttention:
    """The blocks of a stack on one cache, with buffers for up to ``max_rows`` tokens a call."""

    def __init__(self, d, spec, blocks, cache, rope, max_rows=1):
        s = self.spec = spec
        self.d, self.blocks, self.cache, self.rope, self.max_rows = d, blocks, cache, rope, max_rows
        self.max_len = cache.max_pages * s.page_tokens
        self.n_q, self.n_kv, self.n_o = s.heads * (s.d_nope + s.d_rope), s.d_latent + s.d_rope, s.heads * s.d_v
        dev = "cuda"
        self.qb = torch.empty(max_rows, s.heads, s.d_nope + s.d_rope, dtype=torch.float16, device=dev)
        self.kvb = torch.empty(max_rows, self.n_kv, dtype=torch.float32, device=dev)
        self.ob = torch.empty(max_rows, s.heads, s.d_v, dtype=torch.float16, device=dev)
        rank = max(b.rank for b in blocks)
        shapes = ((self.n_q, d), (self.n_kv, d), (d, self.n_o))
        self.ws = self._ws(max(B.linear_workspace_bytes(o, i, rank, max_rows) for o, i in shapes))
        rows = min(max_rows, len(cache.ids))
        self.ws_decode = self._ws(B.latent_decode_workspace_bytes(s, rows, self.max_len))
        self.ws_prefill = None

    @staticmethod
    def _ws(n):
        return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")

    def _project(self, n, x, seq, pos):
        b, T = self.blocks[n], x.shape[0]
        q, kv = self.qb[:T], self.kvb[:T]
        B.linear_int4(b.q, self.n_q, self.d, b.rank, b.lora_scale, x, q.view(T, -1), self.ws)
        B.linear_int4(b.kv, self.n_kv, self.d, b.rank, b.lora_scale, x, kv, self.ws)
        B.latent_append(self.spec, self.cache.layers[n], kv, b.gamma, self.rope, seq, pos, self.cache.status, q=q, q_out=q)
        return q

    def _out(self, n, r):
        b, T = self.blocks[n], r.shape[0]
        B.linear_int4(b.o, self.d, self.n_o, b.rank, b.lora_scale, self.ob[:T].view(T, -1), r, self.ws, add=True)

    def decode(self, n, x, r, seq, pos, kv_len, max_len=None):
        """Layer ``n`` for one token of each of the first ``len(x)`` table rows: ``x`` fp16 ``[B, d]`` (the normed
        residual), ``r`` fp32 ``[B, d]`` in and out; ``seq``, ``pos`` and ``kv_len`` (the token among them) int32
        ``[B]`` on the GPU. ``max_len``: a bound on kv_len (the table's, if none). Capturable."""
        q = self._project(n, x, seq, pos)
        B.latent_decode(self.spec, self.cache.layers[n], self.blocks[n].w_kvb, q, kv_len,
                        self.max_len if max_len is None else max_len, self.ob[:x.shape[0]], self.cache.status,
                        self.ws_decode)
        self._out(n, r)

    def prefill(self, n, x, r, seq, pos, q_start, kv_start, kv_total, max_q):
        """Layer ``n`` for chunks of prompts: the ragged batch of ``moe_latent_prefill``, sequence b in table row b.
        Rows of padding behind the last sequence (``seq`` -1) keep their ``r``. Eager only: its workspace grows with
        ``kv_total``, ``H (d_nope + d_v)`` halves a token, for one layer at a time."""
        q = self._project(n, x, seq, pos)
        need = B.latent_prefill_workspace_bytes(self.spec, q_start.numel() - 1, kv_total)
        if self.ws_prefill is None or self.ws_prefill.nbytes < need:
            self.ws_prefill = self._ws(need)
        o = self.ob[:x.shape[0]].zero_()                 # (rows of padding are not written, and W_o 0 = 0)
        B.latent_prefill(self.spec, self.cache.layers[n], self.blocks[n].w_kvb, q, q_start, kv_start, kv_total, max_q, o,
                         self.cache.status, self.ws_prefill)
        self._out(n, r)


class ChainAttention:
    """The blocks as a decode chain's attention: one sequence, one token a step. ``pos`` and ``kv_len`` live on
    the GPU, so that captured steps replay at any token; ``at`` sets them before a token. What the calls find wrong
    is in ``cache.status``, not in the chain's."""

    def __init__(self, d, spec, blocks, n_tokens):
        self.cache = LatentCache(spec, len(blocks), -(-n_tokens // spec.page_tokens), 1, n_tokens)
        self.cache.grow(self.cache.start(), n_tokens)
        self.attn = LatentAttention(d, spec, blocks, self.cache, rope_table(n_tokens, spec.d_rope))
        self.n_tokens = n_tokens
        self.seq, self.pos = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
        self.kv_len = torch.ones(1, dtype=torch.int32, device="cuda")

    def at(self, t):
        if not 0 <= t < self.n_tokens:
            raise ValueError("token %d: the cache has room for %d" % (t, self.n_tokens))
        self.pos.fill_(t)
        self.kv_len.fill_(t + 1)

    def step(self, n, x, r):
        """r = r + attention of layer ``n`` on x = rmsnorm(r); x is overwritten with rmsnorm of the new r."""
        B.rmsnorm_f16(r, x)
        self.attn.decode(n, x, r, self.seq, self.pos, self.kv_len)
        B.rmsnorm_f16(r, x)

