"""A LlamaGen-shaped decoder around the ADSA attention, with random weights (Section 5 integrates the method with
LlamaGen; trained weights are not available, so this shell has the decoder's shapes and data flow and nothing of
its quality).

What runs where: the attention, the KV cache, the rotary embedding, the normalisations, the gated activation and
the sampling are libadsa calls; the projections, the residual additions and the embedding look-up are torch
(cuBLAS GEMMs: plain library contractions); the token ids go to a pinned host buffer as they are drawn, one
asynchronous copy per step (Section 4.2: generated ids are kept on the host until the image is decoded).

One block: x -> RMSNorm -> q, k, v projections -> 2-D RoPE on q and k -> ADSA layer-step -> output projection
(+ residual) -> RMSNorm -> gate/up projection -> silu(gate) * up -> down projection (+ residual).  Classifier-free
guidance doubles the batch: rows [0, n_images) are conditional, rows [n_images, 2 n_images) unconditional; both
halves are fed the same sampled ids.

SharedPromptShell is the same decoder for several images of ONE prompt, nothing evicted: the condition's rows are kept
once per guidance half in a paged cache and every decode step sweeps them once for all images, the new rows are rotated
on their way into the cache, the residual additions and normalisations are one call each, and a whole decode step is one
CUDA graph (every length and position it needs lies on the device).
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as B


@dataclass(frozen=True)
class ShellConfig:
    n_layers: int
    dim: int
    n_heads: int
    ffn_hidden: int
    vocab: int = 16384
    n_text: int = 120
    grid_h: int = 32
    grid_w: int = 32
    n_images: int = 16
    budget_fraction: float = 0.5
    cfg_scale: float = 7.5
    top_k: int = 2000
    temperature: float = 1.0
    norm_eps: float = 1e-5
    sandwich_norm: bool = False         # SharedPromptShell: a normalisation after each block too, before its residual addition

    @property
    def head_dim(self) -> int:
        return self.dim // self.n_heads

    @property
    def batch(self) -> int:
        return 2 * self.n_images

    @property
    def capacity(self) -> int:
        return int(self.budget_fraction * (self.n_text + self.grid_h * self.grid_w) + 1e-9)


# the three decoder sizes the benchmark configurations are shaped after (hidden sizes: 2/3 * 4 * dim rounded up to 256)
SHAPES = {
    "B": dict(n_layers=12, dim=768, n_heads=12, ffn_hidden=2048),
    "L": dict(n_layers=24, dim=1024, n_heads=16, ffn_hidden=2816),
    "XL": dict(n_layers=36, dim=1280, n_heads=20, ffn_hidden=3584),
}


class _Decoder:
    """Random weights and the buffers of a decode step; what both shells share."""

    def __init__(self, cfg: ShellConfig, seed: int, device: str):
        self.cfg, self.dev = cfg, torch.device(device)
        g = torch.Generator(device=self.dev).manual_seed(seed)
        bf = dict(dtype=torch.bfloat16, device=self.dev)

        def w(*shape):
            return (0.02 * torch.randn(*shape, generator=g, device=self.dev)).to(torch.bfloat16)

        L, D, Hd, V = cfg.n_layers, cfg.dim, cfg.ffn_hidden, cfg.vocab
        self.tok_emb = w(V, D)
        self.wqkv_t = w(L, 3, D, D)         # q, k, v projections, stored transposed: [layer][which][in][out]
        self.wo = w(L, D, D)
        self.w13 = w(L, 2 * Hd, D)          # gate and up projections side by side
        self.w2 = w(L, D, Hd)
        self.norm1 = torch.ones(L, D, **bf)
        self.norm2 = torch.ones(L, D, **bf)
        self.norm_f = torch.ones(D, **bf)
        self.head = w(V, D)
        Bt, H, d = cfg.batch, cfg.n_heads, cfg.head_dim
        self.qkv = torch.empty(3, Bt, H, d, **bf)    # q, k, v of a decode step, each dense [batch, heads, head_dim]
        self.q, self.k, self.v = self.qkv[0], self.qkv[1], self.qkv[2]
        self.o = torch.empty(Bt, H, d, **bf)
        self.h = torch.empty(Bt, D, **bf)
        self.gu = torch.empty(Bt, 2 * Hd, **bf)
        self.act = torch.empty(Bt, Hd, **bf)
        self.logits = torch.empty(Bt, V, **bf)
        self.tokens = torch.zeros(cfg.n_images, dtype=torch.int32, device=self.dev)
        self.ids_host = torch.zeros(cfg.grid_h * cfg.grid_w, cfg.n_images, dtype=torch.int32).pin_memory()
        # the random numbers of the whole generation, drawn once (the sampling call takes them as an input)
        self.uniforms = torch.rand(cfg.grid_h * cfg.grid_w, cfg.n_images, generator=g, device=self.dev, dtype=torch.float32)
        self.kernel_calls = 0               # libadsa calls made (each is at least one kernel of the library)
        self.x = torch.empty(Bt, D, **bf)   # the residual stream of a decode step
        self.u = torch.zeros(cfg.n_images, dtype=torch.float32, device=self.dev)   # this step's uniform numbers

    # the projections in the usual [out][in] orientation (views)
    wq = property(lambda self: self.wqkv_t[:, 0].transpose(1, 2))
    wk = property(lambda self: self.wqkv_t[:, 1].transpose(1, 2))
    wv = property(lambda self: self.wqkv_t[:, 2].transpose(1, 2))

    def generate(self, text_emb, n_cells=None):
        """Prefill and decode `n_cells` grid cells (default: the whole grid); returns the ids on the host, [cells, n_images]."""
        n = self.cfg.grid_h * self.cfg.grid_w if n_cells is None else n_cells
        self.prefill(text_emb)
        for cell in range(1, n):
            self.decode_step(cell)
        torch.cuda.synchronize(self.dev)
        return self.ids_host[:n]


class LlamaGenShell(_Decoder):
    def __init__(self, cfg: ShellConfig, seed: int = 0, device: str = "cuda:0", use_graphs: bool = True):
        super().__init__(cfg, seed, device)
        self.use_graphs, self.graphs = use_graphs, None
        C = self.budget = max(cfg.capacity, cfg.n_text + 1)   # rows a stream may hold (a row is evicted before one is inserted)
        # rows per pool page: the largest divisor of the capacity up to 1024 rows, so that a full stream fills whole pages
        page_rows = next((pr for pr in range(min(C, 1024), 15, -1) if C % pr == 0), 32)
        self.eng = B.AdsaEngine(n_layers=cfg.n_layers, batch=cfg.batch, n_heads=cfg.n_heads, head_dim=cfg.head_dim, n_text=cfg.n_text,
                                grid_h=cfg.grid_h, grid_w=cfg.grid_w, max_rows_per_stream=C,
                                page_rows=page_rows, device=device)
        self.pos = torch.zeros(2 * cfg.batch * cfg.n_heads, dtype=torch.int32, device=self.dev)   # one per row of q and of k

    # -- one block on a [rows, dim] activation; `attend` does the attention for this layer ------------------------
    def _block(self, layer, x, attend):
        c = self.cfg
        step = x.shape[0] == c.batch                                       # a decode step reuses its buffers
        h = B.rmsnorm(x, self.norm1[layer], out=self.h if step else None, eps=c.norm_eps)
        attn = attend(layer, h)                                            # [rows, dim]
        x.addmm_(attn, self.wo[layer].t())
        h = B.rmsnorm(x, self.norm2[layer], out=self.h if step else None, eps=c.norm_eps)
        gu = torch.mm(h, self.w13[layer].t(), out=self.gu) if step else h @ self.w13[layer].t()
        act = B.swiglu(gu[:, :c.ffn_hidden], gu[:, c.ffn_hidden:], out=self.act if step else None)
        x.addmm_(act, self.w2[layer].t())
        self.kernel_calls += 3
        return x

    def prefill(self, text_emb):
        """The condition: text_emb [batch, n_text, dim] bf16 (rows of the unconditional half are the caller's null
        condition).  Fills the caches through dense causal attention and returns the first image tokens."""
        c = self.cfg
        Bt, T, H, d = c.batch, c.n_text, c.n_heads, c.head_dim
        self.eng.reset()
        x = text_emb.reshape(Bt * T, c.dim).clone()
        pos = torch.arange(T, dtype=torch.int32, device=self.dev).repeat(Bt * H)            # condition rows are not rotated
        out = torch.empty(Bt, H, T, d, dtype=torch.bfloat16, device=self.dev)

        def attend(layer, h):
            q, k, v = ((h @ self.wqkv_t[layer, i]).view(Bt, T, H, d).transpose(1, 2).contiguous() for i in range(3))
            self.eng.rope_2d(q, pos)
            self.eng.rope_2d(k, pos)
            self.eng.prefill_attn(layer, q, k, v, 0, out)
            self.kernel_calls += 3
            return out.transpose(1, 2).reshape(Bt * T, c.dim)

        for layer in range(c.n_layers):
            x = self._block(layer, x, attend)
        return self._sample(x.view(Bt, T, c.dim)[:, -1].contiguous(), 0)

    # -- a decode step as CUDA graphs around the attention launches ---------------------------------------------------
    # Everything between two attention launches works on fixed buffers with fixed arguments, so it is captured once:
    # graph 0 = embedding look-up and the first block's part before the attention; graph l + 1 = block l's part after
    # the attention and block l + 1's part before it (the last one ends with the LM head and the sampling).  The
    # attention launches stay outside: their arguments (position, budget, carried state) change every step.
    def _pre(self, layer):
        c = self.cfg
        B.rmsnorm(self.x, self.norm1[layer], out=self.h, eps=c.norm_eps)
        torch.bmm(self.h.unsqueeze(0).expand(3, -1, -1), self.wqkv_t[layer], out=self.qkv.view(3, c.batch, c.dim))
        self.eng.rope_2d(self.qkv[:2], self.pos)

    def _post(self, layer):
        c = self.cfg
        self.x.addmm_(self.o.view(c.batch, c.dim), self.wo[layer].t())
        B.rmsnorm(self.x, self.norm2[layer], out=self.h, eps=c.norm_eps)
        torch.mm(self.h, self.w13[layer].t(), out=self.gu)
        B.swiglu(self.gu[:, :c.ffn_hidden], self.gu[:, c.ffn_hidden:], out=self.act)
        self.x.addmm_(self.act, self.w2[layer].t())

    def _first(self):
        n = self.cfg.n_images
        torch.index_select(self.tok_emb, 0, self.tokens, out=self.x[:n])
        self.x[n:].copy_(self.x[:n])                                       # conditional and unconditional rows
        self._pre(0)

    def _last(self):
        c = self.cfg
        B.rmsnorm(self.x, self.norm_f, out=self.h, eps=c.norm_eps)
        torch.mm(self.h, self.head.t(), out=self.logits)
        B.cfg_sample(self.logits, c.cfg_scale, min(c.top_k, c.vocab), c.temperature, self.u, tokens=self.tokens)

    def _segments(self):
        L = self.cfg.n_layers
        segs = [self._first]
        for layer in range(L):
            nxt = (lambda l=layer: (self._post(l), self._pre(l + 1))) if layer + 1 < L else (lambda l=layer: (self._post(l), self._last()))
            segs.append(nxt)
        return segs

    def _capture(self):
        segs = self._segments()
        side = torch.cuda.Stream(device=self.dev)
        side.wait_stream(torch.cuda.current_stream(self.dev))
        with torch.cuda.stream(side):                                      # once eagerly: libraries make their handles and workspaces
            for seg in segs:
                seg()
        torch.cuda.current_stream(self.dev).wait_stream(side)
        torch.cuda.synchronize(self.dev)
        graphs = []
        for seg in segs:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                seg()
            graphs.append(g)
        self.graphs = graphs

    def decode_step(self, cell):
        """The image token of grid cell `cell` (>= 1) from the token of cell - 1: one pass through every layer."""
        c = self.cfg
        cur = c.n_text + cell - 1                                          # position of the token that is fed in
        if self.use_graphs:
            if self.graphs is None:
                saved = self.tokens.clone()
                self._capture()                                            # (the capture's trial run overwrote the ids)
                self.tokens.copy_(saved)
            self.pos.fill_(cur)
            self.u.copy_(self.uniforms[cell])
            self.graphs[0].replay()
            for layer in range(c.n_layers):
                self.eng.layer_step(layer, cur, self.budget, self.q, self.k, self.v, self.o)
                self.graphs[layer + 1].replay()
            self.ids_host[cell].copy_(self.tokens, non_blocking=True)
            self.kernel_calls += 5 * c.n_layers + 3
            return self.tokens
        emb = self.tok_emb[self.tokens.long()]
        x = torch.cat([emb, emb], dim=0)                                   # conditional and unconditional rows
        self.pos.fill_(cur)

        def attend(layer, h):
            torch.bmm(h.unsqueeze(0).expand(3, -1, -1), self.wqkv_t[layer], out=self.qkv.view(3, c.batch, c.dim))   # one batched GEMM
            self.eng.rope_2d(self.qkv[:2], self.pos)                       # q and k in one call
            self.eng.layer_step(layer, cur, self.budget, self.q, self.k, self.v, self.o)
            self.kernel_calls += 2
            return self.o.view(c.batch, c.dim)

        for layer in range(c.n_layers):
            x = self._block(layer, x, attend)
        return self._sample(x, cell)

    def _sample(self, x_last, cell):
        c = self.cfg
        h = B.rmsnorm(x_last, self.norm_f, eps=c.norm_eps)
        torch.mm(h, self.head.t(), out=self.logits)
        B.cfg_sample(self.logits, c.cfg_scale, min(c.top_k, c.vocab), c.temperature, self.uniforms[cell], tokens=self.tokens)
        self.ids_host[cell].copy_(self.tokens, non_blocking=True)          # ids leave the GPU as they are drawn
        self.kernel_calls += 2
        return self.tokens


class SharedPromptShell(_Decoder):
    """n_images images of one prompt with guidance: two groups of batch rows (conditional, unconditional), each with its
    condition's rows kept once.  Nothing is evicted."""

    PAGE_ROWS = 64
    ATTN_ROWS = 4096            # query rows that one attention call takes

    def __init__(self, cfg: ShellConfig, seed: int = 0, device: str = "cuda:0", use_graphs: bool = True):
        if cfg.n_text < 1:
            raise ValueError("SharedPromptShell: the condition needs a row at least (the first token is drawn from its last)")
        super().__init__(cfg, seed, device)
        self.use_graphs, self.graph = use_graphs, None
        self.next_cell = None                                              # the grid cell decode_step makes next; None before a prefill
        L, H, d, n, pr = cfg.n_layers, cfg.n_heads, cfg.head_dim, cfg.n_images, self.PAGE_ROWS
        bf, i32 = dict(dtype=torch.bfloat16, device=self.dev), dict(dtype=torch.int32, device=self.dev)
        cells = cfg.grid_h * cfg.grid_w
        own, text = (cells + pr - 1) // pr, (cfg.n_text + pr - 1) // pr      # pages per batch row, per condition
        pages = 2 * text + cfg.batch * own
        self.k_pool, self.v_pool = torch.zeros(L, pages, H, pr, d, **bf), torch.zeros(L, pages, H, pr, d, **bf)
        self.prefix_table = torch.arange(2 * text, **i32).view(2, text)
        self.page_table = torch.arange(2 * text, pages, **i32).view(cfg.batch, own)
        self.prefix_rows = torch.full((2,), cfg.n_text, **i32)
        self.group_start = torch.tensor([0, n, 2 * n], **i32)
        # rows in the cache before and after this step's append, and the cell that is fed in: moved on by the step itself
        self.n_before, self.n_after = torch.zeros(cfg.batch, **i32), torch.ones(cfg.batch, **i32)
        self.cell = torch.zeros(1, dtype=torch.int64, device=self.dev)
        # grid row and column of every cell; the condition is not rotated (position 0, 0)
        c = torch.arange(cells, device=self.dev)
        self.positions = torch.stack([c // cfg.grid_w, c % cfg.grid_w], 1).to(torch.int32).contiguous()
        self.pos = torch.zeros(cfg.batch, 2, **i32)
        self.rotary = B.Rotary(d, (d // 4, d // 4))
        self.y = torch.empty(cfg.batch, cfg.dim, **bf)                       # a block's output, before the residual addition
        self.post1 = torch.ones(L, cfg.dim, **bf) if cfg.sandwich_norm else None
        self.post2 = torch.ones(L, cfg.dim, **bf) if cfg.sandwich_norm else None
        self.workspace = B.shared_prefix_workspace(self.q, self.k_pool[0], self.page_table, self.prefix_table)
        self.status = torch.zeros(1, **i32)

    # -- one block: h = norm1(x) of `rows` rows in, the residual stream x moved on, h = the next block's norm1 (or the last norm) out
    def _block(self, layer, x, h, y, attend):
        c = self.cfg
        post = (None, None) if self.post1 is None else (self.post1[layer], self.post2[layer])
        torch.mm(attend(layer, h), self.wo[layer].t(), out=y)
        B.norm_residual(y, x, self.norm2[layer], w_post=post[0], eps=c.norm_eps, x_out=x, h=h)
        step = x is self.x
        gu = torch.mm(h, self.w13[layer].t(), out=self.gu if step else None)
        act = B.swiglu(gu[:, :c.ffn_hidden], gu[:, c.ffn_hidden:], out=self.act if step else None)
        torch.mm(act, self.w2[layer].t(), out=y)
        after = self.norm1[layer + 1] if layer + 1 < c.n_layers else self.norm_f
        B.norm_residual(y, x, after, w_post=post[1], eps=c.norm_eps, x_out=x, h=h)

    def prefill(self, text_emb):
        """The condition, text_emb [2, n_text, dim] bf16 (conditional, unconditional), enters the shared pages; row i of it
        attends rows 0 .. i, as so many queries over the same pages with lengths 1, 2, ..  Draws the first tokens."""
        self.next_cell = None                                              # (until the condition is whole)
        with torch.cuda.device(self.dev):                                  # (calls go to the current device's stream)
            return self._prefill(text_emb)

    def _prefill(self, text_emb):
        c, T, H, d = self.cfg, self.cfg.n_text, self.cfg.n_heads, self.cfg.head_dim
        i32 = dict(dtype=torch.int32, device=self.dev)
        x = text_emb.reshape(2 * T, c.dim).clone()
        h, y = B.rmsnorm(x, self.norm1[0], eps=c.norm_eps), torch.empty_like(x)
        pos, none = torch.zeros(2 * T, 2, **i32), torch.zeros(2, **i32)
        tables = self.prefix_table.repeat_interleave(T, 0)
        lengths = torch.arange(1, T + 1, **i32).repeat(2)
        out = torch.empty(2 * T, H, d, dtype=torch.bfloat16, device=self.dev)

        def attend(layer, h):
            q, k, v = torch.matmul(h.unsqueeze(0), self.wqkv_t[layer]).view(3, 2 * T, H, d)
            B.rope_axes(self.rotary, q, pos, out=q)
            B.paged_append(k, v, self.k_pool[layer], self.v_pool[layer], self.prefix_table, none, rotary=self.rotary, pos=pos, status=self.status)
            for i in range(0, 2 * T, self.ATTN_ROWS):
                part = slice(i, i + self.ATTN_ROWS)
                B.shared_prefix_attn(q[part], self.k_pool[layer], self.v_pool[layer], tables[part], lengths[part], out=out[part], status=self.status)
            return out.view(2 * T, c.dim)

        for layer in range(c.n_layers):
            self._block(layer, x, h, y, attend)
        self.kernel_calls += 1 + (5 + len(range(0, 2 * T, self.ATTN_ROWS))) * c.n_layers + 1
        self.n_before.zero_()
        self.n_after.fill_(1)
        self.cell.fill_(0)
        self.h.copy_(h.view(2, T, c.dim)[:, -1].repeat_interleave(c.n_images, 0))   # every image starts from the same row
        self._sample()
        self.ids_host[0].copy_(self.tokens, non_blocking=True)
        self.next_cell = 1
        return self.tokens

    def _sample(self):
        """The next token of every image from h, with the uniform numbers of `cell`."""
        c = self.cfg
        torch.mm(self.h, self.head.t(), out=self.logits)
        torch.index_select(self.uniforms, 0, self.cell, out=self.u.view(1, -1))
        B.cfg_sample(self.logits, c.cfg_scale, min(c.top_k, c.vocab), c.temperature, self.u, tokens=self.tokens)

    def _attend(self, layer, h):
        c = self.cfg
        torch.bmm(h.unsqueeze(0).expand(3, -1, -1), self.wqkv_t[layer], out=self.qkv.view(3, c.batch, c.dim))
        B.paged_append(self.k, self.v, self.k_pool[layer], self.v_pool[layer], self.page_table, self.n_before, rotary=self.rotary, pos=self.pos,
                       q=self.q, q_out=self.q, status=self.status)
        B.shared_prefix_attn(self.q, self.k_pool[layer], self.v_pool[layer], self.page_table, self.n_after, self.prefix_table, self.prefix_rows,
                             self.group_start, out=self.o, workspace=self.workspace, status=self.status)
        return self.o.view(c.batch, c.dim)

    def _step(self):
        c, n = self.cfg, self.cfg.n_images
        self.pos.copy_(self.positions.index_select(0, self.cell).expand(c.batch, 2))
        torch.index_select(self.tok_emb, 0, self.tokens, out=self.x[:n])
        self.x[n:].copy_(self.x[:n])                                       # conditional and unconditional rows
        B.rmsnorm(self.x, self.norm1[0], out=self.h, eps=c.norm_eps)
        for layer in range(c.n_layers):
            self._block(layer, self.x, self.h, self.y, self._attend)
        for t in (self.n_before, self.n_after, self.cell):
            t.add_(1)
        self._sample()

    def decode_step(self, cell):
        """The image token of grid cell `cell` (after prefill: 1, 2, .. to the end of the grid) from the token of cell - 1."""
        cells = self.cfg.grid_h * self.cfg.grid_w
        if cell != self.next_cell or cell >= cells:                        # (the step follows counters on the device, past the grid's tables too)
            raise ValueError(f"decode_step: cell {cell} cannot follow, the next is {self.next_cell} of {cells} (None: prefill first)")
        with torch.cuda.device(self.dev):
            if not self.use_graphs:
                self._step()
            else:
                if self.graph is None:
                    side = torch.cuda.Stream(device=self.dev)
                    kept = [t.clone() for t in (self.n_before, self.n_after, self.cell, self.tokens)]
                    side.wait_stream(torch.cuda.current_stream(self.dev))
                    with torch.cuda.stream(side):                              # once eagerly: libraries make their handles and workspaces
                        self._step()
                    torch.cuda.current_stream(self.dev).wait_stream(side)
                    torch.cuda.synchronize(self.dev)
                    self.graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(self.graph):
                        self._step()
                    for t, was in zip((self.n_before, self.n_after, self.cell, self.tokens), kept):
                        t.copy_(was)                                           # (the trial run moved them on; its rows are written again)
                self.graph.replay()
            self.ids_host[cell].copy_(self.tokens, non_blocking=True)
        self.kernel_calls += 1 + 5 * self.cfg.n_layers + 1
        self.next_cell = cell + 1
        return self.tokens
