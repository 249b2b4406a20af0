"""Buffer management around the C-ABI calls for one model: per-layer core sets, compacted
weights and workspaces, allocated once with torch and reused.  No arithmetic here: selection,
compaction and decoding all run in the library's kernels."""
from __future__ import annotations

import operator

import torch

from . import binding as B
from .workloads import Config


class CoreSparseStack:
    """Core-sparse FFN stack of `cfg.L` layers (Section 4.2): `prefill()` fixes each layer's
    sentence-wise core set from its pre-fill activations and compacts the weights;
    `decode()` then pushes one token through all layers in one launch."""

    def __init__(self, cfg: Config, device="cuda", alpha=None, beta=None):
        self.cfg = cfg
        self.alpha = cfg.alpha if alpha is None else alpha
        self.beta = cfg.beta if beta is None else beta
        self.kind = B.FFN_RELU_GATED if cfg.gated else B.FFN_RELU
        self.K = B.coreinfer_count(self.beta, cfg.d_ff)
        dt, d, K, L = cfg.torch_dtype, cfg.d_model, self.K, cfg.L
        new = lambda *s, dtype=dt: torch.empty(s, dtype=dtype, device=device)
        self.core_idx = [new(K, dtype=torch.int32) for _ in range(L)]
        self.w_up_c = [new(K, d) for _ in range(L)]
        self.w_gate_c = [new(K, d) if cfg.gated else None for _ in range(L)]
        self.w_downT_c = [new(K, d) for _ in range(L)]
        self.select_ws = None
        self._side = None               # side stream and events of prefill(), created on first use
        self._events = None
        self.stack_ws = new(B.coreinfer_ffn_decode_stack_workspace_bytes(L, 1, d, K), dtype=torch.uint8)
        self.layer_ws = new(B.coreinfer_ffn_decode_workspace_bytes(B.MAX_BATCH, d, K), dtype=torch.uint8)
        self.layers = B.make_layers([(self.w_up_c[l], self.w_gate_c[l], self.w_downT_c[l], None, None)
                                     for l in range(L)])

    # kernels launched by one prefill() per layer / one decode() call, for launch accounting
    SELECT_KERNELS_PER_LAYER = 3
    COMPACT_KERNELS_PER_LAYER = 2
    DECODE_KERNELS_PER_TOKEN = 1

    def compacted_bytes_per_token(self) -> int:
        c = self.cfg
        return c.L * c.n_mat * self.K * c.d_model * c.esize

    def select_layer(self, l: int, act: torch.Tensor, counts_out=None, stream=None):
        need = B.coreinfer_select_workspace_bytes(act.shape[0], act.shape[1])
        if self.select_ws is None or self.select_ws.numel() < need:
            self.select_ws = torch.empty(need, dtype=torch.uint8, device=act.device)
        B.coreinfer_select_core(act, self.alpha, self.beta, self.core_idx[l], counts_out, self.select_ws, stream)

    def compact_layer(self, l: int, w_up, w_gate, w_down, stream=None):
        B.coreinfer_compact(w_up, w_gate, w_down, None, self.core_idx[l], self.K, self.w_up_c[l],
                            self.w_gate_c[l], self.w_downT_c[l], None, stream)

    def prefill(self, acts, weights, stream=None, overlap=True):
        """acts[l]: [T, d_ff] fp32 activations of layer l; weights[l] = (w_up, w_gate | None, w_down).

        Selection is a chain of small latency-bound kernels, compaction is bandwidth-bound: with
        `overlap` the compaction of layer l runs on a side stream while `stream` goes on with the
        selection of layer l + 1.  On return `stream` has been made to wait for the side stream."""
        main = torch.cuda.current_stream() if stream is None else stream
        if not overlap:
            for l in range(self.cfg.L):
                self.select_layer(l, acts[l], None, main)
                self.compact_layer(l, *weights[l], stream=main)
            return
        if self._side is None:
            self._side = torch.cuda.Stream(device=self.core_idx[0].device)
            self._events = [torch.cuda.Event() for _ in range(self.cfg.L + 2)]
        side, ev = self._side, self._events
        ev[-2].record(main)                 # earlier work on `stream` may still read the compacted buffers
        side.wait_event(ev[-2])
        for l in range(self.cfg.L):
            self.select_layer(l, acts[l], None, main)
            ev[l].record(main)
            side.wait_event(ev[l])
            self.compact_layer(l, *weights[l], stream=side)
        ev[-1].record(side)
        main.wait_event(ev[-1])

    def decode(self, x0, y_last, y_layers=None, x_layers=None, stream=None):
        """x0 [1, d] -> y_last [1, d] fp32 (FFN output of the last layer)."""
        B.coreinfer_ffn_decode_stack(self.layers, x0, self.kind, y_last, y_layers, x_layers, self.stack_ws, stream)

    def decode_layer(self, l: int, x, y, stream=None):
        """One layer, any batch 1..8."""
        B.coreinfer_ffn_decode(x, self.kind, self.w_up_c[l], self.w_gate_c[l], self.w_downT_c[l], None, None,
                               y, self.layer_ws, stream)

    def check(self, stream=None):
        B.coreinfer_workspace_status(self.stack_ws, stream)


class W4Linear:
    """A weight matrix [N, K] (any strides) held in four bits: `linear(x, y)` is y = act(x W^T + bias) * mul."""

    def __init__(self, weight, group=128, bias=None, act=B.ACT_NONE, stream=None):
        N, K = weight.shape
        new = lambda n: torch.empty(n, dtype=torch.uint8, device=weight.device)
        self.codes, self.pairs = new(B.coreinfer_w4_codes_bytes(N, K)), new(B.coreinfer_w4_pairs_bytes(N, K, group))
        self.bias, self.act = bias, act
        self.matrix = B.make_w4_matrix(self.codes, self.pairs, N, K, group)
        self.load(weight, stream)

    def load(self, weight, stream=None):
        """Other weights of the same shape into the same buffers, so that a captured graph runs on with them."""
        if tuple(weight.shape) != (self.matrix.N, self.matrix.K):
            raise B.CoreInferError(B.ERR_INVALID_ARG, "weights of shape %s do not fit the %d x %d matrix"
                                   % (tuple(weight.shape), self.matrix.N, self.matrix.K))
        B.coreinfer_w4_quantize(weight, self.matrix.group, self.codes, self.pairs, stream)

    def __call__(self, x, y, mul=None, stream=None):
        B.coreinfer_w4_matvec(self.matrix, x, self.act, self.bias, mul, y, stream)


class KV4Cache:
    """Keys, values, weights and positions of one layer's 4-bit cache, and the workspace of its calls.  The workspace holds an fp32
    logit per slot and query row of the longest call, max_tokens tokens (64 bytes per slot and head where heads are not
    shared, beside 2 * (head_dim / 2 + 4 * head_dim / group) + 8 of the cache); a caller with many layers can use the
    binding's calls with one workspace for all."""

    def __init__(self, batch, q_heads, kv_heads, capacity, head_dim, group=64, device="cuda"):
        new = lambda *s, dtype: torch.empty((batch, kv_heads, capacity) + s, dtype=dtype, device=device)
        self.q_heads = q_heads
        self.k_codes, self.v_codes = (new(head_dim // 2, dtype=torch.uint8) for _ in range(2))
        self.k_pairs, self.v_pairs = (new(head_dim // group, 2, dtype=torch.float16) for _ in range(2))
        self.weight, self.position = new(dtype=torch.float32), new(dtype=torch.int32)
        self.state = torch.zeros(batch, 4, dtype=torch.int32, device=device)
        self.cache = B.make_kv4_cache(self.k_codes, self.k_pairs, self.v_codes, self.v_pairs, self.state, self.weight, self.position)
        # tokens of one attend() at most: with many query heads per key head the rows are the limit
        self.max_tokens = min(B.KV4_MAX_QUERIES, B.KV4_MAX_ROWS * kv_heads // q_heads)
        need = max(B.coreinfer_kv4_attention_workspace_bytes(self.cache, q_heads, self.max_tokens),
                   B.coreinfer_kv4_evict_workspace_bytes(self.cache))
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)

    def append(self, k, v, k_stored=None, v_stored=None, stream=None):
        B.coreinfer_kv4_append(self.cache, k, v, k_stored, v_stored, stream)

    def attend(self, q, out, scale=None, accumulate=True, stream=None):
        B.coreinfer_kv4_attention(self.cache, q, self.cache.head_dim ** -0.5 if scale is None else scale, out, accumulate,
                                  self.ws, stream)

    def evict(self, budget, recent, first, stream=None):
        B.coreinfer_kv4_evict(self.cache, self.cache, budget, recent, first, self.ws, stream)

    def lengths(self):
        """Slots in use per sequence (synchronises)."""
        return self.state[:, 0].tolist()

    def check(self):
        """Raises if a sequence had to refuse tokens for want of room (synchronises)."""
        refused = self.state[:, 2].tolist()
        if any(refused):
            raise B.CoreInferError(B.ERR_INVALID_ARG, "tokens refused by a full cache: %s" % refused)


class Rotary:
    """Rotary positions of queries and keys (binding.ROPE_* scalings) and, where weights [head_dim] are given, the norms of
    their heads that go before.  Keeps the table of frequencies on the device."""

    def __init__(self, rot_dim, base=10000.0, scaling=B.ROPE_PLAIN, factor=1.0, original_context=0, interleaved=False, q_norm=None,
                 k_norm=None, eps=1e-6, device="cuda"):
        self.turns, magnitude = B.coreinfer_rope_frequencies(rot_dim, base, scaling, factor, original_context, device=device)
        self.norms = q_norm, k_norm
        self.rope = B.make_rope(self.turns, interleaved, magnitude, q_norm, k_norm, eps)

    def __call__(self, positions, q, k, q_out=None, k_out=None, stream=None):
        """q, k [tokens, heads, head_dim] to the positions int32 [tokens]; in place unless outputs are given."""
        B.coreinfer_rope_apply(self.rope, positions, q, k, q if q_out is None else q_out, k if k_out is None else k_out, stream)


class Pages:
    """Which pages hold which sequence's tokens: the table and lengths that the caches of all layers share, and the packing of
    a call's new tokens.  Pages are given out and taken back on the host."""

    def __init__(self, batch, n_pages, page_size, max_tokens, device="cuda"):
        self.page_size, self.n_pages = page_size, n_pages
        self.max_pages = -(-max_tokens // page_size)
        self.free = list(range(n_pages - 1, -1, -1))
        self.held = [[] for _ in range(batch)]
        self.tokens = [0] * batch
        self.table = torch.full((batch, self.max_pages), -1, dtype=torch.int32, device=device)
        self.length = torch.zeros(batch, dtype=torch.int32, device=device)
        self.start = torch.zeros(batch + 1, dtype=torch.int32, device=device)
        self.total = 0                                       # rows of the packing
        # who takes part in steps: who holds tokens, or before the first add() everybody
        self.runs, self._runs = [1] * batch, torch.ones(batch, dtype=torch.int32, device=device)

    def _per_sequence(self, numbers):
        try:
            numbers = [operator.index(n) for n in numbers]
        except TypeError:
            numbers = []
        if len(numbers) != len(self.held) or min(numbers) < 0:
            raise B.CoreInferError(B.ERR_INVALID_ARG, "%d numbers >= 0 were expected, one per sequence" % len(self.held))
        return numbers

    def reserve(self, tokens):
        """Pages for that many tokens of every sequence (a number or one per sequence), so that a captured step may run on."""
        want = self._per_sequence([tokens] * len(self.held) if isinstance(tokens, int) else tokens)
        need = [max(0, -(-n // self.page_size) - len(h)) for n, h in zip(want, self.held)]
        if max(want) > self.max_pages * self.page_size or sum(need) > len(self.free):
            raise B.CoreInferError(B.ERR_INVALID_ARG, "%d pages of %d left, %d needed for %s tokens; a sequence takes %d tokens at most"
                                   % (len(self.free), self.n_pages, sum(need), want, self.max_pages * self.page_size))
        for b, n in enumerate(need):
            if n:
                at = len(self.held[b])
                self.held[b] += [self.free.pop() for _ in range(n)]
                self.table[b, at:at + n] = torch.tensor(self.held[b][at:], dtype=torch.int32)

    def add(self, new):
        """Room for new[b] more tokens of each sequence, which the next calls bring: sets lengths and packing.  The total."""
        new = self._per_sequence(new)
        self.reserve([t + n for t, n in zip(self.tokens, new)])
        self.tokens = [t + n for t, n in zip(self.tokens, new)]
        self.length.copy_(torch.tensor(self.tokens, dtype=torch.int32))
        self.runs = [int(t > 0) for t in self.tokens]
        self._runs.copy_(torch.tensor(self.runs, dtype=torch.int32))
        self.start.copy_(torch.tensor([sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32))
        self.total = sum(new)
        return self.total

    def decoding(self):
        """Packing for one token of every sequence.  One that has ended or not begun keeps its row, which is at position -1: it is stored
        nowhere and attends to nothing."""
        self.start.copy_(torch.arange(len(self.held) + 1, dtype=torch.int32))
        self.total = len(self.held)

    def one_more(self):
        """Lengths for the next token of every sequence that holds some, on the device alone: what a captured step does in add()'s
        place, behind decoding() and within what reserve() has given.  Replays are told to counted()."""
        self.length += self._runs

    def counted(self, steps):
        """That many steps by one_more() have run.  Raises where they went on behind the pages that reserve() had given: the tokens there
        were not stored, and the sequence holds what its pages do."""
        if steps < 0:
            raise B.CoreInferError(B.ERR_INVALID_ARG, "%d steps" % steps)
        ran = [t + steps * runs for t, runs in zip(self.tokens, self.runs)]
        self.tokens = [min(t, len(h) * self.page_size) for t, h in zip(ran, self.held)]
        if self.tokens != ran:
            self.length.copy_(torch.tensor(self.tokens, dtype=torch.int32))
            raise B.CoreInferError(B.ERR_INVALID_ARG, "steps to %s tokens ran behind the reserved pages: %s are held" % (ran, self.tokens))

    def release(self, b):
        """Sequence b has ended: its pages are free, and it sits out the steps until add() brings it new tokens."""
        if b not in range(len(self.held)) or not hasattr(b, "__index__"):
            raise B.CoreInferError(B.ERR_INVALID_ARG, "sequence %s of %d" % (b, len(self.held)))
        self.free += reversed(self.held[b])
        self.held[b], self.tokens[b], self.runs[b] = [], 0, 0
        self.table[b] = -1
        self.length[b] = 0
        self._runs[b] = 0


class PagedKVCache:
    """Keys and values of one layer in pages, and attention over them: up to max_tokens new tokens a call, or the workspace grows (at most
    a few times: the forms of the attention differ in it, not the lengths) and the ones before stay, as captured calls may use them."""

    def __init__(self, pages, q_heads, kv_heads, head_dim, dtype=torch.bfloat16, max_tokens=1):
        dev = pages.table.device
        self.pages, self.q_heads, self.head_dim = pages, q_heads, head_dim
        self.k, self.v = (torch.zeros(pages.n_pages, kv_heads, pages.page_size, head_dim, dtype=dtype, device=dev) for _ in range(2))
        self.cache = B.make_paged_cache(self.k, self.v, pages.table, pages.length)
        self.ws, self._outgrown = self._workspace(max_tokens), []

    def _workspace(self, tokens):
        ws = torch.empty(B.coreinfer_paged_attention_workspace_bytes(self.cache, self.q_heads, tokens), dtype=torch.uint8, device=self.k.device)
        ws[:16] = 0                                          # no wait of a call has given up yet
        return ws

    def append(self, k, v, rotary=None, q=None, q_out=None, positions=None, stream=None):
        B.coreinfer_paged_append(self.cache, self.pages.start, k, v, None if rotary is None else rotary.rope, positions, q, q_out, stream)

    def attend(self, q, out, scale=None, window=0, sinks=0, stream=None):
        if B.coreinfer_paged_attention_workspace_bytes(self.cache, self.q_heads, q.shape[0]) > self.ws.numel():
            # more tokens than were announced; calls captured before, or under way on another stream, still write the old one
            self._outgrown.append(self.ws)
            with torch.cuda.stream(stream):
                self.ws = self._workspace(q.shape[0])
        B.coreinfer_paged_attention(self.cache, self.pages.start, q, self.head_dim ** -0.5 if scale is None else scale, out, self.ws, window, sinks, stream)

    def check(self, stream=None):
        """Raises if a wait of the last attend(), or of the last in a workspace since outgrown, gave up (synchronises)."""
        for ws in self._outgrown + [self.ws]:
            B.coreinfer_workspace_status(ws, stream)


class CorePagedLayer:
    """A decoder layer in 16 bits whose prompts arrive in pieces: rotary positions, a paged cache, attention with an optional window
    and first tokens that stay visible, and the FFN, dense for the prompt's tokens and over the core neurons afterwards.  Counts of
    the pieces add up (Eq. 3 is a sum over tokens); `fix_core()` ends the prompt: it takes the top beta of the counts and compacts.

    weights as Core4Layer's; the residual stream is fp32, norms of the stream have no parameters and there are no biases.  All layers of a
    model share one Pages.  `piece` and `step` take what Pages.add() announced; up to 8 sequences decode together."""

    def __init__(self, cfg: Config, pages, q_heads, kv_heads, head_dim, weights, rotary=None, window=0, sinks=0, max_piece=512):
        dev = pages.table.device
        self.cfg, self.pages, self.heads, self.rotary, self.span = cfg, pages, (q_heads, kv_heads, head_dim), rotary, (window, sinks)
        self.w_qkv, self.w_o, *self.w_ffn = weights
        self.cache = PagedKVCache(pages, q_heads, kv_heads, head_dim, cfg.torch_dtype, max_piece)
        self.kind = B.FFN_RELU_GATED if cfg.gated else B.FFN_RELU
        self.K = B.coreinfer_count(cfg.beta, cfg.d_ff)
        new = lambda *s, dtype=cfg.torch_dtype: torch.empty(s, dtype=dtype, device=dev)
        self.counts, self.seen = torch.zeros(cfg.d_ff, dtype=torch.int32, device=dev), 0
        self._f, self._top, self.core_idx = new(cfg.d_ff, dtype=torch.int32), new(self.K, dtype=torch.int32), new(self.K, dtype=torch.int32)
        self.up, self.down = new(self.K, cfg.d_model), new(self.K, cfg.d_model)
        self.gate = new(self.K, cfg.d_model) if cfg.gated else None
        self.deployed = False                                # whether up, gate and down hold the neurons of core_idx
        self._ffn_ws = new(B.coreinfer_ffn_decode_workspace_bytes(B.MAX_BATCH, cfg.d_model, self.K), dtype=torch.uint8)
        self._act_ws = new(B.coreinfer_prefill_activations_workspace_bytes(), dtype=torch.uint8)

    def _norm(self, h):
        return torch.nn.functional.layer_norm(h, (self.cfg.d_model,)).to(self.cfg.torch_dtype)

    def _attention(self, h, most=None):
        if h.shape != (self.pages.total, self.cfg.d_model) or h.shape[0] > (most or h.shape[0]):
            raise B.CoreInferError(B.ERR_INVALID_ARG, "rows [%d, %d] were announced%s, got %s"
                                   % (self.pages.total, self.cfg.d_model, ", up to %d are taken" % most if most else "", tuple(h.shape)))
        Hq, H, D = self.heads
        q, k, v = torch.nn.functional.linear(self._norm(h), self.w_qkv).split((Hq * D, H * D, H * D), dim=-1)
        q, k, v = q.unflatten(-1, (Hq, D)), k.unflatten(-1, (H, D)), v.unflatten(-1, (H, D))
        if self.rotary is None:
            self.cache.append(k, v)
        else:
            self.cache.append(k, v, self.rotary, q, q)
        ctx = torch.empty(h.shape[0], Hq, D, dtype=q.dtype, device=h.device)
        self.cache.attend(q, ctx, None, *self.span)
        h += torch.nn.functional.linear(ctx.flatten(1), self.w_o)

    def piece(self, h):
        """h [tokens, d] fp32, packed pieces of prompts: updated in place; their activations are counted."""
        cfg = self.cfg
        self._attention(h)
        w_up, w_gate, w_down = self.w_ffn
        x = self._norm(h)
        act = torch.empty(h.shape[0], cfg.d_ff, dtype=cfg.torch_dtype, device=h.device)
        B.coreinfer_prefill_activations(x, self.kind, w_up, w_gate, None, act, self._act_ws)
        h += torch.nn.functional.linear(act, w_down)
        ws = torch.empty(B.coreinfer_select_workspace_bytes(*act.shape), dtype=torch.uint8, device=h.device)
        B.coreinfer_select_core(act, cfg.alpha, cfg.beta, self._top, self._f, ws)        # the counts are what is wanted of it
        B.coreinfer_counts_add(self.counts, self._f)
        self.seen += h.shape[0]

    def fix_core(self):
        """Deploys the top beta of the neurons by the counts of the pieces so far, which start anew."""
        if not self.seen:
            raise B.CoreInferError(B.ERR_INVALID_ARG, "no piece has been counted since the last core set")
        w_up, w_gate, w_down = self.w_ffn
        B.coreinfer_top_by_count(self.counts, self.seen, self.cfg.beta, self.core_idx)
        B.coreinfer_compact(w_up, w_gate, w_down, None, self.core_idx, self.K, self.up, self.gate, self.down, None)
        self.counts.zero_()
        self.seen, self.deployed = 0, True

    def step(self, h):
        """h [batch, d] fp32, one new token per sequence: updated in place."""
        if not self.deployed:
            raise B.CoreInferError(B.ERR_INVALID_ARG, "a step decodes over the core set, which fix_core() chooses")
        self._attention(h, B.MAX_BATCH)
        y = torch.empty_like(h)
        B.coreinfer_ffn_decode(self._norm(h), self.kind, self.up, self.gate, self.down, None, None, y, self._ffn_ws)
        h += y


class Core4Layer:
    """A decoder layer whose decode step streams four bits per weight and per cached value: projections,
    attention over a cache that is kept within `budget` slots per head, and the FFN over the core neurons
    that the prompt selected.  Up to 8 sequences decode together and share the core set.

    weights = (w_qkv [(q_heads + 2 kv_heads) * head_dim, d], w_o [d, q_heads * head_dim], w_up, w_gate | None,
    w_down) in the configuration's 16-bit type; the residual stream is fp32, norms have no parameters, there are no biases, positions
    are rotary where a Rotary is given and not marked otherwise, and the FFN is ReLU or ReLU-gated as the configurations' are: a part of a decoder to build on rather than
    one of the models.  The 16-bit weights stay for the next prompt beside their 4-bit copies, so four bits save the bytes of
    a decode step and not memory.  The prompt's dense products and the norms are torch's; a decode step runs in the library's kernels but for
    the norms and the two additions, and can be captured in a CUDA graph, which stays valid over later prompts."""

    def __init__(self, cfg: Config, batch, q_heads, kv_heads, head_dim, budget, weights, recent=32, first=4, max_prompt=None,
                 group=128, cache_group=64, device="cuda", rotary=None):
        self.cfg, self.batch, self.heads = cfg, batch, (q_heads, kv_heads, head_dim)
        self.budget, self.recent, self.first, self.group = budget, recent, first, group
        self.w_qkv, self.w_o, *self.w_ffn = weights
        self.qkv, self.o = W4Linear(self.w_qkv, group), W4Linear(self.w_o, group)
        most = max(cfg.T if max_prompt is None else max_prompt, budget + 1)
        self.cache = KV4Cache(batch, q_heads, kv_heads, -(-most // 16) * 16, head_dim, cache_group, device)
        self.K = B.coreinfer_count(cfg.beta, cfg.d_ff)
        self.core_idx = torch.empty(self.K, dtype=torch.int32, device=device)
        self.up = self.gate = self.down = None               # core-sparse FFN, from prompt()
        new = lambda n, dtype=cfg.torch_dtype: torch.empty(batch, n, dtype=dtype, device=device)
        self._qkv, self._ctx = new(self.w_qkv.shape[0]), new(q_heads * head_dim)
        self._g, self._h, self._y = new(self.K), new(self.K), new(cfg.d_model, torch.float32)
        self.rotary, self._position = rotary, torch.zeros(batch, dtype=torch.int32, device=device)   # of the next token

    def _norm(self, h):
        return torch.nn.functional.layer_norm(h, (self.cfg.d_model,)).to(self.cfg.torch_dtype)

    def _split(self, qkv, T):
        Hq, H, D = self.heads
        q, k, v = qkv.view(self.batch, T, -1).split((Hq * D, H * D, H * D), dim=-1)
        return q.unflatten(-1, (Hq, D)), k.unflatten(-1, (H, D)), v.unflatten(-1, (H, D))

    def prompt(self, h):
        """h [batch, T, d] fp32, the prompts' residual stream: updated in place.  Fills the cache, lets the last
        tokens' attention decide which slots the budget keeps, and fixes the core set.  T is at most what the cache holds."""
        cfg, T, (Hq, H, D) = self.cfg, h.shape[1], self.heads
        if h.shape != (self.batch, T, cfg.d_model) or not 1 <= T <= self.cache.cache.capacity:
            raise B.CoreInferError(B.ERR_INVALID_ARG, "a prompt of shape %s: %d sequences of 1 to %d tokens were expected"
                                   % (tuple(h.shape), self.batch, self.cache.cache.capacity))
        q, k, v = self._split(torch.nn.functional.linear(self._norm(h), self.w_qkv), T)
        if self.rotary is not None:
            at = torch.arange(T, dtype=torch.int32, device=h.device).repeat(self.batch)
            self.rotary(at, q.flatten(0, 1), k.flatten(0, 1))
            self._position.fill_(T)
        self.cache.state.zero_()
        k_stored, v_stored = (torch.empty(self.batch, T, H, D, dtype=k.dtype, device=h.device) for _ in range(2))
        self.cache.append(k, v, k_stored, v_stored)
        # the prompt attends to what the cache holds, as later tokens will
        ctx = torch.nn.functional.scaled_dot_product_attention(q.transpose(1, 2), k_stored.transpose(1, 2), v_stored.transpose(1, 2),
                                                               is_causal=True, enable_gqa=Hq != H).transpose(1, 2)
        h += torch.nn.functional.linear(ctx.reshape(self.batch, T, Hq * D), self.w_o)
        seen = min(T, self.cache.max_tokens)
        last = q[:, T - seen:].contiguous()
        self.cache.attend(last, torch.empty_like(last))      # for its weights
        self.cache.evict(self.budget, self.recent, self.first)
        # FFN: dense for the prompt's own tokens, then over the core
        w_up, w_gate, w_down = self.w_ffn
        x = self._norm(h).view(self.batch * T, cfg.d_model)
        act = torch.empty(self.batch * T, cfg.d_ff, dtype=cfg.torch_dtype, device=h.device)
        kind = B.FFN_RELU_GATED if cfg.gated else B.FFN_RELU
        new_bytes = lambda n: torch.empty(n, dtype=torch.uint8, device=h.device)
        B.coreinfer_prefill_activations(x, kind, w_up, w_gate, None, act, new_bytes(B.coreinfer_prefill_activations_workspace_bytes()))
        h += torch.nn.functional.linear(act, w_down).view_as(h)
        B.coreinfer_select_core(act, cfg.alpha, cfg.beta, self.core_idx, None,
                                new_bytes(B.coreinfer_select_workspace_bytes(*act.shape)))
        up, down = (torch.empty(self.K, cfg.d_model, dtype=cfg.torch_dtype, device=h.device) for _ in range(2))
        gate = torch.empty_like(up) if cfg.gated else None
        B.coreinfer_compact(w_up, w_gate, w_down, None, self.core_idx, self.K, up, gate, down, None)
        if self.up is None:
            self.up = W4Linear(up, self.group, act=B.ACT_NONE if cfg.gated else B.ACT_RELU)
            self.gate = W4Linear(gate, self.group, act=B.ACT_RELU) if cfg.gated else None
            self.down = W4Linear(down.t(), self.group)       # the transposed down projection, by its strides
        else:                                                # a step captured in a graph keeps the buffers
            self.up.load(up)
            if cfg.gated:
                self.gate.load(gate)
            self.down.load(down.t())

    def step(self, h):
        """h [batch, d] fp32, one new token per sequence: updated in place."""
        self.qkv(self._norm(h), self._qkv)
        q, k, v = self._split(self._qkv, 1)
        if self.rotary is not None:
            self.rotary(self._position, q.flatten(0, 1), k.flatten(0, 1))
            self._position += 1
        self.cache.append(k, v)
        self.cache.attend(q, self._ctx.view_as(q))
        self.cache.evict(self.budget, self.recent, self.first)
        self.o(self._ctx, self._y)
        h += self._y
        x = self._norm(h)
        if self.gate is not None:
            self.gate(x, self._g)
        self.up(x, self._h, self._g if self.gate is not None else None)
        self.down(self._h, self._y)
        h += self._y
