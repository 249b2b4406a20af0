"""Buffer management around the C-ABI calls for one model: per-layer core sets, compacted
weights and workspaces, allocated once with torch and reused.  No arithmetic here: selection,
compaction and decoding all run in the library's kernels."""
from __future__ import annotations

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


class Core4Layer:
    """A decoder layer whose decode step streams four bits per weight and per cached value: projections,
    attention over a cache that is kept within `budget` slots per head, and the FFN over the core neurons
    that the prompt selected.  Up to 8 sequences decode together and share the core set.

    weights = (w_qkv [(q_heads + 2 kv_heads) * head_dim, d], w_o [d, q_heads * head_dim], w_up, w_gate | None,
    w_down) in the configuration's 16-bit type; the residual stream is fp32, norms have no parameters, there are no biases and no
    rotary positions, and the FFN is ReLU or ReLU-gated as the configurations' are: a part of a decoder to build on rather than
    one of the models.  The 16-bit weights stay for the next prompt beside their 4-bit copies, so four bits save the bytes of
    a decode step and not memory.  The prompt's dense products and the norms are torch's; a decode step runs in the library's kernels but for
    the norms and the two additions, and can be captured in a CUDA graph, which stays valid over later prompts."""

    def __init__(self, cfg: Config, batch, q_heads, kv_heads, head_dim, budget, weights, recent=32, first=4, max_prompt=None,
                 group=128, cache_group=64, device="cuda"):
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
