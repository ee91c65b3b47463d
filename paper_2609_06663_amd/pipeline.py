"""The whole eviction pass (score -> select -> compact) on torch device tensors.

`EvictionPass` allocates every output and the workspace once for a given
shape, so that `run()` only enqueues the three library calls -- the form the
benchmark times.  All arithmetic happens inside libecokv.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import ecokv as E


class EvictionPass:
    def __init__(self, shape: E.Shape, budget, mode: int = E.PER_HEAD,
                 params: Optional[E.Params] = None, dtype: torch.dtype = torch.bfloat16,
                 device: str = "cuda", workspace: Optional[torch.Tensor] = None):
        self.shape, self.budget, self.mode = shape, E._flat_ints(budget), mode
        self.params = params or E.Params()
        c = shape.c
        L, Hkv, D, w, B = c.num_layers, c.num_kv_heads, c.head_dim, c.window, c.num_seqs
        cu = shape.cu_seqlens
        self.Ptot = cu[-1] - B * w
        U = L * Hkv * B
        self.scores = torch.empty(L * Hkv * self.Ptot, dtype=torch.float32, device=device)
        self.lambda_ = torch.empty(U, dtype=torch.float32, device=device)
        self.stats = torch.empty(U * E.NSTATS, dtype=torch.float32, device=device)
        ws = E.ecokv_workspace_size(shape, self.params)
        if workspace is not None and workspace.numel() >= ws:
            self.workspace = workspace  # (shared with passes that never run at the same time)
        else:
            # zero-filled: its first word is the status that ecokv_workspace_status reads
            self.workspace = torch.zeros(max(ws, 256), dtype=torch.uint8, device=device)
        # zero-filled before its first use
        self.sel_workspace = torch.zeros(max(E.ecokv_select_workspace_size(shape, mode), 256), dtype=torch.uint8,
                                         device=device)
        self.n_idx = E.ecokv_index_count_mode(shape, mode, self.budget)
        self.idx = torch.empty(max(self.n_idx, 1), dtype=torch.int32, device=device)
        self.counts = torch.empty(max(U, 1), dtype=torch.int32, device=device)
        self.offsets = torch.empty(max(U, 1), dtype=torch.int32, device=device)
        self.Kc = torch.empty((max(self.n_idx, 1), D), dtype=dtype, device=device)
        self.Vc = torch.empty((max(self.n_idx, 1), D), dtype=dtype, device=device)

    def score(self, K: torch.Tensor, Q_win: torch.Tensor, stream=None, V: Optional[torch.Tensor] = None,
              pre: Optional[torch.Tensor] = None):
        if pre is not None:
            E.ecokv_score_pre(K, V, Q_win, self.shape, self.params, pre, self.scores, self.lambda_, self.stats,
                              self.workspace, stream)
        elif self.params.imp_mode == E.IMP_ATTN_VNORM:
            E.ecokv_score_v(K, V, Q_win, self.shape, self.params, self.scores, self.lambda_, self.stats,
                            self.workspace, stream)
        else:
            E.ecokv_score(K, Q_win, self.shape, self.params, self.scores, self.lambda_, self.stats,
                          self.workspace, stream)

    def select(self, stream=None):
        E.ecokv_select(self.scores, self.shape, self.mode, self.budget, self.idx, self.counts,
                       self.offsets, self.sel_workspace, stream)

    def compact(self, K: torch.Tensor, V: torch.Tensor, stream=None):
        E.ecokv_compact(K, V, self.shape, self.mode, self.budget, self.idx, self.counts, self.offsets,
                        self.Kc, self.Vc, stream)

    def run(self, K: torch.Tensor, V: torch.Tensor, Q_win: torch.Tensor, stream=None,
            pre: Optional[torch.Tensor] = None):
        self.score(K, Q_win, stream, V, pre)
        self.select(stream)
        self.compact(K, V, stream)
        return self

    def check(self, stream=None):
        """Synchronise `stream` and raise if a score call since the last check
        had a wait between blocks give up (see ecokv_workspace_status)."""
        E.ecokv_workspace_status(self.workspace, stream)


class LayerwiseEviction:
    """The pass layer by layer as a prefill finishes the layers, one call per
    layer or per group of consecutive layers.

    `shape` is the shape of one call: num_layers = 1 for a call per layer, or
    k > 1 for a call per group of k consecutive layers (whose K, V and Q_win
    the caller passes as [k][...] tensors, e.g. views of a cache laid out layer
    by layer).  Call c runs on the c % 2-th of two side streams (default
    priority), with its own outputs (`passes[c]`: scores, idx, counts, offsets,
    Kc, Vc) and the workspace of its stream.  One call's select and epilogue
    occupy only a few compute units; on two streams they overlap the next
    call's sweeps (28 layers of 28q/4kv at 32768 tokens: 77 -> 48 us per layer
    with a call per layer); a group of layers per call fills more of the chip
    per launch.  `run_layer` / `run_group` order the call after the work
    already queued on the caller's stream; `wait` makes the caller's stream
    wait for every call queued so far.  The caller keeps a call's K, V and
    Q_win alive until `wait` (they are read on a side stream, which torch's
    allocator does not track).  The host work per call is one event record
    and wait plus the three library calls.
    """

    def __init__(self, shape: E.Shape, budget, num_layers: int, mode: int = E.PER_HEAD,
                 params: Optional[E.Params] = None, dtype: torch.dtype = torch.bfloat16, device: str = "cuda"):
        k = shape.c.num_layers
        if k < 1 or num_layers % k != 0:
            raise ValueError(f"the call shape's {k} layers must divide the {num_layers} layers")
        self.layers_per_call = k
        params = params or E.Params()
        ws = max(E.ecokv_workspace_size(shape, params), 256)
        self.streams = [torch.cuda.Stream(device=device), torch.cuda.Stream(device=device)]
        self.workspaces = [torch.zeros(ws, dtype=torch.uint8, device=device) for _ in range(2)]
        self.passes = [EvictionPass(shape, budget, mode, params, dtype, device, self.workspaces[c % 2])
                       for c in range(num_layers // k)]
        self._ready = [torch.cuda.Event(), torch.cuda.Event()]
        self._done = [torch.cuda.Event(), torch.cuda.Event()]

    def run_group(self, call: int, K: torch.Tensor, V: torch.Tensor, Q_win: torch.Tensor) -> EvictionPass:
        """Call `call`: layers call * k .. call * k + k - 1 (K, V, Q_win over them)."""
        i = call % 2
        s, ready = self.streams[i], self._ready[i]
        ready.record(torch.cuda.current_stream(K.device))
        s.wait_event(ready)
        return self.passes[call].run(K, V, Q_win, stream=s)

    def run_layer(self, layer: int, K: torch.Tensor, V: torch.Tensor, Q_win: torch.Tensor) -> EvictionPass:
        """One layer per call (the call shape's num_layers = 1)."""
        if self.layers_per_call != 1:
            raise ValueError("this instance takes groups of layers: use run_group")
        return self.run_group(layer, K, V, Q_win)

    def run_layers(self, calls, K, V, Q_win):
        """Several calls whose inputs are all ready: one ordering event for
        all of them (per-call events cost 48 -> 54 us per layer on the
        28-layer stack with a call per layer).  K, V, Q_win: sequences indexed
        like `calls`."""
        cur = torch.cuda.current_stream(self.workspaces[0].device)
        for s, ready in zip(self.streams, self._ready):
            ready.record(cur)
            s.wait_event(ready)
        for j, c in enumerate(calls):
            self.passes[c].run(K[j], V[j], Q_win[j], stream=self.streams[c % 2])

    def wait(self):
        cur = torch.cuda.current_stream(self.workspaces[0].device)
        for s, done in zip(self.streams, self._done):
            done.record(s)
            cur.wait_event(done)

    def check(self):
        """Synchronise both side streams and raise if a layer's score call had a
        wait between blocks give up (see ecokv_workspace_status)."""
        for s, ws in zip(self.streams, self.workspaces):
            E.ecokv_workspace_status(ws, s)


class Continuations:
    """Generation from the compressed prompts of an `EvictionPass`.

    Prompt s is continued by fan_out[s] continuations of up to `max_new` tokens
    each, whose keys and values lie in paged tails; all continuations of a
    prompt share its kept rows.  For every generated token, `step` takes the new
    queries, keys and values as the projections wrote them ([L][N][heads][D],
    views of a fused tensor will do), norms and rotates queries and keys (`rope`),
    appends keys and values and attends: O [L][H_q][N][D] float32 and lse; then
    `advance` moves on.  Positions go on from the prompts' own lengths, whatever
    was evicted.  All continuations go on together: one that has ended keeps its
    place, with any token and its output unused (`rows`, `tail_counts` and
    `positions` are advanced for all).  The pass may hold one layer or several;
    with a pass per layer, each layer has its own instance, advanced with the
    others.

    `step` and `advance` only enqueue work, on one stream at a time (they share a
    workspace): `advance` goes where the last `step` went, to the stream that it
    was given or else to the current one.  Who changes the stream between calls
    orders the one after the other.  To capture them in a HIP graph, pass `step`
    max_tail=max_new: by default it is the present length, which a replay would
    not raise.  A replay moves the device's counters only; `length` is the
    caller's to keep."""

    def __init__(self, ep: EvictionPass, fan_out, max_new: int, rope: E.Rope, page_size: int = 64):
        shape = ep.shape
        c = shape.c
        fan_out = E._flat_ints(fan_out)
        if len(fan_out) != c.num_seqs or min(fan_out) < 0:
            raise ValueError("fan_out has the number of continuations of each prompt")
        if sum(fan_out) < 1:
            raise ValueError("fan_out has no continuation")
        if max_new < 1:
            raise ValueError(f"max_new {max_new} < 1")
        self.ep, self.rope, self.max_new, self.length = ep, rope, int(max_new), 0
        self._stream = None  # that the last step was given
        self.fan = [0]
        for f in fan_out:
            self.fan.append(self.fan[-1] + f)
        N, L, Hq, Hkv, D = self.fan[-1], c.num_layers, c.num_q_heads, c.num_kv_heads, c.head_dim
        dev, dtype = ep.Kc.device, ep.Kc.dtype
        per = -(-self.max_new // page_size)
        self.tails = E.Tails(*(torch.empty((L, N * per, Hkv, page_size, D), dtype=dtype, device=dev) for _ in range(2)),
                             torch.arange(N * per, dtype=torch.int32, device=dev).view(N, per))
        cu = shape.cu_seqlens
        start = [cu[s + 1] - cu[s] for s in range(c.num_seqs) for _ in range(fan_out[s])]
        # row of the next token, rows with it, its position
        self._at = torch.tensor([[0] * N, [1] * N, start], dtype=torch.int32, device=dev)
        self.rows, self.tail_counts, self.positions = self._at
        # rows that one head can keep: the budget, or what the heads of a layer share
        w, lens = c.window, [cu[s + 1] - cu[s] for s in range(c.num_seqs)]
        if ep.mode == E.LAYER_FLAT:
            self.max_count = max(min(t, Hkv * (b - w) + w) for t, b in zip(lens, ep.budget))
        elif ep.mode == E.HEAD_BUDGETS:
            self.max_count = min(max(lens), max(ep.budget))
        else:
            self.max_count = max(min(t, b) for t, b in zip(lens, ep.budget))
        self.Q_dec = torch.empty((L, Hq, N, D), dtype=dtype, device=dev)
        self.O = torch.empty((L, Hq, N, D), dtype=torch.float32, device=dev)
        self.lse = torch.empty((L, Hq, N), dtype=torch.float32, device=dev)
        self.workspace = torch.empty(
            max(E.ecokv_decode_shared_workspace_size(shape, self.fan, self.max_count, self.max_new), 256), dtype=torch.uint8, device=dev)

    def step(self, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, stream=None, max_tail: Optional[int] = None) -> torch.Tensor:
        """Append the next token of every continuation and attend; returns O."""
        if self.length >= self.max_new:
            raise ValueError(f"the tails hold {self.max_new} tokens")
        N = self.fan[-1]
        if isinstance(K, torch.Tensor) and K.shape[-3:-2] != (N,):  # (fewer would leave Q_dec laid out for fewer)
            raise ValueError(f"K has shape {tuple(K.shape)}, a step takes a token of each of the {N} continuations")
        self._stream = stream
        E.ecokv_append(Q, K, V, self.ep.shape, self.rope, self.positions, None, self.rows, self.tails, self.Q_dec, stream)
        E.ecokv_decode_shared(self.Q_dec, self.ep.Kc, self.ep.Vc, self.ep.shape, self.fan, self.ep.counts, self.ep.offsets, self.max_count,
                              self.tails, self.tail_counts, self.length + 1 if max_tail is None else max_tail, self.O, self.lse,
                              self.workspace, stream)
        return self.O

    def advance(self, stream=None) -> None:
        """On to the next token (enqueued on `stream`, or else on the last step's)."""
        with torch.cuda.stream(self._stream if stream is None else stream):  # (None: the current stream stays)
            self._at.add_(1)
        self.length += 1
