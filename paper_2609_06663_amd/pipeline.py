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
        self.evictions = 0  # by Continuations, which move rows of Kc and Vc

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

    Prompt s is continued by fan_out[s] continuations whose tails hold up to
    `max_new` tokens each, keys and values in pages; all continuations of a
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

    With `max_nodes` > 0 several drafted tokens of each continuation are attended
    at once: `tree` lays out what sees what, `draft` takes the place of `step` and
    `commit` of `advance`, which adds to each tail the nodes that were accepted,
    as many as there are.  With `masses`, `accumulate` after a step or a commit
    adds up what weight every row gets (`mass`, `tail_mass`; a row whose own step or
    commit was not accumulated begins with 0), and between tokens
    `evict` bounds the tails and `evict_kept` the prompts' rows (of the pass
    itself) by dropping those of the least: with a limit below `max_new`
    generation need not end.

    The calls only enqueue work, on one stream at a time (they share a
    workspace): `advance` goes where the last `step` went, to the stream that it
    was given or else to the current one.  Who changes the stream between calls
    orders the one after the other, and keeps this and the pass until other streams
    than the one it was made on have done their work.  To capture them in a HIP graph, pass them
    max_tail (max_new, or the limit's bound): by default it is the present length,
    which a replay would not raise.  A replay moves the device's counters only;
    `length`, the tails' rows or more, is the caller's to keep."""

    def __init__(self, ep: EvictionPass, fan_out, max_new: int, rope: E.Rope, page_size: int = 64, max_nodes: int = 0,
                 masses: bool = False):
        shape = ep.shape
        c = shape.c
        fan_out = E._flat_ints(fan_out)
        if len(fan_out) != c.num_seqs or min(fan_out) < 0:
            raise ValueError("fan_out has the number of continuations of each prompt")
        if sum(fan_out) < 1:
            raise ValueError("fan_out has no continuation")
        if max_new < 1:
            raise ValueError(f"max_new {max_new} < 1")
        if not 0 <= max_nodes <= E.MAX_NODES:
            raise ValueError(f"max_nodes {max_nodes} outside [0, {E.MAX_NODES}]")
        self.ep, self.rope, self.max_new, self.max_nodes, self.length = ep, rope, int(max_new), int(max_nodes), 0
        self._stream = None  # that the last step was given
        self._pending = None  # "step" or "draft": rows that are not the tails' yet
        self._unweighed = None  # "step", or the path of a commit: what accumulate may add
        self._ahead = False  # whether the masses behind the tails hold those of a step that was not advanced
        self.fan = [0]
        for f in fan_out:
            self.fan.append(self.fan[-1] + f)
        N, L, Hq, Hkv, D = self.fan[-1], c.num_layers, c.num_q_heads, c.num_kv_heads, c.head_dim
        dev, dtype = ep.Kc.device, ep.Kc.dtype
        per = -(-(self.max_new + self.max_nodes) // page_size)
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
        need = max(E.ecokv_decode_shared_workspace_size(shape, self.fan, self.max_count, self.max_new), 256)
        if self.max_nodes:
            need = max(need, E.ecokv_decode_tree_workspace_size(shape, self.fan, self.max_count, self.max_new, self.max_nodes))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        self._outgrown = []  # workspaces that a captured graph may still use
        self._captured = []  # trees that one reads
        # of drafts: of max_nodes nodes each, of fewer the beginning
        n = L * Hq * N * self.max_nodes
        self._nodes = torch.empty(n * D, dtype=dtype, device=dev), torch.empty(n * D, dtype=dtype, device=dev), torch.empty(n, device=dev)
        self.Q_nodes = self.O_nodes = self.lse_nodes = None
        self._taken = torch.zeros(N, dtype=torch.int32, device=dev)  # by the last commit
        self.mass = self.tail_mass = None
        if masses:
            self._evictions = ep.evictions
            self.mass = torch.zeros(ep.Kc.shape[0], dtype=torch.float32, device=dev)
            self.tail_mass = torch.zeros((L, N * per, Hkv, page_size), dtype=torch.float32, device=dev)

    def _need(self, nbytes: int, stream) -> None:
        """A workspace of nbytes (in order with `stream`, where it is given).  One that is
        too small makes way for one of twice its size at least: those that are kept are
        smaller together than the last."""
        if self.workspace.numel() < nbytes:
            self._outgrown.append(self.workspace)
            with torch.cuda.stream(stream):  # (None: the current stream stays)
                self.workspace = torch.empty(max(nbytes, 2 * self.workspace.numel()), dtype=torch.uint8, device=self.workspace.device)

    def step(self, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, stream=None, max_tail: Optional[int] = None) -> torch.Tensor:
        """Append the next token of every continuation and attend; returns O."""
        if self.length >= self.max_new:
            raise ValueError(f"the tails hold {self.max_new} tokens")
        N = self.fan[-1]
        if isinstance(K, torch.Tensor) and K.shape[-3:-2] != (N,):  # (fewer would leave Q_dec laid out for fewer)
            raise ValueError(f"K has shape {tuple(K.shape)}, a step takes a token of each of the {N} continuations")
        E.ecokv_append(Q, K, V, self.ep.shape, self.rope, self.positions, None, self.rows, self.tails, self.Q_dec, stream)
        self._appended(stream)
        E.ecokv_decode_shared(self.Q_dec, self.ep.Kc, self.ep.Vc, self.ep.shape, self.fan, self.ep.counts, self.ep.offsets, self.max_count,
                              self.tails, self.tail_counts, self.length + 1 if max_tail is None else max_tail, self.O, self.lse,
                              self.workspace, stream)
        self._pending = self._unweighed = "step"
        return self.O

    def advance(self, stream=None) -> None:
        """On to the next token (enqueued on `stream`, or else on the last step's)."""
        if self._pending == "draft":
            raise ValueError("a draft goes on with commit")
        with torch.cuda.stream(self._stream if stream is None else stream):  # (None: the current stream stays)
            self._at.add_(1)
        self._pending, self._ahead = None, False
        self.length += 1

    def tree(self, parents) -> "Tree":
        """Trees for `draft`: the parents of each node (earlier nodes, or -1: the tail's
        last token), one list for all continuations or one for each, of up to max_nodes
        nodes; where they differ in length, the shorter ones are padded."""
        N = self.fan[-1]
        lists = [list(p) for p in parents] if len(parents) and not isinstance(parents[0], int) else [list(parents)] * N
        if len(lists) != N:
            raise ValueError(f"{len(lists)} trees for {N} continuations")
        M = max(map(len, lists))
        if not 1 <= M <= self.max_nodes:
            raise ValueError(f"a tree of {M} nodes, max_nodes is {self.max_nodes}")
        return Tree(lists, M, self.rows.device)

    def draft(self, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, tree: "Tree", stream=None,
              max_tail: Optional[int] = None) -> torch.Tensor:
        """Append the nodes of every continuation's tree behind its tail and attend.
        Q, K, V: [L][N nodes][heads][D], node i of continuation c at c nodes + i (of
        padding, anything).  Returns O [L][H_q][N nodes][D] of the element type; it and
        lse_nodes stay until the next draft."""
        if self.length >= self.max_new:
            raise ValueError(f"the tails hold {self.max_new} tokens")
        c, N, M = self.ep.shape.c, self.fan[-1], tree.nodes
        if tree.masks.shape[0] != N or M > self.max_nodes:
            raise ValueError(f"trees of {tree.masks.shape[0]} continuations and {M} nodes, made for {N} and {self.max_nodes}")
        if isinstance(K, torch.Tensor) and K.shape[-3:-2] != (N * M,):
            raise ValueError(f"K has shape {tuple(K.shape)}, the draft has {N} x {M} nodes")
        L, Hq, D = c.num_layers, c.num_q_heads, c.head_dim
        n, max_tail = L * Hq * N * M, self.length if max_tail is None else max_tail
        Q_nodes, O_nodes = (t[:n * D].view(L, Hq, N * M, D) for t in self._nodes[:2])
        lse_nodes = self._nodes[2][:n].view(L, Hq, N * M)
        self._need(E.ecokv_decode_tree_workspace_size(self.ep.shape, self.fan, self.max_count, max_tail, M), stream)
        tree._used_on(stream)
        with torch.cuda.stream(stream):  # (None: the current stream stays)
            rows, positions = self._at[0::2, :, None] + tree.steps
            if tree.masks.is_cuda and torch.cuda.is_current_stream_capturing():
                self._captured.append(tree)
        E.ecokv_append(Q, K, V, self.ep.shape, self.rope, positions, tree.conts, rows, self.tails, Q_nodes, stream)
        self._appended(stream)
        E.ecokv_decode_tree(Q_nodes, self.ep.Kc, self.ep.Vc, self.ep.shape, self.fan, self.ep.counts, self.ep.offsets, self.max_count,
                            self.tails, self.rows, max_tail, tree.masks, O_nodes, lse_nodes, self.workspace, stream)
        self.Q_nodes, self.O_nodes, self.lse_nodes, self._pending = Q_nodes, O_nodes, lse_nodes, "draft"
        return O_nodes

    def commit(self, path: torch.Tensor, accepted: torch.Tensor, longest: Optional[int] = None, stream=None) -> None:
        """The accepted nodes of the draft become the tails' next rows: path int32
        [N][nodes], of which the first accepted[c] (int32 [N]) count, ascending.  Of a
        continuation with another path, or accepted[c] outside [0, nodes], none are.
        `longest`: the rows of the longest tail afterwards or more, where the caller
        knows better than `nodes` more than before."""
        if self._pending != "draft":
            raise ValueError("commit goes with a draft")
        N, M = self.fan[-1], self.lse_nodes.shape[2] // self.fan[-1]
        if tuple(path.shape) != (N, M):
            raise ValueError(f"path has shape {tuple(path.shape)}, the draft has ({N}, {M}) nodes")
        if not isinstance(accepted, torch.Tensor):
            raise TypeError("accepted must be a torch tensor")
        if tuple(accepted.shape) != (N,):
            raise ValueError(f"accepted has shape {tuple(accepted.shape)}, the call needs ({N},)")
        length = self.length + M if longest is None else min(self.length + M, int(longest))
        stream = self._stream if stream is None else stream
        with torch.cuda.stream(stream):
            self._taken.copy_(accepted)
        E.ecokv_commit(self.ep.shape, self.tails, self.rows, path, accepted, stream, taken=self._taken)
        _used_on(stream, path, accepted)
        with torch.cuda.stream(stream):
            self._at.add_(self._taken)
        self.length, self._pending, self._unweighed = length, None, (path, self._taken)

    def accumulate(self, decay: float = 1.0, stream=None, max_tail: Optional[int] = None) -> None:
        """Add the weights of the last step, or of the accepted nodes of the last
        commit, to the masses, once."""
        self._with_masses(False)
        if self._unweighed is None:
            raise ValueError("accumulate goes with a step or a commit, once")
        self._with_order()
        if self._unweighed == "step":
            Q, lse, path, accepted = self.Q_dec, self.lse, None, None
        else:
            Q, lse, (path, accepted) = self.Q_nodes, self.lse_nodes, self._unweighed
        # (a step's row is the tail's last, whether it was advanced or not)
        counts, most = (self.tail_counts, self.length + 1) if self._pending == "step" else (self.rows, self.length)
        stream = self._stream if stream is None else stream
        E.ecokv_accumulate(Q, lse, self.ep.Kc, self.ep.shape, self.fan, self.ep.counts, self.ep.offsets, self.max_count, self.tails, counts,
                           most if max_tail is None else max_tail, self.mass, self.tail_mass, path, accepted, decay, stream=stream)
        if path is not None:
            _used_on(stream, path, accepted)
        self._unweighed, self._ahead = None, self._pending == "step"

    def _appended(self, stream) -> None:
        """New queries and rows took the place of the last step's or draft's: what was not
        advanced, committed or accumulated of these is gone, whatever comes of the new
        ones, and a row of a step that was weighed and not advanced leaves no mass."""
        self._stream, self._pending, self._unweighed = stream, None, None
        if self._ahead:
            table, pages, size = self.tails.table, *self.tails.K.shape[1:4:2]
            with torch.cuda.stream(stream):
                i = torch.arange(max(table.shape[1], size), device=table.device)
                # the first row of each page that is behind its tail (of pages of nobody, none)
                first = torch.full((pages + 1,), size, dtype=torch.int64, device=table.device)
                page = torch.where((table >= 0) & (table < pages), table, pages).long()
                first.scatter_(0, page.flatten(), (self.rows.long()[:, None] - size * i[:table.shape[1]]).flatten())
                self.tail_mass.masked_fill_((i[:size] >= first[:pages, None])[None, :, None], 0)
            self._ahead = False

    def evict(self, limit: int, keep: int, recent: int, stream=None, max_tail: Optional[int] = None) -> None:
        """Tails of more than `limit` rows keep `keep` of them: the last `recent`, and of
        the others those of the largest mass."""
        self._with_masses(True)
        max_tail = self.length if max_tail is None else max_tail
        stream = self._stream if stream is None else stream
        self._need(E.ecokv_evict_workspace_size(self.ep.shape, self.fan[-1], max_tail, keep), stream)
        E.ecokv_evict_tails(self.ep.shape, self.tails, self.rows, max_tail, limit, keep, recent, self.tail_mass,
                            workspace=self.workspace, stream=stream)
        with torch.cuda.stream(stream):
            torch.add(self.rows, 1, out=self.tail_counts)
        self.length, self._unweighed = min(self.length, limit), None

    def evict_kept(self, limit: int, keep: int, recent: int, stream=None) -> None:
        """The same for the prompts' kept rows, each (layer, KV head, prompt) on its own:
        the pass's Kc, Vc and counts change, and other instances on it that have masses
        can no longer accumulate or evict those."""
        self._with_masses(True)
        self._with_order()
        shape = self.ep.shape
        stream = self._stream if stream is None else stream
        self._need(max(E.ecokv_evict_workspace_size(shape, shape.c.num_seqs, self.max_count, keep),
                       E.ecokv_decode_shared_workspace_size(shape, self.fan, min(self.max_count, limit), self.max_new)), stream)
        E.ecokv_evict(self.ep.Kc, self.ep.Vc, shape, self.ep.counts, self.ep.offsets, self.max_count, limit, keep, recent, self.mass,
                      workspace=self.workspace, stream=stream)
        self.max_count, self._unweighed = min(self.max_count, limit), None
        self._evictions = self.ep.evictions = self.ep.evictions + 1

    def _with_order(self) -> None:
        if self._evictions != self.ep.evictions:
            raise ValueError("another instance has moved the pass's rows since: `mass` is of their old order")

    def _with_masses(self, between: bool) -> None:
        if self.mass is None:
            raise ValueError("made without masses")
        if between and self._pending:
            raise ValueError(f"a {self._pending} is not finished: rows are evicted between tokens")


def _used_on(stream, *tensors: torch.Tensor) -> None:
    """A call on `stream` (None: the current one) reads these: whoever drops them, their
    memory is nobody else's before it has."""
    for t in tensors:
        if t.is_cuda:
            t.record_stream(torch.cuda.current_stream(t.device) if stream is None else stream)


class Tree:
    """Drafted trees of continuations on the device (made by Continuations.tree).  A draft
    that was enqueued does not need the Tree kept, nor does a captured one."""

    def __init__(self, parents, nodes: int, device):
        masks, steps = [], [[], []]  # (row behind the tail, depth)
        for p in parents:
            m, depths = E.ecokv_tree_masks(p) if p else ([], [])
            pad = nodes - len(p)
            masks.append(m + [0] * pad)
            steps[0].append(list(range(len(p))) + [-(1 << 30)] * pad)  # (a negative row is not written)
            steps[1].append(depths + [0] * pad)
        self.nodes = nodes
        self.masks = torch.tensor(masks, dtype=torch.int64, device=device)
        self.steps = torch.tensor(steps, dtype=torch.int32, device=device)
        self.conts = torch.tensor([c for c in range(len(parents)) for _ in range(nodes)], dtype=torch.int32, device=device)

    def _used_on(self, stream) -> None:
        _used_on(stream, self.masks, self.steps, self.conts)
