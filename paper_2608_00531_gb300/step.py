"""One CURE repair-verify step over a batch, through the C ABI.

``RepairVerifyStep`` owns the device buffers of every stage's outputs (and the
tree-attention workspace) for a fixed shape, and runs the six stages in order
on one stream:

  score_draft -> build_tree -> tree_attn x layers -> accept -> resync_kv

Inputs of a step (``StepInputs``) are the draft logits, the tree's target
Q/K/V per layer and the target logits; the KV caches are persistent state
owned by the caller.  Nothing here computes: every stage is a libcure call.
The Q/K/V may come as the rows of each layer's fused projection instead; the
step then norms and rotates them itself (``rope``).

``PromptPass`` fills the caches that a step starts from: the attention layers
of the target over packed prompts, chunks of prompts or single tokens.

Both also take caches held in 8 bits: float8_e4m3fn codes, and their scales
(``cure.kv8_scale_shape``) beside them.

``run_from_host`` takes the same inputs in (pinned) host memory and streams
them in on a copy stream in the order the stages consume them (draft logits,
then each layer's Q/K/V, then the target logits of the tree's nodes); each
stage waits only for its own inputs, so the copies overlap the stages before
them.
"""
from __future__ import annotations

import contextlib
import dataclasses
from typing import List, Optional

import torch

from . import cure


@dataclasses.dataclass
class StepInputs:
    draft_logits: torch.Tensor      # bf16 [B][K][V]
    root_tok: torch.Tensor          # int32 [B]
    cache_len: torch.Tensor         # int32 [B]
    redraft: Optional[torch.Tensor]  # int32 [B][K][branches-1] or None
    q: torch.Tensor                 # bf16 [layers][B][n_max][Hq][D]
    tree_k: torch.Tensor            # bf16 [layers][B][n_max][Hkv][D]
    tree_v: torch.Tensor            # bf16 [layers][B][n_max][Hkv][D]
    target_logits: torch.Tensor     # bf16 [B][n_max][V]
    # bf16 [layers][B][n_max][(Hq + 2 Hkv) D]: Q, K and V as the projections give them, before the head norms and the
    # rotation; q, tree_k and tree_v are then None
    qkv: Optional[torch.Tensor] = None
    # int32 [B]: the position of each sequence's root token where that is not its slot cache_len[b], as behind a prompt
    # whose images' tokens stand at fewer positions than they are (the `pos` and `axes` of PromptPass.layer); not negative.
    # The tree's tokens are text: they count on from there, the same on every axis, and so do the accepted ones.
    next_pos: Optional[torch.Tensor] = None


def _parts(qkv: torch.Tensor, heads_q: int, heads_kv: int, head_dim: int):
    """q, k and v [...][heads][D] within the rows of a fused projection."""
    if qkv.shape[-1] != (heads_q + 2 * heads_kv) * head_dim:
        raise ValueError("a projection's rows must hold (heads_q + 2 heads_kv) heads")
    x = qkv.unflatten(-1, (-1, head_dim))
    return (x[..., :heads_q, :], x[..., heads_q:heads_q + heads_kv, :], x[..., heads_q + heads_kv:, :])


def _of_layer(norms, l: int):
    return None if norms is None else norms[l]


class PromptPass:
    """The target's attention layers over packed rows (Alg. 1's input): per layer the head norms and the rotation,
    K and V behind what the cache holds, and causal attention over the cache.

    Sequence b's rows row_start[b] .. row_start[b+1] - 1 stand at positions cache_len[b], cache_len[b] + 1, ..; all
    layers run at the same lengths, and ``advance`` gives the lengths after the pass.  q_norm, k_norm: a weight
    (bf16 [D]) per layer, or None.  Up to 256 sequences and 2^22 rows, as cure_prompt_attn takes.  A pass holds the
    rotated rows and the attention's workspace: its layers run in one order, not on several streams at once."""

    def __init__(self, rows: int, batch: int, heads_q: int, kv: cure.KVDesc, rope: Optional[cure.Rope],
                 device: torch.device, q_norm=None, k_norm=None, eps: float = 1e-6):
        self.rows, self.B, self.Hq, self.kv, self.rope = rows, batch, heads_q, kv, rope
        self.q_norm, self.k_norm, self.eps = q_norm, k_norm, eps
        self.scale = 1.0 / float(kv.head_dim) ** 0.5
        ws = self._workspace_size(rows, batch)
        self.q = torch.empty(rows, heads_q, kv.head_dim, dtype=torch.bfloat16, device=device)
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=device)

    def _workspace_size(self, rows: int, batch: int) -> int:
        ws = cure.cure_prompt_attn_workspace_size(rows, batch, self.Hq, self.kv)
        if ws == 0:
            raise ValueError(f"PromptPass: cure_prompt_attn does not take {rows} rows of {batch} sequences with "
                             f"{self.Hq} / {self.kv.heads_kv} heads of {self.kv.head_dim}")
        return ws

    def layer(self, l: int, qkv: torch.Tensor, row_start: torch.Tensor, cache_len: torch.Tensor, k_cache: torch.Tensor,
              v_cache: torch.Tensor, *, scales=None, pos: Optional[torch.Tensor] = None,
              axes: Optional[cure.RopeAxes] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Layer l: qkv bf16 [rows][(Hq + 2 Hkv) D] -> attention output [rows][Hq][D]; the cache gains the rows.

        scales: (k_scale, v_scale) of a cache held in 8 bits.  pos, axes: the rows' positions, where they are not their
        places in their sequences (cure_append_kv); rows see the keys up to their own place whatever their positions,
        so none may be negative.  Steps behind such rows take the position that the text goes on from as
        StepInputs.next_pos."""
        n = qkv.shape[0]
        if n > self.rows:
            raise ValueError(f"PromptPass was made for {self.rows} rows, got {n}")
        q, k, v = _parts(qkv, self.Hq, self.kv.heads_kv, self.kv.head_dim)
        # what the attention would refuse is refused before anything is appended
        if cache_len.numel() > self.B:
            self._workspace_size(n, cache_len.numel())
        rows = self.q[:n]
        caches = (k_cache, v_cache) if scales is None else (k_cache, v_cache, *scales)
        of = cure._prompt_attn_args if scales is None else cure._prompt_attn8_args
        out, _, args = of(rows, *caches, self.kv, row_start, cache_len, self.scale, out, self.workspace, stream)
        if out.data_ptr() % 16:
            raise ValueError("out must be 16-byte aligned")
        append = cure.cure_append_kv if scales is None else cure.cure_append_kv8
        append(k, v, *caches, self.kv, row_start, cache_len, self.rope, q=q, pos=pos, axes=axes,
               q_norm=_of_layer(self.q_norm, l), k_norm=_of_layer(self.k_norm, l), eps=self.eps, out=rows,
               stream=stream)
        if scales is None:
            cure.check("cure_prompt_attn", cure._lib.load().cure_prompt_attn(*args))
        else:
            cure.check("cure_prompt_attn8", cure._lib.load().cure_prompt_attn8(*args))
        return out

    @staticmethod
    def advance(row_start: torch.Tensor, cache_len: torch.Tensor) -> torch.Tensor:
        """The lengths behind the appended rows."""
        return cache_len + (row_start[1:] - row_start[:-1])


class RepairVerifyStep:
    # target logits of at least this many bytes are copied by node rows
    NODE_ROWS_MIN_BYTES = 64 << 20

    def __init__(self, batch: int, block: int, vocab: int, topk: int, tau: float, budget: int,
                 branches: int, repair_depth: int, layers: int, heads_q: int, kv: cure.KVDesc,
                 device: torch.device, max_ufp: int = 0, layer_map: Optional[List[int]] = None,
                 rope: Optional[cure.Rope] = None, q_norm=None, k_norm=None, eps: float = 1e-6):
        self.B, self.K, self.V, self.k = batch, block, vocab, topk
        self.tau, self.R, self.branches, self.depth = tau, budget, branches, repair_depth
        self.max_ufp = max_ufp
        self.layers, self.Hq, self.kv = layers, heads_q, kv
        self.n_max = 1 + block + budget
        self.D = kv.head_dim
        self.scale = 1.0 / float(self.D) ** 0.5
        # logical layer -> physical cache index (aliasing when the caches of all
        # layers do not fit in device memory)
        self.layer_map = layer_map or list(range(layers))
        dev = device
        B, K, N = batch, block, self.n_max
        W = (N + 63) // 64
        i32 = dict(dtype=torch.int32, device=dev)
        self.score = (torch.empty(B, K, topk, **i32), torch.empty(B, K, topk, dtype=torch.float32, device=dev),
                      torch.empty(B, K, dtype=torch.float32, device=dev),
                      torch.empty(B, K, dtype=torch.float32, device=dev))
        self.tree = dict(n_nodes=torch.empty(B, **i32), tok=torch.empty(B, N, **i32),
                         pos=torch.empty(B, N, **i32), parent=torch.empty(B, N, **i32),
                         depth=torch.empty(B, N, **i32),
                         anc=torch.empty(B, N, W, dtype=torch.int64, device=dev),
                         ufp_pos=torch.empty(B, K, **i32), n_ufp=torch.empty(B, **i32))
        self.attn_out = torch.empty(layers, B, N, heads_q, self.D, dtype=torch.bfloat16, device=dev)
        ws = cure.cure_tree_attn_workspace_size(B, N, heads_q, kv)
        self.workspace = torch.empty(max(ws, 256), dtype=torch.uint8, device=dev)
        self.targ = torch.empty(B, N, **i32)
        P = K + 2
        self.acc = dict(accept_len=torch.empty(B, **i32), best_node=torch.empty(B, **i32),
                        path_nodes=torch.empty(B, P, **i32), out_tokens=torch.empty(B, P, **i32),
                        diverge_depth=torch.empty(B, **i32))
        self.rs = dict(draft_valid_len=torch.empty(B, **i32), replay_tokens=torch.empty(B, P, **i32),
                       n_replay=torch.empty(B, **i32))
        self.cache_len_out = torch.empty(B, **i32)
        # for inputs that come as projections: the rotation, norm weights per layer, and the rows made of them
        self.rope, self.q_norm, self.k_norm, self.eps = rope, q_norm, k_norm, eps
        self._rows = None
        # for caches in 8 bits: the trees' rows in a packed batch, the workspace, what the sequences' last blocks hold
        self._starts = self._workspace8 = self._held = None
        self._more_launches = 0  # of the last step
        self._dev_inputs = None
        self._copy_stream = None
        self._n_host = None
        self.last_h2d_bytes = 0  # host-to-device bytes of the last run_from_host

    def run(self, x: StepInputs, k_caches: List[torch.Tensor], v_caches: List[torch.Tensor],
            stream=None, scales=None) -> dict:
        """One step.  scales: (k_scales, v_scales), a tensor for each cache, where the caches are held in 8 bits; the
        tree's rows then go into the caches, behind the sequences' tokens (where there must be room for all of a
        sequence's nodes), and are attended to there.  They leave
        the caches again before the accepted path's rows are written: what a sequence holds keeps its codes and scales
        whatever the rejected rows are.  (The step's own attention reads a sequence's last, shared block under the scale
        that all of its rows give it.)  Layers that share a cache (layer_map) cannot be held in 8 bits."""
        if scales is not None and len(set(self.layer_map[:self.layers])) < self.layers:
            raise ValueError("layers that share a cache cannot be held in 8 bits")
        root_pos = x.cache_len if x.next_pos is None else x.next_pos
        if x.next_pos is not None:
            cure._sized(x.next_pos, "next_pos", self.B, cure._current(stream)[0])
        ids, vals, margin, logp1 = cure.cure_score_draft(x.draft_logits, self.k, out=self.score,
                                                         stream=stream)
        tree = cure.cure_build_tree(ids, margin, x.root_tok, root_pos, self.tau, self.R,
                                    self.branches, self.depth, x.redraft, self.max_ufp,
                                    out=self.tree, stream=stream)
        kl = [k_caches[self.layer_map[l]] for l in range(self.layers)]
        vl = [v_caches[self.layer_map[l]] for l in range(self.layers)]
        self._more_launches = (0 if x.qkv is None else self.layers) + (0 if scales is None else self.layers + 3)
        if x.qkv is not None:
            x = self._rotate(x, tree["pos"], stream)
        if scales is not None:
            sl = [[t[self.layer_map[l]] for l in range(self.layers)] for t in scales]
            self._attend8(x, kl, vl, *sl, tree, stream)
        elif all(isinstance(t, torch.Tensor) and t.is_contiguous() and t.dim() == 5 and t.shape[0] == self.layers
               for t in (x.q, x.tree_k, x.tree_v)):
            cure.cure_tree_attn_layers(x.q, x.tree_k, x.tree_v, kl, vl, self.kv, x.cache_len, tree["n_nodes"],
                                       tree["anc"], self.scale, self.attn_out, self.workspace, stream=stream)
        else:  # layers apart in memory
            for l in range(self.layers):
                cure.cure_tree_attn(x.q[l], x.tree_k[l], x.tree_v[l], kl[l], vl[l], self.kv, x.cache_len,
                                    tree["n_nodes"], tree["anc"], self.scale, out=self.attn_out[l],
                                    workspace=self.workspace, stream=stream)
        acc = cure.cure_accept(tree, self.K, target_logits=x.target_logits, targ=self.targ,
                               out=self.acc, stream=stream)
        if scales is not None:
            rs = cure.cure_resync_kv8(kl, vl, *sl, self.kv, x.tree_k, x.tree_v, acc, x.cache_len, self.K,
                                      cache_len_out=self.cache_len_out, out=self.rs, stream=stream)
        else:
            rs = cure.cure_resync_kv(kl, vl, self.kv, x.tree_k, x.tree_v, acc, x.cache_len, self.K,
                                     cache_len_out=self.cache_len_out, out=self.rs, stream=stream)
        return dict(score=self.score, tree=tree, attn=self.attn_out, acc=acc, resync=rs)

    def _attend8(self, x: StepInputs, kl, vl, ksl, vsl, tree: dict, stream) -> None:
        """The layers' tree attention over caches in 8 bits, each layer's tree rows appended in place before it.  A
        tree's first rows share a block, and its scale, with a sequence's last tokens: those are saved before, and put
        back behind the attention, also where a call of it is refused."""
        if self._starts is None:
            with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
                if torch.cuda.is_current_stream_capturing():
                    raise RuntimeError("a step over caches in 8 bits must have run once before it is captured")
                dev = self.attn_out.device
                self._starts = torch.arange(0, (self.B + 1) * self.n_max, self.n_max, dtype=torch.int32, device=dev)
                size = cure.cure_tree_attn8_workspace_size(self.B, self.n_max, self.Hq, self.kv)
                self._workspace8 = torch.empty(max(size, 256), dtype=torch.uint8, device=dev)
                self._held = torch.empty(max(cure.cure_save_kv8_size(self.layers, self.B, self.kv), 256),
                                         dtype=torch.uint8, device=dev)
        dev, s = cure._current(stream)
        of = cure._layers8(kl, vl, ksl, vsl, self.kv, self.B, dev)
        cure._held8("cure_save_kv8", of, self.kv, self.B, x.cache_len, self._held, dev, s)
        try:
            for l in range(self.layers):
                caches = (kl[l], vl[l], ksl[l], vsl[l])
                cure.cure_append_kv8(x.tree_k[l], x.tree_v[l], *caches, self.kv, self._starts, x.cache_len, None,
                                     pos=tree["pos"], stream=stream)
                cure.cure_tree_attn8(x.q[l], *caches, self.kv, x.cache_len, tree["n_nodes"], tree["anc"], self.scale,
                                     out=self.attn_out[l], workspace=self._workspace8, stream=stream)
        finally:
            cure._held8("cure_restore_kv8", of, self.kv, self.B, x.cache_len, self._held, dev, s)

    def _rotate(self, x: StepInputs, pos: torch.Tensor, stream) -> StepInputs:
        """The step's Q/K/V from the layers' projections at the tree's positions (``StepInputs.next_pos`` where those
        are not slots; rows past a sequence's nodes keep what they held)."""
        if x.qkv.shape[:3] != (self.layers, self.B, self.n_max):
            raise ValueError("qkv must be [layers][batch][n_max][..]")
        if self._rows is None:
            with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
                if torch.cuda.is_current_stream_capturing():  # the zeros would be part of the graph, not of the step
                    raise RuntimeError("a step from projections must have run once before it is captured")
                self._rows = [torch.zeros(self.layers, self.B, self.n_max, h, self.D, dtype=torch.bfloat16,
                                          device=self.attn_out.device)
                              for h in (self.Hq, self.kv.heads_kv, self.kv.heads_kv)]
        for l in range(self.layers):
            cure.cure_rope_qkv(*_parts(x.qkv[l], self.Hq, self.kv.heads_kv, self.D), pos, self.rope,
                               q_norm=_of_layer(self.q_norm, l), k_norm=_of_layer(self.k_norm, l), eps=self.eps,
                               out=tuple(t[l] for t in self._rows), stream=stream)
        q, tk, tv = self._rows
        return dataclasses.replace(x, q=q, tree_k=tk, tree_v=tv, qkv=None)

    def run_from_host(self, xh: StepInputs, k_caches: List[torch.Tensor], v_caches: List[torch.Tensor],
                      stream=None) -> dict:
        """One step with its inputs in host memory (pinned, for copies that
        overlap the stages): copies on a side stream, each stage waiting for
        the copy of its own inputs.  When the target logits are large (at
        least NODE_ROWS_MIN_BYTES), only the rows of the tree's nodes are
        copied (rows j < n_nodes[b] of each sequence, the rows stage 5 reads):
        their count is known once the tree is built, so the host reads the
        node counts back before it queues those copies, behind the layers'
        Q/K/V.  Smaller ones are copied whole, without that read-back.
        Results stay on the device, as in run()."""
        if xh.qkv is not None:
            raise ValueError("run_from_host takes q, tree_k and tree_v, not the layers' projections")
        if xh.next_pos is not None and (xh.next_pos.dtype is not torch.int32 or xh.next_pos.numel() != self.B):
            raise ValueError(f"next_pos must hold {self.B} int32 positions")
        fields = ("draft_logits", "root_tok", "cache_len", "q", "tree_k", "tree_v", "target_logits")
        dev = self.attn_out.device
        if self._dev_inputs is None or any(self._dev_inputs[f].shape != getattr(xh, f).shape for f in fields):
            self._dev_inputs = {f: torch.empty(getattr(xh, f).shape, dtype=getattr(xh, f).dtype, device=dev)
                                for f in fields}
            self._copy_stream = torch.cuda.Stream(device=dev)
        if self._n_host is None:
            self._n_host = torch.empty(self.B, dtype=torch.int32).pin_memory()
        d = self._dev_inputs
        main = stream if stream is not None else torch.cuda.current_stream(dev)
        cs = self._copy_stream
        cs.wait_stream(main)  # the previous step's reads of the staging buffers come first
        ev_first = torch.cuda.Event()
        ev_layer = [torch.cuda.Event() for _ in range(self.layers)]
        ev_nodes = torch.cuda.Event()
        ev_target = torch.cuda.Event()
        h2d = 0
        with torch.cuda.stream(cs):
            for f in ("draft_logits", "root_tok", "cache_len"):
                d[f].copy_(getattr(xh, f), non_blocking=True)
                h2d += getattr(xh, f).numel() * getattr(xh, f).element_size()
            ev_first.record(cs)
            for l in range(self.layers):
                for f in ("q", "tree_k", "tree_v"):
                    d[f][l].copy_(getattr(xh, f)[l], non_blocking=True)
                    h2d += getattr(xh, f)[l].numel() * getattr(xh, f)[l].element_size()
                ev_layer[l].record(cs)
        redraft = None
        if xh.redraft is not None:
            redraft = xh.redraft.to(dev, non_blocking=True)
            h2d += xh.redraft.numel() * xh.redraft.element_size()
        x = StepInputs(d["draft_logits"], d["root_tok"], d["cache_len"], redraft, d["q"], d["tree_k"],
                       d["tree_v"], d["target_logits"])
        with torch.cuda.stream(main):
            main.wait_event(ev_first)
            root_pos = x.cache_len
            if xh.next_pos is not None:
                root_pos = xh.next_pos.to(dev, non_blocking=True)
                h2d += xh.next_pos.numel() * 4
            ids, vals, margin, logp1 = cure.cure_score_draft(x.draft_logits, self.k, out=self.score,
                                                             stream=main)
            tree = cure.cure_build_tree(ids, margin, x.root_tok, root_pos, self.tau, self.R,
                                        self.branches, self.depth, x.redraft, self.max_ufp,
                                        out=self.tree, stream=main)
            node_rows = xh.target_logits.numel() * xh.target_logits.element_size() >= self.NODE_ROWS_MIN_BYTES
            if node_rows:
                self._n_host.copy_(tree["n_nodes"], non_blocking=True)
                ev_nodes.record(main)
            for l in range(self.layers):
                main.wait_event(ev_layer[l])
                p = self.layer_map[l]
                cure.cure_tree_attn(x.q[l], x.tree_k[l], x.tree_v[l], k_caches[p], v_caches[p], self.kv,
                                    x.cache_len, tree["n_nodes"], tree["anc"], self.scale,
                                    out=self.attn_out[l], workspace=self.workspace, stream=main)
        with torch.cuda.stream(cs):
            if node_rows:
                ev_nodes.synchronize()
                n_max = xh.target_logits.shape[1]
                row_bytes = xh.target_logits.shape[2] * xh.target_logits.element_size()
                for b, nb in enumerate(self._n_host.tolist()):
                    nb = max(0, min(int(nb), n_max))
                    if nb:
                        d["target_logits"][b, :nb].copy_(xh.target_logits[b, :nb], non_blocking=True)
                        h2d += nb * row_bytes
            else:
                d["target_logits"].copy_(xh.target_logits, non_blocking=True)
                h2d += xh.target_logits.numel() * xh.target_logits.element_size()
            ev_target.record(cs)
        with torch.cuda.stream(main):
            main.wait_event(ev_target)
            acc = cure.cure_accept(tree, self.K, target_logits=x.target_logits, targ=self.targ,
                                   out=self.acc, stream=main)
            kl = [k_caches[self.layer_map[l]] for l in range(self.layers)]
            vl = [v_caches[self.layer_map[l]] for l in range(self.layers)]
            rs = cure.cure_resync_kv(kl, vl, self.kv, x.tree_k, x.tree_v, acc, x.cache_len, self.K,
                                     cache_len_out=self.cache_len_out, out=self.rs, stream=main)
        self.last_h2d_bytes = h2d
        self._more_launches = 0
        return dict(score=self.score, tree=tree, attn=self.attn_out, acc=acc, resync=rs)

    @property
    def launches_per_step(self) -> int:
        """Library kernels that a step like the last one launches (before the first: one over bf16 caches, from Q, K and V):
        scan, tree, one attention kernel per layer, target argmax + walk, and the resync gather (its finalize runs in
        the gather's grid, since the step's new lengths do not alias the old).
        Inputs that come as projections take one more per layer; caches in 8 bits one more per layer, and three in all
        (what the last blocks hold saved and put back, the lengths)."""
        return 1 + 1 + self.layers + 2 + 1 + self._more_launches
