"""Python binding of the C ABI (include/cure.h), one function per entry point.

Argument marshalling only: every stage runs in the CUDA kernels of
libcure.so.  Tensors must live on the current CUDA device; outputs are
allocated with torch when not given.  Calls are asynchronous on the current
torch stream (or the ``stream`` argument).
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from . import _lib
from ._lib import KVDesc, Rope, RopeAxes, RopeScaling, TreeParams, check

_BF16, _I32, _F32, _E4M3 = torch.bfloat16, torch.int32, torch.float32, torch.float8_e4m3fn

DEVERR_PAGE, DEVERR_SLOT, DEVERR_NODES = _lib.DEVERR_PAGE, _lib.DEVERR_SLOT, _lib.DEVERR_NODES


def _stream(stream) -> int:
    if stream is None:
        # the raw handle: a Stream object per call costs more than the launch of a small kernel
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _p(t: Optional[torch.Tensor]) -> Optional[int]:
    """Address of a tensor for the c_void_p arguments (plain ints, which ctypes converts in C)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libcure takes CUDA tensors")
    if not t.is_contiguous():
        raise ValueError("libcure takes contiguous tensors")
    return t.data_ptr()


def _need(t: torch.Tensor, dtype, name: str) -> None:
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


def kv_desc(heads_kv: int, head_dim: int, max_len: int, block_table: Optional[torch.Tensor] = None,
            page_size: int = 16, num_pages: int = 0) -> KVDesc:
    """Cache geometry: contiguous [B][max_len][Hkv][D], or paged [num_pages][page_size][Hkv][D]
    with block_table int32 [B][max_len] (then max_len counts pages)."""
    d = KVDesc()
    d.layout = 0 if block_table is None else 1
    d.heads_kv, d.head_dim, d.max_len = heads_kv, head_dim, max_len
    d.page_size = page_size
    d.num_pages = num_pages
    if block_table is not None:
        _need(block_table, torch.int32, "block_table")
        d.block_table = _p(block_table)
        d._keep = block_table  # keep the table alive with the descriptor
    return d


def cure_score_draft(logits: torch.Tensor, topk: int, *, out=None, stream=None):
    """Stage 1 (Sec. 3.3, Eq. 2): (top_ids, top_vals, margin, logp1) per row."""
    _need(logits, torch.bfloat16, "logits")
    V = logits.shape[-1]
    lead = logits.shape[:-1]
    rows = logits.numel() // V if V else 0
    dev = logits.device
    if out is None:
        out = (torch.empty(*lead, topk, dtype=torch.int32, device=dev),
               torch.empty(*lead, topk, dtype=torch.float32, device=dev),
               torch.empty(*lead, dtype=torch.float32, device=dev),
               torch.empty(*lead, dtype=torch.float32, device=dev))
    ids, vals, margin, logp1 = out
    lib = _lib.load()
    check("cure_score_draft", lib.cure_score_draft(_p(logits), rows, V, topk, _p(ids), _p(vals),
                                                   _p(margin), _p(logp1), _stream(stream)))
    return ids, vals, margin, logp1


def tree_params(batch, block, topk, tau, budget, branches, repair_depth=1, max_ufp=0,
                margin_scale=0.0, branch_min=1, max_depth=0, beam=0) -> TreeParams:
    p = TreeParams()
    p.batch, p.block, p.topk, p.tau = batch, block, topk, float(tau)
    p.budget, p.branches, p.repair_depth, p.max_ufp = budget, branches, repair_depth, max_ufp
    p.margin_scale, p.branch_min = float(margin_scale), branch_min
    p.max_depth, p.beam = max_depth, beam
    return p


def cure_build_tree(top_ids: torch.Tensor, margin: torch.Tensor, root_tok: torch.Tensor,
                    cache_len: torch.Tensor, tau: float, budget: int, branches: int,
                    repair_depth: int = 1, redraft: Optional[torch.Tensor] = None,
                    max_ufp: int = 0, margin_scale: float = 0.0, branch_min: int = 1,
                    max_depth: int = 0, beam: int = 0, *, out=None, stream=None) -> dict:
    """Stages 2+3 (Sec. 3.1 Eq. 1, Sec. 3.3, Sec. 3.4): the flattened repair tree.

    margin_scale > 0 turns on the dynamic branch budget of Eq. (3): UFP i then
    offers b_i alternatives, from branch_min up to branches - 1.  max_depth and
    beam (0 = none) are the structural caps on repair branches (Sec. 3.3-3.4)."""
    _need(top_ids, torch.int32, "top_ids")
    _need(margin, torch.float32, "margin")
    B, K, k = top_ids.shape
    n_max = 1 + K + budget
    W = (n_max + 63) // 64
    dev = top_ids.device
    if out is None:
        out = dict(n_nodes=torch.empty(B, dtype=torch.int32, device=dev),
                   tok=torch.empty(B, n_max, dtype=torch.int32, device=dev),
                   pos=torch.empty(B, n_max, dtype=torch.int32, device=dev),
                   parent=torch.empty(B, n_max, dtype=torch.int32, device=dev),
                   depth=torch.empty(B, n_max, dtype=torch.int32, device=dev),
                   anc=torch.empty(B, n_max, W, dtype=torch.int64, device=dev),
                   ufp_pos=torch.empty(B, K, dtype=torch.int32, device=dev),
                   n_ufp=torch.empty(B, dtype=torch.int32, device=dev))
    p = tree_params(B, K, k, tau, budget, branches, repair_depth, max_ufp, margin_scale, branch_min,
                    max_depth, beam)
    lib = _lib.load()
    check("cure_build_tree", lib.cure_build_tree(
        C.byref(p), _p(top_ids), _p(margin), _p(root_tok), _p(cache_len), _p(redraft),
        _p(out["n_nodes"]), _p(out["tok"]), _p(out["pos"]), _p(out["parent"]), _p(out["depth"]),
        _p(out["anc"]), _p(out["ufp_pos"]), _p(out["n_ufp"]), _stream(stream)))
    return out


def cure_tree_attn_workspace_size(batch: int, n_max: int, heads_q: int, kv: KVDesc) -> int:
    return int(_lib.load().cure_tree_attn_workspace_size(batch, n_max, heads_q, C.byref(kv)))


def cure_tree_attn(q: torch.Tensor, tree_k: Optional[torch.Tensor], tree_v: Optional[torch.Tensor],
                   k_cache: torch.Tensor, v_cache: torch.Tensor, kv: KVDesc,
                   cache_len: torch.Tensor, n_nodes: torch.Tensor, anc: torch.Tensor,
                   scale: float, *, out: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Stage 4 (Sec. 3.2/3.4/3.5): tree-masked GQA attention for one layer.

    tree_k = tree_v = None: the in-place layout, node j's K/V rows at cache
    slot cache_len[b] + j."""
    _need(q, torch.bfloat16, "q")
    if tree_k is not None:
        _need(tree_k, torch.bfloat16, "tree_k")
    if tree_v is not None:
        _need(tree_v, torch.bfloat16, "tree_v")
    _need(k_cache, torch.bfloat16, "k_cache")
    _need(v_cache, torch.bfloat16, "v_cache")
    B, n_max, Hq, D = q.shape
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        need = cure_tree_attn_workspace_size(B, n_max, Hq, kv)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    lib = _lib.load()
    check("cure_tree_attn", lib.cure_tree_attn(
        _p(q), _p(tree_k), _p(tree_v), _p(k_cache), _p(v_cache), C.byref(kv), _p(cache_len),
        _p(n_nodes), _p(anc), B, n_max, Hq, float(scale), _p(out), _p(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))
    return out


def cure_tree_attn_layers(q: torch.Tensor, tree_k: torch.Tensor, tree_v: torch.Tensor,
                          k_caches: Sequence[torch.Tensor], v_caches: Sequence[torch.Tensor], kv: KVDesc,
                          cache_len: torch.Tensor, n_nodes: torch.Tensor, anc: torch.Tensor, scale: float,
                          out: torch.Tensor, workspace: torch.Tensor, *, stream=None) -> torch.Tensor:
    """cure_tree_attn of every layer in turn: q, tree_k, tree_v and out are
    contiguous [layers][...] tensors, the caches one tensor per layer.  The
    arguments that the layers share are checked and converted once, and a
    layer's rows are addressed without making views: at one sequence the host
    work of a call would otherwise outlast its kernel."""
    for t, nm in ((q, "q"), (tree_k, "tree_k"), (tree_v, "tree_v"), (out, "out")):
        _need(t, torch.bfloat16, nm)
    layers, B, n_max, Hq, _ = q.shape
    if not (len(k_caches) == len(v_caches) == tree_k.shape[0] == tree_v.shape[0] == out.shape[0] == layers):
        raise ValueError("cure_tree_attn_layers: one cache and one slice per layer")
    ptrs = [_p(t) for t in (q, tree_k, tree_v, out)]
    steps = [t.stride(0) * 2 for t in (q, tree_k, tree_v, out)]  # bf16
    shared = (C.byref(kv), _p(cache_len), _p(n_nodes), _p(anc), B, n_max, Hq, float(scale))
    ws, ws_bytes, s = _p(workspace), workspace.numel() * workspace.element_size(), _stream(stream)
    fn = _lib.load().cure_tree_attn
    (pq, ptk, ptv, po), (sq, stk, stv, so) = ptrs, steps
    for l in range(layers):
        k, v = k_caches[l], v_caches[l]
        _need(k, torch.bfloat16, "k_cache")
        _need(v, torch.bfloat16, "v_cache")
        check("cure_tree_attn", fn(pq + l * sq, ptk + l * stk, ptv + l * stv, _p(k), _p(v), *shared, po + l * so,
                                   ws, ws_bytes, s))
    return out


def cure_accept(tree: dict, block: int, *, target_logits: Optional[torch.Tensor] = None,
                targ: Optional[torch.Tensor] = None, out=None, stream=None) -> dict:
    """Stage 5 (Sec. 3.5 Eq. 4): target argmax per node and the longest accepted path.

    Give ``target_logits`` (bf16 [B][n_max][V]) to compute the argmax, or
    ``targ`` (int32 [B][n_max]) already holding the target's tokens.
    """
    B, n_max = tree["tok"].shape
    dev = tree["tok"].device
    V = 0
    if target_logits is not None:
        _need(target_logits, torch.bfloat16, "target_logits")
        V = target_logits.shape[-1]
        if targ is None:
            targ = torch.empty(B, n_max, dtype=torch.int32, device=dev)
    elif targ is None:
        raise ValueError("cure_accept needs target_logits or targ")
    P = block + 2
    if out is None:
        out = dict(accept_len=torch.empty(B, dtype=torch.int32, device=dev),
                   best_node=torch.empty(B, dtype=torch.int32, device=dev),
                   path_nodes=torch.empty(B, P, dtype=torch.int32, device=dev),
                   out_tokens=torch.empty(B, P, dtype=torch.int32, device=dev),
                   diverge_depth=torch.empty(B, dtype=torch.int32, device=dev))
    lib = _lib.load()
    check("cure_accept", lib.cure_accept(
        _p(target_logits), _p(targ), B, n_max, V, block, _p(tree["n_nodes"]), _p(tree["tok"]),
        _p(tree["parent"]), _p(tree["depth"]), _p(tree["anc"]), _p(out["accept_len"]),
        _p(out["best_node"]), _p(out["path_nodes"]), _p(out["out_tokens"]),
        _p(out["diverge_depth"]), _stream(stream)))
    out["targ"] = targ
    return out


def cure_sample_target(target_logits: torch.Tensor, n_nodes: torch.Tensor, uniforms: torch.Tensor,
                       temperature: float, *, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Stochastic verification (Sec. 2, T > 0): the target's token at every tree
    node sampled by inverse CDF with uniforms[b][j]; pass the result to
    cure_accept as ``targ`` (without target_logits) for the walk."""
    _need(target_logits, torch.bfloat16, "target_logits")
    _need(uniforms, torch.float32, "uniforms")
    B, n_max, V = target_logits.shape
    if out is None:
        out = torch.empty(B, n_max, dtype=torch.int32, device=target_logits.device)
    lib = _lib.load()
    check("cure_sample_target", lib.cure_sample_target(
        _p(target_logits), _p(uniforms), float(temperature), B, n_max, V, _p(n_nodes), _p(out),
        _stream(stream)))
    return out


def cure_lm_head_workspace_size(rows: int, vocab: int) -> int:
    return int(_lib.load().cure_lm_head_workspace_size(rows, vocab))


def cure_lm_head_argmax(hidden: torch.Tensor, w_lm: torch.Tensor, *, out_index: Optional[torch.Tensor] = None,
                        out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """Stage 5 fused with the LM head (Sec. 3.5, Sec. 4.1): the first argmax of
    hidden[r] . w_lm[v] over v for every row, without writing the logits.

    hidden bf16 [rows][d_model], w_lm bf16 [vocab][d_model].  ``out_index``
    (int32 [rows]) places row r at out.view(-1)[out_index[r]]; without it the
    result is int32 [rows].
    """
    _need(hidden, torch.bfloat16, "hidden")
    _need(w_lm, torch.bfloat16, "w_lm")
    rows, d = hidden.shape
    V = w_lm.shape[0]
    dev = hidden.device
    if out is None:
        out = torch.empty(rows, dtype=torch.int32, device=dev)
    lib = _lib.load()
    ws = int(lib.cure_lm_head_workspace_size(rows, V))
    if workspace is None or workspace.numel() < ws:
        workspace = torch.empty(max(ws, 256), dtype=torch.uint8, device=dev)
    check("cure_lm_head_argmax", lib.cure_lm_head_argmax(
        _p(hidden), _p(w_lm), rows, d, V, _p(out_index), _p(out), _p(workspace), workspace.numel(),
        _stream(stream)))
    return out


def cure_resync_kv(k_caches: Sequence[torch.Tensor], v_caches: Sequence[torch.Tensor], kv: KVDesc,
                   tree_k: Optional[torch.Tensor], tree_v: Optional[torch.Tensor], acc: dict,
                   cache_len_in: torch.Tensor, block: int, *, n_max: Optional[int] = None,
                   cache_len_out: Optional[torch.Tensor] = None, out=None, stream=None) -> dict:
    """Stage 6 (Sec. 3.5, Alg. 1): write the path into every layer's cache, realign the draft.

    tree_k/tree_v: bf16 [layers][B][n_max][Hkv][D], or None for the in-place
    layout (the path rows are then read from cache slots L + node, and only
    the rows past the divergence move; give n_max).
    """
    layers = len(k_caches)
    B = cache_len_in.shape[0]
    if n_max is None:
        if layers and tree_k is None:
            raise ValueError("cure_resync_kv: the in-place layout needs n_max")
        n_max = tree_k.shape[2] if layers else block + 1
    dev = cache_len_in.device
    P = block + 2
    if cache_len_out is None:
        cache_len_out = torch.empty_like(cache_len_in)
    if out is None:
        out = dict(draft_valid_len=torch.empty(B, dtype=torch.int32, device=dev),
                   replay_tokens=torch.empty(B, P, dtype=torch.int32, device=dev),
                   n_replay=torch.empty(B, dtype=torch.int32, device=dev))
    kp = (C.c_void_p * max(1, layers))(*[_p(t) for t in k_caches])
    vp = (C.c_void_p * max(1, layers))(*[_p(t) for t in v_caches])
    lib = _lib.load()
    check("cure_resync_kv", lib.cure_resync_kv(
        layers, kp, vp, C.byref(kv), _p(tree_k), _p(tree_v), B, n_max, block,
        _p(acc["path_nodes"]), _p(acc["accept_len"]), _p(acc["diverge_depth"]),
        _p(acc["out_tokens"]), _p(cache_len_in), _p(cache_len_out), _p(out["draft_valid_len"]),
        _p(out["replay_tokens"]), _p(out["n_replay"]), _stream(stream)))
    out["cache_len"] = cache_len_out
    return out


_SCALINGS = {"linear": 1, "base": 2, "bands": 3, "ramp": 4}


def rope_desc(rot_dim: int = 128, base: float = 10000.0, *, style: str = "half", scaling: Optional[dict] = None,
              amplitude: float = 1.0, freqs: Optional[Sequence[float]] = None) -> Rope:
    """The rotation of a head's first ``rot_dim`` values, a host struct to keep with the model: pairs
    (i, i + rot_dim / 2) with style "half", (2i, 2i + 1) with "interleaved".

    The frequencies are base^(-2i / rot_dim), scaled by ``scaling``: dict(kind="linear" | "base", factor=) or
    dict(kind="bands" | "ramp", factor=, low=, high=, original=) (the formulas are in include/cure.h; "ramp" also
    takes its two numbers of turns as slow= and fast=).  Or they are ``freqs``, rot_dim / 2 values in radians per
    position.  ``amplitude`` multiplies cosines and sines."""
    if style not in ("half", "interleaved"):
        raise ValueError(f"rope_desc: style must be 'half' or 'interleaved', got {style!r}")
    st, r, lib = int(style == "interleaved"), Rope(), _lib.load()
    if freqs is not None:
        if scaling is not None:
            raise ValueError("rope_desc: freqs are taken as they are; scaling goes with base")
        f = [float(x) for x in freqs]
        if len(f) != rot_dim // 2:
            raise ValueError(f"rope_desc: {rot_dim // 2} frequencies expected, got {len(f)}")
        check("cure_rope_init_freqs", lib.cure_rope_init_freqs(C.byref(r), st, rot_dim, (C.c_double * max(1, len(f)))(*f),
                                                               float(amplitude)))
        return r
    sc = None
    if scaling is not None:
        d = dict(scaling)
        kind = d.pop("kind", None)
        if kind not in _SCALINGS:
            raise ValueError(f"rope_desc: unknown scaling {kind!r}")
        if kind == "ramp":
            d = {dict(slow="low", fast="high").get(k, k): v for k, v in d.items()}
        want = {"factor"} | ({"low", "high", "original"} if kind in ("bands", "ramp") else set())
        if set(d) != want:
            raise ValueError(f"rope_desc: scaling {kind!r} takes {sorted(want)}, got {sorted(d)}")
        sc = C.byref(RopeScaling(kind=_SCALINGS[kind], **{k: float(v) for k, v in d.items()}))
    check("cure_rope_init", lib.cure_rope_init(C.byref(r), st, rot_dim, float(base), sc, float(amplitude)))
    return r


def rope_axes(axis: Sequence[int]) -> RopeAxes:
    """The axis whose position each pair of a head turns by, pair 0 first (e.g. [0] * 16 + [1] * 24 + [2] * 24 for
    time, height and width in a run each): a host struct for the ``axes`` of cure_rope_qkv, cure_append_kv and
    cure_append_kv8, whose ``pos`` then holds a position on each axis for every row, [axes][rows].  Up to 8 axes; pairs
    that are not given (of a rotation of fewer dims) turn by axis 0."""
    a = [int(x) for x in axis]
    if not a or len(a) > 64:
        raise ValueError(f"rope_axes: 1 to 64 pairs expected, got {len(a)}")
    if min(a) < 0 or max(a) > 7:
        raise ValueError("rope_axes: axes are numbered from 0 to 7")
    return RopeAxes(axes=max(a) + 1, axis=(C.c_uint8 * 64)(*a))


def _here(t: torch.Tensor, name: str, dtype, dev: int) -> int:
    """_p() of a tensor that must also be on device `dev` and of a type."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on the current CUDA device")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _new(shape, dtype, stream) -> torch.Tensor:
    """A tensor that the call fills on `stream`: allocated there, so that its memory is not in use on another."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device="cuda")
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device="cuda")


def _current(stream) -> tuple[int, int]:
    """The current device, and the handle of `stream` (None: the current one), which must be on it."""
    dev = torch._C._cuda_getDevice()
    if stream is None:
        return dev, torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        raise ValueError("stream must be on the current CUDA device")
    return dev, stream.cuda_stream


def _head_rows(t: torch.Tensor, name: str, dev: int):
    """(address, values from row to row, rows, heads, head_dim) of bf16 [...][heads][D]: heads end to end, the
    leading dimensions one even step apart, as in a part of a fused projection's rows.  (Written for few
    attribute reads: a small call's host work outlasts its kernel.)"""
    if t.dtype is not _BF16:
        raise TypeError(f"{name} must be torch.bfloat16, got {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on the current CUDA device")
    sh = t.shape
    if len(sh) == 3:
        rows, H, D = sh
        outer, inner = 1, rows
    elif len(sh) == 4:
        outer, inner, H, D = sh
        rows = outer * inner
    else:
        raise ValueError(f"{name} must be [rows][heads][head_dim] or [batch][rows][heads][head_dim]")
    ld = H * D
    if t.is_contiguous():
        return t.data_ptr(), ld, rows, H, D
    st = t.stride()
    if rows > 1:
        ld = st[-3] if inner > 1 else st[0]
        if outer > 1 and inner > 1 and st[0] != inner * ld:
            raise ValueError(f"{name}: rows must lie one even step apart")
    if (D > 1 and st[-1] != 1) or (H > 1 and st[-2] != D):
        raise ValueError(f"{name}: a row's heads must lie end to end")
    return t.data_ptr(), ld, rows, H, D


_NO_ROWS = (None, 0, 0, 0, 0)


def cure_rope_qkv(q: Optional[torch.Tensor], k: Optional[torch.Tensor], v: Optional[torch.Tensor],
                  pos: torch.Tensor, rope: Optional[Rope], *, q_norm: Optional[torch.Tensor] = None,
                  k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, axes: Optional[RopeAxes] = None, out=None,
                  stream=None):
    """Per-head norms and the rotation of q and k at the rows' positions, v copied: (q, k, v) as cure_tree_attn
    takes them, from (parts of) the rows of a fused projection.

    q bf16 [rows][heads_q][D] or [batch][rows][heads_q][D], k and v the same with heads_kv; pos int32, one per row
    (the tree's ``pos``): rows with pos < 0 are left out.  rope = None: no rotation.  Any of q, k, v may be None, and
    its output with it.  With ``axes`` (rope_axes) pos holds a position on each axis, [axes][rows], and a row is left
    out where any of them is negative."""
    dev, s = _current(stream)
    if out is None:
        out = tuple(None if t is None else _new(t.shape, t.dtype, stream) for t in (q, k, v))
    qo, ko, vo = out
    rows = pos.numel() if axes is None else _rows_of_axes(pos, axes)
    pq, lq, nq, hq, dq = _NO_ROWS if q is None else _head_rows(q, "q", dev)
    pk, lk, nk, hk, dk = _NO_ROWS if k is None else _head_rows(k, "k", dev)
    pv, lv, nv, hv, dv = _NO_ROWS if v is None else _head_rows(v, "v", dev)
    oq, loq, noq, hoq, doq = _NO_ROWS if qo is None else _head_rows(qo, "q's output", dev)
    ok, lok, nok, hok, dok = _NO_ROWS if ko is None else _head_rows(ko, "k's output", dev)
    ov, lov, nov, hov, dov = _NO_ROWS if vo is None else _head_rows(vo, "v's output", dev)
    if nq != noq or nk != nok or nv != nov or hq != hoq or hk != hok or hv != hov or dq != doq or dk != dok or dv != dov:
        raise ValueError("cure_rope_qkv: an output must have its input's rows and heads")
    D = dq or dk or dv or 128
    if (q is not None and (nq != rows or dq != D)) or (k is not None and (nk != rows or dk != D)) or (
            v is not None and (nv != rows or dv != D or (k is not None and hv != hk))):
        raise ValueError("cure_rope_qkv: q, k, v and pos must have the same rows, k and v the same heads, and all one "
                         "head_dim")
    args = (None if rope is None else C.byref(rope), None if q_norm is None else _norm(q_norm, "q_norm", dev),
            None if k_norm is None else _norm(k_norm, "k_norm", dev), eps, oq, ok, ov, loq, lok, lov, s)
    p = _here(pos, "pos", _I32, dev)
    if axes is None:
        check("cure_rope_qkv", _lib.load().cure_rope_qkv(pq, pk, pv, lq, lk, lv, rows, hq, hk or hv, D, p, *args))
    else:
        check("cure_rope_qkv_axes", _lib.load().cure_rope_qkv_axes(pq, pk, pv, lq, lk, lv, rows, hq, hk or hv, D, p,
                                                                   C.byref(axes), *args))
    return out


def _rows_of_axes(pos: torch.Tensor, axes: RopeAxes) -> int:
    if pos.dim() < 2 or pos.shape[0] != axes.axes:
        raise ValueError(f"pos must hold a row of positions for each of {axes.axes} axes")
    return pos.numel() // axes.axes


def _norm(w: torch.Tensor, name: str, dev: int) -> int:
    if w.numel() != 128:
        raise ValueError(f"{name} must hold one weight for each of a head's 128 values")
    return _here(w, name, _BF16, dev)


def _caches(k: torch.Tensor, v: torch.Tensor, kv: KVDesc, batch: int, dev: int, dtype=_BF16) -> tuple[int, int]:
    """Addresses of a layer's caches, which must hold what their geometry says."""
    size = (batch * kv.max_len if kv.layout == 0 else kv.num_pages * kv.page_size) * kv.heads_kv * kv.head_dim
    if k.numel() < size or v.numel() < size:
        raise ValueError("a cache is smaller than its geometry")
    return _here(k, "k_cache", dtype, dev), _here(v, "v_cache", dtype, dev)


def _ragged(row_start: torch.Tensor, cache_len: torch.Tensor, kv: KVDesc) -> int:
    """Sequences of a packed batch, whose tensors must agree on it."""
    B = cache_len.numel()
    if row_start.numel() != B + 1:
        raise ValueError("row_start must hold one entry more than cache_len")
    table = getattr(kv, "_keep", None)
    if table is not None and table.numel() < B * kv.max_len:
        raise ValueError("block_table has fewer rows than the batch has sequences")
    return B


def _append_args(k, v, k_cache, v_cache, kv: KVDesc, row_start, cache_len, rope, q, pos, axes, q_norm, k_norm, eps, out,
                 stream, dtype):
    """The arguments of an append, checked: q's output, those before the caches, the caches, those behind."""
    dev, s = _current(stream)
    B = _ragged(row_start, cache_len, kv)
    Hkv, D = kv.heads_kv, kv.head_dim
    pk, lk, rows, hk, dk = _head_rows(k, "k", dev)
    pv, lv, nv, hv, dv = _head_rows(v, "v", dev)
    if nv != rows or hk != Hkv or hv != Hkv or dk != D or dv != D:
        raise ValueError("cure_append_kv: k and v must have the same rows, the cache's heads and its head_dim")
    if q is None:
        out, (pq, lq, _, hq, _), (po, lo, _, _, _) = None, _NO_ROWS, _NO_ROWS
    else:
        if out is None:
            out = _new(q.shape, q.dtype, stream)
        pq, lq, nq, hq, dq = _head_rows(q, "q", dev)
        po, lo, no, ho, do = _head_rows(out, "out", dev)
        if nq != rows or no != rows or ho != hq or dq != D or do != D:
            raise ValueError("cure_append_kv: q, its output and k must have the same rows and head_dim")
    if axes is not None:
        if pos is None:
            raise ValueError("cure_append_kv: axes need positions")
        if _rows_of_axes(pos, axes) != rows:
            raise ValueError("cure_append_kv: pos must have an entry for every row")
    elif pos is not None and pos.numel() != rows:
        raise ValueError("cure_append_kv: pos must have an entry for every row")
    kc, vc = _caches(k_cache, v_cache, kv, B, dev, dtype)
    front = (pq, pk, pv, lq, lk, lv, rows, hq, B, _here(row_start, "row_start", _I32, dev),
             _here(cache_len, "cache_len", _I32, dev), None if pos is None else _here(pos, "pos", _I32, dev))
    back = (None if rope is None else C.byref(rope), None if q_norm is None else _norm(q_norm, "q_norm", dev),
            None if k_norm is None else _norm(k_norm, "k_norm", dev), eps, po, lo, s)
    return out, front, (kc, vc), back, B, dev


def cure_append_kv(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, kv: KVDesc,
                   row_start: torch.Tensor, cache_len: torch.Tensor, rope: Optional[Rope], *,
                   q: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None,
                   axes: Optional[RopeAxes] = None, q_norm: Optional[torch.Tensor] = None,
                   k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, out: Optional[torch.Tensor] = None,
                   stream=None) -> Optional[torch.Tensor]:
    """cure_rope_qkv of packed rows whose K and V go into the cache, sequence b's rows row_start[b] ..
    row_start[b+1] - 1 to slots cache_len[b], cache_len[b] + 1, ..; returns q's rows (None without q).

    A row's position is its slot, or its entry of ``pos`` (int32; < 0 leaves the row out), or with ``axes`` its
    entries of pos [axes][rows].  cache_len is not advanced.  In-place tree rows: row_start = 0, n_max, 2 n_max, ..,
    pos = the tree's ``pos``."""
    out, front, caches, back, _, _ = _append_args(k, v, k_cache, v_cache, kv, row_start, cache_len, rope, q, pos, axes,
                                                  q_norm, k_norm, eps, out, stream, _BF16)
    if axes is None:
        check("cure_append_kv", _lib.load().cure_append_kv(*front, C.byref(kv), *caches, *back))
    else:
        check("cure_append_kv_axes", _lib.load().cure_append_kv_axes(*front, C.byref(axes), C.byref(kv), *caches, *back))
    return out


KV8_BLOCK = 16  # slots of a scale of a cache in 8 bits


def kv8_scale_shape(kv: KVDesc, batch: int) -> tuple[int, int, int]:
    """The shape of the scales of a layer's K (or V) cache in 8 bits: a float32 for each block of 16 slots and head."""
    if kv.layout == 0:
        return batch, -(-kv.max_len // KV8_BLOCK), kv.heads_kv
    return kv.num_pages, kv.page_size // KV8_BLOCK, kv.heads_kv


def _scales(k: torch.Tensor, v: torch.Tensor, kv: KVDesc, batch: int, dev: int) -> tuple[int, int]:
    a, b, c = kv8_scale_shape(kv, batch)
    if k.numel() < a * b * c or v.numel() < a * b * c:
        raise ValueError("scales are fewer than the cache's blocks and heads")
    return _here(k, "k_scale", _F32, dev), _here(v, "v_scale", _F32, dev)


def cure_append_kv8(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                    k_scale: torch.Tensor, v_scale: torch.Tensor, kv: KVDesc, row_start: torch.Tensor,
                    cache_len: torch.Tensor, rope: Optional[Rope], *, q: Optional[torch.Tensor] = None,
                    pos: Optional[torch.Tensor] = None, axes: Optional[RopeAxes] = None,
                    q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6,
                    out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """cure_append_kv into a cache held in 8 bits: k_cache, v_cache float8_e4m3fn codes in the geometry ``kv``,
    k_scale, v_scale float32 (kv8_scale_shape), value = code * scale.

    The scale of a block that gains rows becomes the least power of two for which all that the block then holds lies
    within 448 of it.  Pages of 16, 32 or 64 tokens."""
    out, front, caches, back, B, dev = _append_args(k, v, k_cache, v_cache, kv, row_start, cache_len, rope, q, pos, axes,
                                                    q_norm, k_norm, eps, out, stream, _E4M3)
    check("cure_append_kv8", _lib.load().cure_append_kv8(
        *front, None if axes is None else C.byref(axes), C.byref(kv), *caches, *_scales(k_scale, v_scale, kv, B, dev),
        *back))
    return out


def cure_prompt_attn_workspace_size(rows: int, batch: int, heads_q: int, kv: KVDesc) -> int:
    return int(_lib.load().cure_prompt_attn_workspace_size(rows, batch, heads_q, C.byref(kv)))


def _prompt_attn_args(q, k_cache, v_cache, kv: KVDesc, row_start, cache_len, scale, out, workspace, stream):
    """cure_prompt_attn's output, its workspace (to be held until the call is launched) and its C arguments, checked."""
    dev, s = _current(stream)
    B = _ragged(row_start, cache_len, kv)
    shape = q.shape
    if len(shape) != 3 or shape[2] != kv.head_dim:
        raise ValueError("q must be [rows][heads_q][head_dim]")
    if out is None:
        out = _new(shape, torch.bfloat16, stream)
    elif out.shape != shape:
        raise ValueError("out must have q's shape")
    if workspace is None:
        size = cure_prompt_attn_workspace_size(shape[0], B, shape[1], kv)
        workspace = _new((max(size, 256),), torch.uint8, stream)
    kc, vc = _caches(k_cache, v_cache, kv, B, dev)
    return out, workspace, (
        _here(q, "q", _BF16, dev), kc, vc, C.byref(kv), _here(row_start, "row_start", _I32, dev),
        _here(cache_len, "cache_len", _I32, dev), shape[0], B, shape[1], scale, _here(out, "out", _BF16, dev),
        _here(workspace, "workspace", torch.uint8, dev), workspace.numel(), s)


def cure_prompt_attn(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, kv: KVDesc,
                     row_start: torch.Tensor, cache_len: torch.Tensor, scale: float, *,
                     out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """Causal attention of packed rows over the cache for one layer: whole prompts, further chunks, single tokens.

    q bf16 [rows][heads_q][D]; sequence b's rows row_start[b] .. row_start[b+1] - 1 stand at positions cache_len[b],
    cache_len[b] + 1, .., and their K and V are in the cache already (cure_append_kv at the same lengths).  Up to 256
    sequences and 2^22 rows."""
    out, held, args = _prompt_attn_args(q, k_cache, v_cache, kv, row_start, cache_len, scale, out, workspace, stream)
    check("cure_prompt_attn", _lib.load().cure_prompt_attn(*args))
    return out


def cure_prompt_attn8_workspace_size(rows: int, batch: int, heads_q: int, kv: KVDesc) -> int:
    return int(_lib.load().cure_prompt_attn8_workspace_size(rows, batch, heads_q, C.byref(kv)))


def _prompt_attn8_args(q, k_cache, v_cache, k_scale, v_scale, kv: KVDesc, row_start, cache_len, scale, out, workspace,
                       stream):
    """As _prompt_attn_args, of cure_prompt_attn8."""
    dev, s = _current(stream)
    B = _ragged(row_start, cache_len, kv)
    shape = q.shape
    if len(shape) != 3 or shape[2] != kv.head_dim:
        raise ValueError("q must be [rows][heads_q][head_dim]")
    if out is None:
        out = _new(shape, torch.bfloat16, stream)
    elif out.shape != shape:
        raise ValueError("out must have q's shape")
    if workspace is None:
        size = cure_prompt_attn8_workspace_size(shape[0], B, shape[1], kv)
        workspace = _new((max(size, 256),), torch.uint8, stream)
    kc, vc = _caches(k_cache, v_cache, kv, B, dev, _E4M3)
    ks, vs = _scales(k_scale, v_scale, kv, B, dev)
    return out, workspace, (
        _here(q, "q", _BF16, dev), kc, vc, ks, vs, C.byref(kv), _here(row_start, "row_start", _I32, dev),
        _here(cache_len, "cache_len", _I32, dev), shape[0], B, shape[1], scale, _here(out, "out", _BF16, dev),
        _here(workspace, "workspace", torch.uint8, dev), workspace.numel(), s)


def cure_prompt_attn8(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: torch.Tensor,
                      v_scale: torch.Tensor, kv: KVDesc, row_start: torch.Tensor, cache_len: torch.Tensor, scale: float,
                      *, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """cure_prompt_attn over a cache held in 8 bits (cure_append_kv8): float8_e4m3fn codes and a float32 scale for
    each block of 16 slots and head."""
    out, held, args = _prompt_attn8_args(q, k_cache, v_cache, k_scale, v_scale, kv, row_start, cache_len, scale, out,
                                         workspace, stream)
    check("cure_prompt_attn8", _lib.load().cure_prompt_attn8(*args))
    return out


def cure_tree_attn8_workspace_size(batch: int, n_max: int, heads_q: int, kv: KVDesc) -> int:
    return int(_lib.load().cure_tree_attn8_workspace_size(batch, n_max, heads_q, C.byref(kv)))


def cure_tree_attn8(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: torch.Tensor,
                    v_scale: torch.Tensor, kv: KVDesc, cache_len: torch.Tensor, n_nodes: torch.Tensor,
                    anc: torch.Tensor, scale: float, *, out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """cure_tree_attn over a cache held in 8 bits, in the in-place layout: q bf16 [B][n_max][heads_q][D], node j's K/V
    rows at slot cache_len[b] + j (cure_append_kv8 with row_start = 0, n_max, 2 n_max, .. and the tree's ``pos``; around
    rows that may not stay, cure_save_kv8 and cure_restore_kv8)."""
    out, held, args = _tree_attn8_args(q, k_cache, v_cache, k_scale, v_scale, kv, cache_len, n_nodes, anc, scale, out,
                                       workspace, stream)
    check("cure_tree_attn8", _lib.load().cure_tree_attn8(*args))
    return out


def _tree_attn8_args(q, k_cache, v_cache, k_scale, v_scale, kv: KVDesc, cache_len, n_nodes, anc, scale, out, workspace,
                     stream):
    """As _prompt_attn_args, of cure_tree_attn8."""
    dev, s = _current(stream)
    shape = q.shape
    if len(shape) != 4 or shape[3] != kv.head_dim:
        raise ValueError("q must be [batch][n_max][heads_q][head_dim]")
    B, n_max, Hq, _ = shape
    if cache_len.numel() != B or n_nodes.numel() != B or anc.numel() != B * n_max * ((n_max + 63) // 64):
        raise ValueError("cache_len and n_nodes must hold an entry for every sequence, anc the words of every node")
    table = getattr(kv, "_keep", None)
    if table is not None and table.numel() < B * kv.max_len:
        raise ValueError("block_table has fewer rows than the batch has sequences")
    if out is None:
        out = _new(shape, torch.bfloat16, stream)
    elif out.shape != shape:
        raise ValueError("out must have q's shape")
    if workspace is None:
        workspace = _new((max(cure_tree_attn8_workspace_size(B, n_max, Hq, kv), 256),), torch.uint8, stream)
    kc, vc = _caches(k_cache, v_cache, kv, B, dev, _E4M3)
    ks, vs = _scales(k_scale, v_scale, kv, B, dev)
    return out, workspace, (
        _here(q, "q", _BF16, dev), kc, vc, ks, vs, C.byref(kv), _here(cache_len, "cache_len", _I32, dev),
        _here(n_nodes, "n_nodes", _I32, dev), _here(anc, "anc", torch.int64, dev), B, n_max, Hq, scale,
        _here(out, "out", _BF16, dev), _here(workspace, "workspace", torch.uint8, dev), workspace.numel(), s)


def cure_resync_kv8(k_caches: Sequence[torch.Tensor], v_caches: Sequence[torch.Tensor],
                    k_scales: Sequence[torch.Tensor], v_scales: Sequence[torch.Tensor], kv: KVDesc,
                    tree_k: torch.Tensor, tree_v: torch.Tensor, acc: dict, cache_len_in: torch.Tensor, block: int, *,
                    cache_len_out: Optional[torch.Tensor] = None, out=None, stream=None) -> dict:
    """cure_resync_kv for caches held in 8 bits: the accepted path's rows of tree_k/tree_v (bf16
    [layers][B][n_max][Hkv][D]) into every layer's cache, and the step's new lengths and replay lists."""
    dev, s = _current(stream)
    layers, B, n_max, Hkv, D = tree_k.shape
    if tree_v.shape != tree_k.shape or Hkv != kv.heads_kv or D != kv.head_dim:
        raise ValueError("cure_resync_kv8: tree_k and tree_v must have the same shape, the cache's heads and its head_dim")
    if not len(k_caches) == len(v_caches) == len(k_scales) == len(v_scales) == layers:
        raise ValueError("cure_resync_kv8: one cache, its scales and one slice of the tree per layer")
    P = block + 2
    i32 = lambda t, name, n: _sized(t, name, n, dev)  # noqa: E731
    if cache_len_out is None:
        cache_len_out = _new((B,), _I32, stream)
    if out is None:
        out = dict(draft_valid_len=_new((B,), _I32, stream), replay_tokens=_new((B, P), _I32, stream),
                   n_replay=_new((B,), _I32, stream))
    _, kp, vp, ksp, vsp = _layers8(k_caches, v_caches, k_scales, v_scales, kv, B, dev)
    check("cure_resync_kv8", _lib.load().cure_resync_kv8(
        layers, kp, vp, ksp, vsp, C.byref(kv), _here(tree_k, "tree_k", _BF16, dev), _here(tree_v, "tree_v", _BF16, dev), B,
        n_max, block, i32(acc["path_nodes"], "path_nodes", B * P), i32(acc["accept_len"], "accept_len", B),
        i32(acc["diverge_depth"], "diverge_depth", B), i32(acc["out_tokens"], "out_tokens", B * P),
        i32(cache_len_in, "cache_len_in", B), i32(cache_len_out, "cache_len_out", B),
        i32(out["draft_valid_len"], "draft_valid_len", B), i32(out["replay_tokens"], "replay_tokens", B * P),
        i32(out["n_replay"], "n_replay", B), s))
    out["cache_len"] = cache_len_out
    return out


def cure_save_kv8_size(layers: int, batch: int, kv: KVDesc) -> int:
    return int(_lib.load().cure_save_kv8_size(layers, batch, C.byref(kv)))


def cure_save_kv8(k_caches: Sequence[torch.Tensor], v_caches: Sequence[torch.Tensor], k_scales: Sequence[torch.Tensor],
                  v_scales: Sequence[torch.Tensor], kv: KVDesc, cache_len: torch.Tensor, *,
                  out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """What the sequences hold of the blocks that rows appended behind them would share, of every layer's cache in
    8 bits, for cure_restore_kv8 (uint8, cure_save_kv8_size bytes): before rows are appended that may not stay."""
    (dev, s), B = _current(stream), cache_len.numel()
    of = _layers8(k_caches, v_caches, k_scales, v_scales, kv, B, dev)
    if out is None:
        out = _new((cure_save_kv8_size(of[0], B, kv),), torch.uint8, stream)
    _held8("cure_save_kv8", of, kv, B, cache_len, out, dev, s)
    return out


def cure_restore_kv8(k_caches: Sequence[torch.Tensor], v_caches: Sequence[torch.Tensor],
                     k_scales: Sequence[torch.Tensor], v_scales: Sequence[torch.Tensor], kv: KVDesc,
                     cache_len: torch.Tensor, saved: torch.Tensor, *, stream=None) -> None:
    """Puts back what cure_save_kv8 saved at the same lengths: the tokens' codes and scales, to the bit.  The slots behind
    them hold nothing then."""
    (dev, s), B = _current(stream), cache_len.numel()
    of = _layers8(k_caches, v_caches, k_scales, v_scales, kv, B, dev)
    _held8("cure_restore_kv8", of, kv, B, cache_len, saved, dev, s)


def _layers8(k_caches, v_caches, k_scales, v_scales, kv: KVDesc, batch: int, dev: int) -> tuple:
    """The number of layers, and the arrays of their caches' and scales' addresses, checked."""
    layers = len(k_caches)
    if not layers == len(v_caches) == len(k_scales) == len(v_scales):
        raise ValueError("one k_cache, v_cache, k_scale and v_scale per layer")
    table = getattr(kv, "_keep", None)
    if table is not None and table.numel() < batch * kv.max_len:
        raise ValueError("block_table has fewer rows than the batch has sequences")
    size = (batch * kv.max_len if kv.layout == 0 else kv.num_pages * kv.page_size) * kv.heads_kv * kv.head_dim
    a, b, c = kv8_scale_shape(kv, batch)
    array = C.c_void_p * max(1, layers)
    return (layers, *(array(*_pointers(t, nm, dtype, n, dev)) for t, nm, dtype, n in (
        (k_caches, "a k_cache", _E4M3, size), (v_caches, "a v_cache", _E4M3, size),
        (k_scales, "a k_scale", _F32, a * b * c), (v_scales, "a v_scale", _F32, a * b * c))))


def _held8(name: str, of: tuple, kv: KVDesc, batch: int, cache_len: torch.Tensor, saved: torch.Tensor, dev: int,
           s: int) -> None:
    """cure_save_kv8 or cure_restore_kv8 of layers that _layers8 has checked for `batch` sequences."""
    check(name, getattr(_lib.load(), name)(*of, C.byref(kv), batch, _sized(cache_len, "cache_len", batch, dev),
                                           _here(saved, "saved", torch.uint8, dev), saved.numel(), s))


def _pointers(tensors, name: str, dtype, n: int, dev: int) -> list:
    """Addresses of the layers' tensors, each of a type, on device `dev`, contiguous and of at least n entries.  (In one
    loop: hundreds of calls' checks would outlast their kernel.)"""
    out = []
    for t in tensors:
        if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or t.numel() < n:
            _here(t, name, dtype, dev)
            raise ValueError(f"{name} is smaller than its geometry")
        out.append(t.data_ptr())
    return out


def _sized(t: torch.Tensor, name: str, n: int, dev: int) -> int:
    """_here() of an int32 tensor that must hold n entries."""
    if t.numel() != n:
        raise ValueError(f"{name} must hold {n} entries")
    return _here(t, name, _I32, dev)


def cure_device_error(stream=None) -> int:
    """Synchronise and return (and clear) the device error word's bits."""
    bits = C.c_int32(0)
    code = _lib.load().cure_device_error(_stream(stream), C.byref(bits))
    if code not in (0, 4):
        check("cure_device_error", code)
    return int(bits.value)


def cure_selftest_wait_timeout(limit_cycles: int = 1 << 24, stream=None) -> None:
    """Runs the library's bounded wait on a barrier nothing completes (a
    failure-detection self-test); read the outcome with cure_device_error()."""
    check("cure_selftest_wait_timeout", _lib.load().cure_selftest_wait_timeout(int(limit_cycles), _stream(stream)))


def cure_selftest_lm_head_timeout(hidden: torch.Tensor, w_lm: torch.Tensor, rank: int, out: torch.Tensor,
                                  workspace: torch.Tensor, limit_cycles: int = 1 << 22, *, stream=None) -> torch.Tensor:
    """cure_lm_head_argmax with a wait that runs out in one CTA of every pair (a
    failure-detection self-test); read the outcome with cure_device_error()."""
    rows, d = hidden.shape
    check("cure_selftest_lm_head_timeout", _lib.load().cure_selftest_lm_head_timeout(
        _p(hidden), _p(w_lm), rows, d, w_lm.shape[0], _p(out), _p(workspace),
        workspace.numel() * workspace.element_size(), int(rank), int(limit_cycles), _stream(stream)))
    return out


def cure_selftest_prompt_timeout(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, kv: KVDesc,
                                 row_start: torch.Tensor, cache_len: torch.Tensor, scale: float, warp: int, wait: int, *,
                                 out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                 stream=None) -> torch.Tensor:
    """cure_prompt_attn with the `wait`-th wait of one warp of its first CTA running out (a failure-detection
    self-test); read the outcome with cure_device_error()."""
    out, held, args = _prompt_attn_args(q, k_cache, v_cache, kv, row_start, cache_len, scale, out, workspace, stream)
    check("cure_selftest_prompt_timeout",
          _lib.load().cure_selftest_prompt_timeout(*args[:-1], int(warp), int(wait), args[-1]))
    return out


def cure_selftest_prompt8_timeout(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: torch.Tensor,
                                  v_scale: torch.Tensor, kv: KVDesc, row_start: torch.Tensor, cache_len: torch.Tensor,
                                  scale: float, warp: int, wait: int, *, out: Optional[torch.Tensor] = None,
                                  workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """cure_prompt_attn8 with a wait that runs out, as cure_selftest_prompt_timeout."""
    out, held, args = _prompt_attn8_args(q, k_cache, v_cache, k_scale, v_scale, kv, row_start, cache_len, scale, out,
                                         workspace, stream)
    check("cure_selftest_prompt8_timeout",
          _lib.load().cure_selftest_prompt8_timeout(*args[:-1], int(warp), int(wait), args[-1]))
    return out


def cure_selftest_tree8_timeout(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: torch.Tensor,
                                v_scale: torch.Tensor, kv: KVDesc, cache_len: torch.Tensor, n_nodes: torch.Tensor,
                                anc: torch.Tensor, scale: float, warp: int, wait: int, *,
                                out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                stream=None) -> torch.Tensor:
    """cure_tree_attn8 with a wait that runs out, as cure_selftest_prompt_timeout."""
    out, held, args = _tree_attn8_args(q, k_cache, v_cache, k_scale, v_scale, kv, cache_len, n_nodes, anc, scale, out,
                                       workspace, stream)
    check("cure_selftest_tree8_timeout",
          _lib.load().cure_selftest_tree8_timeout(*args[:-1], int(warp), int(wait), args[-1]))
    return out


def cure_selftest_attn_route(batch: int, n_max: int, heads_q: int, kv: KVDesc, in_place: bool) -> tuple[int, bool, int]:
    """The form a tree-attention call of this shape takes: CTAs per unit's cluster
    (0: persistent), pieces in two tile slots in turn, CTAs of the grid."""
    r = (C.c_int32 * 3)()
    check("cure_selftest_attn_route",
          _lib.load().cure_selftest_attn_route(batch, n_max, heads_q, C.byref(kv), int(in_place), r))
    return r[0], bool(r[1]), r[2]


def cure_status_string(code: int) -> str:
    return _lib.load().cure_status_string(code).decode()


def cure_abi_version() -> int:
    return int(_lib.load().cure_abi_version())
