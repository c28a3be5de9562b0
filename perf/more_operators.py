"""Cases of the target model's layers over a cache that is held in 8 bits, and of rotations with several positions.

``axes``    per-head norms and the rotation of Q and K rows whose tokens have a position on each of several axes
            (time, height, width), from the rows of the fused projection
``append``  the same for packed rows, K and V written as e4m3 into the cache, with a scale for each block of 16
            tokens and head
``prompt``  causal grouped-head attention of packed rows over such a cache: whole prompts, chunks, single tokens
``tree``    attention of a repair tree's nodes over it, the tree's rows in the cache behind the sequence's tokens
``commit``  the accepted path's K and V rows of every layer into it, and the step's new lengths

Where ``own`` is false ``run`` computes them in elementary torch operations; where it is true, by the calls
of ``paper_2608_00531_gb300.cure``.
"""
import math
import random

import torch

own = False

D = 128
BLOCK = 16  # tokens of a scale
LARGEST = 448.0  # of an e4m3 value
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-6
E4M3 = torch.float8_e4m3fn
# pairs of a head that turn by the positions of time, height and width: in a run each, or in turns
SECTIONS = (16, 24, 24)


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # the trees of a serving batch of a model that reads images: few rows, three positions each
        dict(name="axes_tree", op="axes", batch=32, heads_q=28, heads_kv=4, lo=33, hi=33, past_lo=100, past_hi=8000,
             style="half", base=1000000.0, order="runs", norm=False, lens=1),
        # prompts of text and images, interleaved pairs that take the axes in turns, heads normed
        dict(name="axes_images", op="axes", batch=4, heads_q=32, heads_kv=8, lo=3001, hi=9000, past_lo=0, past_hi=0,
             style="interleaved", base=500000.0, order="turns", norm=True, lens=2),
        # plain decoding, one new token for each of 200 sequences: most blocks are begun already
        dict(name="append_tokens", op="append", batch=200, heads_q=32, heads_kv=8, lo=1, hi=1, past_lo=60, past_hi=500,
             page=16, style="half", base=500000.0, order="", norm=False, lens=3),
        # chunks of prompts with images behind what their sequences hold
        dict(name="append_images", op="append", batch=32, heads_q=28, heads_kv=4, lo=37, hi=3000, past_lo=1, past_hi=3000,
             page=16, style="half", base=1000000.0, order="runs", norm=True, lens=4),
        # the first token's wait of one user: one short prompt
        dict(name="prompt_short", op="prompt", batch=1, heads_q=32, heads_kv=8, lo=200, hi=200, past_lo=0, past_hi=0,
             page=16, lens=5),
        # a packed batch of ragged prompts, 7 query heads a kv head
        dict(name="prompt_packed", op="prompt", batch=32, heads_q=28, heads_kv=4, lo=33, hi=4096, past_lo=0, past_hi=0,
             page=16, lens=6),
        # one long document, 70B-class heads, contiguous
        dict(name="prompt_document", op="prompt", batch=1, heads_q=64, heads_kv=8, lo=16384, hi=16384, past_lo=0,
             past_hi=0, page=0, lens=7),
        # plain decoding, one token for each of 64 sequences: the cache's bytes are the work
        dict(name="prompt_tokens", op="prompt", batch=64, heads_q=28, heads_kv=4, lo=1, hi=1, past_lo=500, past_hi=16000,
             page=16, lens=8),
        # the tree of one sequence, 8B-class heads: latency counts
        dict(name="tree_single", op="tree", batch=1, heads_q=32, heads_kv=8, lo=21, hi=25, past_lo=4096, past_hi=4096,
             page=16, lens=9),
        # a serving batch's trees
        dict(name="tree_serve", op="tree", batch=32, heads_q=28, heads_kv=4, lo=17, hi=33, past_lo=1024, past_hi=8192,
             page=16, lens=10),
        # one sequence's accepted path in 32 layers
        dict(name="commit_single", op="commit", batch=1, heads_kv=8, lo=9, hi=9, past_lo=500, past_hi=500, page=16,
             layers=32, block=16, lens=11),
        # a serving batch's accepted paths in 28 layers
        dict(name="commit_serve", op="commit", batch=32, heads_kv=4, lo=1, hi=17, past_lo=100, past_hi=1000, page=16,
             layers=28, block=16, lens=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads_q, heads_kv = rng.choice([(28, 4), (32, 8), (64, 8), (8, 2), (16, 16), (40, 8)])
    c = dict(heads_q=heads_q, heads_kv=heads_kv, lens=rng.randint(100, 10 ** 6))
    form = dict(style=rng.choice(["half", "half", "interleaved"]), base=rng.choice([10000.0, 500000.0, 1000000.0]),
                norm=rng.random() < 0.5)
    op = rng.choice(["axes", "append", "prompt", "prompt", "tree", "commit"])
    if op == "axes":
        batch = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 24000 // batch)
        return dict(op=op, batch=batch, lo=max(1, int(hi * rng.random())), hi=hi, past_lo=0,
                    past_hi=_log_int(rng, 1, 100000), order=rng.choice(["runs", "turns"]), **c, **form)
    page = rng.choice([0, 16, 16, 32, 64])
    if op == "append":
        batch = _log_int(rng, 1, 256)
        hi = _log_int(rng, 1, max(2, 32768 // batch))
        return dict(op=op, batch=batch, lo=max(1, int(hi * rng.random())), hi=hi, past_lo=0,
                    past_hi=_log_int(rng, 1, max(2, 32768 // batch)), page=page,
                    order=rng.choice(["", "runs", "turns"]), **c, **form)
    if op == "commit":
        del c["heads_q"]
        block, layers = rng.choice([8, 16, 31]), rng.randint(1, 40)
        batch = _log_int(rng, 1, 64)
        return dict(op=op, batch=batch, lo=1, hi=rng.randint(1, block + 1), past_lo=0,
                    past_hi=_log_int(rng, 16, 40000 // batch), page=page, layers=layers, block=block, **c)
    batch = _log_int(rng, 1, 64)
    if op == "tree":
        hi = rng.randint(4, 97)
        past = _log_int(rng, 16, min(65536, 400000 // batch))
    elif rng.random() < 0.35:  # a token or a few for each sequence
        hi = rng.randint(1, 8)
        past = _log_int(rng, 16, min(65536, 1000000 // batch))
    else:
        # the scores of all sequences stay below half of the longest listed document's
        hi = _log_int(rng, 2, int(16384 / math.sqrt(batch)))
        past = _log_int(rng, 1, max(2, int(16384 * 16384 * 0.25 / (batch * hi))))
        past = min(past, 65536) if rng.random() < 0.5 else 0
    past = min(past, (1 << 23) // (batch * heads_kv))  # a cache of some 2 GB at most
    return dict(op=op, batch=batch, lo=max(1, int(hi * rng.random())), hi=hi, past_lo=int(past * rng.random()),
                past_hi=past, page=page, **c)


def _lengths(c):
    """Rows of each sequence (nodes of its tree, or of its accepted path), and the tokens that its cache holds already."""
    rng = random.Random(c["lens"])

    def log_between(lo, hi):
        return max(lo, hi) if lo >= hi else min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))
    rows = [log_between(c["lo"], c["hi"]) for _ in range(c["batch"])]
    past = [rng.randint(c["past_lo"], c["past_hi"]) for _ in range(c["batch"])]
    return rows, past


# ---------------------------------------------------------------- inputs
def _cuda(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _randn(g, *shape, std=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=g)


def _cache(g, c, ends, layers=0):
    """K and V of a layer (or of `layers`) with room for every sequence's `ends` tokens: codes and scales as earlier
    appends leave them, and the pages' table. Some blocks hold larger values than others."""
    B, H, ps = c["batch"], c["heads_kv"], c["page"]
    lead = (layers,) if layers else ()
    if ps == 0:
        cap = max(ends)
        blocks = (cap + BLOCK - 1) // BLOCK
        shape, of_scales, table, pages = (B, cap, H, D), (B, blocks, H), None, 0
    else:  # a pool that is somewhat larger than what is in use, its pages in any order
        need = [(e + ps - 1) // ps for e in ends]
        pages = sum(need) + B
        order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32).tolist()
        rows, o = [], 0
        for n in need:
            rows.append(order[o:o + n] + [-1] * (max(need) - n))
            o += n
        table = _cuda(rows)
        shape, of_scales = (pages, ps, H, D), (pages, ps // BLOCK, H)
    codes = [torch.empty(lead + shape, dtype=torch.float32, device="cuda").normal_(0.0, 96.0, generator=g)
             .clamp_(-LARGEST, LARGEST).to(E4M3) for _ in range(2)]
    scales = [torch.exp2(torch.randint(-8, -5, lead + of_scales, device="cuda", generator=g).float()) for _ in range(2)]
    return codes[0], codes[1], scales[0], scales[1], table, pages


def _positions(c, rows, past):
    """[3][all rows]: runs of text, whose positions are the same on all axes, and images, whose rows and columns count
    on from where they begin; the next text follows behind the largest position. (Trees: text alone.)"""
    rng = random.Random(c["lens"] + 1)
    axes = [[], [], []]
    for n, p in zip(rows, past):
        if c["hi"] <= 97:  # a tree: a chain of up to 16 nodes, then repairs at its depths
            d = [p + (j if j <= 16 else 1 + (7 * j) % 16) for j in range(n)]
            for a in axes:
                a.extend(d)
            continue
        at, left = p, n
        while left > 0:
            m = min(left, rng.randint(5, 200))
            for a in axes:
                a.extend(range(at, at + m))
            at, left = at + m, left - m
            h, w = rng.randint(4, 40), rng.randint(4, 40)
            m = min(left, h * w)
            axes[0].extend([at] * m)
            axes[1].extend(at + j // w for j in range(m))
            axes[2].extend(at + j % w for j in range(m))
            at, left = at + max(h, w), left - m
    return _cuda(axes)


def _axis_of_pair(c):
    if c["order"] == "turns":
        return [i % 3 for i in range(D // 2)]
    return [a for a, n in enumerate(SECTIONS) for _ in range(n)]


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 31)
    B, Hkv = c["batch"], c["heads_kv"]
    rows, past = _lengths(c)
    s = dict(c=c, rows=rows, past=past)
    if c["op"] == "commit":
        return _prepare_commit(c, s, g)
    Hq, start = c["heads_q"], [0]
    for n in rows:
        start.append(start[-1] + n)
    N = start[-1]
    s["row_start"], s["cache_len"] = _cuda(start), _cuda(past)
    if c["op"] != "axes":
        s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["pages"] = _cache(
            g, c, [n + p for n, p in zip(rows, past)])
    if c["op"] == "prompt":
        s["q"] = _randn(g, N, Hq, D, std=1.5)
        s["out"] = torch.zeros_like(s["q"])
    elif c["op"] == "tree":
        n_max = c["hi"]
        s["q"] = _randn(g, B, n_max, Hq, D, std=1.5)
        s["out"] = torch.zeros_like(s["q"])
        s["n_nodes"] = _cuda(rows)
        s["anc"] = _ancestors(rows, n_max)
    else:  # the rows of the fused projection: Hq heads of Q, then Hkv of K, then Hkv of V
        qkv = _randn(g, N, (Hq + 2 * Hkv) * D).unflatten(-1, (-1, D))
        s["q"], s["k"], s["v"] = qkv[..., :Hq, :], qkv[..., Hq:Hq + Hkv, :], qkv[..., Hq + Hkv:, :]
        s["q_norm"] = s["k_norm"] = None
        if c["norm"]:
            s["q_norm"], s["k_norm"] = ((1.0 + 0.1 * torch.randn(D, device="cuda", generator=g)).to(torch.bfloat16)
                                        for _ in range(2))
        s["q_out"] = torch.zeros(N, Hq, D, dtype=torch.bfloat16, device="cuda")
        if c["op"] == "axes":
            s["k_out"], s["v_out"] = (torch.zeros(N, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s["pos"] = _positions(c, rows, past) if c["order"] else None
    if own:
        from paper_2608_00531_gb300 import cure
        if c["op"] != "axes":
            s["kv"] = _geometry(c, s)
        if c["op"] in ("axes", "append"):
            s["rope"] = cure.rope_desc(D, c["base"], style=c["style"])
            s["axes"] = cure.rope_axes(_axis_of_pair(c)) if c["order"] else None
        if c["op"] == "prompt":
            size = cure.cure_prompt_attn8_workspace_size(N, B, Hq, s["kv"])
        if c["op"] == "tree":
            size = cure.cure_tree_attn8_workspace_size(B, c["hi"], Hq, s["kv"])
        if c["op"] in ("prompt", "tree"):
            s["ws"] = torch.empty(max(256, size), dtype=torch.uint8, device="cuda")
    return s


def _ancestors(rows, n_max):
    """The trees' ancestor bits [B][n_max][words]: a chain of up to 16 nodes, then repairs that leave it."""
    words = (n_max + 63) // 64
    bits = []
    for j in range(n_max):
        if j <= 16:
            bits.append((1 << (j + 1)) - 1)
        else:
            bits.append((1 << (1 + (7 * j) % 16)) - 1 | 1 << j)
    signed = lambda v: v - (1 << 64) if v >> 63 else v  # noqa: E731
    one = [[signed(b >> (64 * w) & (1 << 64) - 1) for w in range(words)] for b in bits]
    return torch.tensor([[w if j < n else [0] * words for j, w in enumerate(one)] for n in rows], dtype=torch.int64,
                        device="cuda")


def _prepare_commit(c, s, g):
    """A step's tree rows of all layers, and what the acceptance walk gave for them."""
    B, H, K, layers = c["batch"], c["heads_kv"], c["block"], c["layers"]
    n_max = 2 * K + 1
    rng = random.Random(c["lens"] + 2)
    s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["pages"] = _cache(
        g, c, [p + n_max for p in s["past"]], layers)
    s["tree_k"], s["tree_v"] = (_randn(g, layers, B, n_max, H, D) for _ in range(2))
    paths, diverge = [], []
    for n in s["rows"]:  # n nodes: the root, then the draft's up to where a repair took over
        d = rng.randint(1, n) if n > 1 else 1
        nodes = [j if j < d else K + j for j in range(n)]
        paths.append(nodes + [-1] * (K + 2 - n))
        diverge.append(d if d < n else -1)
    s["acc"] = dict(path_nodes=_cuda(paths), accept_len=_cuda([n - 1 for n in s["rows"]]), diverge_depth=_cuda(diverge),
                    out_tokens=torch.randint(0, 150000, (B, K + 2), device="cuda", generator=g, dtype=torch.int32))
    s["cache_len"] = _cuda(s["past"])
    s["new_len"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    s["resync"] = dict(draft_valid_len=torch.zeros(B, dtype=torch.int32, device="cuda"),
                       replay_tokens=torch.zeros(B, K + 2, dtype=torch.int32, device="cuda"),
                       n_replay=torch.zeros(B, dtype=torch.int32, device="cuda"))
    if own:
        s["kv"] = _geometry(c, s)
    return s


def _geometry(c, s):
    from paper_2608_00531_gb300 import cure
    if s["table"] is None:
        return cure.kv_desc(c["heads_kv"], D, s["k_cache"].shape[-3])
    return cure.kv_desc(c["heads_kv"], D, s["table"].shape[1], block_table=s["table"], page_size=c["page"],
                        num_pages=s["pages"])


# ---------------------------------------------------------------- one pass
def run(state):
    s, c = state, state["c"]
    if own:
        from paper_2608_00531_gb300 import cure
        if c["op"] == "axes":
            return cure.cure_rope_qkv(s["q"], s["k"], s["v"], s["pos"], s["rope"], axes=s["axes"], q_norm=s["q_norm"],
                                      k_norm=s["k_norm"], eps=EPS, out=(s["q_out"], s["k_out"], s["v_out"]))
        if c["op"] == "append":
            q = cure.cure_append_kv8(s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["kv"],
                                     s["row_start"], s["cache_len"], s["rope"], q=s["q"], pos=s["pos"], axes=s["axes"],
                                     q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS, out=s["q_out"])
            return q, s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]
        if c["op"] == "prompt":
            return cure.cure_prompt_attn8(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["kv"],
                                          s["row_start"], s["cache_len"], SCALE, out=s["out"], workspace=s["ws"])
        if c["op"] == "tree":
            return cure.cure_tree_attn8(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["kv"],
                                        s["cache_len"], s["n_nodes"], s["anc"], SCALE, out=s["out"], workspace=s["ws"])
        r = cure.cure_resync_kv8(list(s["k_cache"]), list(s["v_cache"]), list(s["k_scale"]), list(s["v_scale"]), s["kv"],
                                 s["tree_k"], s["tree_v"], s["acc"], s["cache_len"], c["block"],
                                 cache_len_out=s["new_len"], out=s["resync"])
        return (s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], r["cache_len"], r["draft_valid_len"],
                r["replay_tokens"], r["n_replay"])
    if c["op"] == "axes":
        cos, sin = _angles(c, s["pos"])
        s["q_out"].copy_(_turn(c, _normed(s["q"], s["q_norm"]), cos, sin))
        s["k_out"].copy_(_turn(c, _normed(s["k"], s["k_norm"]), cos, sin))
        s["v_out"].copy_(s["v"])
        return s["q_out"], s["k_out"], s["v_out"]
    if c["op"] == "append":
        row = torch.arange(s["q"].shape[0], dtype=torch.int32, device="cuda")
        seq = (row[:, None] >= s["row_start"][None, 1:]).sum(1)
        slot = (row - s["row_start"][seq] + s["cache_len"][seq]).long()
        cos, sin = _angles(c, slot.expand(3, -1) if s["pos"] is None else s["pos"])
        s["q_out"].copy_(_turn(c, _normed(s["q"], s["q_norm"]), cos, sin))
        k = _turn(c, _normed(s["k"], s["k_norm"]), cos, sin)
        for codes, scale, x in ((s["k_cache"], s["k_scale"], k), (s["v_cache"], s["v_scale"], s["v"].float())):
            _quantise(s, codes, scale, x, seq, slot)
        return s["q_out"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]
    if c["op"] == "commit":
        return _commit(s, c)
    if c["op"] == "tree":
        q, out = s["q"].flatten(0, 1), s["out"].flatten(0, 1)
        first = [b * c["hi"] for b in range(c["batch"])]
    else:
        q, out, first = s["q"], s["out"], [0]
        for n in s["rows"]:
            first.append(first[-1] + n)
    for lo, hi, i, m in _parts(c, s["rows"], s["past"]):
        _attend(s, c, q, out, first, lo, hi, i, m)
    return s["out"]


# ---------------------------------------------------------------- the plain forms
def _frequencies(c):
    """Radians per position of each pair, in 64 bits."""
    i = torch.arange(D // 2, dtype=torch.float64, device="cuda")
    return torch.exp(i * (-2.0 * math.log(c["base"]) / D))


def _angles(c, pos):
    """Cosines and sines [rows][1][pairs] of positions [axes][rows], the angles in 64 bits."""
    axis = torch.tensor(_axis_of_pair(c), device="cuda")
    a = pos.double()[axis].T * _frequencies(c)
    return torch.cos(a).float()[:, None, :], torch.sin(a).float()[:, None, :]


def _normed(x, weight):
    x = x.float()
    if weight is None:
        return x
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()


def _turn(c, x, cos, sin):
    half = c["style"] == "half"
    a, b = (x[..., :D // 2], x[..., D // 2:]) if half else (x[..., 0::2], x[..., 1::2])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    return torch.cat([ya, yb], -1) if half else torch.stack([ya, yb], -1).flatten(-2)


def _places(s, seq, slot, cap, scales):
    """Rows in the flattened cache (or, by blocks, in its scales) of slots (blocks) `slot` of sequences `seq`."""
    if s["table"] is None:
        return seq * cap + slot
    per = s["c"]["page"] // BLOCK if scales else s["c"]["page"]
    return s["table"][seq, slot // per].long() * per + slot % per


def _quantise(s, codes, scale, x, seq, slot, layer=0, layers=1):
    """Rows x [n][Hkv][D] (32 bits) of sequences `seq` (and layers `layer`) into the cache's slots `slot`: each block that
    gains rows gets the least power of two s for which its tokens, held and new, lie within 448 s, and its values are
    rounded to it."""
    H, B = x.shape[1], s["c"]["batch"]
    flat, flat_scale = codes.view(-1, H, D), scale.view(-1, H)
    rows, places = len(flat) // layers, len(flat_scale) // layers  # of a layer
    which, item = torch.unique((layer * B + seq) * (1 << 32) + slot // BLOCK, return_inverse=True)
    b_layer, b_seq, b_block = (which >> 32) // B, (which >> 32) % B, which & (1 << 32) - 1
    at_scale = b_layer * places + _places(s, b_seq, b_block, scale.shape[-2], True)
    # the tokens that the block holds already: its slots below the sequence's length
    t = b_block[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    held = t < s["cache_len"][b_seq][:, None]
    h_item, h_slot = held.nonzero()[:, 0], t[held]
    at_held = b_layer[h_item] * rows + _places(s, b_seq[h_item], h_slot, codes.shape[-3], False)
    old = flat[at_held].float() * flat_scale[at_scale[h_item]][..., None]
    amax = torch.zeros(len(which), H, device="cuda")
    amax.index_reduce_(0, item, x.abs().amax(-1), "amax")
    amax.index_reduce_(0, h_item, old.abs().amax(-1), "amax")
    new = _power_above(amax / LARGEST)
    flat_scale[at_scale] = new
    at = layer * rows + _places(s, seq, slot, codes.shape[-3], False)
    flat.view(torch.uint8)[at] = (x / new[item][..., None]).to(E4M3).view(torch.uint8)
    flat.view(torch.uint8)[at_held] = (old / new[h_item][..., None]).to(E4M3).view(torch.uint8)


def _power_above(x):
    """The least power of two from 2^-40 to 2^40 that is not below x."""
    m, e = torch.frexp(x)
    return torch.exp2((e - (m == 0.5).to(e.dtype)).clamp(-40, 40).float()).where(x > 0, 2.0 ** -40)


def _commit(s, c):
    K = c["block"]
    path, a, d = (s["acc"][n] for n in ("path_nodes", "accept_len", "diverge_depth"))
    depth = torch.arange(K + 2, device="cuda")
    taken = (depth[None, :K + 1] <= a[:, None]).expand(c["layers"], -1, -1)
    layer, seq, t = taken.nonzero().unbind(1)
    node, slot = path[seq, t].long(), s["cache_len"][seq].long() + t
    for codes, scale, x in ((s["k_cache"], s["k_scale"], s["tree_k"]), (s["v_cache"], s["v_scale"], s["tree_v"])):
        _quantise(s, codes, scale, x[layer, seq, node].float(), seq, slot, layer, c["layers"])
    s["new_len"].copy_(s["cache_len"] + a + 1)
    r = s["resync"]
    r["draft_valid_len"].copy_(torch.where(d >= 0, s["cache_len"] + d, s["cache_len"] + a + 1))
    r["n_replay"].copy_(torch.where(d >= 0, a + 2 - d, 1))
    begin = torch.where(d >= 0, d - 1, a).long()
    shifted = s["acc"]["out_tokens"].gather(1, (begin[:, None] + depth[None]).clamp(max=K + 1))
    r["replay_tokens"].copy_(torch.where(depth[None] < r["n_replay"][:, None], shifted, -1))
    return (s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["new_len"], r["draft_valid_len"],
            r["replay_tokens"], r["n_replay"])


def _parts(c, rows, past, most=1 << 28):
    """Sequences lo .. hi - 1 whose scores fit 1 GiB at once, padded to the longest; or rows i .. i + m - 1 of one."""
    lo, parts = 0, []
    while lo < len(rows):
        hi = lo + 1
        while hi < len(rows) and ((hi + 1 - lo) * c["heads_q"] * max(rows[lo:hi + 1]) *
                                  max(n + p for n, p in zip(rows[lo:hi + 1], past[lo:hi + 1]))) <= most:
            hi += 1
        m = max(rows[lo:hi])
        if hi == lo + 1:
            m = max(1, min(m, most // (c["heads_q"] * (rows[lo] + past[lo]))))
        parts += [(lo, hi, i, min(m, max(rows[lo:hi]) - i)) for i in range(0, max(rows[lo:hi]), m)]
        lo = hi
    return parts


def _attend(s, c, q, out, first, lo, hi, i, m):
    """Rows i .. i + m - 1 of sequences lo .. hi - 1, as far as they have them, in 32 bits."""
    H, seq = c["heads_kv"], torch.arange(lo, hi, device="cuda")
    n, p = (torch.tensor(x[lo:hi], device="cuda") for x in (s["rows"], s["past"]))
    keys = max(b + (a if c["op"] == "tree" else min(a, i + m)) for a, b in zip(s["rows"][lo:hi], s["past"][lo:hi]))
    j = torch.arange(keys, device="cuda")
    held = j < (n + p)[:, None]
    slot = torch.where(held, j, 0)
    at = _places(s, seq[:, None], slot, s["k_cache"].shape[1], False)
    at_scale = _places(s, seq[:, None], slot // BLOCK, s["k_scale"].shape[1], True)
    k, v = ((s[x + "_cache"].view(-1, H, D)[at].float() * s[x + "_scale"].view(-1, H)[at_scale][..., None])
            .transpose(1, 2) for x in "kv")                                     # [B][Hkv][keys][D]
    r = i + torch.arange(m, device="cuda")
    there = r < n[:, None]
    row = torch.tensor(first[lo:hi], device="cuda")[:, None] + torch.where(there, r, 0)
    x = q[row].float().unflatten(2, (H, -1)).permute(0, 2, 3, 1, 4)             # [B][Hkv][G][m][D]
    x = torch.matmul(x.flatten(2, 3), k.transpose(2, 3)).mul_(SCALE).unflatten(2, (-1, m))
    if c["op"] == "tree":
        node = (j - p[:, None]).clamp(min=0)                                    # [B][keys]
        word = s["anc"][lo:hi, i:i + m].gather(2, (node // 64).clamp(max=s["anc"].shape[2] - 1)[:, None].expand(-1, m, -1))
        seen = (word >> (node % 64)[:, None] & 1 == 1) | (j < p[:, None])[:, None]
        seen = seen & held[:, None]
    else:
        seen = j <= (p[:, None] + r)[..., None]                                 # [B][m][keys]
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    x = torch.exp(x.sub_(x.amax(-1, keepdim=True)))
    o = torch.matmul(x.flatten(2, 3), v).unflatten(2, (-1, m)) / x.sum(-1, keepdim=True)
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3).to(torch.bfloat16)               # [B][m][Hq][D]
    out[row[there]] = o[there]


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    rows, past = _lengths(c)
    n, Hkv = sum(rows), c["heads_kv"]
    # blocks that a call's rows lie in, and the tokens that those hold already
    gain = sum((p + m - 1) // BLOCK - p // BLOCK + 1 for m, p in zip(rows, past))
    begun = sum(p % BLOCK for p in past)
    if c["op"] == "commit":
        each = 2 * Hkv * (D * 3.0 * n + D * 2.0 * begun + 8.0 * gain)
        return dict(bytes=c["layers"] * each, flops=c["layers"] * 2.0 * Hkv * D * 2 * (n + begun))
    Hq = c["heads_q"]
    if c["op"] in ("prompt", "tree"):
        seen = sum(m * p + (m * (m + 1) // 2 if c["op"] == "prompt" else m * min(m, 9)) for m, p in zip(rows, past))
        held = sum(m + p for m, p in zip(rows, past))
        return dict(bytes=4.0 * D * n * Hq + 2.0 * held * Hkv * (D + 4.0 / BLOCK), flops=4.0 * D * Hq * seen)
    flops = n * (Hq + Hkv) * (3.0 * D + (4.0 * D if c["norm"] else 0.0))
    if c["op"] == "axes":
        return dict(bytes=n * (4.0 * D * (Hq + 2 * Hkv) + 12), flops=flops)
    return dict(bytes=n * (4.0 * D * Hq + 6.0 * D * Hkv + 12) + 2 * Hkv * (D * 2.0 * begun + 8.0 * gain),
                flops=flops + 4.0 * n * D * Hkv)


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_rows(c, x, weight, pos):
    """Heads of rows x at positions pos [axes][rows], from the definition: norm, then each pair as a complex number turned."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + EPS) * weight.double()
    axis = _axis_of_pair(c)
    angle = torch.stack([pos[axis[i]].double() * c["base"] ** (-2.0 * i / D) for i in range(D // 2)], -1)[:, None]
    turn = torch.polar(torch.ones_like(angle), angle)
    if c["style"] == "half":
        z = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous()) * turn
        return torch.cat([z.real, z.imag], -1)
    z = torch.view_as_complex(x.contiguous().unflatten(-1, (-1, 2))) * turn
    return torch.view_as_real(z).flatten(-2)


def _exact_blocks(s, codes, scale, x, seq_rows):
    """Codes (not rounded) and scales of one layer's K or V after the rows x; seq_rows: (sequence, its first row, rows)."""
    H = x.shape[1]
    old, old_scale = codes.double().view(-1, H, D), scale.double().view(-1, H)
    new, new_scale = old.clone(), old_scale.clone()
    page = s["c"]["page"]
    table = None if s["table"] is None else s["table"].tolist()
    powers = torch.ldexp(torch.ones(81, dtype=torch.float64), torch.arange(-40, 41)).to(codes.device)
    for b, r0, n in seq_rows:
        p = s["past"][b]
        for blk in range(p // BLOCK, (p + n - 1) // BLOCK + 1):
            t0 = blk * BLOCK
            begin, end = max(p, t0), min(p + n, t0 + BLOCK)
            if table is None:
                first, place = b * codes.shape[-3] + t0, b * scale.shape[-2] + blk
            else:
                first = table[b][t0 // page] * page + t0 % page
                place = table[b][t0 // page] * (page // BLOCK) + t0 % page // BLOCK
            h = old[first:first + max(0, begin - t0)] * old_scale[place][None, :, None]
            values = torch.cat([h, x[r0 + begin - p:r0 + end - p].double()])
            amax = values.abs().amax((0, 2))
            new_scale[place] = powers[(LARGEST * powers[None] < amax[:, None]).sum(1).clamp(max=80)]
            new[first:first + end - t0] = values / new_scale[place][None, :, None]
    return new.view(codes.shape), new_scale.view(scale.shape)


def exact(case, seed):
    c = case
    rows, past = _lengths(c)
    if c["op"] in ("prompt", "tree"):
        if c["heads_q"] * sum(m * (m + p) for m, p in zip(rows, past)) > 6e9:
            return None
    elif c["op"] == "commit" and c["layers"] * sum(r // BLOCK + 2 for r in rows) > 20000:
        return None
    s = prepare(case, seed)
    H = c["heads_kv"]
    start = [0]
    for n in rows:
        start.append(start[-1] + n)
    if c["op"] == "axes":
        return (_exact_rows(c, s["q"], s["q_norm"], s["pos"]), _exact_rows(c, s["k"], s["k_norm"], s["pos"]),
                s["v"].double())
    if c["op"] == "append":
        pos = s["pos"]
        if pos is None:
            pos = torch.cat([torch.arange(p, p + n, device="cuda") for n, p in zip(rows, past)]).expand(3, -1)
        seq_rows = [(b, start[b], rows[b]) for b in range(c["batch"])]
        k, ks = _exact_blocks(s, s["k_cache"], s["k_scale"], _exact_rows(c, s["k"], s["k_norm"], pos), seq_rows)
        v, vs = _exact_blocks(s, s["v_cache"], s["v_scale"], s["v"], seq_rows)
        return _exact_rows(c, s["q"], s["q_norm"], pos), k, v, ks, vs
    if c["op"] == "commit":
        outs = [[], [], [], []]
        paths = s["acc"]["path_nodes"].tolist()
        for layer in range(c["layers"]):
            for o, name in enumerate("kv"):
                tree = s["tree_" + name][layer]
                x = torch.cat([tree[b, paths[b][:n]] for b, n in enumerate(rows)])
                codes, scale = _exact_blocks(s, s[name + "_cache"][layer], s[name + "_scale"][layer], x,
                                             [(b, start[b], n) for b, n in enumerate(rows)])
                outs[o].append(codes)
                outs[2 + o].append(scale)
        return (*(torch.stack(x) for x in outs), None, None, None, None)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    G = c["heads_q"] // H
    kc, vc, ks, vs = (s[n].flatten(0, 1) for n in ("k_cache", "v_cache", "k_scale", "v_scale"))
    for b, (n, p) in enumerate(zip(rows, past)):
        held = torch.arange(p + n, device="cuda")
        block = torch.div(held, BLOCK, rounding_mode="floor")
        if s["table"] is None:
            at, of = b * s["k_cache"].shape[1] + held, b * s["k_scale"].shape[1] + block
        else:
            pg = s["table"][b].long()[torch.div(held, c["page"], rounding_mode="floor")]
            at, of = pg * c["page"] + held % c["page"], pg * (c["page"] // BLOCK) + block % (c["page"] // BLOCK)
        if c["op"] == "tree":
            mask = torch.zeros(n, p + n, dtype=torch.bool, device="cuda")
            words = s["anc"][b, :n].tolist()
            for i in range(n):
                for a in range(n):
                    mask[i, p + a] = not words[i][a // 64] >> (a % 64) & 1
        for h in range(c["heads_q"]):
            k = kc[at, h // G].double() * ks[of, h // G].double()[:, None]
            v = vc[at, h // G].double() * vs[of, h // G].double()[:, None]
            if c["op"] == "tree":
                x = (s["q"][b, :n, h].double() @ k.T * SCALE).masked_fill(mask, -math.inf)
                out[b, :n, h] = torch.softmax(x, 1) @ v
                continue
            step = max(1, (1 << 27) // (p + n))
            for i in range(0, n, step):
                m = min(step, n - i)
                end = p + i + m
                x = (s["q"][start[b] + i:start[b] + i + m, h].double() @ k[:end].T) * SCALE
                x.masked_fill_(torch.ones(m, end, dtype=torch.bool, device="cuda").triu(end - m + 1), -math.inf)
                out[start[b] + i:start[b] + i + m, h] = torch.softmax(x, 1) @ v[:end]
    return out
