"""Cases of the target model's attention operators around the repair-verify step: what stands between a
layer's Q/K/V projection and the tree attention, and what fills the cache that the tree attention reads.

``rope``    per-head norms and the rotation of the tree's Q and K rows at their positions (V passed along),
            from the rows of the fused projection into the tensors that the tree attention takes
``append``  the same for packed prompt (or single-token) rows, K and V written into the cache
``prompt``  causal grouped-head attention of packed prompt rows over the cache, whole prompts, later
            chunks of one, or one token a sequence

Where ``own`` is false ``run`` computes them in elementary torch operations; where it is true, by the calls
of ``paper_2608_00531_gb300.cure``.
"""
import math
import random

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-6
# scaled rotations, by the text that a case names them with
SCALINGS = {
    "": None,
    "linear": dict(kind="linear", factor=4.0),
    "bands": dict(kind="bands", factor=8.0, low=1.0, high=4.0, original=8192),
    "ramp": dict(kind="ramp", factor=4.0, slow=1.0, fast=32.0, original=32768),
}


# ---------------------------------------------------------------- the cases
def _rope(style, rot, base, scaling, norm):
    return dict(style=style, rot=rot, base=base, scaling=scaling, norm=norm)


def listed():
    half = _rope("half", 128, 500000.0, "", False)
    normed = _rope("half", 128, 1000000.0, "", True)
    return [
        # the tree of one sequence (21 of 25 nodes or so), 8B-class heads: latency counts
        dict(name="rope_single", op="rope", batch=1, heads_q=32, heads_kv=8, nodes=25, lo=17, hi=25, past_lo=4096,
             past_hi=4096, lens=1, **half),
        # a serving batch's trees, heads normed as well
        dict(name="rope_serve", op="rope", batch=32, heads_q=28, heads_kv=4, nodes=33, lo=17, hi=33, past_lo=1024,
             past_hi=8192, lens=2, **normed),
        # 64 wide trees at far positions: interleaved pairs, half of the head rotated, frequencies scaled in bands
        dict(name="rope_long", op="rope", batch=64, heads_q=64, heads_kv=8, nodes=49, lo=30, hi=49, past_lo=32768,
             past_hi=1000000, lens=3, **_rope("interleaved", 64, 500000.0, "bands", False)),
        # one new token for each of 200 sequences, plain decoding
        dict(name="append_decode", op="append", batch=200, heads_q=32, heads_kv=8, lo=1, hi=1, past_lo=60, past_hi=500,
             page=16, lens=4, **half),
        # prompt chunks of a serving batch behind what their sequences hold already, 16-token pages
        dict(name="append_chunks", op="append", batch=32, heads_q=28, heads_kv=4, lo=37, hi=1000, past_lo=1, past_hi=3000,
             page=16, lens=5, **normed),
        # one long document, 70B-class heads, contiguous cache, rotation scaled for long contexts
        dict(name="append_document", op="append", batch=1, heads_q=64, heads_kv=8, lo=32768, hi=32768, past_lo=0,
             past_hi=0, page=0, lens=6, **_rope("half", 128, 1000000.0, "ramp", False)),
        # the first token's wait of one user: one short prompt
        dict(name="prompt_short", op="prompt", batch=1, heads_q=32, heads_kv=8, lo=200, hi=200, past_lo=0, past_hi=0,
             page=16, lens=7),
        # a packed batch of ragged prompts, 7 query heads a kv head, 16-token pages
        dict(name="prompt_packed", op="prompt", batch=32, heads_q=28, heads_kv=4, lo=33, hi=4096, past_lo=0, past_hi=0,
             page=16, lens=8),
        # chunks of prompts that were begun earlier: many keys before the chunk's own
        dict(name="prompt_chunks", op="prompt", batch=8, heads_q=28, heads_kv=4, lo=200, hi=1024, past_lo=1024,
             past_hi=16000, page=16, lens=9),
        # one long document, 70B-class heads, contiguous
        dict(name="prompt_document", op="prompt", batch=1, heads_q=64, heads_kv=8, lo=16384, hi=16384, past_lo=0,
             past_hi=0, page=0, lens=10),
        # plain decoding, one token for each of 64 sequences: the cache's bytes are the work
        dict(name="prompt_tokens", op="prompt", batch=64, heads_q=28, heads_kv=4, lo=1, hi=1, past_lo=500, past_hi=16000,
             page=16, lens=11),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads_q, heads_kv = rng.choice([(28, 4), (32, 8), (64, 8), (8, 2), (16, 16), (40, 8)])
    heads = dict(heads_q=heads_q, heads_kv=heads_kv, lens=rng.randint(100, 10 ** 6))
    form = _rope(rng.choice(["half", "half", "interleaved"]), rng.choice([128, 128, 96, 64, 32]),
                 rng.choice([10000.0, 500000.0, 1000000.0]), rng.choice(sorted(SCALINGS)), rng.random() < 0.5)
    op = rng.choice(["rope", "append", "prompt", "prompt"])
    if op == "rope":
        nodes = rng.randint(6, 97)
        past = _log_int(rng, 16, 1000000)
        return dict(op=op, batch=_log_int(rng, 1, 128), nodes=nodes, lo=rng.randint(1, nodes), hi=nodes,
                    past_lo=int(past * rng.random()), past_hi=past, **heads, **form)
    page = rng.choice([0, 8, 16, 16, 32, 64])
    if op == "append":
        batch = _log_int(rng, 1, 256)
        hi = _log_int(rng, 1, max(2, 32768 // batch))
        return dict(op=op, batch=batch, lo=max(1, int(hi * rng.random())), hi=hi, past_lo=0,
                    past_hi=_log_int(rng, 1, max(2, 32768 // batch)), page=page, **heads, **form)
    batch = _log_int(rng, 1, 64)
    if rng.random() < 0.25:  # a token or a few for each sequence
        hi = rng.randint(1, 8)
        past = _log_int(rng, 16, min(65536, 1000000 // batch))
    else:
        # the scores of all sequences stay below half of the longest listed document's
        hi = _log_int(rng, 2, int(16384 / math.sqrt(batch)))
        past = _log_int(rng, 1, max(2, int(16384 * 16384 * 0.25 / (batch * hi))))
        past = min(past, 65536) if rng.random() < 0.5 else 0
    past = min(past, (1 << 23) // (batch * heads_kv))  # a cache of some 4 GB at most
    return dict(op=op, batch=batch, lo=max(1, int(hi * rng.random())), hi=hi, past_lo=int(past * rng.random()),
                past_hi=past, page=page, **heads)


def _lengths(c):
    """Rows of each sequence (or nodes of its tree), and the tokens that its cache holds already."""
    rng = random.Random(c["lens"])

    def log_between(lo, hi):
        if hi <= 0 or lo >= hi:
            return max(lo, hi)
        return min(hi, max(lo, int(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi + 1))))))
    rows = [log_between(c["lo"], c["hi"]) for _ in range(c["batch"])]
    past = [rng.randint(c["past_lo"], c["past_hi"]) for _ in range(c["batch"])]
    return rows, past


# ---------------------------------------------------------------- inputs
def _cuda(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _randn(g, *shape, std=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=g)


def _cache(g, c, ends):
    """K and V of one layer with room for every sequence's `ends` tokens, and the pages' table."""
    B, H, ps = c["batch"], c["heads_kv"], c["page"]
    if ps == 0:
        shape, table, pages = (B, max(ends), H, D), None, 0
    else:  # a pool that is somewhat larger than what is in use, its pages in any order
        need = [(e + ps - 1) // ps for e in ends]
        pages = sum(need) + B
        order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32).tolist()
        rows, o = [], 0
        for n in need:
            rows.append(order[o:o + n] + [-1] * (max(need) - n))
            o += n
        table = _cuda(rows)
        shape = (pages, ps, H, D)
    return _randn(g, *shape), _randn(g, *shape), table, pages


def _geometry(c, s):
    from paper_2608_00531_gb300 import cure
    if s["table"] is None:
        return cure.kv_desc(c["heads_kv"], D, s["k_cache"].shape[1])
    return cure.kv_desc(c["heads_kv"], D, s["table"].shape[1], block_table=s["table"], page_size=c["page"],
                        num_pages=s["pages"])


def _amplitude(c):
    return 0.1 * math.log(SCALINGS["ramp"]["factor"]) + 1.0 if c["scaling"] == "ramp" else 1.0


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 29)
    B, Hq, Hkv = c["batch"], c["heads_q"], c["heads_kv"]
    rows, past = _lengths(c)
    s = dict(c=c, rows=rows, past=past)
    if c["op"] != "rope":
        start = [0]
        for n in rows:
            start.append(start[-1] + n)
        s.update(row_start=_cuda(start), cache_len=_cuda(past))
        s["k_cache"], s["v_cache"], s["table"], s["pages"] = _cache(g, c, [n + p for n, p in zip(rows, past)])
    if c["op"] == "prompt":
        s["q"] = _randn(g, start[-1], Hq, D, std=1.5)
        s["out"] = torch.zeros_like(s["q"])
        if own:
            from paper_2608_00531_gb300 import cure
            s["kv"] = _geometry(c, s)
            s["ws"] = torch.empty(max(256, cure.cure_prompt_attn_workspace_size(start[-1], B, Hq, s["kv"])),
                                  dtype=torch.uint8, device="cuda")
        return s
    # the rows of the fused projection: Hq heads of Q, then Hkv of K, then Hkv of V
    lead = (B, c["nodes"]) if c["op"] == "rope" else (start[-1],)
    qkv = _randn(g, *lead, (Hq + 2 * Hkv) * D).unflatten(-1, (-1, D))
    s["q"], s["k"], s["v"] = qkv[..., :Hq, :], qkv[..., Hq:Hq + Hkv, :], qkv[..., Hq + Hkv:, :]
    s["q_norm"] = s["k_norm"] = None
    if c["norm"]:
        s["q_norm"], s["k_norm"] = ((1.0 + 0.1 * torch.randn(D, device="cuda", generator=g)).to(torch.bfloat16)
                                    for _ in range(2))
    s["q_out"] = torch.zeros(*lead, Hq, D, dtype=torch.bfloat16, device="cuda")
    if c["op"] == "rope":
        s["k_out"], s["v_out"] = (torch.zeros(*lead, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        # a chain of up to 16 nodes, then repairs at its depths; rows past the last node hold no position
        depth = [[j if j <= 16 else 1 + (7 * j) % 16 for j in range(n)] for n in rows]
        s["pos"] = _cuda([[p + d for d in ds] + [-1] * (c["nodes"] - len(ds)) for p, ds in zip(past, depth)])
    if own:
        from paper_2608_00531_gb300 import cure
        s["rope"] = cure.rope_desc(c["rot"], c["base"], style=c["style"], scaling=SCALINGS[c["scaling"]],
                                   amplitude=_amplitude(c))
        if c["op"] == "append":
            s["kv"] = _geometry(c, s)
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    s, c = state, state["c"]
    if own:
        from paper_2608_00531_gb300 import cure
        if c["op"] == "rope":
            return cure.cure_rope_qkv(s["q"], s["k"], s["v"], s["pos"], s["rope"], q_norm=s["q_norm"],
                                      k_norm=s["k_norm"], eps=EPS, out=(s["q_out"], s["k_out"], s["v_out"]))
        if c["op"] == "append":
            q = cure.cure_append_kv(s["k"], s["v"], s["k_cache"], s["v_cache"], s["kv"], s["row_start"], s["cache_len"],
                                    s["rope"], q=s["q"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS,
                                    out=s["q_out"])
            return q, s["k_cache"], s["v_cache"]
        return cure.cure_prompt_attn(s["q"], s["k_cache"], s["v_cache"], s["kv"], s["row_start"], s["cache_len"], SCALE,
                                     out=s["out"], workspace=s["ws"])
    if c["op"] == "rope":
        keep = s["pos"] >= 0
        cos, sin = _angles(c, s["pos"][keep])
        s["q_out"][keep] = _turn(c, _normed(s["q"][keep], s["q_norm"]), cos, sin).to(torch.bfloat16)
        s["k_out"][keep] = _turn(c, _normed(s["k"][keep], s["k_norm"]), cos, sin).to(torch.bfloat16)
        s["v_out"][keep] = s["v"][keep]
        return s["q_out"], s["k_out"], s["v_out"]
    if c["op"] == "append":
        row = torch.arange(s["q"].shape[0], dtype=torch.int32, device="cuda")
        seq = (row[:, None] >= s["row_start"][None, 1:]).sum(1)
        pos = row - s["row_start"][seq] + s["cache_len"][seq]
        at = _rows_of(s, seq, pos.long())
        cos, sin = _angles(c, pos)
        s["q_out"].copy_(_turn(c, _normed(s["q"], s["q_norm"]), cos, sin))
        s["k_cache"].view(-1, c["heads_kv"], D)[at] = _turn(c, _normed(s["k"], s["k_norm"]), cos, sin).to(torch.bfloat16)
        s["v_cache"].view(-1, c["heads_kv"], D)[at] = s["v"]
        return s["q_out"], s["k_cache"], s["v_cache"]
    r0 = 0
    for b, (n, p) in enumerate(zip(s["rows"], s["past"])):
        at = _rows_of(s, b, torch.arange(p + n, device="cuda"))
        k, v = (x.view(-1, c["heads_kv"], D)[at].float().transpose(0, 1) for x in (s["k_cache"], s["v_cache"]))
        step = max(1, (1 << 28) // (c["heads_q"] * (p + n)))  # scores of 1 GiB at most
        for i in range(0, n, step):
            m = min(step, n - i)
            s["out"][r0 + i:r0 + i + m] = _attend(c, s["q"][r0 + i:r0 + i + m].float(), k[:, :p + i + m],
                                                  v[:, :p + i + m], p + i)
        r0 += n
    return s["out"]


# ---------------------------------------------------------------- the plain forms
def _frequencies(c):
    """Radians per position of each pair, in 64 bits."""
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda")
    f = torch.exp(i * (-2.0 * math.log(c["base"]) / c["rot"]))
    sc = SCALINGS[c["scaling"]]
    if sc is None:
        return f
    if sc["kind"] == "linear":
        return f / sc["factor"]
    turns = f * sc["original"] / (2.0 * math.pi)  # of a pair within the original context
    if sc["kind"] == "bands":  # few turns: slowed; many: kept; between: in proportion
        part = ((turns - sc["low"]) / (sc["high"] - sc["low"])).clamp(0.0, 1.0)
        return f * (part + (1.0 - part) / sc["factor"])
    first, last = _ramp(c, sc)
    part = ((i - first) / (last - first)).clamp(0.0, 1.0)
    return f * (1.0 - part) + f / sc["factor"] * part


def _ramp(c, sc):
    """The pairs between which the slowing grows from nothing to the whole factor."""
    def pair(turns):
        return c["rot"] * math.log(sc["original"] / (turns * 2.0 * math.pi)) / (2.0 * math.log(c["base"]))
    first, last = max(math.floor(pair(sc["fast"])), 0), min(math.ceil(pair(sc["slow"])), c["rot"] - 1)
    return first, (last if last > first else first + 0.001)


def _angles(c, pos):
    a = pos.double()[:, None] * _frequencies(c)
    return (torch.cos(a) * _amplitude(c)).float()[:, None, :], (torch.sin(a) * _amplitude(c)).float()[:, None, :]


def _normed(x, weight):
    x = x.float()
    if weight is None:
        return x
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()


def _turn(c, x, cos, sin):
    r = c["rot"]
    y = x.clone()
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if c["style"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    if c["style"] == "half":
        y[..., :r // 2], y[..., r // 2:r] = ya, yb
    else:
        y[..., 0:r:2], y[..., 1:r:2] = ya, yb
    return y


def _rows_of(s, seq, slot):
    """Rows in the flattened cache of slots `slot` of sequences `seq`."""
    if s["table"] is None:
        return seq * s["k_cache"].shape[1] + slot
    ps = s["k_cache"].shape[1]
    return s["table"][seq, slot // ps].long() * ps + slot % ps


def _attend(c, q, k, v, first):
    """q [m][Hq][D] at positions first, first + 1, ..; k, v [Hkv][keys][D]; all in 32 bits."""
    m, H = q.shape[0], c["heads_kv"]
    q = q.view(m, H, -1, D).permute(1, 2, 0, 3)                # [Hkv][G][m][D]
    x = torch.matmul(q.reshape(H, -1, D), k.transpose(1, 2)).view(H, -1, m, k.shape[1]) * SCALE
    later = torch.arange(k.shape[1], device="cuda")[None, :] > first + torch.arange(m, device="cuda")[:, None]
    x = x.masked_fill_(later, -math.inf)
    x = torch.exp(x.sub_(x.amax(-1, keepdim=True)))
    o = torch.matmul(x.view(H, -1, k.shape[1]), v).view(H, -1, m, D) / x.sum(-1, keepdim=True)
    return o.permute(2, 0, 1, 3).reshape(m, -1, D).to(torch.bfloat16)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    rows, past = _lengths(c)
    n, Hq, Hkv = sum(rows), c["heads_q"], c["heads_kv"]
    if c["op"] == "prompt":
        seen = sum(m * p + m * (m + 1) // 2 for m, p in zip(rows, past))
        held = sum(m + p for m, p in zip(rows, past))
        return dict(bytes=2.0 * D * (2 * n * Hq + 2 * held * Hkv), flops=4.0 * D * Hq * seen)
    # read and written once each; four products and two sums a pair, and with norms about four operations a value
    flops = n * (Hq + Hkv) * (3.0 * c["rot"] + (4.0 * D if c["norm"] else 0.0))
    return dict(bytes=n * (4.0 * D * (Hq + 2 * Hkv) + 4), flops=flops)


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_rows(c, x, weight, pos):
    """Heads of rows x at positions pos, from the definition: norm, then each pair as a complex number turned."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + EPS) * weight.double()
    r = c["rot"]
    w = []
    for i in range(r // 2):
        f = c["base"] ** (-2.0 * i / r)
        sc = SCALINGS[c["scaling"]] or dict(kind="")
        if sc["kind"] == "linear":
            f /= sc["factor"]
        elif sc["kind"] == "bands":
            length = 2.0 * math.pi / f
            if length > sc["original"] / sc["low"]:
                f /= sc["factor"]
            elif length >= sc["original"] / sc["high"]:
                t = (sc["original"] / length - sc["low"]) / (sc["high"] - sc["low"])
                f = (1.0 - t) * f / sc["factor"] + t * f
        elif sc["kind"] == "ramp":
            first, last = _ramp(c, sc)
            t = min(1.0, max(0.0, (i - first) / (last - first)))
            f = f / sc["factor"] * t + f * (1.0 - t)
        w.append(f)
    angle = pos.double()[:, None, None] * torch.tensor(w, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(angle, _amplitude(c)), angle)
    y = x.clone()
    if c["style"] == "half":
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * turn
        y[..., :r] = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.view_as_complex(x[..., :r].contiguous().unflatten(-1, (-1, 2))) * turn
        y[..., :r] = torch.view_as_real(z).flatten(-2)
    return y


def exact(case, seed):
    c, s = case, prepare(case, seed)
    H = c["heads_kv"]
    if c["op"] == "rope":
        q, k, v = (torch.zeros_like(s[n], dtype=torch.float64) for n in ("q_out", "k_out", "v_out"))
        for b, n in enumerate(s["rows"]):
            pos = s["pos"][b, :n]
            q[b, :n] = _exact_rows(c, s["q"][b, :n], s["q_norm"], pos)
            k[b, :n] = _exact_rows(c, s["k"][b, :n], s["k_norm"], pos)
            v[b, :n] = s["v"][b, :n].double()
        return q, k, v
    r0 = 0
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    kc, vc = s["k_cache"].flatten(0, 1), s["v_cache"].flatten(0, 1)
    if c["op"] == "append":
        kc, vc = kc.double(), vc.double()
    for b, (n, p) in enumerate(zip(s["rows"], s["past"])):
        held = torch.arange(p + n, device="cuda")
        if s["table"] is None:
            held += b * s["k_cache"].shape[1]
        else:
            held = s["table"][b].long()[torch.div(held, c["page"], rounding_mode="floor")] * c["page"] + held % c["page"]
        if c["op"] == "append":
            pos = torch.arange(p, p + n, device="cuda")
            out[r0:r0 + n] = _exact_rows(c, s["q"][r0:r0 + n], s["q_norm"], pos)
            kc[held[p:]] = _exact_rows(c, s["k"][r0:r0 + n], s["k_norm"], pos)
            vc[held[p:]] = s["v"][r0:r0 + n].double()
            r0 += n
            continue
        G = c["heads_q"] // H
        step = max(1, (1 << 27) // (p + n))
        for h in range(c["heads_q"]):
            k, v = kc[held, h // G].double(), vc[held, h // G].double()
            for i in range(0, n, step):
                m = min(step, n - i)
                end = p + i + m
                x = (s["q"][r0 + i:r0 + i + m, h].double() @ k[:end].T) * SCALE
                x.masked_fill_(torch.ones(m, end, dtype=torch.bool, device="cuda").triu(end - m + 1), -math.inf)
                out[r0 + i:r0 + i + m, h] = torch.softmax(x, 1) @ v[:end]
        r0 += n
    if c["op"] == "append":
        return out, kc.view(s["k_cache"].shape), vc.view(s["v_cache"].shape)
    return out
