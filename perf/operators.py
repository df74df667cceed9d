"""Measured cases of the operators around the attention kernels: query/key normalisation with rotation, attention
under a sliding window with visible first tokens, and the paged key/value cache (append, and one new token's attention).

listed() and draw() give the cases, prepare() makes their inputs, run() is one pass (the plain torch form, or the
library's entry points when `own` is true), work() counts the bytes and operations that a pass cannot do without,
and exact() computes the outputs in 64 bits from the definitions.

Definitions
  rows:    n = x / sqrt(mean(x^2) + eps) * weight over one head's D values, then the first R values rotated:
           pair i (i, i + R/2, or 2i, 2i + 1 when interleaved) turns by the angle whose cosine and sine are row
           `position` of the table.
  window:  key j is visible to query i, at position p = i + q_offset, iff j <= p and (j > p - window or j < sinks).
  cache:   key j of sequence b lies in slot j % page_size of page block_table[b, j // page_size].
"""
import math

import torch

own = False

EPS = 1e-6
THETA = 1e6
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------ cases

def listed():
    return [
        # --- per-head norm + rotation + head-major layout of a fused projection, as it feeds the attention kernels
        # the shortest prompt of the repository's configurations: a launch-bound call
        dict(name="prep_short", op="prep", type="fp16", B=1, S=128, H=2, Hkv=2, D=64, R=64, interleaved=False),
        # the long-context configuration with grouped heads: a prompt that is bound by memory bandwidth
        dict(name="prep_long", op="prep", type="bf16", B=1, S=16384, H=32, Hkv=8, D=128, R=128, interleaved=False),
        # training, ragged length, rotation of half of each head, adjacent pairs
        dict(name="prep_grad_ragged", op="prep_grad", type="fp16", B=3, S=1999, H=16, Hkv=4, D=64, R=32, interleaved=True),
        # training at the batched causal configuration
        dict(name="prep_grad_batch", op="prep_grad", type="bf16", B=4, S=2048, H=32, Hkv=8, D=128, R=128, interleaved=False),
        # --- sliding window with first tokens that stay visible
        # a short ragged prompt and a window that ends inside a tile
        dict(name="window_ragged", op="window", type="fp16", B=2, H=16, Hkv=16, Sq=1000, Sk=1000, D=64, window=255, sinks=1),
        # a long prompt
        dict(name="window_long", op="window", type="bf16", B=1, H=32, Hkv=8, Sq=16384, Sk=16384, D=128, window=1024, sinks=4),
        # a training step (forward and backward) of the same layer
        dict(name="window_train", op="window_train", type="bf16", B=1, H=32, Hkv=8, Sq=8192, Sk=8192, D=128, window=1024, sinks=4),
        # --- paged cache
        # one serving step of a batch: every sequence appends its new token
        dict(name="append_step", op="append", type="bf16", B=64, low=1, high=2048, new=1, H=32, Hkv=8, D=128, R=128, page=16,
             layout="head", interleaved=False),
        # prompts of many lengths written at once, slots before heads in a page, padded at the end of the batch
        dict(name="append_prompts", op="append", type="fp16", B=8, low=100, high=4000, new=0, H=16, Hkv=16, D=64, R=64, page=64,
             layout="slot", interleaved=True),
        # one short conversation: a latency-bound call
        dict(name="decode_single", op="decode", type="bf16", B=1, low=1000, high=1000, H=32, Hkv=8, D=128, page=16, layout="head",
             window=0, sinks=0),
        # a serving batch of ragged lengths, one to 8192 tokens
        dict(name="decode_batch", op="decode", type="bf16", B=64, low=1, high=8192, H=32, Hkv=8, D=128, page=16, layout="slot",
             window=0, sinks=0),
        # long conversations of which a window and the first tokens are visible; no grouped heads
        dict(name="decode_window", op="decode", type="fp16", B=32, low=500, high=20000, H=16, Hkv=16, D=64, page=64, layout="head",
             window=4096, sinks=4),
    ]


def _spread(rng, low, high):
    """A whole number whose logarithm is spread evenly over low .. high."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["prep", "prep_grad", "window", "window_train", "append", "decode"])
    kind, D = rng.choice(["bf16", "fp16"]), rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    H = Hkv * rng.choice([1, 2, 4, 8] if Hkv < 8 else [1, 2, 4])
    c = dict(op=op, type=kind, H=H, Hkv=Hkv, D=D)
    if op in ("prep", "prep_grad"):
        # at most the elements of the longest listed case
        tokens = _spread(rng, 1, min(32768, (16384 if op == "prep" else 8192) * 48 * 128 // ((H + 2 * Hkv) * D)))
        c["B"] = rng.randint(1, min(8, tokens))
        c["S"] = max(1, tokens // c["B"])
        c |= dict(R=rng.choice([D, D // 2, 32]), interleaved=rng.random() < 0.5)
    elif op in ("window", "window_train"):
        c["B"] = rng.randint(1, 4)
        most = (16384 if op == "window" else 8192) * 32 * 1024
        # training sequences have some length: where every query sees one key alone, the gradients of Q and K are zero
        least = 1 if op == "window" else 32
        c["window"] = _spread(rng, least, 2048)
        c["sinks"] = rng.choice([0, 1, 4, 16, 130])
        c["Sq"] = _spread(rng, least, max(least, min(8192, most // (c["B"] * H * (c["window"] + 256)))))
        # a chunk behind tokens that are already there (Sk > Sq), or the whole sequence
        c["Sk"] = c["Sq"] + (rng.randint(0, 4096) if rng.random() < 0.5 else 0)
    elif op == "append":
        c["B"] = _spread(rng, 1, 128)
        c["high"] = _spread(rng, 2, max(2, 32768 // c["B"]))
        c["low"] = _spread(rng, 1, c["high"])
        c |= dict(new=rng.choice([0, 1]), R=rng.choice([D, D // 2]), page=rng.choice([8, 16, 64, 128]), layout=rng.choice(["head", "slot"]),
                  interleaved=rng.random() < 0.5)
    else:
        c["B"] = _spread(rng, 1, 128)
        c["high"] = _spread(rng, 2, max(2, min(65536, 64 * 4096 * 8 * 128 // (c["B"] * Hkv * D))))
        c["low"] = _spread(rng, 1, c["high"])
        c |= dict(page=rng.choice([8, 16, 64, 128]), layout=rng.choice(["head", "slot"]))
        c |= rng.choice([dict(window=0, sinks=0), dict(window=_spread(rng, 1, 8192), sinks=rng.choice([0, 4, 33]))])
    return c


def _lengths(c):
    """The sequences' lengths: spread over low .. high, both ends among them; the same for every seed."""
    B, low, high = c["B"], c["low"], c["high"]
    if B == 1:
        return [high]
    at = [(b * 0.6180339887498949) % 1.0 for b in range(B)]
    at[B // 2] = 1.0
    return [low + int(round(f * (high - low))) for f in at]


def _new_tokens(c):
    """How many tokens each sequence appends: one, or its whole length."""
    return [1 if c["new"] else n for n in _lengths(c)]


def _visible(c, length):
    """How many keys the newest token of a sequence sees."""
    if not c["window"] or c["window"] >= length:
        return length
    return c["window"] + min(c["sinks"], length - c["window"])


def _pairs(c):
    """Visible (query, key) pairs of one head."""
    off, total = c["Sk"] - c["Sq"], 0
    for i in range(c["Sq"]):
        p = i + off
        seen = min(c["window"], p + 1)
        total += seen + min(c["sinks"], p + 1 - seen)
    return total


def work(case):
    c = case
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    if c["op"] in ("prep", "prep_grad"):
        rows = c["B"] * c["S"]
        table = c["S"] * c["R"] * 4 + 4 * D
        if c["op"] == "prep":
            return {"bytes": rows * (H + 2 * Hkv) * D * 2 * 2 + table, "flops": rows * (H + Hkv) * D * 7}
        # gradients in and out for q, k, v; q and k themselves; two weight gradients in 32 bits
        return {"bytes": rows * D * 2 * (2 * (H + 2 * Hkv) + H + Hkv) + table + 8 * D, "flops": rows * (H + Hkv) * D * 16}
    if c["op"] in ("window", "window_train"):
        pairs = c["B"] * H * _pairs(c)
        q, kv, lse = c["B"] * H * c["Sq"] * D * 2, c["B"] * Hkv * D * 2, c["B"] * H * c["Sq"] * 4
        run = min(c["Sk"], c["Sq"] + c["window"] - 1)                      # keys that some query sees
        seen = run + min(c["sinks"], c["Sk"] - run)
        if c["op"] == "window":
            return {"bytes": 2 * q + 2 * kv * seen + lse, "flops": 4 * D * pairs}
        return {"bytes": 4 * q + 2 * kv * (seen + c["Sk"]) + lse, "flops": 14 * D * pairs}
    if c["op"] == "append":
        tokens = sum(_new_tokens(c))
        return {"bytes": tokens * ((H + 2 * Hkv) * D * 2 * 2 + c["R"] * 4) + 4 * D + tokens * 4, "flops": tokens * (H + Hkv) * D * 7}
    keys = sum(_visible(c, n) for n in _lengths(c))
    pages = sum(-(-_visible(c, n) // c["page"]) for n in _lengths(c))
    return {"bytes": keys * Hkv * D * 4 + c["B"] * H * (4 * D + 4) + pages * 4 + c["B"] * 4, "flops": 4 * keys * H * D}


# ------------------------------------------------------------------ inputs

def _table(length, R, device):
    """cos | sin of position * THETA^(-2i/R), from angles in 64 bits."""
    f = THETA ** (-torch.arange(0, R, 2, dtype=torch.float64, device=device) / R)
    a = torch.arange(length, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([a.cos(), a.sin()], dim=1).float().contiguous()


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    dt = TYPES[c["type"]]
    H, Hkv, D = c["H"], c["Hkv"], c["D"]

    def normal(*shape, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32) * scale + shift).to(dt)

    s = dict(case=dict(c), scale=1.0 / math.sqrt(D))
    if c["op"] in ("prep", "prep_grad"):
        B, S = c["B"], c["S"]
        # one projection's output, of which q, k and v are strided views
        qkv = normal(B, S, H + 2 * Hkv, D, scale=1.5)
        s |= dict(q=qkv[:, :, :H], k=qkv[:, :, H:H + Hkv], v=qkv[:, :, H + Hkv:], q_weight=normal(D, scale=0.2, shift=1.0),
                  k_weight=normal(D, scale=0.2, shift=1.0), table=_table(S, c["R"], dev))
        if c["op"] == "prep_grad":
            s |= dict(dq=normal(B, H, S, D), dk=normal(B, Hkv, S, D), dv=normal(B, Hkv, S, D))
    elif c["op"] in ("window", "window_train"):
        B, Sq, Sk = c["B"], c["Sq"], c["Sk"]
        s |= dict(q=normal(B, H, Sq, D), k=normal(B, Hkv, Sk, D), v=normal(B, Hkv, Sk, D), q_offset=Sk - Sq)
        if c["op"] == "window_train":
            s["dout"] = normal(B, H, Sq, D)
    else:
        B, P, lens = c["B"], c["page"], _lengths(c)
        per_seq = -(-max(lens) // P)
        used = sum(-(-n // P) for n in lens)
        pages = used + 3
        order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
        table = torch.full((B, per_seq), -1, dtype=torch.int32)
        owner, at = order.cpu(), 0
        for b, n in enumerate(lens):     # the pages of a sequence, in the order in which they were handed out
            m = -(-n // P)
            table[b, :m] = owner[at:at + m]
            at += m
        shape = (pages, Hkv, P, D) if c["layout"] == "head" else (pages, P, Hkv, D)
        kc, vc = normal(*shape), normal(*shape)
        if c["layout"] == "slot":
            kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
        s |= dict(k_cache=kc, v_cache=vc, block_table=table.to(dev), seq_lens=torch.tensor(lens, dtype=torch.int32, device=dev))
        if c["op"] == "append":
            new = _new_tokens(c)
            tokens = sum(new)
            padded = tokens if c["new"] else -(-tokens // 64) * 64 + 64   # a prompt batch is padded to whole blocks
            qkv = normal(padded, H + 2 * Hkv, D, scale=1.5)
            starts = [0]
            for n in new:
                starts.append(starts[-1] + n)
            s |= dict(q=qkv[:, :H], k=qkv[:, H:H + Hkv], v=qkv[:, H + Hkv:], q_weight=normal(D, scale=0.2, shift=1.0),
                      k_weight=normal(D, scale=0.2, shift=1.0), table=_table(max(lens), c["R"], dev), q_out=torch.zeros(padded, H, D, dtype=dt, device=dev),
                      cu_seqlens=None if c["new"] else torch.tensor(starts, dtype=torch.int32, device=dev))
        else:
            s["q"] = normal(B, H, D)
    return s


# ------------------------------------------------------------------ plain forms

def _turn(x, cos, sin, R, interleaved, back=False):
    """The rotation of the first R values of each row, or its transpose."""
    if back:
        sin = -sin
    a, b, rest = (x[..., 0:R:2], x[..., 1:R:2], x[..., R:]) if interleaved else (x[..., :R // 2], x[..., R // 2:R], x[..., R:])
    y, z = a * cos - b * sin, b * cos + a * sin
    return torch.cat([torch.stack([y, z], -1).flatten(-2) if interleaved else torch.cat([y, z], -1), rest], -1)


def _plain_rows(x, weight, cos, sin, R, interleaved):
    x = x.float()
    n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    return _turn(n, cos, sin, R, interleaved)


def _plain_rows_grad(g, x, weight, cos, sin, R, interleaved):
    x, w = x.float(), weight.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    g = _turn(g.float(), cos, sin, R, interleaved, back=True)
    gw = g * w
    dx = r * gw - x * (r * r * r * (gw * x).mean(-1, keepdim=True))
    return dx, (g * x * r).sum((0, 1, 2))


def _angles(table, R):
    return table[..., :R // 2], table[..., R // 2:]


def _plain_prep(s):
    c = s["case"]
    cos, sin = (t[None, :, None] for t in _angles(s["table"], c["R"]))
    out = [_plain_rows(s[n], s[n + "_weight"], cos, sin, c["R"], c["interleaved"]).transpose(1, 2).to(s[n].dtype).contiguous() for n in "qk"]
    return out[0], out[1], s["v"].transpose(1, 2).contiguous()


def _plain_prep_grad(s):
    c = s["case"]
    cos, sin = (t[None, :, None] for t in _angles(s["table"], c["R"]))
    dq, dqw = _plain_rows_grad(s["dq"].transpose(1, 2), s["q"], s["q_weight"], cos, sin, c["R"], c["interleaved"])
    dk, dkw = _plain_rows_grad(s["dk"].transpose(1, 2), s["k"], s["k_weight"], cos, sin, c["R"], c["interleaved"])
    dt = s["q"].dtype
    return dq.to(dt), dk.to(dt), s["dv"].transpose(1, 2).contiguous(), dqw, dkw


def _window_blocks(s):
    """Blocks of queries beside the keys that any of them sees: the first tokens, then a run of keys.
    Returns (rows per block, blocks, key numbers [blocks, n], visible [blocks, rows, n])."""
    c, dev = s["case"], s["q"].device
    rows = min(512, c["Sq"])
    blocks = -(-c["Sq"] // rows)
    first = s["q_offset"] + torch.arange(blocks, device=dev) * rows                 # position of each block's first query
    run = first[:, None] - (c["window"] - 1) + torch.arange(min(c["window"] + rows - 1, c["Sk"] + c["window"]), device=dev)
    lead = torch.arange(c["sinks"], device=dev).expand(blocks, -1)
    keys = torch.cat([lead, run], 1)
    is_lead = torch.arange(keys.shape[1], device=dev) < c["sinks"]
    p = (first[:, None] + torch.arange(rows, device=dev))[:, :, None]
    j = keys[:, None, :]
    near = (j > p - c["window"]) & (j <= p) & (j >= 0) & (j < c["Sk"])
    # a first token inside the window is counted where the run has it
    seen = torch.where(is_lead, (j <= p - c["window"]) & (j < c["Sk"]), near)
    return rows, blocks, keys.clamp(0, c["Sk"] - 1), seen


def _plain_window(s, dout=None):
    c = s["case"]
    B, H, Hkv, D, Sq = c["B"], c["H"], c["Hkv"], c["D"], c["Sq"]
    rows, blocks, keys, seen = _window_blocks(s)
    extra = rows * blocks - Sq

    def split(x):      # [B,H,Sq,D] -> [B,Hkv,blocks,G*rows,D]
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, extra)).view(B, Hkv, H // Hkv, blocks, rows, D)
        return x.transpose(2, 3).reshape(B, Hkv, blocks, -1, D)

    def join(x):
        return x.view(B, Hkv, blocks, H // Hkv, rows, -1).transpose(2, 3).reshape(B, H, blocks * rows, -1)[:, :, :Sq]

    q, k, v = split(s["q"]), s["k"].float()[:, :, keys], s["v"].float()[:, :, keys]
    hidden = ~seen[:, None].expand(-1, H // Hkv, -1, -1).reshape(blocks, -1, keys.shape[1])
    x = (q @ k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(hidden, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = (x - m).exp_()
    l = p.sum(-1, keepdim=True)
    lse = (m + l.log())
    p = p / torch.where(l > 0, l, 1.0)
    o = p @ v
    out, lse = join(o).to(s["q"].dtype).contiguous(), join(lse).squeeze(-1).contiguous()
    if dout is None:
        return out, lse
    g = split(dout)
    dv = p.transpose(-1, -2) @ g
    ds = p * (g @ v.transpose(-1, -2) - (g * o).sum(-1, keepdim=True)) * s["scale"]
    dq = join(ds @ k)
    dk = ds.transpose(-1, -2) @ q
    dt, at = s["q"].dtype, keys.reshape(-1)
    dk = torch.zeros(s["k"].shape, dtype=torch.float32, device=dk.device).index_add_(2, at, dk.reshape(B, Hkv, -1, D))
    dv = torch.zeros(s["v"].shape, dtype=torch.float32, device=dv.device).index_add_(2, at, dv.reshape(B, Hkv, -1, D))
    return out, lse, dq.to(dt).contiguous(), dk.to(dt), dv.to(dt)


def _token_slots(s):
    """(live tokens, their positions, their pages) of a batch of new tokens."""
    c, dev = s["case"], s["q"].device
    lens, table = s["seq_lens"].long(), s["block_table"].long()
    t = torch.arange(s["q"].shape[0], device=dev)
    if s["cu_seqlens"] is None:
        seq, pos = t, lens - 1
    else:
        ends = s["cu_seqlens"].long()[1:]
        t = t[t < ends[-1]]
        seq = torch.searchsorted(ends, t, right=True)
        pos = lens[seq] - (ends[seq] - t)
    return t, pos, table[seq, pos // c["page"]]


def _plain_append(s):
    c = s["case"]
    t, pos, page = _token_slots(s)
    cos, sin = (x[pos][:, None] for x in _angles(s["table"], c["R"]))
    dt = s["q"].dtype
    s["q_out"][t] = _plain_rows(s["q"][t], s["q_weight"], cos, sin, c["R"], c["interleaved"]).to(dt)
    s["k_cache"][page, :, pos % c["page"]] = _plain_rows(s["k"][t], s["k_weight"], cos, sin, c["R"], c["interleaved"]).to(dt)
    s["v_cache"][page, :, pos % c["page"]] = s["v"][t]
    return s["q_out"], s["k_cache"], s["v_cache"]


def _plain_decode(s):
    c = s["case"]
    B, H, Hkv, D = c["B"], c["H"], c["Hkv"], c["D"]
    pages = s["block_table"].long().clamp(min=0)
    k = s["k_cache"][pages].transpose(2, 3).flatten(1, 2).transpose(1, 2).float()     # [B,Hkv,keys,D]
    v = s["v_cache"][pages].transpose(2, 3).flatten(1, 2).transpose(1, 2).float()
    j, n = torch.arange(k.shape[2], device=k.device), s["seq_lens"].long()[:, None]
    seen = j < n
    if c["window"]:
        seen = seen & ((j >= n - c["window"]) | (j < c["sinks"]))
    q = s["q"].float().view(B, Hkv, H // Hkv, D)
    x = (q @ k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = (x - m).exp_()
    l = p.sum(-1, keepdim=True)
    o = (p @ v) / l
    return o.view(B, H, D).to(s["q"].dtype), (m + l.log()).view(B, H)


# ------------------------------------------------------------------ one pass

def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2506_12355_b200 import api
        if c["op"] == "prep":
            return api.attn_qk_norm_rope(s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["table"], eps=EPS, interleaved=c["interleaved"])
        if c["op"] == "prep_grad":
            return api.attn_qk_norm_rope_bwd(s["dq"], s["dk"], s["dv"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["table"], eps=EPS,
                                             interleaved=c["interleaved"])
        if c["op"] == "window":
            return api.attn_fwd_window(s["q"], s["k"], s["v"], s["scale"], c["window"], c["sinks"], s["q_offset"])
        if c["op"] == "window_train":
            o, lse = api.attn_fwd_window(s["q"], s["k"], s["v"], s["scale"], c["window"], c["sinks"], s["q_offset"])
            return (o, lse) + api.attn_bwd_window(s["q"], s["k"], s["v"], o, lse, s["dout"], s["scale"], c["window"], c["sinks"], s["q_offset"])
        if c["op"] == "append":
            api.attn_paged_append(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["block_table"], s["seq_lens"], s["q_weight"], s["k_weight"],
                                  s["table"], cu_seqlens=s["cu_seqlens"], eps=EPS, interleaved=c["interleaved"], q_out=s["q_out"])
            return s["q_out"], s["k_cache"], s["v_cache"]
        return api.attn_paged_decode(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["seq_lens"], s["scale"], c["window"], c["sinks"])
    if c["op"] == "prep":
        return _plain_prep(s)
    if c["op"] == "prep_grad":
        return _plain_prep_grad(s)
    if c["op"] == "window":
        return _plain_window(s)
    if c["op"] == "window_train":
        return _plain_window(s, s["dout"])
    if c["op"] == "append":
        return _plain_append(s)
    return _plain_decode(s)


# ------------------------------------------------------------------ 64 bits

def _exact_rows(x, w, table, pos, R, interleaved):
    """One matrix of rows [N, heads, D] at positions [N], pair by pair from the definition."""
    x = x.double()
    y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * w.double()
    out = y.clone()
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        cos, sin = table[pos, i].double()[:, None], table[pos, R // 2 + i].double()[:, None]
        out[..., a] = y[..., a] * cos - y[..., b] * sin
        out[..., b] = y[..., a] * sin + y[..., b] * cos
    return out


def _exact_rows_grad(g, x, w, table, pos, R, interleaved):
    g, x, w = g.double(), x.double(), w.double()
    h = g.clone()
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        cos, sin = table[pos, i].double()[:, None], table[pos, R // 2 + i].double()[:, None]
        h[..., a] = g[..., a] * cos + g[..., b] * sin
        h[..., b] = g[..., b] * cos - g[..., a] * sin
    size = torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS)
    unit = x / size
    hw = h * w
    dx = (hw - unit * (hw * unit).sum(-1, keepdim=True) / x.shape[-1]) / size
    return dx, (h * unit).flatten(0, 1).sum(0)


def _exact_window(s):
    c = s["case"]
    G, W, off, train = c["H"] // c["Hkv"], c["window"], s["q_offset"], "dout" in s
    o, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["q"].shape[:3], dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(o), torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["v"].shape, dtype=torch.float64, device="cuda")
    for i in range(0, c["Sq"], 1024):
        n = min(1024, c["Sq"] - i)
        pos = torch.arange(i, i + n, device="cuda") + off
        j = torch.arange(c["Sk"], device="cuda")
        j = j[(j < c["sinks"]) | ((j > i + off - W) & (j < i + off + n))]
        vis = (j <= pos[:, None]) & ((j > pos[:, None] - W) | (j < c["sinks"]))
        for b in range(c["B"]):
            for g in range(c["Hkv"]):
                k, v = s["k"][b, g, j].double(), s["v"][b, g, j].double()
                h = slice(g * G, g * G + G)
                q = s["q"][b, h, i:i + n].double()
                x = torch.where(vis, q @ k.T * s["scale"], -math.inf)
                e = torch.logsumexp(x, -1)
                p = torch.where(vis, torch.exp(x - torch.where(e == -math.inf, 0.0, e)[..., None]), 0.0)
                o[b, h, i:i + n], lse[b, h, i:i + n] = p @ v, e
                if train:
                    do = s["dout"][b, h, i:i + n].double()
                    dp = do @ v.T
                    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * s["scale"]
                    dq[b, h, i:i + n] = ds @ k
                    dk[b, g, j] += (ds.transpose(1, 2) @ q).sum(0)
                    dv[b, g, j] += (p.transpose(1, 2) @ do).sum(0)
    return (o, lse, dq, dk, dv) if train else (o, lse)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] in ("prep", "prep_grad"):
        B, S = c["B"], c["S"]
        pos = torch.arange(S, device="cuda").repeat(B)
        more = (s["table"], pos, c["R"], c["interleaved"])

        def rows(x):     # [B,S,heads,D] -> [B*S,heads,D]
            return x.reshape(B * S, x.shape[2], c["D"])

        if c["op"] == "prep":
            q, k = (_exact_rows(rows(s[n]), s[n + "_weight"], *more).view(B, S, -1, c["D"]).transpose(1, 2) for n in "qk")
            return q, k, s["v"].double().transpose(1, 2)
        (dq, dqw), (dk, dkw) = (_exact_rows_grad(rows(s["d" + n].transpose(1, 2)), rows(s[n]), s[n + "_weight"], *more) for n in "qk")
        return dq.view(B, S, -1, c["D"]), dk.view(B, S, -1, c["D"]), s["dv"].double().transpose(1, 2), dqw, dkw
    if c["op"] in ("window", "window_train"):
        return _exact_window(s)
    lens = _lengths(c)
    if c["op"] == "append":
        qo, kc, vc = s["q_out"].double(), s["k_cache"].double(), s["v_cache"].double()
        at = 0
        for b, (n, new) in enumerate(zip(lens, _new_tokens(c))):
            pos = torch.arange(n - new, n, device="cuda")
            more, t = (s["table"], pos, c["R"], c["interleaved"]), slice(at, at + new)
            page, slot = s["block_table"][b].long()[pos // c["page"]], pos % c["page"]
            qo[t] = _exact_rows(s["q"][t], s["q_weight"], *more)
            kc[page, :, slot] = _exact_rows(s["k"][t], s["k_weight"], *more)
            vc[page, :, slot] = s["v"][t].double()
            at += new
        return qo, kc, vc
    G = c["H"] // c["Hkv"]
    o, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        j = torch.arange(n, device="cuda")
        if c["window"]:
            j = j[(j >= n - c["window"]) | (j < c["sinks"])]
        page, slot = s["block_table"][b].long()[j // c["page"]], j % c["page"]
        k, v = s["k_cache"][page, :, slot].double(), s["v_cache"][page, :, slot].double()      # [keys,Hkv,D]
        x = torch.einsum("gid,jgd->gij", s["q"][b].double().view(-1, G, c["D"]), k) * s["scale"]
        lse[b] = torch.logsumexp(x, -1).flatten()
        o[b] = torch.einsum("gij,jgd->gid", torch.softmax(x, -1), v).flatten(0, 1)
    return o, lse
