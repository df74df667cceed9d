"""Measured cases of three further operators around the attention kernels: query/key normalisation with a rotation over several
position axes (and its gradient, and the same on the way into the paged cache), attention of prompts over the paged cache, and one
new token's attention for a batch whose sequences share long prefixes.

listed() and draw() give the cases, prepare() makes their inputs, run() is one pass (the plain torch form, or the
library's entry points when `own` is true), work() counts the bytes and operations that a pass cannot do without,
and exact() computes the outputs in 64 bits from the definitions.

Definitions
  rows:     n = x / sqrt(mean(x^2) + eps) * weight over one head's D values, then the first R values rotated: pair i (i, i + R/2, or
            2i, 2i + 1 when interleaved) belongs to one of the axes (time, height, width, ..) and turns by the angle whose cosine
            and sine are column i of the table's row positions[axis of i][token].
  cache:    key j of sequence b lies in slot j % page_size of page block_table[b, j // page_size].
  prefill:  token i of the n new ones of a sequence of length len sees its keys j <= len - n + i.
  prefix:   the newest token of a sequence sees all its keys j < len; the sequences of a group have their first prefix_len keys in
            common.  Whole pages of those are the same pages; a page that the prefix fills in part is each sequence's own copy.
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
        # --- rotation over several axes
        # one small image before a vision encoder's attention, height and width: a launch-bound call
        dict(name="axes_image", op="axes", type="fp16", B=1, S=196, H=16, Hkv=16, D=64, R=64, axes=2, order="blocks", text=0, interleaved=False),
        # a long prompt with a video in it, time, height and width, runs of pairs per axis
        dict(name="axes_video", op="axes", type="bf16", B=1, S=16384, H=32, Hkv=8, D=128, R=128, axes=3, order="blocks", text=500, interleaved=False),
        # training on ragged sequences, half of each head rotated, adjacent pairs
        dict(name="axes_grad_ragged", op="axes_grad", type="fp16", B=3, S=1999, H=16, Hkv=4, D=64, R=32, axes=2, order="blocks", text=99,
             interleaved=True),
        # training at the batched causal configuration, the axes taking turns pair by pair
        dict(name="axes_grad_batch", op="axes_grad", type="bf16", B=4, S=2048, H=32, Hkv=8, D=128, R=128, axes=3, order="cyclic", text=100,
             interleaved=False),
        # prompts with images appended to the cache at once, padded at the end of the batch
        dict(name="axes_append_prompts", op="axes_append", type="bf16", B=8, low=100, high=4000, new=0, H=32, Hkv=8, D=128, R=128, axes=3,
             order="cyclic", page=64, layout="slot", interleaved=False),
        # one serving step of a batch: every sequence appends its new token
        dict(name="axes_append_step", op="axes_append", type="fp16", B=64, low=1, high=2048, new=1, H=16, Hkv=16, D=64, R=64, axes=3, order="blocks",
             page=16, layout="head", interleaved=False),
        # --- prompts over the paged cache
        # the next piece of a long prompt: few query tiles, a long key axis
        dict(name="prefill_chunk", op="prefill", type="bf16", B=1, past_low=14336, past_high=14336, new_low=2048, new_high=2048, shared=0, H=32,
             Hkv=8, D=128, page=16, layout="head"),
        # prompts of many lengths from their first token, no grouped heads
        dict(name="prefill_ragged", op="prefill", type="fp16", B=8, past_low=0, past_high=0, new_low=100, new_high=4000, shared=0, H=16, Hkv=16, D=64,
             page=64, layout="slot"),
        # short questions behind one long instruction
        dict(name="prefill_questions", op="prefill", type="bf16", B=32, past_low=4096, past_high=4096, new_low=10, new_high=200, shared=4096, H=32,
             Hkv=8, D=128, page=16, layout="head"),
        # --- shared prefixes
        # four samples of one short prompt: a latency-bound call
        dict(name="prefix_samples", op="prefix", type="bf16", B=4, groups=1, prefix=2000, low=1, high=100, H=32, Hkv=8, D=128, page=16, layout="head"),
        # a serving batch behind one long instruction
        dict(name="prefix_batch", op="prefix", type="bf16", B=64, groups=1, prefix=8192, low=1, high=1024, H=32, Hkv=8, D=128, page=16, layout="slot"),
        # three instructions of different lengths in one batch; no grouped heads
        dict(name="prefix_groups", op="prefix", type="fp16", B=100, groups=3, prefix=16000, low=1, high=2000, H=16, Hkv=16, D=64, page=64,
             layout="head"),
    ]


def _spread(rng, low, high):
    """A whole number whose logarithm is spread evenly over low .. high."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["axes", "axes_grad", "axes_append", "prefill", "prefill", "prefix", "prefix"])
    kind, D = rng.choice(["bf16", "fp16"]), rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    H = Hkv * rng.choice([1, 2, 3, 4, 8] if Hkv < 8 else [1, 2, 3, 4])
    c = dict(op=op, type=kind, H=H, Hkv=Hkv, D=D)
    if op.startswith("axes"):
        c |= dict(R=rng.choice([D, D // 2, 32]), axes=rng.choice([2, 3, 4]), order=rng.choice(["blocks", "cyclic"]), interleaved=rng.random() < 0.5)
    if op in ("axes", "axes_grad"):
        # at most the elements of the longest listed case
        tokens = _spread(rng, 1, min(32768, (16384 if op == "axes" else 8192) * 48 * 128 // ((H + 2 * Hkv) * D)))
        c["B"] = rng.randint(1, min(8, tokens))
        c["S"] = max(1, tokens // c["B"])
        c["text"] = rng.randint(0, c["S"])
    elif op == "axes_append":
        c["B"] = _spread(rng, 1, 128)
        c["high"] = _spread(rng, 2, max(2, 16384 // c["B"]))
        c["low"] = _spread(rng, 1, c["high"])
        c |= dict(new=rng.choice([0, 1]), page=rng.choice([8, 16, 64, 128]), layout=rng.choice(["head", "slot"]))
    elif op == "prefill":
        c["B"] = _spread(rng, 1, 64)
        most = 2048 * 15360 * 32 * 128 // (c["B"] * H * D)               # visible pairs of a head and sequence
        c["new_high"] = _spread(rng, 1, max(1, min(8192, 65536 // c["B"], int(math.sqrt(2 * most)))))
        c["new_low"] = _spread(rng, 1, c["new_high"])
        c["past_high"] = rng.choice([0, _spread(rng, 1, max(1, min(32768, 131072 // c["B"], (most - c["new_high"] ** 2 // 2) // c["new_high"] + 1)))])
        c["past_low"] = rng.randint(0, c["past_high"])
        c["shared"] = rng.choice([0, c["past_low"]])
        c |= dict(page=rng.choice([8, 16, 64, 128, 256]), layout=rng.choice(["head", "slot"]))
    else:
        c["B"] = _spread(rng, 1, 128)
        c["groups"] = rng.randint(1, min(4, c["B"]))
        c["prefix"] = _spread(rng, 1, 16384)
        c["high"] = _spread(rng, 2, max(2, min(16384, 64 * 1024 * 8 * 128 // (c["B"] * Hkv * D))))
        c["low"] = _spread(rng, 1, c["high"])
        c |= dict(page=rng.choice([8, 16, 64, 128]), layout=rng.choice(["head", "slot"]))
    return c


def _between(n, low, high):
    """n lengths spread over low .. high, the upper end among them; the same for every seed."""
    if n == 1:
        return [high]
    at = [(b * 0.6180339887498949) % 1.0 for b in range(n)]
    at[n // 2] = 1.0
    return [low + int(round(f * (high - low))) for f in at]


def _groups(c):
    """The groups of a batch with shared prefixes: (first sequences and the end, prefix lengths)."""
    n = c["groups"]
    return [c["B"] * g // n for g in range(n + 1)], [max(1, c["prefix"] * (g + 1) // n) for g in range(n)]


def _lengths(c):
    """The sequences' lengths, new tokens included."""
    if c["op"] == "axes_append":
        return _between(c["B"], c["low"], c["high"])
    if c["op"] == "prefill":
        return [p + n for p, n in zip(_past(c), _new_tokens(c))]
    starts, prefix = _groups(c)
    own_part = _between(c["B"], c["low"], c["high"])
    return [own_part[b] + prefix[g] for g in range(c["groups"]) for b in range(starts[g], starts[g + 1])]


def _past(c):
    return _between(c["B"], c["past_low"], c["past_high"])


def _new_tokens(c):
    """How many tokens each sequence brings to the call."""
    if c["op"] == "prefill":
        return _between(c["B"], c["new_low"], c["new_high"])[::-1]
    return [1 if c["new"] else n for n in _lengths(c)]


def _shared_runs(c):
    """Runs of sequences with common first keys: (first sequence, end, common keys)."""
    if c["op"] == "prefix":
        starts, prefix = _groups(c)
        return [(starts[g], starts[g + 1], prefix[g]) for g in range(c["groups"])]
    return [(0, c["B"], c["shared"])] if c["op"] == "prefill" and c["shared"] else []


def _pairs(c):
    """Visible (query, key) pairs of one head."""
    return sum(n * (length - n) + n * (n + 1) // 2 for n, length in zip(_new_tokens(c), _lengths(c)))


def _keys(c):
    """Keys that the call has to read, common ones once."""
    return sum(_lengths(c)) - sum((end - first - 1) * n for first, end, n in _shared_runs(c))


def work(case):
    c = case
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    if c["op"] in ("axes", "axes_grad"):
        rows = c["B"] * c["S"]
        table = _table_length(c) * c["R"] * 4 + 4 * D + rows * c["axes"] * 4
        if c["op"] == "axes":
            return {"bytes": rows * (H + 2 * Hkv) * D * 2 * 2 + table, "flops": rows * (H + Hkv) * D * 7}
        # gradients in and out for q, k, v; q and k themselves; two weight gradients in 32 bits
        return {"bytes": rows * D * 2 * (2 * (H + 2 * Hkv) + H + Hkv) + table + 8 * D, "flops": rows * (H + Hkv) * D * 16}
    if c["op"] == "axes_append":
        tokens = sum(_new_tokens(c))
        table = min(tokens * c["axes"], _table_length(c)) * c["R"] * 4
        return {"bytes": tokens * ((H + 2 * Hkv) * D * 2 * 2 + c["axes"] * 4 + 4) + table + 4 * D, "flops": tokens * (H + Hkv) * D * 7}
    keys = _keys(c) * (Hkv * D * 4) + -(-_keys(c) // c["page"]) * 4
    if c["op"] == "prefill":
        return {"bytes": keys + sum(_new_tokens(c)) * H * (4 * D + 4) + c["B"] * 8, "flops": 4 * D * H * _pairs(c)}
    return {"bytes": keys + c["B"] * (H * (4 * D + 4) + 4), "flops": 4 * D * H * sum(_lengths(c))}


# ------------------------------------------------------------------ inputs

def _grid(axes, n, text):
    """Positions [axes, n] of a prompt: `text` words, which have the same position on every axis, then pictures of 14 x 14 (or, with
    four axes, 7 x 14 x 2) patches, each axis counting from the last word on."""
    shape = {2: (14, 14), 3: (10 ** 6, 14, 14), 4: (10 ** 6, 7, 14, 2)}[axes]
    t = torch.arange(n)
    at, rest = [], (t - text).clamp(min=0)
    for size in reversed(shape[1:]):
        at.append(rest % size)
        rest = rest // size
    at.append(rest)
    return torch.stack([torch.where(t < text, t, text + a) for a in reversed(at)]).to(torch.int32)


def _table_length(c):
    """Rows of the rotation's table: the largest position and one more."""
    n = c["S"] if c["op"] in ("axes", "axes_grad") else max(_lengths(c))
    return int(_grid(c["axes"], n, c["text"] if "text" in c else n // 4).max()) + 1


def _sections(c):
    """Pairs of each axis: the first axis has what the even split of the others leaves."""
    pairs, n = c["R"] // 2, c["axes"]
    other = pairs // n if c["R"] < 64 else pairs // n // 4 * 4
    return [pairs - other * (n - 1)] + [other] * (n - 1)


def _pair_axes(c):
    """The axis of each pair: runs of pairs, or the axes in turn until their pairs are used up."""
    left = _sections(c)
    if c["order"] == "blocks":
        return [a for a, n in enumerate(left) for _ in range(n)]
    of = []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                of.append(a)
    return of


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
    if c["op"].startswith("axes"):
        s |= dict(q_weight=normal(D, scale=0.2, shift=1.0), k_weight=normal(D, scale=0.2, shift=1.0), table=_table(_table_length(c), c["R"], dev),
                  axis_of=torch.tensor(_pair_axes(c), device=dev), pair_axes=bytes(_pair_axes(c)))
    if c["op"] in ("axes", "axes_grad"):
        B, S = c["B"], c["S"]
        # one projection's output, of which q, k and v are strided views
        qkv = normal(B, S, H + 2 * Hkv, D, scale=1.5)
        s |= dict(q=qkv[:, :, :H], k=qkv[:, :, H:H + Hkv], v=qkv[:, :, H + Hkv:],
                  positions=_grid(c["axes"], S, c["text"]).to(dev)[:, None].expand(-1, B, -1).contiguous())
        if c["op"] == "axes_grad":
            s |= dict(dq=normal(B, H, S, D), dk=normal(B, Hkv, S, D), dv=normal(B, Hkv, S, D))
        return s
    B, P, lens = c["B"], c["page"], _lengths(c)
    per_seq = -(-max(lens) // P)
    table = torch.full((B, per_seq), -1, dtype=torch.int32)
    first_own = [0] * B                      # a sequence's first page that is not shared
    common = [(first, end, n // P) for first, end, n in _shared_runs(c)]
    pages = sum(-(-n // P) for n in lens) - sum((end - first - 1) * n for first, end, n in common) + 3
    owner, at = torch.randperm(pages, generator=gen, device=dev).to(torch.int32).cpu(), 0     # pages in the order in which they were handed out
    for first, end, n in common:
        table[first:end, :n] = owner[at:at + n]
        first_own[first:end] = [n] * (end - first)
        at += n
    for b, n in enumerate(lens):
        m = -(-n // P) - first_own[b]
        table[b, first_own[b]:first_own[b] + m] = owner[at:at + m]
        at += m
    shape = (pages, Hkv, P, D) if c["layout"] == "head" else (pages, P, Hkv, D)
    kc, vc = normal(*shape), normal(*shape)
    if c["layout"] == "slot":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    for first, end, n in _shared_runs(c):    # the page that a prefix fills in part
        if n % P:
            own_copies = table[first:end, n // P].long().to(dev)
            for cache in (kc, vc):
                cache[own_copies, :, :n % P] = cache[own_copies[0], :, :n % P].clone()
    s |= dict(k_cache=kc, v_cache=vc, block_table=table.to(dev), seq_lens=torch.tensor(lens, dtype=torch.int32, device=dev))
    if c["op"] == "prefix":
        starts, prefix = _groups(c)
        s |= dict(q=normal(B, H, D), group_starts=torch.tensor(starts, dtype=torch.int32, device=dev),
                  prefix_lens=torch.tensor(prefix, dtype=torch.int32, device=dev))
        return s
    new = _new_tokens(c)
    tokens = sum(new)
    padded = tokens if c["op"] == "axes_append" and c["new"] else -(-tokens // 64) * 64 + 64      # prompts come padded to whole blocks
    ends = [0]
    for n in new:
        ends.append(ends[-1] + n)
    cu = torch.tensor(ends, dtype=torch.int32, device=dev)
    if c["op"] == "prefill":
        s |= dict(q=normal(padded, H, D), cu_seqlens=cu, out=torch.zeros(padded, H, D, dtype=dt, device=dev),
                  lse=torch.zeros(padded, H, dtype=torch.float32, device=dev))
        return s
    qkv = normal(padded, H + 2 * Hkv, D, scale=1.5)
    positions = torch.zeros(c["axes"], padded, dtype=torch.int32)
    for b, n in enumerate(lens):
        positions[:, ends[b]:ends[b + 1]] = _grid(c["axes"], n, n // 4)[:, n - new[b]:]
    s |= dict(q=qkv[:, :H], k=qkv[:, H:H + Hkv], v=qkv[:, H + Hkv:], positions=positions.to(dev),
              q_out=torch.zeros(padded, H, D, dtype=dt, device=dev), cu_seqlens=None if c["new"] else cu)
    return s


# ------------------------------------------------------------------ plain forms

def _factors(s, positions):
    """Cosines and sines [.., R/2] of tokens with positions [axes, ..]."""
    R = s["case"]["R"]
    at = positions.long().movedim(0, -1)[..., s["axis_of"]]              # [.., R/2]: each pair's position
    col = torch.arange(R // 2, device=at.device)
    return s["table"][at, col], s["table"][at, R // 2 + col]


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


def _plain_axes(s):
    c = s["case"]
    cos, sin = (t[:, :, None] for t in _factors(s, s["positions"]))
    out = [_plain_rows(s[n], s[n + "_weight"], cos, sin, c["R"], c["interleaved"]).transpose(1, 2).to(s[n].dtype).contiguous() for n in "qk"]
    return out[0], out[1], s["v"].transpose(1, 2).contiguous()


def _plain_axes_grad(s):
    c = s["case"]
    cos, sin = (t[:, :, None] for t in _factors(s, s["positions"]))
    dq, dqw = _plain_rows_grad(s["dq"].transpose(1, 2), s["q"], s["q_weight"], cos, sin, c["R"], c["interleaved"])
    dk, dkw = _plain_rows_grad(s["dk"].transpose(1, 2), s["k"], s["k_weight"], cos, sin, c["R"], c["interleaved"])
    dt = s["q"].dtype
    return dq.to(dt), dk.to(dt), s["dv"].transpose(1, 2).contiguous(), dqw, dkw


def _plain_append(s):
    c, dev = s["case"], s["q"].device
    lens, table = s["seq_lens"].long(), s["block_table"].long()
    t = torch.arange(s["q"].shape[0], device=dev)
    if s["cu_seqlens"] is None:
        seq, slot = t, lens - 1
    else:
        ends = s["cu_seqlens"].long()[1:]
        t = t[t < ends[-1]]
        seq = torch.searchsorted(ends, t, right=True)
        slot = lens[seq] - (ends[seq] - t)
    page = table[seq, slot // c["page"]]
    cos, sin = (x[:, None] for x in _factors(s, s["positions"][:, t]))
    dt = s["q"].dtype
    s["q_out"][t] = _plain_rows(s["q"][t], s["q_weight"], cos, sin, c["R"], c["interleaved"]).to(dt)
    s["k_cache"][page, :, slot % c["page"]] = _plain_rows(s["k"][t], s["k_weight"], cos, sin, c["R"], c["interleaved"]).to(dt)
    s["v_cache"][page, :, slot % c["page"]] = s["v"][t]
    return s["q_out"], s["k_cache"], s["v_cache"]


def _gather(cache, pages):
    """Rows of the cache [.., Hkv, keys, D] in 32 bits, for pages [.., n]."""
    return cache[pages.clamp(min=0)].transpose(-4, -3).flatten(-3, -2).float()


def _plain_prefill(s):
    c = s["case"]
    H, Hkv, D, P = c["H"], c["Hkv"], c["D"], c["page"]
    at = 0
    for b, (n, length) in enumerate(zip(_new_tokens(c), _lengths(c))):
        pages = s["block_table"][b, :-(-length // P)].long()
        k, v = (_gather(s[name], pages)[:, :length] for name in ("k_cache", "v_cache"))
        q = s["q"][at:at + n].float().view(n, Hkv, H // Hkv, D).transpose(0, 1)
        pos = torch.arange(length - n, length, device=k.device)
        hidden = torch.arange(length, device=k.device) > pos[:, None]
        step = max(1, min(n, 2 ** 28 // (H * length)))                    # query tokens at a time
        for i in range(0, n, step):
            x = (q[:, i:i + step].flatten(1, 2) @ k.transpose(-1, -2)).mul_(s["scale"]).view(Hkv, -1, H // Hkv, length)
            x.masked_fill_(hidden[i:i + step, None], -math.inf)
            m = x.amax(-1, keepdim=True)
            p = x.sub_(m).exp_()
            l = p.sum(-1, keepdim=True)
            o = (p.flatten(1, 2) @ v).view(Hkv, -1, H // Hkv, D) / l
            s["out"][at + i:at + min(n, i + step)] = o.transpose(0, 1).flatten(1, 2).to(s["q"].dtype)
            s["lse"][at + i:at + min(n, i + step)] = (m + l.log()).transpose(0, 1).flatten(1)
        at += n
    return s["out"], s["lse"]


def _plain_prefix(s):
    c = s["case"]
    H, Hkv, D, P = c["H"], c["Hkv"], c["D"], c["page"]
    outs, lses = [], []
    starts, prefix = _groups(c)
    lens = _lengths(c)
    for g in range(c["groups"]):
        b0, b1, n = starts[g], starts[g + 1], prefix[g]
        q = s["q"][b0:b1].float().view(-1, Hkv, H // Hkv, D)
        # the prefix once for the group: the rows of all its sequences side by side
        kp, vp = (_gather(s[name], s["block_table"][b0, :-(-n // P)].long())[:, :n] for name in ("k_cache", "v_cache"))
        xp = (q.transpose(0, 1).flatten(1, 2) @ kp.transpose(-1, -2)).mul_(s["scale"]).view(Hkv, b1 - b0, -1, n).transpose(0, 1)
        # each sequence's own keys, from the page in which the prefix ends
        skip, longest = n // P, max(lens[b0:b1])
        k, v = (_gather(s[name], s["block_table"][b0:b1, skip:-(-longest // P)].long()) for name in ("k_cache", "v_cache"))
        j = torch.arange(k.shape[2], device=k.device) + skip * P
        hidden = (j < n) | (j >= s["seq_lens"][b0:b1].long()[:, None])
        xs = (q @ k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(hidden[:, None, None], -math.inf)
        v = v.masked_fill(hidden[:, None, :, None], 0.0)
        m = torch.maximum(xp.amax(-1, keepdim=True), xs.amax(-1, keepdim=True))
        pp, ps = (xp - m).exp_(), (xs - m).exp_()
        l = pp.sum(-1, keepdim=True) + ps.sum(-1, keepdim=True)
        o = (pp.transpose(0, 1).flatten(1, 2) @ vp).view(Hkv, b1 - b0, -1, D).transpose(0, 1) + ps @ v
        outs.append((o / l).reshape(b1 - b0, H, D).to(s["q"].dtype))
        lses.append((m + l.log()).reshape(b1 - b0, H))
    return torch.cat(outs), torch.cat(lses)


# ------------------------------------------------------------------ one pass

def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2506_12355_b200 import api
        if c["op"] == "axes":
            return api.attn_qk_norm_rope_axes(s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["table"], s["positions"], s["pair_axes"], eps=EPS,
                                              interleaved=c["interleaved"])
        if c["op"] == "axes_grad":
            return api.attn_qk_norm_rope_axes_bwd(s["dq"], s["dk"], s["dv"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["table"], s["positions"],
                                                  s["pair_axes"], eps=EPS, interleaved=c["interleaved"])
        if c["op"] == "axes_append":
            api.attn_paged_append_axes(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["block_table"], s["seq_lens"], s["positions"],
                                       s["pair_axes"], s["q_weight"], s["k_weight"], s["table"], cu_seqlens=s["cu_seqlens"], eps=EPS,
                                       interleaved=c["interleaved"], q_out=s["q_out"])
            return s["q_out"], s["k_cache"], s["v_cache"]
        if c["op"] == "prefill":
            return api.attn_paged_prefill(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["seq_lens"], s["cu_seqlens"], s["scale"],
                                          out=s["out"], lse=s["lse"])
        return api.attn_paged_prefix_decode(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["seq_lens"], s["group_starts"],
                                            s["prefix_lens"], s["scale"])
    if c["op"] == "axes":
        return _plain_axes(s)
    if c["op"] == "axes_grad":
        return _plain_axes_grad(s)
    if c["op"] == "axes_append":
        return _plain_append(s)
    if c["op"] == "prefill":
        return _plain_prefill(s)
    return _plain_prefix(s)


# ------------------------------------------------------------------ 64 bits

def _exact_rows(s, x, w, pos, back=False):
    """One matrix of rows [N, heads, D] at positions [axes, N], pair by pair from the definition; back: the transposed rotation
    of x alone."""
    c = s["case"]
    R, of = c["R"], _pair_axes(c)
    y = x.double()
    if not back:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / y.shape[-1] + EPS) * w.double()
    out = y.clone()
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + R // 2)
        row = s["table"][pos[of[i]].long()].double()
        cos, sin = row[:, i, None], row[:, R // 2 + i, None] * (-1 if back else 1)
        out[..., a] = y[..., a] * cos - y[..., b] * sin
        out[..., b] = y[..., a] * sin + y[..., b] * cos
    return out


def _exact_rows_grad(s, g, x, w, pos):
    h, x = _exact_rows(s, g, None, pos, back=True), x.double()
    size = torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS)
    unit = x / size
    hw = h * w.double()
    dx = (hw - unit * (hw * unit).sum(-1, keepdim=True) / x.shape[-1]) / size
    return dx, (h * unit).flatten(0, 1).sum(0)


def _sequence(s, b, length):
    """Keys and values [length, Hkv, D] of sequence b."""
    j = torch.arange(length, device="cuda")
    page, slot = s["block_table"][b].long()[j // s["case"]["page"]], j % s["case"]["page"]
    return s["k_cache"][page, :, slot].double(), s["v_cache"][page, :, slot].double()


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] in ("axes", "axes_grad"):
        B, S = c["B"], c["S"]
        pos = s["positions"].flatten(1)

        def rows(x):     # [B,S,heads,D] -> [B*S,heads,D]
            return x.reshape(B * S, x.shape[2], c["D"])

        if c["op"] == "axes":
            q, k = (_exact_rows(s, rows(s[n]), s[n + "_weight"], pos).view(B, S, -1, c["D"]).transpose(1, 2) for n in "qk")
            return q, k, s["v"].double().transpose(1, 2)
        (dq, dqw), (dk, dkw) = (_exact_rows_grad(s, rows(s["d" + n].transpose(1, 2)), rows(s[n]), s[n + "_weight"], pos) for n in "qk")
        return dq.view(B, S, -1, c["D"]), dk.view(B, S, -1, c["D"]), s["dv"].double().transpose(1, 2), dqw, dkw
    lens, G = _lengths(c), c["H"] // c["Hkv"]
    at = 0
    if c["op"] == "axes_append":
        qo, kc, vc = s["q_out"].double(), s["k_cache"].double(), s["v_cache"].double()
        for b, (n, new) in enumerate(zip(lens, _new_tokens(c))):
            j, t = torch.arange(n - new, n, device="cuda"), slice(at, at + new)
            page, slot = s["block_table"][b].long()[j // c["page"]], j % c["page"]
            qo[t] = _exact_rows(s, s["q"][t], s["q_weight"], s["positions"][:, t])
            kc[page, :, slot] = _exact_rows(s, s["k"][t], s["k_weight"], s["positions"][:, t])
            vc[page, :, slot] = s["v"][t].double()
            at += new
        return qo, kc, vc
    if c["op"] == "prefix":
        o, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            k, v = _sequence(s, b, n)
            x = torch.einsum("gid,jgd->gij", s["q"][b].double().view(-1, G, c["D"]), k) * s["scale"]
            lse[b] = torch.logsumexp(x, -1).flatten()
            o[b] = torch.einsum("gij,jgd->gid", torch.softmax(x, -1), v).flatten(0, 1)
        return o, lse
    o, lse = s["out"].double(), s["lse"].double()
    for b, (n, length) in enumerate(zip(_new_tokens(c), lens)):
        k, v = _sequence(s, b, length)
        j = torch.arange(length, device="cuda")
        for i in range(0, n, 256):
            rows = slice(at + i, at + min(n, i + 256))
            q = s["q"][rows].double().view(-1, c["Hkv"], G, c["D"])
            x = torch.einsum("igrd,jgd->girj", q, k) * s["scale"]
            p = torch.arange(length - n + i, length - n + i + q.shape[0], device="cuda")
            x.masked_fill_((j > p[:, None])[None, :, None], -math.inf)
            lse[rows] = torch.logsumexp(x, -1).transpose(0, 1).flatten(1)
            o[rows] = torch.einsum("girj,jgd->igrd", torch.softmax(x, -1), v).flatten(1, 2)
        at += n
    return o, lse
