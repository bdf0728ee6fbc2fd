"""A paged key-value cache made smaller, as cases that can be timed and compared: held in 8 bits,
and without the slots that attention has had no use for.

In 8 bits: the pools hold e4m3 codes, and every block of 16 slots of a KV-head has a scale for its
keys and one for its values (fp32, powers of two when `append8` has set them), a value being code
times scale. `append8` rotates and quantises new tokens into the pages of their sequences; a block
that is partly filled keeps the larger scale and has its older codes brought to it. `decode8`
attends from one new token of every sequence, `prefill8` from several.

Eviction: `weigh` adds up, slot by slot, the attention weights that new tokens give to the slots
they see, over the query heads of a KV-head; `decode_weigh` does so beside the attention of one new
token per sequence; `evict` keeps, of every sequence and KV-head, the first slots, the last ones and
the heaviest of the others, in their order, in pages of a cache of their own.

Caches are pools of pages [n_pages, page, H, d] (in memory slots before heads or heads before
slots) with an optional logit bias per slot [n_pages, H, page] (fp32), weights have the layout of
biases, and a table lists every sequence's pages. `lens` counts a sequence's slots with this call's
tokens, which are its last ones.

With `own` false the calls are written in elementary torch operations in fp32; `exact` restates
them in 64 bits, one sequence and KV-head at a time.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
E4M3 = torch.float8_e4m3fn
BLOCK = 16             # slots of a KV-head that share a scale
_MOST_SLOTS = 250_000  # of a drawn case's cache, with 8 KV-heads of 128 channels
_MOST_SCORES = 0.9e9   # of a drawn case of many tokens with 128 channels: queries x heads x slots


def listed():
    return [
        # a decode step of a small model for three sequences, inside blocks: latency
        dict(name="append8_step_3x_h2", op="append8", B=3, past="777:790", new="1", H=2, Hq=8, d=64,
             page=16, beta=False, heads_first=False, theta=1e4, offset=0),
        # a chunk of a long prompt on its way into the cache, behind a block that is partly filled
        dict(name="append8_chunk_8k", op="append8", B=1, past="8185", new="8192", H=8, Hq=32, d=128,
             page=64, beta=False, heads_first=False, theta=1e6, offset=0),
        # eight compacted documents (t = 1311, biases) and what was said since
        dict(name="decode8_8x_compacted", op="decode8", B=8, past="1311:5407", new="1", H=8, Hq=32,
             d=128, page=32, beta=True, heads_first=False, offset=64225),
        # uncompacted documents of ragged length, seven query heads to a KV-head
        dict(name="decode8_24x_8k_32k", op="decode8", B=24, past="8192:32768", new="1", H=4, Hq=28,
             d=128, page=64, beta=False, heads_first=True, offset=0),
        # a question of odd length after each of four compacted documents
        dict(name="prefill8_question_4x", op="prefill8", B=4, past="655:1311", new="17:101", H=8,
             Hq=32, d=128, page=32, beta=True, heads_first=False, offset=64225),
        # a whole prompt, seven query heads to a KV-head
        dict(name="prefill8_prompt_8k_g7", op="prefill8", B=1, past="0", new="8192", H=4, Hq=28,
             d=128, page=64, beta=False, heads_first=True, offset=0),
        # a decode step that keeps count for later evictions, ragged documents, one place idle
        dict(name="decode_weigh_8x_8k", op="decode_weigh", B=8, past="5000:9001", new="1", H=8,
             Hq=32, d=128, page=32, beta=False, heads_first=False, idle=1, decay=1.0),
        # the same of one very long document, 256 channels, older steps counting less
        dict(name="decode_weigh_131072_d256", op="decode_weigh", B=1, past="131071", new="1", H=8,
             Hq=16, d=256, page=128, beta=False, heads_first=False, decay=0.95),
        # the last 64 tokens of four prompts look back: what their answers will need
        dict(name="weigh_window_4x_32k", op="weigh", B=4, past="9000:32700", new="64", H=8, Hq=32,
             d=128, page=64, beta=True, heads_first=False, decay=0.0),
        # all tokens of an odd prompt, seven query heads to a KV-head
        dict(name="weigh_prompt_6k_g7", op="weigh", B=1, past="0", new="6001", H=4, Hq=28, d=128,
             page=64, beta=False, heads_first=True, decay=1.0),
        # a batch of short conversations of a small model, down to 164 slots
        dict(name="evict_32x_short", op="evict", B=32, past="700:1500", new="0", H=2, d=64, page=16,
             beta=True, heads_first=False, offset=0, keep=164, sinks=4, recent=32),
        # one very long document, to an eighth
        dict(name="evict_131072_to_16384", op="evict", B=1, past="131072", new="0", H=8, d=128,
             page=64, beta=False, heads_first=False, offset=0, keep=16384, sinks=4, recent=256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append8", "decode8", "decode8", "prefill8", "prefill8", "decode_weigh",
                     "weigh", "weigh", "evict", "evict"])
    d = rng.choice([64, 128, 128, 256])
    H = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 3, 4, 5, 7, 8, 16])
    c = dict(op=op, H=H, Hq=H * g, d=d, page=rng.choice([16, 32, 64, 128, 256]),
             beta=rng.random() < 0.5, heads_first=rng.random() < 0.4)
    if op not in ("decode_weigh", "weigh"):
        c["offset"] = rng.choice([0, 0, rng.randint(1, 1 << 20)])
    else:
        c["decay"] = rng.choice([0.0, 1.0, 1.0, round(rng.uniform(0.5, 0.999), 3)])
    if op == "append8":
        c["theta"] = rng.choice([1e4, 1e6])
        if rng.random() < 0.3:  # compact slots
            c |= dict(theta=0.0, Hq=0)
        total = _log(rng, 1, 8192 * 1024 // (H * d * min(g, 4)))
        c["B"] = min(total, rng.choice([1, 1, 3, 8, 32]))
        new = max(1, total // c["B"])
        c |= dict(new="%d:%d" % (max(1, new // 2), new), past="0:%d" % rng.choice([0, 100, 4000]))
        return c
    if op in ("decode8", "decode_weigh", "evict"):
        slots = _log(rng, 1, _MOST_SLOTS * 1024 // (H * d))
        c["B"] = min(slots, rng.choice([1, 1, 2, 8, 32, 128]))
        most = min(max(1, slots // c["B"]), 262144)
        c["past"] = "%d:%d" % (max(1, most // rng.choice([1, 3])), most)
        if op != "evict":
            c |= dict(new="1", idle=rng.choice([0, 0, 1]) if c["B"] > 1 else 0)
            return c
        del c["Hq"]
        keep = _log(rng, 1, most)
        keep = max(1, min(keep, most * 3 // 4))
        recent = rng.randint(0, keep // 2)
        c |= dict(new="0", keep=keep, recent=recent, sinks=rng.randint(0, min(4, keep - recent)))
        return c
    scores = math.exp(rng.uniform(math.log(1e4), math.log(_MOST_SCORES * min(1, 128 / d))))
    c["B"] = rng.choice([1, 1, 2, 5])
    new = max(1, min(8192, _log(rng, 2, max(3, int(math.sqrt(scores / (c["B"] * H * g)))))))
    past = int(min(65536, scores / (c["B"] * H * g * new), _MOST_SLOTS * 1024 / (c["B"] * H * d)))
    past = max(0, past - new)
    least = rng.choice([1, 2])
    c |= dict(new="%d:%d" % (max(1, new // least), new), past="%d:%d" % (past // least, past))
    return c


def _spread(text, count, salt):
    """`count` whole numbers spread evenly in "lo:hi" (or all of them "n"), in a mixed order."""
    lo, _, hi = text.partition(":")
    lo, hi = int(lo), int(hi or lo)
    got = [lo + (hi - lo) * i // max(1, count - 1) for i in range(count)]
    random.Random(salt).shuffle(got)
    return got if count > 1 else [hi]


def _counts(case):
    """New tokens and slots (with them) of every sequence; idle places of a batch have none."""
    B = case["B"]
    new = _spread(case["new"], B, 1)
    lens = [p + n for p, n in zip(_spread(case["past"], B, 2), new)]
    for b in range(case.get("idle", 0)):
        lens[(7 * b + 1) % B] = 0
    return new, lens


# ------------------------------------------------------------------------------ states

def _least_scale(top):
    """The smallest power of two, 2^-126 at least, by which values up to `top` are 448 at most."""
    m, e = torch.frexp(top)
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(top > 0, e.clamp_min(-126), -126)
    return torch.ldexp(torch.ones_like(top), e)


def _laid_out(x, case):
    """[n_pages, page, H, d] in the case's order of memory."""
    return x.transpose(1, 2).contiguous().transpose(1, 2) if case["heads_first"] else x


def _pools(gen, case, n_pages):
    """Keys and values of every slot, bf16, one outlier key channel per head as in real caches."""
    H, d, page = case["H"], case["d"], case["page"]
    K, V = (torch.empty(n_pages, page, H, d, device=DEVICE, dtype=torch.bfloat16).normal_(
        generator=gen) for _ in range(2))
    heavy = torch.randint(0, d, (H, 1), generator=gen, device=DEVICE)
    K *= 1 + 7 * torch.zeros(H, d, device=DEVICE, dtype=torch.bfloat16).scatter_(1, heavy, 1)
    return K, V


def _quantised(x, case):
    """A pool in 8 bits, and its scales [n_pages, H, page / 16]."""
    n_pages, page, H, d = x.shape
    scale = _least_scale(x.view(n_pages, -1, BLOCK, H, d).abs().amax((2, 4)).float())
    rows = scale.repeat_interleave(BLOCK, 1)[..., None]
    return _laid_out((x.float() / rows).to(E4M3), case), scale.transpose(1, 2).contiguous()


def _table(gen, lens, page):
    """Pages for so many slots per sequence, in the order that an allocator left them."""
    need = [max(1, -(-x // page)) for x in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device=DEVICE).to(torch.int32)
    table = torch.zeros(len(lens), max(need), dtype=torch.int32, device=DEVICE)
    taken = 0
    for b, k in enumerate(need):
        table[b, :k] = order[taken:taken + k]
        taken += k
    return table, n_pages


def prepare(case, seed):
    """A program's cache (what is in no sequence stale), table and lengths, the rows of the fused
    q, k, v projection of its new tokens, and the buffers that its calls write."""
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    H, Hq, d, page, B = case["H"], case.get("Hq", 0), case["d"], case["page"], case["B"]
    new, lens = _counts(case)
    table, n_pages = _table(gen, lens, page)
    s = dict(case=case, n=sum(new), new=new, table=table, beta=None, cu_new=None,
             lens=torch.tensor(lens, dtype=torch.int32, device=DEVICE),
             offset=torch.full((B,), case.get("offset", 0), dtype=torch.int64, device=DEVICE))
    K, V = _pools(gen, case, n_pages)
    if case["op"].endswith("8"):
        s["K"], s["k_scale"] = _quantised(K, case)
        s["V"], s["v_scale"] = _quantised(V, case)
    else:
        s["K"], s["V"] = _laid_out(K, case), _laid_out(V, case)
    del K, V
    if case["beta"]:
        s["beta"] = torch.empty(n_pages, H, page, device=DEVICE).normal_(generator=gen)
    if "weigh" in case["op"] or case["op"] == "evict":  # of some earlier steps: many of none
        w = torch.empty(n_pages, H, page, device=DEVICE).normal_(generator=gen)
        s["weight"] = torch.where(w > -1, (2 * w).exp() * (4.0 / max(lens)), 0.0)
    if case["op"] == "evict":
        kept = [min(x, case["keep"]) for x in lens]
        s["to_table"], to_pages = _table(gen, kept, page)
        shape = (to_pages, page, H, d)
        s["to_K"], s["to_V"] = (_laid_out(torch.zeros(shape, device=DEVICE, dtype=torch.bfloat16),
                                          case) for _ in range(2))
        s["to_beta"] = torch.zeros(to_pages, H, page, device=DEVICE) if case["beta"] else None
        s["to_weight"] = torch.zeros(to_pages, H, page, device=DEVICE)
        s["kept"] = torch.empty(B, H, case["keep"], dtype=torch.int32, device=DEVICE)
        s["to_lens"], s["to_offset"] = torch.empty_like(s["lens"]), torch.empty_like(s["offset"])
        return s
    # cumulative new tokens: absent where every sequence has one
    if "decode" not in case["op"] and any(x != 1 for x in new):
        s["cu_new"] = torch.tensor([0] + new, device=DEVICE).cumsum(0).to(torch.int32)
    rows = torch.empty(s["n"], (Hq + 2 * H) * d, device=DEVICE,
                       dtype=torch.bfloat16).normal_(generator=gen)
    q, k, v = rows.split([Hq * d, H * d, H * d], 1)
    s["q"] = q.unflatten(1, (Hq, d)) if Hq else None
    s["out"] = None
    if Hq and case["op"] != "weigh":
        s["out"] = torch.empty(s["n"], Hq, d, device=DEVICE, dtype=torch.bfloat16)
    if case["op"] == "append8":
        s["k"], s["v"] = k.unflatten(1, (H, d)), v.unflatten(1, (H, d))
        s["new_beta"] = None
        if case["beta"] and not case["theta"]:  # compact slots come with their biases
            s["new_beta"] = torch.empty(s["n"], H, device=DEVICE).normal_(generator=gen)
    return s


# ------------------------------------------------------------------------------ passes

_context = None


def _own(s):
    """The calls of the framework, with the handles and scratch that a program makes once."""
    global _context
    from paper_2606_07878_gb300 import still
    if _context is None:
        _context = still.still_create(0)
    c = s["case"]
    op = c["op"]
    if "cache" not in s:
        s["batch"] = still.PagedBatch(s["table"], s["lens"], s["cu_new"], s["offset"])
        if op.endswith("8"):
            s["cache"] = still.PagedCacheQuant(s["K"], s["V"], s["k_scale"], s["v_scale"],
                                               s["beta"])
        else:
            s["cache"] = still.PagedCache(s["K"], s["V"], s["beta"])
        if "weigh" in op:
            size = still.still_paged_weigh_scratch(s["cache"], s["n"], c["Hq"])
            s["scratch"] = torch.empty(size, dtype=torch.uint8, device=DEVICE)
        if op == "evict":
            s["to"] = still.PagedCache(s["to_K"], s["to_V"], s["to_beta"])
    if op == "append8":
        still.still_paged_append_quant(_context, s["cache"], s["batch"], s["k"], s["v"],
                                       q=s["q"], q_out=s["out"], beta=s["new_beta"],
                                       rope_theta=c["theta"])
    elif op == "decode8":
        still.still_paged_decode_quant(_context, s["cache"], s["batch"], s["q"], s["out"])
    elif op == "prefill8":
        still.still_paged_prefill_quant(_context, s["cache"], s["batch"], s["q"], s["out"])
    elif op == "decode_weigh":
        still.still_paged_decode_weigh(_context, s["cache"], s["batch"], s["q"], s["out"],
                                       s["weight"], s["scratch"], decay=c["decay"])
    elif op == "weigh":
        still.still_paged_weigh(_context, s["cache"], s["batch"], s["q"], s["weight"],
                                s["scratch"], decay=c["decay"])
    else:
        still.still_paged_evict(_context, s["cache"], s["batch"], s["weight"], c["keep"],
                                c["sinks"], c["recent"], s["to"], s["to_table"], s["kept"],
                                s["to_lens"], to_weight=s["to_weight"], to_offset=s["to_offset"])
    return _outputs(s)


def _outputs(s):
    op = s["case"]["op"]
    if op == "append8":  # 8-bit values, and what they are multiples of
        names = ["K", "V", "k_scale", "v_scale", "beta", "out"]
    elif op == "evict":
        names = ["to_K", "to_V", "to_beta", "to_weight", "kept", "to_lens", "to_offset"]
    else:
        names = ["out", "weight"]
    return {x: s[x] for x in names if s.get(x) is not None}


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    if op == "append8":
        _plain_append(s)
    elif op == "evict":
        _plain_evict(s)
    else:
        _plain_attention(s)
    return _outputs(s)


def _places(s):
    """Sequence and slot of every new token."""
    B, n = s["case"]["B"], s["n"]
    if s["cu_new"] is None:
        seq = torch.arange(B, device=DEVICE)
        return seq, s["lens"].long() - 1
    cu = s["cu_new"].long()
    at = torch.arange(n, device=DEVICE)
    seq = torch.bucketize(at, cu[1:], right=True)
    return seq, s["lens"].long()[seq] - cu[seq + 1] + at


def _rotated(x, pos, theta):
    """x [n, heads, d] rotated in pairs (m, m + d/2); angles from 64-bit products."""
    x = x.float()
    half = x.shape[2] // 2
    m = torch.arange(half, device=DEVICE, dtype=torch.float64)
    a = pos.double()[:, None] * theta ** (-m / half)
    cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
    lo, hi = x[..., :half], x[..., half:]
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], 2)


def _plain_put(pool, scales, x, page, at):
    """Rows x [n, H, d] into slots `at` of pages `page`: codes, and scales of their blocks."""
    H, d = x.shape[1:]
    per = scales.shape[2]
    blocks, seat = torch.unique(page * per + at // BLOCK, return_inverse=True)
    where, which = blocks // per, blocks % per
    new = torch.zeros(len(blocks), H, device=DEVICE)
    new.scatter_reduce_(0, seat[:, None].expand(-1, H), x.float().abs().amax(2), "amax")
    first = torch.full((len(blocks),), BLOCK, device=DEVICE)
    first.scatter_reduce_(0, seat, at % BLOCK, "amin")
    old = torch.where(first[:, None] > 0, scales[where, :, which], 0.0)
    scale = torch.maximum(_least_scale(new), old)
    scales[where, :, which] = scale
    codes = pool.view(torch.uint8)
    slots = which[:, None] * BLOCK + torch.arange(BLOCK, device=DEVICE)  # [blocks, 16]
    held = codes[where[:, None], slots].view(E4M3)  # [blocks, 16, H, d]
    brought = (held.float() * (old / scale)[:, None, :, None]).to(E4M3)
    older = (torch.arange(BLOCK, device=DEVICE) < first[:, None])[..., None, None]
    codes[where[:, None], slots] = torch.where(older, brought.view(torch.uint8),
                                               held.view(torch.uint8))
    codes[page, at] = (x.float() / scale[seat][..., None]).to(E4M3).view(torch.uint8)


def _plain_append(s):
    c = s["case"]
    seq, slot = _places(s)
    k, theta = s["k"], c["theta"]
    if theta:
        pos = slot + s["offset"][seq]
        k = _rotated(k, pos, theta).bfloat16()  # the key that a cache of 16 bits would hold
        if s["q"] is not None:
            s["out"].copy_(_rotated(s["q"], pos, theta))
    page, at = s["table"].long()[seq, slot // c["page"]], slot % c["page"]
    _plain_put(s["K"], s["k_scale"], k, page, at)
    _plain_put(s["V"], s["v_scale"], s["v"], page, at)
    if s["beta"] is not None:
        s["beta"][page, :, at] = s["new_beta"] if s["new_beta"] is not None else 0.0


def _read(s, name):
    """Keys or values of every sequence's slots [B, slots, H, d], fp32."""
    table, pool = s["table"].long(), s[name]
    if pool.dtype != E4M3:
        return pool[table].flatten(1, 2).float()
    x = pool.view(torch.uint8)[table].view(E4M3).flatten(1, 2).float()
    scale = s[name.lower() + "_scale"][table].transpose(2, 3).flatten(1, 2)  # [B, blocks, H]
    return x.mul_(scale.repeat_interleave(BLOCK, 1)[..., None])


def _plain_attention(s):
    c = s["case"]
    B, H, Hq, d, page = c["B"], c["H"], c["Hq"], c["d"], c["page"]
    seq, slot = _places(s)
    wide = max(s["new"])
    first = s["cu_new"].long()[seq] if s["cu_new"] is not None else seq
    col = torch.arange(s["n"], device=DEVICE) - first
    q = torch.zeros(B, wide, Hq, d, device=DEVICE)
    q[seq, col] = s["q"].float()
    seen = torch.zeros(B, wide, dtype=torch.long, device=DEVICE)
    seen[seq, col] = slot + 1
    table = s["table"].long()
    k = _read(s, "K")
    T = k.shape[1]
    q = q.view(B, wide, H, Hq // H, d).permute(0, 2, 3, 1, 4).reshape(B, H, -1, d)
    x = torch.matmul(q * d ** -0.5, k.permute(0, 2, 3, 1)).view(B, H, Hq // H, wide, T)
    del k
    if s["beta"] is not None:
        x += s["beta"][table].permute(0, 2, 1, 3).reshape(B, H, 1, 1, T)
    hidden = torch.arange(T, device=DEVICE) >= seen[:, :, None]  # [B, wide, slots]
    x.masked_fill_(hidden[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    if s["out"] is not None:
        o = torch.matmul(x.view(B, H, -1, T), _read(s, "V").transpose(1, 2))
        o = o.view(B, H, Hq // H, wide, d)
        o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, wide, Hq, d)
        s["out"].copy_(o[seq, col])
    if "weight" in s:
        x = x.div_(torch.where(total > 0, total, 1.0)).sum((2, 3))  # [B, H, slots]
        lens = s["lens"].long()[:, None]
        new = torch.tensor(s["new"], device=DEVICE)[:, None]
        at = torch.arange(T, device=DEVICE).expand(B, T)
        before = s["weight"][table].transpose(1, 2).reshape(B, H, T)
        if c["decay"] == 0:
            before = torch.zeros_like(before)
        x += torch.where((at < lens - new)[:, None], c["decay"] * before, 0.0)
        b, j = (at < lens).nonzero(as_tuple=True)
        s["weight"][table[b, j // page], :, j % page] = x[b, :, j]


def _plain_evict(s):
    c = s["case"]
    B, H, page, keep = c["B"], c["H"], c["page"], c["keep"]
    table, lens = s["table"].long(), s["lens"].long()
    T = table.shape[1] * page
    at = torch.arange(T, device=DEVICE)
    w = s["weight"][table].transpose(1, 2).reshape(B, H, T)
    end = lens[:, None, None]
    w = torch.where((at < c["sinks"]) | (at >= end - c["recent"]), math.inf, w)
    w = torch.where(at < end, w, -math.inf)
    order = torch.sort(w, dim=2, descending=True, stable=True).indices
    kept = min(T, keep)
    count = lens.clamp_max(keep)
    rank = torch.arange(kept, device=DEVICE)
    real = rank < count[:, None]  # [B, kept]
    idx = torch.where(real[:, None], order[..., :kept], T).sort(2).values
    s["kept"].fill_(-1)
    s["kept"][..., :kept] = torch.where(real[:, None], idx, -1)
    s["to_lens"].copy_(count)
    s["to_offset"].copy_(s["offset"] + lens - count)
    b, r = real.nonzero(as_tuple=True)
    j = idx[b, :, r]  # [rows, H]
    h = torch.arange(H, device=DEVICE)
    src, dst = table[b[:, None], j // page], s["to_table"].long()[b, r // page][:, None]
    r, j = (r % page)[:, None], j % page
    s["to_K"][dst, r, h] = s["K"][src, j, h]
    s["to_V"][dst, r, h] = s["V"][src, j, h]
    s["to_weight"][dst, h, r] = s["weight"][src, h, j]
    if s["beta"] is not None:
        s["to_beta"][dst, h, r] = s["beta"][src, h, j]


# ------------------------------------------------------------------------------ in 64 bits

def _exact_rotation(x, pos, theta):
    half = x.shape[-1] // 2
    w = torch.tensor([theta ** (-2.0 * m / (2 * half)) for m in range(half)],
                     dtype=torch.float64, device=DEVICE)
    turn = torch.polar(torch.ones_like(w), pos.double().unsqueeze(-1) * w)[:, None]
    z = torch.complex(x[..., :half].double(), x[..., half:].double()) * turn
    return torch.cat([z.real, z.imag], -1)


def _exact_put(got, name, rows, slots, pages, page):
    """Rows [n, H, d] of consecutive slots into got[name], codes not rounded."""
    scales = got[name.lower() + "_scale"]
    held = rows.to(torch.bfloat16).double().abs().amax(2)  # [n, H], as rounded
    at = 0
    while at < len(slots):
        j = int(slots[at])
        n = min(len(slots) - at, BLOCK - j % BLOCK)
        p, i = int(pages[at]), j % page
        top = held[at:at + n].amax(0)
        need = torch.exp2(torch.ceil(torch.log2(top / 448)).clamp_min(-126))
        block = slice(i // BLOCK * BLOCK, i)
        if j % BLOCK:
            old = scales[p, :, i // BLOCK].clone()
            need = torch.maximum(need, old)
            got[name][p, block] *= (old / need)[:, None]
        scales[p, :, i // BLOCK] = need
        got[name][p, i:i + n] = rows[at:at + n] / need[:, None]
        at += n


def exact(case, seed):
    s = prepare(case, seed)
    H, d, page, op = case["H"], case["d"], case["page"], case["op"]
    new, lens = _counts(case)
    if op == "evict":
        return _exact_evict(s, case, lens)
    group = case["Hq"] // H
    if op == "append8":
        got = {key: x.double() for key, x in _outputs(s).items()}
        at = 0
        for b in range(case["B"]):
            rows = slice(at, at + new[b])
            at += new[b]
            slots = torch.arange(lens[b] - new[b], lens[b], device=DEVICE)
            pages = s["table"][b].long()[slots // page]
            k = s["k"][rows].double()
            if case["theta"]:
                k = _exact_rotation(s["k"][rows], slots + case["offset"], case["theta"])
                if s["q"] is not None:
                    got["out"][rows] = _exact_rotation(s["q"][rows], slots + case["offset"],
                                                       case["theta"])
            _exact_put(got, "K", k, slots.tolist(), pages.tolist(), page)
            _exact_put(got, "V", s["v"][rows].double(), slots.tolist(), pages.tolist(), page)
            if s["beta"] is not None:
                x = s["new_beta"]
                got["beta"][pages, :, slots % page] = x[rows].double() if x is not None else 0.0
        return got
    got = {}
    if s["out"] is not None:
        got["out"] = torch.zeros(s["n"], case["Hq"], d, dtype=torch.float64, device=DEVICE)
    if "weight" in s:
        got["weight"] = s["weight"].double()
    at = 0
    for b in range(case["B"]):
        rows = slice(at, at + new[b])
        at += new[b]
        if lens[b] == 0:
            continue
        pages = s["table"][b, :-(-lens[b] // page)].long()
        reach = torch.arange(lens[b] - new[b], lens[b], device=DEVICE)[:, None]
        late = torch.arange(lens[b], device=DEVICE)[None] > reach
        for h in range(H):
            k, v = (_exact_rows(s, x, pages, h)[:lens[b]] for x in "KV")
            bias = s["beta"][pages, h].reshape(-1)[:lens[b]].double() if case["beta"] else 0.0
            total = torch.zeros(lens[b], dtype=torch.float64, device=DEVICE)
            for i in range(h * group, (h + 1) * group):
                logit = s["q"][rows, i].double() @ k.T / math.sqrt(d) + bias
                weight = torch.softmax(logit.masked_fill_(late, -math.inf), -1)
                if "out" in got:
                    got["out"][rows, i] = weight @ v
                total += weight.sum(0)
            if "weight" in got:
                old = got["weight"][pages, h].reshape(-1)
                old[:lens[b] - new[b]] *= case["decay"]
                old[lens[b] - new[b]:lens[b]] = 0
                old[:lens[b]] += total
                got["weight"][pages, h] = old.view(-1, page)
    return got


def _exact_rows(s, name, pages, h):
    pool = s[name]
    if pool.dtype != E4M3:
        return pool[pages, :, h].reshape(-1, pool.shape[3]).double()
    x = pool.view(torch.uint8)[pages, :, h].view(E4M3).double()
    scale = s[name.lower() + "_scale"][pages, h].double()
    return (x.unflatten(1, (-1, BLOCK)) * scale[..., None, None]).reshape(-1, pool.shape[3])


def _exact_evict(s, case, lens):
    """Nothing is computed: numbers are chosen and moved."""
    H, page, keep = case["H"], case["page"], case["keep"]
    got = {key: x.double() if x.is_floating_point() else x.clone()
           for key, x in _outputs(s).items()}
    got["kept"].fill_(-1)
    for b, n in enumerate(lens):
        pages = s["table"][b].long()
        count = min(n, keep)
        got["to_lens"][b] = count
        got["to_offset"][b] = case["offset"] + n - count
        r = torch.arange(count, device=DEVICE)
        to = s["to_table"][b].long()[r // page]
        for h in range(H):
            w = s["weight"][pages, h].reshape(-1)[:n].tolist()
            free = sorted(range(case["sinks"], n - case["recent"]), key=lambda j: (-w[j], j))
            fixed = list(range(min(n, case["sinks"])))
            fixed += range(max(len(fixed), n - case["recent"]), n)
            idx = list(range(n)) if n <= keep else sorted(fixed + free[:keep - len(fixed)])
            got["kept"][b, h, :count] = torch.tensor(idx, device=DEVICE)
            j = got["kept"][b, h, :count].long()
            src = pages[j // page], j % page
            got["to_K"][to, r % page, h] = s["K"][src[0], src[1], h].double()
            got["to_V"][to, r % page, h] = s["V"][src[0], src[1], h].double()
            got["to_weight"][to, h, r % page] = s["weight"][src[0], h, src[1]].double()
            if s["beta"] is not None:
                got["to_beta"][to, h, r % page] = s["beta"][src[0], h, src[1]].double()
    return got


# ------------------------------------------------------------------------------ work

def work(case):
    """Every input once and every output once; products of visible slots only."""
    H, Hq, d, B, op = case["H"], case.get("Hq", 0), case["d"], case["B"], case["op"]
    new, lens = _counts(case)
    n = sum(new)
    plan = 4 * (sum(max(1, -(-x // case["page"])) for x in lens) + 2 * B) + 8 * B
    if op == "append8":
        # q both ways, k and v in 16 bits and out in 8, and a scale for every block
        beta = 4 * n * H * (1 + (not case["theta"])) if case["beta"] else 0
        moved = n * d * (4 * Hq + 6 * H) + 8 * H * (n // BLOCK + B)
        return {"bytes": moved + beta + plan, "flops": 3 * n * (Hq + H) * d if case["theta"] else 0}
    if op == "evict":
        kept = sum(min(x, case["keep"]) for x in lens)
        row = 8 * d + 8 + (8 if case["beta"] else 0) + 4
        return {"bytes": (4 * sum(lens) + kept * row) * H + plan, "flops": 0}
    beta = 4 if case["beta"] else 0
    pairs = sum((x - k + 1 + x) * k / 2.0 for k, x in zip(new, lens) if x >= k)
    if op.endswith("8"):
        cache = sum(lens) * H * (2 * d + 8 / BLOCK + beta)
        return {"bytes": cache + 4 * n * Hq * d + plan, "flops": 4.0 * pairs * Hq * d}
    out = op == "decode_weigh"
    weight = 4 if case["decay"] == 0 else 8
    cache = sum(lens) * H * ((4 if out else 2) * d + beta + weight)
    rows = (4 if out else 2) * n * Hq * d
    return {"bytes": cache + rows + plan, "flops": (4.0 if out else 2.0) * pairs * Hq * d}
