"""A paged key-value cache and the attention that reads it, as cases that can be timed and compared.

Three calls of a served model whose caches may have been compacted: `append` puts the keys and
values of new tokens (or the slots of a compact cache) into the pages of their sequences and
rotates keys and queries to their positions, `decode` attends from one new token of every sequence,
`prefill` from several. A cache is a pool of pages [n_pages, page, H, d] (bf16; in memory slots
before heads or heads before slots), with an optional logit bias per slot [n_pages, H, page]
(fp32) and a table of pages per sequence. `lens` counts a sequence's slots with this call's tokens,
which are its last ones; the token in slot j has position j + offset, and the offset is what a
compaction took out (tokens less slots).

With `own` false the calls are written in elementary torch operations in fp32; `exact` restates
them in 64 bits, one sequence and KV-head at a time.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
_MOST_SLOTS = 250_000  # of a drawn case's cache, with 8 KV-heads of 128 channels
_MOST_SCORES = 0.9e9   # of a drawn prefill with 128 channels: padded queries x heads x padded slots


def listed():
    return [
        # a decode step's append for one sequence of a small model: latency
        dict(name="append_step_1x_h2", op="append", B=1, past="777", new="1", H=2, Hq=8, d=64,
             page=16, beta=False, heads_first=False, theta=1e4, offset=0),
        # a chunk of a long prompt on its way into the cache
        dict(name="append_chunk_8k", op="append", B=1, past="8192", new="8192", H=8, Hq=32, d=128,
             page=64, beta=False, heads_first=False, theta=1e6, offset=0),
        # the compact caches of eight documents into their pages, with their biases, not rotated
        dict(name="install_8x1311", op="append", B=8, past="0", new="1311", H=8, Hq=0, d=128,
             page=32, beta=True, heads_first=False, theta=0.0, offset=0),
        # one short sequence of a small model
        dict(name="decode_1x778_h2", op="decode", B=1, past="777", new="1", H=2, Hq=8, d=64,
             page=16, beta=False, heads_first=False, offset=0),
        # eight compacted documents (t = 1311, biases) and what was said since
        dict(name="decode_8x_compacted", op="decode", B=8, past="1311:5407", new="1", H=8, Hq=32,
             d=128, page=32, beta=True, heads_first=False, offset=64225),
        # a full batch of small compact caches, two of its places idle
        dict(name="decode_256x_short", op="decode", B=256, past="164:700", new="1", H=8, Hq=32,
             d=128, page=16, beta=True, heads_first=False, offset=8028, idle=2),
        # uncompacted documents of ragged length, seven query heads to a KV-head
        dict(name="decode_24x_8k_32k", op="decode", B=24, past="8192:32768", new="1", H=4, Hq=28,
             d=128, page=64, beta=False, heads_first=True, offset=0),
        # one very long document, 256 channels
        dict(name="decode_1x131072_d256", op="decode", B=1, past="131071", new="1", H=8, Hq=16,
             d=256, page=128, beta=False, heads_first=False, offset=0),
        # a question of odd length after each of four compacted documents
        dict(name="prefill_question_4x", op="prefill", B=4, past="655:1311", new="17:101", H=8,
             Hq=32, d=128, page=32, beta=True, heads_first=False, offset=64225),
        # a pass of the lookahead schedule: a chunk against five compact chunks and one raw chunk
        dict(name="prefill_lookahead_4k", op="prefill", B=1, past="4736", new="4096", H=8, Hq=32,
             d=128, page=128, beta=True, heads_first=False, offset=19840),
        # a whole prompt, seven query heads to a KV-head
        dict(name="prefill_prompt_8k_g7", op="prefill", B=1, past="0", new="8192", H=4, Hq=28,
             d=128, page=64, beta=False, heads_first=True, offset=0),
        # ragged prompts on ragged pasts, 256 channels
        dict(name="prefill_3x_ragged_d256", op="prefill", B=3, past="0:2500", new="900:2300", H=8,
             Hq=16, d=256, page=16, beta=False, heads_first=False, offset=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "prefill", "prefill"])
    d = rng.choice([64, 128, 128, 256])
    H = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 3, 4, 5, 7, 8, 16])
    c = dict(op=op, H=H, Hq=H * g, d=d, page=rng.choice([16, 32, 64, 128, 256]),
             beta=rng.random() < 0.5, heads_first=rng.random() < 0.4,
             offset=rng.choice([0, 0, rng.randint(1, 1 << 20)]))
    if op == "append":
        c["theta"] = rng.choice([1e4, 1e6])
        if rng.random() < 0.3:  # compact slots
            c |= dict(theta=0.0, Hq=0)
        total = _log(rng, 1, 8192 * 1024 // (H * d * min(g, 4)))
        c["B"] = min(total, rng.choice([1, 1, 3, 8, 32]))
        new = max(1, total // c["B"])
        c |= dict(new="%d:%d" % (max(1, new // 2), new), past="0:%d" % rng.choice([0, 100, 4000]))
        return c
    if op == "decode":
        slots = _log(rng, 1, _MOST_SLOTS * 1024 // (H * d))
        c["B"] = min(slots, rng.choice([1, 1, 2, 8, 32, 128]))
        most = min(max(1, slots // c["B"]), 262144)
        c |= dict(past="%d:%d" % (max(1, most // rng.choice([1, 3])), most), new="1",
                  idle=rng.choice([0, 0, 1]) if c["B"] > 1 else 0)
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

def _pool(gen, case, n_pages):
    H, d, page = case["H"], case["d"], case["page"]
    shape = (n_pages, H, page, d) if case["heads_first"] else (n_pages, page, H, d)
    x = torch.empty(shape, device=DEVICE, dtype=torch.bfloat16).normal_(generator=gen)
    return x.transpose(1, 2) if case["heads_first"] else x


def prepare(case, seed):
    """A program's cache (pages in the order that an allocator left them, what is in no sequence
    stale), table and lengths, and the rows of the fused q, k, v projection of its new tokens."""
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    H, Hq, d, page, B = case["H"], case["Hq"], case["d"], case["page"], case["B"]
    new, lens = _counts(case)
    need = [max(1, -(-x // page)) for x in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device=DEVICE).to(torch.int32)
    table = torch.zeros(B, max(need), dtype=torch.int32, device=DEVICE)
    taken = 0
    for b, k in enumerate(need):
        table[b, :k] = order[taken:taken + k]
        taken += k
    s = dict(case=case, n=sum(new), new=new, table=table,
             lens=torch.tensor(lens, dtype=torch.int32, device=DEVICE),
             offset=torch.full((B,), case["offset"], dtype=torch.int64, device=DEVICE))
    s["K"], s["V"] = _pool(gen, case, n_pages), _pool(gen, case, n_pages)
    # one outlier key channel per head, as in real caches
    heavy = torch.randint(0, d, (H, 1), generator=gen, device=DEVICE)
    s["K"] *= 1 + 7 * torch.zeros(H, d, device=DEVICE, dtype=torch.bfloat16).scatter_(1, heavy, 1)
    s["beta"] = None
    if case["beta"]:
        s["beta"] = torch.empty(n_pages, H, page, device=DEVICE).normal_(generator=gen)
    # cumulative new tokens: absent where every sequence has one
    s["cu_new"] = None
    if case["op"] != "decode" and any(x != 1 for x in new):
        s["cu_new"] = torch.tensor([0] + new, device=DEVICE).cumsum(0).to(torch.int32)
    rows = torch.empty(s["n"], (Hq + 2 * H) * d, device=DEVICE,
                       dtype=torch.bfloat16).normal_(generator=gen)
    q, k, v = rows.split([Hq * d, H * d, H * d], 1)
    s["q"] = q.unflatten(1, (Hq, d)) if Hq else None
    s["out"] = torch.empty(s["n"], Hq, d, device=DEVICE, dtype=torch.bfloat16) if Hq else None
    if case["op"] == "append":
        s["k"], s["v"] = k.unflatten(1, (H, d)), v.unflatten(1, (H, d))
        s["new_beta"] = None
        if case["beta"] and not case["theta"]:  # compact slots come with their biases
            s["new_beta"] = torch.empty(s["n"], H, device=DEVICE).normal_(generator=gen)
    return s


# ------------------------------------------------------------------------------ passes

_context = None


def _own(s):
    """The calls of the framework, with the handles that a program makes once."""
    global _context
    from paper_2606_07878_gb300 import still
    if _context is None:
        _context = still.still_create(0)
    if "cache" not in s:
        s["cache"] = still.PagedCache(s["K"], s["V"], s["beta"])
        s["batch"] = still.PagedBatch(s["table"], s["lens"], s["cu_new"], s["offset"])
    c = s["case"]
    if c["op"] == "append":
        still.still_paged_append(_context, s["cache"], s["batch"], s["k"], s["v"], q=s["q"],
                                 q_out=s["out"], beta=s["new_beta"], rope_theta=c["theta"])
        return _appended(s)
    call = still.still_paged_decode if c["op"] == "decode" else still.still_paged_prefill
    call(_context, s["cache"], s["batch"], s["q"], s["out"])
    return s["out"]


def _appended(s):
    got = dict(K=s["K"], V=s["V"])
    if s["out"] is not None:
        got["q"] = s["out"]
    if s["beta"] is not None:
        got["beta"] = s["beta"]
    return got


def run(s):
    if own:
        return _own(s)
    return _plain_append(s) if s["case"]["op"] == "append" else _plain_attention(s)


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


def _plain_append(s):
    c = s["case"]
    seq, slot = _places(s)
    k, theta = s["k"], c["theta"]
    if theta:
        pos = slot + s["offset"][seq]
        k = _rotated(k, pos, theta).bfloat16()
        if s["q"] is not None:
            s["out"].copy_(_rotated(s["q"], pos, theta))
    page, at = s["table"].long()[seq, slot // c["page"]], slot % c["page"]
    s["K"][page, at] = k
    s["V"][page, at] = s["v"]
    if s["beta"] is not None:
        s["beta"][page, :, at] = s["new_beta"] if s["new_beta"] is not None else 0.0
    return _appended(s)


def _plain_attention(s):
    c = s["case"]
    B, H, Hq, d = c["B"], c["H"], c["Hq"], c["d"]
    seq, slot = _places(s)
    wide = max(s["new"])
    first = s["cu_new"].long()[seq] if s["cu_new"] is not None else seq
    col = torch.arange(s["n"], device=DEVICE) - first
    q = torch.zeros(B, wide, Hq, d, device=DEVICE)
    q[seq, col] = s["q"].float()
    seen = torch.zeros(B, wide, dtype=torch.long, device=DEVICE)
    seen[seq, col] = slot + 1
    table = s["table"].long()
    k = s["K"][table].flatten(1, 2).float()  # [B, slots, H, d]
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
    v = s["V"][table].flatten(1, 2).float()
    o = torch.matmul(x.view(B, H, -1, T), v.transpose(1, 2)).view(B, H, Hq // H, wide, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, wide, Hq, d)
    s["out"].copy_(o[seq, col])
    return s["out"]


# ------------------------------------------------------------------------------ in 64 bits

def _exact_rotation(x, pos, theta):
    half = x.shape[-1] // 2
    w = torch.tensor([theta ** (-2.0 * m / (2 * half)) for m in range(half)],
                     dtype=torch.float64, device=DEVICE)
    turn = torch.polar(torch.ones_like(w), pos.double().unsqueeze(-1) * w)[:, None]
    z = torch.complex(x[..., :half].double(), x[..., half:].double()) * turn
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    s = prepare(case, seed)
    H, d, page = case["H"], case["d"], case["page"]
    new, lens = _counts(case)
    group = case["Hq"] // H
    if case["op"] == "append":
        got = {key: x.double() for key, x in _appended(s).items()}
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
                    got["q"][rows] = _exact_rotation(s["q"][rows], slots + case["offset"],
                                                     case["theta"])
            got["K"][pages, slots % page] = k
            got["V"][pages, slots % page] = s["v"][rows].double()
            if s["beta"] is not None:
                x = s["new_beta"]
                got["beta"][pages, :, slots % page] = x[rows].double() if x is not None else 0.0
        return got
    out = torch.zeros(s["n"], case["Hq"], d, dtype=torch.float64, device=DEVICE)
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
            k = s["K"][pages, :, h].reshape(-1, d)[:lens[b]].double()
            v = s["V"][pages, :, h].reshape(-1, d)[:lens[b]].double()
            bias = s["beta"][pages, h].reshape(-1)[:lens[b]].double() if case["beta"] else 0.0
            for i in range(h * group, (h + 1) * group):
                logit = s["q"][rows, i].double() @ k.T / math.sqrt(d) + bias
                weight = torch.softmax(logit.masked_fill_(late, -math.inf), -1)
                out[rows, i] = weight @ v
    return out


# ------------------------------------------------------------------------------ work

def work(case):
    """Every input once and every output once; products of visible slots only."""
    H, Hq, d, B = case["H"], case["Hq"], case["d"], case["B"]
    new, lens = _counts(case)
    n = sum(new)
    plan = 4 * (sum(max(1, -(-x // case["page"])) for x in lens) + 2 * B) + 8 * B
    if case["op"] == "append":
        rows = n * (Hq + 2 * H) * d * 2
        beta = 4 * n * H * (1 + (not case["theta"])) if case["beta"] else 0
        return {"bytes": 2 * rows + beta + plan, "flops": 3 * n * (Hq + H) * d if case["theta"] else 0}
    cache = sum(lens) * H * (4 * d + (4 if case["beta"] else 0))
    pairs = sum((x - k + 1 + x) * k / 2.0 for k, x in zip(new, lens) if x >= k)
    return {"bytes": cache + 4 * n * Hq * d + plan, "flops": 4.0 * pairs * Hq * d}
