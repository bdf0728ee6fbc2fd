"""A document served from a paged cache that is compacted as it grows (Sec. 2.3, "Iterative chunked
compaction"; App. B): one layer's part of it, with synthetic rows in place of a base model's.

    python -m paper_2606_07878_gb300.paged_serving

The document comes in chunks of c * t tokens. A pass appends a chunk to the cache (keys rotated to
their positions), attends from its tokens to [compact chunks | raw chunk | the chunk itself],
compacts the oldest raw chunk to t slots and puts those into pages of their own. The raw chunk's
pages then leave the sequence's table and the compact ones take their place: nothing else moves, and
positions run ahead of slots by what the compactions took out. A question of some tokens and an
answer, token by token, follow.
"""
from __future__ import annotations

import torch

from paper_2606_07878_gb300 import still, synth


class Document:
    """The pages of one sequence in a pool that keeps slots before heads, so that a chunk's
    consecutive pages are also the [tokens, H, d] rows that the compactor reads."""

    def __init__(self, H, d, n_pages, page, device):
        self.H, self.d, self.page = H, d, page
        self.K = torch.zeros(n_pages, page, H, d, dtype=torch.bfloat16, device=device)
        self.V = torch.zeros_like(self.K)
        self.cache = still.PagedCache(self.K, self.V)
        i32 = dict(dtype=torch.int32, device=device)
        self.table = torch.zeros(1, n_pages, **i32)
        self.lens, self.cu_new = torch.zeros(1, **i32), torch.zeros(2, **i32)
        self.offset = torch.zeros(1, dtype=torch.int64, device=device)
        self.many = still.PagedBatch(self.table, self.lens, self.cu_new, self.offset)
        self.one = still.PagedBatch(self.table, self.lens, None, self.offset)
        self.compact, self.raw = [], []  # page numbers; of every raw chunk
        self.used = 0     # pages taken so far (none are reused here)
        self.slots = 0    # in use

    def take(self, tokens):
        """Consecutive pages for so many tokens."""
        n = -(-tokens // self.page)
        self.used += n
        return list(range(self.used - n, self.used))

    def link(self):
        pages = self.compact + [p for chunk in self.raw for p in chunk]
        self.table[0, :len(pages)] = torch.tensor(pages, dtype=torch.int32)

    def rows(self, pool, pages):
        return pool[pages[0]:pages[-1] + 1].view(-1, self.H, self.d)

    def extend(self, ctx, rows, start, theta, group):
        """Appends the tokens of `rows` (a fused projection, first position `start`) and attends
        from them; their pages are linked already. Returns [n, Hq, d]."""
        n, d, H = rows.shape[0], self.d, self.H
        q, k, v = rows.split([group * H * d, H * d, H * d], 1)
        q, k, v = q.unflatten(1, (-1, d)), k.unflatten(1, (H, d)), v.unflatten(1, (H, d))
        self.offset.fill_(start - self.slots)
        self.slots += n
        self.lens.fill_(self.slots)
        self.cu_new[1] = n
        out = torch.empty(n, group * H, d, dtype=torch.bfloat16, device=rows.device)
        batch = self.one if n == 1 else self.many
        rotated = torch.empty_like(out)
        still.still_paged_append(ctx, self.cache, batch, k, v, q=q, q_out=rotated,
                                 rope_theta=theta)
        attend = still.still_paged_decode if n == 1 else still.still_paged_prefill
        attend(ctx, self.cache, batch, rotated, out)
        return out

    def compact_oldest(self, ctx, k, c, t):
        """Chunk k, the oldest raw one, becomes t compact slots."""
        chunk = self.raw.pop(0)
        Ck = torch.empty(t, self.H, self.d, dtype=torch.bfloat16, device=self.K.device)
        Cv = torch.empty_like(Ck)
        still.still_lookahead_compact_layer(ctx, 0, self.rows(self.K, chunk),
                                            self.rows(self.V, chunk), [k], c, t, Ck, Cv)
        pages = self.take(t)
        i32 = dict(dtype=torch.int32, device=self.K.device)
        slots = still.PagedBatch(torch.tensor([pages], **i32), torch.tensor([t], **i32),
                                 torch.tensor([0, t], **i32))
        still.still_paged_append(ctx, self.cache, slots, Ck, Cv)  # at their positions already
        self.compact += pages
        self.slots -= c * t - t
        self.link()


def serve(wl, chunks=4, c=8, t=128, page=32, group=4, question=37, answer=8, seed=0,
          device="cuda:0"):
    """Serves `chunks` chunks of c * t tokens, a question and an answer. t and c * t are multiples
    of the page. Returns the document and the outputs of the question and of the answer."""
    H, d, theta = wl["H"], wl["d"], wl["theta"]
    assert t % page == 0 and chunks >= 2
    gen = torch.Generator(device=device).manual_seed(seed)

    def rows(n):  # of the base model's fused projection
        return torch.randn(n, (group + 2) * H * d, generator=gen, device=device).bfloat16()

    ctx = still.still_create(torch.device(device).index or 0)
    try:
        still.still_load_layer_weights(ctx, 0, still.config_from_workload(wl, t),
                                       synth.gen_weights(wl, 0, t, device))
        need = chunks * (c * t + t) + question + answer
        doc = Document(H, d, -(-need // page) + chunks + 1, page, device)
        for k in range(chunks - 1):
            p = still.still_lookahead_pass_info(k, c, t)
            for _ in range(p["prefill_len"] // (c * t)):
                doc.raw.append(doc.take(c * t))
            doc.link()
            assert doc.slots == p["prefill_past"]
            doc.extend(ctx, rows(p["prefill_len"]), p["prefill_start"], theta, group)
            doc.compact_oldest(ctx, k, c, t)
            assert doc.slots == p["retained_after"]
        position = chunks * c * t
        doc.raw.append(doc.take(question + answer))
        doc.link()
        asked = doc.extend(ctx, rows(question), position, theta, group)
        answered = [doc.extend(ctx, rows(1), position + question + i, theta, group)
                    for i in range(answer)]
        code, detail = still.still_get_device_status(ctx)
        if code != 0:
            raise RuntimeError(f"device status {still.STATUS.get(code)} {detail}")
        return doc, asked, answered
    finally:
        still.still_destroy(ctx)


def main():
    wl = synth.WORKLOADS["qwen3_4b_64k"]
    chunks, c, t = 5, 16, 256
    doc, asked, answered = serve(wl, chunks, c, t)
    tokens = chunks * c * t + asked.shape[0] + len(answered)
    print(f"{tokens} tokens in {doc.slots} slots of {doc.page} a page; "
          f"{still.still_kv_bytes(1, wl['H'], wl['d'], 2, doc.slots) / 2 ** 20:.1f} MiB a layer "
          f"instead of {still.still_kv_bytes(1, wl['H'], wl['d'], 2, tokens) / 2 ** 20:.1f}")


if __name__ == "__main__":
    main()
