"""A document served from a paged cache that is compacted as it grows: the slots that it ends with,
and the attention over them, against 64 bits."""
import math

import pytest
import torch

from paper_2606_07878_gb300 import paged_serving, still, synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("family,t,c,page", [("tiny_1k", 32, 4, 16), ("qwen3_4b_64k", 64, 8, 64)])
def test_served_document_matches_64_bits(family, t, c, page):
    wl = synth.WORKLOADS[family]
    chunks, group, question, answer = 4, 3, 21, 3
    H, d, theta = wl["H"], wl["d"], wl["theta"]
    doc, asked, answered = paged_serving.serve(wl, chunks, c, t, page, group, question, answer)
    passes, retained = still.still_lookahead_totals((chunks - 1) * c * t, c, t)
    assert passes == chunks - 1 and doc.slots == retained + question + answer

    # the rows again, in the order in which they were drawn
    gen = torch.Generator(device="cuda:0").manual_seed(0)
    counts = [2 * c * t] + [c * t] * (chunks - 2) + [question] + [1] * answer
    rows = torch.cat([torch.randn(n, (group + 2) * H * d, generator=gen, device="cuda:0").bfloat16()
                      for n in counts])
    pos = torch.arange(rows.shape[0], device="cuda:0").double()
    half = d // 2
    w = theta ** (-torch.arange(half, device="cuda:0", dtype=torch.float64) / half)
    turn = torch.polar(torch.ones_like(w), pos[:, None] * w)[:, None]

    def rotated(x):
        x = x.double()
        z = torch.complex(x[..., :half], x[..., half:]) * turn
        return torch.cat([z.real, z.imag], -1).bfloat16()

    q, k, v = rows.split([group * H * d, H * d, H * d], 1)
    q = rotated(q.unflatten(1, (-1, d)))
    k, v = rotated(k.unflatten(1, (H, d))), v.unflatten(1, (H, d))

    # the compact chunks by the layer call, then what is raw
    ctx = still.still_create(0)
    try:
        still.still_load_layer_weights(ctx, 0, still.config_from_workload(wl, t),
                                       synth.gen_weights(wl, 0, t, "cuda:0"))
        K, V = [], []
        n = c * t
        raw = doc.K[doc.table[0, :-(-doc.slots // page)].long()].flatten(0, 1)[:doc.slots]
        rawv = doc.V[doc.table[0, :-(-doc.slots // page)].long()].flatten(0, 1)[:doc.slots]
        for i in range(chunks - 1):
            Ck = torch.empty(t, H, d, dtype=torch.bfloat16, device="cuda:0")
            Cv = torch.empty_like(Ck)
            still.still_compact_layer(ctx, 0, k[i * n:(i + 1) * n].contiguous(),
                                      v[i * n:(i + 1) * n].contiguous(), t, Ck, Cv,
                                      segments=[(i * n, 1, n)])
            K.append(Ck)
            V.append(Cv)
            # keys that differ by the rounding of a rotation give other compact slots
            for got, ref in ((raw[i * t:(i + 1) * t], Ck), (rawv[i * t:(i + 1) * t], Cv)):
                err = (got.double() - ref.double()).norm() / ref.double().norm()
                assert err <= 2e-2, float(err)
    finally:
        still.still_destroy(ctx)
    kept = (chunks - 1) * n
    assert torch.equal(rawv[(chunks - 1) * t:], v[kept:])
    # an angle within 2^-22 rad and bf16 rounding: at most an ulp, 2^-7 of the value, apart
    err = (raw[(chunks - 1) * t:].double() - k[kept:].double()).abs()
    assert (err <= 2.0 ** -7 * k[kept:].double().abs() + 2.0 ** -18).all()

    # question and answer over the slots that there are
    out = torch.cat([asked] + answered)
    K, V = raw.double(), rawv.double()
    first = doc.slots - out.shape[0]
    for i in range(out.shape[0]):
        see = first + i + 1
        for h in range(H):
            qi = q[kept + n + i, h * group:(h + 1) * group].double()
            p = torch.softmax(qi @ K[:see, h].T / math.sqrt(d), -1)
            ref, size = p @ V[:see, h], p @ V[:see, h].abs()
            err = (out[i, h * group:(h + 1) * group].double() - ref).abs()
            # as for the attention alone, and queries that may be an ulp apart: a logit of |q| |k|
            # / sqrt(d), below 2^5 here, moves by 2^-7 of it at the very most, and few channels are
            assert (err <= 2.0 ** -8 * ref.abs() + 2.0 ** -5 * size).all()
