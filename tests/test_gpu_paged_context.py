"""A context whose paged calls were captured, and what it is used for afterwards."""
import pytest
import torch

from paper_2606_07878_gb300 import still, synth
from test_gpu_paged import DEV, NAN, WEIGHTS, Pages, assert_rows, attention64, batch_of, fused_rows

pytestmark = pytest.mark.gpu


@pytest.fixture
def ctx():
    c = still.still_create(0)
    yield c
    code, det = still.still_get_device_status(c)
    still.still_destroy(c)
    assert code == 0, (still.STATUS[code], det)


def captured(call, out):
    """A graph of one call (on a side stream); replays it into `out` filled with NaN."""
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        call(stream)

    def replay():
        out.fill_(NAN)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
    return replay


def test_captured_calls_outlive_larger_ones(ctx):
    """A decode step captured after calls of its own size alone, a prefill captured as the first one
    of its kernel: both replay into a workspace that stays where it is through attention of other
    head sizes, biased decode attention and compactions of growing sizes. Memory that these free is
    taken and overwritten before the replay."""
    p = Pages(50, [3000, 900], 2, 64, 16)
    q, = fused_rows(51, 2, [4], 64)
    out = torch.empty_like(q)
    batch, cache = batch_of(p), p.cache()
    decode = lambda s=None: still.still_paged_decode(ctx, cache, batch, q, out, stream=s)
    decode()
    replay = captured(decode, out)
    r = Pages(52, [2500], 2, 128, 64, beta=True)
    new = [70]
    rq, = fused_rows(53, 70, [8], 128)
    rout = torch.empty_like(rq)
    rbatch, rcache = batch_of(r, new), r.cache()
    replay_r = captured(lambda s: still.still_paged_prefill(ctx, rcache, rbatch, rq, rout, stream=s),
                        rout)

    wl = synth.WORKLOADS["tiny_1k"]
    t = wl["ts"][0]
    still.still_load_layer_weights(ctx, 0, still.config_from_workload(wl, t),
                                   synth.gen_weights(wl, 0, t, DEV))
    taken = []
    for size in (256, 512, 1024):
        K, V = synth.gen_kv(wl, 0, N=size, device=DEV)
        Ck = torch.empty(t, wl["H"], wl["d"], dtype=torch.bfloat16, device=DEV)
        still.still_compact_layer(ctx, 0, K, V, t, Ck, torch.empty_like(Ck))
        big = Pages(54, [size], 1, 256, 16)
        bq, = fused_rows(55, 130, [3], 256)
        still.still_paged_prefill(ctx, big.cache(), batch_of(big, [130]), bq, torch.empty_like(bq))
        k = torch.randn(40 * size, 1, 256, device=DEV).bfloat16()
        still.still_attend_biased(ctx, bq[:4].contiguous(), k[:0], k[:0], None, k, k,
                                  torch.empty_like(bq[:4]))
        torch.cuda.synchronize()
        taken.append(torch.full((1 << 26,), NAN, device=DEV))
    replay()
    assert_rows(out, *attention64(p, q, [1, 1]), WEIGHTS)
    replay_r()
    assert_rows(rout, *attention64(r, rq, new), WEIGHTS)
    # and the other way round: what the calls in between gave is what they give now
    first = out.clone()
    decode()
    assert torch.equal(out, first)


def test_workspace_is_allocated_once(ctx):
    """The first call of either kind takes device memory, no later one of any size does."""
    calls = []
    for d, n in ((64, 1), (64, 9), (128, 1), (128, 12), (128, 300), (256, 1), (256, 40), (256, 300)):
        p = Pages(56, [n + 100], 1, d, 16)
        q, = fused_rows(57, n, [1], d)
        calls.append((p.cache(), batch_of(p, [n]), q, torch.empty_like(q)))
    other = still.still_create(0)  # the driver loads a kernel's code at its first launch
    try:
        for call in calls:
            still.still_paged_prefill(other, *call)
    finally:
        still.still_destroy(other)
    still.still_paged_prefill(ctx, *calls[0])
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for call in calls:
        still.still_paged_prefill(ctx, *call)
        torch.cuda.synchronize()
        assert torch.cuda.mem_get_info()[0] == free


@pytest.mark.parametrize("new,n", [([7, 3], 11), ([30, 10], 90), ([0, 0], 3)])
@pytest.mark.parametrize("first", [0, 1])
def test_tokens_of_no_sequence_are_recorded(new, n, first):
    """Rows before the first offset or behind the last one: the record says so, their own outputs
    stay, and everybody else's are right. One call of each kind, and both kernels of prefill."""
    c = still.still_create(0)
    try:
        p = Pages(60, [x + 70 for x in new], 1, 64, 16)
        cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device=DEV) + first
        lens = torch.tensor(p.lens, dtype=torch.int32, device=DEV)
        mine = slice(first, first + sum(new))
        for Hq in (1, 8):  # the seven and three tokens: few rows, then many
            q, k, v = fused_rows(61, n + first, [Hq, 1, 1], 64)
            out = torch.full((n + first, Hq, 64), 7.0, device=DEV, dtype=torch.bfloat16)
            batch = still.PagedBatch(p.table, lens, cu)
            K0 = p.K.clone()
            still.still_paged_prefill(c, p.cache(), batch, q, out)
            code, det = still.still_get_device_status(c)
            assert still.STATUS[code] == "STILL_ERR_CUDA" and det[0] == 2
            assert_rows(out[mine], *attention64(p, q[mine], new), WEIGHTS)
            assert (out[:first] == 7).all() and (out[first + sum(new):] == 7).all()
            still.still_paged_append(c, p.cache(), batch, k, v)
            code, det = still.still_get_device_status(c)
            assert still.STATUS[code] == "STILL_ERR_CUDA" and det[0] == 2
            rest = torch.ones(p.K.shape[:2], dtype=torch.bool, device=DEV)
            at = first
            for b, m in enumerate(new):
                slots = torch.arange(p.lens[b] - m, p.lens[b], device=DEV)
                pages = p.table[b].long()[slots // 16]
                assert torch.equal(p.K[pages, slots % 16], k[at:at + m])
                rest[pages, slots % 16] = False
                at += m
            assert torch.equal(p.K[rest].view(torch.int16), K0[rest].view(torch.int16))
    finally:
        still.still_destroy(c)
