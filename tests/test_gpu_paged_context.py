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
