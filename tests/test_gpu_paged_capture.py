"""Captured attention calls beside eager ones of other sizes on the same stream."""
import pytest
import torch

import paper_2205_11622_amd as slnr
from tests import paged_util as pu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sparse", [False, True])
def test_a_captured_step_outlives_larger_calls_on_its_stream(gpu, sparse):
    """A step of a few tokens is captured after one eager call of a few tokens; a prompt, a call of
    another type and width, and a selection that goes by pages then run on the stream between the replays."""
    b = pu.Batch([4000, 90], [2, 2], 8, 2, 128, 64, torch.bfloat16, seed=70)
    q, kc, vc, table, seq, qptr = b.upload(gpu)
    sel = torch.arange(64, dtype=torch.int32, device=gpu).expand(4, 2, 64).contiguous()
    big = pu.Batch([700], [900], 8, 8, 128, 64, torch.bfloat16, seed=71)
    wide = pu.Batch([200], [300], 2, 2, 256, 64, torch.float16, seed=72)
    up, up_wide = big.upload(gpu), wide.upload(gpu)
    many = torch.arange(12, dtype=torch.int32, device=gpu).expand(900, 8, 12).contiguous()
    stream = torch.cuda.Stream()

    def step():
        if sparse:
            return slnr.sparselnr_block_attention(q, kc, vc, table, seq, qptr, sel)
        return slnr.sparselnr_paged_attention(q, kc, vc, table, seq, qptr)

    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = step()
    x = torch.randn(3, *q.shape, device=gpu, generator=torch.Generator(device=gpu).manual_seed(1)).to(q.dtype)
    with torch.cuda.stream(stream):
        for i in range(3):
            q.copy_(x[i])
            graph.replay()
            slnr.sparselnr_paged_attention(*up)
            slnr.sparselnr_paged_attention(*up_wide)
            slnr.sparselnr_block_attention(*up, many)
            out.zero_()
            graph.replay()
            want = step()
            stream.synchronize()
            assert torch.equal(out.view(torch.int16), want.view(torch.int16)), i
    ref = pu.attention(x[2].cpu(), b.kc, b.vc, b.table, b.seq, b.qptr, 128 ** -0.5, sel=sel.tolist() if sparse else None)
    pu.check(out.cpu(), None, ref, torch.bfloat16, max(b.seq), 128, float(b.vc.float().nan_to_num(0.0).abs().max()))


def test_two_host_threads_on_one_stream(gpu):
    """Each thread's calls give what they give alone."""
    import threading
    batches = [pu.Batch([5000, 900], [1, 3], 8, 2, 128, 64, torch.bfloat16, seed=73 + i) for i in range(2)]
    ups = [b.upload(gpu) for b in batches]
    sel = torch.arange(64, dtype=torch.int32, device=gpu).expand(4, 2, 64).contiguous()
    calls = [lambda u: slnr.sparselnr_paged_attention(*u), lambda u: slnr.sparselnr_block_attention(*u, sel)]
    want = [[call(u) for call in calls] for u in ups]
    torch.cuda.synchronize()
    got = [[], []]

    def work(i):
        for _ in range(40):
            got[i].append([call(ups[i]) for call in calls])

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(2):
        assert len(got[i]) == 40
        for outs in got[i]:
            for x, y in zip(outs, want[i]):
                assert torch.equal(x.view(torch.int16), y.view(torch.int16))
