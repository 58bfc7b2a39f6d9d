"""The operators without a context on other streams and in captured graphs, against the same calls on
the current stream.

Collected last: once a process has used a second stream, launches may begin on another XCD, and
contexts created afterwards find that workgroup i is not on XCD i % 8 and leave out the kernels that
need it, which other tests compare."""
import pytest
import torch

from test_gpu_paged import BF, DEV, ints, make_cache, make_step
from test_gpu_scaled import F32, make

pytestmark = pytest.mark.gpu


def test_two_streams_and_graph_replays():
    """The same step on another stream, and captured and replayed between other work."""
    page, H, G, dh = 64, 2, 4, 128
    lens = [(700, 8), (30, 8)]
    kv = make_cache(20, page, H, dh, 41)
    step, *_ = make_step(lens, page, 20, 41)
    q = torch.randn((16, H * G, dh), device=DEV).to(BF)
    x = torch.randn((16, 2 * H, dh), device=DEV).to(BF)
    kv.append(step, x[:, :H], x[:, H:])
    want = kv.attend(step, q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        kv.append(step, x[:, :H], x[:, H:])
        got = kv.attend(step, q)
    s.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.append(step, x[:, :H], x[:, H:])
        kv.attend(step, q, out=out)
    for i in range(3):
        out.zero_()
        x.copy_(torch.randn_like(x))
        graph.replay()
        torch.cuda.synchronize()
        mine = out.clone()
        kv.append(step, x[:, :H], x[:, H:])
        assert torch.equal(mine, kv.attend(step, q))


def test_plan_in_a_graph():
    """A captured plan, append and attention of a growing sequence, replayed step after step."""
    from paper_2509_04185_amd import PagedKV, PageTable
    B, page, H, dh = 2, 16, 1, 64

    def fresh():
        return PageTable.empty(B, 128, 20, page), PagedKV.empty(20, page, H, dh)
    x = torch.zeros((B, 3 * H, dh), dtype=BF, device=DEV)
    n_new = ints([1, 1])
    (pa, ka), (pb, kb) = fresh(), fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step = pa.plan(n_new, B)
        ka.append(step, x[:, H:2 * H], x[:, 2 * H:])
        out = ka.attend(step, x[:, :H])
        pa.cached.add_(n_new)
    g = torch.Generator().manual_seed(51)
    for i in range(40):
        x.copy_(torch.randn(x.shape, generator=g).to(BF))
        graph.replay()
        torch.cuda.synchronize()
        s2 = pb.plan(n_new, B)
        kb.append(s2, x[:, H:2 * H], x[:, 2 * H:])
        want = kb.attend(s2, x[:, :H])
        pb.cached += n_new
        assert torch.equal(out, want)
        assert torch.equal(pa.table, pb.table)


def test_matmul_same_bits_again_and_in_a_graph():
    """The order of the sums is fixed: the same call gives the same bits, captured too."""
    from paper_2509_04185_amd import scaled_matmul
    for m, n, k in ((16, 1024, 14336), (100, 1024, 4096), (300, 512, 1024)):
        a, sa, b, sb = make(m, n, k, 3)
        want = scaled_matmul(a, sa, b, sb, out_dtype=F32)
        out = torch.empty_like(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            scaled_matmul(a, sa, b, sb, out=out)
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            assert torch.equal(scaled_matmul(a, sa, b, sb, out_dtype=F32), want)
