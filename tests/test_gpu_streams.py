"""Calls that make their own outputs and scratch on a stream that is not the current
one, while work queued on the current stream still writes to memory that it has just
given back: the results are those of the same calls on an idle GPU."""

import pytest

from tests._util import ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    ensure_built()
    from paper_2607_14107_amd import polestar
    return polestar


def _normal(*shape, seed=0, dtype=None):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed + sum(shape))
    return torch.randn(shape, generator=g, device="cuda").to(dtype or torch.bfloat16)


def _beside_work_in_progress(call, sizes):
    """call(stream) -> tensors: its results on a side stream, issued while the current stream is about to fill
    blocks of these sizes (bytes) that were freed already."""
    import torch
    want = call(None)
    want = [t.clone() for t in want]
    busy = _normal(4096, 4096)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    for _ in range(40):                                  # some milliseconds
        busy = (busy @ busy).clamp_(-1, 1)
    for b in blocks:
        b.fill_(0xFF)
    del blocks, b
    got = call(side)
    torch.cuda.synchronize()
    assert len(got) == len(want)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_microscaled_rows_and_their_scales(P):
    x = _normal(3, 200, 4096)
    n = x.numel()
    _beside_work_in_progress(lambda s: P.mx_quantize(P.MXFP8, x, stream=s), [n, n // 32])


def test_microscaled_product(P):
    import torch
    w = P.mx_quantize(P.MXFP4, _normal(512, 4096))
    h = P.mx_quantize(P.MXFP8, _normal(80, 4096))
    y = torch.zeros((80, 512), dtype=torch.bfloat16, device="cuda")
    need = P.mx_linear_workspace_size(P.MXFP8, P.BF16, 80, 512, 4096)
    assert need                                          # a split product: sums pass through the scratch
    _beside_work_in_progress(lambda s: [P.mx_linear(P.MXFP8, *h, *w, y, stream=s)], [need])


def test_microscaled_product_of_rows(P):
    import torch
    w = P.mx_quantize(P.MXFP4, _normal(512, 4096))
    x = _normal(1, 80, 4096)
    y = torch.zeros((1, 80, 512), dtype=torch.bfloat16, device="cuda")
    need = P.mx_quantize_linear_workspace_size(P.MXFP8, P.BF16, 1, 80, 512, 4096)
    assert need
    _beside_work_in_progress(lambda s: [P.mx_quantize_linear(P.MXFP8, x, 0, 80, *w, y, stream=s)], [need])


def test_microscaled_attention(P):
    caches = [t.view(2, 1, 4096, -1) for i in range(2) for t in P.mx_quantize(P.MXFP4, _normal(8192, 128, seed=i))]
    q = _normal(2, 3, 5, 128)
    need = P.mx_attend_workspace_size(P.BF16, 2, 4096, 5, 1, 128, 3)
    assert need
    _beside_work_in_progress(lambda s: [P.mx_attend(q, *caches, stream=s)], [need, 2 * q.numel()])


def test_attention_over_a_cache(P):
    k, v, q = _normal(1, 2048, 2, 128), _normal(1, 2048, 2, 128, seed=1), _normal(1, 32, 2, 128)
    need = P.attend_workspace_size(P.BF16, 1, 2048, 256, 2, 2, 128, 32)
    assert need
    _beside_work_in_progress(lambda s: [P.attend(None, None, k, v, 64, 32, 2, q_buf=q, stream=s)[0]],
                             [need, 2 * q.numel()])


def test_product_of_dense_rows(P):
    import torch
    x, w = _normal(1, 128, 4096), _normal(1024, 4096)
    y = torch.zeros((1, 96, 1024), dtype=torch.bfloat16, device="cuda")
    need = P.linear_workspace_size(P.BF16, 1, 96, 1024, 4096)
    assert need
    _beside_work_in_progress(lambda s: [P.linear(x, 8, 96, w, y, stream=s)], [need])


def test_drift_and_select(P):
    a, b = _normal(2, 3000, 1024), _normal(2, 3000, 1024, seed=1)

    def both(s):
        d = P.drift(a, b, stream=s)
        return [d, *P.select(d, 40, 64, 32, stream=s)]
    _beside_work_in_progress(both, [4 * 2 * 3000, 4 * 2 * 40, 8])


def test_commit(P):
    import torch
    logits = _normal(1, 32, 126464)
    masked = torch.ones((1, 32), dtype=torch.uint8, device="cuda")
    need = P.commit_workspace_size(P.BF16, 1, 32, 126464)
    assert need
    _beside_work_in_progress(lambda s: P.suffix_commit(logits, masked, masked, stream=s), [need, 128, 128, 32])


def test_microscaled_calls_on_a_forked_stream_in_a_graph(P):
    """Captured on a stream that joins the captured one, outputs and scratch made by the calls: every replay gives
    the eager bits, with eager work that allocates and fills between them."""
    import torch
    w = P.mx_quantize(P.MXFP4, _normal(512, 4096))
    x = _normal(80, 4096)
    caches = [t.view(2, 1, 4096, -1) for i in range(2) for t in P.mx_quantize(P.MXFP4, _normal(8192, 128, seed=i))]
    q = _normal(2, 3, 5, 128)
    y = torch.zeros((80, 512), dtype=torch.bfloat16, device="cuda")

    def calls(s):
        h = P.mx_quantize(P.MXFP8, x, stream=s)
        P.mx_linear(P.MXFP8, *h, *w, y, stream=s)
        return [*h, y, P.mx_attend(q, *caches, stream=s)]
    want = [t.clone() for t in calls(None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = calls(side)
        torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(calls(None)[:2], want))
        torch.full((1 << 24,), i, dtype=torch.uint8, device="cuda")
