"""Norm, projection with adapters, norm, projection: the operators of a block one behind the other, as a decode step or a prompt runs them.
Every stage is compared with its own reference on the inputs that it got, and the whole run with its replay from a graph."""
import numpy as np
import pytest

import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_adapters import check as check_adapters, reference as reference_adapters  # noqa: E402
from test_residual_norm import check as check_norm, reference as reference_norm  # noqa: E402


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2604_04701_b200 as m
    m.lib()
    return m


class Block:
    """Two projections, D -> F and F -> D, with a norm before each part of the residual stream and adapters beside both."""

    def __init__(self, mx, M, D, F, vector, seed):
        gen = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=gen)
        self.mx, self.M = mx, M
        self.p = mx.MuxqParams(gran=mx.MUXQ_PER_VECTOR if vector else mx.MUXQ_PER_TENSOR)
        self.w = [(r(D, F) * 0.03).half().cuda(), (r(F, D) * 0.03).half().cuda()]
        load = mx.Workspace(mx.muxq_small_workspace_bytes(max(D, F)))
        self.q = [mx.muxq_quantize(w, self.p, True, load) for w in self.w]
        self.bias = [(r(F) * 0.1).cuda(), (r(D) * 0.1).cuda()]
        ids = torch.randint(-1, 3, (M,), generator=gen).int().cuda()
        rank = torch.tensor([16, 5, 9], dtype=torch.int32).cuda()
        scale = torch.tensor([0.5, 1.0, 2.0]).cuda()
        pair = lambda K, N: mx.Adapters((r(3, 16, K) / K ** 0.5).half().cuda(), (r(3, N, 16) * 0.1).half().cuda(), ids, scale, rank)
        self.adapters = [pair(D, F), pair(F, D)]
        self.pre = mx.Norm(mx.MUXQ_NORM_LAYER, (1 + 0.1 * r(D)).cuda(), (0.1 * r(D)).cuda())
        self.mid = mx.Norm(mx.MUXQ_NORM_RMS, (1 + 0.1 * r(F)).cuda())
        self.post = mx.Norm(mx.MUXQ_NORM_RMS, (1 + 0.1 * r(D)).cuda())
        self.next = mx.Norm(mx.MUXQ_NORM_LAYER, (1 + 0.1 * r(D)).cuda(), None)
        self.gate = (0.5 * r(D)).cuda()
        self.stream = r(M, D).cuda()
        self.stream[:, 3] *= 40.0
        self.ws = mx.Workspace(max(mx.muxq_workspace_bytes(M, D, F, self.p), mx.muxq_workspace_bytes(M, F, D, self.p)))
        self.x0 = torch.empty(M, D, dtype=torch.float16, device="cuda")
        self.y1 = torch.empty(M, F, dtype=torch.float16, device="cuda")
        self.x1 = torch.empty(M, F, dtype=torch.float16, device="cuda")
        self.y2 = torch.empty(M, D, device="cuda")
        self.h = torch.empty(M, D, device="cuda")
        self.x2 = torch.empty(M, D, dtype=torch.float16, device="cuda")

    def run(self):
        mx, p, ws = self.mx, self.p, self.ws
        mx.muxq_residual_norm(self.stream, None, self.pre, X=self.x0)
        mx.muxq_linear(self.x0, *self.q[0], p, ws, mx.MUXQ_OUT_F16, out=self.y1, bias=self.bias[0], adapters=self.adapters[0])
        mx.muxq_residual_norm(None, self.y1, None, post=self.mid, X=self.x1, want_h=False)
        mx.muxq_linear(self.x1, *self.q[1], p, ws, mx.MUXQ_OUT_F32, out=self.y2, bias=self.bias[1], adapters=self.adapters[1])
        mx.muxq_residual_norm(self.stream, self.y2, self.next, post=self.post, gate=self.gate, scale=0.7, H=self.h, X=self.x2)

    def results(self):
        return [t.clone() for t in (self.x0, self.y1, self.x1, self.y2, self.h, self.x2)]


def _linear(b, i, x, y_before):
    """The projection alone: against the oracle, bit for bit in fp32 and to the last place in fp16."""
    vector = b.p.gran == b.mx.MUXQ_PER_VECTOR
    w_q, s_w = oracle.quantize_weight(b.w[i].cpu().numpy(), per_channel=vector)
    want = oracle.linear(x.cpu().numpy(), w_q, s_w, per_vector=vector, bias=b.bias[i].cpu().numpy())
    got = y_before.cpu().numpy()
    if got.dtype == np.float32:
        assert np.array_equal(got, want.y32)
    else:
        a, c = got.view(np.int16).astype(np.int32), want.y16.view(np.int16).astype(np.int32)
        assert np.abs(np.where(a < 0, -(a & 0x7fff), a) - np.where(c < 0, -(c & 0x7fff), c)).max() <= 1


@pytest.mark.parametrize("vector", [False, True])
@pytest.mark.parametrize("M", [1, 5, 16, 130, 700])
def test_a_block(mx, M, vector):
    b = Block(mx, M, 256, 640, vector, seed=M)
    b.run()
    torch.cuda.synchronize()
    assert mx.muxq_read_status(b.ws) == mx.MUXQ_OK
    x0, y1, x1, y2, h, x2 = b.results()
    _, _, want, err = reference_norm(b.stream, None, b.pre, None, None, 1, 1.0)
    check_norm(x0, torch.float16, want, err, "x0")
    for i, (x, y, kind) in enumerate(((x0, y1, mx.MUXQ_OUT_F16), (x1, y2, mx.MUXQ_OUT_F32))):
        alone = mx.muxq_linear(x, *b.q[i], b.p, b.ws, kind, bias=b.bias[i])
        _linear(b, i, x, alone)
        a = b.adapters[i]
        check_adapters(y, *reference_adapters(x, a.A, a.B, a.row_slot, a.scale, a.rank, alone))
    _, _, want, err = reference_norm(None, y1, None, b.mid, None, 1, 1.0)
    check_norm(x1, torch.float16, want, err, "x1")
    want_h, err_h, want, err = reference_norm(b.stream, y2, b.next, b.post, b.gate, 1, 0.7)
    check_norm(h, torch.float32, want_h, err_h, "h")
    check_norm(x2, torch.float16, want, err, "x2")


@pytest.mark.parametrize("M", [1, 16, 130])
def test_a_block_from_a_graph(mx, M):
    """Captured once and replayed over other contents of the stream and other requests in the rows, against plain calls."""
    b = Block(mx, M, 256, 640, False, seed=50 + M)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.run()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.run()
    torch.cuda.synchronize()
    gen = torch.Generator().manual_seed(M)
    for _ in range(3):
        b.stream.copy_(torch.randn(b.stream.shape, generator=gen) * 2)
        b.adapters[0].row_slot.copy_(torch.randint(-1, 3, (M,), generator=gen).int())
        b.run()
        torch.cuda.synchronize()
        want = b.results()
        for t in (b.x0, b.y1, b.x1, b.y2, b.h, b.x2):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(b.results(), want):
            assert torch.equal(got, w)


def test_adapters_do_not_go_with_the_accumulator(mx):
    b = Block(mx, 4, 256, 640, False, seed=9)
    with pytest.raises(mx.MuxqError):
        mx.muxq_linear(b.x0, *b.q[0], b.p, b.ws, mx.MUXQ_OUT_ACC_I32, adapters=b.adapters[0])
