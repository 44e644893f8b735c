"""muxq_adapters on long inputs where a CTA runs through many steps of N: every stage of its rings is used again and again, its accumulators too.
Formulas and tolerances are those of test_adapters.py; the references are made on the GPU, in 64 bits, for their size."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_adapters import F16, F32, _inputs, _run, _runs  # noqa: E402


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2604_04701_b200 as m
    m.lib()
    return m


def _grids(call):
    """(mangled name, grid) of every kernel that `call` launches, from a capture of it."""
    from cuda.bindings import driver as d

    def ok(r):
        assert r[0] == d.CUresult.CUDA_SUCCESS, r[0]
        return r[1:] if len(r) > 2 else r[1]

    graph, side = torch.cuda.CUDAGraph(keep_graph=True), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    raw, out = d.CUgraph(graph.raw_cuda_graph()), []
    for node in ok(d.cuGraphGetNodes(raw, ok(d.cuGraphGetNodes(raw, 0))[1]))[0]:
        if ok(d.cuGraphNodeGetType(node)) == d.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            p = ok(d.cuGraphKernelNodeGetParams(node))
            name = ok(d.cuFuncGetName(p.func)) if int(p.func) else ok(d.cuKernelGetName(p.kern))
            out.append((name.decode(), (p.gridDimX, p.gridDimY)))
    return out


def _reference(X, A, B, ids, scale, ranks, base):
    """(Y, bound of its error before it is rounded) in 64 bits, on the GPU"""
    M, K, N = X.shape[0], X.shape[1], B.shape[1]
    Y = torch.zeros(M, N, dtype=torch.float64, device="cuda") if base is None else base.double()
    E = torch.zeros_like(Y)
    for a, r in enumerate(ranks):
        rows = (ids == a).nonzero()[:, 0]
        if not r or not len(rows):
            continue
        x, A1, B1, s = X[rows].double(), A[a, :r].double(), B[a, :, :r].double(), float(scale[a])
        T = x @ A1.T
        eT = (K / 16 + 16) * 2.0 ** -22 * (x.abs() @ A1.abs().T) + 2.0 ** -22 * T.abs() + 2.0 ** -38 * T.abs().amax(1, keepdim=True)
        d = s * (T @ B1.T)
        Y[rows] += d
        E[rows] = abs(s) * (eT @ B1.abs().T + (r / 8 + 4) * 2.0 ** -22 * (T.abs() @ B1.abs().T)) + 2 * 2.0 ** -24 * d.abs()
    return Y, E


def _check(got, want, err):
    half = (lambda v: v * 2.0 ** -11 + 2.0 ** -25) if got.dtype == F16 else (lambda v: v * 2.0 ** -24)
    assert torch.isfinite(got).all()
    off, tol = (got.double() - want).abs(), err + half(want.abs() + err)
    assert (off <= tol).all(), float((off / tol.clamp(min=1e-300)).max())


@pytest.mark.parametrize("out", [F16, F32])
@pytest.mark.parametrize("run,R,ranks", [(1024, 16, (16, 9, 16)), (1024, 64, (64, 33, 64)), (1024, 128, (128, 100, 128)), (64, 16, (16, 16, 5)),
                                         (64, 128, (128, 96, 128)), (32, 32, (32, 16, 32)), (32, 64, (64, 40, 48))])
@pytest.mark.parametrize("M,N", [(14700, 1544), (9473, 3848)])
def test_many_steps_of_columns(gpu, M, N, run, R, ranks, out):
    """Windows of one, two and four adapters, some rows of each without one; with base, in place and without base."""
    mx, K, slots = gpu, 64, 5
    gen = torch.Generator(device="cuda")
    gen.manual_seed(M + N + run + R)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    ranks = [ranks[i % len(ranks)] for i in range(slots)]
    X, A, B = rand(M, K).half(), (rand(slots, R, K) / 8).half(), (rand(slots, N, R) * 0.2).half()
    for i, r in enumerate(ranks):  # what lies beyond a slot's rank is not looked at
        A[i, r:] = float("nan")
        B[i, :, r:] = float("inf")
    ids = (torch.arange(M, device="cuda") // run % slots).int()
    ids[torch.rand(M, device="cuda", generator=gen) < 0.1] = -1
    scale, rank = 0.5 + torch.rand(slots, device="cuda", generator=gen), torch.tensor(ranks, dtype=torch.int32, device="cuda")
    base, whole = rand(M, N).to(out), rand(M + 1, N + 8).to(out)
    before, status = whole.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    call = lambda base, Y: mx.muxq_adapters(X, A, B, ids, status, scale, rank, base, out=Y)
    grids = [g for name, g in _grids(lambda: call(base, whole[:M, :N])) if "k_adapter_tiles" in name]
    assert len(grids) == 1 and grids[0][0] == -(-M // 128) and -(-N // 64) // grids[0][1] >= 20  # steps of every CTA
    Y = call(base, whole[:M, :N])
    _check(Y, *_reference(X, A, B, ids, scale, ranks, base))
    assert torch.equal(whole[M:], before[M:]) and torch.equal(whole[:, N:], before[:, N:])
    again = base.clone()
    call(again, again)
    assert torch.equal(again, Y)
    _check(call(None, whole[:M, :N]), *_reference(X, A, B, ids, scale, ranks, None))
    assert int(status) == 0


@pytest.mark.parametrize("out", [F16, F32])
@pytest.mark.parametrize("size", [1e-7, 1e-3, 1.0, 6e4])
def test_magnitudes(gpu, size, out):
    """Rows of X whose products leave the range of fp16 in either direction, and a row of zeros, on tensor memory."""
    v, whole = _inputs(1300, 264, 136, 3, 16, None, out, big=False)
    v["X"] = (v["X"].float().clamp(-1, 1) * size).half()
    v["X"][0] = 0.0
    v["X"][700:800:7] = 0.0
    v["ids"] = _runs(torch.Generator().manual_seed(2), 1300, 3, (300, 90, 129))
    v["ids"][0] = 1
    v["base"] = None
    if out == F16:  # results beyond fp16 are infinities there
        v["scale"] = v["scale"] * min(1.0, 1.0 / size)
    _run(gpu, v, whole)
    if out == F32 and size > 1:
        v["A"] = v["A"] * 16
        _run(gpu, v, whole)


@pytest.mark.parametrize("K", [1296, 2568, 5120])
def test_long_rows(gpu, K):
    """The stages of X and A come round many times."""
    v, whole = _inputs(1100, K, 136, 4, 32, (32, 9, 24, 32), F32)
    v["ids"] = _runs(torch.Generator().manual_seed(K), 1100, 4, (300, 90, 40, 129))
    _run(gpu, v, whole)


@pytest.mark.parametrize("out", [F16, F32])
@pytest.mark.parametrize("N,ranks", [(72, (32,)), (72, (32, 9)), (1544, (32,))])
def test_a_time_out_behind_copies_that_were_all_started(gpu, N, ranks, out):
    """The loads of a part of X and A are left out by a test hook.  B and the first tiles of base were asked for long before: with few columns all of
    them, so that the warps that bring them have nothing left to wait for."""
    mx = gpu
    v, whole = _inputs(1500, 776, N, 2, 32, ranks, out)
    v["ids"].fill_(1)
    want = _run(mx, v, whole).clone()
    for chunk in (1, 12):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        mx.muxq_test_hooks(spin_limit=20000, gemm_skip_k_block=chunk)
        try:
            mx.muxq_adapters(v["X"], v["A"], v["B"], v["ids"], status, v["scale"], v["rank"], v["base"], out=whole[:1500, :N])
            torch.cuda.synchronize()
        finally:
            mx.muxq_test_hooks()
        assert int(status) == mx.MUXQ_ERR_TIMEOUT
        assert torch.equal(_run(mx, v, whole), want)
